// library.hip -- the optimizer step's source and, in the same translation unit, what uses its
// device code (momentum.hip) and what lends its host side to the other sources (host.h).
#include "lazytrain.hip"

#include "host.h"

#include "momentum.hip"

namespace host {

lt_err fail(lt_err code, const std::string& msg) { return ::fail(code, msg); }

lt_err caught() noexcept
{
    try {
        return ::fail(LT_ERR_HOST, "host memory ran out");
    } catch (...) {
        return LT_ERR_HOST;
    }
}

void clear_error() { g_last_error.clear(); }

lt_err put_descriptors(std::vector<uint8_t>& image, void* ws, hipStream_t st, Guard* guard)
{
    static_assert(kTagBytes == ::kTagBytes, "one tag slot");
    WsGuard g;
    if (lt_err e = ::put_descriptors(
            image, ws, st, &g, [&](const PutWords& a) { return put_words(a, ws, st); }, true))
        return e;
    *guard = Guard{g.at, g.tag};
    return LT_OK;
}

lt_err workspace_written(const void* ws, size_t bytes, hipStream_t st)
{
    return ::workspace_written(ws, bytes, st);
}

lt_err compute_units(int* cus) { return ::compute_units(cus); }

bool aligned(const void* p, size_t a) { return ::aligned(p, a); }

bool valid_block_size(int block) { return ::valid_block_size(block); }

std::string overlap(std::vector<Range>& ranges)
{
    ByteRanges r;
    r.v.reserve(ranges.size());
    for (const Range& x : ranges)
        r.v.push_back({x.lo, x.hi, x.written});
    r.ends.push_back(r.v.size());
    return overlap_error(r);
}

}  // namespace host
