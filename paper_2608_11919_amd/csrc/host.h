// host.h -- what the library's source files share on the host side: errors, descriptors in
// workspaces and launch sizes (defined in library.hip over those of lazytrain.hip), and the
// launches that one file makes for another.
#ifndef LAZYTRAIN_HOST_H
#define LAZYTRAIN_HOST_H

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "lazytrain.h"

namespace host {

// The workspace's tag word and the tag a launch expects there: a kernel whose workspace does
// not hold its descriptors returns before it reads one.
struct Guard {
    const uint64_t* at;
    uint64_t tag;
};

constexpr size_t kTagBytes = 64;  // at the head of every workspace with descriptors

constexpr size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
constexpr int64_t ceil_div(int64_t x, int64_t a) { return (x + a - 1) / a; }

// Records the calling thread's error message and returns the code.
lt_err fail(lt_err code, const std::string& msg);
void clear_error();

// Makes the workspace hold `image` (its first kTagBytes are the tag slot) before the work
// enqueued next on the stream reads it; nothing is copied when it already does.  Under capture
// the graph writes it, at every replay.
lt_err put_descriptors(std::vector<uint8_t>& image, void* ws, hipStream_t st, Guard* guard);

// Before work on the stream writes [ws, ws + bytes) as anything but descriptors: a list call that
// finds its workspace there writes its descriptors again.
lt_err workspace_written(const void* ws, size_t bytes, hipStream_t st);

lt_err compute_units(int* cus);

// For an entry point's handler of all exceptions, none of which leaves it: a list that does not
// fit host memory is an error like any other.
lt_err caught() noexcept;

bool aligned(const void* p, size_t a);
bool valid_block_size(int block);

// Byte ranges of a call's arrays, for the rule that no array it writes overlaps another.
struct Range {
    uintptr_t lo, hi;
    bool written;
};
// Empty when nothing overlaps, else a message.
std::string overlap(std::vector<Range>& ranges);

inline bool overlaps(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && a_bytes && b_bytes && x < y + b_bytes && y < x + a_bytes;
}

// ------------------------------------------------------- 8-bit momentum (momentum.hip)

// One matrix of a momentum launch.
struct MomentumTensor {
    const void* g;   // gradient, fp32 or bf16
    int8_t* mq;      // codes and block scales, read and written
    float* ma;
    float* u;        // the update, unnormalised
    double* partial; // a sum of squares of u for every unit
    int64_t numel;
};

struct MomentumScalars {
    float beta, rest;  // fp32(momentum), fp32(1 - momentum)
    int nesterov;
};

// Elements of one unit (one workgroup's pass, whole blocks) at a block size.
int64_t momentum_unit(int block);

// The momentum pass over matrices [first, first + n): `prefix` holds units before each
// matrix of the whole list.
lt_err launch_momentum(const Guard& guard, const int64_t* prefix, const MomentumTensor* desc,
                       int first, int n, int64_t first_unit, int64_t units, int grad_dtype,
                       int block, int code_map, const MomentumScalars& s, const float* coef,
                       const int32_t* status, const void* step_state, hipStream_t st);

}  // namespace host

#define LT_TRY_HIP(call)                                                                \
    do {                                                                                \
        hipError_t e_ = (call);                                                         \
        if (e_ != hipSuccess)                                                           \
            return host::fail(LT_ERR_HIP, std::string(#call) + ": " + hipGetErrorString(e_)); \
    } while (0)

#endif
