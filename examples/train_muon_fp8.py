"""Trains a small character-level model whose linear layers multiply in 8-bit floating point and
whose matrices are updated by Muon with 8-bit momentum.

    python -m examples.train_muon_fp8 [--steps 60]     (from the repository's root)

One step, as a training program runs it:

1. forward and backward through ``Fp8Linear``, which reads the 8-bit weights and leaves bf16
   gradients;
2. ``HybridMuon.step``: global norm, clip coefficient, AdamW for embedding and output head, Muon
   for the hidden matrices, fp32 master weights and their bf16 copies;
3. ``Fp8Weight.update``: the masters quantized again for the next step.

At the end a few characters are answered one at a time, through the kernel for few tokens.
"""
import argparse

import torch

import paper_2608_11919_amd as lt

TEXT = ("the moment of a block is stored in eight bits, the weights in thirty-two; "
        "a step reads them, a step writes them, and the sum of all squares bounds it. ") * 8


class Layer:
    """A linear layer: fp32 master weights, their bf16 copy in the graph, and the 8-bit weight."""

    def __init__(self, rows, cols, gen):
        self.master = torch.randn(rows, cols, device="cuda", generator=gen) / cols ** 0.5
        self.weight = lt.Fp8Weight.from_master(self.master)
        self.copy = None  # the optimizer's bf16 copy, which the gradient belongs to

    def __call__(self, x):
        return lt.Fp8Linear.apply(x, self.copy, self.weight)


def build(vocab, width, depth, context, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    embedding = torch.randn(vocab, width, device="cuda", generator=gen) * 0.3
    layers = [Layer(4 * width if i % 2 == 0 else width,
                    context * width if i == 0 else (width if i % 2 == 0 else 4 * width), gen)
              for i in range(2 * depth)]
    head = Layer(vocab, width, gen)
    return embedding, layers, head


def forward(embedding, layers, head, tokens):
    """tokens (batch, context) -> logits of the next character."""
    h = embedding[tokens].flatten(1)
    for i in range(0, len(layers), 2):
        out = layers[i + 1](torch.relu(layers[i](h)))
        h = out if i == 0 else h + out  # the first pair narrows the context to the width
    return head(h).float()


def train(steps=60, width=128, depth=2, context=16, batch=256, lr=4e-3, seed=0, verbose=True):
    letters = sorted(set(TEXT))
    text = torch.tensor([letters.index(c) for c in TEXT], device="cuda")
    embedding, layers, head = build(len(letters), width, depth, context, seed)
    modules = layers + [head]
    masters = [embedding] + [m.master for m in modules]
    # Muon for the hidden matrices; embedding and head stay with AdamW
    opt = lt.HybridMuon(masters, lr=lr, weight_decay=0.01, max_norm=1.0, block_size=256,
                        bf16_copy=True, matrices=[False] + [True] * len(layers) + [False])
    for p, c in zip(opt.params, opt.params_bf16):
        c.copy_(p.view(-1))
    graph = [c.view(p.shape).requires_grad_() for p, c in zip(opt.params, opt.params_bf16)]
    for m, g in zip(modules, graph[1:]):
        m.copy = g
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    losses = []
    for step in range(steps):
        at = torch.randint(0, len(text) - context, (batch,), device="cuda", generator=gen)
        window = text[at[:, None] + torch.arange(context + 1, device="cuda")]
        logits = forward(graph[0], layers, head, window[:, :-1])
        loss = torch.nn.functional.cross_entropy(logits, window[:, -1])
        grads = torch.autograd.grad(loss, graph)
        opt.step([g.contiguous() for g in grads])
        for m in modules:
            m.weight.update(m.master)
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    if opt.last_status() != lt.LT_STATUS_OK:
        raise RuntimeError("the last step was skipped")

    answer = list(text[:context])
    with torch.no_grad():
        for _ in range(40):
            h = embedding[torch.stack(answer[-context:])].view(1, -1).bfloat16()
            for i in range(0, len(layers), 2):
                out = lt.fp8_linear(torch.relu(lt.fp8_linear(h, layers[i].weight)),
                                    layers[i + 1].weight)
                h = out if i == 0 else h + out
            answer.append(lt.fp8_linear(h, head.weight).argmax())
    said = "".join(letters[int(t)] for t in answer)
    if verbose:
        print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")
        print(f"answers: {said!r}")
    return losses, said


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=60)
    train(p.parse_args().steps)
