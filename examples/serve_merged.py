"""Agents decode over merged caches held in 8-bit pages.

Each agent's deliveries are rendered to a merged cache (the order of delivery does not
matter), which is laid into 8-bit pages; a question is appended to it; then all agents
decode together, one token a step. The model is a stand-in of random weights: per layer
projections to q, k and v, attention, a projection back and a residual sum, which is what
decides how the operators are called.

    python examples/serve_merged.py [--agents 4] [--steps 32]

prints the milliseconds of a step, and how far the last step's attention is from the same
attention over the tokens' own bf16 keys and values (what the 8 bits cost)."""

from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2607_01308_amd as cm  # noqa: E402
import synth  # noqa: E402

BF16 = torch.bfloat16


class Decoder:
    """Random weights of L layers; KV heads shared by `group` query heads."""

    def __init__(self, L: int, H: int, group: int, d: int, width: int, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape):
            w = torch.randn(shape, generator=g, device="cuda") * shape[-2] ** -0.5
            return w.to(BF16)

        self.L, self.H, self.group, self.d, self.width = L, H, group, d, width
        self.qkv = weight(L, width, (group + 2) * H * d)
        self.back = weight(L, group * H * d, width)

    def step(self, x: torch.Tensor, sc: cm.ServingCache, new, keep=None) -> torch.Tensor:
        """The rows x of the places' new tokens through all layers."""
        step = sc.extend(new)
        Hq = self.H * self.group
        for layer in range(self.L):
            y = torch.nn.functional.rms_norm(x, (self.width,)) @ self.qkv[layer]
            q, k, v = y.view(-1, Hq + 2 * self.H, self.d).split((Hq, self.H, self.H), 1)
            sc.write(layer, k, v, step)
            out, _ = sc.attend(layer, q, step)
            if keep is not None:
                keep(layer, q, k, v, out)
            x = x + out.view(-1, Hq * self.d) @ self.back[layer]
        return x


def last_rows(x: torch.Tensor, new) -> torch.Tensor:
    """The last row of each place."""
    ends = torch.tensor(new).cumsum(0) - 1
    return x[ends.to(x.device)]


def main(agents: int = 4, steps: int = 32, question: int = 24, block: int = 16,
         lengths=(512, 768, 700), L: int = 4, H: int = 8, group: int = 2, d: int = 128) -> dict:
    merged = []
    for a in range(agents):
        w = synth.custom(lengths=tuple(n + 16 * a for n in lengths), deliveries=(1, 0, 2, 0),
                         dtype="bfloat16", d=d, L=L, H=H)
        deliveries = synth.make_deliveries(w, synth.make_fragments(w, device="cuda"))
        merged.append(cm.render_deliveries(deliveries, w.routing_layer, w.rope_base).cache)
    tokens = [c[0][0].shape[2] for c in merged]
    max_len = max(tokens) + question + max(steps, 4)     # (three steps untimed, one at least timed)
    pages = agents * -(-max_len // block)
    sc = cm.ServingCache(cm.QCache.empty(L, H, d, pages, block), agents, max_len)
    for a, cache in enumerate(merged):
        sc.load(a, cache)

    model = Decoder(L, H, group, d, width=group * H * d)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    seen = []                                            # (layer, q, k, v, out) of every step

    def keep(*step):
        seen.append(step)

    # the questions, each with several rows, then one token a step
    ask = [question] * agents
    x = torch.randn((agents * question, model.width), generator=g, device="cuda").to(BF16)
    x = last_rows(model.step(x, sc, ask, keep), ask)
    one = [1] * agents
    for _ in range(3):                                   # (the first calls load the kernels)
        x = model.step(x, sc, one, keep)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    timed = max(steps - 4, 1)
    for _ in range(timed):
        x = model.step(x, sc, one, keep)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / timed * 1e3

    # the last step's attention over the tokens' own keys and values, in 64 bits
    far = 0.0
    for layer in range(L):
        steps_of = [step[1:] for step in seen if step[0] == layer]
        q, out = steps_of[-1][0], steps_of[-1][3]
        for a in range(agents):
            own = [[x[0].transpose(0, 1)] for x in merged[a][layer]]
            for _, k, v, _ in steps_of:
                rows = k.shape[0] // agents
                for to, x in zip(own, (k, v)):
                    to.append(x[a * rows:(a + 1) * rows])
            K, V = (torch.cat(x).double() for x in own)
            for h in range(H):
                s = q[a, h * group:(h + 1) * group].double() @ K[:, h].T * d ** -0.5
                exact = torch.softmax(s, 1) @ V[:, h]
                got = out[a, h * group:(h + 1) * group].double()
                far = max(far, float((got - exact).norm() / exact.norm()))
    for a in range(agents):
        sc.release(a)
    result = {"agents": agents, "tokens": tokens, "ms_per_step": ms, "relative_error": far,
              "free_pages": sc.free_pages, "pages": pages}
    print(f"{agents} agents over {tokens} merged tokens, {L} layers: {ms:.3f} ms a step; attention "
          f"from 8 bits off by {far:.4f} of its norm at most", flush=True)
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--agents", type=int, default=4)
    ap.add_argument("--steps", type=int, default=32)
    args = ap.parse_args()
    main(args.agents, args.steps)
