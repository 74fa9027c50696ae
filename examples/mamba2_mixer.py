"""Two Mamba-2 mixer layers served end to end: ragged prompts, then single tokens.

    python examples/mamba2_mixer.py [--batch 64] [--prompt 500] [--tokens 64] [--rank 16] [--window 16]

Weights and inputs are random, of the shapes of the decode path's Mamba-2
layers (128 heads of 64 values, 128 keys, 8 groups, hidden size 4096).  Prompts
of different lengths are packed one after the other; each request then decodes
`--tokens` tokens from its state through the sketch.  Prints the times of both,
and, with exact reads, how far the last prompt token's output is when it is
decoded after the others instead of being prefilled with them.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2609_33051_amd.mixer import Mamba2Mixer  # noqa: E402

HIDDEN, H, G, K, V = 4096, 128, 8, 128, 64


def weights(seed: int) -> dict:
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    C = H * V + 2 * G * K
    return dict(norm=1 + 0.1 * r(HIDDEN), in_proj=r(H * V + C + H, HIDDEN) * HIDDEN ** -0.5, taps=r(C, 4) * 0.5, conv_bias=r(C) * 0.1,
                dt_bias=r(H) - 4.0, A=-torch.exp(r(H)), D=r(H), out_norm=1 + 0.1 * r(H * V), out_proj=r(HIDDEN, H * V) * (H * V) ** -0.5)


def mixer(seed: int, batch: int, rank: int, window: int) -> Mamba2Mixer:
    """rank K: the sketch is the state itself, and its reads are exact."""
    omega = torch.eye(K, device="cuda")[:, :rank].expand(H, K, rank).contiguous()
    coef = omega.transpose(1, 2).contiguous()
    return Mamba2Mixer(weights(seed), batch, H, G, K, V, rank, window, omega, coef)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--prompt", type=int, default=500, help="mean prompt length")
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--rank", type=int, default=16)
    p.add_argument("--window", type=int, default=16)
    a = p.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    lengths = torch.randint(1, 2 * a.prompt, (a.batch,), generator=g, device="cuda")
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)]).to(torch.int32)
    T = int(offsets[-1])
    x = torch.randn((T, HIDDEN), generator=g, device="cuda").bfloat16()
    token = torch.randn((a.batch, HIDDEN), generator=g, device="cuda").bfloat16()

    def prefill(layers, x, offsets):
        h, res = x, torch.zeros_like(x)
        for m in layers:
            h, res = m.prefill(h, res, offsets)
        return h

    def step(layers, x):
        h, res = x, torch.zeros_like(x)
        for m in layers:
            h, res = m.step(h, res)
        return h

    def run(n):
        """The prompts, then n tokens: the seconds of both."""
        layers = [mixer(s, a.batch, a.rank, a.window) for s in (1, 2)]
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        prefill(layers, x, offsets)
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        h = token
        for _ in range(n):
            h = step(layers, h)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(h.float()).all())
        return t1 - t0, time.perf_counter() - t1

    run(a.window)  # first launches
    prompts, decode = run(a.tokens)
    print(f"prompts: {T} tokens of {a.batch} requests, two layers: {prompts * 1e3:.2f} ms, {T / prompts:.0f} tokens/s")
    print(f"decode:  {a.tokens} tokens of {a.batch} requests: {decode * 1e3:.2f} ms, {a.batch * a.tokens / decode:.0f} tokens/s")

    last = (offsets[1:] - 1).long()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[last] = False
    exact = lambda: [mixer(s, a.batch, K, a.window) for s in (1, 2)]  # noqa: E731
    whole = prefill(exact(), x, offsets)[last]
    layers = exact()
    prefill(layers, x[rest], offsets - torch.arange(a.batch + 1, dtype=torch.int32, device="cuda"))
    off = float((step(layers, x[last]).float() - whole.float()).norm() / whole.float().norm())
    print(f"the last prompt token decoded instead of prefilled: relative difference {off:.4f} (both round to 8 and 16 bits)")
    assert off < 0.1


if __name__ == "__main__":
    main()
