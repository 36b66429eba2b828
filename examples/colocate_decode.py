#!/usr/bin/env python3
"""Which served models may share an MI355X?

Traces the decode step of a few model shapes on this GPU, and the prompts of one
with 8-bit floating weights, predicts every pair's slowdown from the traces and
places the models on simulated GPUs of the same kind:

    python examples/colocate_decode.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2607_16784_amd import api, decode, workloads as W  # noqa: E402

SHAPES = [
    # name, layers, width, heads, kv_heads, head_dim, hidden, sequences, tokens held
    ("small, 4 sequences", 6, 1024, 8, 2, 128, 2816, 4, 500),
    ("small, 64 sequences", 6, 1024, 8, 2, 128, 2816, 64, 1000),
    ("middle, 16 sequences", 4, 2048, 16, 4, 128, 5632, 16, 2000),
    ("wide, 1 sequence", 4, 4096, 32, 8, 128, 14336, 1, 8000),
]
# prompts of different lengths, behind each other
PROMPTS = ("middle, 4 prompts", 4, 2048, 16, 4, 128, 5632, [900, 37, 2000, 411])


def main():
    models = []
    for i, (name, layers, width, heads, kv, dim, hidden, n, held) in enumerate(SHAPES):
        model = decode.DecodeModel(layers, width, heads, kv, dim, hidden, seed=i)
        state = model.new_state(n, held + 64)
        for at in range(0, held, 512):          # prompts, 512 tokens at a time
            new = min(512, held - at)
            model.step(torch.randn((n * new, width), device="cuda").bfloat16(), state, new)
        models.append((model, state))
    name, layers, width, heads, kv, dim, hidden, lengths = PROMPTS
    model = decode.DecodeModel(layers, width, heads, kv, dim, hidden, seed=len(SHAPES),
                               weights="f8", head_norm=True)
    models.append((model, model.new_state(len(lengths), max(lengths) + 64), lengths))
    lib = decode.trace_library(models)
    dev = api.library_to_device(lib)
    status = api.new_status()
    out = api.rm_pair_slowdown_matrix(W.MI355X, dev["offsets"], dev["grid"], dev["threads"],
                                      dev["regs"], dev["smem"], dev["duration"], status=status)
    events = torch.arange(len(models), dtype=torch.int32, device="cuda")
    placed = api.rm_place(out["delay"], out["iso_time"], out["kernel_count"], n_devices=3,
                          capacity=2, events=events, lam=1.0)
    names = [s[0] for s in SHAPES] + [PROMPTS[0]]
    for name, state in zip(names, [m[1] for m in models]):
        if int(state["status"].item()):
            raise SystemExit(f"{name}: status {int(state['status'].item())}")
    if int(status.item()):
        raise SystemExit(f"pair matrix: status {int(status.item())}")
    count, iso = out["kernel_count"].tolist(), out["iso_time"].tolist()
    slow = out["slowdown"].view(len(models), -1).tolist()
    where = placed["placed_device"].tolist()
    print("model                  kernels  step alone   predicted slowdown beside each    GPU")
    for i, name in enumerate(names):
        print(f"{name:22s} {count[i]:7d} {iso[i]:8.1f} us   "
              + "  ".join(f"{v:5.2f}" for v in slow[i]) + f"   {where[i]:4d}")


if __name__ == "__main__":
    main()
