"""Runs the fused SC+LWP update over plain arrays, and a plain copy of known size beside it.

Used under `rocprofv3 --pmc FETCH_SIZE` / `--pmc WRITE_SIZE` to read the HBM traffic of the update
kernel: the copy kernel (torch's `copy_`, n floats read and n written) calibrates what the counter
reports per byte moved.

    python3 -m paper_2003_11666_amd.update_bench [--elements N] [--reps R] [--adamw 32|8]

--adamw: also the AdamW step over as many weights, in 16 tensors, with moments in so many bits.
"""
from __future__ import annotations

import argparse
import json
import time


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--elements", type=int, default=256 * 1024 * 1024)
    ap.add_argument("--reps", type=int, default=5)
    ap.add_argument("--adamw", type=int, choices=(32, 8))
    args = ap.parse_args()
    import torch
    from paper_2003_11666_amd import update_standalone

    dev = torch.device("cuda:0")
    n = args.elements
    w = torch.randn(n, device=dev)
    v = torch.zeros(n, device=dev)
    g = torch.randn(n, device=dev)
    wh = torch.empty(n, device=dev)
    dst = torch.empty(n, device=dev)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.reps):
        update_standalone(w, v, g, wh, 0.005, 0.9, 0.5, 4.0, 0.05)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    for _ in range(args.reps):
        dst.copy_(w)
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    out = {"elements": n, "reps": args.reps,
           "update_bytes_per_launch": 24 * n, "update_us": 1e6 * (t1 - t0) / args.reps,
           "copy_bytes_per_launch": 8 * n, "copy_us": 1e6 * (t2 - t1) / args.reps}
    if args.adamw:
        from paper_2003_11666_amd import ADAMW_BLOCK, adamw_elements, adamw_step
        ws, gs = w.chunk(16), g.chunk(16)
        total, kind = adamw_elements(ws), torch.uint8 if args.adamw == 8 else torch.float32
        ms = [torch.zeros(total, dtype=kind, device=dev) for _ in range(2)]
        exps = [torch.zeros(total // ADAMW_BLOCK, dtype=torch.uint8, device=dev) if args.adamw == 8 else None for _ in range(2)]

        def step(t):
            adamw_step(ws, gs, *ms, m_exp=exps[0], v_exp=exps[1], step=t, lr=1e-3)

        step(1)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for t in range(args.reps):
            step(2 + t)
        torch.cuda.synchronize()
        out |= {"adamw_moment_bits": args.adamw, "adamw_bytes_per_step": (28 if args.adamw == 32 else 16) * n + (4 * n // ADAMW_BLOCK if args.adamw == 8 else 0),
                "adamw_us": 1e6 * (time.perf_counter() - t0) / args.reps}
    print(json.dumps(out))


if __name__ == "__main__":
    main()
