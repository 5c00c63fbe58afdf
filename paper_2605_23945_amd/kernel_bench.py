"""Micro-benchmark of the weight-streaming projection kernels on the shapes of a configuration.

    python -m paper_2605_23945_amd.kernel_bench [--config 7b_tp1] [--batch 1,16,32,64,256] [--iters 30]
                                                 [--only gateup,down,...,barrier,append,attend,f8] [--copy-gib 1]

Each projection is run on 6 distinct weight copies in rotation (more than the 256 MB
memory-side cache holds), timed with events on the launch stream.  `--copy-gib` first runs a
plain device-to-device copy of known size: under `rocprofv3 --pmc FETCH_SIZE` / `WRITE_SIZE` its
counters calibrate the unit of the projection kernels' counters.  `--only barrier` times the device-wide barrier
of the fused layer kernel instead (pat_op_barrier_probe) among 32, 64, 128 and 256 resident workgroups.
`--only append,attend,f8` times the operators of group rollouts on the configuration's shapes: rotation and append of a step's
rows, attention of the batch as groups of eight answers to prompts of `--prefix` tokens with `--suffix` of their own, and the projections on
8-bit weights.
"""
from __future__ import annotations

import argparse
import ctypes
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def _us(run, iters):
    """Mean microseconds of a call, by events around `iters` of them."""
    import torch
    for i in range(6):
        run(i)
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for i in range(iters):
        run(i)
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) * 1e3 / iters


def operators(s, kinds, batches, shapes, args, dev="cuda:0"):
    """The operators of include/pat_operators.h on shard `s`."""
    import torch
    import paper_2605_23945_amd as pat
    bf = torch.bfloat16
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32, device=dev)
    randn = lambda *shape: torch.randn(*shape, device=dev, dtype=bf)
    hq, hkv, d, P = s.hq, s.hkv, s.head_dim, 64
    for b in batches:
        if "append" in kinds or "attend" in kinds:
            members = min(8, b)
            start = list(range(0, b, members)) + [b]
            whole, own = args.prefix // P, -(-(args.prefix % P + args.suffix) // P)
            n_pages = (len(start) - 1) * whole + b * own
            order, table, at = torch.randperm(n_pages).tolist(), [], (len(start) - 1) * whole
            for i in range(b):
                g = i // members
                table.append(order[g * whole:(g + 1) * whole] + order[at:at + own])
                at += own
            table, length = i32(table), args.prefix + args.suffix
            pools = [[randn(n_pages, hkv, P, d) for _ in range(2)] for _ in range(2)]
        if "append" in kinds:
            cs, qkv, q = pat.pat_op_rope_table(length, d, s.model.rope_base, dev), randn(b, (hq + 2 * hkv) * d), randn(b, hq, d)
            seq, pos = i32(range(b)), i32([length - 1] * b)
            us = _us(lambda i: pat.pat_op_kv_append(qkv, seq, pos, cs, *pools[i % 2], table, q), args.iters)
            print(f"append   B={b:4d} heads {hq}+{hkv}+{hkv} x {d}  {us:8.1f} us", flush=True)
        if "attend" in kinds:
            q, out = randn(b, hq, d), randn(b, hq, d)
            plan = pat.pat_op_attn_plan(i32([length] * b), i32(start), i32([args.prefix] * (len(start) - 1)), length, hq, hkv, d)
            us = _us(lambda i: pat.pat_op_attn_shared(q, *pools[i % 2], table, plan, out), args.iters)
            nbytes = ((len(start) - 1) * args.prefix + b * args.suffix) * hkv * d * 4
            print(f"attend   B={b:4d} groups of {members}, {args.prefix} + {args.suffix} tokens  {us:8.1f} us  {nbytes} B  {nbytes / us / 1e6:6.2f} TB/s", flush=True)
        if "f8" in kinds:
            for name, (n, k, _) in shapes.items():
                ws = [pat.pat_op_f8_pack_weight(randn(n, k)) for _ in range(max(1, args.copies))]
                x, y = randn(b, k), randn(b, n)
                us = _us(lambda i: pat.pat_op_f8_gemm(*ws[i % len(ws)], n, x, y), args.iters)
                print(f"f8 {name:8s} N={n:6d} K={k:6d} B={b:4d}  {us:8.1f} us  weights {n * k} B  {n * k / us / 1e6:6.2f} TB/s  {2 * n * k * b / us / 1e6:7.1f} TFLOP/s", flush=True)


def main():
    import torch
    import pat_inputs as pi
    import paper_2605_23945_amd as pat

    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="7b_tp1")
    ap.add_argument("--batch", default="1,16,32,64,256")
    ap.add_argument("--iters", type=int, default=30)
    ap.add_argument("--only", default="")
    ap.add_argument("--copy-gib", type=float, default=0.0)
    ap.add_argument("--copies", type=int, default=6, help="distinct weight copies used in rotation (1 = cache-resident if it fits)")
    ap.add_argument("--prefix", type=int, default=1024, help="shared tokens of a group (attend)")
    ap.add_argument("--suffix", type=int, default=512, help="own tokens of an answer (attend)")
    args = ap.parse_args()
    lib = pat.load_library()
    dev = "cuda:0"
    s = pi.CONFIGS[args.config]["shard"]
    H, d = s.hidden, s.head_dim
    shapes = {"qkv": (s.qkv_rows, H, 0), "o": (H, s.hq * d, 1), "gateup": (2 * s.ffn, H, 2), "down": (H, s.ffn, 1),
              "lm_head": (s.vocab, H, 0)}
    only = [x for x in args.only.split(",") if x]
    stream = torch.cuda.current_stream().cuda_stream
    if args.copy_gib > 0:
        n = int(args.copy_gib * (1 << 30))
        a = torch.empty(n, dtype=torch.uint8, device=dev).fill_(1)
        b = torch.empty_like(a)
        for _ in range(3):
            b.copy_(a)
        torch.cuda.synchronize()
        print(f"copy  {n} bytes read + {n} bytes written per launch", flush=True)
        del a, b
    if "barrier" in only:
        n_cu = torch.cuda.get_device_properties(0).multi_processor_count
        for n_wg in (32, 64, 128, 256):
            if n_wg > n_cu:
                continue
            us = [pat.pat_op_barrier_probe(n_wg, iters=500) for _ in range(3)]
            print(f"barrier  workgroups={n_wg:4d}  {min(us):6.2f} us per barrier (best of 3 x 500; others {sorted(us)[1]:.2f}, {max(us):.2f})", flush=True)
        only = [x for x in only if x != "barrier"]
        if not only:
            return
    kinds = [x for x in only if x in ("append", "attend", "f8")]
    if kinds:
        operators(s, kinds, [int(x) for x in args.batch.split(",")], shapes, args, dev)
        only = [x for x in only if x not in kinds]
        if not only:
            return
    ncopy = max(1, args.copies)
    for name, (n, k, mode) in shapes.items():
        if only and name not in only:
            continue
        wps = []
        for c in range(ncopy):
            idx = torch.arange(n * k, dtype=torch.int64, device=dev)
            w = pi.normal_bf16(pi.stream_key(77, c, len(name)), idx, 0.02).view(n, k)
            wps.append(pat.pat_op_pack_weight(w[: n // 2], w[n // 2:]) if mode == 2 else pat.pat_op_pack_weight(w))
            del w, idx
        for b in [int(x) for x in args.batch.split(",")]:
            x = torch.randn(b, k, device=dev, generator=torch.Generator(device=dev).manual_seed(b))
            hi, lo = pat.pat_op_pack_act(x)
            y = torch.zeros(b, n, device=dev) if mode != 2 else None
            nb = lib.pat_op_packed_act_bytes(b, n // 2) if mode == 2 else 0
            yh = torch.zeros(max(nb, 16), dtype=torch.uint8, device=dev)
            yl = torch.zeros_like(yh)
            sb = lib.pat_op_gemm_scratch_bytes(n, k, b)
            scratch = torch.empty(max(sb, 256), dtype=torch.uint8, device=dev)

            def run(i):
                rc = lib.pat_op_gemm(wps[i % ncopy].data_ptr(), n, k, hi.data_ptr(), lo.data_ptr(), b,
                                     y.data_ptr() if y is not None else None, n if y is not None else 0,
                                     yh.data_ptr() if mode == 2 else None, yl.data_ptr() if mode == 2 else None, mode,
                                     scratch.data_ptr() if sb > 0 else None, stream)
                assert rc == 0, rc

            for i in range(ncopy):
                run(i)
            torch.cuda.synchronize()
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            for i in range(args.iters):
                run(i)
            e1.record()
            torch.cuda.synchronize()
            us = e0.elapsed_time(e1) * 1e3 / args.iters
            plan = (ctypes.c_int32 * 4)()
            lib.pat_op_gemm_plan(n, k, b, plan)
            print(f"{name:8s} N={n:6d} K={k:6d} B={b:4d}  {us:8.1f} us  weights {n * k * 2} B  {n * k * 2 / us / 1e6:6.2f} TB/s  "
                  f"{n * k * 2 / us / 1e6 / 8.0:6.1%} of 8 TB/s  plan(kernel,Kb,Rg,tiles)={list(plan)}", flush=True)


if __name__ == "__main__":
    main()
