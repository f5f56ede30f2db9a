#!/usr/bin/env python3
"""Benchmark of the Hanayo per-rank hot path on one MI355X.

A "step" is one pass of the whole hot path over one batch of synthetic input:
rank 0's complete ordered task list of the workload's (P, W, M) wave schedule
(generated by the library), every task a chunk forward or backward in the
library's HIP kernels, gradients accumulated, inputs resident in HBM.

Prints ONE JSON line: chunk fwd+bwd tokens/s over the step (plus TFLOP/s and the
fraction of the bf16 MFMA peak), a `roofline` object for the dominant kernel
(the bf16 MFMA GEMM, timed live with HIP events over the GEMM launches of one
chunk forward+backward at the workload's shapes) and a `cpu_baseline` object
(the numpy oracle timed on the host cores on a bounded sample).
"""

import argparse
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

PEAK_BF16_TFLOPS = 2500.0     # MI355X dense bf16 MFMA, published
PEAK_HBM_GBS = 8000.0
CAL_COPY_BYTES = 256 << 20


def pairs_sum(wl, valid_len_all):
    """Sum over sequences of allowed (query, key) pairs of one micro-batch, averaged over micro-batches."""
    s = wl.seq
    if wl.causal:
        return wl.mb * s * (s + 1) / 2.0
    if valid_len_all is not None:
        return float(sum(int(v) for vl in valid_len_all for v in vl)) * s / len(valid_len_all)
    return wl.mb * float(s) * s


def flops_pair(wl, pairs):
    """Algorithmic forward+backward flops of one (micro-batch, chunk): per block
    72 T H^2 for the linears (F = 4H) plus 12 H * pairs for attention; masked work is not counted."""
    T, H, F = wl.tokens, wl.hidden, wl.ffn
    gemm = 3 * 2.0 * T * (H * 3 * H + H * H + 2 * H * F)
    attn = 12.0 * H * pairs
    return wl.n_blocks * (gemm + attn)


def time_gemms(wl, iters):
    """The dominant kernel, timed live: the bf16 MFMA GEMM launches of one block forward+backward
    exactly as the chunk path issues them (four forward linears with their epilogues, four
    input-gradient GEMMs, and the four weight-gradient GEMMs as one grouped launch with the bias
    gradients folded in), back to back on one stream between two HIP events, each launch with
    operands of its own.  Returns (average seconds per launch, flops per launch, launches)."""
    import torch
    from paper_2308_15762_amd import hanayo as hn
    T, H, F = wl.tokens, wl.hidden, wl.ffn
    bf = torch.bfloat16

    def act(rows, cols):
        return torch.randn((rows, cols), device="cuda").to(bf)

    def weight(k, n):
        return (0.02 * torch.randn((k, n), device="cuda")).to(bf)

    lin = [("qkv", H, 3 * H, hn.EPI_BIAS), ("o", H, H, hn.EPI_BIAS_RES), ("fc1", H, F, hn.EPI_BIAS_GELU),
           ("fc2", F, H, hn.EPI_BIAS_RES)]
    calls, group, flops = [], [], 0.0
    for name, K, N, epi in lin:
        x, W, dy = act(T, K), weight(K, N), act(T, N)
        y, bias = torch.empty((T, N), device="cuda", dtype=bf), torch.zeros(N, device="cuda", dtype=bf)
        res = act(T, N) if epi == hn.EPI_BIAS_RES else None
        pre = torch.empty((T, N), device="cuda", dtype=bf) if epi == hn.EPI_BIAS_GELU else None
        calls.append((x, W, y, T, N, K, K, N, N, False, True, epi, bias, res, pre))          # y = x W + b ...
        dx = torch.empty((T, K), device="cuda", dtype=bf)
        dgelu = name == "fc2"                                                                   # d(pre-activation)
        calls.append((dy, W, dx, T, K, N, N, N, K, False, False, hn.EPI_MUL_DGELU if dgelu else hn.EPI_NONE,
                      None, act(T, K) if dgelu else None, None))                               # dx = dy W^T
        group.append(dict(A=x, B=dy, C=torch.zeros((K, N), device="cuda"), M=K, N=N, K=T, lda=K, ldb=N, ldc=N,
                          colsum=torch.zeros(N, device="cuda"),
                          colsum_scratch=torch.empty(64 * N, device="cuda")))                  # dW += x^T dy
        flops += 3 * 2.0 * T * K * N

    # arguments marshalled once, so that the launch loop keeps the GPU's queue full
    bound = [hn.bound_op_gemm(hn.BF16, *c) for c in calls]
    bound.append(hn.bound_op_gemm_group(hn.BF16, True, True, hn.EPI_ACCUM_F32, group))

    def once():
        for f in bound:
            f()

    launches = len(bound)
    once()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(iters):
        once()
    e1.record()
    torch.cuda.synchronize()
    avg_s = e0.elapsed_time(e1) * 1e-3 / (iters * launches)
    return avg_s, flops / launches, launches


def stored_traffic(wl):
    """HBM-side bytes per GEMM launch from the committed counter summary of this workload
    (rocprofv3 FETCH_SIZE + WRITE_SIZE, scaled by the calibration copy); None if there is none."""
    path = os.path.join(ROOT, "profiles", "gemm_dma_kernel_%s_hbm_traffic.txt" % wl.name)
    try:
        for line in open(path):
            if line.startswith("traffic_bytes_per_launch:"):
                return int(line.split(":")[1])
    except OSError:
        pass
    return None


def cpu_baseline(wl, budget_s=20.0):
    """The numpy oracle, as it stands, on the host cores: forward+backward pairs of one chunk.
    `cores` = the cores this process may run on (its affinity mask); the oracle's matrix products run on the
    BLAS thread pool, whose size is stated in `sample`."""
    import numpy as np
    from oracle import block as OB
    from paper_2308_15762_amd import synth
    cores = len(os.sched_getaffinity(0))
    try:
        from threadpoolctl import threadpool_info
        blas_threads = max([p.get("num_threads", 1) for p in threadpool_info()] or [1])
    except Exception:
        blas_threads = cores
    # a bounded sample: the chunk at the workload's H/F/heads, with fewer sequences and then fewer blocks
    # if one full pair would take longer than the budget (the oracle's cost is linear in both)
    sample = wl
    cfg = OB.BlockCfg(wl.hidden, wl.heads, wl.ffn, norm=wl.norm, causal=wl.causal)
    pairs = lambda w: pairs_sum(w, None if w.valid_len_range is None else [[w.seq] * w.mb])
    assumed_rate = 50e9 * max(1, min(cores, blas_threads) / 8)     # fp64 numpy, as the parity tests use it
    if flops_pair(sample, pairs(sample)) / assumed_rate > budget_s and sample.mb > 1:
        sample = sample.scaled(mb=1)
    if flops_pair(sample, pairs(sample)) / assumed_rate > budget_s and sample.n_blocks > 1:
        sample = sample.scaled(n_blocks=1)
    params = synth.chunk_params(sample, 0)
    x = synth.forward_input(sample, 0, 0)
    dy = synth.upstream_grad(sample, 0, 0)
    vl = synth.valid_lengths(sample, 0)
    t0 = time.perf_counter()
    n = 0
    while True:
        y, st = OB.chunk_forward(params, x, cfg, vl)
        OB.chunk_backward(cfg, st, dy)
        n += 1
        el = time.perf_counter() - t0
        if el > budget_s * 0.5 or n >= 8:
            break
    tok_s = n * sample.tokens / el
    # tokens through a whole chunk per second: a sample of fewer blocks is scaled to the chunk's block count
    tok_s *= sample.n_blocks / wl.n_blocks
    return {"value": tok_s, "unit": "chunk fwd+bwd tokens/s", "cores": int(cores), "kind": "oracle",
            "sample": "%d fwd+bwd pair(s) of %d of the chunk's %d blocks, %d tokens each (mb=%d of %d), numpy fp64 on a "
                      "BLAS pool of %d threads, %.1f s"
                      % (n, sample.n_blocks, wl.n_blocks, sample.tokens, sample.mb, wl.mb, blas_threads, el)}


def copy_yardstick(mibs):
    """What a plain device copy reaches at a given tensor size: the yardstick for the memory-bound kernels,
    whose launches at the workloads' tensor sizes are over before the memory system is saturated.  Times the
    library's copy kernel, rotating over enough buffer pairs (1 GiB) that nothing stays cache-resident."""
    import torch
    from paper_2308_15762_amd import hanayo as hn
    for mib in mibs:
        n = mib << 20
        pairs = max(2, (1024 << 20) // (2 * n))
        bufs = [(torch.empty(n, dtype=torch.uint8, device="cuda").random_(0, 255),
                 torch.empty(n, dtype=torch.uint8, device="cuda")) for _ in range(pairs)]
        for a, b in bufs:
            hn.hanayo_op_copy(b, a, n)
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        count = 0
        e0.record()
        for _ in range(4):
            for a, b in bufs:
                hn.hanayo_op_copy(b, a, n)
                count += 1
        e1.record()
        torch.cuda.synchronize()
        us = e0.elapsed_time(e1) * 1e3 / count
        print("copy_kernel %4d MiB read + %4d MiB written (%3d buffer pairs in rotation): %8.2f us  %7.1f GB/s"
              % (mib, mib, pairs, us, 2 * n / us / 1e3), flush=True)
        del bufs


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--workload", default="gpt_4096_bf16",
                    help="default: the largest single-GPU configuration (rank 0 of P=16, W=2, M=32 at H=4096); "
                         "gpt_1024_bf16, bert_1024_bf16, gpt_2560_wave4_bf16 and tiny_gpt_fp32 are the others")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--gemm-config", type=int, default=-1, help="measurement knob, see hanayo_op_gemm_config")
    ap.add_argument("--stash", choices=["full", "input"], default="full",
                    help="what a stash entry holds: everything the forward materialises, or the chunk input only "
                         "(backward then recomputes the forward)")
    ap.add_argument("--lanes", type=int, default=4, help="HIP streams the executor spreads independent tasks over")
    ap.add_argument("--ends", action="store_true",
                    help="rank 0 also embeds the tokens in front of stage 0 and ends the last stage in head + loss "
                         "(not part of the headline metric's step; its flops are added to the TFLOP/s figure)")
    ap.add_argument("--adam", action="store_true", help="every step ends with the Adam update of all the rank's parameters")
    ap.add_argument("--max-norm", type=float, default=None, help="with --adam: the gradients are clipped to this norm in the update")
    ap.add_argument("--copy-yardstick", type=int, nargs="*", metavar="MIB", default=None,
                    help="instead of the benchmark: time the plain copy kernel at these sizes (MiB read and as many "
                         "written; default 4 8 16 32 64 256), the yardstick of the memory-bound kernels")
    args = ap.parse_args()
    if args.max_norm is not None and not args.adam:
        ap.error("--max-norm clips in the Adam update: it needs --adam")
    if args.gpus != 1:
        sys.exit("bench.py: this build covers one GPU's share of the pipeline (one rank); --gpus must be 1")

    import torch
    from paper_2308_15762_amd import hanayo as hn
    from paper_2308_15762_amd import synth
    from paper_2308_15762_amd.runner import GpuRank

    if not torch.cuda.is_available():
        sys.exit("bench.py: no GPU")
    if args.copy_yardstick is not None:
        copy_yardstick(args.copy_yardstick or [4, 8, 16, 32, 64, 256])
        return
    wl = synth.WORKLOADS[args.workload]
    hn.hanayo_op_gemm_config(args.gemm_config)
    rank = 0
    gpu = GpuRank(wl, rank, lanes=args.lanes, stash_mode=1 if args.stash == "input" else 0, ends=args.ends)
    n_tasks = len(gpu.tasks)
    pairs_per_step = n_tasks // 2
    vls = None if wl.valid_len_range is None else [synth.valid_lengths(wl, m) for m in range(wl.M)]
    flops_step = pairs_per_step * flops_pair(wl, pairs_sum(wl, vls))
    if args.ends:
        flops_step += wl.M * 3 * 2.0 * wl.tokens * wl.hidden * wl.vocab      # logits, d_head, d_hidden per micro-batch
    if args.adam:
        gpu.init_optimizer()

    def step():
        if not args.adam:
            gpu.zero_grads()
        peak = gpu.run()
        if args.adam:
            gpu.adam_step(1e-4, weight_decay=0.01, max_norm=args.max_norm)         # clears the gradients as it goes
        return peak

    # one plain copy of known size: the dispatch the HBM traffic counters of a profiler run are scaled by
    cal = torch.empty(2, CAL_COPY_BYTES, dtype=torch.uint8, device="cuda")
    hn.hanayo_op_copy(cal[1], cal[0], CAL_COPY_BYTES)
    del cal

    for _ in range(args.warmup):
        step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        peak = step()
    torch.cuda.synchronize()
    el = time.perf_counter() - t0
    ms_per_step = el / args.steps * 1e3
    tok_s = pairs_per_step * wl.tokens / (ms_per_step * 1e-3)
    tflops = flops_step / (ms_per_step * 1e-3) / 1e12

    avg_s, gemm_flops, n_gemm = time_gemms(wl, iters=10)
    achieved = gemm_flops / avg_s / 1e12
    out = {
        "metric": "chunk fwd+bwd tokens/sec and TFLOP/s (% bf16 MFMA peak) per MI355X",
        "value": tok_s, "unit": "chunk fwd+bwd tokens/s",
        "n_gpus": 1, "steps": args.steps, "warmup": args.warmup, "ms_per_step": ms_per_step,
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None,
        "dtype": "bf16" if wl.dtype == "bf16" else "f32", "data": "synthetic",
        "tflops": tflops, "pct_bf16_mfma_peak": 100.0 * tflops / PEAK_BF16_TFLOPS,
        "block_tokens_per_s": tok_s * wl.n_blocks,                      # the same per transformer block
        "rank_tokens_per_s": wl.M * wl.tokens / (ms_per_step * 1e-3),   # micro-batch tokens through the whole rank
        "config": {"workload": "%s: rank %d of P=%d W=%d M=%d, %d tasks/step, chunk = %d %s-LN blocks H=%d heads=%d "
                               "F=%d seq=%d mb=%d" % (wl.name, rank, wl.P, wl.W, wl.M, n_tasks, wl.n_blocks, wl.norm,
                                                      wl.hidden, wl.heads, wl.ffn, wl.seq, wl.mb),
                   "executor_lanes": args.lanes, "stash": args.stash, "model_ends": bool(args.ends), "adam": bool(args.adam), "max_norm": args.max_norm, "stash_peak": peak, "stash_arena_gib": gpu.arena_bytes / 2 ** 30},
        "roofline": {"bound": "mfma", "achieved": achieved, "peak": PEAK_BF16_TFLOPS, "unit": "TFLOP/s",
                     "frac": achieved / PEAK_BF16_TFLOPS, "traffic": stored_traffic(wl),
                     "kernel": "gemm_dma_kernel (bf16 MFMA; the %d GEMM launches of one block fwd+bwd, alone on the chip)" % n_gemm,
                     "avg_launch_us": avg_s * 1e6, "flops_per_launch": gemm_flops},
    }
    if not args.no_cpu_baseline:
        out["cpu_baseline"] = cpu_baseline(wl)
    print(json.dumps(out))


if __name__ == "__main__":
    main()
