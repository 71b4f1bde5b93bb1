#!/usr/bin/env python3
"""Benchmark of the hot path on one MI355X.

A "step" is one pass of the whole hot path over one batch of synthetic input: one
nt_gemm / nt_bmm / nt_conv2d_implicit call (arrangement build, lowering, kernel).  The
default workload is the one the headline metric is quoted on: the square 8192^3 fp16 GEMM
with fp32 accumulation and fp16 output.  Inputs are resident in HBM before the timed region.

Prints ONE JSON line: throughput (TFLOP/s, true 2*M*N*K flops), the roofline of the
dominant kernel from HIP-event timings of each launch, and the CPU oracle timed on a
bounded sample of the same workload (reported baseline only).
"""
from __future__ import annotations

import argparse
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

METRIC = "GEMM TFLOP/s and % of MI355X fp16 MFMA peak, 1 GPU, 8192^3 fp16"
MFMA_PEAK_TFLOPS = 2500.0          # MI355X dense fp16/bf16 matrix peak (published)
HBM_PEAK_GBS = 8000.0

# HBM bytes per launch of the dominant kernel, measured with rocprofv3 --pmc (FETCH_SIZE and WRITE_SIZE runs, scaled by a copy
# kernel of known size): profiles/traffic.json holds, per workload, the bytes, the kernel and the library version they were measured on; a
# figure measured on another version of the kernels is not reported.
def measured_traffic(workload, version):
    try:
        with open(os.path.join(ROOT, "profiles", "traffic.json")) as f:
            entry = json.load(f).get(workload)
    except (OSError, ValueError):
        return None
    if not entry or entry.get("library_version") != version:
        return None
    return int(entry["hbm_bytes_per_launch"])


def _torch_dt():
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def to_gpu(bits, dtype):
    """uint16 bit patterns -> device tensor of the 16-bit float type (no value conversion)."""
    import numpy as np
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(_torch_dt()[dtype]).cuda()


def to_f64(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


class ClockSampler:
    """Shader clock while the timed region runs, from the driver's sysfs file (the line marked '*' is the current clock)."""

    def __init__(self):
        import glob
        import threading
        self.files = sorted(glob.glob("/sys/class/drm/card*/device/pp_dpm_sclk"))
        self.samples = []
        self._stop = threading.Event()
        self._thread = threading.Thread(target=self._run, daemon=True) if self.files else None

    def _run(self):
        while not self._stop.is_set():
            try:
                for line in open(self.files[0]):
                    if "*" in line:
                        self.samples.append(int(line.split(":")[1].strip().split("Mhz")[0].split("MHz")[0]))
            except (OSError, ValueError, IndexError):
                return
            time.sleep(0.002)

    def __enter__(self):
        if self._thread:
            self._thread.start()
        return self

    def __exit__(self, *exc):
        self._stop.set()
        if self._thread:
            self._thread.join(timeout=1.0)

    def summary(self):
        if not self.samples:
            return None
        return {"mean": round(sum(self.samples) / len(self.samples), 1), "min": min(self.samples), "max": max(self.samples), "samples": len(self.samples)}


def settle_clock(step, ms=40.0):
    """The first tens of milliseconds of work after an idle period run at clocks that are still moving: untimed steps until
    `ms` of stream time have passed, whatever the warm-up count asked for.  Returns the steps taken."""
    import torch
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    n, total = 0, 0.0
    while total < ms and n < 100000:
        e0.record()
        for _ in range(8):
            step()
        e1.record()
        torch.cuda.synchronize()
        total += e0.elapsed_time(e1)
        n += 8
    return n


def mfma_only_rate(nt, data, seconds=0.25):
    """Sustained rate of the product kernels' matrix instruction alone on this workload's operand values (nt_mfma_probe)."""
    import torch
    out = torch.empty(1024 * 256, dtype=torch.float32, device="cuda")
    flat = data.reshape(-1)
    flat = flat[: min(flat.numel(), 1 << 22)]
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    flops, total, warm = 0.0, 0.0, 0.0
    while warm < seconds * 500:                                        # half the time again to settle, then the timed part
        e0.record(); nt.mfma_probe(flat, out); e1.record(); torch.cuda.synchronize()
        warm += e0.elapsed_time(e1)
    while total < seconds * 1000:
        e0.record()
        f = sum(nt.mfma_probe(flat, out) for _ in range(4))
        e1.record(); torch.cuda.synchronize()
        total += e0.elapsed_time(e1)
        flops += f
    return flops / (total * 1e-3) / 1e12


def parse_args():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=None, help="timed steps (default 50; 2000 for the kernels that run for tens of microseconds)")
    ap.add_argument("--warmup", type=int, default=None, help="untimed steps (default 50; 1000 for those short kernels)")
    ap.add_argument("--workload", default="p_f16_8192",
                    help="p_f16_8192 (default, headline), c2_f16_4096, c3_bf16_ragged, c4_f16_bmm, c5_f16_conv, c5_f16_conv_krsc, f2_f16_conv_views, c6_f16_conv_paper, c1_f16_256, f1_f16_addmm, f1_f16_bias_gelu, f3_f16_add, f3_f16_silu, f3_f16_softmax, f3_f16_rms_norm, f4_f16_sdpa, f4_bf16_sdpa, f4_f16_sdpa_4k")
    ap.add_argument("--tile", default=None, help="bm,bn,bk (default: library choice)")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--no-check", action="store_true")
    ap.add_argument("--calibrate-copy", action="store_true",
                    help="run a plain device copy of known size instead (reference for the FETCH_SIZE / WRITE_SIZE counters)")
    args = ap.parse_args()
    # The device needs some tens of milliseconds of continuous work after an idle period before its clocks settle;
    # a 10-launch warm-up of a 15 - 100 us kernel ends long before that and the timed launches then sample the transient.
    short = args.workload.startswith(("f3_", "f4_", "c6_"))
    if args.steps is None:
        args.steps = 2000 if short else 50
    if args.warmup is None:
        args.warmup = 1000 if short else 50
    return args


def flops_and_bytes(cfg):
    """True flops per step and algorithmic HBM bytes (inputs read once, output written once)."""
    osz = 4 if cfg["out"] == "f32" else 2
    if cfg["kind"] == "conv":
        N, C, H, W, K, R, S = (cfg[k] for k in ("N", "C", "H", "W", "K", "R", "S"))
        P = (H + 2 * cfg["pad"] - R) // cfg["stride"] + 1
        Q = (W + 2 * cfg["pad"] - S) // cfg["stride"] + 1
        return 2.0 * N * P * Q * K * C * R * S, 2 * (N * C * H * W + K * C * R * S) + osz * N * K * P * Q
    b = cfg.get("batch", 1)
    M, N, K = cfg["M"], cfg["N"], cfg["K"]
    extra = 0
    if cfg["kind"] == "addmm":                                       # the added input is read once
        extra = osz * N if cfg.get("bias") == "row" else osz * M * N
    return 2.0 * b * M * N * K, b * (2 * (M * K + K * N) + osz * M * N) + extra


def time_short_kernel(step, steps):
    """K back-to-back launches of a kernel that runs for tens of microseconds: one HIP event before the
    first and one after the last, so that the average is the stream time per launch and holds no event
    record between launches.  Returns (wall ms per step, kernel ms per launch)."""
    import torch
    first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    first.record()
    for _ in range(steps):
        step()
    last.record()
    torch.cuda.synchronize()
    wall = time.perf_counter() - t0
    return wall * 1e3 / steps, first.elapsed_time(last) / steps


def bench_memory_bound(args, cfg):
    """The memory-bound kernels (add, silu, softmax, rms_norm): value and roofline in GB/s of
    algorithmic HBM traffic (every input read once, the output written once)."""
    import numpy as np
    import torch
    import paper_2507_11978_amd as nt
    import synthetic_inputs as si
    TORCH_DT = _torch_dt()
    from oracle import elementwise as oe

    dt, kind = cfg["dtype"], cfg["kind"]
    if kind in ("add", "silu"):
        n = cfg["n"]
        xb = si.normal_bits((n,), dt, cfg["seed"], 2.0)
        x = to_gpu(xb, dt)
        out = torch.empty(n, dtype=TORCH_DT[dt], device="cuda")
        if kind == "add":
            yb = si.normal_bits((n,), dt, cfg["seed"] + 1, 2.0)
            y = to_gpu(yb, dt)
            step = nt.prepare(nt.add, x, y, out)              # (the call marshalled once; measured: no faster than calling nt.add each time)
            ref_fn = lambda sl: oe.add(xb[sl], yb[sl], dt)
            alg_bytes = 3 * 2 * n
        else:
            step = nt.prepare(nt.silu, x, out)
            ref_fn = lambda sl: oe.silu(xb[sl], dt)
            alg_bytes = 2 * 2 * n
        shape = {"n": n}
        sample_sl, sample_desc = slice(0, 1 << 22), "elements 0..4194303"
    else:
        rows, cols = cfg["rows"], cfg["cols"]
        xb = si.normal_bits((rows, cols), dt, cfg["seed"], 2.0)
        x = to_gpu(xb, dt)
        out = torch.empty((rows, cols), dtype=TORCH_DT[dt], device="cuda")
        if kind == "softmax":
            step = nt.prepare(nt.softmax, x, out)
            ref_fn = lambda sl: oe.softmax(xb[sl], dt)
        else:
            step = nt.prepare(nt.rms_norm, x, out, eps=cfg["eps"])
            ref_fn = lambda sl: oe.rms_norm(xb[sl], dt, cfg["eps"])
        alg_bytes = 2 * 2 * rows * cols
        shape = {"rows": rows, "cols": cols}
        sample_sl, sample_desc = slice(0, 1024), "rows 0..1023"
    for _ in range(args.warmup):
        step()
    ms_per_step, kern_avg = time_short_kernel(step, args.steps)
    achieved = alg_bytes / (kern_avg * 1e-3) / 1e9
    result = {
        "metric": f"{kind}: GB/s of algorithmic HBM traffic, 1 GPU", "value": round(alg_bytes / (ms_per_step * 1e-3) / 1e9, 1), "unit": "GB/s",
        "n_gpus": 1, "steps": args.steps, "warmup": args.warmup, "ms_per_step": round(ms_per_step, 4), "higher_is_better": True,
        "scaling": "weak", "vs_baseline": None, "dtype": dt, "data": "synthetic",
        "config": {"workload": args.workload, "shape": shape, "in_dtype": dt, "out_dtype": dt, "arithmetic": "f32"},
        "roofline": {"bound": "hbm", "achieved": round(achieved, 1), "peak": HBM_PEAK_GBS, "unit": "GB/s", "frac": round(achieved / HBM_PEAK_GBS, 4),
                     "traffic": measured_traffic(args.workload, nt.version()), "kernel_ms_avg": round(kern_avg, 5), "algorithmic_bytes": int(alg_bytes),
                     # the paper's task sizes (67 - 101 MB per launch, the same buffers every launch) fit the 256 MB Infinity Cache:
                     # part of the traffic never reaches HBM, so `frac` can exceed what HBM alone would allow
                     "working_set_fits_infinity_cache": bool(alg_bytes < 256 * 2 ** 20)},
    }
    if not args.no_check:
        got = oe.decode(out[sample_sl].contiguous().view(torch.int16).cpu().numpy().view(np.uint16), dt)
        ref = ref_fn(sample_sl)
        result["parity"] = {"sample": sample_desc, "max_abs_err": float(np.abs(got - ref).max()),
                            "max_err_in_output_ulps": float((np.abs(got - ref) / (np.abs(ref) * 2.0 ** (-10 if dt == "f16" else -7) + 2.0 ** -24)).max())}
    if not args.no_cpu_baseline:
        t1 = time.perf_counter()
        reps = 0
        while time.perf_counter() - t1 < 10.0:
            ref_fn(sample_sl)
            reps += 1
        dt_cpu = (time.perf_counter() - t1) / reps
        frac = (sample_sl.stop - sample_sl.start) / (cfg["n"] if kind in ("add", "silu") else cfg["rows"])
        result["cpu_baseline"] = {"value": round(alg_bytes * frac / dt_cpu / 1e9, 3), "unit": "GB/s", "cores": 1, "kind": "oracle",
                                  "seconds": round(dt_cpu * reps, 2), "sample": f"{sample_desc}, repeated {reps} times (numpy fp64)"}
    print(json.dumps(result), flush=True)


def bench_sdpa(args, cfg):
    """Attention forward at the paper's task shape: TFLOP/s over the 4 * B * H * S^2 * D flops of the two products."""
    import numpy as np
    import torch
    import paper_2507_11978_amd as nt
    import synthetic_inputs as si
    TORCH_DT = _torch_dt()
    from oracle import attention as oat

    dt, B, H, S, D = cfg["dtype"], cfg["B"], cfg["H"], cfg["S"], cfg["D"]
    qb, kb, vb = (si.normal_bits((B, H, S, D), dt, cfg["seed"] + i, 1.0) for i in range(3))
    q, k, v = to_gpu(qb, dt), to_gpu(kb, dt), to_gpu(vb, dt)
    out = torch.empty((B, H, S, D), dtype=TORCH_DT[dt], device="cuda")
    step = nt.prepare(nt.sdpa, q, k, v, out)
    flops = 4.0 * B * H * S * S * D
    alg_bytes = 4 * 2 * B * H * S * D
    for _ in range(args.warmup):
        step()
    ms_per_step, kern_avg = time_short_kernel(step, args.steps)
    achieved = flops / (kern_avg * 1e-3) / 1e12
    result = {
        "metric": "sdpa forward TFLOP/s (4*B*H*S^2*D flops), 1 GPU", "value": round(flops / (ms_per_step * 1e-3) / 1e12, 2), "unit": "TFLOP/s",
        "n_gpus": 1, "steps": args.steps, "warmup": args.warmup, "ms_per_step": round(ms_per_step, 4), "higher_is_better": True,
        "scaling": "weak", "vs_baseline": None, "dtype": dt, "data": "synthetic",
        "config": {"workload": args.workload, "shape": {"B": B, "H": H, "S": S, "D": D}, "in_dtype": dt, "out_dtype": dt, "accumulate": "f32"},
        "roofline": {"bound": "mfma", "achieved": round(achieved, 2), "peak": MFMA_PEAK_TFLOPS, "unit": "TFLOP/s", "frac": round(achieved / MFMA_PEAK_TFLOPS, 4),
                     "traffic": measured_traffic(args.workload, nt.version()), "kernel_ms_avg": round(kern_avg, 5), "algorithmic_bytes": int(alg_bytes),
                     # the paper's task sizes (67 - 101 MB per launch, the same buffers every launch) fit the 256 MB Infinity Cache:
                     # part of the traffic never reaches HBM, so `frac` can exceed what HBM alone would allow
                     "working_set_fits_infinity_cache": bool(alg_bytes < 256 * 2 ** 20)},
    }
    if not args.no_check:
        ref = oat.sdpa(qb[B - 1, H - 1, :256], kb[B - 1, H - 1], vb[B - 1, H - 1], dt)
        got = to_f64(out[B - 1, H - 1, :256])
        result["parity"] = {"sample": "last batch and head, query rows 0..255", "max_abs_err": float(np.abs(got - ref).max()),
                            "rel_frobenius_err": float(np.linalg.norm(got - ref) / np.linalg.norm(ref))}
    if not args.no_cpu_baseline:
        t1 = time.perf_counter()
        heads = 0
        while time.perf_counter() - t1 < 10.0:
            oat.sdpa(qb[0, heads % H], kb[0, heads % H], vb[0, heads % H], dt)
            heads += 1
        dt_cpu = time.perf_counter() - t1
        result["cpu_baseline"] = {"value": round(4.0 * S * S * D * heads / dt_cpu / 1e12, 6), "unit": "TFLOP/s", "cores": 1, "kind": "oracle",
                                  "seconds": round(dt_cpu, 2), "sample": f"{heads} heads of batch 0 (numpy fp64)"}
    print(json.dumps(result), flush=True)


def main():
    args = parse_args()
    if args.gpus != 1 or int(os.environ.get("WORLD_SIZE", "1")) != 1:
        print("bench.py: this build targets one GPU; run with --gpus 1 (no multi-GPU path exists)", file=sys.stderr)
        sys.exit(2)

    import numpy as np
    import torch
    import paper_2507_11978_amd as nt
    import synthetic_inputs as si
    TORCH_DT = _torch_dt()

    if not torch.cuda.is_available():
        print("bench.py: no GPU visible; the hot path has no CPU fallback", file=sys.stderr)
        sys.exit(3)
    if args.calibrate_copy:
        n = 1 << 30                                     # 1 GiB read + 1 GiB written per copy
        src = torch.randint(0, 255, (n,), dtype=torch.uint8, device="cuda")
        dst = torch.empty_like(src)
        torch.cuda.synchronize()
        for _ in range(args.steps):
            dst.copy_(src)
        torch.cuda.synchronize()
        print(json.dumps({"calibration": "device copy", "bytes_read_per_copy": n, "bytes_written_per_copy": n, "copies": args.steps}))
        return
    nt.load()
    cfg = si.CONFIGS[args.workload]
    if cfg["kind"] in ("add", "silu", "softmax", "rms_norm"):
        return bench_memory_bound(args, cfg)
    if cfg["kind"] == "sdpa":
        return bench_sdpa(args, cfg)
    tile = tuple(int(x) for x in args.tile.split(",")) if args.tile else cfg.get("tile")
    dt, out = cfg["dtype"], cfg["out"]

    # ---- inputs, resident in HBM before timing starts
    if cfg["kind"] == "conv":
        Xb, Wb = si.conv_inputs(cfg["N"], cfg["C"], cfg["H"], cfg["W"], cfg["K"], cfg["R"], cfg["S"], dt, cfg["seed"])
        x, w = to_gpu(Xb, dt), to_gpu(Wb, dt)
        if cfg.get("filter") == "krsc":
            w = w.permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2)       # the same tensor, stored (f, r, s, c)
        P = (cfg["H"] + 2 * cfg["pad"] - cfg["R"]) // cfg["stride"] + 1
        Q = (cfg["W"] + 2 * cfg["pad"] - cfg["S"]) // cfg["stride"] + 1
        y = torch.empty((cfg["N"], cfg["K"], P, Q), dtype=TORCH_DT[out], device="cuda")
        st, pd = (cfg["stride"],) * 2, (cfg["pad"],) * 2
        step = lambda: nt.conv2d_implicit(x, w, y, st, pd, tile=tile)
        if cfg.get("via") == "views":
            # the arrangement of Section 4.3 as a caller writes it: the input tiled by (1, C, R, S) with the convolution's
            # strides and padding and flattened to (N P Q, C R S), the filter to (C R S, K), the output to (N P Q, K)
            hi_h = (P - 1) * st[0] + cfg["R"] - cfg["H"] - pd[0]
            hi_w = (Q - 1) * st[1] + cfg["S"] - cfg["W"] - pd[1]
            px = [("tile", (1, cfg["C"], cfg["R"], cfg["S"]), (-1, -1, st[0], st[1]), ((0, 0), (0, 0), (pd[0], hi_h), (pd[1], hi_w))),
                  ("squeeze", 1), ("descend",), ("squeeze", 0), ("ascend",), ("ravel",), ("flatten", 0, 3), ("flatten", 1, 4)]
            pw = [("flatten", 1, 4), ("permute", (1, 0))]
            py = [("permute", (0, 2, 3, 1)), ("flatten", 0, 3)]
            step = lambda: nt.matmul_views(x, px, w, pw, y, py, tile=tile)
        grid, kt = nt.arrange_conv2d(x, w, y, st, pd, tile=tile)
    else:
        Ab, Bb = si.gemm_inputs(cfg["M"], cfg["N"], cfg["K"], dt, cfg["seed"], cfg["dist"], batch=cfg.get("batch"))
        a, b = to_gpu(Ab, dt), to_gpu(Bb, dt)
        shape = (cfg["batch"], cfg["M"], cfg["N"]) if cfg["kind"] == "bmm" else (cfg["M"], cfg["N"])
        y = torch.empty(shape, dtype=TORCH_DT[out], device="cuda")
        if cfg["kind"] == "addmm":
            Ib = si.normal_bits((cfg["N"],) if cfg.get("bias") == "row" else (cfg["M"], cfg["N"]), out, cfg["seed"] + 2, 1.0)
            inp = to_gpu(Ib, out)
            step = lambda: nt.addmm(inp, a, b, y, alpha=cfg["alpha"], beta=cfg["beta"], tile=tile, act=cfg.get("act"))
        else:
            fn = nt.gemm if cfg["kind"] == "gemm" else nt.bmm
            step = lambda: fn(a, b, y, tile=tile)
        grid, kt = (nt.arrange_bmm if cfg["kind"] == "bmm" else nt.arrange_gemm)(a, b, y, tile=tile)
    flops, alg_bytes = flops_and_bytes(cfg)

    # ---- clocks settled, warm-up, then exactly K timed steps bracketed by synchronisation
    settle_steps = settle_clock(step)
    for _ in range(args.warmup):
        step()
    torch.cuda.synchronize()
    sampler = ClockSampler()
    sampler.__enter__()
    if args.workload.startswith("c6_"):
        # a step of some tens of microseconds (two dependent launches: the k-split convolution and the sum of its
        # partial tiles): one event before the first step and one after the last, none in between
        ms_per_step, kern_avg = time_short_kernel(step, args.steps)
        kern_ms = np.array([kern_avg])
    else:
        starts = [torch.cuda.Event(enable_timing=True) for _ in range(args.steps)]
        ends = [torch.cuda.Event(enable_timing=True) for _ in range(args.steps)]
        t0 = time.perf_counter()
        for i in range(args.steps):
            starts[i].record()          # events on the stream the kernel is launched on (torch's current)
            step()
            ends[i].record()
        torch.cuda.synchronize()
        wall = time.perf_counter() - t0
        kern_ms = np.array([s.elapsed_time(e) for s, e in zip(starts, ends)])
        ms_per_step = wall * 1e3 / args.steps
        kern_avg = float(kern_ms.mean())
    sampler.__exit__()
    value = flops / (ms_per_step * 1e-3) / 1e12
    achieved = flops / (kern_avg * 1e-3) / 1e12
    # the matrix instruction alone on the same operand values, right behind the timed run (same clock regime)
    mfma_only = mfma_only_rate(nt, x if cfg["kind"] == "conv" else a)

    result = {
        # (the headline metric's name only for the headline workload; the other workloads say what they are)
        "metric": METRIC if args.workload == "p_f16_8192" else f"TFLOP/s and % of MI355X MFMA peak, 1 GPU, workload {args.workload}",
        "value": round(value, 2), "unit": "TFLOP/s", "n_gpus": 1,
        "steps": args.steps, "warmup": args.warmup, "ms_per_step": round(ms_per_step, 4),
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None, "dtype": dt, "data": "synthetic",
        "pct_of_mfma_peak": round(100.0 * value / MFMA_PEAK_TFLOPS, 2),
        "config": {"workload": args.workload, "shape": {k: cfg[k] for k in cfg if k in ("M", "N", "K", "batch", "C", "H", "W", "R", "S", "stride", "pad")},
                   "in_dtype": dt, "out_dtype": out, "accumulate": "f32",
                   "grid": list(grid), "k_tiles": int(kt), "tile": list(tile) if tile else "library default"},
        "roofline": {"bound": "mfma", "achieved": round(achieved, 2), "peak": MFMA_PEAK_TFLOPS, "unit": "TFLOP/s",
                     "frac": round(achieved / MFMA_PEAK_TFLOPS, 4), "traffic": measured_traffic(args.workload, nt.version()),
                     "kernel_ms_avg": round(kern_avg, 4), "kernel_ms_min": round(float(kern_ms.min()), 4),
                     "kernel_ms_median": round(float(np.median(kern_ms)), 4),
                     "algorithmic_bytes": int(alg_bytes),
                     "hbm_gbs_algorithmic": round(alg_bytes / (kern_avg * 1e-3) / 1e9, 1), "hbm_peak_gbs": HBM_PEAK_GBS,
                     "mfma_only_tflops_same_data": round(mfma_only, 1), "frac_of_mfma_only": round(achieved / mfma_only, 4),
                     "sclk_mhz": sampler.summary(), "settle_steps": settle_steps},
    }

    # ---- the CPU oracle on a bounded part of the same workload: timed (reported baseline only) and then used as the
    #      reference for every output element of that part; without it, sampled outputs one by one
    from oracle import numeric as onum
    cores = min(os.cpu_count() or 1, 16)
    gates_ok = True
    if cfg["kind"] != "conv":
        M, N, K = cfg["M"], cfg["N"], cfg["K"]
        bsel = 0
        A2, B2 = (Ab[bsel], Bb[bsel]) if cfg["kind"] == "bmm" else (Ab, Bb)
        yy = y[bsel] if cfg["kind"] == "bmm" else y

        def epilogue(prod, ms=None, ns=None):
            if cfg["kind"] != "addmm":
                return prod
            Iv = onum.decode(Ib, out)
            if ms is not None:
                Iv = Iv[ns] if cfg.get("bias") == "row" else Iv[ms, ns]
            return onum.activation(cfg["beta"] * Iv + cfg["alpha"] * prod, cfg.get("act"))

        if not args.no_cpu_baseline:
            t1 = time.perf_counter()
            prod = onum.gemm(A2, B2, dt, nthreads=cores)             # the whole product (one batch entry of a batched one)
            dt_cpu = time.perf_counter() - t1
            rows1 = max(1, min(M, int(2.5e10 / (2.0 * N * K))))      # about 10 s of one core
            t1 = time.perf_counter()
            onum.gemm(A2[:rows1], B2, dt, nthreads=1)
            dt_one = time.perf_counter() - t1
            result["cpu_baseline"] = {"value": round(2.0 * M * N * K / dt_cpu / 1e12, 6), "unit": "TFLOP/s", "cores": cores,
                                      "kind": "oracle", "seconds": round(dt_cpu, 2),
                                      "sample": f"the whole {M} x {N} x {K} product" + (" of batch entry 0" if cfg["kind"] == "bmm" else "") + " (fp64 triple loop, rows dealt to the threads)",
                                      "single_thread": {"value": round(2.0 * rows1 * N * K / dt_one / 1e12, 6), "unit": "TFLOP/s", "cores": 1,
                                                        "seconds": round(dt_one, 2), "sample": f"rows 0..{rows1 - 1} of the same product"}}
            if not args.no_check:
                ref, got, what = epilogue(prod), to_f64(yy), "every element" + (" of batch entry 0" if cfg["kind"] == "bmm" else "")
        if not args.no_check and args.no_cpu_baseline:
            rng = np.random.default_rng(7)
            ms, ns = rng.integers(0, M, 64), rng.integers(0, N, 64)
            ref = epilogue(onum.gemm_samples(A2, B2, dt, ms, ns), ms, ns)
            got, what = to_f64(yy[torch.from_numpy(ms).cuda(), torch.from_numpy(ns).cuda()]), "64 random elements"
    else:
        nf = 64
        if not args.no_cpu_baseline:
            t1 = time.perf_counter()
            slab = onum.conv2d(Xb[:1], Wb[:nf], dt, st, pd, nthreads=cores)
            dt_cpu = time.perf_counter() - t1
            fl = 2.0 * P * Q * nf * cfg["C"] * cfg["R"] * cfg["S"]
            t1 = time.perf_counter()
            onum.conv2d(Xb[:1], Wb[:4], dt, st, pd, nthreads=1)
            dt_one = time.perf_counter() - t1
            result["cpu_baseline"] = {"value": round(fl / dt_cpu / 1e12, 6), "unit": "TFLOP/s", "cores": cores, "kind": "oracle",
                                      "seconds": round(dt_cpu, 2), "sample": f"image 0, filters 0..{nf - 1} (direct fp64 convolution)",
                                      "single_thread": {"value": round(fl * 4 / nf / dt_one / 1e12, 6), "unit": "TFLOP/s", "cores": 1,
                                                        "seconds": round(dt_one, 2), "sample": "image 0, filters 0..3"}}
            if not args.no_check:
                ref, got, what = slab[0], to_f64(y[0, :nf]), f"every output of image 0, filters 0..{nf - 1}"
        if not args.no_check and args.no_cpu_baseline:
            rng = np.random.default_rng(7)
            idx = np.stack([rng.integers(0, s, 64) for s in y.shape], 1)
            ref = onum.conv2d_samples(Xb, Wb, dt, idx, st, pd)
            ti = torch.from_numpy(idx).cuda()
            got, what = to_f64(y[ti[:, 0], ti[:, 1], ti[:, 2], ti[:, 3]]), "64 random outputs"
    if not args.no_check:
        # the benchmark's gates on the output of the timed run: max |err| <= 2e-2 (16-bit outputs of unit-scale problems) and
        # relative Frobenius error <= 1e-2; an fp32 output carries fp32 accumulation error only
        max_abs = float(np.abs(got - ref).max())
        rel = float(np.linalg.norm((got - ref).ravel()) / np.linalg.norm(ref.ravel()))
        gates_ok = bool(np.isfinite(got).all()) and max_abs <= 2e-2 and rel <= (2e-5 if out == "f32" else 1e-2)
        result["parity"] = {"samples": int(ref.size), "compared": what, "max_abs_err": max_abs, "rel_frobenius_err": rel, "gates_passed": gates_ok}
    print(json.dumps(result), flush=True)
    if not gates_ok:
        print("bench.py: the timed output fails the parity gates against the oracle", file=sys.stderr)
        sys.exit(1)


if __name__ == "__main__":
    main()
