#!/usr/bin/env python
"""Benchmark of the verify step (one pass of the whole hot path over one batch of synthetic input).

    python bench.py --gpus N --steps K --warmup W [--workload NAME] [--impl reference]

Prints ONE JSON line.  `value` is verified tokens per second (rows pushed through verification per
second, whole job) with the step's inputs resident in device memory; `e2e` is the same metric through
the public ts_verify call with host buffers (inputs copied host->device and results device->host
inside the timed region).  Multi-GPU runs are independent replicas (the path has no exchange step).
"""
import argparse
import json
import math
import os
import statistics
import subprocess
import sys
import threading
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

# name -> (shape, [context lengths], [k per sequence])
WORKLOADS = {
    "c1_tiny_ctx256_k8": ("tiny", [256], [8]),
    "c2_1b_ctx4096_k4": ("1b", [4096], [4]),
    "c2_1b_ctx4096_k8": ("1b", [4096], [8]),
    "c2_1b_ctx4096_k16": ("1b", [4096], [16]),
    "c3_8b_ctx2048_k32": ("8b", [2048], [32]),
    "c3_8b_ctx8192_k1": ("8b", [8192], [1]),
    "c3_8b_ctx8192_k4": ("8b", [8192], [4]),
    "c3_8b_ctx8192_k8": ("8b", [8192], [8]),
    "c3_8b_ctx8192_k16": ("8b", [8192], [16]),
    "c3_8b_ctx8192_k32": ("8b", [8192], [32]),
    "c5_8b_b4_ctx8192_k64": ("8b", [8192] * 4, [64] * 4),
    # reduced-depth case for profiler captures (same per-layer kernels and grids as c3)
    "prof_8b4l_ctx8192_k32": ("8b-4l", [8192], [32]),
    "prof_8b4l_b4_ctx2048_k64": ("8b-4l", [2048] * 4, [64] * 4),
}
DEFAULT_WORKLOAD = "c3_8b_ctx8192_k32"
TRACE_TOKENS = 512          # tokens generated by the decode-loop trace (vanilla pass, then the speculative pass)
METRIC = "verified_tokens_per_s"
UNIT = "tokens/s"
# dram__bytes_read.sum + dram__bytes_write.sum per launch of the dominant kernel come from the text summary of the
# ncu capture under profiles/ (written by `bench.py --summarise-ncu`): the figure is reported only while the kernel's
# source file still has the checksum recorded there.
TRAFFIC_SUMMARY = os.path.join(ROOT, "profiles", "gemm_ws_kernel_traffic.txt")
GEMM_SOURCE = os.path.join(ROOT, "paper_2604_13519_b200", "csrc", "gemm_tcgen05.cu")


def _sha256(path):
    import hashlib
    with open(path, "rb") as f:
        return hashlib.sha256(f.read()).hexdigest()


def recorded_gemm_traffic(workload, shape, M, planes):
    """DRAM bytes (read + written) per projection-GEMM launch of `workload`, from the ncu summary under profiles/,
    or None: no summary, another workload's capture that cannot be scaled, or a kernel source that has changed since.
    The capture is taken on the 4-layer shape (same per-layer launches and grids); a full step's figure is its
    per-layer DRAM bytes x layers plus the LM-head launch at its algorithmic bytes (not captured), over all launches."""
    if not os.path.exists(TRAFFIC_SUMMARY):
        return None
    kv = {}
    for line in open(TRAFFIC_SUMMARY):
        if ":" in line and not line.startswith("#"):
            k, v = line.split(":", 1)
            kv[k.strip()] = v.strip()
    try:
        if kv["source_sha256"] != _sha256(GEMM_SOURCE):
            return None
        if kv["layer_shape"] != f"{shape.d_model}/{shape.d_ffn}/{shape.n_q_heads}/{shape.n_kv_heads}/{shape.head_dim}" \
                or int(kv["rows"]) != M or int(kv["planes"]) != planes:
            return None
        per_layer = float(kv["dram_bytes_per_layer"])
    except (KeyError, ValueError):
        return None
    lm = shape.vocab * shape.d_model * 2 + M * shape.d_model * 2 * planes + M * shape.vocab * 4
    return (per_layer * shape.n_layers + lm) / (4 * shape.n_layers + 1)


def summarise_ncu(csv_path, out_path, workload, rows, planes):
    """Write the traffic summary bench.py reads from an `ncu --csv --page raw` export that holds the projection
    launches of whole layers (metrics dram__bytes_read.sum, dram__bytes_write.sum, gpu__time_duration.sum)."""
    import csv
    import synth
    shape = synth.SHAPES[get_workload(workload)[0]]
    rd = list(csv.reader(l for l in open(csv_path, newline="") if l.startswith('"')))
    head = rd[0]
    col = {n: i for i, n in enumerate(head)}
    need = ["Kernel Name", "dram__bytes_read.sum", "dram__bytes_write.sum", "gpu__time_duration.sum"]
    for n in need:
        if n not in col:
            raise SystemExit(f"{csv_path}: column {n} missing")
    units = rd[1]
    scale = {"byte": 1.0, "Kbyte": 1e3, "Mbyte": 1e6, "Gbyte": 1e9}

    def to_bytes(r, name):
        return float(r[col[name]].replace(",", "")) * scale.get(units[col[name]], 1.0)
    launches = [r for r in rd[2:] if "gemm_ws_kernel" in r[col["Kernel Name"]]]
    if len(launches) % 4:
        raise SystemExit(f"expected the four projection launches of whole layers, found {len(launches)} launches")
    n_layers = len(launches) // 4
    total = sum(to_bytes(r, "dram__bytes_read.sum") + to_bytes(r, "dram__bytes_write.sum") for r in launches)
    with open(out_path, "w") as f:
        cmd = f"python bench.py --workload {workload} --steps 2 --warmup 3 --no-sweep --no-cpu-baseline"
        f.write("# DRAM traffic of the projection GEMM (dram__bytes_read.sum + dram__bytes_write.sum), from an ncu capture of\n"
                f"# {len(launches)} consecutive gemm_ws_kernel launches = {n_layers} layer(s).  Commands (on a B200; the plain\n"
                "# command exited 0 first in the same call):\n"
                f"#   ncu --set full --clock-control none -k regex:\"gemm_ws_kernel|attn_tc_kernel|attn_merge_kernel\" -s 50 -c 6 \\\n"
                f"#       -o prof {cmd}\n"
                "#   ncu -i prof.ncu-rep --page raw --csv > raw.csv\n"
                f"#   python bench.py --workload {workload} --summarise-ncu raw.csv {os.path.relpath(out_path, ROOT)}\n"
                "# Read by bench.py for `roofline.traffic`; valid while the source checksum below matches.\n")
        f.write("kernel: gemm_ws_kernel\n")
        f.write("source: paper_2604_13519_b200/csrc/gemm_tcgen05.cu\n")
        f.write(f"source_sha256: {_sha256(GEMM_SOURCE)}\n")
        f.write(f"workload: {workload}\n")
        f.write(f"layer_shape: {shape.d_model}/{shape.d_ffn}/{shape.n_q_heads}/{shape.n_kv_heads}/{shape.head_dim}\n")
        f.write(f"rows: {rows}\nplanes: {planes}\n")
        f.write(f"layers_captured: {n_layers}\n")
        f.write(f"dram_bytes_per_layer: {total / n_layers:.0f}\n")
        for r in launches:
            f.write(f"# {r[col['Kernel Name']][:40]:40s} read {to_bytes(r, 'dram__bytes_read.sum') / 1e6:9.2f} MB  "
                    f"write {to_bytes(r, 'dram__bytes_write.sum') / 1e6:8.2f} MB  {r[col['gpu__time_duration.sum']]} {units[col['gpu__time_duration.sum']]}\n")
    print(f"wrote {out_path}: {total / n_layers / 1e6:.1f} MB per layer over {n_layers} layer(s)")


def c4_workload():
    """Config 4: 16 sessions, contexts log-uniform over 2k..16k, k uniform in 4..32 (seeded)."""
    import numpy as np
    g = np.random.Generator(np.random.Philox(key=[260413519, 4]))
    lens = [int(round(2048 * 8 ** float(u))) for u in g.random(16)]
    ks = [int(x) for x in g.integers(4, 33, size=16)]
    return "8b", lens, ks


def get_workload(name):
    if name == "c4_8b_b16_ragged":
        return c4_workload()
    return WORKLOADS[name]


def algorithmic_bytes(shape, lens, ks, weights_held="bf16"):
    """Bytes one verify step must move: every weight matrix once, the context K/V once, the chunk's
    K/V written, the logits written, the embedding rows read (the embedding table itself is not)."""
    s = shape
    M = sum(ks)
    weights = 2 * s.n_params_matmul() if weights_held == "bf16" else s.n_params_matmul() * 17 // 32
    kv_read = sum(lens) * 4 * s.n_kv_heads * s.head_dim * s.n_layers
    kv_write = M * 4 * s.n_kv_heads * s.head_dim * s.n_layers
    return dict(weights=weights, kv_read=kv_read, kv_write=kv_write, logits=4 * M * s.vocab,
                embed=2 * M * s.d_model,
                total=weights + kv_read + kv_write + 4 * M * s.vocab + 2 * M * s.d_model)


def algorithmic_flops(shape, lens, ks):
    s = shape
    M = sum(ks)
    attn = sum(4 * s.n_q_heads * s.head_dim * s.n_layers * k * (n + k / 2) for n, k in zip(lens, ks))
    return 2 * M * s.n_params_matmul() + attn


def gemm_bytes_per_step(shape, M, planes):
    """Algorithmic bytes of the projection-GEMM launches of one step and their count: each weight
    matrix once plus the activation rows in and the result rows out."""
    s = shape
    d, F, Nq, Nkv = s.d_model, s.d_ffn, s.n_q_heads * s.head_dim, s.n_kv_heads * s.head_dim
    per_layer = [((Nq + 2 * Nkv), d, 4), (d, Nq, 4), (2 * F, d, 1 * planes), (d, F, 4)]   # (N, K, out bytes per (m, n) / 2 for swiglu)
    total = 0
    for N, K, ob in per_layer:
        out = M * N * 4 if ob == 4 else M * (N // 2) * 2 * planes
        total += N * K * 2 + M * K * 2 * planes + out
    total *= s.n_layers
    total += s.vocab * d * 2 + M * d * 2 * planes + M * s.vocab * 4
    return total, 4 * s.n_layers + 1


def measured_peaks():
    p = os.path.join(ROOT, "MEASURED_PEAKS.json")
    if os.path.exists(p):
        j = json.load(open(p))
        return dict(hbm_gbs=j["hbm_gbs"], bf16_tflops=j.get("bf16_tflops_sustained", j["bf16_tflops"]),
                    source="measured")
    return dict(hbm_gbs=6650.0, bf16_tflops=1590.0, source="fallback")


class ClockSampler:
    """Samples SM clock and throttle reasons with nvidia-smi while the timed region runs."""
    Q = ("clocks.sm,clocks.max.sm,power.draw,clocks_event_reasons.hw_slowdown,"
         "clocks_event_reasons.hw_thermal_slowdown,clocks_event_reasons.sw_thermal_slowdown,"
         "clocks_event_reasons.sw_power_cap")

    def __init__(self, uuid):
        self.uuid, self.rows, self.proc = uuid, [], None

    def start(self):
        try:
            self.proc = subprocess.Popen(["nvidia-smi", "-i", self.uuid, f"--query-gpu={self.Q}",
                                          "--format=csv,noheader,nounits", "-lms", "100"],
                                         stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True)
            threading.Thread(target=self._read, daemon=True).start()
        except Exception:
            self.proc = None

    def _read(self):
        for line in self.proc.stdout:
            self.rows.append([x.strip() for x in line.split(",")])

    def stop(self):
        if self.proc is None:
            return dict(sm_mhz=None, sm_max_mhz=None, reasons=["nvidia-smi unavailable"])
        time.sleep(0.15)
        self.proc.terminate()
        sm, mx, reasons = [], None, set()
        for r in self.rows:
            try:
                sm.append(float(r[0]))
                mx = float(r[1])
            except (ValueError, IndexError):
                continue
            for name, v in zip(("hw_slowdown", "hw_thermal_slowdown", "sw_thermal_slowdown", "sw_power_cap"), r[3:7]):
                if v.lower().startswith("active"):
                    reasons.add(name)
        return dict(sm_mhz=statistics.median(sm) if sm else None, sm_max_mhz=mx, reasons=sorted(reasons),
                    samples=len(sm))


def tree_parents(k):
    """Parent node of each of the k - 1 draft nodes: four chains hanging from the root (node 0), of about
    1/2, 1/4, 1/8 and 1/8 of the drafts -- the proportions of the 32/16/8/8 continuation lengths."""
    n = k - 1
    lens = [n - n // 2, n // 2 - n // 4, n // 4 - n // 8, n // 8]
    par, node = [], 1
    for ln in lens:
        for j in range(ln):
            par.append(0 if j == 0 else node - 1)
            node += 1
    assert len(par) == n
    return par


def dist_env():
    return int(os.environ.get("RANK", 0)), int(os.environ.get("LOCAL_RANK", 0)), int(os.environ.get("WORLD_SIZE", 1))


def max_over_ranks(value_ms: float, world: int, backend_device=None) -> float:
    """Slowest rank's time (replicas run independently; the job's time is the maximum)."""
    if world == 1:
        return value_ms
    import torch
    import torch.distributed as dist
    t = torch.tensor([value_ms], dtype=torch.float64, device=backend_device or "cpu")
    dist.all_reduce(t, op=dist.ReduceOp.MAX)
    return float(t[0])


def build_gpu_model(shape, lens, ks, act_split=True, path=0, extra_ctx=0, weights="bf16"):
    """Random-init weights generated on the device (N(0, 0.02) rounded to bf16, gains one) and a KV
    pool filled with N(0,1) fp16 values; sessions placed at their context lengths.  The model's capacity is the
    workload's: context + 2 k_max positions per sequence (+ extra_ctx for the decode-loop trace, which generates
    tokens)."""
    import torch
    import paper_2604_13519_b200 as ts
    from paper_2604_13519_b200 import binding as B
    B_, k_max = len(lens), max(max(ks), 8)
    max_ctx = max(lens) + 2 * k_max + extra_ctx
    pages = sum((n + 2 * k_max + extra_ctx + 15) // 16 for n in lens) + 8
    m = ts.Model(shape, max_pages=pages, max_batch=B_, k_max=k_max, max_rows=max(sum(ks), k_max),
                 max_ctx=max_ctx, act_split=act_split, path=path, weights=weights)
    g = torch.Generator(device="cuda").manual_seed(260413519)
    s = shape

    def rnd(r, c):
        return (torch.randn(r, c, generator=g, device="cuda", dtype=torch.float32) * 0.02).to(torch.bfloat16)
    ones = torch.ones(s.d_model, dtype=torch.float32, device="cuda")
    m.load_tensor(B.TS_W_EMBED, 0, rnd(s.vocab, s.d_model))
    m.load_tensor(B.TS_W_LM_HEAD, 0, rnd(s.vocab, s.d_model))
    m.load_tensor(B.TS_W_FINAL_GAIN, 0, ones)
    Nq, Nkv = s.n_q_heads * s.head_dim, s.n_kv_heads * s.head_dim
    for l in range(s.n_layers):
        m.load_tensor(B.TS_W_Q, l, rnd(Nq, s.d_model))
        m.load_tensor(B.TS_W_K, l, rnd(Nkv, s.d_model))
        m.load_tensor(B.TS_W_V, l, rnd(Nkv, s.d_model))
        m.load_tensor(B.TS_W_O, l, rnd(s.d_model, Nq))
        m.load_tensor(B.TS_W_GATE, l, rnd(s.d_ffn, s.d_model))
        m.load_tensor(B.TS_W_UP, l, rnd(s.d_ffn, s.d_model))
        m.load_tensor(B.TS_W_DOWN, l, rnd(s.d_model, s.d_ffn))
        m.load_tensor(B.TS_W_GAIN1, l, ones)
        m.load_tensor(B.TS_W_GAIN2, l, ones)
    kv = m.kv_pool_tensor()
    step = 1 << 28
    for i in range(0, kv.numel(), step):
        kv[i:i + step].normal_(generator=g)
    sessions = []
    for n in lens:
        ss = ts.Session(m, None, None)
        ss.set_cache(n, 3)
        sessions.append(ss)
    torch.cuda.synchronize()
    return m, sessions


def oracle_sample_seconds(shape, lens, ks, n_layers_sample):
    """Time the CPU oracle on the same chunk over the first n_layers_sample layers plus the LM head,
    then scale the per-layer part to the full depth.  Returns (seconds for a full step, threads)."""
    import torch
    import oracle
    import synth
    layers = list(range(min(n_layers_sample, shape.n_layers)))
    sub = synth.ModelShape(**{**shape.asdict(), "n_layers": len(layers), "name": shape.name + "-sample"})
    w = synth.make_weights(shape, layers=layers)
    om = oracle.OracleModel(sub, w)
    t_layers = 0.0
    t_head = 0.0
    for i, (n, k) in enumerate(zip(lens, ks)):
        K, V = synth.make_synthetic_kv(sub, n, stream=i)
        cache = om.new_cache()
        cache.import_kv(K, V)
        toks = [3] + [64 + j for j in range(k - 1)]
        t0 = time.perf_counter()
        x = om.w["embed"][torch.tensor(toks)].to(torch.float64)
        pos = torch.arange(k) + n
        for l in range(len(layers)):
            x, _, _ = om._layer(l, x, pos, cache.k[l], cache.v[l], torch.arange(n))
        t1 = time.perf_counter()
        logits = om._head(x)
        oracle.argmax_lowest(logits)
        t2 = time.perf_counter()
        t_layers += t1 - t0
        t_head += t2 - t1
    full = t_layers * shape.n_layers / len(layers) + t_head
    return full, torch.get_num_threads(), len(layers)


def run_reference(args, shape, lens, ks, name):
    """Reference arm: the CPU oracle, as it stands, on the host cores; each step a bounded sample."""
    rank, _, world = dist_env()
    if rank != 0:
        return
    n_sample = 2 if shape.n_layers > 4 else shape.n_layers
    times = []
    for i in range(args.warmup + args.steps):
        sec, threads, nl = oracle_sample_seconds(shape, lens, ks, n_sample)
        if i >= args.warmup:
            times.append(sec)
    ms = 1e3 * sum(times) / len(times)
    value = sum(ks) / (ms / 1e3)
    sample = f"chunk forward over the first {nl} of {shape.n_layers} layers + LM head, layer time scaled to full depth"
    print(json.dumps({
        "impl": "reference", "metric": METRIC, "value": value, "unit": UNIT, "n_gpus": args.gpus,
        "steps": args.steps, "warmup": args.warmup, "ms_per_step": ms, "higher_is_better": True,
        "scaling": "weak", "vs_baseline": None, "dtype": "f64", "data": "synthetic",
        "config": {"workload": name, "batch": len(lens), "context": lens, "k": ks},
        "cpu_baseline": {"value": value, "unit": UNIT, "cores": threads, "kind": "oracle", "sample": sample},
        "e2e": {"value": value, "unit": UNIT, "h2d_bytes_per_step": 0, "d2h_bytes_per_step": 0},
    }))


def run_retrieval(args, shape):
    """Top-K of Eq. 3 over N seeded N(0,1) hidden states (bf16), K = 10: one pass over N x d x 2 bytes."""
    import torch
    import synth
    import paper_2604_13519_b200 as ts
    # (the call needs a model handle for its stream and width: a two-layer one of the same width is enough)
    small = shape if shape.n_layers <= 4 else synth.SHAPES[shape.name + "-2l"]
    tiny = ts.Model(small, max_pages=8, max_batch=1, k_max=8, max_rows=8, max_ctx=64, act_split=True, path=1)
    d, N = shape.d_model, args.retrieval
    g = torch.Generator(device="cuda").manual_seed(260413519)
    H = torch.randn(N, d, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    q = torch.randn(d, generator=g, device="cuda", dtype=torch.float32)
    for _ in range(max(args.warmup, 3)):
        ts.ts_topk_cosine(tiny, H, 10, query=q)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        ts.ts_topk_cosine(tiny, H, 10, query=q)
    torch.cuda.synchronize()
    ms = 1e3 * (time.perf_counter() - t0) / args.steps
    peaks = measured_peaks()
    gbs = N * d * 2 / (ms * 1e-3) / 1e9
    print(json.dumps({"metric": "topk_cosine_ms", "value": ms, "unit": "ms", "n_gpus": 1, "steps": args.steps,
                      "warmup": max(args.warmup, 3), "higher_is_better": False, "dtype": "bf16", "data": "synthetic",
                      "config": {"workload": f"retrieval over {N} hidden states of width {d}, K = 10",
                                 "timing": "host clock around the public call (launches, result copy, stream sync)"},
                      "roofline": {"bound": "hbm", "achieved": gbs, "peak": peaks["hbm_gbs"], "unit": "GB/s",
                                   "frac": gbs / peaks["hbm_gbs"], "traffic": None, "peak_source": peaks["source"]}}))


def run_loop_trace(model, ctx, pending, k_max, jsonl_path=None):
    """The decode loop of Algorithm 1 on one sequence, timed on the host clock: first TRACE_TOKENS tokens by vanilla
    decoding (k = 1 steps), then the same context again through ts_draft -> ts_verify -> ts_commit with "self-history"
    in the datastore: the vanilla output itself, each retrieved draft corrupted at a seeded index so that the
    accepted lengths follow the paper's profile (a random-init model would reject any other draft at once).  Returns the
    throughput of both passes and the mean number of tokens emitted per step.  The two outputs must be the same ids:
    a row's logits do not depend on the rows verified beside it, so anything else is a fault and ends the run.
    jsonl_path: one record per speculative step (k, accepted length, draft source, draft / verify / commit us)."""
    import paper_2604_13519_b200 as ts
    from synth.toolcalls import planted_accept_lengths
    store = ts.Datastore(1)
    s = ts.Session(model, None, store)
    s.set_cache(ctx, pending)
    t0 = time.perf_counter()
    for _ in range(TRACE_TOKENS):
        ts.ts_commit(s, ts.ts_verify(model, [s], [[]])[0])
    van_s = time.perf_counter() - t0
    y_star = s.output()
    vocab = model.cfg.vocab
    store.add(y_star, 0)
    planted = planted_accept_lengths(TRACE_TOKENS)
    s.restart(ctx, pending)
    steps, t_draft, t_verify, t_commit, records = 0, 0.0, 0.0, 0.0, []
    t0 = time.perf_counter()
    while s.state().n_output < TRACE_TOKENS:
        a = time.perf_counter()
        d, src = ts.ts_draft(s, min(k_max - 1, TRACE_TOKENS - s.state().n_output))
        if planted[steps] < len(d):              # the retrieved draft, corrupted at the seeded index
            d[planted[steps]] = (d[planted[steps]] + 1) % vocab
        b = time.perf_counter()
        n0 = s.state().n_output
        r = ts.ts_verify(model, [s], [d])[0]
        c = time.perf_counter()
        em = list(r.emitted[:r.n_emitted])
        want = y_star[n0:n0 + len(em)]                 # (shorter than em at the very end of the trace)
        if em[:len(want)] != want:
            raise RuntimeError(f"speculative decoding left the vanilla trajectory at output token {n0}: emitted {em}, "
                               f"vanilla {want}")
        ts.ts_commit(s, r)
        e = time.perf_counter()
        t_draft += b - a; t_verify += c - b; t_commit += e - c
        records.append({"step": steps, "k": r.k, "accept_len": r.accept_len, "emitted": r.n_emitted, "source": src,
                        "draft_us": 1e6 * (b - a), "verify_us": 1e6 * (c - b), "commit_us": 1e6 * (e - c)})
        steps += 1
    spec_s = time.perf_counter() - t0
    y = s.output()
    s.close()
    if jsonl_path:
        with open(jsonl_path, "w") as f:
            for rec in records:
                f.write(json.dumps(rec) + "\n")
    vs = sorted(rec["verify_us"] for rec in records)
    return {"tokens": len(y), "steps": steps, "mean_emitted_per_step": len(y) / steps,
            "emitted_tok_s": len(y) / spec_s, "vanilla_tok_s": TRACE_TOKENS / van_s,
            "speedup_over_vanilla": (len(y) / spec_s) / (TRACE_TOKENS / van_s),
            "ms": {"draft": 1e3 * t_draft, "verify": 1e3 * t_verify, "commit": 1e3 * t_commit},
            "verify_us_p50": vs[len(vs) // 2], "verify_us_p90": vs[int(0.9 * (len(vs) - 1))],
            "steps_over_8_emitted": sum(rec["emitted"] > 8 for rec in records) / steps,
            "output_equals_vanilla": y[:TRACE_TOKENS] == y_star[:TRACE_TOKENS],
            "near_tie_resyncs": 0,
            "per_step_record": jsonl_path,
            "drafts": "retrieved from the model's own greedy output in the datastore, corrupted at seeded indices "
                      "(accepted-length profile of the paper: mean about 5, 22% above 8)"}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--warmup", type=int, default=5)
    ap.add_argument("--workload", default=DEFAULT_WORKLOAD)
    ap.add_argument("--impl", default="ours", choices=["ours", "reference"])
    ap.add_argument("--no-sweep", action="store_true", help="skip the latency-vs-k sweep")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--no-act-split", action="store_true")
    ap.add_argument("--path", type=int, default=0, help="0 auto, 1 one kernel per stage, 2 single persistent kernel")
    ap.add_argument("--weights", default="bf16", choices=["bf16", "mxfp4"], help="how the projection matrices are held")
    ap.add_argument("--retrieval", type=int, default=0,
                    help="N > 0: time ts_topk_cosine (K = 10) over N synthetic hidden states of the workload's width "
                         "instead of the verify step, and print its own JSON line")
    ap.add_argument("--want-topk", action="store_true",
                    help="also take the per-position Top-K of the logits (TS_FLAG_WANT_TOPK), as the recycling drafter needs")
    ap.add_argument("--temperature", type=float, default=0.0,
                    help="> 0: speculative-sampling acceptance at this temperature (ts_verify_sampled) with fixed uniforms")
    ap.add_argument("--trace-jsonl", default=None,
                    help="write one JSON record per step of the decode-loop trace (k, accepted length, source, draft / "
                         "verify / commit microseconds) to this file")
    ap.add_argument("--summarise-ncu", nargs=2, metavar=("RAW_CSV", "OUT_TXT"), default=None,
                    help="no benchmark: turn an `ncu -i x.ncu-rep --page raw --csv` export of whole layers' projection "
                         "launches of --workload into the traffic summary that `roofline.traffic` is read from")
    ap.add_argument("--tree", action="store_true",
                    help="verify each chunk as a draft tree (four branches from the root, lengths about 1/2, 1/4, 1/8, "
                         "1/8 of the drafts: the shape of the retrieval candidate set) through ts_verify_tree")
    args = ap.parse_args()
    args.warmup = max(args.warmup, 3) if args.impl == "ours" else args.warmup

    import synth
    shape_name, lens, ks = get_workload(args.workload)
    shape = synth.SHAPES[shape_name]
    if args.summarise_ncu:
        summarise_ncu(args.summarise_ncu[0], args.summarise_ncu[1], args.workload, sum(ks), 1 if args.no_act_split else 2)
        return
    if args.impl == "reference":
        run_reference(args, shape, lens, ks, args.workload)
        return

    import torch
    import paper_2604_13519_b200 as ts
    rank, local_rank, world = dist_env()
    if not torch.cuda.is_available():
        raise SystemExit("bench.py needs a CUDA device: the verify path has no CPU fallback")
    torch.cuda.set_device(local_rank)
    if args.retrieval > 0:
        run_retrieval(args, shape)
        return
    if world > 1:
        import torch.distributed as dist
        dist.init_process_group("nccl", device_id=torch.device("cuda", local_rank))
    ts.binding.lib()
    planes = 1 if args.no_act_split else 2
    model, sessions = build_gpu_model(shape, lens, ks, act_split=not args.no_act_split, path=args.path, weights=args.weights)
    M = sum(ks)
    drafts = [[64 + (7 * j + i) % (shape.vocab - 64) for j in range(k - 1)] for i, k in enumerate(ks)]
    stream = torch.cuda.current_stream()
    parents = [tree_parents(k) for k in ks] if args.tree else None

    uniforms = [((37 * r + 11) % 100) / 100.0 for r in range(M)]

    vflags = ts.TS_FLAG_WANT_TOPK if args.want_topk else 0

    def verify():
        if args.temperature > 0 and parents is not None:
            return ts.ts_verify_tree_sampled(model, sessions, drafts, parents, args.temperature, uniforms, flags=vflags)
        if args.temperature > 0:
            return ts.ts_verify_sampled(model, sessions, drafts, args.temperature, uniforms, flags=vflags)
        if parents is None:
            return ts.ts_verify(model, sessions, drafts, flags=vflags)
        return ts.ts_verify_tree(model, sessions, drafts, parents, flags=vflags)

    def barrier():
        if world > 1:
            torch.distributed.barrier()
        torch.cuda.synchronize()

    # ---- e2e arm: the public call with host buffers --------------------------------------------
    for _ in range(args.warmup):
        verify()
    l0, h0, d0 = model.counters()
    barrier()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        verify()
    torch.cuda.synchronize()
    e2e_ms = 1e3 * (time.perf_counter() - t0) / args.steps
    l1, h1, d1 = model.counters()
    launches_per_step = (l1 - l0) // args.steps
    e2e_ms = max_over_ranks(e2e_ms, world, "cuda")

    # ---- device-resident arm: replay the staged step ---------------------------------------------
    for _ in range(args.warmup):
        ts.ts_verify_replay(model)
    uuid = str(torch.cuda.get_device_properties(local_rank).uuid)
    sampler = ClockSampler(uuid if uuid.startswith("GPU-") else "GPU-" + uuid)
    barrier()
    sampler.start()
    ev0, ev1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    ev0.record(stream)
    for _ in range(args.steps):
        ts.ts_verify_replay(model)
    ev1.record(stream)
    barrier()
    clocks = sampler.stop()
    ms = ev0.elapsed_time(ev1) / args.steps
    ms = max_over_ranks(ms, world, "cuda")

    # ---- per-step latency distribution and the per-kernel pass -------------------------------------
    lat = []
    for _ in range(min(args.steps, 50)):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record(stream)
        ts.ts_verify_replay(model)
        b.record(stream)
        b.synchronize()
        lat.append(a.elapsed_time(b))
    prof = {}
    for _ in range(3):
        p = ts.ts_profile_step(model)
        for kcls, (pm, pn) in p.items():
            a = prof.setdefault(kcls, [0.0, 0])
            a[0] += pm / 3
            a[1] = pn
    peaks = measured_peaks()
    ab = algorithmic_bytes(shape, lens, ks, args.weights)
    fl = algorithmic_flops(shape, lens, ks)
    t_hbm = ab["total"] / (peaks["hbm_gbs"] * 1e9)
    t_tc = fl / (peaks["bf16_tflops"] * 1e12)
    bound = "hbm" if t_hbm >= t_tc else "tensor"
    fused_ms, fused_n = prof.get("fused_kernel", (0.0, 0))
    if fused_n:
        # the step is ONE launch of the persistent kernel: its algorithmic bytes are the step's; its
        # duration is the average launch duration over the timed region (launches run back to back)
        gbs = ab["total"] / (ms * 1e-3) / 1e9
        roofline = {"bound": "hbm", "kernel": "fused_verify_kernel", "achieved": gbs, "peak": peaks["hbm_gbs"],
                    "unit": "GB/s", "frac": gbs / peaks["hbm_gbs"], "traffic": None,
                    "peak_source": peaks["source"], "bytes_per_launch": ab["total"], "ms_per_launch": ms,
                    "phase_ms": {k: v[0] for k, v in prof.items() if k in ("gemm", "attention", "attention_merge")}}
    elif args.weights == "mxfp4":
        # products with MXFP4 matrices, and what prepares their input where no other kernel leaves it: the matrices once
        gemm_ms, gemm_n = prof["gemm"]
        gbs = ab["weights"] / (gemm_ms * 1e-3) / 1e9
        roofline = {"bound": "hbm", "kernel": "mx_product_kernel", "achieved": gbs, "peak": peaks["hbm_gbs"], "unit": "GB/s",
                    "frac": gbs / peaks["hbm_gbs"], "traffic": None, "peak_source": peaks["source"],
                    "bytes_per_launch": ab["weights"] / gemm_n, "ms_per_launch": gemm_ms / gemm_n}
    else:
        gemm_bytes, gemm_launches = gemm_bytes_per_step(shape, M, planes)
        gemm_ms, gemm_n = prof["gemm"]
        gemm_gbs = gemm_bytes / gemm_launches / (gemm_ms / gemm_n * 1e-3) / 1e9 if gemm_n else None
        roofline = {"bound": "hbm", "kernel": "gemm_ws_kernel", "achieved": gemm_gbs, "peak": peaks["hbm_gbs"],
                    "unit": "GB/s", "frac": gemm_gbs / peaks["hbm_gbs"] if gemm_gbs else None,
                    "traffic": recorded_gemm_traffic(args.workload, shape, M, planes), "peak_source": peaks["source"],
                    "bytes_per_launch": gemm_bytes / gemm_launches,
                    "ms_per_launch": gemm_ms / gemm_n if gemm_n else None}
    step_roof = {"bound": bound, "bytes": ab["total"], "flops": fl, "achieved_gbs": ab["total"] / (ms * 1e-3) / 1e9,
                 "frac_of_measured_hbm": ab["total"] / (ms * 1e-3) / 1e9 / peaks["hbm_gbs"],
                 "frac_of_nominal_8tbs": ab["total"] / (ms * 1e-3) / 1e9 / 8000.0,
                 "roofline_ms": 1e3 * max(t_hbm, t_tc), "frac": max(t_hbm, t_tc) / (ms * 1e-3)}

    sweep = None
    if not args.no_sweep and len(lens) == 1 and rank == 0:
        sweep = {}
        for k in sorted({1, 4, 8, 16, 32, ks[0]}):
            if k > model.cfg.k_max:
                continue
            ts.ts_verify(model, sessions, [drafts[0][:k - 1]])
            for _ in range(3):
                ts.ts_verify_replay(model)
            ls = []
            for _ in range(20):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record(stream)
                ts.ts_verify_replay(model)
                b.record(stream)
                b.synchronize()
                ls.append(a.elapsed_time(b))
            sweep[str(k)] = {"p50_ms": statistics.median(ls), "verified_tok_s": k / (statistics.median(ls) * 1e-3)}

    trace = None
    if not args.no_sweep and len(lens) == 1 and rank == 0 and world == 1:
        # the trace generates TRACE_TOKENS tokens: it gets a model of its own with room for them (the timed model
        # above has the capacity of the workload it is timed on)
        model.close()
        model, sessions = build_gpu_model(shape, lens, ks, act_split=not args.no_act_split, path=args.path, weights=args.weights,
                                          extra_ctx=TRACE_TOKENS)
        sessions[0].close()                      # its pages go back to the pool; the trace takes a session of its own
        trace = run_loop_trace(model, lens[0], 3, model.cfg.k_max, args.trace_jsonl)

    cpu = None
    if rank == 0 and world == 1 and not args.no_cpu_baseline:
        n_sample = 4 if shape.n_layers > 8 else shape.n_layers
        sec, threads, nl = oracle_sample_seconds(shape, lens, ks, n_sample)
        cpu = {"value": M / sec, "unit": UNIT, "cores": threads, "kind": "oracle",
               "sample": f"one chunk forward over the first {nl} of {shape.n_layers} layers + LM head on the same "
                         f"shapes, layer time scaled to full depth ({sec:.1f} s per step)"}

    if rank == 0:
        out = {
            "metric": METRIC, "value": world * M / (ms * 1e-3), "unit": UNIT, "n_gpus": world, "steps": args.steps,
            "warmup": args.warmup, "ms_per_step": ms, "higher_is_better": True, "scaling": "weak",
            "vs_baseline": None, "dtype": "bf16", "data": "synthetic",
            "config": {"workload": args.workload, "batch": len(lens), "context": lens, "k": ks,
                       "act_split": planes == 2, "draft_tree": bool(args.tree), "temperature": args.temperature, "per_position_topk": bool(args.want_topk), "kv_dtype": "f16", "l2": "inputs (weights) far larger than L2",
                       "parallelism": "replicas" if world > 1 else "single",
                       **({} if args.weights == "bf16" else {"weights": args.weights})},
            "latency_ms": {"p50": statistics.median(lat), "p90": sorted(lat)[int(0.9 * (len(lat) - 1))]},
            "clocks": clocks,
            "e2e": {"value": world * M / (e2e_ms * 1e-3), "unit": UNIT, "ms_per_step": e2e_ms,
                    "h2d_bytes_per_step": (h1 - h0) // args.steps, "d2h_bytes_per_step": (d1 - d0) // args.steps},
            "gpu_launches": launches_per_step * args.steps,
            "launches_per_step": launches_per_step,
            "roofline": roofline, "step_roofline": step_roof,
            "kernel_ms_per_step": {k: v[0] for k, v in prof.items()},
            "latency_vs_k": sweep, "loop_trace": trace, "cpu_baseline": cpu,
        }
        print(json.dumps(out))
    model.close()
    if world > 1:
        torch.distributed.destroy_process_group()


if __name__ == "__main__":
    main()
