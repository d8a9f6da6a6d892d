#!/usr/bin/env python3
"""Benchmark of the Swimba token-mixer hot path on one MI355X.

A step = one swimba_mixer_fwd call (router + mixing, the SSM's forward) over one batch of synthetic input resident in HBM.  The headline workload is the
largest single-GPU one (long sequence, 8 B/C groups, 16 experts); the two Mamba-2-shaped layers
and the decode step ride along as extra keys of the same JSON line.  Prints ONE JSON line:
whole-path tokens/s by host clock over exactly K steps, median / min per-step times from HIP
events on the launch stream, the roofline of the whole call on its irreducible bytes, per-kernel
MFMA and HBM fractions (each kernel timed alone), the decode step, and the CPU oracle timed on
the host cores.

  python bench.py [--gpus 1] [--steps K] [--warmup W] [--workload 1|2|3] [--no-cpu] [--no-others]
"""
from __future__ import annotations

import argparse
import json
import os
import statistics
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

# MI355X published peaks
PEAK_HBM_GBS = 8000.0
PEAK_BF16_TFLOPS = 2500.0
IO_NAMES = ("x", "dt", "B_experts", "C_experts", "router_logits")


def work_model(w, live=1.0, nseg=2):
    """Algorithmic work of one forward and of each of its kernels.

    irreducible bytes: tensors that cross the library's boundary (x, y, dt, logits, the k selected
    rows of the B and C streams per token) - what any implementation has to move.
    moved bytes: what this design's kernels move, intermediates in the workspace included.
    flops: dense counts (causally skipped tiles are counted; recomputation is not)."""
    T, H, P, N, G, E, k, Q = w.tokens, w.nheads, w.headdim, w.dstate, w.ngroups, w.nexperts, w.top_k, w.chunk
    nchunks = w.batch * ((w.seqlen + Q - 1) // Q)
    state_elems = nchunks * H * P * N
    NT = Q // 32
    cb_bytes = nchunks * G * (NT * (NT + 1) // 2) * 2048
    call = {
        "irreducible_bytes": T * (2 * H * P * 2 + H * 2 + E * 2 + 2 * k * G * N * 2),
        "flops": T * (2.0 * Q * N * G + 2.0 * Q * P * H + 4.0 * N * P * H),
    }
    kernels = {
        # router + mixing: reads logits and the k active B and C rows; writes top-k, the mixed C
        # rows and the mixed B rows in two layouts (bf16)
        "mix": {"moved": T * (E * 2 + k * 8 + 2 * k * G * N * 2 + 3 * G * N * 2),
                "irreducible": T * (E * 2 + 2 * k * G * N * 2), "flops": 0.0},
        # router + mixing + C.B^T tiles per whole chunk in one persistent kernel: reads logits and the
        # selected rows; writes top-k, the mixed C rows, the mixed B rows once, and the tiles
        "mix_chunk": {"moved": T * (E * 2 + k * 8 + 2 * k * G * N * 2 + 2 * G * N * 2) + cb_bytes,
                      "irreducible": T * (E * 2 + 2 * k * G * N * 2), "flops": 2.0 * T * Q * N * G},
        # the cumsum tables alone
        "tables": {"moved": T * (H * 2 + 3 * H * 4), "irreducible": T * H * 2, "flops": 0.0},
        # C.B^T tiles from the mixed rows, cumsum tables from dt
        "prep": {"moved": T * (2 * G * N * 2 + H * 2 + H * 8) + cb_bytes,
                 "irreducible": T * H * 2, "flops": 2.0 * T * Q * N * G},
        # the single pass: reads x, dt, the tables, the mixed rows and the tiles (once per XCD, from
        # its L2, for all heads of a group), writes y; state build, state readout and the masked
        # intra-chunk contraction on MFMA, the state carried between chunks in registers
        "pass": {"moved": T * (2 * H * P * 2 + H * 2 + H * 8 + 2 * G * N * 2) + cb_bytes + 2 * w.batch * H * P * N * 4,
                 "irreducible": T * (2 * H * P * 2 + H * 2) + w.batch * H * P * N * 4,
                 "flops": 2.0 * T * Q * P * H + 4.0 * T * N * P * H},
        # ---- the staged evaluation (chunk states through memory) ----
        # (filled in below: the whole-head pass moves what the sliced pass moves)
        # cumsum + chunk state: reads x, dt, mixed B; writes cs and the bf16 chunk states
        "chunk_state": {"moved": T * (H * P * 2 + H * 2 + G * N * 2 + H * 4) + state_elems * 2,
                        "irreducible": T * (H * P * 2 + H * 2), "flops": 2.0 * T * N * P * H},
        # reads the bf16 chunk states, writes the carried states in place, and h_final; the same
        # launch reads the mixed rows and writes the causal C.B^T tiles
        "state_scan": {"moved": state_elems * 4 + w.batch * H * P * N * 4 + T * 2 * G * N * 2 + cb_bytes,
                       "irreducible": w.batch * H * P * N * 4, "flops": 2.0 * T * Q * N * G},
        # reads x, dt, cs, carried states, mixed C, C.B^T tiles; writes y
        "output": {"moved": T * (2 * H * P * 2 + H * 2 + H * 4 + G * N * 2) + state_elems * 2 + cb_bytes,
                   "irreducible": T * (2 * H * P * 2 + H * 2), "flops": 2.0 * T * Q * P * H + 2.0 * T * N * P * H},
    }
    kernels["pass64"] = kernels["pass"]
    # ---- the walk over 64-token steps ----
    # router + mixing per step: writes top-k, the C, B and C.B^T operands of a step (6 KB of 16 x 32 tiles of C.B^T; the
    # states padded to 32, 64 or 128) and, from dt, the decay tables of every head
    nsteps = w.batch * ((w.seqlen + 63) // 64)
    op_bytes = nsteps * G * (8 * (4 if N > 64 else 2 if N > 32 else 1) + 6) * 1024
    tab_bytes = nsteps * (H * (64 * 8 + 12) + G * 8)
    kernels["chain_mix"] = {"moved": T * (E * 2 + k * 8 + 2 * k * G * N * 2 + H * 2) + op_bytes + tab_bytes,
                            "irreducible": T * (E * 2 + 2 * k * G * N * 2 + H * 2), "flops": 2.0 * T * 64 * N * G}
    # x, the operands (once per XCD, from its L2, for the heads of a group) and the tables to y and the final state; cut into
    # segments, the parts in front of the last one are walked for their state alone first (`live` of them, by 64-token steps)
    first = (nseg - 1) / nseg * live
    kernels["chain_walk"] = {"moved": T * 2 * H * P * 2 + op_bytes + tab_bytes + w.batch * H * P * N * 4
                                      + first * (T * H * P * 2 + T * G * N * 2 + tab_bytes),
                             "irreducible": T * 2 * H * P * 2 + w.batch * H * P * N * 4,
                             "flops": T * H * (2.0 * 64 * P + 4.0 * N * P) + first * 2.0 * T * N * P * H}
    # split pass: the chunk states in front of the segment boundaries ((nseg - 1) / nseg of the chunks), of which
    # only the fraction `live` still counts at the boundary behind it (it depends on dt and A; the bench measures
    # it on its inputs), and the boundary states.  Nothing of it is irreducible: x and dt are read a second time.
    front = (nseg - 1) / nseg
    kernels["boundary_states"] = {"moved": front * (live * (T * (H * P * 2 + H * 2) + state_elems * 4) + T * G * N * 2)
                                           + nseg * w.batch * H * P * N * 4,
                                  "irreducible": 0.0, "flops": front * live * 2.0 * T * N * P * H}
    # short sequences: the tiles ride in the chunk-state launch, the output kernel reads the chunk states before
    # its chunk ((nc - 1) / 2 of them on average) instead of one carried state
    nc = (w.seqlen + Q - 1) // Q
    kernels["chunk_state_tiles"] = {"moved": kernels["chunk_state"]["moved"] + T * 2 * G * N * 2 + cb_bytes,
                                    "irreducible": kernels["chunk_state"]["irreducible"],
                                    "flops": kernels["chunk_state"]["flops"] + 2.0 * T * Q * N * G}
    kernels["output_carry"] = {"moved": kernels["output"]["moved"] + state_elems * (nc - 3) + w.batch * H * P * N * 4,
                               "irreducible": kernels["output"]["irreducible"] + w.batch * H * P * N * 4,
                               "flops": kernels["output"]["flops"]}
    return call, kernels


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--warmup", type=int, default=5)
    ap.add_argument("--workload", type=int, default=3, choices=(1, 2, 3),
                    help="headline workload (default: the largest single-GPU one)")
    ap.add_argument("--decode-steps", type=int, default=256)
    ap.add_argument("--no-cpu", action="store_true", help="skip the CPU oracle leg")
    ap.add_argument("--no-decode", action="store_true")
    ap.add_argument("--no-others", action="store_true", help="skip the other prefill workloads")
    ap.add_argument("--proj", type=int, default=0, metavar="D_MODEL",
                    help="also time the routed expert in-projection from token features of this width, and the calls "
                         "that train the routing on them")
    ap.add_argument("--xe", action="store_true",
                    help="also time the forward with one input stream per expert (rank-k injection)")
    ap.add_argument("--contrast", action="store_true",
                    help="also time the separated-SSM contrast (E state trajectories) on the same inputs")
    ap.add_argument("--contrast-sweep", action="store_true",
                    help="mixed against separated forward for E in {1,2,4,8,16} on the headline shape")
    ap.add_argument("--stage", default=None,
                    help="run only this stage in the timed loop (for profilers): "
                         "fwd|chain_mix|chain_walk|mix|mix_chunk|tables|prep|pass|chunk_state|state_scan|output|step|copy")
    ap.add_argument("--graph", action="store_true",
                    help="launch every timed forward call from a HIP graph captured once per input set instead of "
                         "eagerly (measured: no gain on the long-sequence workload, 7 % on the 370M-shaped one)")
    ap.add_argument("--staged", action="store_true",
                    help="also time the kernels of the evaluation the forward does not take for the headline shape "
                         "(chunk states through memory against the single pass)")
    args = ap.parse_args()
    if args.gpus != 1:
        print("bench.py: this build runs on ONE GPU only (no collectives, no sharding); "
              "run with --gpus 1", file=sys.stderr)
        return 2

    import numpy as np
    import torch
    from paper_2603_06938_amd import binding as sw
    from paper_2603_06938_amd import synth

    if not torch.cuda.is_available():
        print("bench.py: no GPU visible", file=sys.stderr)
        return 2
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    io = torch.bfloat16
    K, W = args.steps, args.warmup

    def to_dev(a, is_io):
        t = torch.from_numpy(np.ascontiguousarray(a))
        return (t.to(io) if is_io else t).to(dev)

    def time_loop(fn, n):
        """average ms per call of fn(i), measured with HIP events on the launch stream"""
        e0 = torch.cuda.Event(enable_timing=True)
        e1 = torch.cuda.Event(enable_timing=True)
        e0.record()
        for i in range(n):
            fn(i)
        e1.record()
        e1.synchronize()
        return e0.elapsed_time(e1) / n

    def per_call_times(fn, n):
        """ms of each of n calls of fn(i): one HIP event pair per call on the launch stream"""
        evs = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(n)]
        for i, (a, b) in enumerate(evs):
            a.record()
            fn(i)
            b.record()
        torch.cuda.synchronize()
        return [a.elapsed_time(b) for a, b in evs]

    def graph_of(fn, n):
        """n calls of fn(i) captured into one HIP graph (no host launch path between the kernels)"""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                for i in range(n):
                    fn(i)
        torch.cuda.current_stream().wait_stream(side)
        g.replay()
        torch.cuda.synchronize()
        return g

    class Prefill:
        """input sets of one workload on the device (several, rotated, so that a step does not find
        its inputs in the 256 MB last-level cache left by the previous step) and its step"""

        def __init__(self, w):
            self.w = w
            self.p = synth.make_inputs(w)
            base = {k: to_dev(v, k in IO_NAMES) for k, v in self.p.items()}
            self.dims = sw.dims_of(base["x"], base["B_experts"], w.top_k, w.chunk)
            ws_bytes = sw.swimba_mixer_workspace_bytes(self.dims)
            set_bytes = sum(t.numel() * t.element_size() for t in base.values()) + ws_bytes + base["x"].numel() * 2
            self.nsets = max(2, min(6, int(768e6 // set_bytes) + 1))
            self.sets = []
            for i in range(self.nsets):
                d = base if i == 0 else {k: v.clone() for k, v in base.items()}
                d["ws"] = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
                d["y"] = torch.empty_like(d["x"])
                d["h_final"] = torch.empty((w.batch, w.nheads, w.headdim, w.dstate), dtype=torch.float32, device=dev)
                self.sets.append(d)
            dims = self.dims
            mix = lambda d: sw.swimba_stage_mix(dims, d["B_experts"], d["C_experts"], d["router_logits"], d["ws"])
            # the evaluations of the forward on the MFMA path: the walk over 64-token steps, one pass over the chunks
            # with the state in registers, or chunk states through memory; swimba_mixer_fwd picks by shape
            self.paths = {
                sw.PATH_CHAIN_BF16: {
                    "chain_mix": lambda d: sw.swimba_stage_chain_mix(dims, d["dt"], d["A"], d["B_experts"], d["C_experts"],
                                                                     d["router_logits"], d["ws"]),
                    "chain_walk": lambda d: sw.swimba_stage_chain_walk(dims, d["x"], d["D"], None, d["y"], d["h_final"], d["ws"]),
                },
                sw.PATH_SINGLE_PASS: {
                    "mix": mix,
                    "prep": lambda d: sw.swimba_stage_prep(dims, d["dt"], d["A"], d["ws"]),
                    "pass": lambda d: sw.swimba_stage_pass(dims, d["x"], d["dt"], d["D"], None, d["y"], d["h_final"], d["ws"]),
                },
                sw.PATH_SINGLE_PASS_CHUNK_MIX: {
                    "mix_chunk": lambda d: sw.swimba_stage_mix_chunk(dims, d["B_experts"], d["C_experts"],
                                                                     d["router_logits"], d["ws"]),
                    "tables": lambda d: sw.swimba_stage_tables(dims, d["dt"], d["A"], d["ws"]),
                    "pass": lambda d: sw.swimba_stage_pass(dims, d["x"], d["dt"], d["D"], None, d["y"], d["h_final"], d["ws"]),
                },
                sw.PATH_SINGLE_PASS_HEAD: {
                    "mix": mix,
                    "prep": lambda d: sw.swimba_stage_prep(dims, d["dt"], d["A"], d["ws"]),
                    "pass64": lambda d: sw.swimba_stage_pass64(dims, d["x"], d["dt"], d["D"], None, d["y"], d["h_final"], d["ws"]),
                },
                sw.PATH_SINGLE_PASS_HEAD_CHUNK_MIX: {
                    "mix_chunk": lambda d: sw.swimba_stage_mix_chunk(dims, d["B_experts"], d["C_experts"],
                                                                     d["router_logits"], d["ws"]),
                    "tables": lambda d: sw.swimba_stage_tables(dims, d["dt"], d["A"], d["ws"]),
                    "pass64": lambda d: sw.swimba_stage_pass64(dims, d["x"], d["dt"], d["D"], None, d["y"], d["h_final"], d["ws"]),
                },
                sw.PATH_SINGLE_PASS_HEAD_SPLIT: {
                    "mix": mix,
                    "prep": lambda d: sw.swimba_stage_prep(dims, d["dt"], d["A"], d["ws"]),
                    "boundary_states": lambda d: sw.swimba_stage_boundary_states(dims, d["x"], d["dt"], d["A"], None,
                                                                                 self.nseg, d["ws"]),
                    "pass64": lambda d: sw.swimba_stage_pass64_split(dims, d["x"], d["dt"], d["D"], None, d["y"],
                                                                     d["h_final"], self.nseg, d["ws"]),
                },
                sw.PATH_SINGLE_PASS_HEAD_SPLIT_CHUNK_MIX: {
                    "mix_chunk": lambda d: sw.swimba_stage_mix_chunk(dims, d["B_experts"], d["C_experts"],
                                                                     d["router_logits"], d["ws"]),
                    "tables": lambda d: sw.swimba_stage_tables(dims, d["dt"], d["A"], d["ws"]),
                    "boundary_states": lambda d: sw.swimba_stage_boundary_states(dims, d["x"], d["dt"], d["A"], None,
                                                                                 self.nseg, d["ws"]),
                    "pass64": lambda d: sw.swimba_stage_pass64_split(dims, d["x"], d["dt"], d["D"], None, d["y"],
                                                                     d["h_final"], self.nseg, d["ws"]),
                },
                sw.PATH_STAGED_SHORT: {
                    "mix": mix,
                    "chunk_state_tiles": lambda d: sw.swimba_stage_chunk_state_tiles(dims, d["x"], d["dt"], d["A"], d["ws"]),
                    "output_carry": lambda d: sw.swimba_stage_output_carry(dims, d["x"], d["dt"], d["D"], None, d["y"],
                                                                           d["h_final"], d["ws"]),
                },
                sw.PATH_STAGED: {
                    "mix": mix,
                    "chunk_state": lambda d: sw.swimba_stage_chunk_state(dims, d["x"], d["dt"], d["A"], d["B_experts"], d["ws"]),
                    "state_scan": lambda d: sw.swimba_stage_state_scan(dims, None, d["h_final"], d["ws"]),
                    "output": lambda d: sw.swimba_stage_output(dims, d["x"], d["dt"], d["D"], d["B_experts"],
                                                               d["C_experts"], d["y"], d["ws"]),
                },
            }
            # the pass with one workgroup per (batch, head) instead of per 32-channel slice
            self.extra = {"pass64": lambda d: sw.swimba_stage_pass64(dims, d["x"], d["dt"], d["D"], None, d["y"],
                                                                     d["h_final"], d["ws"])}
            self.path = sw.swimba_forward_path(dims)
            self.nseg = sw.swimba_forward_segments(dims)
            self.live = 1.0
            if self.nseg > 1:
                # fraction of the (chunk, head) pairs in front of a segment boundary whose chunk state reaches
                # it with a factor of at least 2^-150 (what is computed and read for the boundary); of the walk by
                # 64-token steps
                d0 = self.sets[0]
                Q = 64 if self.path == sw.PATH_CHAIN_BF16 else w.chunk
                nper = w.seqlen // Q // self.nseg
                cut = nper * Q * self.nseg
                tot = (d0["dt"].float() * d0["A"].float())[:, :cut].reshape(w.batch, self.nseg, nper, Q, w.nheads).sum(3)
                tot = tot[:, :-1] * 1.4426950408889634
                suf = torch.flip(torch.cumsum(torch.flip(tot, (2,)), 2), (2,)) - tot
                self.live = float((suf >= -150.0).float().mean().item())
            self.path_name = {sw.PATH_CHAIN_BF16: "walk_over_64_token_steps", sw.PATH_SINGLE_PASS: "single_pass", sw.PATH_STAGED: "staged",
                              sw.PATH_SINGLE_PASS_CHUNK_MIX: "single_pass_chunk_mix",
                              sw.PATH_SINGLE_PASS_HEAD: "single_pass_head", sw.PATH_STAGED_SHORT: "staged_short",
                              sw.PATH_SINGLE_PASS_HEAD_CHUNK_MIX: "single_pass_head_chunk_mix",
                              sw.PATH_SINGLE_PASS_HEAD_SPLIT: "single_pass_head_split",
                              sw.PATH_SINGLE_PASS_HEAD_SPLIT_CHUNK_MIX: "single_pass_head_split_chunk_mix"}[self.path]
            self.other = sw.PATH_SINGLE_PASS if self.path in (sw.PATH_STAGED, sw.PATH_STAGED_SHORT) else sw.PATH_STAGED
            # the chunk-level mix takes few experts only, the short staged path few chunks
            nchunks = (w.seqlen + w.chunk - 1) // w.chunk
            self.paths = {pth: fns for pth, fns in self.paths.items()
                          if pth == self.path or not (pth in (sw.PATH_SINGLE_PASS_CHUNK_MIX, sw.PATH_SINGLE_PASS_HEAD_CHUNK_MIX,
                                                              sw.PATH_SINGLE_PASS_HEAD_SPLIT,
                                                              sw.PATH_SINGLE_PASS_HEAD_SPLIT_CHUNK_MIX)
                                                      or (pth == sw.PATH_STAGED_SHORT and nchunks > 8))}

        def step(self, i):
            d, w = self.sets[i % self.nsets], self.w
            sw.swimba_mixer_fwd(d["x"], d["dt"], d["A"], d["D"], d["B_experts"], d["C_experts"],
                                d["router_logits"], w.top_k, w.chunk, None, y=d["y"], h_final=d["h_final"],
                                workspace=d["ws"])

        def describe(self):
            w = self.w
            return "%s: B%d L%d H%d P%d N%d G%d E%d top%d chunk%d, bf16 io / fp32 accumulate" % (
                w.name, w.batch, w.seqlen, w.nheads, w.headdim, w.dstate, w.ngroups, w.nexperts, w.top_k, w.chunk)

        def whole_call(self):
            """exactly K steps by host clock between synchronisations, then K steps with one event
            pair each (median and min).  A step is one swimba_mixer_fwd call, launched eagerly, or
            with --graph from a HIP graph captured once per input set (the library's launches,
            nothing else); the eager host-clock figure is reported either way."""
            w = self.w
            for i in range(W):
                self.step(i)
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            for i in range(K):
                self.step(W + i)
            torch.cuda.synchronize()
            eager = time.perf_counter() - t0
            step = self.step
            if args.graph:
                # every replay must give what the eager call gives: checked on the first input set
                want_y, want_h = self.sets[0]["y"].clone(), self.sets[0]["h_final"].clone()
                self.graphs = [graph_of(lambda _, i=i: self.step(i), 1) for i in range(self.nsets)]
                for _ in range(2):
                    self.sets[0]["y"].zero_()
                    self.graphs[0].replay()
                    torch.cuda.synchronize()
                    if not (torch.equal(self.sets[0]["y"], want_y) and torch.equal(self.sets[0]["h_final"], want_h)):
                        raise SystemExit("a graph replay of the forward differs from the eager call")
                step = lambda i: self.graphs[i % self.nsets].replay()
                for i in range(W):
                    step(i)
                torch.cuda.synchronize()
                t0 = time.perf_counter()
                for i in range(K):
                    step(W + i)
                torch.cuda.synchronize()
            elapsed = time.perf_counter() - t0 if args.graph else eager
            ts = per_call_times(step, max(K, 30))
            self.graphs = None
            call, _ = work_model(w)
            med = statistics.median(ts)
            return {"tokens_per_s": w.tokens * K / elapsed, "ms_per_step": elapsed * 1e3 / K,
                    "ms_per_step_eager": eager * 1e3 / K,
                    "ms_median": med, "ms_min": min(ts), "reps": len(ts),
                    "hbm_frac": call["irreducible_bytes"] / med / 1e6 / PEAK_HBM_GBS,
                    "mfma_frac": call["flops"] / med / 1e9 / PEAK_BF16_TFLOPS,
                    "irreducible_MB": call["irreducible_bytes"] / 1e6, "GFLOP": call["flops"] / 1e9}

        def kernels(self, other=False):
            """each kernel of the path the forward takes for this shape (or of the other one) alone:
            K launches replayed from one HIP graph between two events"""
            _, km = work_model(self.w, self.live, max(self.nseg, 2))
            out = {}
            fns = self.paths[self.other if other else self.path]
            for fn in fns.values():   # every workspace holds this path's intermediates
                for d in self.sets:
                    fn(d)
            for name, fn in fns.items():
                time_loop(lambda i: fn(self.sets[i % self.nsets]), 3)
                g = graph_of(lambda i: fn(self.sets[i % self.nsets]), K)
                ms = time_loop(lambda i: g.replay(), 3) / K
                del g
                m = km[name]
                out[name] = {"ms": round(ms, 5),
                             "mfma_frac": round(m["flops"] / ms / 1e9 / PEAK_BF16_TFLOPS, 4),
                             "hbm_frac": round(m["irreducible"] / ms / 1e6 / PEAK_HBM_GBS, 4),
                             "hbm_frac_with_intermediates": round(m["moved"] / ms / 1e6 / PEAK_HBM_GBS, 4),
                             "mfma_TFLOPs": round(m["flops"] / ms / 1e9, 1),
                             "irreducible_MB": round(m["irreducible"] / 1e6, 2), "moved_MB": round(m["moved"] / 1e6, 2)}
            return out

        def close(self):
            self.sets = None
            self.paths = None
            torch.cuda.empty_cache()

    w = synth.workload(args.workload)
    head = Prefill(w)

    # ---- profiler mode: one stage only --------------------------------------------------
    if args.stage:
        for i in range(head.nsets):
            head.step(i)   # every workspace holds valid router/cumsum/state data
            for fns in head.paths.values():
                for fn in fns.values():
                    fn(head.sets[i])
        torch.cuda.synchronize()
        if args.stage == "copy":
            src = torch.empty(256 << 20, dtype=torch.uint8, device=dev)
            dst = torch.empty_like(src)
            ms = time_loop(lambda i: sw.swimba_probe_copy(dst, src), K)
            print(json.dumps({"stage": "copy", "bytes_per_launch": src.numel(), "ms": ms,
                              "GBps_read_plus_write": 2 * src.numel() / ms / 1e6}))
            return 0
        if args.stage == "fwd":
            ms = time_loop(head.step, K)
            print(json.dumps({"stage": "fwd", "workload": w.name, "ms": ms}))
            return 0
        if args.stage != "step":
            fn = None
            for fns in list(head.paths.values()) + [head.extra]:
                fn = fn or fns.get(args.stage)
            if fn is None:
                raise SystemExit("this workload's paths have no stage %r" % args.stage)
            ms = time_loop(lambda i: fn(head.sets[i % head.nsets]), K)
            print(json.dumps({"stage": args.stage, "workload": w.name, "ms": ms}))
            return 0

    # ---- whole path on the headline workload -----------------------------------------------
    if not args.stage:
        res = head.whole_call()
        ev_ms = res["ms_median"]
        # context: the same step on ONE input set (inputs and workspace partly found in the
        # last-level cache), the K steps replayed from one HIP graph, and what a plain copy and a
        # register-resident MFMA loop reach on this GPU
        warm_ms = time_loop(lambda i: head.step(0), K)
        g = graph_of(head.step, K)
        graph_ms = time_loop(lambda i: g.replay(), 3) / K
        del g
        src = torch.empty(256 << 20, dtype=torch.uint8, device=dev)
        dst = torch.empty_like(src)
        time_loop(lambda i: sw.swimba_probe_copy(dst, src), 2)
        cms = time_loop(lambda i: sw.swimba_probe_copy(dst, src), 10)
        del src, dst
        sink = torch.zeros(1024 * 256, device=dev)
        time_loop(lambda i: sw.swimba_probe_mfma(sink, 1024, 2048), 2)
        mms = time_loop(lambda i: sw.swimba_probe_mfma(sink, 1024, 2048), 5)
        achievable = {"copy_GBps_read_plus_write": round(2 * (256 << 20) / cms / 1e6, 1),
                      "mfma_bf16_TFLOPs": round(1024 * 4 * 2048 * 32768.0 / mms / 1e9, 1)}
        kernels = head.kernels()
        staged_kernels = None
        if args.staged:
            staged_kernels = head.kernels(other=True)

    T, H, P, N, G, E, k, Q = w.tokens, w.nheads, w.headdim, w.dstate, w.ngroups, w.nexperts, w.top_k, w.chunk

    # ---- separated-SSM contrast: E plain SSM passes through the same kernels --------------------
    contrast = None
    if args.contrast and not args.stage:
        sws = torch.empty(sw.swimba_separated_workspace_bytes(head.dims), dtype=torch.uint8, device=dev)

        def sep(i):
            d = head.sets[i % head.nsets]
            sw.swimba_separated_fwd(d["x"], d["dt"], d["A"], d["D"], d["B_experts"], d["C_experts"],
                                    d["router_logits"], w.top_k, w.chunk, y=d["y"], workspace=sws)

        time_loop(sep, 2)
        ms = time_loop(sep, max(3, K // 5))
        contrast = {"what": "MoE of separated SSMs, %d state trajectories" % w.nexperts, "ms_per_step": round(ms, 4),
                    "tokens_per_s": round(w.tokens / ms * 1e3, 1), "slowdown_vs_mixed": round(ms / ev_ms, 2)}
        del sws

    # ---- scaling in the number of experts (complexity theorem): the mixed forward advances one
    # ---- state whatever E is, the separated model advances E of them.  Headline shape, k = min(2, E),
    # ---- device-generated inputs of the workloads' distributions.
    sweep = None
    if args.contrast_sweep and not args.stage:
        sweep = {}
        x0, dt0, A0, D0 = (head.sets[0][n] for n in ("x", "dt", "A", "D"))
        y0 = head.sets[0]["y"]
        for Es in (1, 2, 4, 8, 16):
            ks = min(2, Es)
            gen = torch.Generator(device=dev)
            gen.manual_seed(69380 + 300 + Es)
            Bs = (torch.randn((w.batch, w.seqlen, Es, G, N), generator=gen, device=dev) / N ** 0.5).to(io)
            Cs = (torch.randn((w.batch, w.seqlen, Es, G, N), generator=gen, device=dev) / N ** 0.5).to(io)
            gs = torch.randn((w.batch, w.seqlen, Es), generator=gen, device=dev).to(io)
            ds = sw.dims_of(x0, Bs, ks, Q)
            mws = torch.empty(sw.swimba_mixer_workspace_bytes(ds), dtype=torch.uint8, device=dev)
            sws = torch.empty(sw.swimba_separated_workspace_bytes(ds), dtype=torch.uint8, device=dev)

            def mixed(i):
                sw.swimba_mixer_fwd(x0, dt0, A0, D0, Bs, Cs, gs, ks, Q, None, y=y0, workspace=mws)

            def separated(i):
                sw.swimba_separated_fwd(x0, dt0, A0, D0, Bs, Cs, gs, ks, Q, y=y0, workspace=sws)

            time_loop(mixed, 3)
            mm = statistics.median(per_call_times(mixed, 30))
            time_loop(separated, 1)
            sm = statistics.median(per_call_times(separated, 5 if Es > 4 else 10))
            sweep["E%d" % Es] = {"top_k": ks, "mixed_ms": round(mm, 4), "separated_ms": round(sm, 4),
                                 "ratio": round(sm / mm, 2)}
            del Bs, Cs, gs, mws, sws
            torch.cuda.empty_cache()

    # ---- routed expert in-projection (upstream of the mixer): grouped GEMM on MFMA --------------
    proj_res = None
    if args.proj and not args.stage:
        Dm = args.proj
        gen = torch.Generator(device=dev)
        gen.manual_seed(69380 + 200 + args.workload)
        us = [torch.randn((w.batch, w.seqlen, Dm), generator=gen, device=dev).to(io) for _ in range(3)]
        WBs = (torch.randn((E, G, N, Dm), generator=gen, device=dev) / Dm ** 0.5).to(io)
        WCs = (torch.randn((E, G, N, Dm), generator=gen, device=dev) / Dm ** 0.5).to(io)
        pws = torch.empty(sw.swimba_expert_proj_workspace_bytes(head.dims, Dm), dtype=torch.uint8, device=dev)

        def proj_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_expert_proj(us[i % 3], WBs, WCs, d["router_logits"], w.top_k, B_experts=d["B_experts"],
                                  C_experts=d["C_experts"], workspace=pws)

        time_loop(proj_step, 3)
        ms = time_loop(proj_step, K)
        pflops = 2.0 * T * k * Dm * 2 * G * N
        pbytes = T * (Dm * 2 + E * 2 + k * 2 * G * N * 2) + 2 * E * G * N * Dm * 2
        proj_res = {"what": "routed expert in-projection, d_model %d -> B, C rows of the top-%d experts" % (Dm, k),
                    "ms": round(ms, 5), "mfma_TFLOPs": round(pflops / ms / 1e9, 1),
                    "mfma_frac": round(pflops / ms / 1e9 / PEAK_BF16_TFLOPS, 4),
                    "hbm_GBps": round(pbytes / ms / 1e6, 1), "hbm_frac": round(pbytes / ms / 1e6 / PEAK_HBM_GBS, 4)}
        # the router's linear map on the same features
        Wg = (torch.randn((E, Dm), generator=gen, device=dev) / Dm ** 0.5).to(io)
        lg = torch.empty((w.batch, w.seqlen, E), dtype=io, device=dev)
        time_loop(lambda i: sw.swimba_router_linear(us[i % 3], Wg, lg), 3)
        rl_ms = time_loop(lambda i: sw.swimba_router_linear(us[i % 3], Wg, lg), K)
        proj_res["router_linear"] = {"ms": round(rl_ms, 5),
                                     "hbm_GBps": round(T * (Dm * 2 + E * 2) / rl_ms / 1e6, 1)}
        # token features -> y in one call, selected streams only (no tensor with an expert axis),
        # against projection into the dense layout followed by the mixer forward
        fws = torch.empty(sw.swimba_mixer_proj_workspace_bytes(head.dims, Dm), dtype=torch.uint8, device=dev)

        def fused_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_mixer_fwd_proj(us[i % 3], WBs, WCs, d["x"], d["dt"], d["A"], d["D"], d["router_logits"],
                                     w.top_k, w.chunk, y=d["y"], h_final=d["h_final"], workspace=fws)

        def dense_step(i):
            proj_step(i)
            head.step(i)

        time_loop(fused_step, 3)
        fms = time_loop(fused_step, K)
        time_loop(dense_step, 3)
        dms = time_loop(dense_step, K)
        proj_res["features_to_y"] = {"selected_streams_ms": round(fms, 5), "dense_streams_ms": round(dms, 5),
                                     "tokens_per_s": round(T / fms * 1e3, 1)}
        # the same with the experts' input streams as a third block of columns, [B | C | X], and the
        # expert-X forward on the projected rows
        WXs = (torch.randn((E, H, P, Dm), generator=gen, device=dev) / Dm ** 0.5).to(io)
        xpw = torch.empty(sw.swimba_expert_proj_x_workspace_bytes(head.dims, Dm), dtype=torch.uint8, device=dev)

        def projx_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_expert_proj_x_selected(us[i % 3], WBs, WCs, WXs, d["router_logits"], w.top_k, workspace=xpw,
                                             want_topk=False)

        time_loop(projx_step, 3)
        xms = time_loop(projx_step, K)
        xflops = 2.0 * T * k * Dm * (2 * G * N + H * P)
        xfw = torch.empty(sw.swimba_mixer_xe_proj_workspace_bytes(head.dims, Dm), dtype=torch.uint8, device=dev)

        def fused_x_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_mixer_fwd_xe_proj(us[i % 3], WBs, WCs, WXs, d["dt"], d["A"], d["D"], d["router_logits"],
                                        w.top_k, w.chunk, y=d["y"], h_final=d["h_final"], workspace=xfw)

        time_loop(fused_x_step, 3)
        fxms = time_loop(fused_x_step, K)
        proj_res["with_input_streams"] = {
            "what": "[B | C | X] rows of the top-%d experts, %d output columns" % (k, 2 * G * N + H * P),
            "ms": round(xms, 5), "mfma_TFLOPs": round(xflops / xms / 1e9, 1),
            "mfma_frac": round(xflops / xms / 1e9 / PEAK_BF16_TFLOPS, 4),
            "features_to_y_ms": round(fxms, 5), "tokens_per_s": round(T / fxms * 1e3, 1)}
        # training the routing on the same features: norm (into an fp32 residual stream), router, routing with the balance
        # loss of each sequence, and back through all of them
        gain, bias = torch.ones(Dm, device=dev), torch.zeros(Dm, device=dev)
        stream = torch.randn((w.batch, w.seqlen, Dm), generator=gen, device=dev)
        d_w = torch.randn((w.batch, w.seqlen, k), generator=gen, device=dev) / T
        d_loss = torch.full((w.batch,), 0.01 / w.batch, device=dev)
        norm = sw.swimba_layer_norm(us[0], gain, bias, 1e-5, stream, want_stats=True)
        route = sw.swimba_router_balance(sw.swimba_router_linear(norm.u, Wg), k, per_sequence=True)
        d_lg = sw.swimba_router_bwd(lg, route.topk_idx, d_w, route.counts, d_loss)
        back = sw.swimba_router_linear_bwd(norm.u, Wg, d_lg)

        def routing_step(i):
            n = sw.swimba_layer_norm(us[i % 3], gain, bias, 1e-5, stream, want_stats=True)
            sw.swimba_router_linear(n.u, Wg, lg)
            b = sw.swimba_router_balance(lg, k, per_sequence=True)
            dz = sw.swimba_router_bwd(lg, b.topk_idx, d_w, b.counts, d_loss)
            g = sw.swimba_router_linear_bwd(n.u, Wg, dz)
            sw.swimba_layer_norm_bwd(g.du, n.sum, gain, n.mean, n.rstd)

        proj_res["routing_training"] = {"what": "norm -> router -> routing with a balance loss, forward and backward"}
        for name, fn in (("layer_norm_ms", lambda i: sw.swimba_layer_norm(us[i % 3], gain, bias, 1e-5, stream, want_stats=True)),
                         ("router_balance_ms", lambda i: sw.swimba_router_balance(lg, k, per_sequence=True)),
                         ("router_bwd_ms", lambda i: sw.swimba_router_bwd(lg, route.topk_idx, d_w, route.counts, d_loss)),
                         ("router_linear_bwd_ms", lambda i: sw.swimba_router_linear_bwd(us[i % 3], Wg, d_lg)),
                         ("layer_norm_bwd_ms", lambda i: sw.swimba_layer_norm_bwd(back.du, norm.sum, gain, norm.mean, norm.rstd)),
                         ("step_ms", routing_step)):
            time_loop(fn, 3)
            proj_res["routing_training"][name] = round(time_loop(fn, K), 5)
        # the projection overwrote the synthetic expert rows of every set with its own values
        del stream, norm, route, back, d_w, d_lg
        del us, WBs, WCs, WXs, pws, fws, xpw, xfw

    # ---- one input stream per expert (rank-k injection) -------------------------------------------
    xe_res = None
    if args.xe and not args.stage:
        gen = torch.Generator(device=dev)
        gen.manual_seed(69380 + 100 + args.workload)
        xes = [torch.randn((w.batch, w.seqlen, E, H, P), generator=gen, device=dev, dtype=torch.float32).to(io)
               for _ in range(2)]
        xws = torch.empty(sw.swimba_mixer_xe_workspace_bytes(head.dims), dtype=torch.uint8, device=dev)

        def xe_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_mixer_fwd_xe(xes[i % 2], d["dt"], d["A"], d["D"], d["B_experts"], d["C_experts"],
                                   d["router_logits"], w.top_k, w.chunk, None, y=d["y"], h_final=d["h_final"],
                                   workspace=xws)

        time_loop(xe_step, 3)
        ms = time_loop(xe_step, max(5, K // 2))
        del xes, xws
        # the same forward on the rows of the selected experts only, (B,L,k,...) as a projection
        # restricted to the active set leaves them: no gather
        xss = [torch.randn((w.batch, w.seqlen, k, H, P), generator=gen, device=dev, dtype=torch.float32).to(io)
               for _ in range(2)]
        Bs_ = [torch.randn((w.batch, w.seqlen, k, G, N), generator=gen, device=dev, dtype=torch.float32).mul_(N ** -0.5).to(io)
               for _ in range(4)]
        wsel = torch.rand((w.batch, w.seqlen, k), generator=gen, device=dev, dtype=torch.float32).mul_(0.5)
        sdims = sw.make_dims(w.batch, w.seqlen, H, P, N, G, k, k, w.chunk, head.dims.io_dtype)
        sws = torch.empty(sw.swimba_mixer_xe_selected_workspace_bytes(sdims), dtype=torch.uint8, device=dev)

        def xs_step(i):
            d = head.sets[i % head.nsets]
            sw.swimba_mixer_fwd_xe_selected(xss[i % 2], d["dt"], d["A"], d["D"], Bs_[i % 2], Bs_[2 + i % 2], wsel,
                                            w.chunk, None, y=d["y"], h_final=d["h_final"], workspace=sws)

        time_loop(xs_step, 3)
        sms = time_loop(xs_step, max(5, K // 2))
        xe_res = {"what": "mixed forward with one x stream per expert (rank-%d injection)" % k,
                  "dense_input": {"what": "x_experts (B,L,E,H,P), routed inside, rows gathered once",
                                  "ms_per_step": round(ms, 4), "tokens_per_s": round(w.tokens / ms * 1e3, 1),
                                  "slowdown_vs_shared_x": round(ms / ev_ms, 2)},
                  "selected_input": {"what": "x_sel (B,L,k,H,P), B_sel, C_sel, weights given",
                                     "ms_per_step": round(sms, 4), "tokens_per_s": round(w.tokens / sms * 1e3, 1),
                                     "slowdown_vs_shared_x": round(sms / ev_ms, 2)}}
        del xss, Bs_, sws

    p_head = head.p
    head_desc, head_nsets, head_path = head.describe(), head.nsets, head.path_name
    head_split = {"segments_per_sequence": head.nseg, "states_live_at_boundary": round(head.live, 4)} if head.nseg > 1 else {}
    head.close()
    del head

    # ---- the other prefill workloads: whole call and per-kernel figures ----------------------------
    others = {}
    if not args.stage and not args.no_others:
        for wi in (1, 2, 3):
            if wi == args.workload:
                continue
            o = Prefill(synth.workload(wi))
            r = o.whole_call()
            others[o.w.name] = {"workload": o.describe(), "tokens_per_s": round(r["tokens_per_s"], 1),
                                "ms_median": round(r["ms_median"], 5), "ms_min": round(r["ms_min"], 5),
                                "ms_per_step_eager_launches": round(r["ms_per_step_eager"], 5),
                                "reps": r["reps"], "hbm_frac": round(r["hbm_frac"], 4),
                                "mfma_frac": round(r["mfma_frac"], 4), "input_sets_rotated": o.nsets,
                                "path": o.path_name, "kernels": o.kernels()}
            o.close()
            del o

    # ---- decode step (workload 4) ------------------------------------------------------------
    decode = None
    if not args.no_decode and (not args.stage or args.stage == "step"):
        wd = synth.workload(4)
        S = args.decode_steps
        pd = synth.make_decode_inputs(wd, steps=8)
        dd = {kk: to_dev(v, kk in IO_NAMES) for kk, v in pd.items()}
        xs = dd["x"].transpose(0, 1).contiguous()
        dts = dd["dt"].transpose(0, 1).contiguous()
        Bs = dd["B_experts"].transpose(0, 1).contiguous()
        Cs = dd["C_experts"].transpose(0, 1).contiguous()
        gs = dd["router_logits"].transpose(0, 1).contiguous()
        # four independent state buffers, round-robin: 4 x 134 MB > last-level cache
        states = [dd["state"].clone() for _ in range(4)]
        yd = torch.empty_like(xs[0])
        dws = torch.empty(sw.swimba_step_workspace_bytes(
            sw.make_dims(wd.batch, 1, wd.nheads, wd.headdim, wd.dstate, wd.ngroups, wd.nexperts, wd.top_k, 0, io)),
            dtype=torch.uint8, device=dev)

        def dstep(i):
            t = i % 8
            sw.swimba_step(states[i % 4], xs[t], dts[t], dd["A"], dd["D"], Bs[t], Cs[t], gs[t], wd.top_k, y=yd, workspace=dws)

        time_loop(dstep, 8)
        ms = time_loop(dstep, S)
        dts_each = per_call_times(dstep, 64)
        dbytes = 2 * wd.batch * wd.nheads * wd.headdim * wd.dstate * 4 \
            + wd.batch * (2 * wd.nheads * wd.headdim * 2 + wd.nheads * 2 + wd.nexperts * 2
                          + 2 * wd.top_k * wd.ngroups * wd.dstate * 2)
        decode = {"workload": "decode_step: B64 H64 P64 N128 G1 E8 top2, fp32 state, bf16 io",
                  "us_per_step": round(ms * 1e3, 2), "steps": S, "tokens_per_s": round(wd.batch / ms * 1e3, 1),
                  "us_median_single": round(statistics.median(dts_each) * 1e3, 2),
                  "us_min_single": round(min(dts_each) * 1e3, 2),
                  "bound": "hbm", "achieved": round(dbytes / ms / 1e6, 1), "peak": PEAK_HBM_GBS, "unit": "GB/s",
                  "frac": round(dbytes / ms / 1e6 / PEAK_HBM_GBS, 4), "state_buffers_rotated": 4}
        # the same step with other router / group settings: G = 8 B/C groups (the long-sequence
        # layer's grouping), and 4 experts with top-1 routing (the paper's large model); random
        # device-side inputs of the same distributions, same state buffers
        variants = {}
        for vname, (vG, vE, vk) in {"G8_E8_top2": (8, 8, 2), "G1_E4_top1": (1, 4, 1)}.items():
            gen = torch.Generator(device=dev)
            gen.manual_seed(69384 + vG * 100 + vE)
            vB = (torch.randn((wd.batch, vE, vG, wd.dstate), generator=gen, device=dev) / wd.dstate ** 0.5).to(io)
            vC = (torch.randn((wd.batch, vE, vG, wd.dstate), generator=gen, device=dev) / wd.dstate ** 0.5).to(io)
            vg = torch.randn((wd.batch, vE), generator=gen, device=dev).to(io)
            vws = torch.empty(sw.swimba_step_workspace_bytes(
                sw.make_dims(wd.batch, 1, wd.nheads, wd.headdim, wd.dstate, vG, vE, vk, 0, io)),
                dtype=torch.uint8, device=dev)

            def vstep(i):
                sw.swimba_step(states[i % 4], xs[i % 8], dts[i % 8], dd["A"], dd["D"], vB, vC, vg, vk, y=yd, workspace=vws)

            time_loop(vstep, 8)
            vms = time_loop(vstep, S)
            variants[vname] = {"us_per_step": round(vms * 1e3, 2), "frac": round(dbytes / vms / 1e6 / PEAK_HBM_GBS, 4)}
        decode["variants"] = variants
        # several tokens per call (speculative / short-chunk decoding): same state bytes per call
        multi = {}
        for Lm in (4, 8):
            xm = dd["x"][:, :Lm].contiguous()
            dtm = dd["dt"][:, :Lm].contiguous()
            Bm = dd["B_experts"][:, :Lm].contiguous()
            Cm = dd["C_experts"][:, :Lm].contiguous()
            gm = dd["router_logits"][:, :Lm].contiguous()
            ym = torch.empty_like(xm)
            mws = torch.empty(sw.swimba_step_multi_workspace_bytes(
                sw.make_dims(wd.batch, Lm, wd.nheads, wd.headdim, wd.dstate, wd.ngroups, wd.nexperts, wd.top_k, 0, io)),
                dtype=torch.uint8, device=dev)

            def mstep(i):
                sw.swimba_step_multi(states[i % 4], xm, dtm, dd["A"], dd["D"], Bm, Cm, gm, wd.top_k, y=ym, workspace=mws)

            time_loop(mstep, 8)
            mms = time_loop(mstep, max(32, S // 4))
            multi["L%d" % Lm] = {"us_per_call": round(mms * 1e3, 2), "tokens_per_s": round(wd.batch * Lm / mms * 1e3, 1),
                                  "frac": round(dbytes / mms / 1e6 / PEAK_HBM_GBS, 4)}
        decode["multi_token"] = multi
        if args.stage == "step":
            print(json.dumps(decode))
            return 0
        del states, dd, xs, dts, Bs, Cs, gs
        torch.cuda.empty_cache()

    # ---- CPU oracle on the host cores (reported baseline only) -------------------------------
    cpu = None
    if not args.no_cpu:
        from oracle import swimba_oracle as orc
        # a bounded sample of the headline workload: its first sequence, every head; about 10 s
        sample = {kk: (v[:1] if kk in IO_NAMES else v) for kk, v in p_head.items()}
        stoks = sample["x"].shape[0] * sample["x"].shape[1]
        runs, t_cpu = 0, 0.0
        while t_cpu < 10.0 and runs < 400:
            t0 = time.perf_counter()
            orc.mixer_fwd(sample["x"], sample["dt"], sample["A"], sample["D"], sample["B_experts"],
                          sample["C_experts"], sample["router_logits"], w.top_k)
            t_cpu += time.perf_counter() - t0
            runs += 1
        cpu = {"value": round(stoks * runs / t_cpu, 1), "unit": "tokens/s", "cores": orc.num_threads(),
               "kind": "oracle",
               "sample": "the first sequence of the %s batch (%d tokens, all heads), %d passes, fp64 sequential "
                         "recurrence, OpenMP over (batch, head)" % (w.name, stoks, runs)}

    # ---- the line ---------------------------------------------------------------------------------
    dom = max(kernels, key=lambda n: kernels[n]["ms"])
    call, _ = work_model(w)
    # HBM bytes per call measured with rocprofv3 --pmc FETCH_SIZE / WRITE_SIZE (scaled by a copy
    # kernel of known size), summed over the call's kernels; recorded in profiles/ after a counter run
    traffic = None
    tf = os.path.join(ROOT, "profiles", "hbm_traffic_mixer_fwd_%s.txt" % w.name)
    if os.path.exists(tf):
        for line in open(tf):
            if line.startswith("traffic_bytes_per_launch:"):
                traffic = float(line.split(":")[1])
    roof = {"scope": "one swimba_mixer_fwd call (all kernels), irreducible bytes over the median HIP-event time",
            "bound": "hbm", "achieved": round(call["irreducible_bytes"] / res["ms_median"] / 1e6, 1),
            "peak": PEAK_HBM_GBS, "unit": "GB/s", "frac": round(res["hbm_frac"], 4),
            "mfma_frac": round(res["mfma_frac"], 4), "traffic": traffic,
            "irreducible_bytes": call["irreducible_bytes"], "dense_flops": call["flops"],
            "dominant_kernel": dict(kernels[dom], name=dom)}
    # the targets the kernels are held to, and whether this run met them
    contr = {n: kernels[n]["mfma_frac"] for n in ("chain_walk", "pass", "pass64", "chunk_state", "output", "chunk_state_tiles",
                                                  "output_carry") if n in kernels}
    targets = {
        "contractions_mfma_frac": {"target": 0.5, "value": contr, "met": all(v >= 0.5 for v in contr.values()),
                                   "note": "the forward is HBM-bound (dense flops / irreducible bytes = %d flop/B, "
                                           "ridge 312): at the HBM floor the contractions would sit at %.2f of MFMA peak"
                                           % (round(call["flops"] / call["irreducible_bytes"]),
                                              call["flops"] / call["irreducible_bytes"] / 312.5)},
        "mixing_hbm_frac": {"target": 0.6, "value": (kernels.get("chain_mix") or kernels.get("mix") or kernels.get("mix_chunk") or {}).get("hbm_frac")},
        "scan_hbm_frac": ({"target": 0.6, "value": kernels["state_scan"]["hbm_frac_with_intermediates"],
                           "note": "on the chunk states it reads and writes (intermediates of the staged path)"}
                          if "state_scan" in kernels else
                          {"target": 0.6, "value": None,
                           "note": "the scan between chunks runs in the pass kernel's registers: no bytes of its own"}),
        "decode_hbm_frac": {"target": 0.6, "value": decode["frac"] if decode else None},
    }
    for kk in ("mixing_hbm_frac", "scan_hbm_frac", "decode_hbm_frac"):
        v = targets[kk]["value"]
        targets[kk]["met"] = None if v is None else bool(v >= targets[kk]["target"])
    out = {
        "metric": "Swimba mixer fwd tokens/s + % peak MFMA/HBM at 1 MI355X; decode step us",
        "value": round(res["tokens_per_s"], 1),
        "unit": "tokens/s",
        "n_gpus": 1,
        "steps": K,
        "warmup": W,
        "ms_per_step": round(res["ms_per_step"], 5),
        "ms_per_step_median": round(res["ms_median"], 5),
        "ms_per_step_min": round(res["ms_min"], 5),
        "timed_reps_hip_events": res["reps"],
        "ms_per_step_eager_launches": round(res["ms_per_step_eager"], 5),
        "launch": "eager" if not args.graph else "one HIP graph per step, captured once per input set; replays checked against the eager call",
        "ms_per_step_warm_cache": round(warm_ms, 5),
        "ms_per_step_k_steps_in_one_graph": round(graph_ms, 5),
        "peaks": {"hbm_GBps": PEAK_HBM_GBS, "mfma_bf16_TFLOPs": PEAK_BF16_TFLOPS},
        "achievable": achievable,
        "higher_is_better": True,
        "scaling": "weak",
        "vs_baseline": None,
        "dtype": "bf16",
        "data": "synthetic",
        "config": dict({"workload": head_desc, "input_sets_rotated": head_nsets, "path": head_path}, **head_split),
        "roofline": roof,
        "targets": targets,
        "kernels": kernels,
        "other_workloads": others,
        "decode": decode,
        "cpu_baseline": cpu,
    }
    if staged_kernels:
        out["other_path_kernels"] = staged_kernels
    if contrast:
        out["separated_contrast"] = contrast
    if sweep:
        out["expert_count_sweep"] = sweep
    if xe_res:
        out["expert_x"] = xe_res
    if proj_res:
        out["expert_proj"] = proj_res
    print(json.dumps(out))
    return 0


if __name__ == "__main__":
    sys.exit(main())
