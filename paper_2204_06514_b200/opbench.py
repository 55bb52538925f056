"""Per-operator micro-benchmark through the C ABI: times one operator with CUDA
events on the launching stream and prints one JSON line with its achieved
TFLOP/s or GB/s.  Also the small, self-contained workload to put under a
profiler.

  python -m paper_2204_06514_b200.opbench gemm --m 8192 --n 4096 --k 4096 [--a-mn 0 --b-mn 1 --epi 1 --f32-out 0]
  python -m paper_2204_06514_b200.opbench attn_fwd --batch 4 --seq 2048 --heads 32 --hd 128
  python -m paper_2204_06514_b200.opbench attn_bwd --batch 4 --seq 2048 --heads 32 --hd 128
  python -m paper_2204_06514_b200.opbench ln_fwd --rows 8192 --d 4096
  python -m paper_2204_06514_b200.opbench ln_bwd --rows 8192 --d 4096
  python -m paper_2204_06514_b200.opbench adamw --n 201379840
  python -m paper_2204_06514_b200.opbench adamw8 --n 201379840                 # moments in 8 bits
  python -m paper_2204_06514_b200.opbench fp8_gemm --m 8192 --n 16384 --k 4096 [--b-tile 128 --f32-out 0 --acc 0]
  python -m paper_2204_06514_b200.opbench fp8_quantize --rows 8192 --d 4096 [--tile 1 --only straight|transposed]
  python -m paper_2204_06514_b200.opbench embed_fwd --rows 16384 --d 768 --vocab 50304
  python -m paper_2204_06514_b200.opbench embed_bwd --rows 16384 --d 768 --vocab 50304 [--acc 1]
  python -m paper_2204_06514_b200.opbench rotary --rows 16384 --heads 24 --hd 64 [--rot 64 --layout halves|pairs]   # in place in a fused q | k | v
  python -m paper_2204_06514_b200.opbench dropout --rows 16384 --d 768 [--resid 0]
  python -m paper_2204_06514_b200.opbench recurrence_fwd --batch 16 --seq 1024 --d 768 [--gate 0]
  python -m paper_2204_06514_b200.opbench recurrence_bwd --batch 16 --seq 1024 --d 768 [--gate 0]
  python -m paper_2204_06514_b200.opbench expert_sort --rows 16384 --top-k 2 --experts 8 [--capacity 5120 | --align 128]
  python -m paper_2204_06514_b200.opbench expert_dispatch | expert_combine | expert_combine_bwd --rows 16384 --d 768 (as above)
"""
from __future__ import annotations

import argparse
import ctypes as C
import json

import torch

from . import binding as fx
from . import binding_ops as ops
from . import build
from .state import Session, hparams, rotary_frequencies


def P(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("op", choices=["gemm", "attn_fwd", "attn_bwd", "ln_fwd", "ln_bwd", "adamw", "adamw8", "fp8_gemm",
                                   "fp8_quantize", "embed_fwd", "embed_bwd", "rotary", "dropout", "recurrence_fwd", "recurrence_bwd",
                                   "expert_sort", "expert_dispatch", "expert_combine", "expert_combine_bwd"])
    ap.add_argument("--m", type=int, default=8192); ap.add_argument("--n", type=int, default=4096)
    ap.add_argument("--k", type=int, default=4096)
    ap.add_argument("--a-mn", type=int, default=0); ap.add_argument("--b-mn", type=int, default=1)
    ap.add_argument("--epi", type=int, default=0); ap.add_argument("--f32-out", type=int, default=0)
    ap.add_argument("--batch", type=int, default=4); ap.add_argument("--seq", type=int, default=2048)
    ap.add_argument("--heads", type=int, default=32); ap.add_argument("--hd", type=int, default=128)
    ap.add_argument("--rows", type=int, default=8192); ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--b-tile", type=int, default=128, choices=[1, 128]); ap.add_argument("--acc", type=int, default=0)
    ap.add_argument("--tile", type=int, default=1, choices=[1, 128]); ap.add_argument("--only", choices=["straight", "transposed"])
    ap.add_argument("--vocab", type=int, default=50304)
    ap.add_argument("--rot", type=int, default=0); ap.add_argument("--layout", choices=["halves", "pairs"], default="halves")
    ap.add_argument("--resid", type=int, default=1); ap.add_argument("--gate", type=int, default=1)
    ap.add_argument("--top-k", type=int, default=2); ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--capacity", type=int, default=0); ap.add_argument("--align", type=int, default=128)
    ap.add_argument("--iters", type=int, default=20); ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--l2-budget-mb", type=float, default=-1.0, help="GEMM raster: L2 bytes for resident panels (0: fixed order)")
    a = ap.parse_args()
    build.build()
    s = Session(0)
    if a.l2_budget_mb >= 0:
        fx.fax_set_gemm_l2_budget(s.ctx, int(a.l2_budget_mb * 1e6))
    dev, bf = s.device, torch.bfloat16
    g = torch.Generator(device=dev); g.manual_seed(1)
    rn = lambda *shape: torch.randn(shape, generator=g, device=dev).to(bf)
    flops = bytes_ = 0.0
    if a.op == "gemm":
        M, N, K = a.m, a.n, a.k
        A = rn(K, M) if a.a_mn else rn(M, K)
        B = rn(K, N) if a.b_mn else rn(N, K)
        Cc = torch.zeros((M, N), device=dev, dtype=torch.float32 if a.f32_out else bf)
        bias, aux = rn(N), rn(M, N)
        desc = ops.GemmDesc(M, N, K, P(A), M if a.a_mn else K, a.a_mn, P(B), N if a.b_mn else K, a.b_mn, P(Cc), N,
                            a.f32_out, 0, a.epi, P(bias), P(aux), N, P(aux), N, 1.0, 0)
        fn = lambda: ops.fax_op_gemm(s.ctx, 0, desc)
        flops = 2.0 * M * N * K
    elif a.op in ("attn_fwd", "attn_bwd"):
        Bn, T, H, hd = a.batch, a.seq, a.heads, a.hd
        d = H * hd
        qkv, do = rn(Bn * T, 3 * d), rn(Bn * T, d)
        o = torch.empty((Bn * T, d), device=dev, dtype=bf)
        lse = torch.empty((Bn, H, T), device=dev, dtype=torch.float32)
        ops.fax_op_attention_forward(s.ctx, 0, Bn, T, H, hd, P(qkv), P(o), P(lse))
        if a.op == "attn_fwd":
            fn = lambda: ops.fax_op_attention_forward(s.ctx, 0, Bn, T, H, hd, P(qkv), P(o), P(lse))
            flops = 2.0 * Bn * H * T * T * hd
        else:
            nb = ops.fax_op_attention_backward_scratch_bytes(0, Bn, T, H, hd)
            scratch, dqkv = s.arena(nb), torch.empty_like(qkv)
            fn = lambda: ops.fax_op_attention_backward(s.ctx, 0, Bn, T, H, hd, P(qkv), P(o), P(lse), P(do), P(dqkv),
                                                       P(scratch), nb)
            flops = 4.0 * Bn * H * T * T * hd
    elif a.op in ("ln_fwd", "ln_bwd"):
        R, d = a.rows, a.d
        x, da, gam, bet = rn(R, d), rn(R, d), rn(d), rn(d)
        out = torch.empty_like(x)
        mu = torch.empty(R, device=dev, dtype=torch.float32); rstd = torch.empty_like(mu)
        ops.fax_op_layernorm_forward(s.ctx, 0, R, d, P(x), P(gam), P(bet), 1e-5, P(out), P(mu), P(rstd))
        if a.op == "ln_fwd":
            fn = lambda: ops.fax_op_layernorm_forward(s.ctx, 0, R, d, P(x), P(gam), P(bet), 1e-5, P(out), P(mu), P(rstd))
            bytes_ = 2.0 * R * d * 2
        else:
            nb = ops.fax_op_layernorm_backward_scratch_bytes(R, d)
            scratch = s.arena(nb)
            dg = torch.empty(d, device=dev, dtype=torch.float32); db = torch.empty_like(dg)
            fn = lambda: ops.fax_op_layernorm_backward(s.ctx, 0, R, d, P(da), P(x), P(mu), P(rstd), P(gam), P(x),
                                                       P(out), P(dg), P(db), P(scratch), nb)
            bytes_ = 4.0 * R * d * 2
    elif a.op == "fp8_gemm":
        M, N, K = a.m, a.n, a.k
        up, kb = lambda x: -(-x // 16) * 16, -(-K // 128)
        q8 = lambda r: torch.randn((r, up(K)), generator=g, device=dev).to(torch.float8_e4m3fn)
        A, B = q8(M), q8(N)
        sa = torch.ones((kb, M), device=dev)
        sb = torch.ones((kb, N if a.b_tile == 1 else -(-N // 128)), device=dev)
        Cc = torch.zeros((M, N), device=dev, dtype=torch.float32 if a.f32_out or a.acc else bf)
        desc = ops.Fp8GemmDesc(M, N, K, P(A), up(K), 0, P(sa), sa.shape[1], P(B), up(K), 0, P(sb), sb.shape[1], a.b_tile, P(Cc), N,
                               int(Cc.dtype == torch.float32), a.acc, None)
        fn = lambda: ops.fax_op_fp8_gemm(s.ctx, desc)
        flops = 2.0 * M * N * K
    elif a.op == "fp8_quantize":
        R, d = a.rows, a.d
        up = lambda x: -(-x // 16) * 16
        x = rn(R, d)
        q, sq = torch.empty((R, up(d)), dtype=torch.uint8, device=dev), torch.empty((-(-d // 128), -(-R // a.tile)), device=dev)
        qt, st_ = torch.empty((d, up(R)), dtype=torch.uint8, device=dev), torch.empty((-(-R // 128), -(-d // a.tile)), device=dev)
        if a.only == "straight":
            qt = None
        if a.only == "transposed":
            q = None
        desc = ops.Fp8QuantizeDesc(R, d, P(x), d, 0, a.tile, P(q), up(d), P(sq), sq.shape[1], P(qt), up(R), P(st_), st_.shape[1])
        fn = lambda: ops.fax_op_fp8_quantize(s.ctx, 0, desc)
        bytes_ = float(R) * d * (2 + (q is not None) + (qt is not None))
    elif a.op in ("embed_fwd", "embed_bwd"):
        n, d, V = a.rows, a.d, a.vocab
        ids = torch.exp(torch.rand(n, generator=g, device=dev) * float(torch.tensor(V + 1.0).log())).int().clamp_(1, V) - 1     # Zipf
        x = rn(n, d)
        if a.op == "embed_fwd":
            table = rn(V, d)
            fn = lambda: ops.fax_op_embedding_forward(s.ctx, 0, n, V, d, P(ids), P(table), d ** 0.5, P(x))
            bytes_ = 2.0 * d * (n + int(ids.unique().numel())) + 4.0 * n
        else:
            table = torch.zeros((V, d), device=dev)
            nb = ops.fax_op_embedding_backward_scratch_bytes(n, V, d)
            scratch = s.arena(nb)
            fn = lambda: ops.fax_op_embedding_backward(s.ctx, 0, n, V, d, P(ids), P(x), d ** 0.5, a.acc, P(table), P(scratch), nb)
            bytes_ = 2.0 * n * d + 4.0 * n + 4.0 * d * (2 * int(ids.unique().numel()) if a.acc else V)
    elif a.op == "rotary":
        R, H, hd = a.rows, a.heads, a.hd
        rot = a.rot or hd
        qkv = rn(R, (H + H // 2) * hd)
        table = rotary_frequencies(dev, rot)
        desc = ops.RotaryDesc(R, H, hd, rot, int(a.layout == "pairs"), P(qkv), qkv.shape[1], P(qkv), qkv.shape[1], None, 0, a.seq, P(table), 1.0, 0)
        fn = lambda: ops.fax_op_rotary(s.ctx, 0, desc)
        bytes_ = 4.0 * R * H * rot
    elif a.op == "dropout":
        R, d = a.rows, a.d
        x, r, y = rn(R, d), rn(R, d), rn(R, d)
        desc = ops.DropoutDesc(R, d, P(x), d, P(r) if a.resid else None, d, P(y), d, 0.1, 1, 0, None)
        fn = lambda: ops.fax_op_dropout(s.ctx, 0, desc)
        bytes_ = (4.0 + 2 * (a.resid != 0)) * R * d
    elif a.op in ("recurrence_fwd", "recurrence_bwd"):
        B_, T, d = a.batch, a.seq, a.d
        R, k = B_ * T, 2 + (a.gate != 0)
        proj, dproj, y, dy = rn(R, k * d), rn(R, k * d), rn(R, d), rn(R, d)
        h0 = torch.zeros((B_, d), device=dev)
        states = torch.empty(ops.fax_op_recurrence_states_floats(R, B_, d), device=dev)
        col = lambda t, i: C.c_void_p(t.data_ptr() + 2 * i * d) if i < k else None
        shape = (R, d, B_, T, None, ops.FAX_RECURRENCE_COMPLEMENT, col(proj, 0), k * d, col(proj, 1), k * d, col(proj, 2), k * d, P(h0))
        fwd = ops.RecurrenceDesc(*shape, P(y), d, None, P(states))
        bwd = ops.RecurrenceBackwardDesc(*shape, P(states), P(dy), d, None, col(dproj, 0), k * d, col(dproj, 1), k * d, col(dproj, 2), k * d, None)
        ops.fax_op_recurrence_forward(s.ctx, 0, fwd)
        if a.op == "recurrence_fwd":
            fn = lambda: ops.fax_op_recurrence_forward(s.ctx, 0, fwd)
            bytes_ = 2.0 * (k + 1) * R * d + R * d / 4
        else:
            fn = lambda: ops.fax_op_recurrence_backward(s.ctx, 0, bwd)
            bytes_ = 2.0 * (2 * k + 1) * R * d + R * d / 4
    elif a.op.startswith("expert"):
        R, d, K, E = a.rows, a.d, a.top_k, a.experts
        slots = ops.fax_op_expert_slots(R, K, E, a.capacity, a.align)
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)
        ids = torch.rand((R, E), generator=g, device=dev).topk(K, dim=1).indices.int()
        slot_of, source, offsets, counts = i32(R, K), i32(slots), i32(E + 1), i32(E)
        plan = ops.ExpertSortDesc(R, K, E, a.capacity, a.align, slots, P(ids), P(slot_of), P(source), P(offsets), P(counts))
        ops.fax_op_expert_sort(s.ctx, plan)
        x, z, y = rn(R, d), rn(slots, d), rn(R, d)
        w, dw = torch.rand((R, K), generator=g, device=dev), torch.empty((R, K), device=dev)
        where = (R, K, d, slots, P(slot_of))
        if a.op == "expert_sort":
            fn = lambda: ops.fax_op_expert_sort(s.ctx, plan)
            bytes_ = 4.0 * (2 * R * K + slots + 2 * E)
        elif a.op == "expert_dispatch":
            desc = ops.ExpertDispatchDesc(*where, P(source), P(x), d, P(z), d)
            fn = lambda: ops.fax_op_expert_dispatch(s.ctx, 0, desc)
            bytes_ = 2.0 * d * (R + slots)
        elif a.op == "expert_combine":
            desc = ops.ExpertCombineDesc(*where, P(w), P(z), d, P(x), d, P(y), d)
            fn = lambda: ops.fax_op_expert_combine(s.ctx, 0, desc)
            bytes_ = 2.0 * d * (R * K + 2 * R)
        else:
            desc = ops.ExpertCombineBackwardDesc(*where, P(source), P(w), P(z), d, P(x), d, P(z), d, P(dw))
            fn = lambda: ops.fax_op_expert_combine_backward(s.ctx, 0, desc)
            bytes_ = 2.0 * d * (R * K + slots + R)
    elif a.op == "adamw8":
        n = a.n if a.n > 4096 else 201379840
        w = torch.randn(n, generator=g, device=dev); gr = torch.randn(n, generator=g, device=dev)
        m = torch.zeros(n, dtype=torch.uint8, device=dev); v = torch.zeros_like(m)
        ms = torch.zeros(-(-n // 128), device=dev); vs = torch.zeros_like(ms)
        wc = torch.empty(n, device=dev, dtype=bf)
        t8 = (fx.Adamw8Tensor * 1)(fx.Adamw8Tensor(P(w), P(m), P(v), P(ms), P(vs), P(gr), P(wc), n, 0.1, 1))
        hp = hparams(1e-3, 0.9, 0.95, 1e-8, 1)
        fn = lambda: fx.fax_adamw8_step(s.ctx, t8, hp)
        bytes_ = 18.0 * n + 16.0 * (n / 128)
    else:
        n = a.n if a.n > 4096 else 201379840
        w = torch.randn(n, generator=g, device=dev); m = torch.zeros_like(w); v = torch.zeros_like(w)
        gr = torch.randn(n, generator=g, device=dev); wc = torch.empty(n, device=dev, dtype=bf)
        t = [fx.AdamwTensor(P(w), P(m), P(v), P(gr), P(wc), n, 0.1)]
        hp = hparams(1e-3, 0.9, 0.95, 1e-8, 1)
        fn = lambda: fx.fax_adamw_step(s.ctx, t, hp)
        bytes_ = 30.0 * n
    for _ in range(a.warmup):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record(s.stream)
    for _ in range(a.iters):
        fn()
    e1.record(s.stream)
    torch.cuda.synchronize()
    ms = e0.elapsed_time(e1) / a.iters
    st, detail = fx.fax_check_device_status(s.ctx)
    out = {"op": a.op, "ms": ms, "status": st, "detail": detail}
    if flops:
        out.update(tflops=flops / ms / 1e9, flops=flops)
    else:
        out.update(gbs=bytes_ / ms / 1e6, bytes=bytes_)
    print(json.dumps(out))
    s.close()


if __name__ == "__main__":
    main()
