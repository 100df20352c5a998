"""Ragged attention batches, or ragged batches of experts, through the C ABI: one grouped launch against the alternatives.

    python run_ragged.py [--seqs 64] [--heads 12] [--iters 20] [--draws 4] [--align 8]
    python run_ragged.py --experts 64 [--tokens 4096] [--top-k 8] [--cols 2048] [--inner 1408] [--draws 2]

A batch holds --seqs sequences whose lengths are drawn like the attention configuration's (the
paper's motivation, Sec. 1 / Fig. 1(b): sequence lengths in a batch differ widely and padding them to
the longest wastes most of the work).  For QK^T (K = 64, fp32 scores) and PV (N = 64) the batch is run
  grouped : ONE launch over per-sequence groups (ft_plan_create_grouped), every sequence at its own length
  padded  : one plain batched launch with every sequence padded to the longest of the batch
            (the planner's plan for that shape; useful flops are those of the true lengths)
  looped  : one plain launch per sequence, back to back on one stream
Operands are random bit patterns made on the device (timing only; tests/ checks grouped launches against
the oracle).  Buffers rotate over a ring so that launches do not find them in the caches.  Prints one
line per draw and operator and a JSON summary line.

With --experts the ragged batch is the tokens that a router sends to each of them, and the work a layer of gated experts in
8-bit integers: sort, quantise, product with its gate, quantise, product, combine (bf16 in and out).  It is run
  grouped : the rows of all experts in ONE launch of each product; their numbers stay on the device
  padded  : one product over every expert's rows, padded to the most that any expert has
  looped  : the numbers are known to the host, and every expert that has rows gets a launch of its own
The two products alone are compared; the whole layer's time stands beside them.
"""
import argparse
import json
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--seqs", type=int, default=64)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--iters", type=int, default=20)
    ap.add_argument("--draws", type=int, default=4)
    ap.add_argument("--ring-mb", type=float, default=600.0)
    ap.add_argument("--align", type=int, default=1, help="round every length up to a multiple of this (8: the "
                    "grouped launch then runs the LDS-DMA bodies)")
    ap.add_argument("--b-nk", action="store_true", help="Q K^T with the K matrices stored [L, 64] (FT_B_NK): the LDS-DMA "
                    "bodies at every length")
    ap.add_argument("--experts", type=int, default=0, help="a layer of so many gated experts in 8-bit integers instead of attention")
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--top-k", type=int, default=8)
    ap.add_argument("--cols", type=int, default=2048)
    ap.add_argument("--inner", type=int, default=1408)
    a = ap.parse_args()
    if a.experts:
        rows = measure_experts(a.experts, a.tokens, a.top_k, a.cols, a.inner, a.iters, a.draws, verbose=True)
        print(json.dumps({"workload": "%d tokens to %d of %d gated experts, %d x %d, int8 products, bf16 in and out" % (a.tokens, a.top_k, a.experts, a.cols, a.inner), "rows": rows}))
        return
    rows = measure(a.seqs, a.heads, a.iters, a.draws, a.align, a.ring_mb, verbose=True, b_nk=a.b_nk)
    gm = lambda xs: math.exp(sum(math.log(x) for x in xs) / len(xs))
    print(json.dumps({"workload": "ragged attention batches, %d sequences x %d heads, lengths rounded up to multiples of %d, fp16 in, fp32 out" % (a.seqs, a.heads, a.align),
                      "speedup_vs_padded_geomean": round(gm([r["us_padded"] / r["us_grouped"] for r in rows]), 3),
                      "speedup_vs_looped_geomean": round(gm([r["us_looped"] / r["us_grouped"] for r in rows]), 3),
                      "rows": rows}))


def measure(seqs=64, heads=12, iters=20, draws=4, align=1, ring_mb=600.0, verbose=False, b_nk=False):
    """The measurement itself; returns one row per draw and operator."""
    import argparse as _ap
    a = _ap.Namespace(seqs=seqs, heads=heads, iters=iters, draws=draws, align=align, ring_mb=ring_mb)

    import torch
    import paper_2407_21418_amd as ft
    import synth_inputs as si

    assert torch.cuda.is_available(), "run_ragged needs a GPU"
    stream = torch.cuda.current_stream().cuda_stream
    hw = ft.ft_hw_query(0)
    H = a.heads
    ops = {
        "qk": ft.ft_op_register(ft.ft_op_desc(kind=ft.FT_OP_BMM, dtype=ft.FT_F16, k=64, m_lo=0, m_hi=512, n_lo=0, n_hi=512,
                                              batch_hi=a.seqs * H, b_layout=ft.FT_B_NK if b_nk else ft.FT_B_KN)),
        "pv": ft.ft_op_register(ft.ft_op_desc(kind=ft.FT_OP_BMM, dtype=ft.FT_F16, n=64, m_lo=0, m_hi=512, k_lo=0, k_hi=512,
                                              batch_hi=a.seqs * H)),
    }
    sets = {k: ft.ft_ukernels_derive(op, hw, None) for k, op in ops.items()}

    def dims(which, L):
        return (L, L, 64) if which == "qk" else (L, 64, L)

    def rand16(n):
        return si.device_normal_bits((max(n, 8),), si.F16)

    def timed(plan, na, nb, nc):
        nsets = max(2, min(16, int(math.ceil(a.ring_mb * 1e6 / (2 * (na + nb) + 4 * nc)))))
        A = [rand16(na) for _ in range(nsets)]
        B = [rand16(nb) for _ in range(nsets)]
        Cs = [torch.empty(max(nc, 8), dtype=torch.float32, device="cuda") for _ in range(nsets)]
        pa, pb, pc = [t.data_ptr() for t in A], [t.data_ptr() for t in B], [t.data_ptr() for t in Cs]
        ft.ft_launch_timed(plan, pa, pb, pc, stream, 2)
        return ft.ft_launch_timed(plan, pa, pb, pc, stream, a.iters) * 1e3

    rows = []
    for draw in range(a.draws):
        lengths = [min(512, -(-L // a.align) * a.align) for L in si.ragged_lengths(draw, a.seqs)]
        Lmax = max(lengths)
        for which in ("qk", "pv"):
            op, uks = ops[which], sets[which]
            shape = (lambda L, b: ft.ft_shape(batch=b, m=L, n=L) if which == "qk" else ft.ft_shape(batch=b, m=L, k=L))
            flops = sum(2.0 * H * m * n * k for m, n, k in (dims(which, L) for L in lengths))
            grouped = ft.ft_plan_create_grouped(op, uks, [shape(L, H) for L in lengths])
            na, nb, nc = ft.ft_plan_group_layout(grouped, len(lengths))
            us_grouped = timed(grouped, na, nb, nc)
            m, n, k = dims(which, Lmax)
            padded = ft.ft_plan_create(op, uks, shape(Lmax, a.seqs * H))
            us_padded = timed(padded, a.seqs * H * m * k, a.seqs * H * k * n, a.seqs * H * m * n)
            # one launch per sequence on slices of one packed set (no ring: the operands of 64 launches
            # already exceed the L2s), timed as a whole with events
            plans = [ft.ft_plan_create(op, uks, shape(L, H)) for L in lengths]
            A, B, Cb = rand16(na), rand16(nb), torch.empty(max(nc, 8), dtype=torch.float32, device="cuda")
            offs = [ft.ft_plan_group_layout(grouped, i) for i in range(len(lengths))]

            def loop_once():
                for p, (oa, ob, oc) in zip(plans, offs):
                    ft.ft_launch(p, A.data_ptr() + 2 * oa, B.data_ptr() + 2 * ob, Cb.data_ptr() + 4 * oc, stream)
            loop_once()
            torch.cuda.synchronize()
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            for _ in range(a.iters):
                loop_once()
            e1.record()
            e1.synchronize()
            us_looped = e0.elapsed_time(e1) * 1e3 / a.iters
            st = ft.ft_plan_stats_get(grouped)
            rows.append(dict(draw=draw, op=which, max_len=Lmax, mean_len=round(sum(lengths) / len(lengths), 1),
                             us_grouped=round(us_grouped, 1), us_padded=round(us_padded, 1), us_looped=round(us_looped, 1),
                             tflops_grouped=round(flops / us_grouped / 1e6, 1), tiles=int(st.n_tiles),
                             padded_work_ratio=round(a.seqs * Lmax * Lmax / max(1, sum(L * L for L in lengths)), 2)))
            r = rows[-1]
            if verbose:
                print("draw %d %s: %d seqs x %d heads, L mean %.0f max %d | grouped %7.1f us (%5.1f TFLOP/s useful, %d tiles) | "
                      "padded to max %7.1f us (x%.2f, %.2fx the work) | one launch per sequence %7.1f us (x%.2f)"
                      % (draw, which, a.seqs, H, r["mean_len"], Lmax, us_grouped, r["tflops_grouped"], r["tiles"], us_padded,
                         us_padded / us_grouped, r["padded_work_ratio"], us_looped, us_looped / us_grouped), flush=True)
    return rows


def measure_experts(experts=64, tokens=4096, top_k=8, cols=2048, inner=1408, iters=20, draws=2, verbose=False):
    """A layer of gated experts; returns one row per draw of the router."""
    import torch
    import paper_2407_21418_amd as ft

    assert torch.cuda.is_available(), "run_ragged needs a GPU"
    s = torch.cuda.current_stream().cuda_stream
    pitch = lambda k: (k + 15) // 16 * 16
    entries = tokens * top_k
    i8 = lambda rows, k: torch.randint(-127, 128, (rows, pitch(k)), device="cuda", dtype=torch.int8)
    up, down = i8(experts * 2 * inner, cols), i8(experts * cols, inner)
    up_scale, down_scale = torch.rand(experts * 2 * inner, device="cuda") * 1e-3, torch.rand(experts * cols, device="cuda") * 1e-3
    x = torch.randn(tokens, cols, device="cuda").to(torch.bfloat16)
    weights = torch.softmax(torch.randn(tokens, top_k, device="cuda"), 1)
    int32 = lambda n: torch.empty(n, device="cuda", dtype=torch.int32)
    offsets, row_token, row_of = int32(experts + 1), int32(entries), int32(entries)
    xq, xs = i8(tokens, cols), torch.empty(tokens, device="cuda")
    d_sort = ft.ft_expert_desc(experts=experts, top_k=top_k, cols=cols, dtype=ft.FT_BF16)
    need = ft.ft_expert_workspace(d_sort, tokens)
    work = torch.empty(max(need, 1), device="cuda", dtype=torch.uint8)
    d_x, d_h = ft.ft_quant_desc(cols=cols, dtype=ft.FT_BF16), ft.ft_quant_desc(cols=inner, dtype=ft.FT_F32)
    one_up = dict(n=2 * inner, k=cols, dtype=ft.FT_BF16, out_dtype=ft.FT_OUT_F32, epilogue=ft.FT_EPI_SILU_MUL)
    one_down = dict(n=cols, k=inner, dtype=ft.FT_BF16, out_dtype=ft.FT_OUT_SAME)
    d_up, d_down = ft.ft_i8_desc(experts=experts, **one_up), ft.ft_i8_desc(experts=experts, **one_down)
    d_up1, d_down1 = ft.ft_i8_desc(**one_up), ft.ft_i8_desc(**one_down)
    out = torch.empty(tokens, cols, device="cuda", dtype=torch.bfloat16)

    def timed(f):
        f()
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(iters):
            f()
        e1.record()
        e1.synchronize()
        return e0.elapsed_time(e1) * 1e3 / iters

    rows = []
    for draw in range(draws):
        g = torch.Generator(device="cuda").manual_seed(draw)
        liked = 0.5 * torch.randn(experts, device="cuda", generator=g)
        ids = torch.topk(torch.randn(tokens, experts, device="cuda", generator=g) + liked, top_k, 1)[1].int().contiguous()
        counts = torch.bincount(ids.flatten(), minlength=experts).cpu().tolist()
        most = max(counts)
        h, y = torch.empty(entries, inner, device="cuda"), torch.empty(entries, cols, device="cuda", dtype=torch.bfloat16)
        hq, hs = i8(entries, inner), torch.empty(entries, device="cuda")

        def sort():
            ft.ft_expert_sort(d_sort, tokens, ids.data_ptr(), offsets.data_ptr(), row_token.data_ptr(), row_of.data_ptr(), work.data_ptr(), need, s)

        def products(quantize_between):
            ft.ft_i8_matmul_experts(d_up, entries, offsets.data_ptr(), xq.data_ptr(), xs.data_ptr(), row_token.data_ptr(), tokens, up.data_ptr(), up_scale.data_ptr(), 0, h.data_ptr(), s)
            if quantize_between:
                ft.ft_i8_quantize(d_h, entries, h.data_ptr(), hq.data_ptr(), hs.data_ptr(), s)
            ft.ft_i8_matmul_experts(d_down, entries, offsets.data_ptr(), hq.data_ptr(), hs.data_ptr(), 0, entries, down.data_ptr(), down_scale.data_ptr(), 0, y.data_ptr(), s)

        def layer():
            sort()
            ft.ft_i8_quantize(d_x, tokens, x.data_ptr(), xq.data_ptr(), xs.data_ptr(), s)
            products(True)
            ft.ft_expert_combine(d_sort, tokens, y.data_ptr(), row_of.data_ptr(), weights.data_ptr(), out.data_ptr(), s)
        us_layer = timed(layer)
        us_grouped = timed(lambda: products(False))

        # the same rows, gathered: a launch for each expert
        gathered, gathered_s = xq[row_token.long()].contiguous(), xs[row_token.long()].contiguous()

        def expert(e, at, count):
            ft.ft_i8_matmul(d_up1, count, gathered.data_ptr() + at * pitch(cols), gathered_s.data_ptr() + 4 * at, up.data_ptr() + e * 2 * inner * pitch(cols), up_scale.data_ptr() + 8 * e * inner,
                            0, h.data_ptr() + 4 * at * inner, s)
            ft.ft_i8_matmul(d_down1, count, hq.data_ptr() + at * pitch(inner), hs.data_ptr() + 4 * at, down.data_ptr() + e * cols * pitch(inner), down_scale.data_ptr() + 4 * e * cols, 0,
                            y.data_ptr() + 2 * at * cols, s)

        def looped():
            at = 0
            for e, count in enumerate(counts):
                if count:
                    expert(e, at, count)
                at += count
        us_looped = timed(looped)

        # every expert's rows padded to the most
        all_rows = experts * most
        pad_x, pad_xs, pad_off = i8(all_rows, cols), torch.rand(all_rows, device="cuda"), torch.arange(0, all_rows + 1, most, device="cuda", dtype=torch.int32)
        pad_hq, pad_hs = i8(all_rows, inner), torch.rand(all_rows, device="cuda")
        pad_h, pad_y = torch.empty(all_rows, inner, device="cuda"), torch.empty(all_rows, cols, device="cuda", dtype=torch.bfloat16)

        def padded():
            ft.ft_i8_matmul_experts(d_up, all_rows, pad_off.data_ptr(), pad_x.data_ptr(), pad_xs.data_ptr(), 0, all_rows, up.data_ptr(), up_scale.data_ptr(), 0, pad_h.data_ptr(), s)
            ft.ft_i8_matmul_experts(d_down, all_rows, pad_off.data_ptr(), pad_hq.data_ptr(), pad_hs.data_ptr(), 0, all_rows, down.data_ptr(), down_scale.data_ptr(), 0, pad_y.data_ptr(), s)
        us_padded = timed(padded)
        flops = 2.0 * entries * 3 * cols * inner
        rows.append(dict(draw=draw, most_rows=most, mean_rows=round(entries / experts, 1), us_layer=round(us_layer, 1), us_grouped=round(us_grouped, 1), us_padded=round(us_padded, 1),
                         us_looped=round(us_looped, 1), tops_grouped=round(flops / us_grouped / 1e6, 1), padded_work_ratio=round(all_rows / entries, 2)))
        if verbose:
            print("draw %d: %d entries, rows of an expert mean %.0f most %d | products grouped %7.1f us (%5.1f TOP/s) | padded %7.1f us (x%.2f, %.2fx the work) | a launch for each expert %7.1f us "
                  "(x%.2f) | the layer %7.1f us" % (draw, entries, entries / experts, most, us_grouped, rows[-1]["tops_grouped"], us_padded, us_padded / us_grouped, all_rows / entries,
                                                    us_looped, us_looped / us_grouped, us_layer), flush=True)
    return rows


if __name__ == "__main__":
    main()
