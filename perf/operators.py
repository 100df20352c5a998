"""Products in 8-bit integers and tokens sorted by expert: what is timed, and the operators' plain forms.

Kinds of cases
  linear   a linear layer in 8 bits: the rows of x are quantised, each with a scale of its own (after silu(gate) * up where the
           layer follows a gated activation), and multiplied with a weight that has a scale for each channel
  permute  the tokens of a batch sorted by expert, carried there and back with the router's weights; `grad`: and the gradients
  experts  the feed-forward layer of a mixture of experts in 8 bits: sort, quantise, grouped product up, gated activation and
           quantisation, grouped product down, back to the tokens

`own` false: the plain forms, elementary torch operations.  `own` true: the calls of the framework.
"""
import math

import torch

own = False

MOST_LINEAR = 8192 * 11008 * 4096
MOST_EXPERTS = 8192 * 8 * 2048 * 1408
MOST_PERMUTE = 8192 * 8 * 4096


def listed():
    return [
        # one token of one request through a square projection: the smallest call, latency and one read of the weight
        dict(name="linear 1x4096x4096", kind="linear", m=1, n=4096, k=4096, dtype="bf16", out="same", bias=False, gated=False),
        # a short sentence through a layer of an encoder, with bias and full-width results
        dict(name="linear 77x768x768", kind="linear", m=77, n=768, k=768, dtype="f16", out="f32", bias=True, gated=False),
        # a decode step of many requests with a short prompt; no extent is a multiple of anything
        dict(name="linear 403x1003x1001", kind="linear", m=403, n=1003, k=1001, dtype="bf16", out="same", bias=True, gated=False),
        # the down projection of a gated feed-forward layer over a prompt
        dict(name="linear gated 2048x4096x11008", kind="linear", m=2048, n=4096, k=11008, dtype="bf16", out="same", bias=False, gated=True),
        # prefill of a long prompt up the feed-forward layer: the largest product
        dict(name="linear 8192x11008x4096", kind="linear", m=8192, n=11008, k=4096, dtype="bf16", out="same", bias=False, gated=False),
        # a decode step of five requests
        dict(name="permute 5 top 2", kind="permute", tokens=5, top_k=2, experts=8, cols=1024, dtype="f16", padded=0, grad=False),
        # a training step over a padded batch whose rows end inside every vector width
        dict(name="permute 1234 top 6 grad", kind="permute", tokens=1234, top_k=6, experts=60, cols=1001, dtype="f16", padded=100, grad=True),
        # a training step of a long batch over many experts
        dict(name="permute 8192 top 8 grad", kind="permute", tokens=8192, top_k=8, experts=128, cols=4096, dtype="bf16", padded=0, grad=True),
        # a decode step of four requests: a few experts' weights read once
        dict(name="experts 4 top 2", kind="experts", tokens=4, top_k=2, experts=8, cols=1024, ffn=1408, dtype="f16", padded=0),
        # a decode step of a full batch: every expert's weight read once, for a few rows each
        dict(name="experts 64 top 4", kind="experts", tokens=64, top_k=4, experts=64, cols=2048, ffn=1408, dtype="bf16", padded=0),
        # a padded batch of short prompts through layers of odd extents
        dict(name="experts 1000 top 2 odd", kind="experts", tokens=1000, top_k=2, experts=16, cols=1000, ffn=715, dtype="f16", padded=37),
        # prefill of long prompts
        dict(name="experts 8192 top 8", kind="experts", tokens=8192, top_k=8, experts=64, cols=2048, ffn=1408, dtype="bf16", padded=0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _extent(rng, lo, hi):
    """A layer's extent: whole multiples of 64 mostly, anything else too."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.3 else max(64, n // 64 * 64)


def draw(rng):
    kind = rng.choice(("linear", "permute", "experts"))
    dtype = rng.choice(("f16", "bf16"))
    if kind == "linear":
        gated = rng.random() < 0.3
        n, k = _extent(rng, 64, 11008), _extent(rng, 64, 11008)
        m = _log_int(rng, 1, max(1, min(8192, MOST_LINEAR // (n * k * (2 if gated else 1)))))
        return dict(kind=kind, m=m, n=n, k=k, dtype=dtype, out="same" if gated else rng.choice(("same", "f32")), bias=rng.random() < 0.5, gated=gated)
    top_k = rng.randint(1, 8)
    experts = _log_int(rng, max(4, top_k), 128)
    if kind == "permute":
        cols = _extent(rng, 64, 4096)
        tokens = _log_int(rng, 1, min(16384, MOST_PERMUTE // (top_k * cols)))
        grad = rng.random() < 0.6
        return dict(kind=kind, tokens=tokens, top_k=top_k, experts=experts, cols=cols, dtype=rng.choice(("f16", "bf16", "f32")),
                    padded=rng.randint(0, tokens // 4), grad=grad)
    cols, ffn = _extent(rng, 64, 4096), _extent(rng, 64, 4096)
    experts = max(top_k, min(experts, 64 * 2048 * 1408 // (cols * ffn)))
    tokens = _log_int(rng, 1, max(1, min(8192, MOST_EXPERTS // (4 * top_k * cols * ffn))))
    return dict(kind=kind, tokens=tokens, top_k=top_k, experts=experts, cols=cols, ffn=ffn, dtype=dtype, padded=rng.randint(0, tokens // 4))


# ---- what a program has in hand ------------------------------------------------------------------

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _pitch(k):
    """Rows of 8-bit operands lie on 16-byte blocks."""
    return (k + 15) // 16 * 16


def _activations(gen, rows, cols, dtype):
    """Normal values with a few channels that are several times larger, as activations have them."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    loud = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return torch.where(loud, 6 * x, x).to(TYPES[dtype])


def _weight(gen, rows, k):
    """A quantised weight, each row [k] with its own scale; what lies between a row's end and its pitch is anything."""
    q = torch.empty(rows, _pitch(k), dtype=torch.int8, device="cuda")
    for at in range(0, rows, 32768):
        part = torch.randn(min(32768, rows - at), _pitch(k), generator=gen, device="cuda")
        q[at:at + part.shape[0]] = part.mul_(36.0).round_().clamp_(-127, 127).to(torch.int8)
    return q, torch.rand(rows, generator=gen, device="cuda").add_(0.5).mul_(1 / (36.0 * math.sqrt(k)))


def _router(gen, case):
    """Expert ids [tokens, top_k], distinct for a token, some experts liked more than others; padding tokens have none (-1)."""
    tokens, top_k, experts = case["tokens"], case["top_k"], case["experts"]
    liked = torch.randn(experts, generator=gen, device="cuda").mul_(0.5)
    logits = torch.randn(tokens, experts, generator=gen, device="cuda") + liked
    values, ids = torch.topk(logits, top_k, dim=1)
    weights = torch.softmax(values, dim=1).contiguous()
    ids = ids.to(torch.int32).contiguous()
    if case["padded"]:
        ids[tokens - case["padded"]:] = -1
    return ids, weights


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["x"] = _activations(gen, m, 2 * k if case["gated"] else k, case["dtype"])
        s["w"], s["sw"] = _weight(gen, n, k)
        s["b"] = torch.randn(n, generator=gen, device="cuda") if case["bias"] else None
        s["q"] = torch.zeros(m, _pitch(k), dtype=torch.int8, device="cuda")
        s["sx"] = torch.zeros(m, device="cuda")
        s["y"] = torch.zeros(m, n, dtype=torch.float32 if case["out"] == "f32" else TYPES[case["dtype"]], device="cuda")
        if own:
            import paper_2407_21418_amd as ft
            dtype = ft.FT_F16 if case["dtype"] == "f16" else ft.FT_BF16
            s["quantize"] = ft.ft_quant_desc(cols=k, dtype=dtype, act=ft.FT_ACT_SILU_MUL if case["gated"] else ft.FT_ACT_NONE)
            s["product"] = ft.ft_i8_desc(n=n, k=k, dtype=dtype, out_dtype=ft.FT_OUT_F32 if case["out"] == "f32" else ft.FT_OUT_SAME,
                                         epilogue=ft.FT_EPI_BIAS if case["bias"] else ft.FT_EPI_NONE)
        return s
    tokens, top_k, experts, cols = case["tokens"], case["top_k"], case["experts"], case["cols"]
    rows = tokens * top_k
    s["ids"], s["weights"] = _router(gen, case)
    s["offsets"] = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    s["row_token"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    s["row_of"] = torch.zeros(tokens, top_k, dtype=torch.int32, device="cuda")
    s["x"] = _activations(gen, tokens, cols, case["dtype"])
    s["out"] = torch.zeros_like(s["x"])
    if kind == "permute":
        s["xs"] = torch.zeros(rows, cols, dtype=s["x"].dtype, device="cuda")
        s["ys"] = _activations(gen, rows, cols, case["dtype"])
        if case["grad"]:
            s["dout"], s["dxs"] = _activations(gen, tokens, cols, case["dtype"]), _activations(gen, rows, cols, case["dtype"])
            s["dys"], s["dweights"], s["dx"] = torch.zeros_like(s["xs"]), torch.zeros_like(s["weights"]), torch.zeros_like(s["x"])
    else:
        ffn = case["ffn"]
        s["w1"], s["sw1"] = _weight(gen, experts * 2 * ffn, cols)
        s["w2"], s["sw2"] = _weight(gen, experts * cols, ffn)
        s["q"], s["sx"] = torch.zeros(tokens, _pitch(cols), dtype=torch.int8, device="cuda"), torch.zeros(tokens, device="cuda")
        s["h"] = torch.zeros(rows, 2 * ffn, dtype=s["x"].dtype, device="cuda")
        s["qh"], s["sh"] = torch.zeros(rows, _pitch(ffn), dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
        s["ys"] = torch.zeros(rows, cols, dtype=s["x"].dtype, device="cuda")
    if own:
        import paper_2407_21418_amd as ft
        dtype = {"f16": ft.FT_F16, "bf16": ft.FT_BF16, "f32": ft.FT_F32}[case["dtype"]]
        s["route"] = ft.ft_expert_desc(experts=experts, top_k=top_k, cols=cols, dtype=dtype)
        s["workspace"] = torch.empty(max(16, ft.ft_expert_workspace(s["route"], tokens)), dtype=torch.uint8, device="cuda")
        if kind == "experts":
            s["quantize_x"] = ft.ft_quant_desc(cols=cols, dtype=dtype)
            # (the product's own activation, in 32 bits until it is quantised: gates and values that were rounded to 16 bits before leave an integer in a
            # hundred on another side, 0.010 of the result in bf16 where this way leaves 0.0023)
            s["h"] = torch.zeros(rows, ffn, device="cuda")
            s["up"] = ft.ft_i8_desc(n=2 * ffn, k=cols, dtype=dtype, out_dtype=ft.FT_OUT_F32, epilogue=ft.FT_EPI_SILU_MUL, experts=experts)
            s["quantize_h"] = ft.ft_quant_desc(cols=ffn, dtype=ft.FT_F32)
            s["down"] = ft.ft_i8_desc(n=cols, k=ffn, dtype=dtype, out_dtype=ft.FT_OUT_SAME, experts=experts)
    return s


# ---- the framework's calls -----------------------------------------------------------------------


def _own_linear(s, ft, stream):
    x, q, sx, y, b = s["x"], s["q"], s["sx"], s["y"], s["b"]
    ft.ft_i8_quantize(s["quantize"], s["m"], x.data_ptr(), q.data_ptr(), sx.data_ptr(), stream)
    ft.ft_i8_matmul(s["product"], s["m"], q.data_ptr(), sx.data_ptr(), s["w"].data_ptr(), s["sw"].data_ptr(), b.data_ptr() if b is not None else 0, y.data_ptr(), stream)
    return {"y": y, "scale": sx}


def _own_sort(s, ft, stream):
    ft.ft_expert_sort(s["route"], s["tokens"], s["ids"].data_ptr(), s["offsets"].data_ptr(), s["row_token"].data_ptr(), s["row_of"].data_ptr(),
                      s["workspace"].data_ptr(), s["workspace"].numel(), stream)


def _own_permute(s, ft, stream):
    route, tokens, row_of, w = s["route"], s["tokens"], s["row_of"].data_ptr(), s["weights"].data_ptr()
    _own_sort(s, ft, stream)
    ft.ft_expert_gather(route, tokens, s["x"].data_ptr(), row_of, s["xs"].data_ptr(), stream)
    ft.ft_expert_combine(route, tokens, s["ys"].data_ptr(), row_of, w, s["out"].data_ptr(), stream)
    got = {"offsets": s["offsets"], "row_token": s["row_token"], "row_of": s["row_of"], "xs": s["xs"], "out": s["out"]}
    if s["grad"]:
        ft.ft_expert_combine_grad(route, tokens, s["dout"].data_ptr(), s["ys"].data_ptr(), row_of, w, s["dys"].data_ptr(), s["dweights"].data_ptr(), stream)
        ft.ft_expert_combine(route, tokens, s["dxs"].data_ptr(), row_of, 0, s["dx"].data_ptr(), stream)
        got |= {"dys": s["dys"], "dweights": s["dweights"], "dx": s["dx"]}
    return got


def _own_experts(s, ft, stream):
    tokens, rows, offsets = s["tokens"], s["tokens"] * s["top_k"], s["offsets"].data_ptr()
    _own_sort(s, ft, stream)
    ft.ft_i8_quantize(s["quantize_x"], tokens, s["x"].data_ptr(), s["q"].data_ptr(), s["sx"].data_ptr(), stream)
    ft.ft_i8_matmul_experts(s["up"], rows, offsets, s["q"].data_ptr(), s["sx"].data_ptr(), s["row_token"].data_ptr(), tokens, s["w1"].data_ptr(), s["sw1"].data_ptr(), 0,
                            s["h"].data_ptr(), stream)
    ft.ft_i8_quantize(s["quantize_h"], rows, s["h"].data_ptr(), s["qh"].data_ptr(), s["sh"].data_ptr(), stream)
    ft.ft_i8_matmul_experts(s["down"], rows, offsets, s["qh"].data_ptr(), s["sh"].data_ptr(), 0, rows, s["w2"].data_ptr(), s["sw2"].data_ptr(), 0, s["ys"].data_ptr(), stream)
    ft.ft_expert_combine(s["route"], tokens, s["ys"].data_ptr(), s["row_of"].data_ptr(), s["weights"].data_ptr(), s["out"].data_ptr(), stream)
    return {"offsets": s["offsets"], "row_of": s["row_of"], "out": s["out"]}


# ---- the plain forms -----------------------------------------------------------------------------


def _plain_quantize(x, cols, gated):
    f = x.float()
    if gated:
        gate, up = f[:, :cols], f[:, cols:]
        f = gate / (1 + torch.exp(-gate)) * up
    amax = f.abs().amax(dim=1, keepdim=True)
    q = torch.where(amax > 0, torch.round(f * 127 / amax), torch.zeros_like(f))
    return q, amax / 127


def _plain_linear(s):
    q, sx = _plain_quantize(s["x"], s["k"], s["gated"])
    y = torch.matmul(q, s["w"][:, :s["k"]].float().t()) * sx * s["sw"]
    if s["b"] is not None:
        y = y + s["b"]
    return {"y": y.to(s["y"].dtype), "scale": sx.reshape(-1)}


def _plain_sort(s):
    ids, experts, top_k = s["ids"].reshape(-1).long(), s["experts"], s["top_k"]
    keys = torch.where(ids >= 0, ids, experts)
    order = torch.sort(keys, stable=True)[1]
    counts = (keys[:, None] == torch.arange(experts, device=keys.device)).sum(dim=0)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
    place = torch.arange(keys.numel(), device=keys.device)
    row_token = torch.where(place < offsets[-1], order // top_k, -1)
    row_of = torch.empty_like(place)
    row_of[order] = place
    row_of = torch.where(ids >= 0, row_of, -1)
    return offsets, row_token, row_of


def _plain_carry(values, row_of, rows):
    """values [entries, cols] to their rows; rows that no entry goes to are zeros, as the buffers were."""
    out = torch.zeros(rows + 1, values.shape[1], dtype=values.dtype, device=values.device)
    out[torch.where(row_of >= 0, row_of, rows)] = values
    return out[:rows]


def _plain_fetch(rows, row_of, tokens):
    """[tokens, top_k, cols] in 32 bits, zeros where an entry has no row."""
    got = rows[row_of.clamp(min=0)].float() * (row_of >= 0)[:, None]
    return got.reshape(tokens, -1, rows.shape[1])


def _plain_permute(s):
    tokens, top_k = s["tokens"], s["top_k"]
    offsets, row_token, row_of = _plain_sort(s)
    i32 = torch.int32
    repeated = s["x"][:, None, :].expand(-1, top_k, -1).reshape(tokens * top_k, -1)
    ys = _plain_fetch(s["ys"], row_of, tokens)
    got = {"offsets": offsets.to(i32), "row_token": row_token.to(i32), "row_of": row_of.reshape(tokens, top_k).to(i32),
           "xs": _plain_carry(repeated, row_of, tokens * top_k), "out": (ys * s["weights"][:, :, None]).sum(dim=1).to(s["x"].dtype)}
    if s["grad"]:
        dout = s["dout"].float()[:, None, :]
        dys = (dout * s["weights"][:, :, None]).to(s["x"].dtype).reshape(tokens * top_k, -1)
        got |= {"dys": _plain_carry(dys, row_of, tokens * top_k), "dweights": (ys * dout).sum(dim=2),
                "dx": _plain_fetch(s["dxs"], row_of, tokens).sum(dim=1).to(s["x"].dtype)}
    return got


def _plain_grouped(q, scale, source, w, sw, offsets, n, k):
    """Every expert's rows side by side, as many for each as the fullest has: one batch of products.  source: the row of q that a row takes."""
    experts = offsets.numel() - 1
    counts = offsets[1:] - offsets[:-1]
    most = max(1, int(counts.max()))
    slot = torch.arange(most, device=q.device)
    rows = offsets[:-1, None] + slot
    there = slot < counts[:, None]
    take = source[torch.where(there, rows, 0)]
    products = torch.bmm(q[take], w.reshape(experts, n, -1)[:, :, :k].float().transpose(1, 2))
    products = products * scale[take] * sw.reshape(experts, 1, n)
    return products[there]


def _plain_experts(s):
    tokens, top_k, cols, ffn = s["tokens"], s["top_k"], s["cols"], s["ffn"]
    offsets, row_token, row_of = _plain_sort(s)
    q, sx = _plain_quantize(s["x"], cols, False)
    h = _plain_grouped(q, sx, row_token.clamp(min=0), s["w1"], s["sw1"], offsets, 2 * ffn, cols)
    qh, sh = _plain_quantize(h, ffn, True)
    if h.shape[0]:
        y = _plain_grouped(qh, sh, torch.arange(h.shape[0], device=q.device), s["w2"], s["sw2"], offsets, cols, ffn)
    else:
        y = torch.zeros(1, cols, device=q.device)
    out = (_plain_fetch(y, row_of, tokens) * s["weights"][:, :, None]).sum(dim=1)
    return {"offsets": offsets.to(torch.int32), "row_of": row_of.reshape(tokens, top_k).to(torch.int32), "out": out.to(s["x"].dtype)}


def run(state):
    kind = state["kind"]
    if own:
        import paper_2407_21418_amd as ft
        stream = torch.cuda.current_stream().cuda_stream
        if kind == "linear":
            return _own_linear(state, ft, stream)
        return _own_permute(state, ft, stream) if kind == "permute" else _own_experts(state, ft, stream)
    if kind == "linear":
        return _plain_linear(state)
    return _plain_permute(state) if kind == "permute" else _plain_experts(state)


# ---- what a pass cannot do without ---------------------------------------------------------------


def work(case):
    kind = case["kind"]
    es = 4 if case["dtype"] == "f32" else 2
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": 2 * m * k * (2 if case["gated"] else 1) + n * k + 4 * n + (4 * n if case["bias"] else 0) + 4 * m + out * m * n, "flops": 2 * m * n * k}
    entries, kept, cols = case["tokens"] * case["top_k"], (case["tokens"] - case["padded"]) * case["top_k"], case["cols"]
    kept_tokens = case["tokens"] - case["padded"]
    route = 4 * entries + 4 * entries  # ids read, weights read
    if kind == "permute":
        moved = es * cols * (kept_tokens + kept) + es * cols * (kept + case["tokens"])  # x to its rows; rows back to the tokens
        got = {"bytes": route + 8 * entries + 4 * case["experts"] + moved, "flops": 2 * kept * cols}
        if case["grad"]:  # dout read, dys written (the rows themselves are read once for both); dxs read, dx written
            got["bytes"] += es * cols * (kept_tokens + kept) + 4 * entries + es * cols * (kept + case["tokens"])
            got["flops"] += 4 * kept * cols
        return got
    ffn, experts = case["ffn"], case["experts"]
    hit = experts * (1 - (1 - case["top_k"] / experts) ** kept_tokens)  # experts that a token reaches, if all are liked alike
    weights = hit * (3 * ffn * cols + 4 * (2 * ffn + cols))
    return {"bytes": int(route + 4 * entries + 4 * experts + weights + es * cols * (kept_tokens + case["tokens"])), "flops": 6 * kept * cols * ffn}


# ---- the definitions in 64 bits ------------------------------------------------------------------


def _exact_rows(f):
    """(integers, scale) of each row, from its values in 64 bits."""
    peak = torch.max(torch.abs(f), dim=1)[0]
    safe = torch.where(peak == 0, torch.ones_like(peak), peak)
    return torch.round(f * (127.0 / 1.0) / safe[:, None]), peak / 127.0


def _exact_gated(f):
    half = f.shape[1] // 2
    return f[:, :half] * torch.sigmoid(f[:, :half]) * f[:, half:]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        f = s["x"].double()
        q, scale = _exact_rows(_exact_gated(f) if case["gated"] else f)
        y = scale[:, None] * (q @ s["w"].double()[:, :case["k"]].T) * s["sw"].double()[None, :]
        return {"y": y if s["b"] is None else y + s["b"].double()[None, :], "scale": scale}
    tokens, top_k, experts, cols = case["tokens"], case["top_k"], case["experts"], case["cols"]
    ids = s["ids"].reshape(-1).cpu().tolist()
    members = [[] for _ in range(experts)]
    for entry, e in enumerate(ids):
        if 0 <= e < experts:
            members[e].append(entry)
    packed = [entry for group in members for entry in group]
    at = torch.tensor(packed, dtype=torch.long, device="cuda")
    token, weight = at // top_k, s["weights"].double().reshape(-1)[at]
    offsets = [0]
    for group in members:
        offsets.append(offsets[-1] + len(group))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    row_of = torch.full((tokens * top_k,), -1, dtype=torch.int32, device="cuda")
    row_of[at] = torch.arange(len(packed), dtype=torch.int32, device="cuda")
    got = {"offsets": ints(offsets), "row_of": row_of.reshape(tokens, top_k)}
    back = lambda rows: torch.zeros(tokens, cols, dtype=torch.float64, device="cuda").index_add_(0, token, rows)  # noqa: E731
    if case["kind"] == "permute":
        behind = tokens * top_k - len(packed)
        tail = torch.zeros(behind, cols, dtype=torch.float64, device="cuda")
        kept = s["ys"][:len(packed)].double()
        got["row_token"] = torch.cat([token.to(torch.int32), torch.full((behind,), -1, dtype=torch.int32, device="cuda")])
        got["xs"] = torch.cat([s["x"].double()[token], tail])
        got["out"] = back(kept * weight[:, None])
        if case["grad"]:
            dout = s["dout"].double()[token]
            got["dys"] = torch.cat([dout * weight[:, None], tail])
            dweights = torch.zeros(tokens * top_k, dtype=torch.float64, device="cuda")
            dweights[at] = torch.sum(dout * kept, dim=1)
            got["dweights"] = dweights.reshape(tokens, top_k)
            got["dx"] = back(s["dxs"][:len(packed)].double())
        return got
    ffn, parts = case["ffn"], []
    q, scale = _exact_rows(s["x"].double())
    for e, group in enumerate(members):
        if group:
            t = token[offsets[e]:offsets[e + 1]]
            w1, w2 = (w.reshape(experts, n, -1)[e, :, :k].double() for w, n, k in ((s["w1"], 2 * ffn, cols), (s["w2"], cols, ffn)))
            h = scale[t][:, None] * (q[t] @ w1.T) * s["sw1"].reshape(experts, -1)[e].double()
            qh, sh = _exact_rows(_exact_gated(h))
            parts.append(sh[:, None] * (qh @ w2.T) * s["sw2"].reshape(experts, -1)[e].double())
    got["out"] = back(torch.cat(parts) * weight[:, None]) if parts else back(torch.zeros(0, cols, dtype=torch.float64, device="cuda"))
    return got
