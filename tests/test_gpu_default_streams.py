"""The operators on HIP's default streams by their handles (hipStreamLegacy 1, hipStreamPerThread 2) and by none."""
import pytest
import torch

import paper_2407_21418_amd as ft

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_default_streams(handle):
    tokens, top_k, experts, cols = 300, 2, 5, 96
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, experts, (tokens, top_k), generator=gen, device="cuda", dtype=torch.int32)
    x = torch.randn(tokens, cols, generator=gen, device="cuda").half()
    offsets, row_token, row_of = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (experts + 1, tokens * top_k, tokens * top_k))
    xs, back, c = torch.zeros(tokens * top_k, cols, device="cuda").half(), torch.zeros_like(x), torch.zeros(tokens, 32, device="cuda")
    q, scale = torch.zeros(tokens, cols, dtype=torch.int8, device="cuda"), torch.zeros(tokens, device="cuda")
    w, sw = torch.randint(-128, 128, (32, cols), generator=gen, device="cuda", dtype=torch.int8), torch.ones(32, device="cuda")
    torch.cuda.synchronize()
    d = ft.ft_expert_desc(experts=experts, top_k=top_k, cols=cols)
    ft.ft_expert_sort(d, tokens, ids.data_ptr(), offsets.data_ptr(), row_token.data_ptr(), row_of.data_ptr(), 0, 0, handle)
    ft.ft_expert_gather(d, tokens, x.data_ptr(), row_of.data_ptr(), xs.data_ptr(), handle)
    ft.ft_expert_combine(d, tokens, xs.data_ptr(), row_of.data_ptr(), 0, back.data_ptr(), handle)
    ft.ft_i8_quantize(ft.ft_quant_desc(cols=cols), tokens, x.data_ptr(), q.data_ptr(), scale.data_ptr(), handle)
    ft.ft_i8_matmul(ft.ft_i8_desc(n=32, k=cols), tokens, q.data_ptr(), scale.data_ptr(), w.data_ptr(), sw.data_ptr(), 0, c.data_ptr(), handle)
    torch.cuda.synchronize()
    assert torch.equal(xs, x[row_token.long()]) and torch.equal(back, x + x)
    # (an exact sum, its conversion and one product: two roundings)
    ref = (q.double() @ w.double().t()) * scale.double()[:, None]
    assert bool(((c.double() - ref).abs() <= 2.01 * 2.0 ** -24 * ref.abs()).all())
