"""ft_expert_sort and what lies around its workspace: nothing but the bytes it asks for is written, and what they hold before does not matter."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from test_gpu_experts import route, sort

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (5, 2, 8), (16384, 1, 64), (16385, 1, 64), (8192, 8, 128), (20000, 7, 1000), (300001, 5, 3), (600000, 4, 1024)])
def test_bytes_around_the_workspace(tokens, top_k, experts):
    g = np.random.default_rng(tokens)
    ids = g.integers(-1, experts, size=(tokens, top_k))
    need = ft.ft_expert_workspace(ft.ft_expert_desc(experts=experts, top_k=top_k), tokens)
    assert (need == 0) == (tokens * top_k <= 16384)
    want = route(ids, experts)
    for inside in (0, 255):
        whole = torch.full((need + 2048,), 0xA5, dtype=torch.uint8, device="cuda")
        whole[1024:1024 + need] = inside
        got = sort(ids, experts, workspace=whole[1024:])
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
        assert bool((whole[:1024] == 0xA5).all()) and bool((whole[1024 + need:] == 0xA5).all()), "write outside of the workspace"
