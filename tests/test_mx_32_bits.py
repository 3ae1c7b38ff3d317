"""Sizes that do not fit the library's 32-bit arguments are refused, not cut off to what their low 32 bits say."""
from types import SimpleNamespace

import pytest
import torch

import paper_1711_00244_amd as cl

BIG = 1 << 32


def test_sizes_that_are_asked_about():
    W, experts = SimpleNamespace(shape=(64, 200), K=200), SimpleNamespace(shape=(8, 64, 200), K=200)
    for ask in (lambda: cl.mx_fc_workspace_bytes(W, BIG + 30000, torch.float32), lambda: cl.mx_fc_resolved_form(W, BIG + 3),
                lambda: cl.mx_fc_resolved_form(SimpleNamespace(shape=(BIG + 64, 200), K=200), 3), lambda: cl.mx_experts_resolved_form(experts, BIG + 5, 2),
                lambda: cl.mx_experts_resolved_form(experts, 5, BIG + 2)):
        with pytest.raises(ValueError):
            ask()
    assert cl.mx_fc_workspace_bytes(W, 30000, torch.float32) > 0 and cl.mx_fc_resolved_form(W, 3)[1] == 1


@pytest.mark.gpu
def test_choice_and_lists():
    x = torch.zeros((3, 8), device="cuda")
    for how in (dict(k=BIG + 2), dict(k=2, groups=BIG + 2), dict(k=2, groups=2, groups_kept=BIG + 1)):
        with pytest.raises(ValueError):
            cl.route_experts(x, **how)
    with pytest.raises(ValueError):
        cl.expert_lists(torch.zeros((3, 2), dtype=torch.int32, device="cuda"), BIG + 8)
    for k in (-1, 0, 9, (1 << 31) - 1):                      # (what fits is for the library to refuse, and nothing of that size is allocated)
        before = torch.cuda.max_memory_allocated()
        with pytest.raises(cl.CLError):
            cl.route_experts(x, k)
        assert torch.cuda.max_memory_allocated() - before < 1 << 20


@pytest.mark.gpu
def test_a_row_of_more_elements_than_32_bits_count():
    x = torch.empty((1, BIG + 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        cl.mx_quantize(x)
    del x
    q = cl.mx_quantize(torch.ones((2, 64), device="cuda"))
    q.K = BIG + 64                                           # (as a matrix of that size would have it)
    with pytest.raises(ValueError):
        cl.mx_dequantize(q, out=torch.empty((2, BIG + 64), dtype=torch.bfloat16, device="cuda"))
