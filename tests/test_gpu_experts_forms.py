"""Every kernel that the products of include/lora_experts.h can take, on the GPU against the definitions in 64 bits.  test_experts_rules.py says, without
a GPU, that these sizes take the kernels they stand for, and that there are no others.  The bounds are those of test_gpu_experts.py."""
import pytest
import torch

import test_gpu_experts as E
from paper_2511_22880_amd import binding as L
from test_experts_rules import EXPERTS_FORMS, LAYER_FORMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ordered", [True, False])
@pytest.mark.parametrize("name, bits", EXPERTS_FORMS)
def test_experts(name, bits, ordered):
    sizes, picks, idle, in_f, out_f = EXPERTS_FORMS[name, bits]
    E.run_experts(sizes, picks, in_f, out_f, bits, idle, ordered)


@pytest.mark.parametrize("name", LAYER_FORMS)
def test_one_layer(name):
    rows, in_f, out_f = LAYER_FORMS[name]
    g = E.gen(rows)
    q, s = E.rows8(g, rows, in_f)
    w, ws = E.weights8(g, 1, out_f, in_f)
    y = torch.full((rows + 2, out_f), -7.0, dtype=E.BF, device="cuda")
    L.lora_linear_scaled(q, s, E.packed(w, in_f), ws, y[1:-1])
    if in_f % 128:
        w[:, :, in_f:] = 0.0
    E.close(y[1:-1], *E.product8(q, s, w[0], ws[0]))
    assert (y[[0, -1]] == -7).all()


@pytest.mark.parametrize("name, bits", EXPERTS_FORMS)
def test_the_same_bits_every_time_and_for_a_row_in_any_company(name, bits):
    """sums are taken in an order of their own for every row: neither repetition nor the row's place among its expert's shows"""
    sizes, _, _, in_f, out_f = EXPERTS_FORMS[name, bits]
    g = E.gen(in_f)
    rows = sum(sizes)
    starts = torch.tensor([sum(sizes[:e]) for e in range(len(sizes) + 1)], dtype=torch.int32, device="cuda")
    if bits == 16:
        x = torch.randn(rows, in_f, generator=g, device="cuda").to(E.BF)
        p = E.packed((torch.randn(len(sizes), out_f, in_f, generator=g, device="cuda") * 0.05).to(E.BF))
    else:
        q, s = E.rows8(g, rows, in_f)
        w, ws = E.weights8(g, len(sizes), out_f, in_f)
        p = E.packed(w, in_f)

    def run(order):
        y = torch.empty(rows, out_f, dtype=E.BF, device="cuda")
        order = order.to(torch.int32)
        if bits == 16:
            L.lora_experts_linear(x, starts, order, 1, p, y)
        else:
            L.lora_experts_linear_scaled(q, s, starts, order, 1, p, ws, y)
        return y
    same = torch.arange(rows, device="cuda")
    first = run(same)
    for _ in range(3):
        assert torch.equal(run(same), first)
    perm = torch.cat([int(starts[e]) + torch.randperm(n, generator=g, device="cuda") for e, n in enumerate(sizes)])
    assert torch.equal(run(perm), first[perm])
