"""Every kind of launch that a call of attention takes (csrc/lora_attention.h), on the GPU against the definition in 64 bits, within test_gpu_attention.py's bound."""
import pytest
import torch

from paper_2511_22880_amd import binding as L
from test_attention_rules import FORMS, taken
from test_gpu_attention import Batch, within_guards

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name, bits", [(name, bits) for name in FORMS for bits in (8, 16) if taken(name, bits)])
def test_form(name, dim, bits, tree):
    sizes, most = FORMS[name]
    batch = Batch(sizes, 8, 2, dim, bits=bits, tree=tree, seed=40, spare=2)
    batch.check(most)
    assert (batch.y[-2:] == 9).all()


@pytest.mark.parametrize("name, bits", [(name, bits) for name in FORMS for bits in (8, 16) if taken(name, bits)])
def test_form_in_a_graph_on_what_another_call_left(name, bits):
    """captured twice on one workspace and replayed with eager calls between, whose cuts are elsewhere: what a launch leaves for the join is read by no other"""
    sizes, most = FORMS[name]
    batch, other = Batch(sizes, 8, 2, 64, bits=bits, seed=41), Batch(list(reversed(sizes)), 8, 2, 64, bits=bits, seed=42)
    ref = batch.run(most).clone()
    other_ref = other.run(most).clone()
    other.workspace = batch.workspace
    torch.cuda.synchronize()
    graphs = []
    for b in (batch, other):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            b.run(most, stream=torch.cuda.current_stream())
    for _ in range(3):
        for b, graph, expected in ((batch, graphs[0], ref), (other, graphs[1], other_ref)):
            b.y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(b.y, expected)
            b.y.zero_()
            assert torch.equal(b.run(most), expected)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sizes, heads, kv_heads, most", [
    ([(1, 700), (1, 20), (1, 1500)], 600, 600, 1), ([(2, 600), (1, 3)], 1200, 600, 2), ([(40, 1100), (3, 9)], 600, 600, 40), ([(150, 150), (2, 2500)], 700, 700, 150)])
def test_more_key_heads_than_work_groups(sizes, heads, kv_heads, most, bits):
    """one share of every key head: tiles are cut nowhere, whatever their steps"""
    Batch(sizes, heads, kv_heads, 64, bits=bits, seed=43).check(most)


@pytest.mark.parametrize("most", [1, 0])
def test_pages_that_requests_share(most):
    """three requests that begin with the same pages, two of which are the same to the end"""
    batch = Batch([(1, 600), (3, 520), (40, 600), (1, 100)], 8, 2, 128, page=32, seed=44)
    batch.table[1, :10] = batch.table[0, :10]
    batch.table[2] = batch.table[0]
    batch.check(most)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("n, requests, heads, kv_heads, most", [
    (1, 3, 32, 8, 1), (1, 600, 32, 8, 1), (8, 150, 64, 8, 8), (4096, 1, 64, 2, 4096), (4096, 1, 256, 8, 4096), (30, 300, 32, 8, 30), (0, 5, 8, 2, 0)])
def test_a_table_without_pages(n, requests, heads, kv_heads, most, bits):
    """no request has a key, whatever its length says: zeros, of as many rows as there are, up to more tiles than work groups"""
    batch = Batch([(n, 0)] * requests, heads, kv_heads, 64, bits=bits, spare=2, seed=45)
    batch.table = batch.table[:, :0]
    batch.lengths += 40
    size = L.lora_attention_workspace_bytes(batch.tokens, heads, requests, 0, batch.cache)
    batch.workspace = torch.full((max(16, size) // 4,), float("nan"), device="cuda")
    for said in (most, 0, 1):
        batch.y.fill_(9.0)
        y = batch.run(said)
        assert (y[:-2] == 0).all() and (y[-2:] == 9).all()


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name, bits", [(name, bits) for name in FORMS for bits in (8, 16) if taken(name, bits)])
def test_form_writes_its_rows_and_its_workspace_alone(name, dim, bits, tree):
    sizes, most = FORMS[name]
    batch = Batch(sizes, 8, 2, dim, bits=bits, tree=tree, seed=46)
    ref = batch.run(most).clone()
    untouched = within_guards(batch)
    assert torch.equal(batch.run(most), ref) and untouched()


@pytest.mark.parametrize("page, slots", [(16, 8192), (64, 131072)])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sizes, heads, kv_heads, most", [
    ([(1, 40), (1, 300), (1, 5)], 8, 2, 1), ([(3, 40), (8, 200), (5, 5)], 8, 2, 8), ([(600, 600)], 8, 2, 600), ([(1, 9)] * 40 + [(200, 250), (30, 30)], 8, 2, 200), ([(2, 33)] * 50, 16, 16, 2)])
def test_a_table_wider_than_its_requests(sizes, heads, kv_heads, most, bits, page, slots):
    """as wide as the longest context that a server allows, and a view of the columns that the requests need: the same rows within the bound, pages that are none behind them"""
    batch = Batch(sizes, heads, kv_heads, 64, page=page, bits=bits, seed=47)
    needed = batch.table.shape[1]
    wide = torch.full((len(sizes), slots // page), -7, dtype=torch.int32, device="cuda")
    wide[:, :needed] = batch.table
    size = L.lora_attention_workspace_bytes(batch.tokens, heads, len(sizes), slots // page, batch.cache)
    batch.workspace = torch.full((max(16, size) // 4,), float("nan"), device="cuda")
    for table in (wide, wide[:, :needed]):
        batch.table = table
        batch.check(most)
