"""AdaptedAttention's way from its projections to attention, on what each call of it reads: the queries turned, the turned keys and the values in the cache at the
slots that the page table says, attention over what the cache then holds.

Bounds, each against 64 bits on the values that the call read (half a step of bf16 is 2^-8 of the value): a turned value y of x1, x2 is off by 2^-8 |y| + 2^-21
(|x1| + |x2|), (1 + 2^-7) of it for what the bound itself leaves out; values are copied; a row of attention with M = sum w |v| by (2^-8 |y| + (2^-8 + 2 d +
2^-19 + 4 n 2^-24) M) (1 + 2^-6), d = (dim + 4) 2^-24 A (1 + 2^-3) of the largest A = scale sum |q||k|, n keys (test_gpu_attention.py has the count of roundings).

The checks run on any device: without a GPU on the definition in 64 bits, rounded as the kernels' outputs are, and on the same with one mistake in it each, which
they have to find; with one on a block's run."""
import pytest
import torch

from paper_2511_22880_amd import binding as L

BF = torch.bfloat16
U = 2.0 ** -24


def turned(x, positions, base=10000.0):
    """(values, bound without y's own rounding) in 64 bits; the pairs are the halves of a head"""
    half = x.shape[2] // 2
    f = base ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    a = positions.double()[:, None, None] * f
    x1, x2 = x[..., :half].double(), x[..., half:].double()
    off = (2.0 ** -21 * (x1.abs() + x2.abs())).repeat(1, 1, 2)
    return torch.cat([x1 * a.cos() - x2 * a.sin(), x1 * a.sin() + x2 * a.cos()], dim=2), off


def attended(q, k, v):
    """(values, bound) of the last rows of a request: q [rows][heads][dim], k, v [keys][kv_heads][dim]"""
    rows, heads, dim = q.shape
    keys, group = k.shape[0], heads // k.shape[1]
    q, (k, v) = q.double().permute(1, 0, 2), (t.double().repeat_interleave(group, dim=1).permute(1, 0, 2) for t in (k, v))
    late = torch.arange(keys, device=q.device)[None] > keys - rows + torch.arange(rows, device=q.device)[:, None]
    s = (q @ k.transpose(1, 2).contiguous() / dim ** 0.5).masked_fill(late, float("-inf"))
    a = (q.abs() @ k.abs().transpose(1, 2).contiguous() / dim ** 0.5).masked_fill(late, 0.0).amax(dim=2, keepdim=True)
    w = torch.softmax(s, dim=2)
    y, m = w @ v, w @ v.abs()
    d = (dim + 4) * U * a * (1 + 2.0 ** -3)
    bound = (2.0 ** -8 * y.abs() + (2.0 ** -8 + 2 * d + 2.0 ** -19 + 4 * keys * U) * m) * (1 + 2.0 ** -6)
    return y.permute(1, 0, 2), bound.permute(1, 0, 2)


def check(run):
    """run: q, k, v [tokens][heads][dim] as projected, turned_q, z likewise, held_k, held_v [pages][kv_heads][page][dim] behind the call, table, cached (a request's
    context, (k, v) [keys][kv_heads][dim], before it), positions [tokens], sizes (rows, keys)"""
    at, page = 0, run["held_k"].shape[2]
    ref, off = turned(run["q"], run["positions"])
    assert ((run["turned_q"].double() - ref).abs() <= (2.0 ** -8 * ref.abs() + off) * (1 + 2.0 ** -7)).all(), "queries"
    for r, ((rows, keys), (ck, cv)) in enumerate(zip(run["sizes"], run["cached"])):
        part, j = slice(at, at + rows), torch.arange(keys, device=ref.device)
        k, v = (run[name][run["table"][r, j // page].long(), :, j % page] for name in ("held_k", "held_v"))
        assert torch.equal(k[:keys - rows], ck) and torch.equal(v[:keys - rows], cv), "context"
        ref, off = turned(run["k"][part], run["positions"][part])
        assert ((k[keys - rows:].double() - ref).abs() <= (2.0 ** -8 * ref.abs() + off) * (1 + 2.0 ** -7)).all(), "keys"
        assert torch.equal(v[keys - rows:], run["v"][part]), "values"
        y, bound = attended(run["turned_q"][part], k, v)
        assert ((run["z"][part].double() - y).abs() <= bound).all(), "attention"
        at += rows


# ---- the checks themselves, on the definition with and without a mistake -------------------------------------
def definition(seed=1, turn=True, z=lambda q, k, v: attended(q, k, v)[0], swap=False):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g).to(BF)  # noqa: E731
    heads, kv_heads, dim, page, width = 8, 2, 128, 16, 20
    sizes = [(90, 90), (40, 200)] + [(1, 17 + 9 * i) for i in range(30)]
    tokens = sum(n for n, _ in sizes)
    q, k, v = (normal(tokens, h, dim) for h in (heads, kv_heads, kv_heads))
    positions = torch.tensor([j for n, keys in sizes for j in range(keys - n, keys)])
    held_k, held_v = (normal(width * len(sizes), kv_heads, page, dim) for _ in range(2))
    table = torch.randperm(width * len(sizes), generator=g).view(len(sizes), width)
    turn_of = (lambda x: turned(x, positions)[0].to(BF)) if turn else (lambda x: x)
    turned_q, turned_k, out, cached, at = turn_of(q), turn_of(k), torch.empty_like(q), [], 0
    for r, (rows, keys) in enumerate(sizes):
        j, part = torch.arange(keys), slice(at, at + rows)
        where = table[r, j // page], j % page
        own, before = (where[0][keys - rows:], where[1][keys - rows:]), (where[0][:keys - rows], where[1][:keys - rows])
        cached.append((held_k[before[0], :, before[1]], held_v[before[0], :, before[1]]))
        held_k[own[0], :, own[1]], held_v[own[0], :, own[1]] = turned_k[part], v[part]
        k_seen, v_seen = held_k[where[0], :, where[1]], held_v[where[0], :, where[1]]
        out[part] = z(turned_q[part], *((v_seen, k_seen) if swap else (k_seen, v_seen))).to(BF)
        at += rows
    return dict(q=q, k=k, v=v, turned_q=turned_q, z=out, held_k=held_k, held_v=held_v, table=table, cached=cached, positions=positions, sizes=sizes)


def test_the_definition_passes():
    check(definition())


def bidirectional(q, k, v):
    """rows that see their request's later keys too"""
    group = q.shape[1] // k.shape[1]
    q, k, v = q.double().permute(1, 0, 2), *(t.double().repeat_interleave(group, dim=1).permute(1, 0, 2) for t in (k, v))
    return (torch.softmax(q @ k.transpose(1, 2).contiguous() / q.shape[2] ** 0.5, dim=2) @ v).permute(1, 0, 2)


@pytest.mark.parametrize("mistake, says", [
    (dict(z=lambda q, k, v: torch.zeros_like(q)), "attention"),
    (dict(turn=False), "queries"),
    (dict(z=lambda q, k, v: attended(q.flip(1), k, v)[0]), "attention"),
    (dict(z=lambda q, k, v: attended(q, k.flip(1), v.flip(1))[0]), "attention"),
    (dict(z=lambda q, k, v: attended(q, k.flip(1), v)[0]), "attention"),
    (dict(z=lambda q, k, v: attended(q * 1.0625, k, v)[0]), "attention"),
    (dict(z=lambda q, k, v: 1.03125 * attended(q, k, v)[0]), "attention"),
    (dict(z=bidirectional), "attention"),
    (dict(z=lambda q, k, v: torch.cat([attended(q, k, v)[0][:1]] * q.shape[0])), "attention"),
    (dict(swap=True), "attention"),
], ids=["zeros", "not turned", "query heads reversed", "key heads exchanged", "keys of the other head", "another scale", "a factor", "later keys seen", "one row for all",
        "keys for values"])
def test_a_mistake_is_found(mistake, says):
    with pytest.raises(AssertionError, match=says):
        check(definition(**mistake))


@pytest.mark.parametrize("what, says", [("turned_q", "queries"), ("held_k", "keys"), ("held_v", "values"), ("context", "context")])
def test_a_wrong_place_is_found(what, says):
    run = definition()
    if what == "turned_q":
        run["turned_q"] = turned(run["q"], run["positions"] + 1)[0].to(BF)
    elif what == "context":  # a page of the second request's context overwritten
        run["held_k"][run["table"][1, 0]] = 0
    else:  # a token of the first prompt a slot further on
        page, at = run["table"][0, 2], slice(3, 9)
        run[what][page, :, at] = run[what][page, :, 2:8].clone()
    with pytest.raises(AssertionError, match=says):
        check(run)


# ---- a block's run ------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_a_block_on_what_its_calls_read(monkeypatch):
    from paper_2511_22880_amd import expert_layer as m
    taken, attention = [], L.lora_attention

    def noted(q, starts, lengths, page_table, *rest, **more):
        taken.append(page_table)
        return attention(q, starts, lengths, page_table, *rest, **more)
    monkeypatch.setattr(m.L, "lora_attention", noted)
    g = torch.Generator(device="cuda").manual_seed(18)
    block, adapters, _, _, _, (cached, positions, sizes, dim) = m.attention_example(lambda *shape: torch.randn(*shape, generator=g, device="cuda"))
    heads = lambda t: t.view(t.shape[0], -1, dim)  # noqa: E731
    check(dict(q=heads(block.q), k=heads(block.k), v=heads(block.v), turned_q=heads(block.turned), z=heads(block.z), held_k=block.cache.k, held_v=block.cache.v,
               table=taken[0], cached=cached, positions=positions, sizes=sizes))
    assert len(taken) == 1 and block.z.abs().sum() > 0
    for a in adapters:
        a.close()
