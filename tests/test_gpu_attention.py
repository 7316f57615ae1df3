"""The operators of include/lora_attention.h on the GPU against their definitions in 64 bits, at the sizes and values where they can go wrong.

Bounds.  A rounding to nearest is off by half a step at most: bf16 2^-8 of the value, E4M3 2^-4 (2^-10 scales below its normal range), fp32 2^-24.

Turned values: the angle is kept to 2^-32 turns and read in fp32 within an eighth of a turn, 2^-28 turns: less than 2^-25 radians in all; cosine and sine are
off by 4 of their last places at most (2^-22), their product with the magnitude by 2^-24, the two products and their sum by 2 * 2^-24.  All of it is below
2^-21 m (|x1| + |x2|).

Attention: products of bf16 are exact, so a score s = scale q.k is off by (dim + 4) 2^-24 scale sum |q||k|: dim additions, the scale, the key's scale, the
difference from the maximum and the scale's own rounding.  With A the largest of scale sum |q||k| of a row, a weight is off by the factor
exp(d), d = (dim + 4) 2^-24 A (1 + 2^-3), by 2^-21 in the exponential itself, and by 2^-8 where it is rounded for its product with v (2^-24 more for v's scale); the sums over n keys by
n 2^-24 each, some rescalings by as much as the sums over the steps, n 2^-24 at most.  Numerator and denominator both: with M = sum w |v|,
|y - ref| <= (2^-8 |ref| + (2^-8 + 2 d + 2^-19 + 4 n 2^-24) M) (1 + 2^-6).
"""
import math

import numpy as np
import pytest
import torch

from paper_2511_22880_amd import binding as L

pytestmark = pytest.mark.gpu
F8, BF, I32 = torch.float8_e4m3fn, torch.bfloat16, torch.int32
U = 2.0 ** -24


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen(seed), device="cuda") * scale).to(BF)


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def within(y, ref, bound):
    y = y.double()
    assert torch.equal(y.isnan(), ref.isnan())
    d = torch.where(ref.isnan(), 0.0, (y - ref).abs())
    assert (d <= bound.nan_to_num(0)).all(), f"{(d / bound.clamp(min=1e-300)).nan_to_num(0).max().item():.3f} of the bound"


# ---- rotary positions ---------------------------------------------------------------------------------------
def turned(x, positions, rotary, dims, base=10000.0, inverse=False):
    """(values, bound) of plain frequencies, in 64 bits"""
    f = base ** (-torch.arange(0, dims, 2, dtype=torch.float64, device="cuda") / dims)
    a = positions.double()[:, None, None] * f * (-1 if inverse else 1)
    y, m = x.double().clone(), rotary.magnitude
    off = torch.zeros_like(y)
    s0, s1 = (slice(0, dims, 2), slice(1, dims, 2)) if rotary.interleaved else (slice(0, dims // 2), slice(dims // 2, dims))
    x1, x2 = x[..., s0].double(), x[..., s1].double()
    y[..., s0], y[..., s1] = m * (x1 * a.cos() - x2 * a.sin()), m * (x1 * a.sin() + x2 * a.cos())
    off[..., s0] = off[..., s1] = 2.0 ** -21 * m * (x1.abs() + x2.abs())
    return y, off


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens, heads, dim, dims", [
    (1, 1, 16, 16), (1, 32, 128, 128), (3, 5, 48, 32), (7, 8, 64, 64), (5, 1, 256, 256), (130, 1, 64, 16), (1025, 3, 80, 80), (700, 40, 128, 64),
    (5000, 2, 128, 128), (9, 4096, 16, 16)])
def test_rotary(tokens, heads, dim, dims, interleaved):
    x = normal(tokens, tokens, heads, dim)
    positions = torch.randint(0, 1 << 20, (tokens,), generator=gen(1), device="cuda", dtype=I32)
    positions[0] = 0
    rotary = L.Rotary(dims, interleaved=interleaved)
    y = torch.full_like(x, 7.0)
    L.lora_rotary(x, positions, rotary, y)
    ref, off = turned(x, positions, rotary, dims)
    within(y, ref, (2.0 ** -8 * ref.abs() + off) * (1 + 2.0 ** -7))
    assert torch.equal(y[..., dims:], x[..., dims:]) and torch.equal(y[0], x[0])
    z = x.clone()
    L.lora_rotary(z, positions, rotary)  # in place
    assert torch.equal(z, y)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient(interleaved):
    """dx of y = R x is R^T dy: against the formula, and <R x, dy> = <x, R^T dy> for whatever x and dy; against differences of the values in 64 bits."""
    n, heads, dim, dims = 33, 4, 64, 48
    x, dy = normal(1, n, heads, dim), normal(2, n, heads, dim)
    positions = torch.randint(0, 5000, (n,), generator=gen(3), device="cuda", dtype=I32)
    rotary = L.Rotary(dims, interleaved=interleaved, scaling="dimension", factor=8.0, low=1.0, high=32.0, length=4096.0)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    L.lora_rotary(x, positions, rotary, y)
    L.lora_rotary(dy, positions, rotary, dx, inverse=True)
    forward, back = (y.double() * dy.double()).sum(), (x.double() * dx.double()).sum()
    size = (y.double().abs() * dy.double().abs()).sum() + (x.double().abs() * dx.double().abs()).sum()
    assert rotary.magnitude > 1.2 and (forward - back).abs() <= 2.0 ** -7 * size
    # one element moved: the difference of the loss sum(y dy), linear in x, is the gradient but for y's roundings
    step = 64.0
    for t, h, e in [(5, 1, 0), (20, 3, dims - 1), (32, 0, dims)]:
        far = torch.zeros_like(x)
        far[t, h, e] = step
        moved = torch.empty_like(x)
        L.lora_rotary(far, positions, rotary, moved)
        difference = (moved.double() * dy.double()).sum() / step
        bound = 2.0 ** -7 * ((moved.double() * dy.double()).abs().sum() / step + dx[t, h, e].double().abs())
        assert (difference - dx[t, h, e].double()).abs() <= bound


def test_rotary_far_positions_and_frequencies():
    """positions to the end of 32 bits, by the bits that the library states: exact integers modulo a turn"""
    positions = ints([0, 1, 2, 1 << 20, (1 << 31) - 1, 123456789])
    for kind in L.ROTARY_SCALING:
        rotary = L.Rotary(128, 500000.0, scaling=kind, factor=8.0, low=1.0, high=4.0, length=8192.0)
        x = normal(4, 6, 2, 128)
        y = torch.empty_like(x)
        L.lora_rotary(x, positions, rotary, y)
        turns = [int(t) % (1 << 64) for t in rotary.turns.tolist()]
        a = torch.tensor([[(p * t % (1 << 64)) / 2.0 ** 64 * 2 * math.pi for t in turns] for p in positions.tolist()], dtype=torch.float64, device="cuda")[:, None]
        x1, x2, m = x[..., :64].double(), x[..., 64:].double(), rotary.magnitude
        ref = torch.cat([m * (x1 * a.cos() - x2 * a.sin()), m * (x1 * a.sin() + x2 * a.cos())], dim=2)
        off = 2.0 ** -21 * m * (x1.abs() + x2.abs()).repeat(1, 1, 2)
        within(y, ref, (2.0 ** -8 * ref.abs() + off) * (1 + 2.0 ** -7))


def test_rotary_strides_padding_and_nothing_beside_the_rows():
    wide = torch.full((9, 6, 96), 5.0, dtype=BF, device="cuda")
    wide[:, 1:5, 16:80] = normal(5, 9, 4, 64)
    x, before = wide[:, 1:5, 16:80], wide.clone()
    positions = ints([3, -1, 0, 7, -(1 << 31), 9, 11, 2, 5])
    rotary = L.Rotary(32)
    L.lora_rotary(x, positions, rotary)
    ref, off = turned(before[:, 1:5, 16:80], positions.clamp(min=0), rotary, 32)
    keep = positions >= 0
    within(x[keep], ref[keep], ((2.0 ** -8 * ref.abs() + off) * (1 + 2.0 ** -7))[keep])
    assert torch.equal(x[~keep], before[:, 1:5, 16:80][~keep])
    wide[:, 1:5, 16:80] = before[:, 1:5, 16:80]
    assert torch.equal(wide, before)
    # heads first in memory
    by_head = normal(6, 4, 9, 64)
    y = torch.zeros(4, 9, 64, dtype=BF, device="cuda")
    L.lora_rotary(by_head.transpose(0, 1), positions, rotary, y.transpose(0, 1))
    z = by_head.transpose(0, 1).contiguous()
    L.lora_rotary(z, positions, rotary)
    z[~keep] = 0
    assert torch.equal(y.transpose(0, 1), z)


# ---- the cache ----------------------------------------------------------------------------------------------
def nearest8(v):
    """the nearest E4M3 value in 64 bits, ties to even"""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def new_cache(pages, heads, page, dim, bits, seed=None):
    """tensors of a cache: of noise, or (seed None) of ones"""
    shape = (pages, heads, page, dim)
    x = torch.ones(shape, device="cuda") if seed is None else torch.randn(shape, generator=gen(seed), device="cuda")
    if bits == 16:
        return dict(k=x.to(BF), v=(x * 0.5 if seed is None else torch.randn(shape, generator=gen(seed + 1), device="cuda")).to(BF))
    s = [torch.ones(shape[:3], device="cuda") if seed is None else torch.rand(shape[:3], generator=gen(seed + i), device="cuda") * 0.03 + 0.001 for i in (2, 3)]
    v = x * 0.5 if seed is None else torch.randn(shape, generator=gen(seed + 1), device="cuda")
    return dict(k=(x * 30).to(F8), v=(v * 30).to(F8), k_scales=s[0], v_scales=s[1])


def copied(cache):
    return {n: t.clone() for n, t in cache.items()}


def same(a, b):
    return all(torch.equal(a[n].view(torch.uint8) if a[n].dtype == F8 else a[n], b[n].view(torch.uint8) if b[n].dtype == F8 else b[n]) for n in a)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tokens, heads, kv_heads, dim, dims, page, interleaved", [
    (1, 4, 1, 64, 64, 16, False), (1, 32, 8, 128, 128, 16, False), (17, 6, 2, 128, 32, 32, True), (130, 0, 3, 64, 16, 64, False), (5, 8, 8, 128, 128, 1024, True),
    (2500, 8, 2, 128, 128, 16, False), (3, 2, 1, 64, 0, 16, False)])
def test_append(tokens, heads, kv_heads, dim, dims, page, interleaved, bits):
    kv = normal(tokens, tokens, 2 * kv_heads, dim)
    k, v = kv[:, :kv_heads], kv[:, kv_heads:]
    q = normal(tokens + 1, tokens, heads, dim) if heads and dims else None
    y = torch.full_like(q, 3.0) if q is not None else None
    pages = -(-tokens // page) + 3
    slots = torch.randperm(pages * page, generator=gen(2), device="cuda")[:tokens].to(I32)
    positions = torch.randint(0, 40000, (tokens,), generator=gen(3), device="cuda", dtype=I32)
    if tokens > 4:
        slots[1], slots[3], positions[2] = -1, pages * page, -5
    gone = (slots < 0) | (slots >= pages * page) | (positions < 0)
    tensors = new_cache(pages, kv_heads, page, dim, bits, seed=9)
    before, cache = copied(tensors), L.Cache(**tensors)
    rotary = L.Rotary(dims, interleaved=interleaved) if dims else None
    L.lora_cache_append(k, v, slots, cache, rotary, positions, q, y)
    keep = ~gone
    at, off_at = (slots[keep] // page).long(), (slots[keep] % page).long()
    ref_k, off_k = turned(k, positions, rotary, dims) if dims else (k.double(), torch.zeros(k.shape, device="cuda").double())
    ref_k, off_k = ref_k[keep], off_k[keep]
    if bits == 16:
        within(tensors["k"][at, :, off_at], ref_k, (2.0 ** -8 * ref_k.abs() + off_k) * (1 + 2.0 ** -7))
        assert torch.equal(tensors["v"][at, :, off_at], v[keep])
        before["k"][at, :, off_at], before["v"][at, :, off_at] = tensors["k"][at, :, off_at], v[keep]
    else:
        byte = lambda name: tensors[name].view(torch.uint8)[at, :, off_at].view(F8).double()  # noqa: E731
        top = v[keep].double().abs().amax(dim=2).clamp(min=448 * 2.0 ** -126)
        assert torch.equal(tensors["v_scales"][at, :, off_at], (top / 448).float())
        assert torch.equal(byte("v"), nearest8(v[keep].double() * 448 / top[..., None]))
        ks = tensors["k_scales"][at, :, off_at].double()
        within(ks, ref_k.abs().amax(dim=2) / 448, (off_k.amax(dim=2) / 448 + 2 * U * ks) * (1 + 2.0 ** -7))
        within(byte("k") * ks[..., None], ref_k, (2.0 ** -4 * ref_k.abs() + 2.0 ** -10 * ks[..., None] + 2 * off_k) * (1 + 2.0 ** -6))
        for n in ("k", "v"):
            before[n].view(torch.uint8)[at, :, off_at] = tensors[n].view(torch.uint8)[at, :, off_at]
            before[n + "_scales"][at, :, off_at] = tensors[n + "_scales"][at, :, off_at]
    assert same(tensors, before)  # nothing else was touched
    if q is not None:
        z = q.clone()
        L.lora_rotary(z, positions, rotary)
        z[gone] = 3.0
        assert torch.equal(y, z)


def test_append_infinities_and_nan_in_8_bits():
    v = torch.ones(4, 2, 64, dtype=BF, device="cuda")
    v[0, 0, 3], v[1, 1, 9], v[1, 1, 10] = float("inf"), float("nan"), -float("inf")
    v[2] = 0
    tensors = new_cache(1, 2, 16, 64, 8)
    L.lora_cache_append(v, v, ints([0, 1, 2, 3]), L.Cache(**tensors))
    for n in ("k", "v"):
        held, s = tensors[n].float(), tensors[n + "_scales"]
        assert s[0, 0, 0].isinf() and held[0, 0, 0, 3].isnan() and held[0, 0, 0].nan_to_num(0).abs().sum() == 0
        assert s[0, 1, 1].isnan() and held[0, 1, 1].isnan().all()
        assert (held[0, :, 2] == 0).all() and (s[0, :, 2] == 2.0 ** -126).all() and (held[0, 1, 0] == 448).all() and (held[0, :, 3] == 448).all()


def test_append_two_tokens_with_one_slot_touch_nothing_else():
    tensors = new_cache(2, 1, 16, 64, 16)
    before = copied(tensors)
    x = normal(3, 2, 1, 64)
    L.lora_cache_append(x, x, ints([5, 5]), L.Cache(**tensors))
    for n in ("k", "v"):
        assert ((tensors[n][0, 0, 5] == x[0, 0]) | (tensors[n][0, 0, 5] == x[1, 0])).all()
        tensors[n][0, 0, 5] = before[n][0, 0, 5]
    assert same(tensors, before)


# ---- attention ----------------------------------------------------------------------------------------------
class Batch:
    """Requests of (rows, keys) over a cache of noise, whose pages lie anywhere."""

    def __init__(self, sizes, heads, kv_heads, dim, page=16, bits=16, tree=False, seed=1, spare=0, loud=1.0):
        self.sizes, self.heads, self.kv_heads, self.dim, self.page, self.bits = sizes, heads, kv_heads, dim, page, bits
        counts = [-(-keys // page) for _, keys in sizes]
        pages = sum(counts) + 2
        where = torch.randperm(pages, generator=gen(seed), device="cuda").to(I32)
        self.table = torch.full((len(sizes), max(1, max(counts))), -7, dtype=I32, device="cuda")
        at = 0
        for r, n in enumerate(counts):
            self.table[r, :n] = where[at:at + n]
            at += n
        self.first = [0]
        for n, _ in sizes:
            self.first.append(self.first[-1] + n)
        self.tokens = self.first[-1] + spare
        self.starts, self.lengths = ints(self.first), ints([keys for _, keys in sizes])
        self.tensors = new_cache(pages, kv_heads, page, dim, bits, seed=seed + 10)
        self.cache = L.Cache(**self.tensors)
        self.q = normal(seed + 20, self.tokens, heads, dim, scale=loud)
        self.y = torch.full_like(self.q, 9.0)
        self.tree = None
        if tree:
            words = torch.randint(0, 1 << 62, (self.tokens,), generator=gen(seed + 30), device="cuda") * 4 + 3
            words[::3] = torch.randint(0, 16, words[::3].shape, generator=gen(seed + 31), device="cuda")  # few, or none
            self.tree = words
        n = L.lora_attention_workspace_bytes(self.tokens, heads, len(sizes), self.table.shape[1], self.cache)
        self.workspace = torch.full((max(16, n) // 4,), float("nan"), device="cuda")

    def run(self, most=0, stream=None, **more):
        L.lora_attention(self.q, self.starts, self.lengths, self.table, self.cache, self.y, self.workspace, tree=self.tree, most=most, stream=stream, **more)
        return self.y

    def held(self, name, r):
        """fp64 [kv_heads][keys][dim] of request r, and which keys lie on pages that there are"""
        n, keys = self.sizes[r]
        ids = self.table[r, :-(-keys // self.page)].long()
        there = (ids >= 0) & (ids < self.cache.pages)
        ids = torch.where(there, ids, 0)
        x = self.tensors[name].view(torch.uint8)[ids].view(self.tensors[name].dtype).double()
        if self.bits == 8:
            x = x * self.tensors[name + "_scales"][ids].double()[..., None]
        return x.transpose(0, 1).reshape(self.kv_heads, -1, self.dim)[:, :keys], there.repeat_interleave(self.page)[:keys]

    def sees(self, r):
        n, keys = self.sizes[r]
        own = torch.arange(keys, device="cuda")[None] - (keys - n)
        i = torch.arange(n, device="cuda")[:, None]
        if self.tree is None:
            return own <= i
        word = self.tree[self.first[r]:self.first[r + 1]][:, None]
        return (own < 0) | ((own < 64) & ((word >> own.clamp(0, 63)) & 1 == 1))

    def reference(self, scale=None):
        scale = self.dim ** -0.5 if scale is None else scale
        ref = torch.full(self.q.shape, 9.0, dtype=torch.float64, device="cuda")
        bound = torch.zeros_like(ref)
        group = self.heads // self.kv_heads
        for r, (n, keys) in enumerate(self.sizes):
            (k, there), (v, _) = self.held("k", r), self.held("v", r)
            sees = self.sees(r) & there[None]
            for h in range(self.heads):
                rows = slice(self.first[r], self.first[r + 1])
                q, kk, vv = self.q[rows, h].double(), k[h // group], v[h // group]
                s = torch.where(sees, q @ kk.t() * scale, -math.inf)
                a = torch.where(sees, q.abs() @ kk.abs().t() * abs(scale), 0.0).amax(dim=1, keepdim=True) if keys else torch.zeros(n, 1, device="cuda").double()
                top = s.amax(dim=1, keepdim=True) if keys else torch.zeros(n, 1, device="cuda").double()
                w = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
                total = w.sum(dim=1, keepdim=True)
                w = torch.where(total == 0, 0.0, w / total)
                y, m = torch.zeros(n, self.dim, device="cuda").double(), torch.zeros(n, self.dim, device="cuda").double()
                odd = ~torch.isfinite(vv).all(dim=1)
                y, m = y + w[:, ~odd] @ vv[~odd], m + w[:, ~odd] @ vv[~odd].abs()
                for j in torch.nonzero(odd)[:, 0].tolist():  # (nought times an infinity is none of the definition's where the key is not seen)
                    y = torch.where(sees[:, j, None], y + w[:, j, None] * vv[j], y)
                d = (self.dim + 4) * U * a * (1 + 2.0 ** -3)
                ref[rows, h] = y
                bound[rows, h] = ((2.0 ** -8 * y.abs() + (2.0 ** -8 + 2 * d + 2.0 ** -19 + 4 * keys * U) * m) * (1 + 2.0 ** -6)).nan_to_num(0)
        return ref, bound

    def check(self, most=0, scale=None):
        ref, bound = self.reference(scale)
        self.y.fill_(9.0)
        within(self.run(most, scale=scale), ref, bound)


SHAPES = [(4, 4, 64), (32, 8, 128), (7, 1, 128), (6, 2, 64), (64, 1, 128), (16, 1, 64)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads, kv_heads, dim", SHAPES)
def test_single_tokens(heads, kv_heads, dim, bits):
    lengths = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 2047]
    Batch([(1, n) for n in lengths], heads, kv_heads, dim, bits=bits).check(most=1)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("bits", [16, 8])
def test_pages(page, bits):
    Batch([(1, 700), (3, 1500), (40, 333), (1, 1), (300, 300)], 8, 2, 128, page=page, bits=bits).check()


@pytest.mark.parametrize("length", [1, 100, 5000, 70000])
@pytest.mark.parametrize("heads, kv_heads, dim, bits", [(32, 8, 128, 16), (8, 8, 64, 8), (5, 5, 128, 8)])
def test_one_request(length, heads, kv_heads, dim, bits):
    Batch([(1, length)], heads, kv_heads, dim, bits=bits, page=64).check(most=1)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads, kv_heads, dim", SHAPES)
@pytest.mark.parametrize("sizes", [
    [(2, 2), (3, 70), (4, 4), (5, 1000), (1, 7)], [(16, 16), (17, 300), (8, 9)], [(64, 64), (65, 65), (31, 1031), (33, 40)],
    [(130, 130), (1, 500), (257, 900), (2, 2)], [(1, 3), (600, 1234), (1, 40), (100, 100)]])
def test_prompts_and_pieces(sizes, heads, kv_heads, dim, bits):
    batch = Batch(sizes, heads, kv_heads, dim, bits=bits)
    batch.check(most=max(n for n, _ in sizes))
    batch.check()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads, kv_heads, dim", SHAPES)
@pytest.mark.parametrize("sizes", [
    [(1, 1), (1, 50), (3, 3), (5, 200), (4, 1000)], [(8, 500), (16, 700), (13, 13)], [(24, 400), (40, 1100), (64, 64), (64, 800), (33, 33)]])
def test_trees(sizes, heads, kv_heads, dim, bits):
    batch = Batch(sizes, heads, kv_heads, dim, bits=bits, tree=True)
    batch.check(most=max(n for n, _ in sizes))


def test_trees_of_more_than_64_rows_see_their_first_64_keys():
    Batch([(100, 150), (70, 70), (3, 9)], 8, 2, 64, tree=True).check()


@pytest.mark.parametrize("tree", [False, True])
def test_requests_without_rows_without_keys_and_with_fewer_keys_than_rows(tree):
    for sizes in ([(0, 0), (0, 40), (1, 0), (5, 0), (3, 1), (40, 17), (0, 9), (200, 30), (1, 64), (0, 5)], [(1, 0)], [(0, 3), (0, 0)], [(300, 0)]):
        batch = Batch(sizes, 8, 2, 64, tree=tree, spare=3)
        batch.check()
        batch.check(most=1)
        assert (batch.y[-3:] == 9).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tree", [False, True])
def test_what_a_row_does_not_see_has_no_part_in_it(bits, tree):
    """slots behind a request's last key, whole pages that are nobody's, and its own later keys hold infinities and NaN"""
    sizes = [(1, 5), (1, 33), (6, 100), (20, 47), (50, 203), (64, 64), (300, 321)] if not tree else [(1, 5), (6, 100), (20, 47), (50, 203), (64, 64)]
    batch = Batch(sizes, 8, 2, 128, bits=bits, tree=tree, seed=4)
    used = torch.zeros(batch.cache.pages, batch.page, dtype=torch.bool, device="cuda")
    for r, (n, keys) in enumerate(sizes):
        for j in range(keys):
            used[int(batch.table[r, j // batch.page]), j % batch.page] = True
    bad = (~used)[:, None, :].expand(-1, 2, -1)
    for name in ("k", "v"):
        t = batch.tensors[name]
        t.view(torch.uint8 if bits == 8 else torch.int16)[bad] = 0x7F if bits == 8 else 0x7FC0
        if bits == 8:
            batch.tensors[name + "_scales"][bad] = float("nan")
    # own keys that not every row sees
    for r, (n, keys) in enumerate(sizes):
        if n < 6:
            continue
        for own, value in ((n - 1, float("nan")), (n - 2, float("inf")), (n // 2, -float("inf"))):
            key = keys - n + own
            page, at = int(batch.table[r, key // batch.page]), key % batch.page
            if bits == 8:
                batch.tensors["v"].view(torch.uint8)[page, 1, at, 3] = 0x7F
                batch.tensors["v_scales"][page, 0, at] = value
                batch.tensors["k_scales"][page, 0, at] = float("nan") if own == n - 1 else 1.0
            else:
                batch.tensors["v"][page, :, at, own % 128] = value
                batch.tensors["k"][page, :, at, 5] = float("nan") if own == n - 1 else 1.0
    ref, bound = batch.reference()
    assert ref.isnan().any() and torch.isfinite(ref).any()
    for most in (0, max(n for n, _ in sizes)):
        batch.y.fill_(9.0)
        y = batch.run(most).double()
        assert torch.equal(torch.isfinite(y), torch.isfinite(ref))
        fine = torch.isfinite(ref)
        assert ((y - ref).abs()[fine] <= bound[fine]).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads, dim, most", [(16, 64, 1), (32, 128, 1), (8, 64, 1), (8, 128, 40)])
@pytest.mark.parametrize("tree", [False, True])
def test_a_row_alone_in_its_tile_does_not_see_later_keys(heads, dim, most, bits, tree):
    """one key head: 16 heads are a tile's columns, and 32 keys of a step are looked at by one row only.  Its request's later keys, or (tree) its own, hold infinities"""
    batch = Batch([(2, 20), (1, 33), (3, 75), (1, 1)], heads, 1, dim, bits=bits, tree=tree, seed=6)
    if tree:
        batch.tree.copy_(torch.tensor([1, 1, 0, 1, 0, 1, 0]))
    for r, own in ((0, 1), (1, 0), (2, 1), (2, 2), (3, 0)):
        if not tree and own == 0:
            continue
        n, keys = batch.sizes[r]
        key = keys - n + own
        page, at = int(batch.table[r, key // 16]), key % 16
        if bits == 8:
            batch.tensors["v"].view(torch.uint8)[page, 0, at, 9] = 0x7F
        else:
            batch.tensors["v"][page, 0, at, 9] = float("inf")
    ref, bound = batch.reference()
    y = batch.run(most).double()
    assert torch.isfinite(ref[0]).all() and torch.equal(torch.isfinite(y), torch.isfinite(ref))
    fine = torch.isfinite(ref)
    assert ((y - ref).abs()[fine] <= bound[fine]).all()


@pytest.mark.parametrize("most", [1, 8, 40])
def test_infinities_before_requests_without_keys(most):
    """work groups that have several tiles, some of them of rows that see nothing, behind one whose later keys hold infinities"""
    sizes = [(20, 64), (20, 0), (20, 64), (20, 0), (20, 0)] * 240 + [(1, 9000)]
    batch = Batch(sizes, 4, 2, 128, seed=8)
    for r in range(0, 1200, 5):
        for x in (0, 2):
            batch.tensors["v"][int(batch.table[r + x, 3]), :, 15, r % 128] = float("inf")  # the last key
    ref, bound = batch.reference()
    y = batch.run(most).double()
    assert torch.equal(torch.isfinite(y), torch.isfinite(ref)) and torch.isinf(ref).any()
    fine = torch.isfinite(ref)
    assert ((y - ref).abs()[fine] <= bound[fine]).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("most", [1, 40])
def test_pages_that_are_none_are_seen_by_nobody(bits, most):
    batch = Batch([(1, 200), (1, 16), (40, 500), (2, 90), (1, 30)], 8, 2, 64, bits=bits)
    batch.table[0, 3], batch.table[0, 12] = -1, batch.cache.pages
    batch.table[1, 0] = -(1 << 31)
    batch.table[2, 5:9] = (1 << 31) - 1
    batch.table[2, 30] = -1
    batch.table[4] = -1
    batch.check(most)
    assert (batch.y[batch.first[4]] == 0).all() and (batch.y[batch.first[1]] == 0).all()


def within_guards(batch):
    """The batch's y between other rows, and its workspace, as many bytes as the library asks for, between other bytes.  What asks whether those are as they were."""
    room = torch.full((batch.tokens + 64, batch.heads, batch.dim), 9.0, dtype=BF, device="cuda")
    n = L.lora_attention_workspace_bytes(batch.tokens, batch.heads, batch.lengths.numel(), batch.table.shape[1], batch.cache)
    work = torch.full((4096 + n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, as sums)
    batch.y, batch.workspace = room[32:-32], work[4096:4096 + n]
    return lambda: bool((room[:32] == 9).all() and (room[-32:] == 9).all() and (work[:4096] == 0xFF).all() and (work[4096 + n:] == 0xFF).all())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page, dim", [(16, 64), (64, 128)])
def test_indices_that_fit_nothing_write_nothing_beside_the_rows_and_the_workspace(page, dim, bits):
    """starts that are negative, descend, or lie behind the rows, lengths likewise, pages that are none: y's neighbours, the workspace's and the cache stay as they are"""
    for sizes in ([(3, 50), (1, 20), (70, 90)], [(1, 4000), (1, 3), (1, 9)], [(2, 2500), (200, 3000), (5, 700)]):
        batch = Batch(sizes, 4, 2, dim, page=page, bits=bits)
        held, n = copied(batch.tensors), batch.tokens
        untouched = within_guards(batch)
        batch.table[0, ::2] = batch.cache.pages
        batch.table[2] = ints([-1, (1 << 31) - 1, 3, -(1 << 31), batch.cache.pages - 1]).repeat(batch.table.shape[1])[:batch.table.shape[1]]
        for starts, lengths in (([-5, 9, 3, 1 << 30], [1 << 30, -4, 7]), ([n + 6, 20, n, n], [50, (1 << 31) - 1, 90]), ([0, n, 0, n], [90, 90, 90]),
                                ([0, n, 0, n], [4000, -(1 << 31), 4000]), ([-(1 << 31), (1 << 31) - 1, -(1 << 31), (1 << 31) - 1], [(1 << 31) - 1] * 3)):
            batch.starts, batch.lengths = ints(starts), ints(lengths)
            for most in (0, 1, 8, 70):
                batch.run(most)
                assert untouched(), (sizes, starts, lengths, most)
        assert same(held, batch.tensors)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_writes_nothing_beside_the_cache(bits):
    """slots just outside the cache, and far from it: the memory in front of it and behind it stays as it is"""
    pages, heads, page, dim, n = 3, 2, 16, 64, 9
    room = new_cache(pages + 4, heads, page, dim, bits, seed=5)
    held, cache = copied(room), {name: t[2:-2] for name, t in room.items()}
    kv, q = normal(6, n, 2 * heads, dim), normal(7, n, 4, dim)
    y = torch.full((n + 8, 4, dim), 9.0, dtype=BF, device="cuda")
    last = pages * page
    slots = ints([-1, last, last + 1, -page, 1 << 30, -(1 << 31), (1 << 31) - 1, last + page, -2])
    positions = torch.arange(n, device="cuda", dtype=I32)
    L.lora_cache_append(kv[:, :heads], kv[:, heads:], slots, L.Cache(**cache), L.Rotary(dim), positions, q, y[4:-4])
    assert same(held, room) and (y == 9).all()
    L.lora_cache_append(kv[:, :heads], kv[:, heads:], ints([last - 1, 0, -1, last] + [-1] * 5), L.Cache(**cache), L.Rotary(dim), positions, q, y[4:-4])
    assert all(same({name: t[part] for name, t in held.items()}, {name: t[part] for name, t in room.items()}) for part in (slice(0, 2), slice(-2, None)))
    assert not same(held, room) and (y[:4] == 9).all() and (y[6:] == 9).all() and not (y[4:6] == 9).any()


def test_indices_that_fit_nothing_reach_nothing():
    batch = Batch([(3, 50), (1, 20), (70, 90)], 4, 2, 64)
    guard = [t.clone() for t in batch.tensors.values()]
    for starts, lengths in (([-5, 9, 3, 1 << 30], [1 << 30, -4, 7]), ([80, 20, 74, 74], [50, (1 << 31) - 1, 90]), ([0, 74, 0, 74], [90, 90, 90])):
        batch.starts, batch.lengths = ints(starts), ints(lengths)
        for most in (0, 1, 70):
            batch.y.fill_(9.0)
            batch.run(most)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(guard, batch.tensors.values()))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("keys", [90, 3000])
@pytest.mark.parametrize("starts", [[0, 74, 0, 74], [0, 74, 20, 74, 74], [70, 74, 0, 70], [10, 4, 60, 30, 74]])
def test_rows_that_requests_share_hold_what_one_of_them_gives_or_stay(starts, keys, bits):
    """starts that descend: every element of a row is what it was, or what one of the requests that claim the row gives it by itself"""
    requests, n = len(starts) - 1, 74
    batch = Batch([(1, keys)] * requests, 4, 2, 64, bits=bits, spare=n - requests, seed=9)
    claims = [(r, a, b) for r, (a, b) in enumerate(zip(starts, starts[1:])) if b > a]
    refs = []
    for r, a, b in claims:
        alone = Batch([(b - a, keys)], 4, 2, 64, bits=bits, seed=9)
        alone.tensors, alone.cache, alone.table, alone.first = batch.tensors, batch.cache, batch.table[r:r + 1], [0, b - a]
        alone.q = batch.q[a:b]
        refs.append((a, b, *alone.reference()))
    batch.starts, batch.lengths = ints(starts), ints([keys] * requests)
    for most in (0, 1, 8, 74):
        untouched = within_guards(batch)
        batch.y.fill_(9.0)
        y = batch.run(most).double()
        fits = y == 9
        for a, b, ref, bound in refs:
            fits[a:b] |= (y[a:b] - ref).abs() <= bound
        assert fits.all() and untouched(), most


@pytest.mark.parametrize("most", [1, 30])
def test_requests_that_share_rows_without_end(most):
    """10000 requests that each claim all of 20000 rows over 60000 keys: more steps than 32 bits count, which is found, and nothing is done"""
    batch = Batch([(1, 60000)], 4, 1, 64, page=1024)
    n, requests = 20000, 20001
    batch.q = torch.zeros(n, 4, 64, dtype=BF, device="cuda")
    batch.y = torch.full_like(batch.q, 9.0)
    batch.starts, batch.lengths = ints([0, n] * (requests // 2) + [0, n]), ints([60000] * requests)
    batch.table = batch.table.expand(requests, -1).contiguous()
    batch.workspace = torch.empty(L.lora_attention_workspace_bytes(n, 4, requests, batch.table.shape[1], batch.cache), dtype=torch.uint8, device="cuda")
    batch.run(most)
    assert (batch.y == 9).all()


def test_rows_behind_the_last_request_stay_as_they_are():
    for sizes, most in (([(1, 40), (1, 9)], 1), ([(30, 40), (5, 9)], 30), ([(100, 400)], 100)):
        batch = Batch(sizes, 8, 2, 64, spare=5)
        batch.check(most)
        assert (batch.y[-5:] == 9).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_strides(bits):
    batch = Batch([(1, 40), (30, 100), (3, 3)], 8, 2, 64, bits=bits)
    batch.check()
    ref = batch.y.clone()
    wide = torch.full((batch.tokens, 12, 80), 5.0, dtype=BF, device="cuda")
    wide[:, 2:10, 8:72] = batch.q
    out = torch.full((8, batch.tokens, 64), 5.0, dtype=BF, device="cuda").transpose(0, 1)
    table = torch.full((5, 40), -1, dtype=I32, device="cuda")
    table[:3, :batch.table.shape[1]] = batch.table
    batch.q, batch.y, batch.table = wide[:, 2:10, 8:72], out, table[:3, :batch.table.shape[1]]
    batch.run()
    assert torch.equal(batch.y, ref)
    assert (wide[:, :2] == 5).all() and (wide[:, 10:] == 5).all() and (wide[..., 72:] == 5).all()


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales_and_sharp_scores(scale):
    Batch([(1, 300), (20, 90), (150, 170)], 8, 2, 64, loud=4.0).check(scale=scale)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("power", [105, -100])
def test_large_and_small_values(power, bits):
    """as large as sums of 300 weights of up to 2^8 leave room for, and as small as weights times their scales keep their bits"""
    batch = Batch([(1, 300), (1, 17), (20, 90), (150, 170)], 8, 2, 64, bits=bits, loud=4.0, seed=12)
    if bits == 8:
        batch.tensors["v_scales"].copy_(torch.rand(batch.tensors["v_scales"].shape, generator=gen(13), device="cuda").clamp(min=0.25) * 2.0 ** power)
    else:
        batch.tensors["v"].mul_(2.0 ** power)
    for most in (0, 1, 150):
        batch.check(most)
        assert torch.isfinite(batch.y).all() and batch.y.abs().sum(dtype=torch.float64) > 0


def test_scores_of_minus_infinity_have_no_weight():
    batch = Batch([(1, 40), (20, 60), (100, 130)], 4, 2, 64)
    batch.q.fill_(1.0)
    for r, keys in ((0, range(40)), (1, range(3, 50)), (2, range(0, 64))):
        for j in keys:
            batch.tensors["k"][int(batch.table[r, j // 16]), :, j % 16, 7] = -float("inf")
    batch.check()
    batch.check(most=1)
    assert (batch.y[0] == 0).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("requests, most, top", [(700, 1, 300), (3000, 2, 40), (300, 20, 200)])
def test_many_requests(requests, most, top, bits):
    g = torch.Generator().manual_seed(requests)
    sizes = []
    for _ in range(requests):
        n = int(torch.randint(0, most + 1, (1,), generator=g))
        sizes.append((n, n + int(torch.randint(0, top, (1,), generator=g))))
    Batch(sizes, 4, 2, 64, bits=bits).check(most)


@pytest.mark.parametrize("seed", range(16))
def test_at_random(seed):
    rng = np.random.default_rng(seed)
    heads, kv_heads = [(8, 8), (32, 8), (28, 4), (9, 3), (16, 1), (64, 8)][rng.integers(6)]
    tree = bool(rng.integers(2))
    sizes = []
    for _ in range(int(rng.integers(1, 30))):
        n = int(rng.choice([0, 1, 1, 2, 7, 16, 33, 64])) if tree or rng.random() < 0.8 else int(rng.integers(65, 500))
        sizes.append((n, n + int(rng.integers(0, rng.choice([2, 100, 3000])))))
    batch = Batch(sizes, heads, kv_heads, int(rng.choice([64, 128])), page=int(rng.choice([16, 32, 64, 256])), bits=int(rng.choice([16, 8])), tree=tree, seed=seed + 50)
    batch.check(int(rng.choice([0, 1, max(n for n, _ in sizes)])))


def test_offsets_past_32_bits():
    """4.6 GB of keys, as many of values; the requests' pages at the end and the beginning"""
    page, heads, dim = 64, 8, 128
    pages = 35000
    k, v = (torch.zeros(pages, heads, page, dim, dtype=BF, device="cuda") for _ in range(2))
    cache = L.Cache(k, v)
    assert k.numel() * 2 > 1 << 32
    table = ints([[pages - 1, 0, pages - 2], [pages - 3, pages // 2 + 9, 5]])
    x = normal(7, 2 * 150, heads, dim)
    slots = torch.cat([table[r].long()[torch.arange(150, device="cuda") // page] * page + torch.arange(150, device="cuda") % page for r in range(2)]).to(I32)
    L.lora_cache_append(x, x.flip(2).contiguous(), slots, cache)
    for r in range(2):
        got = k[table[r].long()].transpose(1, 2).reshape(-1, heads, dim)[:150]
        assert torch.equal(got, x[150 * r:150 * r + 150])
    for rows in ((1, 1), (40, 90)):
        q = normal(8, sum(rows), 32, dim)
        y = torch.empty_like(q)
        work = torch.empty(L.lora_attention_workspace_bytes(q.shape[0], 32, 2, 3, cache), dtype=torch.uint8, device="cuda")
        L.lora_attention(q, ints([0, rows[0], sum(rows)]), ints([150, 150]), table, cache, y, work)
        for r in range(2):
            n, at = rows[r], sum(rows[:r])
            kk = x[150 * r:150 * r + 150].double().repeat_interleave(4, dim=1).permute(1, 0, 2)
            vv = x.flip(2)[150 * r:150 * r + 150].double().repeat_interleave(4, dim=1).permute(1, 0, 2)
            qq = q[at:at + n].double().permute(1, 0, 2)
            s = qq @ kk.transpose(1, 2).contiguous() / math.sqrt(dim)
            s = s.masked_fill(torch.arange(150, device="cuda")[None, None] > 150 - n + torch.arange(n, device="cuda")[None, :, None], -math.inf)
            w = torch.softmax(s, dim=2)
            ref, m = w @ vv, w @ vv.abs()
            d = (dim + 4) * U * (qq.abs() @ kk.abs().transpose(1, 2).contiguous()).amax(dim=2, keepdim=True) / math.sqrt(dim) * (1 + 2.0 ** -3)
            within(y[at:at + n].permute(1, 0, 2), ref, (2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * d + 2.0 ** -19 + 600 * U) * m) * (1 + 2.0 ** -6))


# ---- streams, graphs, workspaces ----------------------------------------------------------------------------
@pytest.mark.parametrize("sizes, most", [([(1, 3000)], 1), ([(1, 40), (50, 2000), (400, 600)], 400)])
def test_the_same_bits_every_time_on_another_stream_and_with_a_workspace_of_more(sizes, most):
    batch = Batch(sizes, 32, 8, 128)
    ref = batch.run(most).clone()
    for _ in range(3):
        assert torch.equal(batch.run(most), ref)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    batch.y.zero_()
    batch.workspace = torch.full((batch.workspace.numel() * 2,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    batch.run(most, stream=side)
    side.synchronize()
    assert torch.equal(batch.y, ref)


def test_a_step_in_a_graph_follows_positions_lengths_and_pages():
    """turn, append, attend, captured once with two graphs on one workspace, replayed while the requests grow; eager steps between"""
    requests, heads, kv_heads, dim, page = 6, 8, 2, 64, 16
    tensors = new_cache(80, kv_heads, page, dim, 16, seed=2)
    cache, rotary = L.Cache(**tensors), L.Rotary(dim)
    table = torch.randperm(80, generator=gen(1), device="cuda").to(I32)[:requests * 12].view(requests, 12).contiguous()
    lengths, positions, slots = ints([1, 5, 16, 31, 100, 64]), ints([0] * requests), ints([0] * requests)
    starts, q, kv = ints(list(range(requests + 1))), normal(3, requests, heads, dim), normal(4, requests, 2 * kv_heads, dim)
    turned_q, y = torch.empty_like(q), torch.empty_like(q)
    work = torch.empty(L.lora_attention_workspace_bytes(requests, heads, requests, 12, cache), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        L.lora_cache_append(kv[:, :kv_heads], kv[:, kv_heads:], slots, cache, rotary, positions, q, turned_q, stream)
        L.lora_attention(turned_q, starts, lengths, table, cache, y, work, most=1, stream=stream)

    def place(seed):
        q.copy_(normal(seed, requests, heads, dim))
        kv.copy_(normal(seed + 1, requests, 2 * kv_heads, dim))
        lengths.add_(seed % 5)
        positions.copy_(lengths - 1)
        slots.copy_(table.gather(1, (positions // page).long()[:, None])[:, 0] * page + positions % page)
    place(10)
    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step(torch.cuda.current_stream())
    for seed in range(12, 20):
        place(seed)
        held = copied(tensors)
        step()
        torch.cuda.synchronize()
        ref, after = y.clone(), copied(tensors)
        for graph in graphs:
            for n in tensors:
                tensors[n].copy_(held[n])
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, ref) and same(tensors, after) and torch.isfinite(y).all() and y.abs().sum() > 0


def test_a_prompt_in_pieces_gives_what_the_whole_prompt_gives():
    """appended and attended in one piece, and in pieces of 70, 1, 64 and 165 rows: within both sides' bounds"""
    n, heads, kv_heads, dim, page = 300, 8, 2, 64, 32
    x, q = normal(1, n, 2 * kv_heads, dim), normal(2, n, heads, dim)
    rotary, table = L.Rotary(dim), torch.randperm(10, generator=gen(1), device="cuda").to(I32)[None].contiguous()
    at = torch.arange(n, device="cuda")
    slots, positions = (table[0].long()[at // page] * page + at % page).to(I32), at.to(I32)
    results = []
    for cuts in ([0, 300], [0, 70, 71, 135, 300]):
        cache = L.Cache(**new_cache(10, kv_heads, page, dim, 16, seed=6))
        y = torch.empty_like(q)
        for a, b in zip(cuts, cuts[1:]):
            turned_q = torch.empty_like(q[a:b])
            L.lora_cache_append(x[a:b, :kv_heads], x[a:b, kv_heads:], slots[a:b].contiguous(), cache, rotary, positions[a:b].contiguous(), q[a:b], turned_q)
            work = torch.empty(max(16, L.lora_attention_workspace_bytes(b - a, heads, 1, 10, cache)), dtype=torch.uint8, device="cuda")
            L.lora_attention(turned_q, ints([0, b - a]), ints([b]), table, cache, y[a:b], work)
        results.append((y, cache))
    assert same(dict(k=results[0][1].k, v=results[0][1].v), dict(k=results[1][1].k, v=results[1][1].v))
    d = (results[0][0].double() - results[1][0].double()).abs()
    # each is off by 2^-8 |y| + 2^-8 M and a little; M is at most the largest |v|
    assert (d <= 4 * 2.0 ** -8 * x[:, kv_heads:].abs().max().double() * (1 + 2.0 ** -4)).all()


# ---- between the adapted projections ------------------------------------------------------------------------
def test_attention_between_adapted_projections():
    """All of a block's calls on one batch, a part at a time: what the projections give against 64 bits within what an 8-bit row leaves (2^-3 / sqrt(12) of the
    power of two below a value, in the mean), attention on what they gave within this file's bound, and the turned keys in the cache."""
    from paper_2511_22880_amd import expert_layer as m
    g = gen(17)
    block, adapters, weights, x, y, batch = m.attention_example(lambda *shape: torch.randn(*shape, generator=g, device="cuda"))
    cached, positions, sizes, dim = batch
    step, n = 2.0 ** -3 / 12 ** 0.5, x.shape[0]
    for i, (rows, out) in enumerate(((x, block.q), (x, block.k), (x, block.v), (block.z, y))):
        ref = adapters[i].add(rows, rows.double() @ m._values(*weights[i])[0].t())
        assert (out.double() - ref).norm() <= step * ref.norm()
    q, k, v = (t.view(n, -1, dim) for t in (block.q, block.k, block.v))
    z = m.attention_reference(q, k, v, cached, positions, sizes, dim)
    # (here the queries and keys that attention sees were rounded to bf16 after they were turned, 2^-8 each: their scores are off by twice that of scale sum |q||k|)
    group, at = block.heads // block.cache.kv_heads, 0
    got = block.z.view(n, -1, dim).double()
    for (rows, keys), (ck, cv) in zip(sizes, cached):
        part = slice(at, at + rows)
        # |q . k| <= |q||k| by element, and a turn leaves a pair's length: sum |q||k| <= 2 |q| |k| by pairs
        pairs = lambda t: (t[..., :dim // 2].double() ** 2 + t[..., dim // 2:].double() ** 2).sqrt()  # noqa: E731
        kk = torch.cat([pairs(ck), pairs(k[part])]).repeat_interleave(group, dim=1).permute(1, 0, 2)
        a = (2 * pairs(q[part]).permute(1, 0, 2) @ kk.transpose(1, 2).contiguous()).amax(dim=2).t()[..., None] / dim ** 0.5
        top = torch.cat([cv, v[part]]).abs().double().amax()
        d = (2.0 ** -7 + (dim + 4) * U) * a * (1 + 2.0 ** -3)
        bound = (2.0 ** -8 * z[part].abs() + (2.0 ** -8 + 2 * torch.expm1(d) + 2.0 ** -19 + 4 * keys * U) * top) * (1 + 2.0 ** -6)
        assert ((got[part] - z[part]).abs() <= bound).all()
        at += rows
    for a in adapters:
        a.close()
