"""The operators of include/lora_experts.h on the GPU against their definitions in 64 bits, at the sizes and values where they can go wrong.

Bounds.  A product in bf16: its terms are exact in fp32, n of them added in any order err by at most n 2^-24 of the sum M of their
magnitudes, and y's one rounding by 2^-8 of the result: (2^-8 |y| + (in + 2) 2^-24 M) (1 + 2^-7), as for the rest of this library.  In 8 bits
the matrix instruction may drop of each of a block's 128 products what lies below 2^-17 of the block's largest, 2^-10 of that in all; then come
the roundings of the scales' product, of the scaled sum and of its addition, one per block: (blocks + 3) 2^-24 M.
"""
import numpy as np
import pytest
import torch

from paper_2511_22880_amd import binding as L

pytestmark = pytest.mark.gpu
F8, BF = torch.float8_e4m3fn, torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def blocks_of(n):
    return (n + 127) // 128


def nearest8(v):
    """the nearest E4M3 value in 64 bits, ties to even"""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def quantized(x):
    """the definition of lora_rows_quantize on finite values, in 64 bits: (q, scales)"""
    rows, n = x.shape
    v = torch.nn.functional.pad(x.double(), (0, blocks_of(n) * 128 - n)).view(rows, -1, 128)
    d = v.abs().amax(dim=2).clamp(min=448 * 2.0 ** -126)
    return nearest8(v * 448 / d[:, :, None]).view(rows, -1), (d / 448).float()


def rows8(g, rows, in_f, spread=1.0):
    """rows of 8-bit values and scales, whose padding is zero"""
    x = torch.randn(rows, in_f, generator=g, device="cuda") * torch.exp(spread * torch.randn(rows, in_f, generator=g, device="cuda"))
    q, s = quantized(x.to(BF))
    return q.float().to(F8), s


def weights8(g, experts, out_f, in_f):
    w = torch.randn(experts, out_f, blocks_of(in_f) * 128, generator=g, device="cuda").clamp(-4, 4) * 100
    s = torch.rand(experts, out_f // 128, blocks_of(in_f), generator=g, device="cuda") * 1e-3 + 1e-5
    return w.to(F8), s


def packed(w, in_f=None):
    in_f = w.shape[2] if in_f is None else in_f
    p = torch.empty(L.lora_experts_packed_bytes(w.shape[0], in_f, w.shape[1], 8 * w.element_size()), dtype=torch.uint8, device="cuda")
    L.lora_experts_pack_weight(w, p, in_features=in_f)
    return p


def product16(x, w):
    """(y, bound) of rows of bf16 times W^T [out][in]"""
    x, w = x.double(), w.double()
    y, m = x @ w.t(), x.abs() @ w.abs().t()
    return y, (2.0 ** -8 * y.abs() + (x.shape[1] + 2) * 2.0 ** -24 * m) * (1 + 2.0 ** -7)


def product8(q, s, w, ws):
    """(y, bound) of rows in 8 bits times W^T"""
    y = m = off = 0.0
    for b in range(s.shape[1]):
        k = slice(128 * b, 128 * b + 128)
        a, c = q[:, k].contiguous().double(), w[:, k].contiguous().double()
        scale = s[:, b].double()[:, None] * ws[:, b].double().repeat_interleave(128)
        y = y + a @ c.t() * scale
        m = m + a.abs() @ c.abs().t() * scale.abs()
        top = torch.stack([(a[i].abs() * c.abs()).amax(dim=1) for i in range(a.shape[0])]) if a.shape[0] else a @ c.t()
        off = off + top * scale.abs() * 2.0 ** -10
    return y, (2.0 ** -8 * y.abs() + off + (s.shape[1] + 3) * 2.0 ** -24 * m) * (1 + 2.0 ** -7)


def close(y, ref, bound):
    d = (y.double() - ref).abs()
    assert torch.isfinite(y).all()
    assert (d <= bound).all(), f"{(d / bound.clamp(min=1e-300)).max().item():.3f} of the bound"


# ---- rows to 8 bits -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows, in_f", [(1, 64), (1, 128), (3, 192), (7, 4096), (57, 3008), (130, 640), (4099, 320)])
def test_quantize(rows, in_f):
    x = (torch.randn(rows, in_f, generator=gen(rows), device="cuda") * 30).to(BF)
    q = torch.empty(rows, blocks_of(in_f) * 128, dtype=F8, device="cuda")
    s = torch.empty(rows, blocks_of(in_f), device="cuda")
    L.lora_rows_quantize(x, q, s)
    rq, rs = quantized(x)
    assert torch.equal(s, rs)
    assert torch.equal(q.double(), rq)


def test_quantize_keeps_ties_and_the_ends_of_the_range():
    """every bf16 magnitude beside a largest one that makes the quotients dyadic (448 2^k) and beside others, tiny and huge ones among them"""
    mags = torch.arange(0, 0x7F80, dtype=torch.int32, device="cuda")
    for top in (448.0, 448.0 * 2.0 ** 100, 1.0, 3.0, 2.0 ** -120, 2.0 ** -133, 3.3895313892515355e38):
        top_bits = int(torch.tensor(top).to(BF).view(torch.int16))
        below = mags[mags <= top_bits]
        n = (below.numel() + 126) // 127 * 127
        v = torch.zeros(n, dtype=torch.int32, device="cuda")
        v[:below.numel()] = below
        v[1::2] |= 0x8000
        x = torch.cat([v.view(-1, 127), torch.full((n // 127, 1), top_bits, dtype=torch.int32, device="cuda")], dim=1).to(torch.int16).view(BF)
        q = torch.empty(x.shape, dtype=F8, device="cuda")
        s = torch.empty(x.shape[0], 1, device="cuda")
        L.lora_rows_quantize(x, q, s)
        rq, rs = quantized(x)
        assert torch.equal(s, rs), top
        assert torch.equal(q.double(), rq), top


def test_quantize_infinities_nan_and_zeros():
    x = torch.ones(4, 384, dtype=BF, device="cuda")
    x[0] = 0
    x[1, 5], x[1, 300] = float("inf"), -float("inf")
    x[2, 200], x[2, 201] = float("nan"), float("inf")
    q = torch.empty(4, 384, dtype=F8, device="cuda")
    s = torch.empty(4, 3, device="cuda")
    L.lora_rows_quantize(x, q, s)
    v = q.float()
    assert (v[0] == 0).all() and (s[0] == 2.0 ** -126).all()
    assert s[1].isinf().tolist() == [True, False, True] and (s[1] > 0).all()
    bad = torch.zeros(384, dtype=torch.bool, device="cuda")
    bad[5] = bad[300] = True
    assert torch.equal(v[1].isnan(), bad) and (v[1][:128].nan_to_num(0) == 0).all() and (v[1][128:256] == 448).all()
    assert s[2].isnan().tolist() == [False, True, False] and v[2][128:256].isnan().all() and (v[2][:128] == 448).all()
    assert (v[3] == 448).all()


def test_quantize_strides_and_nothing_beside_the_rows():
    x = torch.full((5, 400), float("nan"), dtype=BF, device="cuda")
    x[:, 8:328] = torch.randn(5, 320, generator=gen(3), device="cuda").to(BF)
    q = torch.full((5, 512), 7.0, device="cuda").to(F8)
    s = torch.full((5, 6), -1.0, device="cuda")
    L.lora_rows_quantize(x[:, 8:328], q[:, 64:448], s[:, 1:4])
    rq, rs = quantized(x[:, 8:328])
    assert torch.equal(q[:, 64:448].double(), rq) and torch.equal(s[:, 1:4], rs)
    assert (q[:, :64].float() == 7).all() and (q[:, 448:].float() == 7).all() and (s[:, [0, 4, 5]] == -1).all()


# ---- one layer in 8 bits ------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows, in_f, out_f", [
    (1, 64, 128), (1, 128, 128), (1, 4096, 1024), (2, 192, 256), (15, 640, 384), (16, 1024, 128), (17, 1024, 128), (33, 2048, 512), (64, 128, 640),
    (65, 320, 640), (127, 896, 256), (128, 1152, 384), (129, 4160, 128), (255, 512, 256), (256, 256, 512), (257, 384, 640), (300, 2048, 1920), (515, 192, 1408),
    (1023, 1088, 768)])
def test_linear_scaled(rows, in_f, out_f):
    g = gen(rows + in_f)
    q, s = rows8(g, rows, in_f)
    w, ws = weights8(g, 1, out_f, in_f)
    y = torch.full((rows, out_f), float("nan"), dtype=BF, device="cuda")
    L.lora_linear_scaled(q, s, packed(w, in_f), ws, y)
    if in_f % 128:
        w[:, :, in_f:] = 0.0
    close(y, *product8(q, s, w[0], ws[0]))


def test_linear_scaled_strides_and_nothing_beside_the_rows():
    g = gen(5)
    q0, s0 = rows8(g, 70, 256)
    w, ws = weights8(g, 1, 384, 256)
    q = torch.full((70, 320), 448.0, device="cuda").to(F8)
    s = torch.full((70, 5), float("nan"), device="cuda")
    q[:, 32:288], s[:, 2:4] = q0, s0
    y = torch.full((72, 512), -7.0, dtype=BF, device="cuda")
    L.lora_linear_scaled(q[:, 32:288], s[:, 2:4], packed(w), ws, y[1:71, 64:448])
    close(y[1:71, 64:448], *product8(q0, s0, w[0], ws[0]))
    y[1:71, 64:448] = -7.0
    assert (y == -7).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_linear_scaled_what_a_row_holds_stays_in_it(rows):
    g = gen(6)
    q, s = rows8(g, rows, 384)
    w, ws = weights8(g, 1, 256, 384)
    ws[0, 1, 2] = 0.0
    p, y = packed(w), torch.empty(rows, 256, dtype=BF, device="cuda")
    L.lora_linear_scaled(q, s, p, ws, y)
    hurt, z = s.clone(), torch.empty_like(y)
    hurt[1, 2], hurt[2, 0] = float("inf"), float("nan")
    L.lora_linear_scaled(q, hurt, p, ws, z)
    assert torch.equal(z[0], y[0]) and torch.equal(z[3:], y[3:])
    assert z[2].isnan().all() and not z[1, :128].isfinite().any() and z[1, 128:].isnan().all()  # infinity times zero


def test_linear_scaled_offsets_past_32_bits():
    g = gen(8)
    rows = 4200
    q0, s = rows8(g, 3, 256)
    w, ws = weights8(g, 1, 128, 256)
    q = torch.empty(rows, 1 << 20, dtype=torch.uint8, device="cuda")[:, :256]
    y = torch.empty(rows, 1 << 19, dtype=BF, device="cuda")[:, :128]
    q.view(torch.uint8).copy_(q0[:1].view(torch.uint8).expand(rows, -1))
    q[rows - 2:] = q0[1:].view(torch.uint8)
    scales = s[:1].expand(rows, -1).contiguous()
    scales[rows - 2:] = s[1:]
    L.lora_linear_scaled(q, scales, packed(w), ws, y)
    ref, bound = product8(q0, s, w[0], ws[0])
    at = torch.cat([torch.zeros(rows - 2, dtype=torch.long), torch.tensor([1, 2])]).cuda()
    close(y, ref[at], bound[at])


# ---- picks by expert ----------------------------------------------------------------------------------------
def grouped(ids, experts):
    flat = ids.cpu().numpy().reshape(-1)
    ok = (flat >= 0) & (flat < experts)
    at = np.flatnonzero(ok)
    order = at[np.argsort(flat[at], kind="stable")].astype(np.int32)
    place = np.full(flat.size, -1, dtype=np.int32)
    place[order] = np.arange(order.size)
    starts = np.concatenate([[0], np.cumsum(np.bincount(flat[at], minlength=experts))]).astype(np.int32)
    return starts, np.concatenate([order, np.full(flat.size - order.size, -1, dtype=np.int32)]), place


def group(ids, experts):
    n = ids.numel()
    st, od, pl = (torch.full((k,), 77, dtype=torch.int32, device="cuda") for k in (experts + 1, n, n))
    need = L.lora_experts_group_workspace_bytes(n, experts)
    ws = torch.randint(0, 255, (need,), dtype=torch.uint8, device="cuda") if need else None
    L.lora_experts_group(ids, st, od, pl, ws)
    return st, od, pl


@pytest.mark.parametrize("tokens, picks, experts", [
    (0, 1, 4), (1, 1, 1), (1, 8, 8), (3, 2, 512), (63, 1, 5), (64, 8, 128), (255, 8, 64), (256, 8, 256), (257, 8, 255), (2049, 1, 7), (3000, 6, 512),
    (19675, 8, 256), (70001, 8, 33), (100, 64, 200), (1024, 1, 100), (1025, 1, 100), (511, 4, 9), (2047, 2, 64), (4097, 1, 12), (8191, 1, 511), (8192, 1, 60), (8193, 1, 60),
    (90000, 6, 17), (140001, 8, 130), (262144, 9, 40)])
@pytest.mark.parametrize("kind", ["any", "one", "none", "wild"])
def test_group(tokens, picks, experts, kind):
    g = gen(tokens + experts)
    ids = torch.randint(0, experts, (tokens, picks), generator=g, device="cuda", dtype=torch.int32)
    if kind == "one":
        ids.fill_(experts - 1)
    elif kind == "none":
        ids.fill_(-1)
    elif kind == "wild":  # ids of no expert here
        far = torch.randint(-2 ** 31, 2 ** 31 - 1, (tokens, picks), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        ids = torch.where(torch.rand(tokens, picks, generator=g, device="cuda") < 0.3, far, ids)
        ids = torch.where(torch.rand(tokens, picks, generator=g, device="cuda") < 0.1, experts, ids)
    got = group(ids, experts)
    for a, b in zip(got, grouped(ids, experts)):
        assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("n, experts", [(1025, 3), (3000, 512), (8191, 8), (8192, 300)])
def test_group_of_picks_that_are_mostly_one_experts(n, experts):
    g = gen(n)
    ids = torch.randint(-1, experts, (n, 1), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.where(torch.rand(n, 1, generator=g, device="cuda") < 0.8, experts // 2, ids)
    for a, b in zip(group(ids, experts), grouped(ids, experts)):
        assert np.array_equal(a.cpu().numpy(), b)


def test_group_reads_rows_of_any_stride():
    ids = torch.randint(0, 9, (300, 12), generator=gen(1), device="cuda", dtype=torch.int32)
    for a, b in zip(group(ids[:, 3:7], 9), grouped(ids[:, 3:7], 9)):
        assert np.array_equal(a.cpu().numpy(), b)


# ---- rows times their expert's weights ----------------------------------------------------------------------
def ids_of(sizes, picks, idle, g):
    """[tokens][picks] ids that give expert e sizes[e] rows, in random order, filled up with picks of no expert"""
    flat = torch.cat([torch.full((n,), e, dtype=torch.int32) for e, n in enumerate(sizes)] + [torch.full((idle,), -1, dtype=torch.int32)])
    flat = torch.cat([flat, torch.full((-flat.numel() % picks,), -1, dtype=torch.int32)]).cuda()
    return flat[torch.randperm(flat.numel(), generator=g, device="cuda")].view(-1, picks)


def run_experts(sizes, picks, in_f, out_f, bits, idle=0, ordered=True, seed=0):
    g = gen(seed + in_f + out_f)
    ids = ids_of(sizes, picks, idle, g)
    tokens, experts = ids.shape[0], len(sizes)
    starts, order, _ = group(ids, experts)
    n, rows = int(starts[-1]), ids.numel()
    if not ordered:
        order, tokens, picks = None, rows, 1
    y = torch.full((rows, out_f), -7.0, dtype=BF, device="cuda")
    at = order[:n].long() // picks if ordered else torch.arange(n, device="cuda")
    if bits == 16:
        x = torch.randn(tokens, in_f, generator=g, device="cuda").to(BF)
        w = (torch.randn(experts, out_f, in_f, generator=g, device="cuda") * 0.05).to(BF)
        L.lora_experts_linear(x, starts, order, picks, packed(w), y)
        one = lambda t, e: product16(x[t], w[e])  # noqa: E731
    else:
        q, s = rows8(g, tokens, in_f)
        w, ws = weights8(g, experts, out_f, in_f)
        L.lora_experts_linear_scaled(q, s, starts, order, picks, packed(w, in_f), ws, y)
        if in_f % 128:
            w[:, :, in_f:] = 0.0
        one = lambda t, e: product8(q.view(torch.uint8)[t].view(F8), s[t], w[e], ws[e])  # noqa: E731
    for e in range(experts):
        a, b = int(starts[e]), int(starts[e + 1])
        if b > a:
            close(y[a:b], *one(at[a:b], e))
    assert (y[n:] == -7).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sizes, picks, in_f, out_f, idle", [
    ([1], 1, 64, 128, 0),
    ([0, 1, 0, 2, 0], 1, 192, 256, 0),
    ([0, 0, 0], 2, 128, 128, 6),                                 # nobody is here
    ([3, 1, 16, 17, 15, 0, 31, 32, 33], 4, 320, 384, 5),
    ([1] * 70 + [0] * 60 + [9], 8, 256, 128, 30),                # more experts than a wavefront has lanes
    ([2] * 512, 8, 128, 128, 0),
    ([63, 64, 65, 0, 127, 128, 129, 1], 2, 448, 256, 10),
    ([255, 0, 256, 257, 1, 300], 1, 640, 640, 0),
    ([1200, 0, 3, 40], 2, 576, 384, 100),                        # one expert has nearly all
    ([900, 700, 512, 513], 2, 1088, 896, 0),
    ([5, 0, 2100], 1, 4096, 256, 7),
])
def test_experts(sizes, picks, in_f, out_f, idle, bits):
    run_experts(sizes, picks, in_f, out_f, bits, idle)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sizes, in_f, out_f", [
    ([65, 128, 90, 1] * 12, 64, 1792),                           # as many tiles of up to 128 rows as give each four strips of columns,
    ([65, 128, 90, 127] * 10, 192, 1920),                        # the last of them two or three
    ([100] * 36 + [0, 20, 64], 448, 2048),
    ([300] * 30 + [90] * 10, 704, 1024),                         # beside whole ones
    ([77, 128, 64, 100] * 10, 2048, 1792),                       # weights that are read past the caches
    ([200] * 15, 320, 2048),                                     # whole tiles cut in two, all of them
    ([256, 129, 255, 200] * 9 + [60] * 10, 192, 2048),           # .. those of the second round, beside some of few rows
    ([2500], 448, 7680),
])
def test_experts_with_many_tiles_of_few_rows(sizes, in_f, out_f, bits):
    run_experts(sizes, 2, in_f, out_f, bits, idle=3)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sizes", [[7, 0, 30], [400, 3, 0, 290]])
def test_experts_rows_in_expert_order(sizes, bits):
    run_experts(sizes, 1, 384, 256, bits, idle=9, ordered=False)


@pytest.mark.parametrize("seed", range(12))
def test_experts_at_random(seed):
    r = np.random.default_rng(seed)
    experts = int(r.integers(1, 40))
    sizes = [int(v) for v in np.exp(r.uniform(0, np.log(r.choice([4, 40, 600])), experts)) * (r.random(experts) > 0.2)]
    run_experts(sizes, int(r.integers(1, 9)), 64 * int(r.integers(1, 24)), 128 * int(r.integers(1, 8)), int(r.choice([8, 16])), int(r.integers(0, 40)), seed=seed)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rows", [40, 700])
def test_experts_indices_that_fit_nothing_reach_nothing(rows, bits):
    """starts beyond the rows, decreasing or negative ones, order entries of no token: rows that are meant are right, the others left alone"""
    g = gen(rows)
    x = torch.randn(rows, 256, generator=g, device="cuda").to(BF)
    w = (torch.randn(3, 256, 256, generator=g, device="cuda") * 0.05).to(BF)
    if bits == 8:
        q, s = rows8(g, rows, 256)
        w, ws = weights8(g, 3, 256, 256)
    p = packed(w)
    order = torch.arange(rows, dtype=torch.int32, device="cuda")
    order[3], order[5], order[7] = -1, rows, 2 ** 31 - 1
    whole = torch.full((rows + 2, 256), -7.0, dtype=BF, device="cuda")
    y = whole[1:-1]
    for st, meant in (([0, 20, 10, rows + 1000], [(0, 20, 0), (10, rows, 2)]), ([-5, 4, 2 ** 31 - 1, 2 ** 31 - 1], [(0, 4, 0), (4, rows, 1)]),
                      ([rows, 0, 0, 9], [(0, 9, 2)])):
        whole.fill_(-7.0)
        starts = torch.tensor(st, dtype=torch.int32, device="cuda")
        if bits == 16:
            L.lora_experts_linear(x, starts, order, 1, p, y)
        else:
            L.lora_experts_linear_scaled(q, s, starts, order, 1, p, ws, y)
        touched = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for a, b, e in meant:
            rows_of = torch.tensor([r for r in range(a, b) if r not in (3, 5, 7)], device="cuda")
            touched[rows_of] = True
            if not any(c < b and a < d for c, d, f in meant if f != e):  # (places that two experts claim hold either's)
                close(y[rows_of], *(product16(x[rows_of], w[e]) if bits == 16 else product8(q.view(torch.uint8)[rows_of].view(F8), s[rows_of], w[e], ws[e])))
        assert (y[~touched] == -7).all() and (whole[0] == -7).all() and (whole[-1] == -7).all()


@pytest.mark.parametrize("rows", [5, 300])
def test_experts_weights_past_32_bits(rows):
    """the last of many experts: its weights lie beyond byte 2^32"""
    g = gen(11)
    experts, in_f, out_f = 300, 2048, 4096
    each = in_f * out_f * 2
    p = torch.empty(experts * each, dtype=torch.uint8, device="cuda")
    w = (torch.randn(1, out_f, in_f, generator=g, device="cuda") * 0.05).to(BF)
    L.lora_experts_pack_weight(w, p[-each:])
    x = torch.randn(rows, in_f, generator=g, device="cuda").to(BF)
    starts = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    starts[-1] = rows
    y = torch.empty(rows, out_f, dtype=BF, device="cuda")
    L.lora_experts_linear(x, starts, None, 1, p, y)
    close(y, *product16(x, w[0]))


@pytest.mark.parametrize("bits, rows", [(16, 12), (8, 12), (16, 600), (8, 600)])
def test_the_same_bits_every_time_and_for_a_row_in_any_company(bits, rows):
    """sums are taken in an order of their own for every row: neither repetition nor the row's place in its tile shows"""
    g = gen(21)
    w = (torch.randn(2, 256, 1024, generator=g, device="cuda") * 0.05).to(BF)
    ws = None
    x = torch.randn(rows, 1024, generator=g, device="cuda").to(BF)
    if bits == 8:
        q, s = rows8(g, rows, 1024)
        w, ws = weights8(g, 2, 256, 1024)
    p = packed(w)

    def run(perm):
        starts = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
        y = torch.empty(rows, 256, dtype=BF, device="cuda")
        if bits == 16:
            L.lora_experts_linear(x, starts, perm.to(torch.int32), 1, p, y)
        else:
            L.lora_experts_linear_scaled(q, s, starts, perm.to(torch.int32), 1, p, ws, y)
        return y
    same = torch.arange(rows, device="cuda")
    first = run(same)
    for _ in range(3):
        assert torch.equal(run(same), first)
    half = rows // 2
    perm = torch.cat([torch.randperm(half, generator=g, device="cuda"), half + torch.randperm(rows - half, generator=g, device="cuda")])
    assert torch.equal(run(perm), first[perm])


# ---- a token's rows together --------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens, picks, out_f, n_rows", [(1, 1, 128, 1), (3, 2, 384, 9), (64, 8, 2048, 512), (57, 6, 640, 100), (5, 64, 128, 400), (1000, 3, 256, 3000)])
def test_combine(tokens, picks, out_f, n_rows):
    g = gen(tokens)
    y = torch.randn(n_rows + 1, out_f, generator=g, device="cuda").to(BF)[:-1]
    place = torch.randint(0, n_rows, (tokens, picks), generator=g, device="cuda", dtype=torch.int32)
    gone = torch.rand(tokens, picks, generator=g, device="cuda") < 0.3
    gone[0] = True  # a token without any
    gone[-1] = tokens == 1
    place[gone] = torch.tensor([-1, n_rows, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")[torch.arange(int(gone.sum()), device="cuda") % 4]
    weights = torch.randn(tokens, picks, generator=g, device="cuda")
    weights[gone] = float("nan")
    z = torch.full((tokens, out_f), float("nan"), dtype=BF, device="cuda")
    L.lora_experts_combine(y, place, weights, z)
    rows = y.double()[place.long().clamp(0, n_rows - 1)] * torch.where(gone, 0.0, weights.double())[:, :, None].nan_to_num(0)
    rows = torch.where(gone[:, :, None], 0.0, rows)
    ref, m = rows.sum(dim=1), rows.abs().sum(dim=1)
    close(z, ref, (2.0 ** -8 * ref.abs() + (picks + 1) * 2.0 ** -24 * m) * (1 + 2.0 ** -7))
    assert (z[0] == 0).all()


def test_combine_reads_no_row_that_is_left_out():
    y = torch.full((4, 128), float("nan"), dtype=BF, device="cuda")
    y[2] = 3.0
    place = torch.tensor([[2, -1], [-1, 2], [4, 2]], dtype=torch.int32, device="cuda")
    z = torch.full((4, 256), -7.0, dtype=BF, device="cuda")
    L.lora_experts_combine(y, place, torch.full((3, 2), 0.5, device="cuda"), z[:3, 64:192])
    assert (z[:3, 64:192] == 1.5).all()
    z[:3, 64:192] = -7.0
    assert (z == -7).all()


# ---- streams and graphs -------------------------------------------------------------------------------------
class Layer:
    """A layer of experts in 8 bits, all of its steps."""

    def __init__(self, tokens, experts, picks, in_f, out_f, seed=1):
        g = gen(seed)
        self.picks = picks
        w, self.ws = weights8(g, experts, out_f, in_f)
        self.p = packed(w)
        n = tokens * picks
        e = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.x, self.ids = e(tokens, in_f, dtype=BF), e(tokens, picks, dtype=torch.int32)
        self.weights = torch.rand(tokens, picks, generator=g, device="cuda")
        self.q, self.s = e(tokens, in_f, dtype=F8), e(tokens, in_f // 128)
        self.st, self.od, self.pl = e(experts + 1, dtype=torch.int32), e(n, dtype=torch.int32), e(n, dtype=torch.int32)
        self.work = e(max(16, L.lora_experts_group_workspace_bytes(n, experts)), dtype=torch.uint8)
        self.y, self.z = e(n, out_f, dtype=BF), e(tokens, out_f, dtype=BF)
        self.experts = experts

    def fill(self, seed):
        self.x.copy_(torch.randn(self.x.shape, generator=gen(seed), device="cuda"))
        self.ids.copy_(torch.randint(-1, self.experts, self.ids.shape, generator=gen(seed + 1), device="cuda", dtype=torch.int32))

    def run(self, stream=None):
        L.lora_rows_quantize(self.x, self.q, self.s, stream)
        L.lora_experts_group(self.ids, self.st, self.od, self.pl, self.work, stream)
        L.lora_experts_linear_scaled(self.q, self.s, self.st, self.od, self.picks, self.p, self.ws, self.y, stream)
        L.lora_experts_combine(self.y, self.pl, self.weights, self.z, stream)


@pytest.mark.parametrize("tokens", [5, 700])
def test_on_another_stream(tokens):
    layer = Layer(tokens, 12, 4, 512, 384)
    layer.fill(3)
    layer.run()
    ref = layer.z.clone()
    layer.z.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    layer.run(side)
    side.synchronize()
    assert torch.equal(layer.z, ref)


@pytest.mark.parametrize("tokens", [5, 700])
def test_in_a_graph(tokens):
    """captured once, replayed on other tokens and other picks: the launches depend on the sizes alone"""
    layer = Layer(tokens, 12, 4, 512, 384)
    layer.fill(3)
    layer.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(torch.cuda.current_stream())
    for seed in range(4):
        layer.fill(10 + seed)
        layer.z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = layer.z.clone()
        layer.run()
        torch.cuda.synchronize()
        assert torch.equal(got, layer.z) and got.abs().sum() > 0


# ---- the block of expert_layer.py ---------------------------------------------------------------------------
def test_adapted_projection_and_layer_of_experts_together(capsys):
    """Every step of both paths on 200 tokens.  What an 8-bit quantiser with a scale per 128 leaves of a normal value, 2^-4 / sqrt(12) of it or less in
    the mean (half of a step of 2^-3 of the power of two below, uniform), is what separates them from 64 bits: once in the projection, twice in the
    experts, whose product of two such rows counts it once more."""
    from paper_2511_22880_amd import expert_layer
    expert_layer.main()
    errors = [float(line.rsplit(" ", 1)[1]) for line in capsys.readouterr().out.splitlines() if "relative error" in line]
    step = 2.0 ** -3 / 12 ** 0.5  # rms of a rounding to 4 bits, of the value at worst
    assert len(errors) == 2 and errors[0] < step and errors[1] < 2 * step


def test_layer_of_experts_on_fewer_tokens_than_it_has_room_for():
    from paper_2511_22880_amd import expert_layer as m
    g = gen(31)
    gate_up, gs = m.weights_to_8_bits(torch.randn(6, 512, 256, generator=g, device="cuda") * 0.05)
    down, ds = m.weights_to_8_bits(torch.randn(6, 256, 256, generator=g, device="cuda") * 0.05)
    layer = m.ExpertLayer(m.Packed(gate_up, gs), m.Packed(down, ds), 2, 64)
    whole = []
    for tokens in (64, 1, 17):
        x = torch.randn(64, 256, generator=gen(5), device="cuda").to(BF)[:tokens]
        ids = torch.randint(-1, 6, (64, 2), generator=gen(6), device="cuda", dtype=torch.int32)[:tokens]
        w = torch.rand(64, 2, generator=gen(7), device="cuda")[:tokens]
        z = torch.empty(tokens, 256, dtype=BF, device="cuda")
        layer(x, ids, w, z)
        ref = m.reference(x, ids, w, m._values(gate_up, gs), m._values(down, ds))
        assert (z.double() - ref).norm() <= 2 * 2.0 ** -3 / 12 ** 0.5 * ref.norm()
        whole.append(z)
    assert torch.isfinite(whole[2]).all() and torch.isfinite(whole[1]).all()


# ---- scales at the ends of their range ----------------------------------------------------------------------
@pytest.mark.parametrize("rows, in_f, out_f", [(3, 512, 256), (300, 256, 2048), (515, 256, 1408), (2200, 256, 4096)])
@pytest.mark.parametrize("x_power, w_power, small", [
    (-126, -10, False), (-126, -19, False), (-100, -45, False), (-73, -73, False), (-20, -126, False),  # scales whose product has few bits left
    (119, 12, True), (12, 119, True),                                                                   # .. or does not fit
    (119, -126, False), (-126, 119, False), (0, 0, False),
])
def test_linear_scaled_where_the_scales_product_is_no_normal_number(rows, in_f, out_f, x_power, w_power, small):
    """y is one: a block's sum lies 2^23 above the scales' product, or 2^-11.  A scale times 1/2 to 1, at 2^-126, has one bit less, so one more
    rounding's worth: still (blocks + 3) 2^-24 in all."""
    g = gen(rows - x_power)
    blocks = in_f // 128
    draw = (lambda *s: torch.randint(1, 4, s, generator=g, device="cuda") * 2.0 ** -9) if small else (  # noqa: E731
        lambda *s: torch.randint(8, 15, s, generator=g, device="cuda") * 32.0)
    q, w = draw(rows, in_f).to(F8), draw(1, out_f, in_f).to(F8)
    scales = lambda power, *s: (torch.rand(*s, generator=g, device="cuda") * 0.9 + 1) * 2.0 ** power  # noqa: E731
    s, ws = scales(x_power, rows, blocks), scales(w_power, 1, out_f // 128, blocks)
    y = torch.full((rows, out_f), float("nan"), dtype=BF, device="cuda")
    L.lora_linear_scaled(q, s, packed(w), ws, y)
    close(y, *product8(q, s, w[0], ws[0]))


@pytest.mark.parametrize("rows", [1, 5])
def test_linear_scaled_on_the_columns_that_are_there_of_rows_of_whole_blocks(rows):
    g = gen(rows)
    q, s = rows8(g, rows, 192)
    w, ws = weights8(g, 1, 128, 192)
    y = torch.empty(rows, 128, dtype=BF, device="cuda")
    L.lora_linear_scaled(q[:, :192], s, packed(w, 192), ws, y)
    w[:, :, 192:] = 0.0
    close(y, *product8(q, s, w[0], ws[0]))


@pytest.mark.parametrize("tokens, room", [(65000, 66000), (131000, 140000), (262143, 262145)])
def test_group_with_the_workspace_of_more_picks(tokens, room):
    """what a program that makes its buffers once, for the most tokens it takes, has at hand"""
    ids = torch.randint(-1, 256, (tokens, 8), generator=gen(tokens), device="cuda", dtype=torch.int32)
    n = ids.numel()
    st, od, pl = (torch.empty(k, dtype=torch.int32, device="cuda") for k in (257, n, n))
    L.lora_experts_group(ids, st, od, pl, torch.empty(L.lora_experts_group_workspace_bytes(room * 8, 256), dtype=torch.uint8, device="cuda"))
    for a, b in zip((st, od, pl), grouped(ids, 256)):
        assert np.array_equal(a.cpu().numpy(), b)


def test_quantize_more_rows_than_a_launch_takes():
    """2^28 + 4099 blocks of 128: 64 GiB of x, in repetitions of 4096 rows, and other rows behind them"""
    torch.cuda.empty_cache()
    pattern = (torch.randn(4096, 128, generator=gen(1), device="cuda") * 30).to(BF)
    rest = (torch.randn(4099, 128, generator=gen(2), device="cuda") * 3).to(BF)
    n = 1 << 28
    x = torch.empty(n + 4099, 128, dtype=BF, device="cuda")
    x[:n].view(-1, 4096, 128).copy_(pattern)
    x[n:] = rest
    q = torch.empty(x.shape, dtype=torch.uint8, device="cuda")
    s = torch.empty(x.shape[0], 1, device="cuda")
    L.lora_rows_quantize(x, q, s)
    del x
    rq, rs = quantized(pattern)
    rq = rq.float().to(F8).view(torch.uint8)
    for a in range(0, n, 1 << 24):
        assert (q[a:a + (1 << 24)].view(-1, 4096, 128) == rq).all() and (s[a:a + (1 << 24)].view(-1, 4096, 1) == rs).all(), a
    rq, rs = quantized(rest)
    assert torch.equal(q[n:].view(F8).double(), rq) and torch.equal(s[n:], rs)
    del q, s
    torch.cuda.empty_cache()


def test_a_step_of_the_layer_of_experts_allocates_nothing():
    from paper_2511_22880_amd import expert_layer as m
    g = gen(32)
    layer = m.ExpertLayer(m.Packed(*m.weights_to_8_bits(torch.randn(4, 512, 256, generator=g, device="cuda") * 0.05)),
                          m.Packed(*m.weights_to_8_bits(torch.randn(4, 256, 256, generator=g, device="cuda") * 0.05)), 2, 50)
    x, z = torch.randn(50, 256, generator=g, device="cuda").to(BF), torch.empty(50, 256, dtype=BF, device="cuda")
    ids, w = torch.randint(-1, 4, (50, 2), generator=g, device="cuda", dtype=torch.int32), torch.rand(50, 2, generator=g, device="cuda")
    for tokens in (50, 33):
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        layer(x[:tokens], ids[:tokens], w[:tokens], z[:tokens])
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
        h = layer.h[:int(layer.starts[-1])].float()  # the same numbers as out of place
        assert torch.equal(layer.act[:h.shape[0]], (torch.nn.functional.silu(h[:, :256]) * h[:, 256:]).to(BF))
