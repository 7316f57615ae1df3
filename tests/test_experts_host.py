"""include/lora_experts.h without a GPU: what the calls refuse, before the device is touched, and the sizes they state."""
import ctypes

import pytest
import torch

from paper_2511_22880_amd import binding as L

P = 0x7F0000000000  # a 256-byte aligned address that is never dereferenced


def status(name, *args):
    return L.STATUS[getattr(L.lib(), name)(*args)]


QUANTIZE = dict(x=P, ldx=256, rows=3, in_f=256, q=P, ldq=256, scales=P, lds=2)
LINEAR = dict(q=P, ldq=256, scales=P, lds=2, rows=3, in_f=256, w=P, ws=P, out=128, y=P, ldy=128)
GROUP = dict(ids=P, ld=2, tokens=5, picks=2, experts=8, starts=P, order=P, place=P, work=None, nwork=0)
EXPERTS = dict(x=P, ldx=256, tokens=5, starts=P, order=P, picks=2, rows=10, experts=8, in_f=256, w=P, out=128, y=P, ldy=128)
SCALED = dict(q=P, ldq=256, scales=P, lds=2, tokens=5, starts=P, order=P, picks=2, rows=10, experts=8, in_f=256, w=P, ws=P, out=128, y=P, ldy=128)
COMBINE = dict(y=P, ldy=128, rows=10, place=P, weights=P, tokens=5, picks=2, out=128, z=P, ldz=128)
PACK = dict(w=P, experts=2, in_f=256, out=128, bits=8, packed=P, n=2 * 128 * 256)

CASES = [("lora_rows_quantize", QUANTIZE, c, s) for c, s in [
    (dict(x=None), "INVALID_ARG"), (dict(x=P + 8), "INVALID_ARG"), (dict(ldx=248), "INVALID_ARG"), (dict(ldx=260), "INVALID_ARG"),
    (dict(rows=-1), "INVALID_ARG"), (dict(in_f=0), "SHAPE"), (dict(in_f=96), "SHAPE"), (dict(q=None), "INVALID_ARG"), (dict(q=P + 4), "INVALID_ARG"),
    (dict(ldq=240), "INVALID_ARG"), (dict(ldq=264), "INVALID_ARG"), (dict(scales=None), "INVALID_ARG"), (dict(scales=P + 2), "INVALID_ARG"),
    (dict(lds=1), "INVALID_ARG"), (dict(in_f=192, ldx=192, ldq=192), "INVALID_ARG")]]
CASES += [("lora_linear_scaled", LINEAR, c, s) for c, s in [
    (dict(q=None), "INVALID_ARG"), (dict(ldq=128), "INVALID_ARG"), (dict(scales=None), "INVALID_ARG"), (dict(lds=1), "INVALID_ARG"),
    (dict(rows=-1), "INVALID_ARG"), (dict(in_f=100), "SHAPE"), (dict(out=192), "SHAPE"), (dict(out=0), "SHAPE"), (dict(w=None), "INVALID_ARG"),
    (dict(w=P + 128), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"), (dict(y=None), "INVALID_ARG"), (dict(ldy=120), "INVALID_ARG"),
    (dict(ldy=132), "INVALID_ARG"), (dict(y=P + 8), "INVALID_ARG"), (dict(ldq=1 << 62), "INVALID_ARG")]]
CASES += [("lora_experts_group", GROUP, c, s) for c, s in [
    (dict(ids=None), "INVALID_ARG"), (dict(ld=1), "INVALID_ARG"), (dict(tokens=-1), "INVALID_ARG"), (dict(picks=0), "SHAPE"), (dict(picks=65), "SHAPE"),
    (dict(tokens=1 << 30, picks=2), "SHAPE"), (dict(experts=0), "SHAPE"), (dict(experts=513), "SHAPE"), (dict(starts=None), "INVALID_ARG"),
    (dict(order=None), "INVALID_ARG"), (dict(place=None), "INVALID_ARG"), (dict(tokens=5000), "WORKSPACE"),
    (dict(tokens=5000, work=P, nwork=8), "WORKSPACE"), (dict(tokens=5000, work=P + 4, nwork=1 << 20), "WORKSPACE")]]
for name, base in (("lora_experts_linear", EXPERTS), ("lora_experts_linear_scaled", SCALED)):
    CASES += [(name, base, c, s) for c, s in [
        ({next(iter(base)): None}, "INVALID_ARG"), (dict(starts=None), "INVALID_ARG"), (dict(starts=P + 1), "INVALID_ARG"),
        (dict(order=P + 2), "INVALID_ARG"), (dict(rows=9), "INVALID_ARG"), (dict(order=None), "INVALID_ARG"), (dict(picks=0), "SHAPE"),
        (dict(experts=0), "SHAPE"), (dict(experts=600), "SHAPE"), (dict(tokens=-5, rows=-10), "INVALID_ARG"), (dict(w=P + 16), "INVALID_ARG"),
        (dict(out=100), "SHAPE"), (dict(in_f=32), "SHAPE"), (dict(y=None), "INVALID_ARG"), (dict(ldy=64), "INVALID_ARG")]]
CASES += [("lora_experts_linear_scaled", SCALED, c, s) for c, s in [
    (dict(scales=None), "INVALID_ARG"), (dict(lds=1), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"), (dict(ldq=264), "INVALID_ARG")]]
CASES += [("lora_experts_combine", COMBINE, c, s) for c, s in [
    (dict(y=None), "INVALID_ARG"), (dict(ldy=64), "INVALID_ARG"), (dict(rows=-1), "INVALID_ARG"), (dict(place=None), "INVALID_ARG"),
    (dict(weights=None), "INVALID_ARG"), (dict(tokens=-1), "INVALID_ARG"), (dict(picks=0), "SHAPE"), (dict(out=64), "SHAPE"),
    (dict(z=None), "INVALID_ARG"), (dict(z=P + 2), "INVALID_ARG"), (dict(ldz=100), "INVALID_ARG")]]
CASES += [("lora_experts_pack_weight", PACK, c, s) for c, s in [
    (dict(w=None), "INVALID_ARG"), (dict(w=P + 4), "INVALID_ARG"), (dict(experts=0), "SHAPE"), (dict(bits=4), "INVALID_ARG"), (dict(in_f=63), "SHAPE"),
    (dict(out=130), "SHAPE"), (dict(packed=None), "INVALID_ARG"), (dict(packed=P + 64), "INVALID_ARG"), (dict(n=100), "OOM")]]


@pytest.mark.parametrize("name, base, change", [
    ("lora_rows_quantize", QUANTIZE, dict(in_f=1 << 30, ldx=1 << 30, ldq=1 << 30, lds=1 << 23)),
    ("lora_experts_pack_weight", PACK, dict(experts=512, in_f=(1 << 31) - 64, out=(1 << 31) - 128)),  # (bytes that are few in 64 bits)
    ("lora_experts_pack_weight", PACK, dict(experts=1, in_f=(1 << 30) + 64, bits=16, n=1 << 62)),
    ("lora_experts_linear", EXPERTS, dict(out=(1 << 24) + 128, ldy=1 << 25)),
    ("lora_linear_scaled", LINEAR, dict(in_f=1 << 25, ldq=1 << 25, lds=1 << 18)),
    ("lora_experts_combine", COMBINE, dict(out=1 << 25, ldy=1 << 25, ldz=1 << 25)),
])
def test_features_whose_bytes_would_not_fit_are_refused(name, base, change):
    assert status(name, *dict(base, **change).values(), None) == "LORA_ERR_SHAPE"


@pytest.mark.parametrize("name, base, change, expected", CASES, ids=lambda v: str(v) if isinstance(v, str) else "")
def test_refusals(name, base, change, expected):
    assert status(name, *dict(base, **change).values(), None) == "LORA_ERR_" + expected
    assert len(L.lora_last_error()) > 5


@pytest.mark.parametrize("name, base, change", [
    ("lora_rows_quantize", QUANTIZE, dict(rows=0, x=None, q=None, scales=None)),
    ("lora_linear_scaled", LINEAR, dict(rows=0, q=None, y=None)),
    ("lora_experts_linear", EXPERTS, dict(tokens=0, rows=0, x=None, y=None)),
    ("lora_experts_linear_scaled", SCALED, dict(tokens=0, rows=0, q=None, order=None)),
    ("lora_experts_combine", COMBINE, dict(tokens=0, y=None, z=None)),
])
def test_nothing_to_do_is_no_error(name, base, change):
    assert status(name, *dict(base, **change).values(), None) == "LORA_OK"


def test_sizes():
    assert L.lora_experts_packed_bytes(1, 4096, 4096, 8) == 4096 * 4096
    assert L.lora_experts_packed_bytes(3, 192, 256, 8) == 3 * 256 * 256  # 8-bit rows are filled up to whole blocks of 128
    assert L.lora_experts_packed_bytes(3, 192, 256, 16) == 3 * 192 * 256 * 2
    assert L.lora_experts_packed_bytes(512, 16384, 16384, 16) == 512 << 29  # past 32 bits
    assert L.lora_experts_group_workspace_bytes(0, 8) == 0
    assert L.lora_experts_group_workspace_bytes(8192, 512) == 0
    assert L.lora_experts_group_workspace_bytes(8193, 512) == 5 * 512 * 4
    assert L.lora_experts_group_workspace_bytes(2 ** 31 - 1, 512) <= 256 * 512 * 4
    for args in ((-1, 8), (2 ** 31, 8), (5, 0), (5, 513)):
        with pytest.raises(L.LoraError):
            L.lora_experts_group_workspace_bytes(*args)
    n = ctypes.c_size_t(0)
    assert status("lora_experts_packed_bytes", 1, 64, 128, 8, None) == "LORA_ERR_INVALID_ARG"
    assert status("lora_experts_packed_bytes", 1, 64, 128, 32, ctypes.addressof(n)) == "LORA_ERR_INVALID_ARG"


def test_the_binding_refuses_tensors_that_are_too_small_or_of_another_type():
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    e = torch.empty
    x, q, s, y = e(4, 256, dtype=bf), e(4, 256, dtype=f8), e(4, 2), e(4, 128, dtype=bf)
    w, ws = e(128 * 256, dtype=torch.uint8), e(1, 2)
    ids, st, od, pl, wt = e(2, 2, dtype=torch.int32), e(9, dtype=torch.int32), e(4, dtype=torch.int32), e(2, 2, dtype=torch.int32), e(2, 2)
    wide = e(8 * 128 * 512, dtype=torch.uint8)
    bad = [
        lambda: L.lora_rows_quantize(x.float(), q, s), lambda: L.lora_rows_quantize(x, q[:, :128], s), lambda: L.lora_rows_quantize(x, q[:3], s),
        lambda: L.lora_rows_quantize(x, q, s[:, :1]), lambda: L.lora_rows_quantize(x.t(), q, s), lambda: L.lora_rows_quantize(x, q, s.double()),
        lambda: L.lora_linear_scaled(q, s, w[:-1], ws, y), lambda: L.lora_linear_scaled(q, s, w, ws[:, :1], y), lambda: L.lora_linear_scaled(q, s[:3], w, ws, y),
        lambda: L.lora_linear_scaled(q, s, w, ws, y[:3]), lambda: L.lora_linear_scaled(x, s, w, ws, y), lambda: L.lora_linear_scaled(q, s, w, ws, y.float()),
        lambda: L.lora_experts_group(ids.long(), st, od, pl), lambda: L.lora_experts_group(ids, st, od[:3], pl), lambda: L.lora_experts_group(ids, st, od, pl[:1]),
        lambda: L.lora_experts_group(ids, st.float().double(), od, pl), lambda: L.lora_experts_group(ids.t(), st, od, pl),
        lambda: L.lora_experts_linear(x[:2], st, od[:3], 2, wide, y), lambda: L.lora_experts_linear(x[:2], st, od, 2, wide[:-1], y),
        lambda: L.lora_experts_linear(x[:2], st, od, 2, wide, y[:3]), lambda: L.lora_experts_linear(q[:2], st, od, 2, wide, y),
        lambda: L.lora_experts_linear_scaled(q[:2], s[:1], st, od, 2, wide, e(8, 1, 2), y), lambda: L.lora_experts_linear_scaled(q[:2], s, st, od, 2, wide, ws, y),
        lambda: L.lora_experts_combine(y, pl[:1], wt, y[:2]), lambda: L.lora_experts_combine(y, pl, wt.double(), y[:2]),
        lambda: L.lora_experts_combine(y[:, :64], pl, wt, y[:2]), lambda: L.lora_experts_combine(y, pl, wt, y[:1]),
        lambda: L.lora_experts_pack_weight(e(1, 128, 192, dtype=f8), w, in_features=256),
        lambda: L.lora_experts_pack_weight(e(1, 256, 128, dtype=f8).transpose(1, 2), w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, L.LoraError)):
            call()
            pytest.fail(f"call {i} went through")


@pytest.mark.parametrize("name, base, change", [
    ("lora_linear_scaled", LINEAR, dict(rows=1 << 16, ldq=(1 << 20) + 1024, lds=2)), ("lora_linear_scaled", LINEAR, dict(rows=1 << 16, lds=1 << 17)),
    ("lora_experts_linear", EXPERTS, dict(tokens=1 << 20, order=None, rows=1 << 20, ldx=1 << 16))])
def test_rows_beyond_what_the_kernels_reach_are_refused(name, base, change):
    assert status(name, *dict(base, **change).values(), None) == "LORA_ERR_SHAPE"


# ---- the binding, on tensors that would do but for one thing ------------------------------------------------
class OnGpu(torch.Tensor):
    """A tensor that stands on the GPU as far as the binding can tell."""
    is_cuda = True


def good():
    """{call: its tensors by name, in order}: 4 rows, 256 -> 128 features, 8 experts, 2 tokens of 2 picks"""
    bf, f8, i32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32
    e = lambda *shape, dtype=torch.float32: torch.zeros(*shape).to(dtype).as_subclass(OnGpu)  # noqa: E731
    x, q, s, y = e(4, 256, dtype=bf), e(4, 256, dtype=f8), e(4, 2), e(4, 128, dtype=bf)
    starts, order, place, ids = e(9, dtype=i32), e(4, dtype=i32), e(2, 2, dtype=i32), e(2, 2, dtype=i32)
    raw = lambda n: e(n, dtype=torch.uint8)  # noqa: E731
    return {
        "lora_rows_quantize": dict(x=x, q=q, scales=s),
        "lora_linear_scaled": dict(q=q, scales=s, w_packed=raw(128 * 256), w_scales=e(1, 2), y=y),
        "lora_experts_group": dict(ids=ids, starts=starts, order=order, place=place),
        "lora_experts_linear": dict(x=x[:2], starts=starts, order=order, picks=2, w_packed=raw(8 * 128 * 512), y=y),
        "lora_experts_linear_scaled": dict(q=q[:2], scales=s[:2], starts=starts, order=order, picks=2, w_packed=raw(8 * 128 * 256), w_scales=e(8, 1, 2), y=y),
        "lora_experts_combine": dict(y=y, place=place, weights=e(2, 2), z=y[:2]),
        "lora_experts_pack_weight": dict(w=e(1, 128, 256, dtype=f8), dev_packed=raw(128 * 256)),
    }


SAME_SIZE = {torch.bfloat16: (torch.float16, torch.int16), torch.float8_e4m3fn: (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.int8, torch.bool),
             torch.float32: (torch.int32,), torch.int32: (torch.float32, torch.uint32)}


@pytest.mark.parametrize("call, name, dtype", [(c, n, d) for c, given in good().items() for n, t in given.items() if isinstance(t, torch.Tensor)
                                               for d in SAME_SIZE.get(t.dtype, ())])
def test_the_binding_refuses_types_of_the_same_size(call, name, dtype):
    given = good()[call]
    given[name] = given[name].to(torch.float32).to(dtype)
    with pytest.raises(ValueError, match=f"^{name}: {dtype} does not do"):
        getattr(L, call)(**given)


@pytest.mark.parametrize("call, name", [(c, n) for c, given in good().items() for n, t in given.items() if isinstance(t, torch.Tensor)]
                         + [("lora_experts_group", "workspace")])
def test_the_binding_refuses_tensors_of_the_host(call, name):
    given = good()[call]
    given[name] = given[name].as_subclass(torch.Tensor) if name in given else torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match=f"^{name}: a tensor on cpu does not do"):
        getattr(L, call)(**given)


def eights(q, scales, call):
    """the tensors of a product in 8 bits, 192 -> 128 features, of one layer or of one expert"""
    e = lambda *shape, dtype=torch.float32: torch.zeros(*shape).to(dtype).as_subclass(OnGpu)  # noqa: E731
    w, ws, y = e(128 * 256, dtype=torch.uint8), e(1, 1, 2), e(q.shape[0], 128, dtype=torch.bfloat16)
    if call == "lora_linear_scaled":
        return q, scales, w, ws[0], y
    return q, scales, e(2, dtype=torch.int32), None, 1, w, ws, y


@pytest.mark.parametrize("call", ["lora_linear_scaled", "lora_experts_linear_scaled"])
@pytest.mark.parametrize("rows", [1, 3])
def test_the_binding_refuses_rows_whose_last_block_is_not_in_memory(call, rows):
    q = torch.zeros(rows, 256, dtype=torch.float8_e4m3fn).as_subclass(OnGpu)[:, 64:]  # 192 columns: the last row has 64 too few
    with pytest.raises(ValueError, match="^q: the last row's block of 128"):
        getattr(L, call)(*eights(q, torch.zeros(rows, 2).as_subclass(OnGpu), call))


@pytest.mark.parametrize("call", ["lora_linear_scaled", "lora_experts_linear_scaled"])
@pytest.mark.parametrize("rows", [1, 3])
def test_the_binding_takes_the_columns_that_are_there_of_rows_of_whole_blocks(call, rows, monkeypatch):
    told = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: told.append((name, *args)) or 0
    monkeypatch.setattr(L, "_lib", Library())
    q = torch.zeros(rows, 256, dtype=torch.float8_e4m3fn).as_subclass(OnGpu)[:, :192]
    getattr(L, call)(*eights(q, torch.zeros(rows, 2).as_subclass(OnGpu), call))
    name, address, ldq, _, _, n = told[0][:6]
    assert (name, address, ldq, n) == (call, q.data_ptr(), 256, rows) and 192 in told[0]


def test_the_binding_refuses_more_picks_than_32_bits_count(monkeypatch):
    told = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: told.append(args) or 0
    monkeypatch.setattr(L, "_lib", Library())
    e = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="meta").as_subclass(OnGpu)  # noqa: E731
    n = 2 ** 32 + 5
    with pytest.raises(ValueError, match="^ids: 4294967301 tokens x 1 picks"):
        L.lora_experts_group(e(n, 1), e(9), e(n), e(n))
    assert not told
    L.lora_experts_group(e(5, 1), e(9), e(5), e(5))
    assert told[0][2] == 5


def test_a_workspace_of_more_picks_is_enough_for_fewer():
    """by what the calls say of themselves: at every line where a work group takes more picks, and on either side of it"""
    ends = sorted({max(0, m * 2 ** k + d) for k in range(9, 26) for m in (1, 3) for d in (-1, 0, 1)} | {65000 * 8, 66000 * 8, 2 ** 31 - 1})
    for experts in (1, 256, 512):
        said = [L.lora_experts_group_workspace_bytes(n, experts) for n in ends]
        assert said == sorted(said)
    assert L.lora_experts_group_workspace_bytes(10 ** 6, 7) <= L.lora_experts_group_workspace_bytes(10 ** 6, 8)


F = 1 << 24  # LORA_EXPERTS_MAX_FEATURES


@pytest.mark.parametrize("name, base, change", [
    ("lora_linear_scaled", LINEAR, dict(rows=1 << 24, out=F, ldy=F)),                                                # tiles of 256 x 256: 2^32 of them
    ("lora_linear_scaled", LINEAR, dict(rows=1 << 21, in_f=128, ldq=128, lds=1, out=F >> 2, ldy=F >> 2)),              # .. 2^27, of 512 threads
    ("lora_experts_linear", EXPERTS, dict(tokens=3584, picks=1, rows=3584, experts=512, in_f=64, out=F, ldy=F)),     # of 32 x 128
    ("lora_experts_linear_scaled", SCALED, dict(tokens=3584, picks=1, rows=3584, experts=512, out=F, ldy=F)),
])
def test_more_tiles_than_a_launch_can_have_are_refused(name, base, change):
    assert status(name, *dict(base, **change).values(), None) == "LORA_ERR_SHAPE"
    assert "tiles" in L.lib().lora_last_error().decode()


@pytest.fixture
def told(monkeypatch):
    """what the binding tells the library, call by call"""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, *args)) or 0
    monkeypatch.setattr(L, "_lib", Library())
    return calls


def test_the_binding_takes_a_single_row_of_any_stride(told):
    e = lambda *shape, dtype=torch.float32: torch.zeros(*shape).to(dtype).as_subclass(OnGpu)  # noqa: E731
    x, q, s = e(1, 128, dtype=torch.bfloat16), e(1, 130, dtype=torch.uint8), e(1, 1)
    L.lora_rows_quantize(x, q, s)
    assert told[-1][1:9] == (x.data_ptr(), 128, 1, 128, q.data_ptr(), 128, s.data_ptr(), 1)
    y, place, z = e(1, 130, dtype=torch.bfloat16), e(1, 2, dtype=torch.int32), e(1, 128, dtype=torch.bfloat16)
    L.lora_experts_combine(y, place, e(1, 2), z)
    assert told[-1][1:4] == (y.data_ptr(), 128, 1) and told[-1][6:11] == (1, 2, 128, z.data_ptr(), 128)


@pytest.mark.parametrize("call", good())
def test_the_binding_takes_bits_for_bf16_and_8_bit_values(call, told):
    given = {n: t.view({torch.bfloat16: torch.uint16, torch.float8_e4m3fn: torch.uint8}.get(t.dtype, t.dtype)) if isinstance(t, torch.Tensor) else t
             for n, t in good()[call].items()}
    getattr(L, call)(**given)
    assert told[-1][0] == call and next(iter(given.values())).data_ptr() == told[-1][1]
