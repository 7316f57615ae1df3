"""What stands between the adapted projections of a layer, as cases that can be timed and compared: rotary positions, a paged cache of keys
and values that is appended to, and the attention that reads it, of single tokens, drafted trees and prompts.

Where `own` is false, run() computes the operators in elementary torch operations, in 32 bits (angles in 64), rounded once at the end;
where it is true, it makes the calls of the package's public entry points (paper_2511_22880_amd.binding).

A case is a dict.  `kind` says which operator one pass goes through:
  rotary     rows of `tokens` x `heads` heads of `dim` values, the first `rotary` of each turned by their position; `inverse` the gradient's way
  append     keys and values of `tokens` x `kv_heads` heads into a paged cache (`bits` 16: bf16, 8: E4M3 with a scale per slot and head), the
             keys turned on the way, and so are the queries (`heads`) of the same tokens; a share `idle` of the tokens is padding
  attention  `requests` requests of `new_lo` .. `new_hi` new tokens each behind `context_lo` .. `context_hi` cached ones, and `prompts` more of
             `prompt_lo` .. `prompt_hi` new tokens and nothing before them; a token sees the context and, among its own request's new tokens,
             those up to itself, or its ancestors and itself where `tree`
The sizes of requests are spread over the logarithm of their ranges, drawn from `routing`; the seed given to prepare() decides every value,
the trees, and which page is where.  Pages hold `page` slots.
"""
import math
import random

import torch

own = False

TOP = 448.0          # largest E4M3 value
LEAST = 2.0 ** -126  # smallest scale
F8 = torch.float8_e4m3fn
BASE = 500000.0
LENGTH = 8192        # positions that frequencies were made for, of the scaled kinds
SCALING = {"none": {}, "linear": dict(factor=4.0), "wavelength": dict(factor=8.0, low=1.0, high=4.0, length=LENGTH),
           "dimension": dict(factor=16.0, low=1.0, high=32.0, length=LENGTH)}


def _rotary(tokens, **more):
    return dict(dict(kind="rotary", tokens=tokens, heads=32, dim=128, rotary=128, interleaved=False, scaling="none", inverse=False,
                     positions=LENGTH, routing=0), **more)


def _append(tokens, **more):
    return dict(dict(kind="append", tokens=tokens, heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False, scaling="none", page=16, bits=16,
                     idle=0.0, positions=LENGTH, routing=0), **more)


def _attention(requests, **more):
    return dict(dict(kind="attention", requests=requests, new_lo=1, new_hi=1, context_lo=1, context_hi=1, prompts=0, prompt_lo=1, prompt_hi=1,
                     tree=False, heads=32, kv_heads=8, dim=128, page=16, bits=16, routing=0), **more)


def listed():
    return [
        # queries of a handful of decode tokens: latency
        _rotary(7, name="rotary_few"),
        # the gradients of the tokens of 32 prompts, half of each head turned, far positions of a context made longer
        _rotary(19675, rotary=64, interleaved=True, scaling="dimension", inverse=True, positions=131072, name="rotary_prompts"),
        # one user's token: the launch is what it costs
        _append(1, name="append_one"),
        # a decode step of the whole batch
        _append(256, scaling="wavelength", positions=65536, idle=0.1, name="append_decode"),
        # the tokens of 32 prompts into a cache in 8 bits
        _append(19675, page=64, bits=8, name="append_prompts"),
        # one user, one token, a short conversation: latency
        _attention(1, context_lo=1500, context_hi=1500, name="attention_one"),
        # a decode step of the whole batch, contexts of very different lengths
        _attention(256, context_lo=200, context_hi=8000, name="attention_decode"),
        # a few users with very long contexts in 8 bits
        _attention(5, context_lo=60000, context_hi=130000, heads=64, page=64, bits=8, name="attention_far"),
        # trees of drafted tokens, up to 24 each
        _attention(40, new_lo=8, new_hi=24, context_lo=300, context_hi=6000, tree=True, page=32, name="attention_trees"),
        # large trees, small heads, one key head for seven query heads
        _attention(13, new_lo=40, new_hi=64, context_lo=2000, context_hi=20000, tree=True, heads=28, kv_heads=4, dim=64, bits=8, name="attention_big_trees"),
        # what a mixed batch holds: eight prompts beside 384 decode tokens
        _attention(384, context_lo=100, context_hi=4000, prompts=8, prompt_lo=256, prompt_hi=2048, name="attention_mixed"),
        # pieces of long prompts behind what came before them
        _attention(3, new_lo=2000, new_hi=4096, context_lo=4000, context_hi=16000, page=64, name="attention_pieces"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(8, 8), (32, 8), (32, 8), (64, 8), (16, 2), (28, 4), (9, 3), (16, 1), (20, 20)]


def draw(rng):
    kind = rng.choice(["rotary", "append", "append", "attention", "attention", "attention", "attention"])
    heads, kv_heads = rng.choice(HEADS)
    dim = rng.choice([64, 128, 128])
    shape = dict(heads=heads, dim=dim, routing=rng.randrange(1, 1 << 20))
    turned = dict(rotary=rng.choice([dim, dim, dim // 2, dim // 4]), interleaved=rng.random() < 0.4, scaling=rng.choice(sorted(SCALING)),
                  positions=_log(rng, 100, 1 << 20))
    if kind == "rotary":
        return _rotary(min(19000, _log(rng, 1, 8e7 / (heads * dim))) | 1, inverse=rng.random() < 0.4, **shape, **turned)
    shape.update(kv_heads=kv_heads, page=rng.choice([16, 16, 32, 64, 128]), bits=rng.choice([16, 16, 8]))
    if kind == "append":
        return _append(min(19000, _log(rng, 1, 8e7 / ((heads + kv_heads) * dim))) | 1, idle=rng.choice([0.0, 0.0, 0.1, 0.5]), **shape, **turned)
    form = rng.choice(["decode", "decode", "trees", "trees", "pieces", "mixed"])
    while True:
        if form == "decode":
            hi = _log(rng, 16, 130000)
            sizes = dict(requests=_log(rng, 1, 300), context_lo=max(1, hi // rng.choice([1, 3, 40])), context_hi=hi)
        elif form == "trees":
            new, hi = _log(rng, 2, 64), _log(rng, 16, 30000)
            sizes = dict(requests=_log(rng, 1, 100), new_lo=rng.choice([1, new]), new_hi=new, tree=rng.random() < 0.8,
                         context_lo=max(1, hi // rng.choice([1, 10])), context_hi=hi)
        elif form == "pieces":
            new, hi = _log(rng, 65, 6000), _log(rng, 1, 16000)
            sizes = dict(requests=_log(rng, 1, 8), new_lo=max(1, new // 3), new_hi=new, context_lo=max(1, hi // 4), context_hi=hi)
        else:
            sizes = dict(requests=_log(rng, 10, 400), context_lo=50, context_hi=_log(rng, 100, 5000), prompts=_log(rng, 1, 10), prompt_lo=65,
                         prompt_hi=_log(rng, 70, 3000))
        case = _attention(**sizes, **shape)
        least = work(case)
        if least["bytes"] < 2.5e9 and least["flops"] < 9e11:
            return case


# ---- sizes --------------------------------------------------------------------------------------------------
def _sizes(case):
    """(new tokens, length with them) of every request."""
    rng = random.Random(7 + case["routing"])
    sizes = []
    for _ in range(case["requests"]):
        new = _log(rng, case["new_lo"], case["new_hi"])
        sizes.append((new, new + _log(rng, case["context_lo"], case["context_hi"])))
    for _ in range(case["prompts"]):
        new = _log(rng, case["prompt_lo"], case["prompt_hi"])
        sizes.append((new, new))
    rng.shuffle(sizes)
    return sizes


def _starts(sizes):
    starts = [0]
    for new, _ in sizes:
        starts.append(starts[-1] + new)
    return starts


# ---- inputs -------------------------------------------------------------------------------------------------
def _values(g, *shape):
    """Activations: normal, with some channels larger than the rest, as they are in earnest."""
    x = torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    loud = torch.rand(shape[-1], generator=g, device="cuda") < 0.02
    return x.mul_(torch.where(loud, 3.0, 1.0).to(torch.bfloat16))


def _to_bits8(x):
    """(E4M3, fp32 scales without the last dimension) of fp32 rows"""
    top = x.abs().amax(dim=-1).clamp(min=TOP * LEAST)
    return (x * (TOP / 512) / top[..., None] * 512).to(F8), top / TOP


def _cache(case, g, pages):
    """{k, v: [pages][kv_heads][page][dim], and in 8 bits k_scales, v_scales: [pages][kv_heads][page]}"""
    cache = {}
    for name in ("k", "v"):
        x = _values(g, pages, case["kv_heads"], case["page"], case["dim"])
        if case["bits"] == 16:
            cache[name] = x
            continue
        cache[name], cache[name + "_scales"] = torch.empty(x.shape, dtype=F8, device="cuda"), torch.empty(x.shape[:-1], device="cuda")
        for at in range(0, pages, 4096):
            q, scales = _to_bits8(x[at:at + 4096].float())
            cache[name][at:at + 4096], cache[name + "_scales"][at:at + 4096] = q, scales
    return cache


def _trees(g, sizes):
    """One word for every new token: bit j says that it sees its request's new token j.  Parents are earlier tokens, near ones rather than far ones."""
    most = max(new for new, _ in sizes)
    pull = torch.rand(len(sizes), most, generator=g, device="cuda").cpu().tolist()
    words = []
    for (new, _), row in zip(sizes, pull):
        seen = []
        for i in range(new):
            parent = i - 1 - int(row[i] ** 2 * min(i, 6)) if i else -1
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        words += seen
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * case["routing"] + seed)
    s, dim = dict(case), case["dim"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["kind"] == "attention":
        sizes = _sizes(case)
        starts = _starts(sizes)
        counts = [-(-length // case["page"]) for _, length in sizes]
        pages = sum(counts) + 3
        where = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        s["table"] = torch.full((len(sizes), max(counts)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, n in enumerate(counts):
            s["table"][r, :n] = where[at:at + n]
            at += n
        s["sizes"], s["starts"], s["lengths"] = sizes, ints(starts), ints([length for _, length in sizes])
        s["most"] = max(new for new, _ in sizes)
        s["words"] = _trees(g, sizes) if case["tree"] else None
        s["q"] = _values(g, starts[-1], case["heads"], dim)
        s["y"] = torch.zeros_like(s["q"])
        s["cache"] = _cache(case, g, pages)
    else:
        t = case["tokens"]
        s["positions"] = torch.randint(0, case["positions"], (t,), generator=g, device="cuda").to(torch.int32)
        s["q"] = _values(g, t, case["heads"], dim)
        s["y"] = torch.zeros_like(s["q"])
        if case["kind"] == "append":
            # (what the fused projection gives: keys and values side by side)
            s["kv"] = _values(g, t, 2 * case["kv_heads"], dim)
            pages = -(-t // case["page"]) + 5
            s["cache"] = _cache(case, g, pages)
            s["slots"] = torch.randperm(pages * case["page"], generator=g, device="cuda")[:t].to(torch.int32)
            if t > 1:
                gone = torch.rand(t, generator=g, device="cuda") < case["idle"]
                s["slots"], s["positions"] = torch.where(gone, -1, s["slots"]), torch.where(gone, -1, s["positions"])
    if own:
        from paper_2511_22880_amd import binding as L
        s["L"] = L
        if "cache" in s:
            s["paged"] = L.Cache(**s["cache"])
        if "rotary" in case:
            s["turn"] = L.Rotary(case["rotary"], BASE, interleaved=case["interleaved"], scaling=case["scaling"], **SCALING[case["scaling"]])
        if case["kind"] == "attention":
            n = L.lora_attention_workspace_bytes(s["q"].shape[0], case["heads"], len(s["sizes"]), s["table"].shape[1], s["paged"])
            s["workspace"] = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass -----------------------------------------------------------------------------------------------
def _frequencies(dims, scaling):
    """(radians a position of every pair, factor of the turned values)"""
    f = BASE ** (-torch.arange(0, dims, 2, dtype=torch.float64, device="cuda") / dims)
    p = SCALING[scaling]
    if scaling == "none":
        return f, 1.0
    if scaling == "linear":
        return f / p["factor"], 1.0
    if scaling == "wavelength":
        turns = p["length"] * f / (2 * math.pi)
        keep = ((turns - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        return f * keep + f / p["factor"] * (1 - keep), 1.0
    first, last = (dims * math.log(p["length"] / (n * 2 * math.pi)) / (2 * math.log(BASE)) for n in (p["high"], p["low"]))
    first, last = max(math.floor(first), 0), min(math.ceil(last), dims - 1)
    ramp = ((torch.arange(dims // 2, dtype=torch.float64, device="cuda") - first) / max(last - first, 0.001)).clamp(0, 1)
    return f / p["factor"] * ramp + f * (1 - ramp), 0.1 * math.log(p["factor"]) + 1.0


def _turned(s, x, inverse=False):
    """fp32 [tokens][heads][dim] of bf16 x, turned"""
    f, m = _frequencies(s["rotary"], s["scaling"])
    angle = s["positions"].double()[:, None] * f
    c, d = (torch.cos(angle) * m).float()[:, None], (torch.sin(angle) * (-m if inverse else m)).float()[:, None]
    y, r = x.float(), s["rotary"]
    y = y.clone() if y is x else y
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = a * c - b * d, a * d + b * c
    return y


def _held(cache, name, page, off):
    """fp32 [..][kv_heads][dim] of the slots `off` of pages `page`"""
    x = cache[name]
    if x.dtype == F8:  # (bytes: indexing knows those)
        return x.view(torch.uint8)[page, :, off].view(F8).float() * cache[name + "_scales"][page, :, off][..., None]
    return x[page, :, off].float()


def _rows(s, rs, i0, i1):
    """Attention of the new tokens i0 .. i1 - 1 of requests rs, those that they have, into y."""
    heads, kv_heads, dim, page = s["heads"], s["kv_heads"], s["dim"], s["page"]
    group, device = heads // kv_heads, s["q"].device
    r = torch.tensor(rs, device=device)
    new = s["starts"][r + 1].long() - s["starts"][r].long()
    length = s["lengths"][r].long()
    top = max(s["sizes"][i][1] for i in rs)
    key = torch.arange(top, device=device)
    at, off = s["table"][r].long().clamp(min=0)[:, key // page], (key % page).expand(len(rs), -1)
    k, v = (_held(s["cache"], name, at, off).permute(0, 2, 1, 3).contiguous() for name in ("k", "v"))
    there = key < length[:, None]
    v = torch.where(there[:, None, :, None], v, 0.0)
    i = torch.arange(i0, i1, device=device)
    row = (s["starts"][r].long()[:, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().view(len(rs), i1 - i0, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(len(rs), kv_heads, -1, dim)
    score = (q @ k.transpose(2, 3).contiguous()).mul_(dim ** -0.5).view(len(rs), kv_heads, i1 - i0, group, top)
    j = key[None] - (length - new)[:, None]  # which new token a key is, negative in the context
    if s["words"] is None:
        sees = j[:, None, :] <= i[None, :, None]
    else:
        bits = (s["words"][row][:, :, None] >> j.clamp(0, 63)[:, None, :]) & 1
        sees = (j[:, None, :] < 0) | (bits == 1)
    sees = (sees & there[:, None, :])[:, None, :, None, :]
    score = torch.where(sees, score, -math.inf)
    weight = (score - score.amax(dim=-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = weight.sum(dim=-1, keepdim=True)
    weight = (weight / torch.where(total > 0, total, 1.0)).view(len(rs), kv_heads, -1, top)
    z = (weight @ v).view(len(rs), kv_heads, i1 - i0, group, dim).permute(0, 2, 1, 3, 4).reshape(len(rs), i1 - i0, heads, dim)
    mine = i[None] < new[:, None]
    s["y"][row[mine]] = z[mine].to(torch.bfloat16)


def _plain(s):
    if s["kind"] == "rotary":
        s["y"].copy_(_turned(s, s["q"], s["inverse"]))
        return s["y"]
    if s["kind"] == "append":
        there = s["slots"] >= 0
        s["y"][there] = _turned(s, s["q"])[there].to(torch.bfloat16)
        slot = s["slots"][there].long()
        page, off, cache, n = slot // s["page"], slot % s["page"], s["cache"], s["kv_heads"]
        for name, x in (("k", _turned(s, s["kv"][:, :n])[there]), ("v", s["kv"][:, n:][there].float())):
            if s["bits"] == 8:
                q, scales = _to_bits8(x)
                cache[name].view(torch.uint8)[page, :, off], cache[name + "_scales"][page, :, off] = q.view(torch.uint8), scales
            else:
                cache[name][page, :, off] = x.to(torch.bfloat16)
        return dict(cache, q=s["y"])
    # requests of few new tokens in batches, those of like lengths together; of many a request at a time, in blocks of rows
    few = sorted((r for r, (new, _) in enumerate(s["sizes"]) if new <= 64), key=lambda r: s["sizes"][r][1])
    while few:
        batch = [few.pop()]
        longest = s["sizes"][batch[0]][1]
        most = max(1, int(2e8 / (longest * max(s["kv_heads"] * s["dim"], s["heads"] * min(64, s["most"])))))
        while few and len(batch) < most and 2 * s["sizes"][few[-1]][1] > longest:
            batch.append(few.pop())
        _rows(s, batch, 0, max(s["sizes"][r][0] for r in batch))
    for r, (new, length) in enumerate(s["sizes"]):
        if new > 64:
            step = max(64, int(4e8 / (length * s["heads"])))
            for i in range(0, new, step):
                _rows(s, [r], i, min(new, i + step))
    return s["y"]


def run(s):
    if not own:
        return _plain(s)
    L = s["L"]
    if s["kind"] == "rotary":
        L.lora_rotary(s["q"], s["positions"], s["turn"], s["y"], inverse=s["inverse"])
        return s["y"]
    if s["kind"] == "append":
        n = s["kv_heads"]
        L.lora_cache_append(s["kv"][:, :n], s["kv"][:, n:], s["slots"], s["paged"], s["turn"], s["positions"], s["q"], s["y"])
        return dict(s["cache"], q=s["y"])
    L.lora_attention(s["q"], s["starts"], s["lengths"], s["table"], s["paged"], s["y"], s["workspace"], tree=s["words"], most=s["most"])
    return s["y"]


# ---- what a pass cannot do without --------------------------------------------------------------------------
def work(case):
    dim = case["dim"]
    if case["kind"] == "rotary":
        n = case["tokens"] * case["heads"] * dim
        return {"bytes": 4 * n + 4 * case["tokens"] + 4 * case["rotary"], "flops": 3 * n}
    held = dim * case["bits"] // 8 + (4 if case["bits"] == 8 else 0)  # bytes of a head's key or value in the cache
    if case["kind"] == "append":
        t = int(round(case["tokens"] * (1.0 - case["idle"])))
        return {"bytes": t * (4 * case["heads"] * dim + 2 * case["kv_heads"] * (2 * dim + held)) + 8 * case["tokens"] + 4 * case["rotary"],
                "flops": 3 * t * (case["heads"] + case["kv_heads"]) * dim}
    tokens = pairs = keys = 0
    for new, length in _sizes(case):
        tokens += new
        keys += length
        pairs += new * (length - new) + new * (new + 1) // 2
    return {"bytes": 4 * tokens * case["heads"] * dim + 2 * keys * case["kv_heads"] * held, "flops": 4 * pairs * case["heads"] * dim}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------
def _angle(case, i):
    """(radians a position of pair i, factor), in 64 bits"""
    dims, p = case["rotary"], SCALING[case["scaling"]]
    f = math.exp(-2.0 * i / dims * math.log(BASE))
    if case["scaling"] == "linear":
        return f / p["factor"], 1.0
    if case["scaling"] == "wavelength":
        wave = 2 * math.pi / f
        if wave < p["length"] / p["high"]:
            return f, 1.0
        if wave > p["length"] / p["low"]:
            return f / p["factor"], 1.0
        mix = (p["length"] / wave - p["low"]) / (p["high"] - p["low"])
        return (1 - mix) * f / p["factor"] + mix * f, 1.0
    if case["scaling"] == "dimension":
        pair = lambda n: 0.5 * dims * math.log(p["length"] / (2 * math.pi * n), BASE)  # noqa: E731
        a, b = max(0, math.floor(pair(p["high"]))), min(dims - 1, math.ceil(pair(p["low"])))
        mix = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
        return mix * f / p["factor"] + (1 - mix) * f, 1.0 + math.log(p["factor"]) / 10
    return f, 1.0


def _turned64(case, positions, x):
    y, half = x.double(), case["rotary"] // 2
    for i in range(half):
        f, m = _angle(case, i)
        z = torch.polar(torch.full_like(positions, m, dtype=torch.float64), positions.double() * (-f if case.get("inverse") else f))
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        pair = torch.complex(y[:, :, a].clone(), y[:, :, b].clone()) * z[:, None]
        y[:, :, a], y[:, :, b] = pair.real, pair.imag
    return y


def _nearest8(v):
    """The nearest E4M3 value (ties to even), in 64 bits, of values up to 448."""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    if case["kind"] == "rotary":
        return _turned64(case, s["positions"], s["q"])
    if case["kind"] == "append":
        there = torch.nonzero(s["slots"] >= 0)[:, 0]
        out = {name: x.view(torch.uint8).view(F8).float().double() if x.dtype == F8 else x.double() for name, x in s["cache"].items()}
        out["q"] = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        out["q"][there] = _turned64(case, s["positions"], s["q"])[there]
        n = case["kv_heads"]
        for name, x in (("k", _turned64(case, s["positions"], s["kv"][:, :n])), ("v", s["kv"][:, n:].double())):
            x = x[there]
            page, off = torch.div(s["slots"][there], case["page"], rounding_mode="floor").long(), torch.remainder(s["slots"][there], case["page"]).long()
            if case["bits"] == 8:
                top = torch.clamp(x.abs().max(dim=2).values, min=TOP * LEAST)
                out[name + "_scales"][page, :, off] = top / TOP
                x = _nearest8(x * TOP / top[:, :, None])
            out[name][page, :, off] = x
        return out
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, table = case["heads"] // case["kv_heads"], s["table"].cpu()
    words = None if s["words"] is None else s["words"].cpu().tolist()
    starts = _starts(s["sizes"])
    for r, (new, length) in enumerate(s["sizes"]):
        pages = table[r, :-(-length // case["page"])].long().cuda()
        held = []
        for name in ("k", "v"):
            x = s["cache"][name].view(torch.uint8)[pages].view(s["cache"][name].dtype).double()
            if case["bits"] == 8:
                x = x * s["cache"][name + "_scales"][pages].double()[..., None]
            held.append(x.transpose(0, 1).reshape(case["kv_heads"], -1, case["dim"])[:, :length])
        k, v = held
        context = length - new
        sees = torch.ones(new, length, dtype=torch.bool)
        if words is None:
            sees = torch.tril(sees, diagonal=context)
        else:
            for i in range(new):
                w = words[starts[r] + i]
                sees[i, context:] = torch.tensor([w >> j & 1 == 1 for j in range(new)])
        sees = sees.cuda()
        for h in range(case["heads"]):
            q = s["q"][starts[r]:starts[r + 1], h].double()
            for i in range(0, new, 2048):
                score = (q[i:i + 2048] @ k[h // group].t()) / math.sqrt(case["dim"])
                score = score.masked_fill(~sees[i:i + 2048], -math.inf)
                y[starts[r] + i:starts[r] + min(new, i + 2048), h] = torch.softmax(score, dim=1) @ v[h // group]
    return y
