"""A block of a mixture-of-experts model whose frozen weights are held in 8 bits, with LoRA adapters on its projections.

Three parts, each one path through the library as a serving program takes it; every buffer is made once, nothing is allocated or waited
for in a step, and the host never learns which tokens picked which experts:

    AdaptedProjection   y = x W + s_a (x A_a) B_a     lora_rows_quantize, lora_linear_scaled, lora_apply
    AdaptedAttention    y = attention(x W_q, x W_k, x W_v) W_o, all four adapted, over a paged cache
                        three projections, lora_cache_append (which turns queries and keys), lora_attention, the fourth
    ExpertLayer         z = sum over picks of weight * W_down_e (silu(W_gate_e x) * W_up_e x)
                        lora_experts_group, lora_rows_quantize, lora_experts_linear_scaled (gate and up side by side), the
                        activation, lora_rows_quantize, lora_experts_linear_scaled on rows in expert order, lora_experts_combine

``python -m paper_2511_22880_amd.expert_layer`` runs them on random weights and checks them against 64 bits.
"""
from __future__ import annotations

import torch

from . import binding as L

BLOCK = 128
F8 = torch.float8_e4m3fn


def weights_to_8_bits(w: torch.Tensor):
    """[experts][out][in] (in a multiple of 128) -> E4M3 values and fp32 scales [experts][out / 128][in / 128]."""
    e, out_f, in_f = w.shape
    b = w.float().view(e, out_f // BLOCK, BLOCK, in_f // BLOCK, BLOCK)
    scales = (b.abs().amax(dim=(2, 4)) / 448.0).clamp(min=2.0 ** -126)
    return (b / scales[:, :, None, :, None]).to(F8).view(e, out_f, in_f), scales


class Packed:
    """Weights of one layer, or of a layer of experts, in operand order, with their scales."""

    def __init__(self, w8: torch.Tensor, scales: torch.Tensor):
        self.experts, self.out_features, self.in_features = w8.shape
        self.scales = scales.contiguous()
        self.packed = torch.empty(L.lora_experts_packed_bytes(*w8.shape[:1], self.in_features, self.out_features, 8), dtype=torch.uint8, device=w8.device)
        L.lora_experts_pack_weight(w8.contiguous(), self.packed, torch.cuda.current_stream())


class Rows8:
    """Room for rows in 8 bits."""

    def __init__(self, rows: int, features: int):
        blocks = (features + BLOCK - 1) // BLOCK
        self.q = torch.empty(rows, blocks * BLOCK, dtype=F8, device="cuda")
        self.scales = torch.empty(rows, blocks, device="cuda")

    def fill(self, x: torch.Tensor, stream):
        n = x.shape[0]
        L.lora_rows_quantize(x, self.q[:n], self.scales[:n], stream)
        return self.q[:n], self.scales[:n]


class AdaptedProjection:
    """One projection: the frozen layer in 8 bits, the adapters of a pool on top."""

    def __init__(self, w: Packed, pool: L.Pool, most_tokens: int):
        self.w, self.pool = w, pool
        self.rows = Rows8(most_tokens, w.in_features)

    def __call__(self, x: torch.Tensor, segments: L.Segments, y: torch.Tensor, workspace: torch.Tensor) -> None:
        """x: bf16 [tokens][in]; segments: the batch's plan on the pool; y: bf16 [tokens][out], written."""
        stream = torch.cuda.current_stream()
        q, scales = self.rows.fill(x, stream)
        L.lora_linear_scaled(q, scales, self.w.packed, self.w.scales[0], y, stream)
        L.lora_apply(self.pool, segments, x, y, workspace, stream)


class AdaptedAttention:
    """What stands between a layer's norm and its experts: queries, keys and values, the cache, attention, the output projection."""

    def __init__(self, q: AdaptedProjection, k: AdaptedProjection, v: AdaptedProjection, o: AdaptedProjection, cache: L.Cache, rotary: L.Rotary, most_tokens: int,
                 most_requests: int, width: int):
        """width: pages a request has at most."""
        self.projections, self.cache, self.rotary, self.width = (q, k, v, o), cache, rotary, width
        self.heads = q.w.out_features // cache.head_dim
        rows = lambda n: torch.empty(most_tokens, n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.turned, self.z = (rows(p.w.out_features) for p in (q, k, v, q, q))
        n = L.lora_attention_workspace_bytes(most_tokens, self.heads, most_requests, width, cache)
        self.workspace = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")

    def __call__(self, x: torch.Tensor, segments, positions: torch.Tensor, slots: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor,
                 page_table: torch.Tensor, y: torch.Tensor, apply_workspace: torch.Tensor, tree=None, most: int = 0) -> None:
        """x: bf16 [tokens][hidden]; segments: the batch's plans on the pools of q, k, v and o; positions, slots: int32 [tokens]; starts, lengths, page_table, tree,
        most: of lora_attention, lengths with this step's tokens, page_table a view of the columns that the longest request needs, where the caller knows that; y: bf16
        [tokens][hidden], written."""
        stream, n, dim = torch.cuda.current_stream(), x.shape[0], self.cache.head_dim
        for projection, segment, out in zip(self.projections, segments, (self.q, self.k, self.v)):
            projection(x, segment, out[:n], apply_workspace)
        heads = lambda t: t[:n].view(n, -1, dim)  # noqa: E731
        L.lora_cache_append(heads(self.k), heads(self.v), slots, self.cache, self.rotary, positions, heads(self.q), heads(self.turned), stream)
        L.lora_attention(heads(self.turned), starts, lengths, page_table, self.cache, heads(self.z), self.workspace, tree=tree, most=most, stream=stream)
        self.projections[3](self.z[:n], segments[3], y, apply_workspace)


class ExpertLayer:
    """The experts: gate_up holds W_gate and W_up of an expert one behind the other ([experts][2 * inner][hidden]), down [experts][hidden][inner]."""

    def __init__(self, gate_up: Packed, down: Packed, picks: int, most_tokens: int):
        self.gate_up, self.down, self.picks = gate_up, down, picks
        rows, inner = most_tokens * picks, down.in_features
        ints = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
        self.starts, self.order, self.place = ints(gate_up.experts + 1), ints(rows), ints(rows)
        self.workspace = torch.empty(max(16, L.lora_experts_group_workspace_bytes(rows, gate_up.experts)), dtype=torch.uint8, device="cuda")
        self.x8, self.h8 = Rows8(most_tokens, gate_up.in_features), Rows8(rows, inner)
        # (the rows behind the last expert's, where picks have none, are never written: they go through the activation and the second quantiser
        # with whatever they hold, and no product or sum reads them)
        self.h = torch.zeros(rows, 2 * inner, dtype=torch.bfloat16, device="cuda")
        self.act32 = torch.empty(rows, inner, device="cuda")
        self.act = torch.empty(rows, inner, dtype=torch.bfloat16, device="cuda")
        self.y = torch.empty(rows, down.out_features, dtype=torch.bfloat16, device="cuda")

    def __call__(self, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, z: torch.Tensor) -> None:
        """x: bf16 [tokens][hidden]; ids, weights: int32 and fp32 [tokens][picks] of the router; z: bf16 [tokens][hidden], written."""
        stream = torch.cuda.current_stream()
        rows, inner = x.shape[0] * self.picks, self.down.in_features
        L.lora_experts_group(ids, self.starts, self.order[:rows], self.place[:rows], self.workspace, stream)
        q, scales = self.x8.fill(x, stream)
        L.lora_experts_linear_scaled(q, scales, self.starts, self.order[:rows], self.picks, self.gate_up.packed, self.gate_up.scales, self.h[:rows], stream)
        act = self.act32[:rows].copy_(self.h[:rows, :inner])  # silu(gate) * up in 32 bits, rounded once
        torch.nn.functional.silu(act, inplace=True).mul_(self.h[:rows, inner:])
        self.act[:rows].copy_(act)
        q, scales = self.h8.fill(self.act[:rows], stream)
        L.lora_experts_linear_scaled(q, scales, self.starts, None, 1, self.down.packed, self.down.scales, self.y[:rows], stream)
        L.lora_experts_combine(self.y[:rows], self.place[:rows].view(-1, self.picks), weights, z, stream)


def _values(w8: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    return w8.double() * scales.double().repeat_interleave(BLOCK, dim=1).repeat_interleave(BLOCK, dim=2)


def reference(x, ids, weights, gate_up, down):
    """The expert layer on the same 8-bit weights, activations in 64 bits throughout."""
    z = torch.zeros(x.shape[0], down.shape[1], dtype=torch.float64, device=x.device)
    inner = down.shape[2]
    for e in range(gate_up.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        h = x[t].double() @ gate_up[e].t()
        z.index_add_(0, t, weights[t, j].double()[:, None] * ((torch.nn.functional.silu(h[:, :inner]) * h[:, inner:]) @ down[e].t()))
    return z


class Adapters:
    """Random adapters of the given ranks on a layer of this shape, and the plan of a batch on them."""

    def __init__(self, in_f: int, out_f: int, ranks, token_adapter, rand):
        import numpy as np
        self.ranks, self.token_adapter = np.asarray(ranks, dtype=np.int32), np.asarray(token_adapter, dtype=np.int32)
        self.scales = (2.0 / self.ranks).astype(np.float32)
        self.arena = torch.zeros(L.lora_pool_bytes(in_f, out_f, self.ranks, self.scales), dtype=torch.uint8, device="cuda")
        self.pool = L.lora_pool_create(in_f, out_f, self.ranks, self.scales, self.arena)
        self.A = [(rand(in_f, int(r)) * 0.02).to(torch.bfloat16) for r in self.ranks]
        self.B = [(rand(int(r), out_f) * 0.02).to(torch.bfloat16) for r in self.ranks]
        for a in range(len(self.ranks)):
            L.lora_pool_load(self.pool, a, self.A[a], self.B[a], src_is_device=True, stream=torch.cuda.current_stream())
        self.segments = L.lora_segments_build(self.pool, self.token_adapter, torch.cuda.current_stream())
        self.workspace_bytes = L.lora_apply_workspace_bytes(self.pool, self.segments)

    def add(self, x: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
        """fp64 y with the deltas of x"""
        for t, a in enumerate(self.token_adapter):
            if a >= 0:
                y[t] += float(self.scales[a]) * (x[t].double() @ self.A[a].double()) @ self.B[a].double()
        return y

    def close(self) -> None:
        L.lora_segments_destroy(self.segments)
        L.lora_pool_destroy(self.pool)


def attention_reference(q, k, v, cached, positions, sizes, dims: int, base: float = 10000.0):
    """Attention in 64 bits: q [tokens][heads][dim], k and v [tokens][kv_heads][dim] of the new tokens, not yet turned; cached: a request's context, (k, v)
    [keys][kv_heads][dim] as the cache holds it; sizes: (rows, keys) of the requests."""
    f = base ** (-torch.arange(0, dims, 2, dtype=torch.float64, device=q.device) / dims)
    angle = positions.double()[:, None, None] * f

    def turned(x):
        x1, x2 = x[..., :dims // 2].double(), x[..., dims // 2:dims].double()
        return torch.cat([x1 * angle.cos() - x2 * angle.sin(), x1 * angle.sin() + x2 * angle.cos(), x[..., dims:].double()], dim=2)

    q, k, z, at = turned(q), turned(k), torch.zeros(q.shape, dtype=torch.float64, device=q.device), 0
    group = q.shape[1] // k.shape[1]
    for (n, keys), (ck, cv) in zip(sizes, cached):
        rows = slice(at, at + n)
        kk, vv = (torch.cat([c.double(), t[rows].double()]).repeat_interleave(group, dim=1).permute(1, 0, 2) for c, t in ((ck, k), (cv, v)))
        s = q[rows].permute(1, 0, 2) @ kk.transpose(1, 2).contiguous() / q.shape[2] ** 0.5
        late = torch.arange(keys, device=q.device)[None] > keys - n + torch.arange(n, device=q.device)[:, None]
        z[rows] = (torch.softmax(s.masked_fill(late, float("-inf")), dim=2) @ vv).permute(1, 0, 2)
        at += n
    return z


def attention_example(rand, seed: int = 1):
    """A prompt, a piece of one and some single tokens through an AdaptedAttention.  (the block, its adapters and weights, x, y, what attention_reference takes
    of the batch)"""
    hidden, heads, kv_heads, dim, page, width = 1024, 8, 2, 128, 16, 20
    sizes = [(90, 90), (40, 200)] + [(1, 17 + 9 * i) for i in range(30)]  # (new tokens, with their context)
    tokens, ranks = sum(n for n, _ in sizes), [8, 16, 32, 64] * 2
    token_adapter = [-1 if t % 5 == 4 else t % len(ranks) for t in range(tokens)]
    x = rand(tokens, hidden).to(torch.bfloat16)
    shapes = [(hidden, heads * dim), (hidden, kv_heads * dim), (hidden, kv_heads * dim), (heads * dim, hidden)]
    adapters = [Adapters(*shape, ranks, token_adapter, rand) for shape in shapes]
    weights = [weights_to_8_bits(rand(1, out_f, in_f) * 0.03) for in_f, out_f in shapes]
    projections = [AdaptedProjection(Packed(*w), a.pool, tokens) for w, a in zip(weights, adapters)]
    pages = width * len(sizes)
    k, v = (rand(pages, kv_heads, page, dim).to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).view(len(sizes), width)
    where = [[(int(table[r, j // page]), j % page) for j in range(keys)] for r, (_, keys) in enumerate(sizes)]
    cached = []
    for (n, keys), slots in zip(sizes, where):
        ids, places = (torch.tensor([s[i] for s in slots[:keys - n]], dtype=torch.long, device="cuda") for i in (0, 1))
        cached.append((k[ids, :, places], v[ids, :, places]))
    ints = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")  # noqa: E731
    positions = ints([j for n, keys in sizes for j in range(keys - n, keys)])
    slots = ints([p * page + j for (n, keys), s in zip(sizes, where) for p, j in s[keys - n:]])
    starts = ints([sum(n for n, _ in sizes[:r]) for r in range(len(sizes) + 1)])
    block = AdaptedAttention(*projections, L.Cache(k, v), L.Rotary(dim), tokens, len(sizes), width)
    y = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    room = torch.empty(max(256, *(a.workspace_bytes for a in adapters)), dtype=torch.uint8, device="cuda")
    block(x, [a.segments for a in adapters], positions, slots, starts, ints([keys for _, keys in sizes]), table.to(torch.int32).cuda(), y, room, most=90)
    return block, adapters, weights, x, y, (cached, positions, sizes, dim)


def main() -> None:
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    hidden, inner, experts, picks, tokens = 1024, 512, 16, 4, 200
    x = rand(tokens, hidden).to(torch.bfloat16)

    # the projection: 8 adapters of ranks 8 to 64, every fifth token without one
    adapters = Adapters(hidden, hidden, [8, 16, 32, 64] * 2, [-1 if t % 5 == 4 else t % 8 for t in range(tokens)], rand)
    workspace = torch.empty(max(256, adapters.workspace_bytes), dtype=torch.uint8, device="cuda")
    w8, ws = weights_to_8_bits(rand(1, hidden, hidden) * 0.03)
    y = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    AdaptedProjection(Packed(w8, ws), adapters.pool, tokens)(x, adapters.segments, y, workspace)
    ref = adapters.add(x, x.double() @ _values(w8, ws)[0].t())
    print(f"adapted projection in 8 bits: relative error {((y.double() - ref).norm() / ref.norm()).item():.4f}")
    adapters.close()

    # attention between four adapted projections
    block, four, layers, x4, y4, batch = attention_example(rand)
    through = lambda i, rows: four[i].add(rows, rows.double() @ _values(*layers[i])[0].t())  # noqa: E731
    q64, k64, v64 = (through(i, x4).view(x4.shape[0], -1, 128) for i in range(3))
    ref = through(3, attention_reference(q64, k64, v64, *batch).flatten(1))
    print(f"attention between adapted projections in 8 bits: off by {((y4.double() - ref).norm() / ref.norm()).item():.4f} of the result")
    for a in four:
        a.close()

    # the experts
    gate_up, gs = weights_to_8_bits(rand(experts, 2 * inner, hidden) * 0.03)
    down, ds = weights_to_8_bits(rand(experts, hidden, inner) * 0.04)
    top, ids = torch.topk(rand(tokens, experts), picks, dim=1)
    weights, ids = torch.softmax(top, dim=1), ids.to(torch.int32)
    ids[::7, 1] = -1  # held elsewhere
    z = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    ExpertLayer(Packed(gate_up, gs), Packed(down, ds), picks, tokens)(x, ids, weights.contiguous(), z)
    ref = reference(x, ids, weights, _values(gate_up, gs), _values(down, ds))
    print(f"layer of experts in 8 bits: relative error {((z.double() - ref).norm() / ref.norm()).item():.4f}")


if __name__ == "__main__":
    main()
