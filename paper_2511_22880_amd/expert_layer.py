"""A block of a mixture-of-experts model whose frozen weights are held in 8 bits, with LoRA adapters on its projection.

Two parts, each one path through the library as a serving program takes it; every buffer is made once, nothing is allocated or waited
for in a step, and the host never learns which tokens picked which experts:

    AdaptedProjection   y = x W + s_a (x A_a) B_a     lora_rows_quantize, lora_linear_scaled, lora_apply
    ExpertLayer         z = sum over picks of weight * W_down_e (silu(W_gate_e x) * W_up_e x)
                        lora_experts_group, lora_rows_quantize, lora_experts_linear_scaled (gate and up side by side), the
                        activation, lora_rows_quantize, lora_experts_linear_scaled on rows in expert order, lora_experts_combine

``python -m paper_2511_22880_amd.expert_layer`` runs both on random weights and checks them against 64 bits.
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


def main() -> None:
    import numpy as np

    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    hidden, inner, experts, picks, tokens = 1024, 512, 16, 4, 200
    x = rand(tokens, hidden).to(torch.bfloat16)

    # the projection: 8 adapters of ranks 8 to 64, every fifth token without one
    ranks = np.array([8, 16, 32, 64] * 2, dtype=np.int32)
    scales = (2.0 / ranks).astype(np.float32)
    arena = torch.zeros(L.lora_pool_bytes(hidden, hidden, ranks, scales), dtype=torch.uint8, device="cuda")
    pool = L.lora_pool_create(hidden, hidden, ranks, scales, arena)
    A = [(rand(hidden, int(r)) * 0.02).to(torch.bfloat16) for r in ranks]
    B = [(rand(int(r), hidden) * 0.02).to(torch.bfloat16) for r in ranks]
    for a in range(len(ranks)):
        L.lora_pool_load(pool, a, A[a], B[a], src_is_device=True, stream=torch.cuda.current_stream())
    token_adapter = np.array([-1 if t % 5 == 4 else t % len(ranks) for t in range(tokens)], dtype=np.int32)
    seg = L.lora_segments_build(pool, token_adapter, torch.cuda.current_stream())
    workspace = torch.empty(max(256, L.lora_apply_workspace_bytes(pool, seg)), dtype=torch.uint8, device="cuda")
    w8, ws = weights_to_8_bits(rand(1, hidden, hidden) * 0.03)
    y = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    AdaptedProjection(Packed(w8, ws), pool, tokens)(x, seg, y, workspace)
    ref = x.double() @ _values(w8, ws)[0].t()
    for t, a in enumerate(token_adapter):
        if a >= 0:
            ref[t] += float(scales[a]) * (x[t].double() @ A[a].double()) @ B[a].double()
    print(f"adapted projection in 8 bits: relative error {((y.double() - ref).norm() / ref.norm()).item():.4f}")
    L.lora_segments_destroy(seg)
    L.lora_pool_destroy(pool)

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
