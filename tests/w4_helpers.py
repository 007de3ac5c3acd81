"""What the tests of the decoding operators share: the operators' definitions in 64 bits, with bounds on what the kernels' roundings
may do to each value.  u32 is the largest relative error of one fp32 addition in any rounding direction (the tensor cores cut
off), half[dtype] that of one rounding to dtype."""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -23
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
COLUMN_OF_NIBBLE = (0, 2, 4, 6, 1, 3, 5, 7)


def decode(codes: torch.Tensor) -> torch.Tensor:
    """codes uint8 [..., C/2] as integers code - 8, float64 [..., C]."""
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
    for nibble, column in enumerate(COLUMN_OF_NIBBLE):
        out[..., column::8] = ((codes[..., nibble // 2::4] >> (4 * (nibble % 2))) & 15).to(torch.float64) - 8.0
    return out


def encode(q: torch.Tensor) -> torch.Tensor:
    """Integers -8..7 [..., C] as codes uint8 [..., C/2]."""
    code = (q + 8).to(torch.uint8)
    out = torch.zeros(*q.shape[:-1], q.shape[-1] // 2, dtype=torch.uint8, device=q.device)
    for nibble, column in enumerate(COLUMN_OF_NIBBLE):
        out[..., nibble // 2::4] |= code[..., column::8] << (4 * (nibble % 2))
    return out


def weights(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    """[..., N, C] in 64 bits."""
    q = decode(codes)
    s = scales.to(torch.float64).transpose(-1, -2)
    return (q.unflatten(-1, (s.shape[-1], -1)) * s.unsqueeze(-1)).flatten(-2)


def random_w4(gen, std, *shape, group):
    """Random codes and scales of matrices `shape` = [..., N, C]; every code occurs."""
    *lead, N, C = shape
    q = torch.empty(*shape, device="cuda").normal_(0.0, 3.0, generator=gen).round_().clamp_(-8, 7)
    scales = torch.empty(*lead, C // group, N, dtype=torch.bfloat16, device="cuda").uniform_(0.5, 1.5, generator=gen).mul_(std / 3.0)
    return encode(q), scales


def matvec(w: torch.Tensor, x: torch.Tensor):
    """x [M, C] times w [N, C] (64 bits): the products, and a bound on fp32 sums in any order before the final rounding (C
    additions and one scaling per group at most)."""
    return x @ w.T, (x.shape[-1] + 8) * U32 * (x.abs() @ w.abs().T)


def layer(x, wr, bias, wg, wu, wd, K, renorm, idx, dtype):
    """The layer in 64 bits on given picks idx [T, K], with a bound per value.  wg, wu, wd: e -> matrix in 64 bits.
    Returns (logits, their bound, weights, y, bound of y)."""
    T, H = x.shape
    logits, dl = matvec(wr, x)
    if bias is not None:
        logits, dl = logits + bias.to(torch.float64), dl + U32 * (logits.abs() + bias.to(torch.float64).abs())
    dmax = dl.masked_fill(~dl.isfinite(), 0).amax(1, keepdim=True)
    p = torch.softmax(logits, 1)
    w = p.gather(1, idx)
    # exponents off by at most two logits' errors, their fp32 difference's rounding, expf's two ulps, a sum of E numbers and a quotient
    rel = 2 * dmax + U32 * (logits.masked_fill(~logits.isfinite(), 0).abs().amax(1, keepdim=True) * 2 + logits.shape[1] + 8)
    if renorm:
        w = w / w.sum(1, keepdim=True)
        rel = 2 * rel + U32 * (K + 2)
    y = torch.zeros_like(x)
    bound = torch.zeros_like(x)
    half = HALF[dtype]
    for e in idx.unique().tolist():
        t, k = (idx == e).nonzero(as_tuple=True)
        a = x[t]
        (g, dg), (u, du) = matvec(wg(e), a), matvec(wu(e), a)
        sg = torch.sigmoid(g)
        s = g * sg * u
        # |silu'| <= 1.1; expf, the sum, the quotient and the product: a few roundings
        ds = 1.1 * dg * (u.abs() + du) + (g * sg).abs() * du + 8 * U32 * s.abs()
        # (held as fp32, or as two bf16 numbers: what a value rounds to, and what that left)
        ds = ds + (half if dtype == torch.float32 else half * half) * (s.abs() + ds)
        down = wd(e)
        o, do = matvec(down, s)
        do = do + ds @ down.abs().T
        wt = w[t, k].unsqueeze(1)
        y[t] += wt * o
        bound[t] += wt * (do + (rel[t] + K * U32) * (o.abs() + do))
    return logits, dl, w, y, bound + half * (y.abs() + bound)


def check_picks(idx, logits, dl):
    """The picks are the K largest of the logits, descending, up to what fp32 sums may differ by."""
    K = idx.shape[1]
    top = logits.gather(1, idx)
    slack = 2 * dl.amax(1)
    assert (top[:, :-1] - top[:, 1:] >= -slack[:, None]).all()
    rest = logits.scatter(1, idx, float("-inf"))
    assert (top[:, K - 1] - rest.amax(1) >= -slack).all()
    assert all(len(set(r)) == K for r in idx.tolist())


def assert_within(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor, what: str):
    excess = ((got.to(torch.float64) - want).abs() / bound.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    assert not np.isnan(excess) and excess <= 1.0, f"{what}: {excess:.3g} times what the roundings allow"
