"""Attention, rotation and 8-bit pages in 64 bits, plain and row by row, with the error that the kernels may have by arithmetic.

Every bound counts roundings: half a step of an output's type (bf16 2^-8, fp32 2^-24 relative to the value), the rounding of weights
to bf16 on the tensor cores, d products summed in fp32 for a logit, N weights summed in fp32."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attend_rows(q, k, v, limits, scale, self_lse=None, weight_half_step=0.0):
    """One head: (out, lse, bound of |out| error but for the last rounding, bound of |lse| error), all fp64.

    q [n][d], k and v [N][d], limits [n].  Rows of v that no row sees are not read (they may hold NaN)."""
    n, d = q.shape
    N = k.shape[0]
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros((n, d), dtype=torch.float64, device=q.device)
    lse = torch.full((n,), -math.inf, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    delta = torch.zeros_like(lse)
    for i in range(n):
        m = int(limits[i])
        extra = -math.inf if self_lse is None else float(self_lse[i])
        if m == 0:
            lse[i] = extra
            continue
        s = k[:m] @ q[i] * scale
        total = torch.logsumexp(torch.cat([s, s.new_tensor([extra])]), 0)
        w = torch.exp(s - total)
        out[i] = w @ v[:m]
        size[i] = w @ v[:m].abs()
        lse[i] = total
        # a logit: d products and sums in fp32 (2^-24 each, of the sum of magnitudes), a few roundings of the scaled difference
        delta[i] = (d + 8) * 2.0 ** -24 * float((k[:m].abs() @ q[i].abs()).max()) * scale + 2.0 ** -21 * (1 + float(s.abs().max()))
    rel = 2 * delta + (N + 64) * 2.0 ** -24
    return out, lse, size * (rel[:, None] + weight_half_step), delta + (N + 64) * 2.0 ** -24 + 2.0 ** -22 * lse.abs().nan_to_num(0, 0, 0)


def check_rows(got, got_lse, want, want_lse, err, lse_err, what=""):
    got64 = got.double()
    room = err + HALF_STEP[got.dtype] * (want.abs() + err) + 1e-30
    off = (got64 - want).abs()
    assert torch.isfinite(got64).all(), f"{what}: not finite"
    worst = float((off / room).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound"
    if got_lse is not None:
        empty = torch.isneginf(want_lse)
        assert torch.equal(torch.isneginf(got_lse), empty), f"{what}: rows that see nothing"
        off = (got_lse.double() - want_lse).abs()[~empty] / lse_err[~empty]
        assert off.numel() == 0 or float(off.max()) <= 1.0, f"{what}: log-sum-exp {float(off.max()):.2f} times the bound"


def turned(x, pos, freq, rotary_dim, pairing, magnitude=1.0):
    """Rows x [..., tokens, d] in fp64, turned with cosines and sines that are rounded to 32 bits."""
    y = x.double().clone()
    half = rotary_dim // 2
    angle = pos.double()[:, None] * torch.as_tensor(freq, dtype=torch.float64, device=x.device)
    c, s = (angle.cos() * magnitude).float().double(), (angle.sin() * magnitude).float().double()
    for t in range(half):
        a, b = (2 * t, 2 * t + 1) if pairing else (t, t + half)
        xa, xb = y[..., a].clone(), y[..., b].clone()
        y[..., a] = xa * c[:, t] - xb * s[:, t]
        y[..., b] = xa * s[:, t] + xb * c[:, t]
    return y


def quantised(rows):
    """A page's 64 rows [..., 64, d] of one head -> (codes uint8, scale fp32), by the definition: a quotient of fp32 numbers each."""
    x = rows.float()
    mag = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    top = mag.amax((-2, -1))
    scale = top / torch.full_like(top, 448.0)
    by = torch.where(scale > 0, scale, torch.ones_like(scale))
    ratio = (x / by[..., None, None]).clamp(-448.0, 448.0)
    return ratio.to(torch.float8_e4m3fn).view(torch.uint8), scale


def dequantised(codes, scale):
    return codes.view(torch.float8_e4m3fn).double() * scale.double()[..., None, None]
