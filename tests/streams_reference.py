"""Plain implementations in 64 bits of rotary positions, the paged cache and windowed attention, and how far a kernel's
result may be from them.

Bounds count roundings.  A value that is rounded to a type once is off by at most eps/2 of itself (u = eps/2: bf16 2^-8, fp32
2^-24).  With q, k, v as they are stored:
  logits   a sum of d products in fp32, in any order: |error| <= (d + 2) u32 sum |q_i k_i| s, with the scaling
           (accumulators that cut instead of rounding: 2 u32 for u32)
  exp2     of x = logit - m in log2 units: the subtraction and the unit's own 2^-22 relative, |x| u32 from rounding x
  weights  p_j off by a factor e^(2 E) with E the error of logit and exp2 (numerator and reference)
  sums     n terms in fp32: 2 n u32 relative to the sum of magnitudes
  bf16 P   one more u of bf16 relative to each weight, not in their sum
so |o - o64| <= (2 E + 4 n u32 [+ u_bf16]) * (weighted mean of |v|) (1 + E) + u_out |o64|, and the log-sum-exp is off by
at most E + 2 n u32 + 4 u32 (1 + |lse|)."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U32 = 2.0 ** -24


def rotate(x, pos, freqs, pairs, adjacent, inverse=False):
    """x [B, H, n, d] float64, pos [B or 1, n, axes]."""
    R = sum(pairs)
    y = x.clone()
    c = 0
    for a, count in enumerate(pairs):
        for _ in range(count):
            t = pos[..., a].double() * freqs[c] * (-1.0 if inverse else 1.0)
            i, j = (2 * c, 2 * c + 1) if adjacent else (c, R + c)
            cos, sin = torch.cos(t).unsqueeze(1), torch.sin(t).unsqueeze(1)
            y[..., i], y[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., i] * sin + x[..., j] * cos
            c += 1
    return y


def rotate_bound(x, pairs, adjacent, dtype, got64):
    """The phase in half turns is rounded to fp32 once (|t| <= pi: pi u32 of the angle), sine and cosine are off by 2 ulp, each
    product and the sum are rounded: (pi + 4 + 3) u32 (|x| + |y|) < 11 u32 (|x| + |y|); then one rounding to the type."""
    R = sum(pairs)
    size = torch.zeros_like(x)
    for c in range(R):
        i, j = (2 * c, 2 * c + 1) if adjacent else (c, R + c)
        size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return 11 * U32 * size + (U[dtype] * got64.abs() if dtype != torch.float32 else 0.0) * (1 + 1e-6) + 1e-38


def attend(q, k, v, visible, scale, storage, bf16_weights):
    """q [r, d], k and v [n, d] float64, visible [r, n].  Result, log-sum-exp and their bounds."""
    s = torch.where(visible, (q @ k.T) * scale, torch.tensor(-math.inf, dtype=torch.float64, device=q.device))
    v = torch.where(visible.any(0).unsqueeze(1), v, torch.zeros((), dtype=torch.float64, device=q.device))
    kk = torch.where(visible.any(0).unsqueeze(1), k, torch.zeros((), dtype=torch.float64, device=q.device))
    lse = torch.logsumexp(s, dim=1) if s.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    empty = torch.isinf(lse) & (lse < 0)
    w = torch.exp(s - torch.where(empty, torch.zeros_like(lse), lse).unsqueeze(1))
    w = torch.where(visible, w, torch.zeros_like(w))
    o = w @ v
    mean = w @ v.abs()
    d, n = q.shape[1], max(1, int(visible.sum(1).max())) if visible.numel() else 1
    sizes = torch.where(visible, (q.abs() @ kk.abs().T) * scale, torch.zeros_like(s))
    top = sizes.amax(1) if s.shape[1] else torch.zeros_like(lse)
    reach = 2 * top / math.log(2.0)                               # |logit - m| in log2 units at most
    E = 2 * (d + 3) * U32 * top + 2.0 ** -22 + 2 * reach * U32
    n_rel = 4 * n * U32
    bound = (2 * E + n_rel + (U[torch.bfloat16] if bf16_weights else 2.0 ** -15)).unsqueeze(1) * mean * (1 + E).unsqueeze(1)
    bound = bound + U[storage] * (o.abs() + bound) + 1e-30
    lse_bound = E + n_rel + 4 * U32 * (1 + torch.where(empty, torch.zeros_like(lse), lse).abs())
    return o, lse, bound, lse_bound, empty


def window_mask(len_q, len_k, left, right, sinks, device):
    p = torch.arange(len_q, device=device).unsqueeze(1) + (len_k - len_q)
    j = torch.arange(len_k, device=device)
    m = torch.ones((len_q, len_k), dtype=torch.bool, device=device)
    if right >= 0:
        m &= j <= p + right
    if left >= 0:
        m &= (j >= p - left) | (j < sinks)
    return m


def check(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    if bad.any():
        at = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} values beyond their bound, first at {at}: {float(got[at])}, "
                             f"{float(want[at])} within {float(bound[at] if torch.is_tensor(bound) else bound)}")


def check_lse(got, want, bound, empty, what):
    assert torch.equal(torch.isinf(got) & (got < 0), empty), f"{what}: rows that see nothing"
    check(torch.where(empty, torch.zeros_like(got), got), torch.where(empty, torch.zeros_like(want), want), bound, what)
