"""The bounds of stream_bounds tell a product that lost its lower half from one that did not: mistakes planted in 64 bits."""
import pytest
import torch

import stream_bounds as sb


def upper(x, bits):
    """x rounded to so many significant bits."""
    m, e = torch.frexp(x)
    return torch.ldexp((m * 2.0 ** bits).round() / 2.0 ** bits, e)


def rows(seed, n, d, dtype):
    g = torch.Generator()
    g.manual_seed(seed)
    q, k = torch.zeros((96, d), dtype=torch.float64), torch.zeros((n, d), dtype=torch.float64)
    at = [0, d // 2 - 3, d // 2 + 1, d - 1]
    q[:, at], k[:, at] = (torch.randn((m, 4), generator=g, dtype=torch.float64).to(dtype).double() for m in (96, n))
    return q, k, torch.randn((n, d), generator=g, dtype=torch.float64).to(dtype).double()


def exceeded(got, want, bound):
    return bool(((got - want).abs() > bound).any())


@pytest.mark.parametrize("n", [1, 2, 7, 12])
@pytest.mark.parametrize("d", [64, 128])
def test_lost_lower_halves_exceed_the_bounds(n, d):
    see = torch.ones((96, n), dtype=torch.bool)
    q, k, v = rows(n, n, d, torch.float32)
    o, lse, bound, lse_bound = sb.attend(q, k, v, see, 0.75, torch.float32, 4, *sb.WINDOW["fp32", 0])
    # tf32 keeps 11 significant bits of an operand
    assert exceeded(sb.attend(q, k, upper(v, 11), see, 0.75, torch.float32, 4, 0.0, 0.0)[0], o, bound)
    assert exceeded(sb.attend(q, upper(k, 11), v, see, 0.75, torch.float32, 4, 0.0, 0.0)[1], lse, lse_bound)
    assert exceeded(sb.attend(upper(q, 11), k, v, see, 0.75, torch.float32, 4, 0.0, 0.0)[1], lse, lse_bound)
    # and weights of 11 bits, normalised by the sum of the whole ones
    w = torch.exp((q @ k.T) * 0.75 - ((q @ k.T) * 0.75).amax(1, keepdim=True))
    if n > 2:
        assert exceeded((upper(w, 11) @ v) / w.sum(1, keepdim=True), o, bound)
