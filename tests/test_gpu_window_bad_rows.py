"""Rows of windows whose every visible score is no number."""
import math

import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("fp32", 0), ("bf16", binding.CA_ATTN_FP32), ("fp32", binding.CA_ATTN_FP32)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["query", "key"])
@pytest.mark.parametrize("shift", [16, 0, 31])
def test_a_row_whose_only_score_is_no_number(dtype, flags, d, kind, shift):
    """Windows of one key, rows and keys apart, so that a tile of rows goes on to keys that the bad row does not see."""
    B, n_q = 33, 128
    n_k = n_q + shift
    g = generator(shift + d)
    q, k, v = (torch.randn((B, 1, n, d), generator=g, device=DEV).to(DT[dtype]) for n in (n_q, n_k, n_k))
    at, items = torch.arange(B, device=DEV), torch.arange(B, device=DEV)
    if kind == "query":
        q[items, 0, at, 7] = math.nan
    else:
        k[items, 0, at + shift, 7] = math.nan
    p = binding.make_window_problem(B, 1, 1, n_q, n_k, d, dtype, 0, 0, flags=flags)
    plan = binding.WindowPlan(p, DEV)
    O, lse = plan.window_attention_fwd(q, k, v)
    assert plan.last_status() == 0
    assert torch.isnan(O[items, 0, at].float()).all() and torch.isnan(lse[items, 0, at]).all()
    # every other row is the value of the one key that it sees, with weight 1 (as tf32 halves 2^-24 of it is cut)
    O[items, 0, at] = v[items, 0, at + shift]
    want = v[:, :, shift:].double()
    ref.check(O, want, want.abs() * 2.0 ** -23, "the other rows")
    lse[items, 0, at] = 0.0
    assert torch.isfinite(lse).all()
