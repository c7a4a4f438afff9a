"""Waits of the bf16 window kernel that give up."""
import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,n,left", [(1, 500, 200), (3, 6000, 700)])
@pytest.mark.parametrize("step", [0, 2, 6])
def test_a_wait_that_runs_out_ends_the_kernel_with_a_status(d, batch, n, left, step):
    """The loader is told (diagnostic hook) to leave out the key rows of one step, with a limit of about a millisecond: the waits for
    them run out, the kernel records CA_ERR_TIMEOUT, releases its tensor memory and returns.  With the hook cleared the next call
    on the same workspace gives what it gave before.  Of few pieces of work (a CTA each) and of more than there are SMs."""
    lib = binding.load_library()
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    q, k, v = (torch.randn((batch, h, n, d), generator=g, device=DEV).to(torch.bfloat16) for h in (8, 2, 2))
    plan = binding.WindowPlan(binding.make_window_problem(batch, 8, 2, n, n, d, "bf16", left, 0, 4), DEV)
    good = [x.clone() for x in plan.window_attention_fwd(q, k, v)]
    assert plan.last_status() == 0
    try:
        lib.ca_debug_attn_wait(2_000_000, step)
        plan.window_attention_fwd(q, k, v)
        torch.cuda.synchronize()
        assert plan.last_status() == binding.CA_ERR_TIMEOUT
    finally:
        lib.ca_debug_attn_wait(0, -1)
    plan.O.zero_()
    O, lse = plan.window_attention_fwd(q, k, v)
    assert plan.last_status() == 0
    assert torch.equal(O, good[0]) and torch.equal(lse, good[1])
    see = ref.window_mask(n, n, left, 0, 4, DEV)[-300:]
    o, l64, bound, lb, empty = ref.attend(q[0, 5, -300:].double(), k[0, 1].double(), v[0, 1].double(), see, d ** -0.5, torch.bfloat16, True)
    ref.check(O[0, 5, -300:], o, bound, "after it")
