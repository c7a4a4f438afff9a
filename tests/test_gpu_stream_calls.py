"""Calls for streams of tokens beside one another and beside other work."""
import threading

import pytest
import torch

from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def busy():
    """Some tens of milliseconds of work on the current stream."""
    torch.cuda._sleep(100_000_000)


def on_a_side_stream(make, call, want):
    """`call` on another stream right behind `make`, which has buffers filled on a busy one: what it gives is not touched afterwards."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy()
    handle = make()
    got = call(handle, side)
    side.synchronize()
    first = [x.clone() for x in got]
    torch.cuda.synchronize()
    for x, y, z in zip(first, got, want):
        assert torch.equal(x, z) and torch.equal(y, z)


def test_a_plan_is_ready_for_any_stream():
    g = generator(1)
    n, d = 700, 64
    q, k, v = (torch.randn((1, h, n, d), generator=g, device=DEV).to(torch.bfloat16) for h in (4, 2, 2))
    problem = binding.make_window_problem(1, 4, 2, n, n, d, "bf16", 60, 0, 4)
    make = lambda: binding.WindowPlan(problem, DEV)
    call = lambda plan, stream: plan.window_attention_fwd(q, k, v, stream=stream)
    on_a_side_stream(make, call, [x.clone() for x in call(make(), None)])


@pytest.mark.parametrize("per", [4, 300])
def test_a_cache_is_ready_for_any_stream(per):
    g = generator(2)
    n, d = 60, 64
    k, v = (torch.randn((1, 2, n, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((1, 4, 1, d), generator=g, device=DEV).to(torch.bfloat16)
    table = torch.arange(per, device=DEV).flip(0).reshape(1, per).int().contiguous()
    problem = binding.make_cache_problem(1, 4, 2, d, "bf16", 16, per, per)

    def call(cache, stream):
        cache.cache_append(k, v, stream=stream)
        return cache.paged_attention_fwd(q, appended=n, stream=stream) + (cache.K_pages, cache.V_pages)

    make = lambda: binding.PagedCache(problem, DEV, page_table=table)
    on_a_side_stream(make, call, [x.clone() for x in call(make(), None)])


@pytest.mark.parametrize("path", ["forward", "adaptive", "basic", "rotary"])
def test_a_clustering_plan_is_ready_for_any_stream(path):
    g = generator(3)
    n, d = 700, 64
    q, k, v = (torch.randn((1, 2, n, d), generator=g, device=DEV) for _ in range(3))
    pos = torch.arange(n, dtype=torch.int32, device=DEV).view(1, n, 1)
    problem = binding.make_problem(1, 2, n, n, d, "fp32", 64, 64, 4)
    make = lambda: binding.Plan(problem, DEV)
    rows_q, rows_k, _ = make().basic_noise_rows()
    noise = [torch.randn((1, 2, r, d), generator=g, device=DEV) for r in (rows_q, rows_k)]

    def call(plan, stream):
        if path == "adaptive":
            return plan.forward_adaptive(q, k, v, 0.7, want_lse=True, stream=stream)
        if path == "basic":
            plan.cluster_qk_basic(q, k, v, *noise, stream=stream)
            plan.select_blocks(stream=stream)
            return plan.cluster_attention_fwd(stream=stream)
        args = dict(rotary=binding.Rotary(d, [16]), positions_q=pos) if path == "rotary" else {}
        return (plan.forward(q, k, v, stream=stream, **args),)

    on_a_side_stream(make, call, [x.clone() for x in call(make(), None)])


def cache_of(B, hq, kv, d, dtype, per, page_rows=16, **kw):
    table = torch.arange(B * per, device=DEV).flip(0).reshape(B, per).int().contiguous()
    return binding.PagedCache(binding.make_cache_problem(B, hq, kv, d, dtype, page_rows, B * per, per, **kw), DEV, page_table=table)


@pytest.mark.parametrize("per", [2, 40])
@pytest.mark.parametrize("batch", [3, 300])
def test_the_error_of_an_append_outlives_the_attention_behind_it(per, batch):
    """Until the next append, in caches of few rows and of many, of few sequences and of many."""
    g = generator(per)
    cache = cache_of(batch, 4, 2, 64, "bf16", per)
    k, v = (torch.randn((batch, 2, 5, 64), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((batch, 4, 1, 64), generator=g, device=DEV).to(torch.bfloat16)
    count = torch.full((batch,), 5, dtype=torch.int32, device=DEV)
    cache.paged_attention_fwd(q)
    assert cache.last_status() == 0                         # (no append so far)
    cache.cache_append(k, v, count=count)
    cache.paged_attention_fwd(q, appended=5)
    assert cache.last_status() == 0
    for bad in (6, -1):
        count[batch - 1] = bad
        cache.cache_append(k, v, count=count)
        for _ in range(2):
            cache.paged_attention_fwd(q, appended=5)
            assert cache.last_status() == binding.CA_ERR_BAD_INDEX
        count[batch - 1] = 5
        cache.cache_append(k, v, count=count)
        assert cache.last_status() == 0
        cache.paged_attention_fwd(q, appended=5)
        assert cache.last_status() == 0


def test_host_threads_call_the_same_kernels_at_other_sizes():
    """Shared memory of a launch goes by the heads that share a key head, by the number of clusters, by the rows."""
    d, calls = 64, []
    g = generator(5)
    for group in (1, 8, 3):
        cache = cache_of(4, group, 1, d, "bf16", 40)
        k, v, q = (torch.randn((4, h, n, d), generator=g, device=DEV).to(torch.bfloat16) for h, n in ((1, 300), (1, 300), (group, 1)))
        cache.cache_append(k, v)
        calls.append((lambda stream, c=cache, q=q: c.paged_attention_fwd(q, appended=300, stream=stream)[0], cache))
    for n in (600, 9000, 3000):
        plan = binding.Plan(binding.make_problem(1, 1, n, n, d, "bf16", 64, 64, 4), DEV)
        q, k, v = (torch.randn((1, 1, n, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(3))
        calls.append((lambda stream, p=plan, x=(q, k, v): p.forward(*x, stream=stream), plan))
    want = [call(None).clone() for call, _ in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    failed, got = [], [None] * len(calls)

    def work(i):
        try:
            for _ in range(60):
                got[i] = calls[i][0](streams[i])
        except Exception as e:  # noqa: BLE001
            failed.append((i, e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_a_problem_that_changes_does_not_change_what_was_made_for_it():
    """A cache that took the caller's later number of pages for its own would read behind its pools."""
    window, cache = binding.make_window_problem(1, 2, 2, 40, 40, 64, "bf16", 3, 0), binding.make_cache_problem(1, 2, 2, 64, "bf16", 16, 4, 4)
    plan = binding.make_problem(1, 1, 64, 64, 64, "fp32", 16, 16, 2)
    made = binding.WindowPlan(window, DEV), binding.PagedCache(cache, DEV), binding.Plan(plan, DEV)
    window.n_q, cache.pages, cache.pages_per_sequence, plan.n_q = 400, 1000, 1000, 640
    assert made[0].problem.n_q == 40 and made[1].problem.pages == made[1].problem.pages_per_sequence == 4 and made[2].problem.n_q == 64
