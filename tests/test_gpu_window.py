"""Attention over a sliding window with first tokens that stay visible, against the plain form in 64 bits."""
import math

import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
KERNELS = [("bf16", 0), ("bf16", binding.CA_ATTN_FP32), ("fp32", 0), ("fp32", binding.CA_ATTN_FP32)]


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows(g, shape, dtype, layout="dense", gain=1.0):
    B, H, n, d = shape
    if layout == "rows_first":
        return (torch.randn((B, n, H, d), generator=g, device=DEV) * gain).to(DT[dtype]).transpose(1, 2)
    if layout == "room":
        return (torch.randn((B, H, n, d + 16), generator=g, device=DEV) * gain).to(DT[dtype])[..., 8:8 + d]
    return (torch.randn(shape, generator=g, device=DEV) * gain).to(DT[dtype])


def check(p, q, k, v, O, lse, len_q=None, len_k=None, heads=None, weights16=None):
    scale = p.softmax_scale if p.softmax_scale > 0 else 1 / math.sqrt(p.head_dim)
    group = p.heads_q // p.heads_kv
    dt = O.dtype
    weights16 = dt == torch.bfloat16 and not p.flags if weights16 is None else weights16
    for b in range(p.batch):
        a, n = (p.n_q if len_q is None else len_q[b]), (p.n_k if len_k is None else len_k[b])
        see = ref.window_mask(a, n, p.left, p.right, p.sinks, DEV)
        for h in heads or range(p.heads_q):
            want, l64, bound, lb, empty = ref.attend(q[b, h, :a].double(), k[b, h // group, :n].double(), v[b, h // group, :n].double(), see, scale,
                                                     dt, weights16)
            ref.check(O[b, h, :a], want, bound, f"item {b}, head {h}")
            ref.check_lse(lse[b, h, :a].double(), l64, lb, empty, f"item {b}, head {h}")


def run(p, q, k, v, **kw):
    plan = binding.WindowPlan(p, DEV)
    O, lse = plan.window_attention_fwd(q, k, v, **kw)
    assert plan.last_status() == 0
    return O, lse


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,n_k", [(1, 1), (1, 200), (7, 5), (64, 64), (127, 127), (128, 128), (129, 129), (200, 131), (131, 300), (257, 513),
                                     (600, 600)])
@pytest.mark.parametrize("left,right,sinks", [(-1, -1, 0), (-1, 0, 0), (0, 0, 0), (10, 0, 4), (100, 30, 1), (5, -1, 140), (64, 63, 0), (130, 0, 260)])
def test_sizes_and_windows(dtype, flags, d, n_q, n_k, left, right, sinks):
    g = generator(n_q + n_k + left)
    p = binding.make_window_problem(2, 2, 1, n_q, n_k, d, dtype, left, right, sinks, flags=flags)
    q, k, v = rows(g, (2, 2, n_q, d), dtype, gain=1.5), rows(g, (2, 1, n_k, d), dtype), rows(g, (2, 1, n_k, d), dtype)
    check(p, q, k, v, *run(p, q, k, v))


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("hq,kv", [(1, 1), (6, 3), (5, 1), (16, 2)])
@pytest.mark.parametrize("layout", ["rows_first", "room"])
def test_heads_and_strides(dtype, flags, hq, kv, layout):
    g = generator(hq)
    n, d = 333, 64
    p = binding.make_window_problem(2, hq, kv, n, n, d, dtype, 50, 20, 3, softmax_scale=0.3, flags=flags)
    q, k, v = rows(g, (2, hq, n, d), dtype, layout), rows(g, (2, kv, n, d), dtype, layout), rows(g, (2, kv, n, d), dtype, "dense")
    room = torch.full((2, n, hq, d + 8), 9.0, dtype=DT[dtype], device=DEV)
    O, lse = run(p, q, k, v, out=room.transpose(1, 2)[..., :d])
    check(p, q, k, v, O, lse)
    assert (room[..., d:] == 9.0).all()


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("d,left,right,sinks", [(64, 40, 0, 4), (128, -1, 0, 0), (128, 20, 7, 130)])
def test_ragged_batch(dtype, flags, d, left, right, sinks):
    """What stands behind a sequence is not a number and is not used; rows behind it are left as they were; more queries than
    keys leave rows that see nothing."""
    g = generator(d)
    len_q, len_k = [300, 1, 0, 129, 64, 300, 200], [300, 300, 77, 0, 10, 128, 200]
    B, n = len(len_q), 300
    p = binding.make_window_problem(B, 2, 2, n, n, d, dtype, left, right, sinks, flags=flags)
    q, k, v = (rows(g, (B, 2, n, d), dtype, "rows_first") for _ in range(3))
    for b in range(B):
        q[b, :, len_q[b]:] = float("nan")
        k[b, :, len_k[b]:] = float("nan")
        v[b, :, len_k[b]:] = float("inf")
    plan = binding.WindowPlan(p, DEV)
    plan.O.fill_(5.0)
    plan.lse.fill_(6.0)
    lq, lk = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (len_q, len_k))
    O, lse = plan.window_attention_fwd(q, k, v, len_q=lq, len_k=lk)
    assert plan.last_status() == 0
    check(p, q, k, v, O, lse, len_q, len_k)
    for b in range(B):
        assert (O[b, :, len_q[b]:] == 5.0).all() and (lse[b, :, len_q[b]:] == 6.0).all()
    # only one of the two
    O, lse = run(p, torch.nan_to_num(q), k, v, len_k=lk)
    check(p, torch.nan_to_num(q), k, v, O, lse, None, len_k)
    # lengths that are none: cut, recorded
    lq[0], lk[1] = 301, -1
    plan.window_attention_fwd(q, k, v, len_q=lq, len_k=lk)
    assert plan.last_status() == binding.CA_ERR_BAD_INDEX
    lq[0], lk[1] = 300, 300
    plan.window_attention_fwd(q, k, v, len_q=lq, len_k=lk)
    assert plan.last_status() == 0


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("left,right,sinks", [(300, 0, 20), (700, 700, 0), (-1, 0, 0), (1, 1, 1000)])
def test_long(dtype, flags, left, right, sinks):
    g = generator(17)
    n, d = 2500, 128
    p = binding.make_window_problem(1, 3, 1, n, n, d, dtype, left, right, sinks, flags=flags)
    q, k, v = rows(g, (1, 3, n, d), dtype, "rows_first", 2.0), rows(g, (1, 1, n, d), dtype, "rows_first"), rows(g, (1, 1, n, d), dtype)
    O, lse = run(p, q, k, v)
    check(p, q, k, v, O, lse)
    again = run(p, q, k, v)
    assert torch.equal(O, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype,flags", KERNELS)
def test_scores_that_climb_and_fall(dtype, flags):
    """The reference of the softmax moves from tile to tile, by more than 2^96 too."""
    n, d = 1000, 64
    g = generator(2)
    p = binding.make_window_problem(1, 2, 2, n, n, d, dtype, -1, -1, 0, softmax_scale=1.0, flags=flags)
    q, k, v = (rows(g, (1, 2, n, d), dtype, gain=0.1) for _ in range(3))
    q[..., 0] = 1.0
    ramp = torch.linspace(-300, 300, n, device=DEV).to(DT[dtype])
    k[0, 0, :, 0], k[0, 1, :, 0] = ramp, ramp.flip(0)
    check(p, q, k, v, *run(p, q, k, v))


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_numbers_outside_the_window(dtype, flags, d):
    """What a row does not see takes no part in it, in the same tile of keys too; rows that see it are not numbers."""
    n = 400
    g = generator(d)
    p = binding.make_window_problem(1, 1, 1, n, n, d, dtype, 30, 5, 2, flags=flags)
    q, k, v = (rows(g, (1, 1, n, d), dtype) for _ in range(3))
    clean = run(p, q, k, v)
    v2, k2 = v.clone(), k.clone()
    v2[0, 0, 150] = float("nan")
    v2[0, 0, 290, 3] = float("inf")
    k2[0, 0, 220] = float("nan")
    O, lse = run(p, q, k2, v2)
    i = torch.arange(n, device=DEV)
    sees = lambda j: (j <= i + 5) & (j >= i - 30)
    assert torch.isnan(O[0, 0, sees(150)].float()).all() and torch.isnan(O[0, 0, sees(220)].float()).all()
    assert torch.isinf(O[0, 0, sees(290), 3].float()).all()
    rest = ~(sees(150) | sees(290) | sees(220))
    see = ref.window_mask(n, n, 30, 5, 2, DEV)
    see[~rest] = False
    want, l64, bound, lb, empty = ref.attend(q[0, 0].double(), k[0, 0].double(), v[0, 0].double(), see, 1 / math.sqrt(d), DT[dtype],
                                             dtype == "bf16" and not flags)
    ref.check(O[0, 0, rest], want[rest], bound[rest], "rows that do not see them")
    # A value that is not a number leaves the weights as they are.  (The rows that see it may come from another kernel, whose sums have
    # another order: each is within its bound of the 64-bit value, so the two are within twice that.)
    _, _, _, lb, _ = ref.attend(q[0, 0].double(), k[0, 0].double(), v[0, 0].double(), ref.window_mask(n, n, 30, 5, 2, DEV), 1 / math.sqrt(d), DT[dtype],
                                dtype == "bf16" and not flags)
    ref.check(lse[0, 0, ~sees(220)], clean[1][0, 0, ~sees(220)].double(), 2 * lb[~sees(220)], "log-sum-exp")
    assert torch.isnan(lse[0, 0, sees(220)]).all()


def test_large_values_next_to_masked_ones():
    """Values near the end of the type's range, and keys whose scores are the lowest and the highest."""
    n, d = 300, 64
    g = generator(8)
    for dtype, flags in KERNELS:
        p = binding.make_window_problem(1, 1, 1, n, n, d, dtype, 20, 0, 1, flags=flags)
        q, k, v = (rows(g, (1, 1, n, d), dtype) for _ in range(3))
        v[0, 0, 100:110] *= 1e37
        k[0, 0, 200] = 1e4 * q[0, 0, 210]
        k[0, 0, 201] = -1e4 * q[0, 0, 210]
        check(p, q, k, v, *run(p, q, k, v))


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("second", [None, 0.0, -1.0, 3.0])
def test_scores_that_jump_by_the_range_of_the_type(dtype, flags, second):
    """A key some 2^120 to 2^130 times as heavy as those before it, and a second one `second` octaves from it, at any place of a step."""
    jumps = [20.0, 31.0, 33.0, 60.0, 100.0, 119.0, 120.0, 124.0, 125.0, 125.5, 126.0, 126.5, 127.0, 127.5, 128.0, 129.0, 130.0, 150.0, 255.0, 1000.0]
    B, n, d = 2 * len(jumps), 500, 64
    g = generator(77)
    q, k = (torch.zeros((B, 1, n, d), dtype=DT[dtype], device=DEV) for _ in range(2))
    v = rows(g, (B, 1, n, d), dtype)
    q[..., 0] = 1.0
    for b in range(B):
        x = jumps[b // 2]
        k[b, 0, 130 + b, 0] = x                             # (even and odd places: exponentials of both units)
        if second is not None:
            k[b, 0, 290 + 3 * b, 0] = x + second
    p = binding.make_window_problem(B, 1, 1, n, n, d, dtype, -1, 0, softmax_scale=math.log(2.0), flags=flags)
    O, lse = run(p, q, k, v)
    check(p, q, k, v, O, lse)


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["key", "gpu's", "infinite", "value", "query"])
@pytest.mark.parametrize("first", [0, 64])
def test_numbers_that_are_none_inside_the_window(dtype, flags, d, kind, first):
    """One bad row in each batch item, at 33 neighbouring places: the rows that see it are not numbers, the others as without it."""
    B, n, left = 33, 200, 40
    g = generator(d)
    q, k, v = (rows(g, (B, 1, n, d), dtype) for _ in range(3))
    q[..., 0] = q[..., 0].abs() + 0.5
    p = binding.make_window_problem(B, 1, 1, n, n, d, dtype, left, 0, flags=flags)
    bad = [x.clone() for x in (q, k, v)]
    words = torch.int16 if dtype == "bf16" else torch.int32
    nan = 0x7fff if dtype == "bf16" else 0x7fffffff
    at, items = torch.arange(B, device=DEV) + first, torch.arange(B, device=DEV)
    if kind == "key":
        bad[1][items, 0, at] = math.nan
    elif kind == "gpu's":
        bad[1].view(words)[items, 0, at, 5] = nan
    elif kind == "infinite":
        bad[1][items, 0, at, 0] = math.inf
    elif kind == "value":
        bad[2].view(words)[items, 0, at, 3] = nan
    else:
        bad[0].view(words)[items, 0, at, 7] = nan
    O, lse = run(p, *bad)
    row = torch.arange(n, device=DEV)
    hit = (row >= at[:, None]) & (row <= at[:, None] + (0 if kind == "query" else left))          # [B, n]
    columns = torch.ones(d, dtype=torch.bool, device=DEV)
    if kind == "value":
        columns = torch.arange(d, device=DEV) == 3
    wrong = hit[:, None, :, None] & columns
    assert torch.isnan(O[wrong]).all(), int((~torch.isnan(O[wrong])).sum())
    want, want_lse = run(p, q, k, v)
    if kind != "value":
        assert torch.isnan(lse[hit[:, None]]).all()
        lse = torch.where(hit[:, None], want_lse, lse)
    check(p, q, k, v, torch.where(wrong, want, O), lse)


@pytest.mark.parametrize("dtype,flags", KERNELS)
@pytest.mark.parametrize("n", [40, 700])
def test_sums_of_the_largest_values(dtype, flags, n):
    """Values of half the largest number, whose sums overflow before the division; behind a key that takes all the weight, nothing."""
    d, at = 64, n - 20
    q, k, v = (torch.zeros((1, 1, n, d), dtype=DT[dtype], device=DEV) for _ in range(3))
    q[..., 0], k[..., 0], v[:] = 1.0, -140.0, torch.finfo(DT[dtype]).max / 2
    k[0, 0, at, 0], v[0, 0, at] = 140.0, torch.linspace(-1, 1, d, device=DEV).to(DT[dtype])
    p = binding.make_window_problem(1, 1, 1, n, n, d, dtype, -1, 0, softmax_scale=1.0, flags=flags)
    O, lse = run(p, q, k, v)
    check(p, q, k, v, O, lse)


def test_graphs_streams_and_shared_workspace():
    g = generator(4)
    plans = []
    for n, left in ((500, 60), (900, 200)):
        p = binding.make_window_problem(1, 4, 2, n, n, 64, "bf16", left, 0, 4)
        q, k, v = rows(g, (1, 4, n, 64), "bf16"), rows(g, (1, 2, n, 64), "bf16"), rows(g, (1, 2, n, 64), "bf16")
        plan = binding.WindowPlan(p, DEV)
        want = plan.window_attention_fwd(q, k, v)[0].clone()
        plans.append((plan, q, k, v, want))
    size = max(x[0].ws.numel() for x in plans)
    shared = torch.zeros(size, dtype=torch.uint8, device=DEV)
    kept = [x[0].ws for x in plans]
    graphs = []
    for plan, q, k, v, _ in plans:
        plan.ws = shared
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.window_attention_fwd(q, k, v)
        graphs.append(graph)
        plan.O.zero_()
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for plan, q, k, v, want in plans:
        assert torch.equal(plan.O, want)
        plan.O.zero_()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for x, ws, s in zip(plans, kept, streams):
        x[0].ws = ws
    for _ in range(10):
        for (plan, q, k, v, _), s in zip(plans, streams):
            plan.window_attention_fwd(q, k, v, stream=s)
    torch.cuda.synchronize()
    for plan, q, k, v, want in plans:
        assert torch.equal(plan.O, want)


@pytest.mark.parametrize("dtype,flags", KERNELS)
def test_strides_beyond_32_bits(dtype, flags):
    """Batch items more than 2^31 elements apart, in inputs and output."""
    n, d = 200, 64
    far = 2 ** 31 + 64
    g = generator(6)
    p = binding.make_window_problem(2, 1, 1, n, n, d, dtype, 30, 0, 2, flags=flags)
    store = torch.empty((far + 4 * n * d,), dtype=DT[dtype], device=DEV)
    view = lambda i: store.as_strided((2, 1, n, d), (far, n * d, d, 1), i * n * d)
    q, k, v, out = (view(i) for i in range(4))
    for x in (q, k, v):
        x.copy_(rows(g, (2, 1, n, d), dtype))
    O, lse = run(p, q, k, v, out=out)
    check(p, q, k, v, O, lse)


@pytest.mark.parametrize("dtype,flags", KERNELS)
def test_broadcast_keys_and_values(dtype, flags):
    """Keys and values that are the same for the whole batch (a stride of zero), one row of keys for all queries, one query."""
    g = generator(31)
    d = 64
    for n_q, n_k, left, right in ((300, 300, 40, 10), (1, 300, -1, -1), (300, 1, -1, -1)):
        p = binding.make_window_problem(3, 4, 2, n_q, n_k, d, dtype, left, right, 2, flags=flags)
        q = rows(g, (3, 4, n_q, d), dtype)
        k, v = (rows(g, (1, 2, n_k, d), dtype).expand(3, 2, n_k, d) for _ in range(2))
        check(p, q, k, v, *run(p, q, k, v))
        q1 = rows(g, (3, 1, n_q, d), dtype).expand(3, 4, n_q, d)
        check(p, q1, k, v, *run(p, q1, k, v))


def test_rows_at_any_16_bytes():
    """Outputs and inputs that start at a multiple of 16 bytes that is none of 32."""
    g = generator(32)
    n, d = 300, 128
    for dtype, flags in KERNELS:
        p = binding.make_window_problem(1, 3, 1, n, n, d, dtype, 70, 3, 1, flags=flags)
        step = 16 // torch.empty((), dtype=DT[dtype]).element_size()
        room = lambda h: (torch.randn((1, h, n, d + step), generator=g, device=DEV)).to(DT[dtype])[..., step:]
        q, k, v, out = room(3), room(1), room(1), room(3)
        assert out.data_ptr() % 32 == 16
        check(p, q, k, v, *run(p, q, k, v, out=out))


def test_many_short_sequences():
    """More pieces of work than SMs, most of a batch's rows missing, pieces of one key tile."""
    g = generator(33)
    B, n, d = 70, 520, 64
    len_q = [(37 * i) % 521 for i in range(B)]
    len_k = [(91 * i + 13) % 521 for i in range(B)]
    for dtype, flags in KERNELS:
        p = binding.make_window_problem(B, 4, 4, n, n, d, dtype, 100, 0, 3, flags=flags)
        q, k, v = (rows(g, (B, 4, n, d), dtype, "rows_first") for _ in range(3))
        plan = binding.WindowPlan(p, DEV)
        plan.O.fill_(3.0)
        O, lse = plan.window_attention_fwd(q, k, v, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (len_q, len_k)))
        assert plan.last_status() == 0
        check(p, q, k, v, O, lse, len_q, len_k, heads=[0, 3])
        for b in range(B):
            assert (O[b, :, len_q[b]:] == 3.0).all()


def test_same_results_as_one_token_at_a_time():
    """The last row of a causal window and the cache's attention of one token see the same keys."""
    g = generator(12)
    n, d, hq, kv = 700, 128, 8, 2
    q, k, v = rows(g, (1, hq, n, d), "bf16"), rows(g, (1, kv, n, d), "bf16"), rows(g, (1, kv, n, d), "bf16")
    p = binding.make_window_problem(1, hq, kv, n, n, d, "bf16", 100, 0, 6)
    O, lse = run(p, q, k, v)
    cache = binding.PagedCache(binding.make_cache_problem(1, hq, kv, d, "bf16", 32, 22, 22, left=100, sinks=6), DEV,
                               page_table=torch.arange(22, device=DEV).flip(0).reshape(1, 22).int().contiguous())
    cache.cache_append(k, v)
    cache.lengths.fill_(n)
    one, l1 = cache.paged_attention_fwd(q[:, :, -1:])
    see = ref.window_mask(n, n, 100, 0, 6, DEV)[-1:]
    for h in range(hq):
        _, _, bound, lb, _ = ref.attend(q[0, h, -1:].double(), k[0, h // 4].double(), v[0, h // 4].double(), see, 1 / math.sqrt(d), torch.bfloat16, True)
        ref.check(one[0, h], O[0, h, -1:].double(), 2 * bound, "one token")
        ref.check(l1[0, h], lse[0, h, -1:].double(), 2 * lb, "one token's log-sum-exp")
