"""Attention of one new token over a cache in pages against the plain form in 64 bits."""
import math

import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def make(seed, lengths, hq, kv, d, dtype, page_rows, left=-1, sinks=0, garbage=True, spare=0, scale=0.0, gain=1.5):
    """A cache whose unused slots and pages are not numbers and whose unused table entries are no pages."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    B, per = len(lengths), max(1, -(-max(lengths) // page_rows)) + spare
    pages = B * per + 1
    table = torch.randperm(pages, generator=g, device=DEV)[:B * per].reshape(B, per).int()
    cache = binding.PagedCache(binding.make_cache_problem(B, hq, kv, d, dtype, page_rows, pages, per, left, sinks, scale), DEV)
    cache.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    for pool in (cache.K_pages, cache.V_pages):
        pool.fill_(float("nan") if garbage else 0.0)
    for b, n in enumerate(lengths):
        for first in range(0, n, page_rows):
            m = min(page_rows, n - first)
            for pool in (cache.K_pages, cache.V_pages):
                pool[table[b, first // page_rows], :, :m] = torch.randn((kv, m, d), generator=g, device=DEV).to(DT[dtype])
        table[b, -(-n // page_rows):] = -7
    cache.page_table.copy_(table)
    q = (torch.randn((B, hq, 1, d), generator=g, device=DEV) * gain).to(DT[dtype])
    return cache, q


def rows_of(cache, b, g, n):
    p = cache.problem
    pages = cache.page_table[b, :-(-n // p.page_rows)].long()
    return [pool[pages, g].reshape(-1, p.head_dim)[:n].double() for pool in (cache.K_pages, cache.V_pages)]


def check(cache, q, lengths, O, lse, only=None):
    p = cache.problem
    scale = p.softmax_scale if p.softmax_scale > 0 else 1 / math.sqrt(p.head_dim)
    group = p.heads_q // p.heads_kv
    for b, n in enumerate(lengths):
        j = torch.arange(n, device=DEV)
        see = (j >= n - 1 - p.left) | (j < p.sinks) if p.left >= 0 else torch.ones_like(j, dtype=torch.bool)
        for g in range(p.heads_kv):
            k, v = rows_of(cache, b, g, n)
            heads = slice(g * group, (g + 1) * group)
            want, l64, bound, lb, empty = ref.attend(q[b, heads, 0].double(), k, v, see.expand(group, n), scale, cache.dtype, False)
            ref.check(O[b, heads, 0], want, bound, f"sequence {b} of {n}, key head {g}")
            ref.check_lse(lse[b, heads, 0].double(), l64, lb, empty, f"sequence {b} of {n}, key head {g}")


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 1000]


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("hq,kv", [(1, 1), (2, 1), (6, 2), (12, 3), (10, 2), (24, 3), (16, 1), (12, 1), (34, 2), (40, 1)])
@pytest.mark.parametrize("page_rows,left,sinks", [(16, -1, 0), (100, 40, 3), (17, 0, 0), (64, 200, 70)])
def test_lengths_heads_windows(dtype, d, hq, kv, page_rows, left, sinks):
    cache, q = make(hq + page_rows, LENGTHS, hq, kv, d, dtype, page_rows, left, sinks)
    O, lse = cache.paged_attention_fwd(q)
    assert cache.last_status() == 0
    check(cache, q, LENGTHS, O, lse)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("lengths", [[20001], [1, 9000, 3], [5000] * 7])
@pytest.mark.parametrize("left,sinks", [(-1, 0), (4097, 130)])
def test_long_rows_are_split_and_joined(dtype, d, lengths, left, sinks):
    cache, q = make(len(lengths), lengths, 8, 2, d, dtype, 32, left, sinks)
    O, lse = cache.paged_attention_fwd(q)
    first = O.clone(), lse.clone()
    check(cache, q, lengths, O, lse)
    for _ in range(20):                                     # whichever CTA is last to arrive
        O, lse = cache.paged_attention_fwd(q)
        assert torch.equal(O, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("spare", [0, 20])
def test_more_sequences_than_threads_of_the_plan(spare):
    """Of a table of few rows (a CTA for each sequence and head) and of many (units added up by a launch of its own)."""
    lengths = [(7 * i) % 41 for i in range(2500)]
    cache, q = make(1, lengths, 2, 2, 64, "bf16", 16, spare=spare)
    O, lse = cache.paged_attention_fwd(q)
    assert cache.last_status() == 0
    check(cache, q, lengths[:60], O, lse)
    for at in (1023, 1024, 1025, 2047, 2048, 2499):
        n = lengths[at]
        k, v = rows_of(cache, at, 1, n)
        want, l64, bound, lb, empty = ref.attend(q[at, 1].double(), k, v, torch.ones((1, n), dtype=torch.bool, device=DEV), 1 / 8, cache.dtype, False)
        ref.check(O[at, 1], want, bound, f"sequence {at}")
        ref.check_lse(lse[at, 1].double(), l64, lb, empty, f"sequence {at}")


@pytest.mark.parametrize("batch", [1, 2, 127, 128, 129, 255, 256, 257, 300])
def test_batches_around_the_threads_of_a_cta(batch):
    g = torch.Generator()
    g.manual_seed(batch)
    lengths = [int(x) for x in torch.randint(0, 500, (batch,), generator=g)]
    lengths[-1] = 700
    cache, q = make(batch, lengths, 4, 2, 64, "bf16", 16, left=300, sinks=5)
    O, lse = cache.paged_attention_fwd(q)
    assert cache.last_status() == 0
    check(cache, q, lengths, O, lse)
    cache.page_table[batch - 1, 40] = cache.problem.pages
    cache.paged_attention_fwd(q)
    assert cache.last_status() == binding.CA_ERR_BAD_INDEX


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scale_large_scores_and_strided_rows(dtype):
    lengths = [300, 77]
    cache, q = make(2, lengths, 6, 2, 64, dtype, 16, scale=2.0, gain=8.0)
    wide = torch.zeros((2, 1, 6, 96), dtype=DT[dtype], device=DEV).transpose(1, 2)[..., 16:80]
    wide.copy_(q)
    out = torch.full((2, 1, 6, 72), 7.0, dtype=DT[dtype], device=DEV)
    O, lse = cache.paged_attention_fwd(wide, out=out.transpose(1, 2)[..., :64])
    check(cache, q, lengths, O, lse)
    assert (out[..., 64:] == 7.0).all()
    assert cache.paged_attention_fwd(q, want_lse=False)[1] is None


def test_rows_that_are_not_numbers_where_they_are_seen():
    cache, q = make(4, [50, 50, 50], 2, 1, 64, "bf16", 16, left=9, sinks=2)
    page = cache.page_table[0].long()
    cache.V_pages[page[1]] = float("inf")              # rows 16 .. 31 of sequence 0 are not visible
    cache.K_pages[page[1]] = float("nan")
    cache.V_pages[cache.page_table[1, 2].long(), :, 10] = float("inf")      # row 42 of sequence 1 is
    cache.K_pages[cache.page_table[2, 2].long(), :, 10] = float("nan")
    O, lse = cache.paged_attention_fwd(q)
    assert torch.isfinite(O[0].float()).all() and torch.isfinite(lse[:2]).all()
    assert torch.isinf(O[1].float()).all() and torch.isnan(O[2].float()).all() and torch.isnan(lse[2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("spare", [0, 20])
@pytest.mark.parametrize("kind", ["key", "infinite", "value"])
def test_a_row_that_is_no_number_anywhere(dtype, spare, kind):
    """One bad row in each sequence, at another place of a step and a unit in each."""
    lengths = [130] * 130
    cache, q = make(9, lengths, 2, 1, 64, dtype, 16, spare=spare)
    q[..., 0] = q[..., 0].abs() + 0.5
    items = torch.arange(130, device=DEV)
    page = cache.page_table[items, items // 16].long()
    words, nan = (torch.int16, 0x7fff) if dtype == "bf16" else (torch.int32, 0x7fffffff)
    if kind == "key":
        cache.K_pages.view(words)[page, 0, items % 16, 5] = nan
    elif kind == "infinite":
        cache.K_pages[page, 0, items % 16, 0] = math.inf
    else:
        cache.V_pages.view(words)[page, 0, items % 16, 3] = nan
    O, lse = cache.paged_attention_fwd(q)
    if kind == "value":
        assert torch.isnan(O[..., 3]).all() and torch.isfinite(lse).all()
        assert torch.isfinite(O.float()).sum() == O.numel() - O.numel() // 64
    else:
        assert torch.isnan(O).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [50, 3000])
def test_the_largest_values_at_weights_of_zero(dtype, n):
    """All keys but one are 400 octaves below it: their weights are zero in fp32, and their values, the largest of the type, nothing.  (Those
    of a part of the rows without that key add up to more than fp32 holds.)"""
    d = 64
    cache = binding.PagedCache(binding.make_cache_problem(1, 2, 1, d, dtype, 16, 200, 200, softmax_scale=1.0), DEV,
                               page_table=torch.arange(200, dtype=torch.int32, device=DEV)[None])
    k, v = torch.zeros((2, 1, 1, n, d), dtype=DT[dtype], device=DEV)
    k[..., 0], v[:] = -140.0, torch.finfo(DT[dtype]).max
    at = n - 20
    k[0, 0, at, 0], v[0, 0, at] = 140.0, torch.linspace(-1, 1, d, device=DEV).to(DT[dtype])
    q = torch.zeros((1, 2, 1, d), dtype=DT[dtype], device=DEV)
    q[..., 0] = 1.0
    cache.cache_append(k, v)
    O, lse = cache.paged_attention_fwd(q, appended=n)
    check(cache, q, [n], O, lse)


@pytest.mark.parametrize("spare", [0, 20])
def test_bad_pages_and_lengths_are_recorded(spare):
    cache, q = make(5, [40, 40], 2, 1, 64, "bf16", 16, garbage=False, spare=spare)
    good = cache.paged_attention_fwd(q)[0].clone()
    kept = cache.page_table[1, 1].clone()
    for bad in (cache.problem.pages, -1, 2 ** 31 - 1, -2 ** 31):
        cache.page_table[1, 1] = bad
        O, _ = cache.paged_attention_fwd(q)
        assert cache.last_status() == binding.CA_ERR_BAD_INDEX
        assert torch.equal(O[0], good[0]) and torch.isfinite(O.float()).all()
    cache.page_table[1, 1] = kept
    cache.lengths[0] = -3
    O, lse = cache.paged_attention_fwd(q)
    assert cache.last_status() == binding.CA_ERR_BAD_INDEX
    assert (O[0] == 0).all() and torch.isinf(lse[0]).all() and torch.equal(O[1], good[1])
    cache.lengths[0] = 2 ** 31 - 1
    O, lse = cache.paged_attention_fwd(q, appended=2 ** 31 - 1)             # both sequences: cut to the table's rows
    assert cache.last_status() == binding.CA_ERR_BAD_INDEX
    cache.lengths.fill_(40)
    assert torch.equal(cache.paged_attention_fwd(q)[0], good) and cache.last_status() == 0


def test_appended_rows_and_a_step_of_a_stream():
    """Rotary positions, rows into pages, attention, one token after another, against the rows of the whole stream: as a program
    that generates runs them.  The same captured into a graph and replayed."""
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    B, hq, kv, d, steps = 3, 8, 2, 64, 40
    rot = binding.Rotary(d, [8, 12, 12])
    start = torch.tensor([0, 5, 30], dtype=torch.int32, device=DEV)
    K, V = (torch.randn((B, kv, 80, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    Q = torch.randn((steps, B, hq, 1, d), generator=g, device=DEV).to(torch.bfloat16)
    pos = torch.stack((torch.arange(80, device=DEV), torch.arange(80, device=DEV) % 7, torch.arange(80, device=DEV) % 5), -1).int()
    Kr = binding.rotary_axes(rot, K, None, pos[None].contiguous())[0]
    per = 5
    problem = binding.make_cache_problem(B, hq, kv, d, "bf16", 16, B * per, per, left=25, sinks=4)
    results = []
    for graph in (False, True):
        cache = binding.PagedCache(problem, DEV, page_table=torch.randperm(B * per, generator=g, device=DEV).reshape(B, per).int())
        cache.cache_append(K[:, :, :30], V[:, :, :30], count=start, rotary=rot, positions=pos[None, :30].contiguous())
        cache.lengths.copy_(start)
        q, k, v = Q[0].clone(), torch.zeros((B, kv, 1, d), dtype=torch.bfloat16, device=DEV), torch.zeros((B, kv, 1, d), dtype=torch.bfloat16, device=DEV)
        at = torch.zeros((B, 1, 3), dtype=torch.int32, device=DEV)

        def step():
            qr = binding.rotary_axes(rot, q, None, at)[0]
            cache.cache_append(k, v, rotary=rot, positions=at)
            O, lse = cache.paged_attention_fwd(qr, appended=1)
            cache.lengths.add_(1)
            return qr, O, lse

        def feed(t):
            i = (start + t).long()
            b = torch.arange(B, device=DEV)
            q.copy_(Q[t])
            k.copy_(K[b, :, i].unsqueeze(2))
            v.copy_(V[b, :, i].unsqueeze(2))
            at.copy_(pos[i].unsqueeze(1))

        run = step
        if graph:
            cuda_graph = torch.cuda.CUDAGraph()
            feed(0)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
            cache.lengths.copy_(start)
            with torch.cuda.graph(cuda_graph):
                outs = step()
            run = lambda: (cuda_graph.replay(), outs)[1]
        kept = []
        for t in range(steps):
            feed(t)
            qr, O, lse = run()
            kept.append((O.clone(), lse.clone()))
            if t % 13 == 0:
                for b in range(B):
                    n = int(start[b]) + t + 1
                    j = torch.arange(n, device=DEV)
                    see = ((j >= n - 26) | (j < 4)).expand(4, n)
                    for h in range(kv):
                        want, l64, bound, lb, empty = ref.attend(qr[b, 4 * h:4 * h + 4, 0].double(), Kr[b, h, :n].double(), V[b, h, :n].double(), see,
                                                                 1 / 8, torch.bfloat16, False)
                        ref.check(O[b, 4 * h:4 * h + 4, 0], want, bound, f"step {t}")
                        ref.check_lse(lse[b, 4 * h:4 * h + 4, 0].double(), l64, lb, empty, f"step {t}")
        assert cache.last_status() == 0
        results.append(kept)
    for a, b in zip(*results):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_two_graphs_share_a_workspace_and_other_streams():
    one, q1 = make(21, [3000, 10], 8, 2, 64, "bf16", 16)
    two, q2 = make(22, [70, 5000], 8, 2, 64, "bf16", 16)
    want = one.paged_attention_fwd(q1)[0].clone(), two.paged_attention_fwd(q2)[0].clone()
    two.ws = one.ws
    graphs = []
    for cache, q in ((one, q1), (two, q2)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.paged_attention_fwd(q)
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(one.O, want[0]) and torch.equal(two.O, want[1])
    own = binding.PagedCache(two.problem, DEV, two.K_pages, two.V_pages, two.page_table, two.lengths)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):                                     # two calls at once, each with its workspace
        one.paged_attention_fwd(q1, stream=streams[0])
        own.paged_attention_fwd(q2, stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(one.O, want[0]) and torch.equal(own.O, want[1])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_one_long_head_over_all_parts(dtype, d):
    """As many parts as the GPU takes at a time for one head: more than a joining thread has loads in flight, by groups."""
    for hq, lengths in ((1, [70001]), (3, [65536]), (16, [40000, 0, 3])):
        cache, q = make(d + hq, lengths, hq, 1, d, dtype, 64)
        O, lse = cache.paged_attention_fwd(q)
        assert cache.last_status() == 0
        check(cache, q, lengths, O, lse)


def test_sequences_that_share_pages():
    """A fork: two sequences read the same pages and differ in their last one."""
    cache, q = make(8, [100, 100], 4, 2, 64, "bf16", 16, garbage=False)
    cache.page_table[1, :6] = cache.page_table[0, :6]
    q[1] = q[0]
    O, lse = cache.paged_attention_fwd(q)
    check(cache, q, [100, 100], O, lse)
    assert not torch.equal(O[0], O[1])
    cache.page_table[1] = cache.page_table[0]
    O, lse = cache.paged_attention_fwd(q)
    assert torch.equal(O[0], O[1]) and torch.equal(lse[0], lse[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pools_beyond_32_bits(dtype):
    """A pool of more than 2^32 bytes and 2^31 elements, rows at its end."""
    d, page_rows, kv, n = 128, 64, 8, 150
    pages = (2 ** 31 + 2 ** 24) // (kv * page_rows * d)
    shape = (pages, kv, page_rows, d)
    K, V = (torch.empty(shape, dtype=DT[dtype], device=DEV) for _ in range(2))
    cache = binding.PagedCache(binding.make_cache_problem(1, kv, kv, d, dtype, page_rows, pages, 4), DEV, K, V,
                               torch.tensor([[pages - 1, 2, pages - 2, 7]], dtype=torch.int32, device=DEV))
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v, q = (torch.randn((1, kv, m, d), generator=g, device=DEV).to(DT[dtype]) for m in (n, n, 1))
    cache.cache_append(k, v)
    assert torch.equal(K[pages - 1], k[0, :, :64]) and torch.equal(V[pages - 2, :, :22], v[0, :, 128:])
    O, lse = cache.paged_attention_fwd(q, appended=n)
    assert cache.last_status() == 0
    check(cache, q, [n], O, lse)


def test_binding_refuses_what_does_not_fit():
    cache, q = make(3, [40, 40], 4, 2, 64, "bf16", 16)
    k = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device=DEV)
    rot = binding.Rotary(64, [4])
    pos = torch.zeros((2, 3, 1), dtype=torch.int32, device=DEV)
    one = q[:1]
    for bad in (q.float(), one, q.transpose(0, 1), q.cpu(), torch.zeros((2, 4, 1, 128), dtype=torch.bfloat16, device=DEV)[..., ::2], None):
        with pytest.raises(binding.ClusterAttnError):
            cache.paged_attention_fwd(bad)
    with pytest.raises(binding.ClusterAttnError):
        cache.paged_attention_fwd(q, out=q.float())
    with pytest.raises(binding.ClusterAttnError):          # 16-byte alignment
        cache.paged_attention_fwd(torch.zeros((2, 4, 1, 72), dtype=torch.bfloat16, device=DEV)[..., 1:65])
    for args, kw in (((k, k[:, :, :2]), {}), ((k, k), dict(rotary=rot)), ((k, k), dict(positions=pos)), ((k, k), dict(rotary=rot, positions=pos.long())),
                     ((k, k), dict(rotary=rot, positions=pos[:, :2])), ((k, k), dict(rotary=binding.Rotary(128, [4]), positions=pos)),
                     ((k, k), dict(count=torch.zeros(3, dtype=torch.int32, device=DEV))), ((k[:, :, :0], k[:, :, :0]), {}), ((k.float(), k.float()), {})):
        with pytest.raises(binding.ClusterAttnError):
            cache.cache_append(*args, **kw)
    with pytest.raises(AttributeError):
        cache.lengths = torch.zeros(2, dtype=torch.int32, device=DEV)
    p = cache.problem
    for kw in (dict(lengths=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(page_table=torch.zeros((2, 1), dtype=torch.int64, device=DEV)),
               dict(K_pages=torch.zeros((1, 2, 16, 64), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(binding.ClusterAttnError):
            binding.PagedCache(p, DEV, **kw)
    for bad_q, bad_k, bad_pos in ((q.half(), None, pos), (k, k.float(), pos), (k, k[:1], pos), (k, k, pos[:, :, :0]), (k, k, pos.cpu()), (k, k, None), (k[..., :32], None, pos)):
        with pytest.raises(binding.ClusterAttnError):
            binding.rotary_axes(rot, bad_q, bad_k, bad_pos)
    with pytest.raises(binding.ClusterAttnError):
        binding.rotary_axes(rot, k, None, pos, out_k=k)
    w = binding.WindowPlan(binding.make_window_problem(2, 4, 2, 3, 3, 64, "bf16", 1, 0), DEV)
    q3 = torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16, device=DEV)
    for args, kw in (((q3, k, k.float()), {}), ((k, k, k), {}), ((q3, k, k), dict(len_q=torch.zeros(2, device=DEV))), ((q3, k, k), dict(out=q3[:, :, :2]))):
        with pytest.raises(binding.ClusterAttnError):
            w.window_attention_fwd(*args, **kw)
    side = torch.cuda.Stream()
    assert cache.paged_attention_fwd(q, stream=side)[0] is cache.O
    torch.cuda.synchronize()
