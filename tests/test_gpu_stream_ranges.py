"""Windows and the cache in pages over the whole range of their types: values and weights near its ends, and the accuracy of the
products where few terms leave little room for errors to hide in."""
import math

import pytest
import torch

import stream_bounds as sb
import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
LOG2 = math.log(2.0)
# attention over n rows of which the last one asks: windows of either storage and kernel, caches of few rows and of many (split)
WAYS = [("window", "bf16", 0), ("window", "fp32", 0), ("window", "bf16", binding.CA_ATTN_FP32), ("window", "fp32", binding.CA_ATTN_FP32),
        ("cache", "bf16", 0), ("cache", "bf16", 17), ("cache", "fp32", 0), ("cache", "fp32", 17)]


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def ask(way, q, k, v, scale, left=-1, sinks=0):
    """q [B, H, 1, d] against k, v [B, G, n, d]: result [B, H, d] in 64 bits and log-sum-exp [B, H]."""
    kind, dtype, form = way
    (B, H, _, d), (G, n) = q.shape, k.shape[1:3]
    if kind == "window":
        plan = binding.WindowPlan(binding.make_window_problem(B, H, G, 1, n, d, dtype, left, 0, sinks, softmax_scale=scale, flags=form), DEV)
        O, lse = plan.window_attention_fwd(q, k, v)
    else:
        per = -(-n // 16) + form                            # (17 more pages are too many rows for one CTA to a sequence and head)
        pages = B * per
        cache = plan = binding.PagedCache(binding.make_cache_problem(B, H, G, d, dtype, 16, pages, per, left, sinks, scale), DEV,
                                          page_table=torch.arange(pages, device=DEV).flip(0).reshape(B, per).int().contiguous())
        cache.cache_append(k, v)
        assert cache.last_status() == 0
        O, lse = cache.paged_attention_fwd(q, appended=n)
    assert plan.last_status() == 0
    return O[:, :, 0].double(), lse[:, :, 0].double()


def check(way, q, k, v, scale, terms, got, what, left=-1, sinks=0):
    O, lse = got
    kind, dtype, form = way
    products, weights = sb.WINDOW[dtype, form] if kind == "window" else sb.CACHE[dtype]
    group, n = q.shape[1] // k.shape[1], k.shape[2]
    j = torch.arange(n, device=DEV)
    see = ((j >= n - 1 - left) | (j < sinks) if left >= 0 else j >= 0)[None]
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            o, l64, bound, lb = sb.attend(q[b, h].double(), k[b, h // group].double(), v[b, h // group].double(), see, scale, DT[dtype], terms,
                                          products, weights)
            ref.check(O[b, h][None], o, bound, f"{what}, item {b}, head {h}")
            ref.check(lse[b, h][None], l64, lb, f"log-sum-exp of {what}, item {b}, head {h}")


def steps(n, B, H, G, d, dtype, logits):
    """Rows whose logits (in log2 units, with softmax_scale log 2) are those numbers, exactly: channel 0 holds them."""
    q, k = torch.zeros((B, H, 1, d), dtype=DT[dtype], device=DEV), torch.zeros((B, G, n, d), dtype=DT[dtype], device=DEV)
    q[..., 0], k[..., 0] = 1.0, logits
    return q, k


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 2), (6, 1)])
@pytest.mark.parametrize("size", [3e-42, 1e-40, 1e-38, 1e-35, 1e-33, 1e-30, 1.0, 1e30, 1e36])
@pytest.mark.parametrize("n", [5, 40, 700])
def test_values_of_any_size(way, d, H, G, size, n):
    """Their weighted mean is as accurate at the ends of the range as in the middle; few of the rows have most of the weight."""
    g = generator(n + d)
    logits = -torch.randint(0, 9, (2, G, n), generator=g, device=DEV).float()
    logits[..., n // 3] = 6.0
    q, k = steps(n, 2, H, G, d, way[1], logits)
    v = (torch.randn((2, G, n, d), generator=g, device=DEV).clamp(-8, 8).double() * size).to(DT[way[1]])
    check(way, q, k, v, LOG2, 1, ask(way, q, k, v, LOG2), "values")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [40, 700])
def test_large_values_at_small_weights(way, d, n):
    """A row 90 to 125 octaves below the heaviest with a value as many octaves above its value: both count the same."""
    g = generator(n + d)
    octaves = torch.arange(90, 126, device=DEV)
    B = octaves.numel()
    logits = torch.full((B, 1, n), -400.0, device=DEV)
    items = torch.arange(B, device=DEV)
    far = items % (n - 9) + 3
    logits[:, 0, 1], logits[items, 0, far] = 0.0, -octaves.float()
    q, k = steps(n, B, 2, 1, d, way[1], logits)
    v = torch.zeros((B, 1, n, d), dtype=torch.float64, device=DEV)
    v[:, 0, 1] = torch.randn((B, d), generator=g, device=DEV).double()
    v[items, 0, far] = (torch.rand((B, d), generator=g, device=DEV).double() + 0.5) * 2.0 ** octaves.double()[:, None]
    v = v.to(DT[way[1]])
    check(way, q, k, v, LOG2, 1, ask(way, q, k, v, LOG2), "small weights")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("n", [40, 700])
def test_an_infinite_value_at_a_small_weight(way, n):
    octaves = torch.arange(0, 126, 5, device=DEV)
    B, d = octaves.numel(), 64
    logits = torch.full((B, 1, n), -400.0, device=DEV)
    logits[:, 0, 1], logits[:, 0, 7] = 0.0, -octaves.float()
    q, k = steps(n, B, 1, 1, d, way[1], logits)
    v = torch.ones((B, 1, n, d), dtype=DT[way[1]], device=DEV)
    v[:, 0, 7, 5], v[:, 0, 7, 9], v[:, 0, 7, 11] = math.inf, -math.inf, math.nan
    O, lse = ask(way, q, k, v, LOG2)
    assert (O[..., 5] == math.inf).all() and (O[..., 9] == -math.inf).all() and torch.isnan(O[..., 11]).all()
    rest = torch.ones(d, dtype=torch.bool, device=DEV)
    rest[[5, 9, 11]] = False
    v[:, 0, 7] = 1.0
    check(way, q, k, v, LOG2, 1, (torch.where(rest, O, torch.ones_like(O)), lse), "columns beside it")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (20, 1), (4, 2)])
@pytest.mark.parametrize("n", [2, 40, 700, 3000])
def test_means_of_the_largest_values(way, d, H, G, n):
    """Columns of the largest values, of one sign, of the other, of either in turn and in halves, next to columns of the smallest."""
    big = torch.finfo(DT[way[1]]).max
    q, k = steps(n, 1, H, G, d, way[1], (torch.arange(n, device=DEV) % 3 - 2).float())
    v = torch.randn((1, G, n, d), generator=generator(n), device=DEV).to(DT[way[1]])
    j = torch.arange(n, device=DEV)
    v[..., 0], v[..., 1], v[..., 2], v[..., 3] = big, -big, torch.where(j % 2 == 0, big, -big), torch.where(j < n // 2, big, -big)
    v[..., 4], v[..., d - 1] = 1e-35, big / 2
    O, lse = ask(way, q, k, v, LOG2)
    assert torch.isfinite(O).all()
    check(way, q, k, v, LOG2, 1, (O, lse), "largest values")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 7, 12])
def test_products_of_few_terms(way, d, n):
    """Scores of four products, sums of a few rows: what a part of a product that is lost would cost stands far above the bounds."""
    g = generator(n + d)
    B, H, G = 24, 4, 2
    dt = DT[way[1]]
    q, k = torch.zeros((B, H, 1, d), dtype=dt, device=DEV), torch.zeros((B, G, n, d), dtype=dt, device=DEV)
    at = torch.tensor([0, d // 2 - 3, d // 2 + 1, d - 1], device=DEV)
    q[..., at] = torch.randn((B, H, 1, 4), generator=g, device=DEV).to(dt)
    k[..., at] = torch.randn((B, G, n, 4), generator=g, device=DEV).to(dt)
    v = torch.randn((B, G, n, d), generator=g, device=DEV).to(dt)
    check(way, q, k, v, 0.75, 4, ask(way, q, k, v, 0.75), "few terms")


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("left,sinks", [(9, 3), (0, 0), (30, 20)])
def test_largest_values_inside_a_window(way, left, sinks):
    """What is not seen takes no part where a row's sums are taken again either."""
    n, d = 900, 64
    g = generator(left)
    big = torch.finfo(DT[way[1]]).max
    q, k = steps(n, 1, 2, 1, d, way[1], torch.zeros(n, device=DEV))
    v = torch.full((1, 1, n, d), big, dtype=DT[way[1]], device=DEV)
    v[0, 0, :, 1::2] = torch.randn((n, d // 2), generator=g, device=DEV).to(DT[way[1]])
    j = torch.arange(n, device=DEV)
    see = (j >= n - 1 - left) | (j < sinks)
    clean = v.clone()
    v[0, 0, ~see] = math.nan
    k[0, 0, ~see] = math.nan
    O, lse = ask(way, q, k, v, LOG2, left, sinks)
    assert torch.isfinite(O).all()
    check(way, q, torch.nan_to_num(k), clean, LOG2, 1, (O, lse), "a window", left, sinks)


@pytest.mark.parametrize("way", [w for w in WAYS if w[0] == "cache"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8, 20])
def test_an_output_in_the_place_of_the_queries(way, d, group):
    """Sums that are taken again read the queries again, before their place is written."""
    g = generator(group)
    n, dt = 700, DT[way[1]]
    per = -(-n // 16) + way[2]
    cache = binding.PagedCache(binding.make_cache_problem(3, 2 * group, 2, d, way[1], 16, 3 * per, per), DEV,
                               page_table=torch.arange(3 * per, device=DEV).reshape(3, per).int())
    cache.lengths.copy_(torch.tensor([n, 3, 40]))
    for pool in (cache.K_pages, cache.V_pages):
        pool.copy_(torch.randn(pool.shape, generator=g, device=DEV).to(dt))
    cache.V_pages[..., 5] = torch.finfo(dt).max
    q = torch.randn((3, 2 * group, 1, d), generator=g, device=DEV).to(dt)
    want = [x.clone() for x in cache.paged_attention_fwd(q)]
    assert torch.isfinite(want[0].float()).all()
    got = cache.paged_attention_fwd(q, out=q)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(got[1], want[1])
