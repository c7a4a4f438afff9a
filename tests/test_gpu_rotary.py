"""Rotary positions with several axes against rotations in 64 bits, and the same on the way into a cache's pages."""
import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def rows(gen, shape, dtype, layout):
    """[B, H, n, d]: dense, rows before heads, or with room between rows."""
    B, H, n, d = shape
    if layout == "rows_first":
        return torch.randn((B, n, H, d), generator=gen, device=DEV).to(dtype).transpose(1, 2)
    if layout == "room":
        return torch.randn((B, H, n, d + 24), generator=gen, device=DEV).to(dtype)[..., 8:8 + d]
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def positions(gen, B, n, axes, far):
    return torch.randint(-far, far, (B, n, axes), generator=gen, device=DEV, dtype=torch.int64).to(torch.int32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,pairs", [(64, [32]), (64, [16, 16]), (128, [22, 21, 21]), (128, [16, 24, 24]), (128, [5, 0, 3, 9]),
                                     (64, [3]), (128, [32])])
@pytest.mark.parametrize("adjacent", [True, False])
@pytest.mark.parametrize("inverse,layout,n", [(False, "dense", 1), (True, "rows_first", 2), (False, "room", 77), (True, "dense", 1001)])
def test_rotary_axes(dtype, d, pairs, adjacent, inverse, layout, n):
    g = generator(d + n)
    B, H, Hk = 3, 6, 2
    rot = binding.Rotary(d, pairs, adjacent=adjacent)
    q, k = rows(g, (B, H, n, d), DT[dtype], layout), rows(g, (B, Hk, n, d), DT[dtype], layout)
    pos = positions(g, B, n, len(pairs), 100000)
    for p in (pos, pos[1:2].contiguous()):
        for x, y in zip((q, k), binding.rotary_axes(rot, q, k, p, inverse=inverse)):
            want = ref.rotate(x.double(), p, rot.frequencies, pairs, adjacent, inverse)
            ref.check(y, want, ref.rotate_bound(x.double(), pairs, adjacent, DT[dtype], want), "rotary")
            R = sum(pairs)
            assert torch.equal(y[..., 2 * R:], x[..., 2 * R:])


def test_far_positions_keep_their_phase():
    """At the ends of 32 bits, of frequencies above a turn per step and below a turn in all of them: the product of position and
    frequency is taken in whole numbers and fractions here."""
    from fractions import Fraction
    import math
    freqs = [1.0, 7.25, 0.1, 1e-9, -2.5, 3.0e5]
    rot = binding.Rotary(64, [6], frequencies=freqs)
    pos = torch.tensor([-2 ** 31, 2 ** 31 - 1, -1, 0, 1, 123456789], dtype=torch.int32, device=DEV).view(1, 6, 1)
    x = torch.zeros((1, 1, 6, 64), device=DEV)
    x[..., 0:12:2] = 1.0
    y = binding.rotary_axes(rot, x, None, pos)[0][0, 0].double().cpu()
    two_pi = Fraction(6283185307179586476925286766559005768394, 10 ** 39)
    for i, p in enumerate(pos.flatten().tolist()):
        for c, f in enumerate(freqs):
            t = Fraction(f) * p / two_pi
            t = float((t - math.floor(t)) * two_pi)
            # the frequency as a fraction of a turn has 64 bits: |p| 2^-64 of a turn at most, 2^-33
            assert abs(y[i, 2 * c] - math.cos(t)) < 11 * 2 ** -24 and abs(y[i, 2 * c + 1] - math.sin(t)) < 11 * 2 ** -24


@pytest.mark.parametrize("adjacent", [True, False])
def test_channels_behind_the_last_pair_stay(adjacent):
    x = torch.full((1, 2, 40, 64), float("nan"), device=DEV)
    x[..., :14] = 1.0
    x[..., 50] = float("inf")
    for dt in (torch.float32, torch.bfloat16):
        y = binding.rotary_axes(binding.Rotary(64, [3, 4], adjacent=adjacent), x.to(dt), None,
                                torch.ones((1, 40, 2), dtype=torch.int32, device=DEV))[0]
        assert torch.isfinite(y[..., :14].float()).all() and torch.isnan(y[..., 14:50].float()).all()
        assert torch.isinf(y[..., 50].float()).all() and torch.isnan(y[..., 51:].float()).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("adjacent,pairs", [(True, [10, 11, 11]), (False, [10, 11, 11]), (False, [5, 6])])
def test_in_place_gives_the_same(dtype, adjacent, pairs):
    g = generator(5)
    rot = binding.Rotary(64, pairs, adjacent=adjacent)
    q, k = rows(g, (2, 5, 300, 64), DT[dtype], "rows_first"), rows(g, (2, 1, 300, 64), DT[dtype], "room")
    pos = positions(g, 2, 300, len(pairs), 1000)
    a, b = binding.rotary_axes(rot, q, k, pos)
    binding.rotary_axes(rot, q, k, pos, out_q=q, out_k=k)
    assert torch.equal(q, a) and torch.equal(k, b)


def test_broadcast_rows_and_many_batch_items():
    """Inputs with strides of zero; more batch items than a block of threads has rows; one key head for all."""
    g = generator(21)
    rot = binding.Rotary(64, [8, 8], adjacent=False)
    for dtype in DT.values():
        q = torch.randn((1, 3, 5, 64), generator=g, device=DEV).to(dtype).expand(700, 3, 5, 64)
        k = torch.randn((700, 1, 1, 64), generator=g, device=DEV).to(dtype).expand(700, 1, 5, 64)
        pos = positions(g, 700, 5, 2, 1000)
        for x, y in zip((q, k), binding.rotary_axes(rot, q, k, pos)):
            want = ref.rotate(x.double(), pos, rot.frequencies, [8, 8], False)
            ref.check(y, want, ref.rotate_bound(x.double(), [8, 8], False, dtype, want), "rotary")


def test_other_stream():
    g = generator(22)
    rot = binding.Rotary(128, [16, 24, 24])
    q = torch.randn((2, 8, 3000, 128), generator=g, device=DEV)
    pos = positions(g, 2, 3000, 3, 100)
    want = binding.rotary_axes(rot, q, None, pos)[0]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [binding.rotary_axes(rot, q, None, pos, stream=side)[0] for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs)


def test_inverse_is_the_gradient():
    """Against the gradient of the 64-bit form, and against differences (the map is linear, so they are exact but for rounding)."""
    g = generator(9)
    pairs = [6, 4, 6]
    rot = binding.Rotary(64, pairs)
    x, up = (torch.randn((2, 3, 9, 64), generator=g, device=DEV) for _ in range(2))
    pos = positions(g, 2, 9, 3, 50)
    leaf = x.double().requires_grad_()
    torch.autograd.backward(ref.rotate(leaf, pos, rot.frequencies, pairs, True), up.double())
    got = binding.rotary_axes(rot, up, None, pos, inverse=True)[0]
    ref.check(got, leaf.grad, ref.rotate_bound(up.double(), pairs, True, torch.float32, leaf.grad), "gradient")
    move = torch.randn((2, 3, 9, 64), generator=g, device=DEV)
    f = lambda z: (binding.rotary_axes(rot, z, None, pos)[0].double() * up.double()).sum()
    # 3,456 products of two normal numbers, each result off by 11 u (|x| + |y|) < 11 u 12 and up below 6: sum below 3456 * 800 u
    diff = (f(x + move) - f(x - move)) / 2
    assert abs(diff - (got.double() * move.double()).sum()) < 3456 * 1600 * ref.U32


def test_whole_path_turns_queries_and_keys_first():
    """Plan.forward with positions: what it gives for rows that were turned before."""
    g = generator(3)
    for n_q, n_k in ((1000, 1000), (700, 1300)):
        p = binding.make_problem(1, 2, n_q, n_k, 64, "bf16", 64, 64, 4)
        q, k = rows(g, (1, 2, n_q, 64), torch.bfloat16, "rows_first"), rows(g, (1, 2, n_k, 64), torch.bfloat16, "rows_first")
        v = rows(g, (1, 2, n_k, 64), torch.bfloat16, "dense")
        rot = binding.Rotary(64, [8, 12, 12])
        pq, pk = positions(g, 1, n_q, 3, 40), positions(g, 1, n_k, 3, 40)
        args = dict(positions_q=pq) if n_q == n_k else dict(positions_q=pq, positions_k=pk)
        got = binding.Plan(p, DEV).forward(q, k, v, rotary=rot, **args).clone()
        a = binding.rotary_axes(rot, q, None, pq)[0]
        b = binding.rotary_axes(rot, k, None, pq if n_q == n_k else pk)[0]
        assert torch.equal(got, binding.Plan(p, DEV).forward(a, b, v))
        ragged = binding.Plan(p, DEV).forward_adaptive(q, k, v, 0.8, rotary=rot, **args)[0].clone()
        assert torch.equal(ragged, binding.Plan(p, DEV).forward_adaptive(a, b, v, 0.8)[0])


# ---- rows into pages

@pytest.mark.parametrize("dtype,d,page_rows", [("bf16", 128, 16), ("bf16", 64, 100), ("fp32", 64, 17), ("fp32", 128, 64)])
@pytest.mark.parametrize("n", [1, 5, 130])
@pytest.mark.parametrize("pairs,adjacent", [(None, True), ([8, 12, 12], True), ([8, 12, 12], False), ([7, 2], False)])
@pytest.mark.parametrize("ragged", [False, True])
def test_cache_append(dtype, d, page_rows, n, pairs, adjacent, ragged):
    g = generator(n + page_rows)
    B, H, per = 4, 3, 300 // page_rows + 2
    pages = B * per + 2
    table = torch.randperm(pages, generator=g, device=DEV)[:B * per].reshape(B, per).int()
    lengths = torch.tensor([0, page_rows - 1, page_rows, 150], dtype=torch.int32, device=DEV)
    count = torch.tensor([n, 0, 1, max(1, n // 2)], dtype=torch.int32, device=DEV) if ragged else None
    fill = torch.randn((pages, H, page_rows, d), generator=g, device=DEV).to(DT[dtype])
    cache = binding.PagedCache(binding.make_cache_problem(B, 2 * H, H, d, dtype, page_rows, pages, per), DEV, K_pages=fill.clone(),
                               V_pages=fill.clone(), page_table=table, lengths=lengths)
    K, V = rows(g, (B, H, n, d), DT[dtype], "rows_first"), rows(g, (B, H, n, d), DT[dtype], "room")
    pos = positions(g, B, n, len(pairs), 5000) if pairs else None
    rot = binding.Rotary(d, pairs, adjacent=adjacent) if pairs else None
    cache.cache_append(K, V, count=count, rotary=rot, positions=pos)
    want_k = binding.rotary_axes(rot, K, None, pos)[0] if pairs else K       # (held against 64 bits above)
    pools = [fill.clone(), fill.clone()]
    for b in range(B):
        for i in range(n if count is None else int(count[b])):
            page, place = divmod(int(lengths[b]) + i, page_rows)
            pools[0][table[b, page], :, place], pools[1][table[b, page], :, place] = want_k[b, :, i], V[b, :, i]
    assert torch.equal(cache.K_pages, pools[0]) and torch.equal(cache.V_pages, pools[1])
    assert cache.last_status() == 0


def test_cache_append_leaves_out_rows_without_a_place():
    B, n, per, page_rows = 5, 20, 2, 16
    table = torch.tensor([[0, 1], [2, 77], [3, 4], [-1, 5], [6, 7]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([0, 10, 20, 0, -1], dtype=torch.int32, device=DEV)
    cache = binding.PagedCache(binding.make_cache_problem(B, 1, 1, 64, "fp32", page_rows, 8, per), DEV, page_table=table, lengths=lengths)
    K = torch.arange(1, B * n + 1, device=DEV).float().view(B, 1, n, 1).expand(B, 1, n, 64).contiguous()
    cache.cache_append(K, -K)
    assert cache.last_status() == binding.CA_ERR_BAD_INDEX
    want = torch.zeros((8, page_rows), device=DEV)
    want[0], want[1, :4] = K[0, 0, :16, 0], K[0, 0, 16:, 0]
    want[2, 10:] = K[1, 0, :6, 0]                # its second page is not one of the pool
    want[4, 4:] = K[2, 0, :12, 0]                # beyond the table's last page
    want[5, :4] = K[3, 0, 16:, 0]
    assert torch.equal(cache.K_pages[:, 0, :, 0], want) and torch.equal(cache.V_pages[:, 0, :, 5], -want)
    # a count that is not one is cut, and the status of the next call is its own
    lengths.zero_()
    table.copy_(torch.arange(10, device=DEV).int().view(5, 2) % 8)
    table[4] = torch.tensor([7, 6])
    count = torch.tensor([0, 0, 0, 21, -5], dtype=torch.int32, device=DEV)
    cache.cache_append(K, -K, count=count)
    assert cache.last_status() == binding.CA_ERR_BAD_INDEX
    cache.cache_append(K, -K, count=torch.zeros_like(count))
    assert cache.last_status() == 0
