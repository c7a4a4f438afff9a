"""Operators for attention over streams of tokens, as cases that can be timed and compared.

  rotary   rotary positions with several axes (time, height, width) on queries and keys, and its
           inverse, which is also the gradient's way back
  append   new keys (rotated on the way) and values into the pages of a cache
  paged    attention of one new token per sequence over that cache
  window   attention over a sliding window with a few first tokens that stay visible

Tensors are [batch, heads, rows, head_dim].  A key j is visible to a query at position p (its row, counted so that the last
query stands at the last key) when j <= p + right and (j >= p - left or j < sinks); a bound of -1 is none.  With `own`
false, `run` computes the operators from elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""
import math

import torch

own = False

DEV = "cuda:0"

_LISTED = [
    # ---- rotary
    # one new token of each of 64 streams, few key heads: all launch latency
    dict(name="rotary-token", op="rotary", batch=64, heads_q=32, heads_kv=8, n=1, d=128, dtype="bf16", pairs="16,24,24",
         adjacent=False, inverse=False, rows_first=True, far=100000),
    # a video layer at 480p, queries and keys as the projections leave them (rows before heads)
    dict(name="rotary-video480", op="rotary", batch=1, heads_q=40, heads_kv=40, n=32760, d=128, dtype="bf16",
         pairs="22,21,21", adjacent=True, inverse=False, rows_first=True, far=0),
    # gradients of the queries and keys of a large picture's patches, two axes, float32 storage
    dict(name="rotary-image-inverse", op="rotary", batch=1, heads_q=12, heads_kv=12, n=16385, d=64, dtype="fp32",
         pairs="16,16", adjacent=True, inverse=True, rows_first=False, far=0),
    # ---- append
    # one new token of each of 64 streams
    dict(name="append-token", op="append", batch=64, heads_q=8, heads_kv=8, n=1, d=128, dtype="bf16", page=16, longest=1024,
         pairs="16,24,24", adjacent=False, rows_first=True),
    # three frames of a 480p video behind the frames that are there
    dict(name="append-frames", op="append", batch=1, heads_q=40, heads_kv=40, n=4680, d=128, dtype="bf16", page=64,
         longest=32760, pairs="22,21,21", adjacent=True, rows_first=True),
    # ---- paged
    # a few streams with a short window, float32 storage: latency
    dict(name="paged-window-fp32", op="paged", batch=4, heads_q=12, heads_kv=12, d=64, dtype="fp32", page=16, shortest=1,
         longest=1370, left=511, sinks=16),
    # a serving batch: streams of very different lengths, four query heads to a key head
    dict(name="paged-batch", op="paged", batch=64, heads_q=32, heads_kv=8, d=128, dtype="bf16", page=16, shortest=1,
         longest=8192, left=-1, sinks=0),
    # two long streams (with and without the condition) that end inside a page, a key head to every query head
    dict(name="paged-long", op="paged", batch=2, heads_q=40, heads_kv=40, d=128, dtype="bf16", page=64, shortest=131001,
         longest=131071, left=-1, sinks=0),
    # ---- window
    # patches of a small picture (14 x 14 and the class token, which all see)
    dict(name="window-image-197", op="window", batch=1, heads_q=12, heads_kv=12, n_q=197, n_k=197, d=64, dtype="bf16",
         left=32, right=32, sinks=1, ragged=False, rows_first=False),
    # patches of an ordinary picture (37 x 37 and the class token), float32 storage
    dict(name="window-fp32-1370", op="window", batch=1, heads_q=12, heads_kv=12, n_q=1370, n_k=1370, d=64, dtype="fp32",
         left=148, right=148, sinks=1, ragged=False, rows_first=False),
    # streams that are read in, causal, padded to the longest, four query heads to a key head
    dict(name="window-causal-ragged", op="window", batch=4, heads_q=32, heads_kv=8, n_q=4999, n_k=4999, d=128, dtype="bf16",
         left=1023, right=0, sinks=4, ragged=True, rows_first=True),
    # a video layer at 480p: two frames to either side, and the first frame
    dict(name="window-video480", op="window", batch=1, heads_q=40, heads_kv=40, n_q=32760, n_k=32760, d=128, dtype="bf16",
         left=3120, right=3120, sinks=1560, ragged=False, rows_first=True),
]
_MOST = {"rotary": 1.3e9, "append": 0.19e9, "paged": 5.3e9, "window": 2.5e12}   # work of a drawn case: bytes, of windows flops


def listed():
    return [dict(c) for c in _LISTED]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _pairs(rng, d):
    axes = rng.choice([1, 2, 3, 3])
    if axes == 1:
        return str(rng.choice([d // 2, d // 4]))
    if axes == 2:
        return "%d,%d" % (d // 4, d // 4)
    a = rng.choice([d // 8, d // 2 - 2 * ((d // 2) // 3)])
    return "%d,%d,%d" % (a, (d // 2 - a) // 2, (d // 2 - a) // 2)


def _heads(rng, most):
    kv, group = rng.choice([1, 2, 4, 8, 12, 40]), rng.choice([1, 1, 2, 4, 5, 8, 16])
    return (kv, kv * group) if kv * group <= most else (kv, kv)


def draw(rng):
    """One more case of an operator at another size."""
    while True:
        op = rng.choice(["rotary", "append", "paged", "paged", "window", "window"])
        d, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp32"])
        kv, hq = _heads(rng, 64)
        batch = _spread(rng, 1, 64)
        case = dict(op=op, batch=batch, heads_q=hq, heads_kv=kv, d=d, dtype=dtype)
        if op == "rotary":
            case.update(n=_spread(rng, 1, 40000), pairs=_pairs(rng, d), adjacent=rng.random() < 0.5,
                        inverse=rng.random() < 0.5, rows_first=rng.random() < 0.5, far=rng.choice([0, 0, 100000, 1000000]))
        elif op == "append":
            longest = _spread(rng, 16, 16384)
            case.update(n=min(longest, _spread(rng, 1, 5000)), page=rng.choice([16, 32, 64, 128, 100]), longest=longest,
                        pairs=rng.choice(["", _pairs(rng, d)]), adjacent=rng.random() < 0.5, rows_first=rng.random() < 0.5)
        elif op == "paged":
            longest = _spread(rng, 1, 131072)
            case.update(page=rng.choice([16, 32, 64, 128, 100]), shortest=rng.choice([0, 1, max(1, longest // 2), longest]),
                        longest=longest, left=rng.choice([-1, -1, _spread(rng, 1, 4096) - 1]), sinks=rng.choice([0, 4, 64, 100]))
        else:
            n_k = _spread(rng, 1, 32760)
            n_q = rng.choice([n_k, n_k, _spread(rng, 1, n_k), min(32760, n_k + rng.randrange(1, 300))])
            bound = _spread(rng, 1, 4096) - 1
            left, right = rng.choice([(bound, 0), (bound, 0), (bound, bound), (bound, rng.randrange(0, 300)), (-1, 0), (bound, -1)])
            case.update(n_q=n_q, n_k=n_k, left=left, right=right, sinks=rng.choice([0, 1, 4, 100, 1560]),
                        ragged=rng.random() < 0.4, rows_first=rng.random() < 0.5)
            case["batch"] = min(batch, rng.choice([1, 2, 4, 8]))
        w, held = work(case), _held(case)
        limit = _MOST[op] * (0.02 if op == "window" and dtype == "fp32" else 1.0)
        if (w["flops"] if op == "window" else w["bytes"]) <= limit and held <= 6e9:
            return case


def _size(case):
    return 4 if case["dtype"] == "fp32" else 2


def _held(case):
    """Bytes of the state: of caches the pages of the longest stream for every stream."""
    wide = case["d"] * _size(case) * case["batch"]
    if case["op"] == "rotary":
        return wide * case["n"] * (case["heads_q"] + case["heads_kv"])
    if case["op"] == "window":
        return wide * (2 * case["n_q"] * case["heads_q"] + 2 * case["n_k"] * case["heads_kv"])
    return 2 * wide * (case["longest"] + case["page"]) * case["heads_kv"]


def _lengths(case, name, count, lo, hi):
    """`count` lengths of a case, the longest among them: from the case alone, so that its work is known."""
    gen = torch.Generator()
    gen.manual_seed(count * 1000003 + lo * 31 + hi * 7 + len(name))
    low = max(lo, 1)
    x = torch.rand((count,), generator=gen, dtype=torch.float64)
    n = torch.exp(math.log(low) + x * (math.log(max(hi, 1)) - math.log(low))).round().long().clamp(lo, hi)
    n[count // 2] = hi
    if lo == 0 and count > 1:
        n[0] = 0
    return [int(v) for v in n]


def _window_lengths(case):
    """Query and key lengths of every batch item."""
    B = case["batch"]
    if not case["ragged"]:
        return [case["n_q"]] * B, [case["n_k"]] * B
    lk = _lengths(case, "keys", B, max(1, case["n_k"] // 8), case["n_k"])
    if case["n_q"] == case["n_k"]:
        return list(lk), lk
    return _lengths(case, "queries", B, max(1, case["n_q"] // 8), case["n_q"]), lk


def _visible(len_q, len_k, left, right, sinks):
    """Pairs of a query and a visible key."""
    p = torch.arange(len_q, dtype=torch.float64) + (len_k - len_q)
    hi = torch.full_like(p, len_k) if right < 0 else (p + right + 1).clamp(0, len_k)     # keys below hi
    lo = torch.zeros_like(p) if left < 0 else (p - left).clamp(min=0)
    first = torch.minimum(torch.full_like(p, sinks), lo)                                 # sinks outside the window
    return float((torch.minimum(first, hi) + (hi - lo).clamp(min=0)).sum())


def work(case):
    """Inputs read once and outputs written once; products of the visible pairs.  Of a cache the rows that are visible or new, not
    the pages that stay as they are."""
    B, hq, kv, d, size = case["batch"], case["heads_q"], case["heads_kv"], case["d"], _size(case)
    if case["op"] == "rotary":
        elements = B * case["n"] * (hq + kv) * d
        return {"bytes": float(2 * size * elements), "flops": float(3 * elements)}
    if case["op"] == "append":
        elements = B * case["n"] * kv * d
        return {"bytes": float(4 * size * elements), "flops": float(3 * elements)}
    if case["op"] == "paged":
        lengths = _lengths(case, "cache", B, case["shortest"], case["longest"])
        keys = sum(_visible(1, n, case["left"], 0, case["sinks"]) for n in lengths if n > 0)
        return {"bytes": float(2 * size * d * (keys * kv + B * hq) + 4 * B * hq), "flops": float(4 * keys * hq * d)}
    len_q, len_k = _window_lengths(case)
    pairs = sum(_visible(a, b, case["left"], case["right"], case["sinks"]) for a, b in zip(len_q, len_k))
    rows = 2 * sum(len_q) * hq + 2 * sum(len_k) * kv
    return {"bytes": float(size * d * rows + 4 * sum(len_q) * hq), "flops": float(4 * pairs * hq * d)}


# ---- inputs -------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _rows(case, gen, heads, n, gain=1.0):
    """[batch, heads, n, d]; rows_first: as a projection leaves them, with the heads of a row side by side.  Some channels are several
    times larger than the others, as in queries and keys of trained layers."""
    B, d = case["batch"], case["d"]
    shape = (B, n, heads, d) if case.get("rows_first") else (B, heads, n, d)
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    channel = torch.ones((d,), device=DEV)
    channel[torch.randint(0, d, (4,), generator=gen, device=DEV)] = 2.5
    x = x.mul_((channel * gain).to(x.dtype))
    return x.transpose(1, 2) if case.get("rows_first") else x


def _frequencies(pairs):
    """Radians per step of position, each axis a series of its own."""
    return [10000.0 ** (-i / n) for n in pairs for i in range(n)]


def _positions(case, gen, pairs, n, start=None):
    """[batch, n, axes] int32: places of a video of some width and height, or of rows behind `start`."""
    axes = len(pairs)
    at = torch.arange(n, device=DEV).expand(case["batch"], n)
    if start is not None:
        at = at + start.long().unsqueeze(-1)
    if case.get("far"):
        at = at + torch.randint(0, case["far"], (case["batch"], 1), generator=gen, device=DEV)
    h, w = 30, 52
    place = {1: [at], 2: [at // 128, at % 128], 3: [at // (h * w), at // w % h, at % w]}[axes]
    if case.get("far"):
        place[0] = at
    return torch.stack(place, dim=-1).int().contiguous()


def _split(pairs):
    return [int(x) for x in pairs.split(",")] if pairs else []


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        _handles(state)
    return state


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    B, hq, kv, d = case["batch"], case["heads_q"], case["heads_kv"], case["d"]
    state = {"case": case}
    pairs = _split(case.get("pairs", ""))
    if pairs:
        state["freq"] = torch.tensor(_frequencies(pairs), dtype=torch.float64, device=DEV)
        state["axis"] = torch.tensor([a for a, n in enumerate(pairs) for _ in range(n)], device=DEV)
    if case["op"] == "rotary":
        state["q"], state["k"] = _rows(case, gen, hq, case["n"]), _rows(case, gen, kv, case["n"])
        state["pos"] = _positions(case, gen, pairs, case["n"])
    elif case["op"] == "window":
        len_q, len_k = _window_lengths(case)
        state["q"], state["k"], state["v"] = (_rows(case, gen, h, n, g) for h, n, g in
                                              ((hq, case["n_q"], 1.5), (kv, case["n_k"], 1.0), (kv, case["n_k"], 1.0)))
        state["host_q"], state["host_k"], state["len_q"], state["len_k"] = len_q, len_k, None, None
        if case["ragged"]:
            state["len_q"] = torch.tensor(len_q, dtype=torch.int32, device=DEV)
            state["len_k"] = torch.tensor(len_k, dtype=torch.int32, device=DEV)
            for x, n in ((state["q"], len_q), (state["k"], len_k), (state["v"], len_k)):     # what stands behind a sequence is no number
                for b in range(B):
                    x[b, :, n[b]:] = float("nan")
    else:
        # pages in the order in which they were handed out and given back: none
        per = -(-case["longest"] // case["page"])
        pages = B * per + 3
        lengths = (_lengths(case, "cache", B, case["shortest"], case["longest"]) if case["op"] == "paged" else
                   [n - case["n"] for n in _lengths(case, "cache", B, case["n"], case["longest"])])
        in_use = [-(-(n + (case["n"] if case["op"] == "append" else 0)) // case["page"]) for n in lengths]
        order = torch.randperm(pages, generator=gen, device=DEV).int()[:B * per].reshape(B, per)
        used = torch.arange(per, device=DEV) < torch.tensor(in_use, device=DEV).unsqueeze(-1)
        state["table"] = torch.where(used, order, torch.full_like(order, -1)).contiguous()
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        shape = (pages, kv, case["page"], d)
        state["k_pages"] = torch.randn(shape, generator=gen, device=DEV, dtype=_dtype(case))
        state["v_pages"] = torch.randn(shape, generator=gen, device=DEV, dtype=_dtype(case))
        if case["op"] == "append":
            state["k"], state["v"] = _rows(case, gen, kv, case["n"]), _rows(case, gen, kv, case["n"])
            state["pos"] = _positions(case, gen, pairs, case["n"], state["lengths"]) if pairs else None
        else:
            state["q"] = _rows(case, gen, hq, 1, 1.5)
            for b, n in enumerate(lengths):                                                  # slots that no row has been put into
                if n % case["page"]:
                    page = int(state["table"][b, n // case["page"]])
                    state["k_pages"][page, :, n % case["page"]:] = float("nan")
                    state["v_pages"][page, :, n % case["page"]:] = float("nan")
    return state


def _handles(state):
    """What a program makes once per shape: frequencies, buffers of outputs, workspaces, the cache."""
    from paper_2608_26965_b200 import binding
    case, pairs = state["case"], _split(state["case"].get("pairs", ""))
    B, hq, kv, d, dtype = case["batch"], case["heads_q"], case["heads_kv"], case["d"], case["dtype"]
    state["rotary"] = binding.Rotary(d, pairs, frequencies=_frequencies(pairs), adjacent=case["adjacent"]) if pairs else None
    if case["op"] == "window":
        problem = binding.make_window_problem(B, hq, kv, case["n_q"], case["n_k"], d, dtype, case["left"], case["right"],
                                              sinks=case["sinks"])
        state["plan"] = binding.WindowPlan(problem, DEV)
    elif case["op"] in ("append", "paged"):
        problem = binding.make_cache_problem(B, hq, kv, d, dtype, case["page"], state["k_pages"].shape[0], state["table"].shape[1],
                                             left=case.get("left", -1), sinks=case.get("sinks", 0))
        state["cache"] = binding.PagedCache(problem, DEV, K_pages=state["k_pages"], V_pages=state["v_pages"],
                                            page_table=state["table"], lengths=state["lengths"])


# ---- plain forms ------------------------------------------------------------------------------------------

def _rotate(x, state, inverse=False):
    """Pairs of channels turned by position times frequency; channels behind the last pair stay."""
    case = state["case"]
    angle = state["pos"].double()[:, None, :, :].index_select(-1, state["axis"]) * state["freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    sin = -sin if inverse else sin
    R = state["freq"].numel()
    f = x.float()
    if case["adjacent"]:
        a, b = f[..., 0:2 * R:2], f[..., 1:2 * R:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = f[..., :R], f[..., R:2 * R]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, f[..., 2 * R:]), dim=-1).to(x.dtype)


def _slots(state, n):
    """Page and place in it of the rows lengths .. lengths + n - 1 of every sequence."""
    page = state["case"]["page"]
    at = state["lengths"].long().unsqueeze(-1) + torch.arange(n, device=DEV)
    return state["table"].long().gather(1, at // page), at % page


def _append(state):
    k = _rotate(state["k"], state) if state["pos"] is not None else state["k"]
    page, place = _slots(state, state["case"]["n"])
    state["k_pages"].transpose(1, 2)[page, place] = k.transpose(1, 2)
    state["v_pages"].transpose(1, 2)[page, place] = state["v"].transpose(1, 2)
    return state["k_pages"], state["v_pages"]


def _softmax(scores, visible, v):
    """Weighted mean of the values and log-sum-exp of the visible scores; of no scores zeros and -inf."""
    scores = scores.masked_fill(~visible, float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    e = torch.exp(scores - top.masked_fill(top == float("-inf"), 0.0))
    total = e.sum(dim=-1, keepdim=True)
    out = (e @ v) / total.masked_fill(total == 0, 1.0)
    return out, (top + torch.log(total)).squeeze(-1)


def _paged(state):
    case = state["case"]
    B, kv, d = case["batch"], case["heads_kv"], case["d"]
    rows = state["table"].shape[1] * case["page"]
    table = state["table"].long().clamp(min=0)
    j = torch.arange(rows, device=DEV)
    n = state["lengths"].long().unsqueeze(-1)
    written = j < n
    visible = written & ((j >= n - 1 - case["left"]) | (j < case["sinks"])) if case["left"] >= 0 else written
    k, v = (x[table].transpose(1, 2).reshape(B, kv, rows, d).float() for x in (state["k_pages"], state["v_pages"]))
    v = v.masked_fill(~written[:, None, :, None], 0.0)
    q = state["q"].float().reshape(B, kv, -1, d)
    out, lse = _softmax(q @ k.transpose(-1, -2) / math.sqrt(d), visible[:, None, None, :], v)
    return out.reshape(B, -1, 1, d).to(_dtype(case)), lse.reshape(B, -1, 1)


def _window(state):
    """Blocks of rows, as many at a time as their scores take 2 GB: all scores of the largest case would be 170 GB."""
    case = state["case"]
    B, hq, kv, d, n_q, n_k = (case[x] for x in ("batch", "heads_q", "heads_kv", "d", "n_q", "n_k"))
    left, right, sinks = case["left"], case["right"], min(case["sinks"], n_k)
    len_q, len_k = (torch.tensor(x, device=DEV).view(B, 1, 1) for x in (state["host_q"], state["host_k"]))
    shift = [b - a for a, b in zip(state["host_q"], state["host_k"])]
    k = state["k"].float()
    v = state["v"].float().masked_fill((torch.arange(n_k, device=DEV) >= len_k).view(B, 1, n_k, 1), 0.0)
    out = torch.zeros((B, hq, n_q, d), dtype=_dtype(case), device=DEV)
    lse = torch.zeros((B, hq, n_q), device=DEV)
    reach = (left if left >= 0 else n_k) + (right if right >= 0 else n_k) + sinks + max(shift) - min(shift)
    block = max(128, min(n_q, int(2 ** 31 / (4 * B * hq * min(n_k, reach + 1024)))))
    for r in range(0, n_q, block):
        end = min(n_q, r + block)
        lo = 0 if left < 0 else min(max(r + min(shift) - left, 0), n_k)
        hi = n_k if right < 0 else min(max(end + max(shift) + right, 0), n_k)
        j = torch.arange(n_k, device=DEV)
        j = torch.cat((j[:min(sinks, lo)], j[lo:hi]))
        i = torch.arange(r, end, device=DEV).view(1, -1, 1)
        p = i + len_k - len_q
        visible = (j < len_k) & (i < len_q)
        if right >= 0:
            visible = visible & (j <= p + right)
        if left >= 0:
            visible = visible & ((j >= p - left) | (j < sinks))
        if j.numel() == 0:
            j, visible = torch.zeros((1,), dtype=torch.long, device=DEV), torch.zeros((B, end - r, 1), dtype=torch.bool, device=DEV)
        q = state["q"][:, :, r:end].float().reshape(B, kv, -1, d)
        scores = q @ k[:, :, j].transpose(-1, -2) / math.sqrt(d)
        # the query heads of a key head one after the other
        seen = visible.unsqueeze(1).repeat(1, 1, hq // kv, 1)
        o, s = _softmax(scores, seen, v[:, :, j])
        there = (i < len_q).view(B, 1, -1)
        out[:, :, r:end] = o.reshape(B, hq, -1, d).masked_fill(~there.unsqueeze(-1), 0.0).to(out.dtype)
        lse[:, :, r:end] = s.reshape(B, hq, -1).masked_fill(~there, 0.0)
    return out, lse


def run(state):
    case = state["case"]
    if own:
        from paper_2608_26965_b200 import binding
        if case["op"] == "rotary":
            return binding.rotary_axes(state["rotary"], state["q"], state["k"], state["pos"], inverse=case["inverse"])
        if case["op"] == "append":
            cache = state["cache"]
            cache.cache_append(state["k"], state["v"], rotary=state["rotary"], positions=state["pos"])
            return cache.K_pages, cache.V_pages
        if case["op"] == "paged":
            return state["cache"].paged_attention_fwd(state["q"])
        return state["plan"].window_attention_fwd(state["q"], state["k"], state["v"], len_q=state["len_q"], len_k=state["len_k"])
    if case["op"] == "rotary":
        return _rotate(state["q"], state, case["inverse"]), _rotate(state["k"], state, case["inverse"])
    return {"append": _append, "paged": _paged, "window": _window}[case["op"]](state)


# ---- 64 bits ------------------------------------------------------------------------------------------------

def _turn64(x, case, pos, inverse):
    """A pair of channels as a complex number, times exp(i angle)."""
    y = x.double().clone()
    sections = [int(s) for s in case["pairs"].split(",")]
    R, c = sum(sections), 0
    for axis, count in enumerate(sections):
        for i in range(count):
            w = 10000.0 ** (-i / count)
            at = pos[:, :, axis].double() * (-w if inverse else w)
            a, b = (2 * c, 2 * c + 1) if case["adjacent"] else (c, R + c)
            z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(at), at)[:, None]
            y[..., a], y[..., b] = z.real.clone(), z.imag.clone()
            c += 1
    return y


def _attend64(q, k, v, keys_of, scale):
    """One head: q [rows, d], k and v [keys, d]; keys_of(first, last) says which keys rows first .. last - 1 see."""
    rows, keys = q.shape[0], k.shape[0]
    o = torch.zeros((rows, v.shape[1]), dtype=torch.float64, device=q.device)
    lse = torch.full((rows,), float("-inf"), dtype=torch.float64, device=q.device)
    step = max(1, int(1e8 // max(keys, 1)))
    for r in range(0, rows, step):
        e = min(rows, r + step)
        s = (q[r:e].double() @ k.double().T) * scale
        s = torch.where(keys_of(r, e), s, torch.tensor(float("-inf"), dtype=torch.float64, device=q.device))
        lse[r:e] = torch.logsumexp(s, dim=1)
        w = torch.exp(s - torch.where(torch.isinf(lse[r:e]), torch.zeros_like(lse[r:e]), lse[r:e])[:, None])
        o[r:e] = w @ v.double()
    return o, lse


def exact(case, seed):
    s = _inputs(case, seed)
    B, hq, kv, d = case["batch"], case["heads_q"], case["heads_kv"], case["d"]
    if case["op"] == "rotary":
        return _turn64(s["q"], case, s["pos"], case["inverse"]), _turn64(s["k"], case, s["pos"], case["inverse"])
    if case["op"] == "append":
        k = _turn64(s["k"], case, s["pos"], False) if case["pairs"] else s["k"].double()
        pools = s["k_pages"].double(), s["v_pages"].double()
        table, lengths = s["table"].tolist(), s["lengths"].tolist()
        for b in range(B):
            i = 0
            while i < case["n"]:                                    # a page's part of the new rows at a time
                page, place = divmod(lengths[b] + i, case["page"])
                m = min(case["n"] - i, case["page"] - place)
                for pool, x in zip(pools, (k, s["v"].double())):
                    pool[table[b][page], :, place:place + m] = x[b, :, i:i + m]
                i += m
        return pools
    scale = 1.0 / math.sqrt(d)
    left = case["left"] if case["left"] >= 0 else 1 << 40
    if case["op"] == "paged":
        if B * hq * case["longest"] > 4e8:
            return None
        out = torch.zeros((B, hq, 1, d), dtype=torch.float64, device=DEV)
        lse = torch.full((B, hq, 1), float("-inf"), dtype=torch.float64, device=DEV)
        for b, n in enumerate(s["lengths"].tolist()):
            if n == 0:
                continue
            pages = s["table"][b, :-(-n // case["page"])].long()
            j = torch.arange(n, device=DEV)
            see = ((j > n - 2 - left) | (j < case["sinks"])).unsqueeze(0)
            for g in range(kv):
                k, v = (x[pages, g].reshape(-1, d)[:n] for x in (s["k_pages"], s["v_pages"]))
                heads = slice(g * (hq // kv), (g + 1) * (hq // kv))
                o, l = _attend64(s["q"][b, heads, 0], k, v, lambda r, e: see, scale)
                out[b, heads, 0], lse[b, heads, 0] = o, l
        return out, lse
    right = case["right"] if case["right"] >= 0 else 1 << 40
    out = torch.zeros((B, hq, case["n_q"], d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((B, hq, case["n_q"]), dtype=torch.float64, device=DEV)
    for b in range(B):
        a, n = s["host_q"][b], s["host_k"][b]
        j = torch.arange(n, device=DEV)

        def keys_of(r, e):
            p = torch.arange(r, e, device=DEV).unsqueeze(1) + (n - a)
            return (j <= p + right) & ((j >= p - left) | (j < case["sinks"]))

        for h in range(hq):
            g = h // (hq // kv)
            out[b, h, :a], lse[b, h, :a] = _attend64(s["q"][b, h, :a], s["k"][b, g, :n], s["v"][b, g, :n], keys_of, scale)
    return out, lse
