"""What attention along the voxels of a batch of grids is timed on: attention over packed sequences with its gradients, the
paged cache that a running sequence keeps its keys and values in, and attention of one new row over that cache.

``own`` chooses the side: the plain form in elementary torch operations (32 bits throughout, one rounding at the end),
or this library's calls on the same data.  A case is a plain dict; ``op`` says what one pass does:

``attn`` / ``attn_grad``  attention of every row over its sequence's rows (or over those of another set of sequences), and
                          its gradients
``cache``                 rows written into the pages of their sequences, in the cache's type, and read back
``step``                  one new row of each of many running sequences over what the cache holds of it

    s_ij = scale q_i . k_j                     j over the keys of i's sequence; causal: i's distance to the last query is at
                                               most j's distance to the last key
    lse_i = log sum_j exp(s_ij),  out_i = sum_j exp(s_ij - lse_i) v_j          (no key: -inf and zeros)

Query head h reads key and value head h // (heads / kv_heads).  A cache of 8 bits holds e4m3 values q and one exponent e for
every row and head, value = q 2^e, e the least with which no finite value of the row passes 448.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
_BIAS = 127


# ------------------------------------------------------------------------------------------ cases
def _attn(op, rows, seqs, heads, kv_heads, dim, dtype, causal, even=False, kv_rows=0, glse=False):
    return dict(op=op, rows=rows, seqs=seqs, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, causal=causal, even=even,
                kv_rows=kv_rows, glse=glse)


def listed():
    return [
        # eight running scenes get one row each: the smallest call, all latency
        dict(name="step_8_bf16_d64", op="step", seqs=8, longest=700, page=64, heads=8, kv_heads=2, dim=64, dtype="bf16", store="bf16"),
        # a LiDAR scan of a million voxels stands in the cache, one more row looks at all of it
        dict(name="step_lidar_bf16_d64", op="step", seqs=1, longest=986_880, page=256, heads=8, kv_heads=2, dim=64, dtype="bf16", store="bf16"),
        # 64 running scenes of up to 32k rows, cache of 8 bits in small pages
        dict(name="step_64_e4m3_d128", op="step", seqs=64, longest=32_768, page=16, heads=16, kv_heads=4, dim=128, dtype="bf16", store="e4m3"),
        # one row of each of 24 scenes into its page, odd sizes
        dict(name="cache_rows_24_f16_d40", op="cache", rows=24, seqs=24, start=500, page=24, kv_heads=3, dim=40, dtype="f16", store="f16"),
        # all voxels of a scan into a cache of 8 bits, and back
        dict(name="cache_lidar_e4m3_d64", op="cache", rows=986_880, seqs=1, start=0, page=256, kv_heads=2, dim=64, dtype="bf16", store="e4m3"),
        # attention inside every leaf of a grid: short sequences, the finest level of a small scene
        _attn("attn", 203_132, 3_400, 4, 4, 32, "f16", False) | dict(name="attn_leaves_f16_d32"),
        # a coarse level of four indoor scenes in voxel order, generated one after the other
        _attn("attn", 65_536, 4, 8, 2, 64, "bf16", True) | dict(name="attn_indoor_bf16_d64"),
        # one long sequence, wide heads in groups of four
        _attn("attn", 32_768, 1, 16, 4, 128, "bf16", True) | dict(name="attn_long_bf16_d128"),
        # odd sizes, keys from another set of rows, full precision
        _attn("attn", 5_003, 7, 3, 1, 45, "f32", False, kv_rows=9_001) | dict(name="attn_odd_f32_d45"),
        # training on the leaves of a grid
        _attn("attn_grad", 203_132, 3_400, 4, 4, 32, "bf16", False) | dict(name="attn_grad_leaves_bf16_d32"),
        # training on windows of 1,024 voxels in index order
        _attn("attn_grad", 131_072, 128, 4, 4, 64, "f16", False, even=True) | dict(name="attn_grad_windows_f16_d64"),
        # training on one long sequence, wide heads in groups of four
        _attn("attn_grad", 16_384, 1, 16, 4, 128, "bf16", True) | dict(name="attn_grad_long_bf16_d128"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn", "attn_grad", "attn_grad", "cache", "step", "step"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    dim = rng.choice((16, 32, 32, 40, 64, 64, 64, 96, 128, 128, _log_int(rng, 8, 256)))
    kv_heads = rng.choice((1, 1, 2, 2, 3, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
    if op in ("cache", "step"):
        store = rng.choice((dtype, "e4m3"))
        page = rng.choice((16, 16, 64, 64, 128, 256, rng.randint(5, 300)))
        seqs = _log_int(rng, 1, 256)
        width = 2 * kv_heads * dim * max(_BYTES[store], 2)          # bytes of a position, keys and values
        if op == "cache":
            rows = _log_int(rng, seqs, max(seqs, min(986_880, (1 << 28) // width)))
            return dict(op=op, rows=rows, seqs=seqs, start=rng.choice((0, _log_int(rng, 1, 1_000))), page=page, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store)
        longest = _log_int(rng, 1, min(986_880, (1 << 30) // (seqs * width)))
        return dict(op=op, seqs=seqs, longest=longest, page=page, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store)
    heads = min(heads, 16 // kv_heads * kv_heads)
    even = rng.random() < 0.4
    seqs = rng.choice((1, 2, 4, _log_int(rng, 1, 2_000)))
    # the pairs of rows and keys, in all heads, of a quarter of the largest listed case at most
    most = (1 << 32) // heads // (4 if dtype == "f32" else 1) // (2 if dim > 128 else 1) // (2 if op == "attn_grad" else 1)
    rows = _log_int(rng, 1, min(200_000, math.isqrt(most * (seqs if even else max(1, seqs // 2)))))
    kv_rows = rng.choice((0, 0, 0, _log_int(rng, 1, max(1, rows))))
    return _attn(op, rows, min(seqs, rows), heads, kv_heads, dim, dtype, rng.random() < 0.5, even, kv_rows, op == "attn_grad" and rng.random() < 0.3)


# ------------------------------------------------------------------------------------------ lengths: the case's own, whatever the seed
def _bounds(rows, seqs, even, salt):
    """First rows of the sequences and the end: equal lengths, or cuts anywhere (some sequences empty where there are many)."""
    if even:
        return np.arange(seqs + 1, dtype=np.int64) * rows // seqs
    rng = np.random.default_rng([rows, seqs, salt])
    return np.concatenate([[0], np.sort(rng.integers(0, rows + 1, size=seqs - 1)), [rows]]).astype(np.int64)


def _attn_bounds(case):
    q = _bounds(case["rows"], case["seqs"], case["even"], 1)
    return q, _bounds(case["kv_rows"], case["seqs"], case["even"], 2) if case["kv_rows"] else q


def _lengths(case):
    """Rows that the cache holds of each sequence: the first has the most, one of many has none."""
    rng = np.random.default_rng([case["longest"], case["seqs"]])
    lens = rng.integers(0, case["longest"] + 1, size=case["seqs"])
    lens[0] = case["longest"]
    if case["seqs"] >= 8:
        lens[1] = 0
    return lens.astype(np.int64)


def _starts(case):
    rng = np.random.default_rng([case["start"], case["seqs"], 3])
    return rng.integers(0, case["start"] + 1, size=case["seqs"]).astype(np.int64)


# ------------------------------------------------------------------------------------------ what a program has in hand
def _normal(shape, gen, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _device(a, dtype=torch.int64):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def _pages(case, ends, seed):
    """The table of pages [seqs, columns] (-1: none) for sequences that reach up to `ends`, in any order, and their number."""
    need = -(-ends // case["page"])
    order = np.random.default_rng([seed, 5]).permutation(int(need.sum()) + 3)
    table = np.full((len(ends), max(1, int(need.max()))), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < need[:, None]] = order[:int(need.sum())]
    return table, len(order)


def _empty_cache(case, pages):
    pitch = -(-case["dim"] // 16) * 16
    shape = (pages, case["kv_heads"], case["page"], pitch)
    if case["store"] != "e4m3":
        return dict(k=torch.zeros(shape, dtype=_DT[case["store"]], device="cuda"), v=torch.zeros(shape, dtype=_DT[case["store"]], device="cuda"))
    new = lambda: torch.zeros(shape, dtype=torch.float8_e4m3fn, device="cuda")
    exp = lambda: torch.zeros(shape[:3], dtype=torch.uint8, device="cuda")
    return dict(k=new(), v=new(), k_exp=exp(), v_exp=exp())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed((7919 * seed + 31) % (1 << 62))
    dt, op, d, kvh = _DT[case["dtype"]], case["op"], case["dim"], case["kv_heads"]
    s = dict(case=case)
    if op in ("attn", "attn_grad"):
        bq, bk = _attn_bounds(case)
        n, m, h = case["rows"], int(bk[-1]), case["heads"]
        if case["kv_rows"]:
            s["q"], s["k"], s["v"] = _normal((n, h, d), gen, dt, 1.5), _normal((m, kvh, d), gen, dt), _normal((m, kvh, d), gen, dt)
        else:               # out of one projection
            both = torch.randn((n, h + 2 * kvh, d), generator=gen, device="cuda")
            both[:, :h] *= 1.5
            both = both.to(dt)
            s["q"], s["k"], s["v"] = both[:, :h], both[:, h:h + kvh], both[:, h + kvh:]
        s["scale"] = d ** -0.5
        s["plan"] = _plan(bq, bk, h)
        if own:
            import paper_2407_01781_amd as fx
            s["seqs"] = fx.build_sequences(np.stack([bq[:-1], bq[1:]], 1))
            s["kv_seqs"] = fx.build_sequences(np.stack([bk[:-1], bk[1:]], 1)) if case["kv_rows"] else None
        if op == "attn_grad":
            s["out"], s["lse"] = _attention(s)      # what the forward pass wrote
            s["gout"] = _normal((n, h, d), gen, dt)
            s["glse"] = _normal((h, n), gen, torch.float32) if case["glse"] else None
        return s
    if op == "cache":
        bounds, start = _bounds(case["rows"], case["seqs"], case["rows"] == case["seqs"], 1), _starts(case)
        lens = np.diff(bounds)
        table, pages = _pages(case, start + lens, seed)
        s.update(_empty_cache(case, pages))
        both = _normal((case["rows"], 2 * kvh, d), gen, dt) * torch.exp(torch.randn((1, 2 * kvh, 1), generator=gen, device="cuda")).to(dt)
        s["new_k"], s["new_v"] = both[:, :kvh], both[:, kvh:]
        seq = np.repeat(np.arange(case["seqs"]), lens)
        s["row_seq"], s["row_pos"] = _device(seq), _device(np.arange(case["rows"]) - bounds[seq] + start[seq])
        s["table"], s["start"] = _device(table, torch.int32), _device(start, torch.int32)
        if own:
            import paper_2407_01781_amd as fx
            s["seqs"] = fx.build_sequences(np.stack([bounds[:-1], bounds[1:]], 1))
    else:
        lens = _lengths(case)
        table, pages = _pages(case, lens, seed)
        s.update(_empty_cache(case, pages))
        shape = (*s["k"].shape[:3], d)
        for name in ("k", "v"):
            rows = torch.randn(shape, generator=gen, device="cuda")
            if case["store"] == "e4m3":
                codes, exp = _quantise(rows.to(dt).float())
                s[name][..., :d].view(torch.uint8).copy_(codes.view(torch.uint8))
                s[name + "_exp"].copy_(exp)
            else:
                s[name][..., :d] = rows.to(dt)
        s["q"] = _normal((case["seqs"], case["heads"], d), gen, dt, 1.5)
        s["scale"] = d ** -0.5
        s["table"], s["lens"] = _device(table, torch.int32), _device(lens, torch.int32)
        s["groups"] = _by_length(np.ones_like(lens), lens, max(case["heads"], 8 * d * kvh))
    if own:
        import paper_2407_01781_amd as fx
        s["cache"] = fx.KVCache(s["k"], s["v"], dim=d, k_exp=s.get("k_exp"), v_exp=s.get("v_exp"))
    return s


# ------------------------------------------------------------------------------------------ the plain forms
_SCORES = 1 << 30           # scores held at a time


def _by_length(lens_q, lens_k, heads):
    """Sequences of like length together, as lists of (numbers, longest of the queries, longest of the keys): padded to the
    longest, a group's scores are _SCORES at most (or one sequence's)."""
    groups, order = [], np.argsort(lens_k * max(1, int(lens_q.max(initial=0))) + lens_q, kind="stable")[::-1].copy()
    at = 0
    while at < len(order):
        size, a, b = 0, 0, 0
        while at + size < len(order):
            a2, b2 = max(a, int(lens_q[order[at + size]])), max(b, int(lens_k[order[at + size]]))
            if size and (size + 1) * a2 * b2 * heads > _SCORES:
                break
            a, b, size = a2, b2, size + 1
        groups.append((_device(order[at:at + size]), max(a, 1), max(b, 1)))
        at += size
    return groups


def _plan(bq, bk, heads):
    return dict(groups=_by_length(np.diff(bq), np.diff(bk), heads), first_q=_device(bq[:-1]), len_q=_device(np.diff(bq)),
                first_k=_device(bk[:-1]), len_k=_device(np.diff(bk)))


def _padded(x, first, lens, longest):
    """Rows of the sequences as [sequences, heads, longest, dim] in 32 bits, zeros behind their ends."""
    at = torch.arange(longest, device=x.device)[None, :]
    some = at < lens[:, None]
    rows = x[torch.where(some, first[:, None] + at, 0).clamp(max=max(0, x.shape[0] - 1))] if x.shape[0] else x.new_zeros((len(lens), longest, *x.shape[1:]))
    return (rows.float() * some[:, :, None, None]).transpose(1, 2).contiguous(), some


def _probabilities(s, ids, lq, lk, heads):
    """q, k, v of the chosen heads and the probabilities [sequences, kv heads, queries of the group, keys] with their lse."""
    p, case = s["plan"], s["case"]
    g = case["heads"] // case["kv_heads"]
    fq, nq, fk, nk = (p[x][ids] for x in ("first_q", "len_q", "first_k", "len_k"))
    q, some_q = _padded(s["q"][:, heads.start * g:heads.stop * g], fq, nq, lq)
    k, some_k = _padded(s["k"][:, heads], fk, nk, lk)
    v, _ = _padded(s["v"][:, heads], fk, nk, lk)
    b, hk = k.shape[:2]
    q = q.reshape(b, hk, g * lq, -1)
    scores = torch.matmul(q, k.transpose(2, 3)).reshape(b, hk, g, lq, lk) * s["scale"]
    seen = some_k[:, None, :] & some_q[:, :, None]
    if case["causal"]:
        i, j = torch.arange(lq, device=q.device), torch.arange(lk, device=q.device)
        seen = seen & ((nq[:, None] - i)[:, :, None] <= (nk[:, None] - j)[:, None, :])
    scores = scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(4, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    e = scores.sub_(top).exp_()
    total = e.sum(4, keepdim=True)
    lse = (top + torch.log(total)).squeeze(4)
    e /= torch.where(total > 0, total, torch.ones_like(total))
    return q, k, v, e.reshape(b, hk, g * lq, lk), lse, some_q, some_k, fq, fk


def _head_sets(s, ids, lq, lk):
    """Key heads a set at a time, so that no more scores are held than _SCORES."""
    case = s["case"]
    a_head = len(ids) * lq * lk * (case["heads"] // case["kv_heads"])
    step = max(1, min(case["kv_heads"], _SCORES // max(1, a_head)))
    return [slice(h, min(h + step, case["kv_heads"])) for h in range(0, case["kv_heads"], step)]


def _put(into, heads, values, some, first):
    """Values [sequences, heads, longest, ...] back to rows."""
    seq, at = some.nonzero(as_tuple=True)
    into[:, heads][first[seq] + at] = values.transpose(1, 2)[seq, at].to(into.dtype)


def _attention(s):
    case = s["case"]
    g = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.full((case["rows"], case["heads"]), -math.inf, device="cuda")
    for ids, lq, lk in s["plan"]["groups"]:
        for heads in _head_sets(s, ids, lq, lk):
            q, k, v, p, part, some_q, _, fq, _ = _probabilities(s, ids, lq, lk, heads)
            b, hk = k.shape[:2]
            mine = slice(heads.start * g, heads.stop * g)
            _put(out, mine, torch.matmul(p, v).reshape(b, hk * g, lq, -1), some_q, fq)
            _put(lse, mine, part.reshape(b, hk * g, lq), some_q, fq)
    return out, lse.t().contiguous()


def _attention_grad(s):
    case = s["case"]
    g = case["heads"] // case["kv_heads"]
    gq, gk, gv = (torch.zeros(s[x].shape, dtype=s[x].dtype, device="cuda") for x in ("q", "k", "v"))
    for ids, lq, lk in s["plan"]["groups"]:
        for heads in _head_sets(s, ids, lq, lk):
            q, k, v, p, _, some_q, some_k, fq, fk = _probabilities(s, ids, lq, lk, heads)
            b, hk = k.shape[:2]
            mine = slice(heads.start * g, heads.stop * g)
            go, _ = _padded(s["gout"][:, mine], fq, some_q.sum(1), lq)
            go = go.reshape(b, hk, g * lq, -1)
            _put(gv, heads, torch.matmul(p.transpose(2, 3), go), some_k, fk)
            dp = torch.matmul(go, v.transpose(2, 3))
            away = (p * dp).sum(3, keepdim=True)
            if s["glse"] is not None:
                more, _ = _padded(s["glse"].t()[:, mine, None], fq, some_q.sum(1), lq)
                away -= more.reshape(b, hk, g * lq, 1)
            ds = dp.sub_(away).mul_(p).mul_(s["scale"])
            _put(gq, mine, torch.matmul(ds, k).reshape(b, hk * g, lq, -1), some_q, fq)
            _put(gk, heads, torch.matmul(ds.transpose(2, 3), q), some_k, fk)
    return gq, gk, gv


def _quantise(x):
    """e4m3 values and exponents (plus _BIAS) of rows in 32 bits."""
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    m, e = torch.frexp(top)                    # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(top > 0, e, torch.full_like(e, -_BIAS)).clamp(min=-_BIAS)
    scaled = torch.where(torch.isfinite(x), torch.ldexp(x, -e[..., None]), torch.full_like(x, math.nan))
    return scaled.to(torch.float8_e4m3fn), (e + _BIAS).to(torch.uint8)


def _values(codes, exp):
    return codes.float() if exp is None else torch.ldexp(codes.float(), exp[..., None].int() - _BIAS)


def _cache(s):
    case, d = s["case"], s["case"]["dim"]
    page = s["table"][s["row_seq"], s["row_pos"] // case["page"]].long()
    slot = s["row_pos"] % case["page"]
    out = []
    for name in ("k", "v"):
        x = s["new_" + name]
        if case["store"] == "e4m3":
            codes, exp = _quantise(x.float())
            s[name].view(torch.uint8)[..., :d][page, :, slot] = codes.view(torch.uint8)
            s[name + "_exp"][page, :, slot] = exp
            held = s[name].view(torch.uint8)[..., :d][page, :, slot].view(torch.float8_e4m3fn)
            out.append(_values(held, s[name + "_exp"][page, :, slot]).to(x.dtype))
        else:
            s[name][..., :d][page, :, slot] = x
            out.append(s[name][..., :d][page, :, slot])
    return tuple(out)


def _step(s):
    case, d, q = s["case"], s["case"]["dim"], s["q"]
    g, kvh = case["heads"] // case["kv_heads"], case["kv_heads"]
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, device="cuda")
    for ids, _, longest in s["groups"]:
        at = torch.arange(longest, device="cuda")
        seen = at[None, :] < s["lens"][ids][:, None]
        page = s["table"][ids][:, at // case["page"]].long().clamp(min=0)
        held = [_values(s[x][..., :d][page, :, at % case["page"]], None if case["store"] != "e4m3" else s[x + "_exp"][page, :, at % case["page"]]).transpose(1, 2).contiguous()
                for x in ("k", "v")]
        scores = torch.matmul(q[ids].float().reshape(-1, kvh, g, d), held[0].transpose(2, 3)) * s["scale"]
        scores = scores.masked_fill_(~seen[:, None, None], -math.inf)
        top = scores.amax(3, keepdim=True)
        top = torch.where(top > -math.inf, top, torch.zeros_like(top))
        e = torch.exp(scores - top)
        total = e.sum(3, keepdim=True)
        lse[ids] = (top + torch.log(total)).reshape(-1, kvh * g)
        e = e / torch.where(total > 0, total, torch.ones_like(total))
        out[ids] = torch.matmul(e, held[1]).reshape(-1, kvh * g, d).to(q.dtype)
    return out, lse


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        return {"attn": _attention, "attn_grad": _attention_grad, "cache": _cache, "step": _step}[op](s)
    import paper_2407_01781_amd as fx
    if op == "attn":
        return fx.attention_fwd(s["seqs"], s["q"], s["k"], s["v"], causal=case["causal"], scale=s["scale"], kv_seqs=s["kv_seqs"])
    if op == "attn_grad":
        return fx.attention_bwd(s["seqs"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["gout"], grad_lse=s["glse"], causal=case["causal"],
                                scale=s["scale"], kv_seqs=s["kv_seqs"])
    if op == "cache":
        fx.cache_write(s["cache"], s["table"], s["start"], s["new_k"], s["new_v"], seqs=s["seqs"])
        return fx.cache_read(s["cache"], s["table"], s["start"], s["seqs"], dtype=s["new_k"].dtype)
    return fx.attention_step(s["cache"], s["table"], s["lens"], s["q"], scale=s["scale"])


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def _pairs(case):
    """Pairs of a query and a key that it sees."""
    bq, bk = _attn_bounds(case)
    a, b = np.diff(bq).astype(np.float64), np.diff(bk).astype(np.float64)
    if not case["causal"]:
        return float((a * b).sum())
    n = np.minimum(a, b)                        # rows that see a key; the last sees all b, each before it one less
    return float((n * b - n * (n - 1) / 2).sum())


def work(case):
    e, h, kvh, d, op = _BYTES[case["dtype"]], case.get("heads"), case["kv_heads"], case["dim"], case["op"]
    if op in ("attn", "attn_grad"):
        n, m = case["rows"], case["kv_rows"] or case["rows"]
        q, kv, lse, pairs = n * h * d * e, m * kvh * d * e, 4 * n * h, _pairs(case) * h
        if op == "attn":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * pairs * d}
        return {"bytes": 4 * q + 4 * kv + lse * (2 if case["glse"] else 1), "flops": 10 * pairs * d}
    held = 2 * kvh * (d * _BYTES[case["store"]] + (case["store"] == "e4m3"))        # bytes of a position
    if op == "cache":
        return {"bytes": case["rows"] * (2 * held + 4 * kvh * d * e), "flops": 4 * case["rows"] * kvh * d}
    total = int(_lengths(case).sum())
    return {"bytes": total * held + case["seqs"] * h * (2 * d * e + 4) + 4 * (total // case["page"]), "flops": 4 * total * h * d}


# ------------------------------------------------------------------------------------------ the definition in 64 bits
def _grid_of_e4m3(x):
    """Rows in 64 bits as what a cache of 8 bits holds of them, from the format's own numbers."""
    top = np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.ceil(np.log2(top / 448.0)), -_BIAS)
    e = np.where(448.0 * np.exp2(e - 1) >= top, e - 1, np.where(448.0 * np.exp2(e) < top, e + 1, e)).clip(min=-_BIAS)     # log2 is off by a digit at powers of two
    u = x * np.exp2(-e)
    with np.errstate(divide="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(u))), -6) - 3)      # three digits behind the leading one, subnormal below 2^-6
    return np.where(u == 0, u, np.rint(u / step) * step) * np.exp2(e)


def exact(case, seed):
    op = case["op"]
    if op == "cache":
        if case["rows"] * case["kv_heads"] * case["dim"] > 1 << 28:
            return None
        s = prepare(case, seed)
        rows = [s[x].double().cpu().numpy() for x in ("new_k", "new_v")]
        return tuple(torch.from_numpy(_grid_of_e4m3(r) if case["store"] == "e4m3" else r) for r in rows)
    s = prepare(case, seed)
    g = case["heads"] // case["kv_heads"]
    if op == "step":
        lens, out, lse = _lengths(case), [], []
        for b, n in enumerate(lens):
            q = s["q"][b].double()
            if n == 0:
                out.append(torch.zeros_like(q))
                lse.append(torch.full((case["heads"],), -math.inf, dtype=torch.float64, device="cuda"))
                continue
            pages = s["table"][b, :-(-int(n) // case["page"])].long()
            rows = []
            for x in ("k", "v"):
                t = s[x][pages][..., :case["dim"]].double()
                if case["store"] == "e4m3":
                    t = t * torch.exp2(s[x + "_exp"][pages].double() - _BIAS)[..., None]
                rows.append(t.transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(g, 0))
            score = (rows[0] * q[:, None, :]).sum(2) * s["scale"]
            lse.append(torch.logsumexp(score, 1))
            out.append((torch.softmax(score, 1)[:, :, None] * rows[1]).sum(1))
        return torch.stack(out), torch.stack(lse)
    bq, bk = _attn_bounds(case)
    a, b = np.diff(bq), np.diff(bk)
    if float((a * b).sum()) * case["heads"] * case["dim"] * (5 if op == "attn_grad" else 2) > 1.2e13:
        return None
    n, h = case["rows"], case["heads"]
    q, k, v = (s[x].double().transpose(0, 1).contiguous() for x in ("q", "k", "v"))         # [heads, rows, dim]
    grad = op == "attn_grad"
    out, lse = torch.zeros_like(q), torch.full((h, n), -math.inf, dtype=torch.float64, device="cuda")
    if grad:
        go = s["gout"].double().transpose(0, 1).contiguous()
        gl = s["glse"].double() if s["glse"] is not None else torch.zeros_like(lse)
        gq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i0, i1, j0, j1 in zip(bq[:-1], bq[1:], bk[:-1], bk[1:]):
        if i1 == i0 or j1 == j0:
            continue
        part = max(1, min(i1 - i0, (1 << 26) // int(j1 - j0)))
        kv_set = max(1, (1 << 27) // int(part * (j1 - j0) * g))             # key heads at a time
        for head in range(0, case["kv_heads"], kv_set):
            kh = slice(head, min(head + kv_set, case["kv_heads"]))
            qh = slice(kh.start * g, kh.stop * g)
            kk, vv = (t[kh, j0:j1].repeat_interleave(g, 0) for t in (k, v))
            for r in range(i0, i1, part):
                rows = slice(r, min(r + part, i1))
                score = torch.bmm(q[qh, rows], kk.transpose(1, 2).contiguous()) * s["scale"]
                if case["causal"]:
                    last = torch.arange(rows.start, rows.stop, device="cuda") - i1 + (j1 - j0)      # the key that a row sees last
                    score.masked_fill_(torch.arange(j1 - j0, device="cuda")[None, :] > last[:, None], -math.inf)
                lse[qh, rows] = torch.logsumexp(score, 2)
                p = torch.nan_to_num(torch.softmax(score, 2), nan=0.0)
                del score
                if not grad:
                    out[qh, rows] = torch.bmm(p, vv)
                    continue
                fold = lambda t: t.reshape(-1, g, *t.shape[1:]).sum(1)
                gv[kh, j0:j1] += fold(torch.bmm(p.transpose(1, 2).contiguous(), go[qh, rows]))
                dp = torch.bmm(go[qh, rows], vv.transpose(1, 2).contiguous())
                ds = p * (dp - (dp * p).sum(2, keepdim=True) + gl[qh, rows, None]) * s["scale"]
                del dp, p
                gq[qh, rows] = torch.bmm(ds, kk)
                gk[kh, j0:j1] += fold(torch.bmm(ds.transpose(1, 2).contiguous(), q[qh, rows]))
    back = lambda t: t.transpose(0, 1).contiguous()
    return (back(gq), back(gk), back(gv)) if grad else (back(out), lse)
