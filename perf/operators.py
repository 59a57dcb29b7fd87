"""What a program that serves (or trains with positions) calls besides the jagged attention steps of cases.py, as a list
of cases: rotary positions on jagged rows, appending rows to a paged cache of keys and values, and the attention of new
rows over that cache, through the public entry points of paper_2508_04711_amd (`own`) or written out in elementary torch
operations in 32 bits (the plain form).

A case is a dict of plain values.  "op" says what a pass calls:
  rotary   hstu_rotary_fwd on (q, k), then hstu_rotary_bwd on (dq, dk): one attention layer of a training step
  append   hstu_cache_append: new rows of k and v (and their timestamps) into the cache, k and q rotated
  attn     hstu_paged_attn_fwd, or hstu_paged_attn_bias_fwd where "buckets" > 0
Lengths ("lo".."hi" of the rotary rows and of the cached histories, "new_lo".."new_hi" of the new rows) are drawn with the
case's own "len_seed", uniform or lognormal with median "mid", so a case's work does not depend on the seed of its values.
"""
import math

import numpy as np
import torch

own = False


def _lib():
    import paper_2508_04711_amd as lib
    return lib


def _case(name, op, dtype, batch, lo, hi, heads, d, *, mid=0, len_seed=0, kv_heads=0, page=64, new_lo=1, new_hi=1,
          causal=True, buckets=0, rotary=0, interleaved=False, scaling="none"):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "lo": lo, "hi": hi, "heads": heads, "d": d, "mid": mid,
            "len_seed": len_seed, "kv_heads": kv_heads or heads, "page": page, "new_lo": new_lo, "new_hi": new_hi,
            "causal": causal, "buckets": buckets, "rotary": rotary, "interleaved": interleaved, "scaling": scaling}


def listed():
    return [
        # positions in a handful of short histories in fp32, half of each head rotated: gradient checks, all latency
        _case("rotary_small", "rotary", "f32", 4, 1, 64, 2, 32, rotary=16, interleaved=True),
        # positions of the largest single-GPU training step: very skewed, very long histories, frequencies stretched
        _case("rotary_train", "rotary", "bf16", 8, 64, 32768, 8, 128, mid=8192, rotary=128, scaling="by_parts"),
        # one new event of each of 64 users joins their cached histories
        _case("append_one", "append", "bf16", 64, 512, 4096, 4, 128, rotary=128),
        # whole histories of new users fill their pages, with the timestamps that the bias needs
        _case("append_histories", "append", "bf16", 16, 512, 4096, 4, 128, new_lo=512, new_hi=4096, rotary=64,
              interleaved=True, buckets=64),
        # one user's next event over a short history: the smallest request, all latency
        _case("attn_one", "attn", "bf16", 1, 200, 200, 4, 128),
        # a reference run in fp32 over ordinary histories
        _case("attn_f32", "attn", "f32", 8, 64, 512, 4, 64, new_hi=4),
        # one new event of each of 64 users over ordinary long histories
        _case("attn_next", "attn", "bf16", 64, 512, 4096, 4, 128),
        # one new event over very skewed, very long histories
        _case("attn_next_long", "attn", "bf16", 8, 64, 32768, 8, 128, mid=8192),
        # many small requests, query heads that share keys and values, small pages
        _case("attn_next_shared", "attn", "bf16", 128, 1, 2048, 8, 64, kv_heads=2, page=16),
        # a few new events over histories with the learned timestamp bias
        _case("attn_bias", "attn", "bf16", 32, 64, 4096, 4, 128, new_hi=4, buckets=64),
        # hundreds of candidates scored against a cached history that they are not part of
        _case("attn_candidates", "attn", "bf16", 8, 1024, 8192, 4, 128, new_lo=200, new_hi=600, causal=False),
        # a burst of new events over long histories, each seeing those before it: the largest
        _case("attn_burst", "attn", "bf16", 4, 4096, 16384, 8, 128, new_lo=512, new_hi=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# No drawn case does more than the largest listed ones.
_MAX = {"rotary": (8.0e8, 1e18), "append": (3.0e8, 1e18), "attn": (2.2e9, 1.2e11)}
_MAX_SCORES = 6.0e8  # padded scores of the plain form


def draw(rng):
    """One more case of the ranges above: the operator first, then sizes over their logarithm."""
    while True:
        op = rng.choice(["rotary", "append", "attn", "attn", "attn"])
        seed = rng.randrange(1 << 30)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([32, 64, 128, 128])
        rotary = rng.choice([d, d, d // 2])
        if op == "rotary":
            hi = _log_int(rng, 16, 32768)
            c = _case("", op, dtype, _log_int(rng, 1, 512), max(1, hi // rng.choice([2, 8, 64])), hi, rng.choice([1, 2, 4, 8]),
                      d, len_seed=seed, rotary=rotary, interleaved=rng.random() < 0.5,
                      scaling=rng.choice(["none", "linear", "base", "by_parts"]))
        elif op == "append":
            hi = _log_int(rng, 64, 8192)
            many = rng.random() < 0.5
            c = _case("", op, dtype, _log_int(rng, 1, 256), max(1, hi // rng.choice([2, 8, 64])), hi, rng.choice([2, 4, 8]),
                      d, len_seed=seed, rotary=rng.choice([0, rotary, rotary]), interleaved=rng.random() < 0.5,
                      page=rng.choice([16, 32, 64, 128]), new_hi=_log_int(rng, 16, 4096) if many else rng.choice([1, 1, 4]),
                      buckets=rng.choice([0, 64]))
            if c["heads"] > 2 and rng.random() < 0.3:
                c["kv_heads"] = c["heads"] // 2
        else:
            hi = _log_int(rng, 16, 32768)
            new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 1024)])
            c = _case("", op, dtype if new <= 64 else "bf16", _log_int(rng, 1, 256), max(1, hi // rng.choice([2, 8, 64])), hi,
                      rng.choice([2, 4, 8]), d, len_seed=seed, page=rng.choice([16, 32, 64, 128]), new_lo=(new + 1) // 2,
                      new_hi=new, causal=rng.random() < 0.7, buckets=rng.choice([0, 0, 0, 32, 64]))
            if rng.random() < 0.3:
                c["kv_heads"] = max(1, c["heads"] // rng.choice([2, 4, 8]))
        w = work(c)
        padded = max(_lengths(c)[0]) * max(_lengths(c)[1]) * c["batch"] * c["heads"] if op == "attn" else 0
        cached = 2 * sum(_lengths(c)[0]) * c["kv_heads"] * d * (2 if dtype == "bf16" else 4)
        if op == "append" and cached > 6.0e8:
            continue
        if w["bytes"] <= _MAX[op][0] and w["flops"] <= _MAX[op][1] and padded <= _MAX_SCORES:
            del c["name"]
            return c


def _lengths(case):
    """(cached lengths with the new rows in them, new rows), one entry per sequence."""
    rng = np.random.default_rng(case["len_seed"])
    if case["mid"]:
        x = np.clip(np.rint(rng.lognormal(math.log(case["mid"]), 0.8, case["batch"])), case["lo"], case["hi"])
    else:
        x = rng.integers(case["lo"], case["hi"], endpoint=True, size=case["batch"])
    new = rng.integers(case["new_lo"], case["new_hi"], endpoint=True, size=case["batch"])
    if case["op"] == "append" and case["new_hi"] == case["hi"]:
        new = x  # whole histories
    if case["causal"] or case["op"] == "append":
        x = np.maximum(x, new)
    return [int(v) for v in x], [int(v) for v in new]


def _offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device="cuda")


def _event_times(rng, n):
    # bursts of events separated by idle hours
    gaps = np.minimum(np.exp(rng.normal(math.log(60.0), 2.0, n)), 1e6).astype(np.int64)
    return rng.integers(0, 2 ** 28) + np.cumsum(gaps)


def _frequencies(case):
    """Angles per position, as hstu_rotary_frequencies gives them: base 10000, for "linear" all of them divided by 4, for
    "base" the base raised so that the lowest one is, for "by_parts" only those that turn less than once (fully) to 32 times
    (not at all) over 4096 positions."""
    dim = case["rotary"]
    j = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    base = 10000.0
    if case["scaling"] == "base":
        base *= 4.0 ** (dim / (dim - 2.0))
    freq = base ** (-2.0 * j / dim)
    if case["scaling"] == "linear":
        freq = freq / 4.0
    elif case["scaling"] == "by_parts":
        turns = 4096.0 * freq / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        freq = freq * keep + freq / 4.0 * (1.0 - keep)
    return freq


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1 + seed)
    total, new = _lengths(case)
    heads, kv_heads, d, ps = case["heads"], case["kv_heads"], case["d"], case["page"]
    dtype, std = (torch.bfloat16, 0.5) if case["dtype"] == "bf16" else (torch.float32, 1.0)

    def values(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)

    s = {"case": case, "total": total, "new": new, "max_kv": max(total), "alpha": 1.0 / math.sqrt(d)}
    if case["rotary"]:
        s["freq"] = _frequencies(case)
    if case["op"] == "rotary":
        rows = sum(total)
        s["off"] = _offsets(total)
        for name in ("q", "k", "dq", "dk"):
            s[name] = values(rows, heads, d)
        return s
    # pages of the cache in the order in which requests of many users happened to take them; rows that no
    # sequence has reached yet hold what their last owner left there
    rng = np.random.default_rng(seed)
    need = [-(-n // ps) for n in total]
    pages = sum(need) + 3
    order = rng.permutation(pages)
    table = np.full((len(total), max(need)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = torch.tensor(table, device="cuda")
    s["lens"] = torch.tensor(np.array(total, dtype=np.int32), device="cuda")
    s["off"] = _offsets(new)
    s["k_pages"], s["v_pages"] = values(pages, kv_heads, ps, d), values(pages, kv_heads, ps, d)
    rows = sum(new)
    s["q"] = values(rows, heads, d)
    s["ts_pages"] = None
    if case["buckets"]:
        # every history's event times, in its pages; the new rows' times for the call
        times = [_event_times(rng, n) for n in total]
        stamps = rng.integers(0, 2 ** 28, size=pages * ps).astype(np.int32)
        if case["op"] == "attn":
            for b, n in enumerate(total):
                p = np.arange(n)
                stamps[table[b, p // ps].astype(np.int64) * ps + p % ps] = times[b]
        s["ts_pages"] = torch.tensor(stamps.reshape(pages, ps), device="cuda")
        ends = [t[-1] + 60 * np.arange(1, m + 1) if not case["causal"] else t[len(t) - m:] for t, m in zip(times, new)]
        s["ts"] = torch.tensor(np.concatenate(ends).astype(np.int32), device="cuda")
    if case["op"] == "append":
        s["k"], s["v"] = values(rows, kv_heads, d), values(rows, kv_heads, d)
    elif case["buckets"]:
        s["weights"] = torch.randn(case["buckets"], generator=gen, device="cuda")
    if own:
        s["cache"] = _lib().HstuPagedCache(s["k_pages"], s["v_pages"], s["table"], s["lens"], ts_pages=s["ts_pages"])
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, hstu = s["case"], _lib()
    if case["op"] == "rotary":
        q, k = hstu.hstu_rotary_fwd([s["q"], s["k"]], s["freq"], seq_offsets=s["off"], interleaved=case["interleaved"])
        dq, dk = hstu.hstu_rotary_bwd([s["dq"], s["dk"]], s["freq"], seq_offsets=s["off"], interleaved=case["interleaved"])
        return q, k, dq, dk
    if case["op"] == "append":
        q = hstu.hstu_cache_append(s["cache"], s["k"], s["v"], s["off"], q=s["q"], inv_freq=s.get("freq"),
                                   interleaved=case["interleaved"], timestamps=s.get("ts"))
        return (q, s["k_pages"], s["v_pages"]) + ((s["ts_pages"],) if case["buckets"] else ())
    n, alpha = s["max_kv"], s["alpha"]
    if case["buckets"]:
        return hstu.hstu_paged_attn_bias_fwd(s["q"], s["cache"], s["off"], s["ts"], s["weights"], 2, n, alpha,
                                             case["causal"], max_kv=n)
    return hstu.hstu_paged_attn_fwd(s["q"], s["cache"], s["off"], n, alpha, case["causal"], max_kv=n)


# ---- the plain form ----------------------------------------------------------------------------------------------------

def _rows_of(off, rows):
    """Sequence and place in it of every row."""
    r = torch.arange(rows, device="cuda")
    seq = torch.bucketize(r, off[1:].long(), right=True)
    return seq, r - off.long()[seq]


def _turned(x, pos, freq, interleaved, sign=1.0):
    if freq is None:
        return x.clone()
    angle = pos.double()[:, None] * freq[None, :]
    c, sn = angle.cos().float()[:, None, :], (sign * angle.sin()).float()[:, None, :]
    half = freq.numel()
    y = x.float()
    if interleaved:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        part = torch.stack((a * c - b * sn, b * c + a * sn), dim=-1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        part = torch.cat((a * c - b * sn, b * c + a * sn), dim=-1)
    return torch.cat((part, y[..., 2 * half:]), dim=-1).to(x.dtype)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "rotary":
        _, pos = _rows_of(s["off"], s["q"].shape[0])
        i = case["interleaved"]
        return (_turned(s["q"], pos, s["freq"], i), _turned(s["k"], pos, s["freq"], i),
                _turned(s["dq"], pos, s["freq"], i, -1.0), _turned(s["dk"], pos, s["freq"], i, -1.0))
    ps, lens, off = case["page"], s["lens"].long(), s["off"].long()
    seq, i = _rows_of(s["off"], s["q"].shape[0])
    pos = lens[seq] - (off[seq + 1] - off[seq]) + i
    if case["op"] == "append":
        page, slot = s["table"].long()[seq, pos // ps], pos % ps
        s["k_pages"][page, :, slot] = _turned(s["k"], pos, s.get("freq"), case["interleaved"])
        s["v_pages"][page, :, slot] = s["v"]
        out = (_turned(s["q"], pos, s.get("freq"), case["interleaved"]), s["k_pages"], s["v_pages"])
        if case["buckets"]:
            s["ts_pages"][page, slot] = s["ts"]
            out += (s["ts_pages"],)
        return out
    # attention: the batch padded to its longest history and its most new rows
    batch, heads, kv_heads, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    n, m, group = max(s["total"]), max(s["new"]), heads // kv_heads
    table = s["table"].long().clamp(min=0)

    def gathered(pages):  # [batch, kv_heads, n, d]
        x = pages[table].permute(0, 2, 1, 3, 4).reshape(batch, kv_heads, -1, d)[:, :, :n]
        return x.float()

    k, v = gathered(s["k_pages"]), gathered(s["v_pages"])
    q = torch.zeros((batch, m, heads, d), device="cuda")
    q[seq, i] = s["q"].float()
    q = q.view(batch, m, kv_heads, group, d).permute(0, 2, 3, 1, 4).reshape(batch, kv_heads, group * m, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(batch, kv_heads, group, m, n)
    key = torch.arange(n, device="cuda")
    if case["buckets"]:
        tq = torch.zeros((batch, m), dtype=torch.int64, device="cuda")
        tq[seq, i] = s["ts"].long()
        tk = s["ts_pages"][table].reshape(batch, -1)[:, :n].long()
        delta = (tq[:, :, None] - tk[:, None, :]).abs()
        e = torch.frexp(delta.double())[1].long() - 1
        e = e.clamp(min=0)
        bucket = (e * 4 + ((delta << 2) >> e) - 4).clamp(max=case["buckets"] - 1)
        bucket = torch.where(delta <= 1, torch.zeros_like(bucket), bucket)
        x = x + s["weights"][bucket][:, None, None]
    x = x * (1.0 / math.sqrt(d))
    p = x / (1.0 + torch.exp(-x))
    if case["causal"]:
        place = lens[:, None] - (off[1:] - off[:-1])[:, None] + torch.arange(m, device="cuda")
        seen = key <= place[:, :, None]
    else:
        seen = (key < lens[:, None, None]).expand(batch, m, n)
    p = torch.where(seen[:, None, None], p, torch.zeros((), device="cuda")) / n
    o = torch.matmul(p.reshape(batch, kv_heads, group * m, n), v)
    o = o.view(batch, heads, m, d).permute(0, 2, 1, 3)
    return o[seq, i].to(s["q"].dtype)


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _exact_rotation(x, positions, freq, interleaved, backward=False):
    x = x.double()
    if freq is None:
        return x
    half = freq.numel()
    first = torch.arange(half, device="cuda") * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    # each pair as a complex number, multiplied by exp(+-i angle)
    z = torch.complex(x[:, :, first], x[:, :, second])
    angle = torch.outer(positions.double(), freq)
    z = z * torch.polar(torch.ones_like(angle), -angle if backward else angle)[:, None]
    out = x.clone()
    out[:, :, first], out[:, :, second] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    freq, inter = s.get("freq"), case["interleaved"]
    if case["op"] == "rotary":
        pos = torch.cat([torch.arange(n, device="cuda") for n in s["total"]])
        return (_exact_rotation(s["q"], pos, freq, inter), _exact_rotation(s["k"], pos, freq, inter),
                _exact_rotation(s["dq"], pos, freq, inter, True), _exact_rotation(s["dk"], pos, freq, inter, True))
    ps, table = case["page"], s["table"].cpu().numpy().astype(np.int64)
    if case["op"] == "append":
        spans = [np.arange(n - m, n) for n, m in zip(s["total"], s["new"])]
        pos = torch.tensor(np.concatenate(spans), device="cuda")
        place = np.concatenate([table[b, p // ps] * ps + p % ps for b, p in enumerate(spans)])
        place = torch.tensor(place, device="cuda")
        out = [_exact_rotation(s["q"], pos, freq, inter)]
        for pages, rows in ((s["k_pages"], _exact_rotation(s["k"], pos, freq, inter)), (s["v_pages"], s["v"].double())):
            flat = pages.double().permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["d"])  # a row per slot
            flat[place] = rows
            out.append(flat.view(-1, ps, case["kv_heads"], case["d"]).permute(0, 2, 1, 3))
        if case["buckets"]:
            stamps = s["ts_pages"].clone().view(-1)
            stamps[place] = s["ts"]
            out.append(stamps.view(-1, ps))
        return tuple(out)
    # attention, one sequence and one head at a time
    most, alpha, group = max(s["total"]), case["d"] ** -0.5, case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, m) in enumerate(zip(s["total"], s["new"])):
        page = torch.tensor(table[b, :-(-n // ps)], device="cuda")
        rows = torch.arange(m, device="cuda")[:, None]
        keys = torch.arange(n, device="cuda")[None, :]
        hidden = keys > rows + (n - m) if case["causal"] else None
        bias = 0.0
        if case["buckets"]:
            gap = (s["ts"][first:first + m].double()[:, None] - s["ts_pages"][page].reshape(-1)[:n].double()[None]).abs()
            octave = torch.floor(torch.log2(gap.clamp(min=1.0)))
            group_of = octave * 4 + torch.floor((gap / 2.0 ** octave - 1.0) * 4)
            index = torch.where(gap <= 1, torch.zeros_like(gap), group_of).long().clamp(max=case["buckets"] - 1)
            bias = s["weights"].double()[index]
        for h in range(case["heads"]):
            k = s["k_pages"][page, h // group].reshape(-1, case["d"])[:n].double()
            v = s["v_pages"][page, h // group].reshape(-1, case["d"])[:n].double()
            x = alpha * (s["q"][first:first + m, h].double() @ k.T + bias)
            weight = x * torch.sigmoid(x)
            if hidden is not None:
                weight = weight.masked_fill(hidden, 0.0)
            out[first:first + m, h] = weight @ v / most
        first += m
    return out


def work(case):
    """Every input row read once (a cached row once for all rows that see it), every output row written once; the products'
    flops of the visible pairs; 3 flops per element for a rotation."""
    total, new = _lengths(case)
    size = 2 if case["dtype"] == "bf16" else 4
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "rotary":
        rows = sum(total)
        return {"bytes": 8 * rows * heads * d * size + 4 * (len(total) + 1), "flops": 4 * 3 * rows * heads * case["rotary"]}
    rows = sum(new)
    small = 4 * (2 * len(total) + 1) + 4 * sum(-(-n // case["page"]) for n in total)
    if case["op"] == "append":
        stamps = 8 * rows if case["buckets"] else 0
        return {"bytes": 2 * rows * (heads + 2 * kv_heads) * d * size + stamps + small,
                "flops": 3 * rows * (heads + kv_heads) * case["rotary"]}
    pairs = sum(sum(range(n - m + 1, n + 1)) if case["causal"] else n * m for n, m in zip(total, new))
    stamps = 4 * (sum(total) + rows + case["buckets"]) if case["buckets"] else 0
    return {"bytes": 2 * sum(total) * kv_heads * d * size + 2 * rows * heads * d * size + stamps + small,
            "flops": 4 * d * heads * pairs}
