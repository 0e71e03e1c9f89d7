"""The 4-bit sequence cache and the 4-bit products of this library as cases that can be timed and compared.

A case is one pass through one operator, as a serving program calls it through paper_2511_12934_b200.binding:
  linear     microscaled 4-bit quantisation of activations, then their product with weights quantised once
  attention  target attention of query rows over behaviour sequences held in 4-bit pages
  snapshot   sequences forked, rows appended to the forks (copy on write), and the forks read back
  ingest     whole sequences appended to emptied ones and read back
  compact    the live pages of a fragmented cache brought into another one, and its sequences read
Beside each call stands its plain form in elementary torch operations, in 32 bits, and its definition in 64 bits.

4-bit values: blocks of 32 along the last dimension share a scale 2^(byte - 127); a code is sign, two exponent bits and one
mantissa bit, two codes to a byte, the first in the low half.
"""
import math
import random

import torch

own = False

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SIGMA = 0.05    # of item vectors and projected sequences, as in the benchmark's workloads


# ---- cases ------------------------------------------------------------------------------------------------------

def _linear(name, m, k, n, dtype="bf16", relu=True):
    return dict(name=name, op="linear", m=m, k=k, n=n, dtype=dtype, relu=relu)


def _attention(name, seqs, rows, longest, d, heads=1, kv_heads=1, shared=True, dtype="bf16", page_rows=64, ragged=False, window=0, sinks=0, layout=1):
    return dict(name=name, op="attention", seqs=seqs, rows=rows, longest=longest, d=d, heads=heads, kv_heads=kv_heads, shared=shared,
                dtype=dtype, page_rows=page_rows, ragged=ragged, window=window, sinks=sinks, layout=layout)


def _pages(name, op, seqs, longest, added, d, kv_heads=1, shared=True, dtype="bf16", page_rows=64, layout=1):
    return dict(name=name, op=op, seqs=seqs, longest=longest, added=added, d=d, kv_heads=kv_heads, shared=shared, dtype=dtype,
                page_rows=page_rows, layout=layout)


def listed():
    return [
        # the first layer of the scoring MLP (wide model: 2816 input columns) for a handful of candidates
        _linear("mlp_few_rows", 7, 2816, 1024),
        # the same layer for one request of 10^4 candidates
        _linear("mlp_request", 10_000, 2816, 1024),
        # first layer of the item tower over a full refresh of 2^19 items (512 raw features, hidden width 256)
        _linear("item_tower", 524_288, 512, 256),
        # an fp32 model's hidden layer, no activation, ragged rows and columns
        _linear("fp32_layer", 4_001, 1024, 520, dtype="f32", relu=False),
        # one item against one user's sequence: the smallest call
        _attention("one_row", 1, 1, 200, 128),
        # the profile rows of 256 concurrent users, sequences of every length up to 10^4
        _attention("profiles_256_users", 256, 1, 10_000, 128, ragged=True),
        # 16 requests of 10^4 candidates against sequences of 10^4 items (the largest)
        _attention("candidates_long", 16, 10_000, 10_000, 128),
        # grouped heads with values of their own, the recent items and the first four visible, a few rows a sequence
        _attention("window_and_sinks", 96, 5, 6_000, 64, heads=8, kv_heads=2, shared=False, ragged=True, window=1024, sinks=4, page_rows=32),
        # the fp32 model: one request of 1000 candidates, 50 items
        _attention("fp32_request", 1, 1000, 50, 64, dtype="f32", page_rows=16),
        # snapshots of 48 users with a few new items each
        _pages("snapshot_48_users", "snapshot", 48, 2_000, 9, 128),
        # the sequences of 64 users taken in
        _pages("ingest_64_users", "ingest", 64, 0, 6_000, 128),
        # a cache of 200 users of which pages are shared and scattered, moved into a smaller one
        _pages("compact_200_users", "compact", 200, 10_000, 0, 128),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "attention", "attention", "attention", "attention", "snapshot", "ingest", "compact"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "linear":
        m, k = _log(rng, 1, 300_000), 32 * _log(rng, 1, 88)
        n = _log(rng, 8, 1024)
        while m * k * n > 524_288 * 512 * 256:
            m = m // 2
        c = _linear("", m, k, n, dtype=dtype, relu=rng.random() < 0.5)
    elif op == "attention":
        d = rng.choice([32, 64, 64, 96, 128, 128, 128, 256])
        heads, kv_heads = rng.choice([(1, 1), (1, 1), (4, 4), (4, 1), (8, 2)])
        seqs, rows, longest = _log(rng, 1, 256), _log(rng, 1, 10_000), _log(rng, 1, 20_000)
        most = 16e8 * 128 if dtype == "bf16" and d in (64, 128, 256) else 4e9   # products of the pass
        while seqs * rows * heads * longest * d > most:
            if rows > 8 and (rows >= seqs or seqs == 1):
                rows = rows // 2
            elif seqs > 1:
                seqs = seqs // 2
            else:
                longest = longest // 2
        windowed = rng.random() < 0.4
        c = _attention("", seqs, rows, longest, d, heads, kv_heads, shared=rng.random() < 0.5, dtype=dtype, page_rows=rng.choice([16, 32, 64, 128]),
                       ragged=rng.random() < 0.7, window=_log(rng, 1, 4096) if windowed else 0, sinks=rng.choice([0, 1, 4, 33]) if windowed else 0,
                       layout=rng.randrange(1 << 30))
    else:
        seqs = _log(rng, 1, 128)
        longest = {"snapshot": _log(rng, 1, 6000), "ingest": 0, "compact": _log(rng, 64, 8000)}[op]
        added = {"snapshot": _log(rng, 1, 200), "ingest": _log(rng, 1, 4000), "compact": 0}[op]
        c = _pages("", op, seqs, longest, added, rng.choice([32, 64, 128, 128, 256]), kv_heads=rng.choice([1, 1, 2]), shared=rng.random() < 0.6,
                   dtype=dtype, page_rows=rng.choice([16, 32, 64, 128]), layout=rng.randrange(1 << 30))
    del c["name"]
    return c


def _lengths(c):
    """Items of every sequence; the longest is always among them, one in sixteen is empty where they differ."""
    n, top = c["seqs"], c["longest"]
    if c["op"] == "attention" and not c["ragged"]:
        return [top] * n
    r = random.Random(c["layout"])
    got = [0 if n > 4 and r.randrange(16) == 0 else r.randint(min(1, top), top) for _ in range(n)]
    got[r.randrange(n)] = top
    return got


def _counts(c):
    """Rows of every sequence that a call brings: queries, or appended rows."""
    n, top = c["seqs"], c["rows"] if c["op"] == "attention" else c["added"]
    if c["op"] == "attention" and not c["ragged"]:
        return [top] * n
    r = random.Random(c["layout"] + 1)
    got = [r.randint(0 if n > 4 else 1, top) if top > 1 else top for _ in range(n)]
    got[r.randrange(n)] = top
    return got


def _visible(c, length):
    if not c["window"] or length <= c["window"]:
        return length
    return c["window"] + min(c["sinks"], length - c["window"])


def _row_bytes(c):
    return (c["d"] // 2 + c["d"] // 32) * c["kv_heads"] * (1 if c["shared"] else 2)


def work(c):
    el = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        return {"bytes": m * k * el + n * k * 17 // 32 + 4 * n + m * n * el, "flops": 2 * m * n * k}
    L = _lengths(c)
    if c["op"] == "attention":
        q = _counts(c)
        seen = [_visible(c, x) if y else 0 for x, y in zip(L, q)]
        return {"bytes": 2 * sum(q) * c["heads"] * c["d"] * el + sum(seen) * _row_bytes(c),
                "flops": 4 * c["d"] * c["heads"] * sum(x * y for x, y in zip(seen, q))}
    a = _counts(c) if c["added"] else [0] * c["seqs"]
    wide = c["d"] * c["kv_heads"] * (1 if c["shared"] else 2) * el
    total = sum(L) + sum(a)
    if c["op"] == "compact":
        live = sum(-(-x // c["page_rows"]) for x in L[: (c["seqs"] + 1) // 2]) * c["page_rows"]
        return {"bytes": 2 * live * _row_bytes(c) + total * (_row_bytes(c) + wide), "flops": 0}
    # rows in, their 4-bit form written, every row of the sequences read and written
    return {"bytes": sum(a) * (wide + _row_bytes(c)) + total * (_row_bytes(c) + wide), "flops": 0}


# ---- plain forms ------------------------------------------------------------------------------------------------

def _quantise(x):
    """[..., w] -> codes [..., w / 2] and scale bytes [..., w / 32]."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    field = (top.view(torch.int32) >> 23) & 255
    byte = torch.where(field == 255, field, (field - 2).clamp(min=0))
    y = (b * torch.exp2(127.0 - byte.clamp(max=252).float())).abs()
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8)
    code = (code + 8 * torch.signbit(b).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], byte.squeeze(-1).to(torch.uint8)


def _values(codes, scales):
    """The fp32 values that codes [..., w / 2] with scale bytes [..., w / 32] stand for."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).int()].flatten(-2).unflatten(-1, (-1, 32))
    return (v * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _store(x, dtype):
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _plain_linear(s):
    c = s["case"]
    y = torch.matmul(_values(*_quantise(s["x"])), _values(s["w_codes"], s["w_scales"]).T) + s["bias"]
    return _store(y.clamp(min=0) if c["relu"] else y, c["dtype"])


def _rows_of(pool, which, table, seq, pos):
    """fp32 rows [..., heads, d] of the sequences `seq` at the positions `pos`."""
    r = pool["k_codes"].shape[2]
    page = table[seq, pos // r].long()
    return _values(pool[which + "_codes"][page, :, pos % r], pool[which + "_scales"][page, :, pos % r])


def _plain_attention(s):
    c, pool = s["case"], s["pool"]
    H, K, d, n = c["heads"], c["kv_heads"], c["d"], c["seqs"]
    longest, most = c["longest"], s["most_rows"]
    dev = s["q"].device
    at = torch.arange(max(longest, 1), device=dev)
    length = pool["lengths"].unsqueeze(1)
    seen = at < length
    if c["window"]:
        seen = seen & ((at >= length - c["window"]) | (at < c["sinks"]))
    seq = torch.arange(n, device=dev).unsqueeze(1)
    pos = torch.where(at < length, at, torch.zeros_like(at))
    table = pool["table"].clamp(min=0)
    keys = _rows_of(pool, "k", table, seq, pos).permute(0, 2, 1, 3)                       # [n, K, L, d]
    vals = keys if c["shared"] else _rows_of(pool, "v", table, seq, pos).permute(0, 2, 1, 3)
    vals = vals * seen[:, None, :, None]
    slot = s["row_seq"] * most + s["row_pos"]
    q = torch.zeros(n * most, H, d, device=dev)
    q[slot] = s["q"].float()
    q = q.view(n, most, K, H // K, d).permute(0, 2, 1, 3, 4).reshape(n, K, most * (H // K), d)
    w = torch.matmul(q, keys.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    w.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w, vals) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.view(n, K, most, H // K, d).permute(0, 2, 1, 3, 4).reshape(n * most, H, d)
    return _store(o[slot], c["dtype"])


def _plain_fork(p, src, dst):
    """Sequences dst (empty before) on the pages of src."""
    table, lengths = p["table"].clone(), p["lengths"].clone()
    table[dst], lengths[dst] = table[src], lengths[src]
    used = table[dst]
    n_pages = p["refs"].numel()
    refs = torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device)
    refs.index_add_(0, torch.where(used >= 0, used, torch.full_like(used, n_pages)).flatten().long(), torch.ones_like(used).flatten())
    return {**p, "table": table, "lengths": lengths, "refs": p["refs"] + refs[:n_pages]}


def _plain_append(p, ids, counts, row_seq, row_pos, rows):
    """Rows appended to the sequences `ids`: pages from the end of the free list, a shared last page copied first."""
    R, W = p["k_codes"].shape[2], p["table"].shape[1]
    n_pages = p["refs"].numel()
    L = p["lengths"][ids]
    have, want = (L + R - 1) // R, (L + counts + R - 1) // R
    old = p["table"][ids]
    last = (L // R).clamp(max=W - 1).unsqueeze(1).long()
    tail = old.gather(1, last).squeeze(1)
    shared = (counts > 0) & (L % R > 0) & (p["refs"][tail.clamp(min=0).long()] > 1)
    need = want - have + shared.int()
    before = torch.cumsum(need, 0) - need
    at = torch.arange(W, device=ids.device).unsqueeze(0)
    fresh = (at >= have.unsqueeze(1)) & (at < want.unsqueeze(1))
    swap = shared.unsqueeze(1) & (at == last)
    pick = before.unsqueeze(1) + torch.where(swap, torch.zeros_like(at), at - have.unsqueeze(1) + shared.int().unsqueeze(1))
    page = p["free_pages"][(p["n_free"] - 1 - pick).clamp(min=0).long()]
    now = torch.where(fresh | swap, page, old)
    count = torch.zeros(n_pages + 1, dtype=torch.int32, device=ids.device)
    count.index_add_(0, torch.where(fresh | swap, page, torch.full_like(page, n_pages)).flatten().long(), torch.ones_like(page).flatten())
    count.index_add_(0, torch.where(shared, tail, torch.full_like(tail, n_pages)).long(), torch.full_like(tail, -1))
    table, lengths = p["table"].clone(), p["lengths"].clone()
    table[ids], lengths[ids] = now, L + counts
    out = {**p, "table": table, "lengths": lengths, "refs": p["refs"] + count[:n_pages], "n_free": p["n_free"] - need.sum(dtype=torch.int32)}
    spare = p["free_pages"][0]   # never handed out here: a copy onto itself where there is nothing to copy
    frm, to = torch.where(shared, tail, spare).long(), torch.where(shared, now.gather(1, last).squeeze(1), spare).long()
    at_row = L[row_seq] + row_pos
    where = now[row_seq, (at_row // R).long()].long()
    for name, x in rows.items():
        p[name + "_codes"][to], p[name + "_scales"][to] = p[name + "_codes"][frm], p[name + "_scales"][frm]
        p[name + "_codes"][where, :, (at_row % R).long()], p[name + "_scales"][where, :, (at_row % R).long()] = _quantise(x)
    return out


def _plain_read(p, row_seq, row_pos, dtype):
    got = [_store(_rows_of(p, "k", p["table"], row_seq, row_pos), dtype)]
    if "v_codes" in p:
        got.append(_store(_rows_of(p, "v", p["table"], row_seq, row_pos), dtype))
    return got


def _plain_compact(p, small):
    """The live pages of p, in their order, in the pages 0, 1, ... of a cache of small["n_pages"] pages."""
    live = p["refs"] > 0
    place = (torch.cumsum(live, 0, dtype=torch.int32) - 1).clamp(min=0)
    n = small["n_pages"]
    to = torch.where(live, place, torch.full_like(place, n)).long()
    refs = torch.zeros(n + 1, dtype=torch.int32, device=live.device)
    refs[to] = p["refs"]
    out = {"table": torch.where(p["table"] >= 0, place[p["table"].clamp(min=0).long()], torch.full_like(p["table"], -1)), "lengths": p["lengths"].clone(),
           "refs": refs[:n], "n_free": (n - live.sum(dtype=torch.int32)).view(1),
           "free_pages": torch.arange(n - 1, -1, -1, dtype=torch.int32, device=live.device)}
    for name in small["data"]:
        data = torch.zeros(n + 1, *p[name].shape[1:], dtype=torch.uint8, device=live.device)
        data[to] = p[name]
        out[name] = data[:n]
    return out


BOOKS = ("table", "lengths", "refs", "free_pages", "n_free")


def _plain_pages(s):
    c, p = s["case"], s["pool"]
    if c["op"] == "snapshot":
        p = _plain_fork(p, s["src"], s["dst"])
    if c["op"] == "compact":
        p = _plain_compact(p, s["small"])
    else:
        p = _plain_append(p, s["dst"], s["counts"], s["row_seq"], s["row_pos"], s["rows"])
    return _plain_read(p, s["dst"][s["read_seq"]], s["read_pos"], c["dtype"]) + [p[name] for name in BOOKS]


# ---- the library's calls ----------------------------------------------------------------------------------------

def _own(s):
    from paper_2511_12934_b200 import binding as B

    c = s["case"]
    if c["op"] == "linear":
        return B.mx4_linear(s["x"], s["w"], s["out"], bias=s["bias"], relu=c["relu"])
    cache = s["cache"]
    if c["op"] == "attention":
        cache.attention(s["q"], s["out"], offsets=s["offsets"], window=c["window"], sinks=c["sinks"])
        return s["out"]
    if c["op"] == "snapshot":
        cache.fork(s["src_ids"], s["dst_ids"])
    elif c["op"] == "ingest":
        cache.free(s["dst_ids"])
    else:
        cache.compact(s["into"])
        cache = s["into"]
    if c["added"]:
        cache.append(s["dst_ids"], s["offsets"], s["rows"]["k"], s["rows"].get("v"))
    cache.read(s["dst_ids"], s["read_offsets"], *s["read"])
    return s["read"] + [getattr(cache, name) for name in BOOKS]


# ---- inputs -----------------------------------------------------------------------------------------------------

def _offsets(counts, dev):
    t = torch.zeros(len(counts) + 1, dtype=torch.int64)
    t[1:] = torch.tensor(counts).cumsum(0)
    return t.to(dev)


def _places(counts, dev):
    """For every row of a ragged batch its sequence and its place in it."""
    t = torch.tensor(counts)
    seq = torch.repeat_interleave(torch.arange(len(counts)), t)
    pos = torch.arange(int(t.sum())) - (t.cumsum(0) - t)[seq]
    return seq.to(dev), pos.to(dev)


def _random_pages(g, n_pages, heads, page_rows, d, dev):
    """Pages of quantised rows of projected sequences."""
    rows = torch.randn(n_pages, heads, page_rows, d, generator=g, device=dev) * SIGMA
    return _quantise(rows)


def _pool(c, g, gh, dev, n_seqs, n_pages, width):
    """A cache of n_seqs sequences over scattered pages, the lengths of `c` in the first of them."""
    L, R = _lengths(c), c["page_rows"]
    order = torch.randperm(n_pages, generator=gh).int()
    table, used = torch.full((n_seqs, width), -1, dtype=torch.int32), 0
    lengths = torch.zeros(n_seqs, dtype=torch.int32)
    own_pages = L if c["op"] != "compact" else [x if i < (len(L) + 1) // 2 else 0 for i, x in enumerate(L)]
    for i, x in enumerate(own_pages):
        n = -(-x // R)
        table[i, :n], lengths[i], used = order[used:used + n], x, used + n
    if c["op"] == "compact":   # the second half of the sequences share the pages of the first
        for i in range((len(L) + 1) // 2, len(L)):
            table[i], lengths[i] = table[i - (len(L) + 1) // 2], lengths[i - (len(L) + 1) // 2]
    refs = torch.zeros(n_pages, dtype=torch.int32)
    named = table[table >= 0].long()
    refs.index_add_(0, named, torch.ones(named.numel(), dtype=torch.int32))
    free = torch.zeros(n_pages, dtype=torch.int32)
    free[: n_pages - used] = order[used:]
    p = {"table": table, "lengths": lengths, "refs": refs, "free_pages": free, "n_free": torch.tensor([n_pages - used], dtype=torch.int32)}
    p = {name: t.to(dev) for name, t in p.items()}
    p["k_codes"], p["k_scales"] = _random_pages(g, n_pages, c["kv_heads"], R, c["d"], dev)
    if not c["shared"]:
        p["v_codes"], p["v_scales"] = _random_pages(g, n_pages, c["kv_heads"], R, c["d"], dev)
    return p


def _cache(c, pool, n_seqs, n_pages, width):
    """The library's cache with the pages and the books of `pool`."""
    from paper_2511_12934_b200 import binding as B

    cache = B.Cache4(d=c["d"], n_pages=n_pages, page_rows=c["page_rows"], n_seqs=n_seqs, max_pages=width, heads=c["kv_heads"], shared=c["shared"])
    for name, t in pool.items():
        getattr(cache, name).copy_(t)
    return cache


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g, gh = torch.Generator(device=dev).manual_seed(seed), torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    s = {"case": c}
    if c["op"] == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        s["x"] = (torch.randn(m, k, generator=g, device=dev) * SIGMA).to(dt)
        w = torch.randn(n, k, generator=g, device=dev) * math.sqrt(2.0 / (k + n))
        s["w_codes"], s["w_scales"] = _quantise(w)
        s["bias"] = torch.randn(n, generator=g, device=dev) * 0.01
        if own:
            from paper_2511_12934_b200 import binding as B
            s["w"] = B.mx4_quantize(w)
        s["out"] = torch.empty(m, n, dtype=dt, device=dev)
        return s
    L, R, n = _lengths(c), c["page_rows"], c["seqs"]
    kv = (c["kv_heads"], c["d"])
    if c["op"] == "attention":
        q = _counts(c)
        n_pages, width = sum(-(-x // R) for x in L) + 5, max(1, -(-max(L) // R))
        s["pool"] = _pool(c, g, gh, dev, n, n_pages, width)
        s["offsets"], s["most_rows"] = _offsets(q, dev), max(q)
        s["row_seq"], s["row_pos"] = _places(q, dev)
        # queries like item vectors, spread so that the weights are neither all alike nor a single one
        s["q"] = (torch.randn(sum(q), c["heads"], c["d"], generator=g, device=dev) / SIGMA).to(dt)
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["cache"] = _cache(c, s["pool"], n, n_pages, width)
        return s
    a = _counts(c) if c["added"] else [0] * n
    n_seqs = 2 * n if c["op"] == "snapshot" else n
    width = max(1, -(-(max(L) + max(a)) // R))
    fresh = sum(-(-(x + y) // R) - -(-x // R) + 1 for x, y in zip(L, a))
    n_pages = sum(-(-x // R) for x in L) + fresh + 3
    s["pool"] = _pool(c, g, gh, dev, n_seqs, n_pages, width)
    first = n if c["op"] == "snapshot" else 0
    s["src"], s["dst"] = torch.arange(n, device=dev), torch.arange(first, first + n, device=dev)
    s["src_ids"], s["dst_ids"] = s["src"].int(), s["dst"].int()
    s["counts"] = torch.tensor(a, dtype=torch.int32, device=dev)
    s["offsets"] = _offsets(a, dev)
    s["row_seq"], s["row_pos"] = _places(a, dev)
    s["rows"] = {name: (torch.randn(sum(a), *kv, generator=g, device=dev) * SIGMA).to(dt) for name in ("k", "v")[: 1 if c["shared"] else 2]}
    half = (n + 1) // 2
    now = [x + y for x, y in zip(L, a)] if c["op"] != "compact" else [L[i % half] for i in range(n)]
    s["read_offsets"] = _offsets(now, dev)
    s["read_seq"], s["read_pos"] = _places(now, dev)
    s["read"] = [torch.empty(sum(now), *kv, dtype=dt, device=dev) for _ in s["rows"]]
    live = sum(-(-x // R) for x in L[:half])
    s["small"] = {"n_pages": live + 7, "data": [name for name in s["pool"] if name.endswith(("codes", "scales"))]}
    if own:
        s["cache"] = _cache(c, s["pool"], n_seqs, n_pages, width)
        if c["op"] == "compact":
            from paper_2511_12934_b200 import binding as B
            s["into"] = B.Cache4(d=c["d"], n_pages=live + 7, page_rows=R, n_seqs=n_seqs, max_pages=width, heads=c["kv_heads"], shared=c["shared"])
    return s


def run(s):
    if own:
        return _own(s)
    return {"linear": _plain_linear, "attention": _plain_attention}.get(s["case"]["op"], _plain_pages)(s)


# ---- definition in 64 bits --------------------------------------------------------------------------------------

def _exact_values(x):
    """What x stands for after quantisation to 4 bits, from the definition: nearest representable multiples of each block's scale."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    exponent = torch.where(top > 0, torch.frexp(top).exponent - 1 - 2, torch.full_like(top, -127).int()).clamp(min=-127)
    scale = torch.ldexp(torch.ones_like(top), exponent)
    y = (b / scale).abs()
    step = torch.where(y >= 4, 2.0, torch.where(y >= 2, 1.0, 0.5)).double()
    y = (torch.round(y / step) * step).clamp(max=6.0)
    return (torch.copysign(y, b) * scale).reshape(x.shape)


def _exact_stored(codes, scales):
    v = torch.tensor(VALUES, dtype=torch.float64, device=codes.device)
    halves = [torch.where(h >= 8, -v[(h % 8).long()], v[(h % 8).long()]) for h in (codes % 16, codes // 16)]
    x = torch.stack(halves, -1).reshape(*scales.shape, 32)
    return torch.ldexp(x, scales.int().unsqueeze(-1) - 127).reshape(*codes.shape[:-1], -1)


def _exact_sequence(pool, which, seq, length):
    R = pool["k_codes"].shape[2]
    pages = pool["table"][seq][: -(-length // R)].long()
    x = _exact_stored(pool[which + "_codes"][pages], pool[which + "_scales"][pages])     # [pages, heads, R, d]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :length]              # [heads, length, d]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "linear":
        w = _exact_stored(s["w_codes"], s["w_scales"]).T
        y = torch.cat([_exact_values(x) @ w for x in s["x"].split(65536)]) + s["bias"].double()
        return torch.where(y < 0, 0.0, y) if c["relu"] else y
    if c["op"] == "attention":
        H, K, d = c["heads"], c["kv_heads"], c["d"]
        out, at = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device), s["offsets"].tolist()
        for i, length in enumerate(_lengths(c)):
            if length == 0 or at[i] == at[i + 1]:
                continue
            k = _exact_sequence(s["pool"], "k", i, length)
            v = k if c["shared"] else _exact_sequence(s["pool"], "v", i, length)
            if c["window"] and length > c["window"]:
                keep = list(range(min(c["sinks"], length - c["window"]))) + list(range(length - c["window"], length))
                k, v = k[:, keep], v[:, keep]
            for h in range(H):
                j = h // (H // K)
                for r in range(at[i], at[i + 1], 4096):
                    z = s["q"][r:min(r + 4096, at[i + 1]), h].double() @ k[j].T / math.sqrt(d)
                    z = torch.exp(z - z.max(1, keepdim=True).values)
                    out[r:r + z.shape[0], h] = z @ v[j] / z.sum(1, keepdim=True)
        return out
    first, L, a, got = s["pool"], _lengths(c), s["counts"].tolist(), []
    half, off = (c["seqs"] + 1) // 2, s["offsets"].tolist()
    for which in s["rows"]:
        parts = []
        for i in range(c["seqs"]):
            j = i % half if c["op"] == "compact" else i
            if L[j]:
                parts.append(_exact_sequence(first, which, j, L[j]).transpose(0, 1))
            if a[i]:
                parts.append(_exact_values(s["rows"][which][off[i]:off[i + 1]]))
        got.append(torch.cat(parts))
    return got + [None] * len(BOOKS)
