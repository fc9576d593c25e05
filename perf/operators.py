"""The work of the windowed attention, of the paged key-value cache and of the
attention that reads it: what serving and training a sequence recommender on
long histories asks of them.  Four kinds of case:

* "window": jagged HSTU attention in which a token sees its `window` most recent
  tokens and the `sinks` first ones of its sequence, forward alone (prompts) or
  forward and backward (training);
* "decode": the same attention for one new token of every sequence, its keys,
  values and timestamps in the pages of a cache;
* "beams": a beam step on the cache's pages: old beams freed, the prompts forked,
  room for one more token (copies of shared last pages), two layers' rows written;
* "fill": prompts enter the cache, tables and rows;
* "compact": the pages that are in use move to the front of their pools.

A case names its batch by numbers alone.  `lens` seeds the sequence lengths and
the pages' places, which belong to the case; the values of the tensors follow
the seed that `prepare` is given.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
LN_EPS = 1e-6
TS_GAP_MEAN = 600.0
RAB_STD = 0.1


# ------------------------------------------------------------------- cases
def _window(name, dtype, B, dist, lo, hi, H, d, window, sinks, pos, time, bwd, p=0.0, nb=128,
            lens=1):
    return dict(name=name, kind="window", dtype=dtype, B=B, dist=dist, p=p, lo=lo, hi=hi, H=H,
                d=d, window=window, sinks=sinks, pos=pos, time=time, nb=nb, bwd=bwd, lens=lens)


def _decode(name, dtype, B, dist, lo, hi, H, d, page, pos, time, window=0, sinks=0, p=0.0,
            nb=128, lens=1):
    return dict(name=name, kind="decode", dtype=dtype, B=B, dist=dist, p=p, lo=lo, hi=hi, H=H,
                d=d, page=page, window=window, sinks=sinks, pos=pos, time=time, nb=nb, lens=lens)


def _cache(name, kind, dtype, B, dist, lo, hi, H, d, page, beams=1, p=0.0, lens=1):
    return dict(name=name, kind=kind, dtype=dtype, B=B, dist=dist, p=p, lo=lo, hi=hi, H=H, d=d,
                page=page, beams=beams, lens=lens)


def listed():
    return [
        # a handful of short histories scored at once: latency
        _window("window_small_serve", "bf16", 8, "uniform", 1, 250, 4, 64, 64, 4, True, True, False),
        # a training step on many short histories
        _window("window_train_powerlaw", "bf16", 128, "powerlaw", 16, 512, 4, 64, 128, 8, True,
                True, True, p=1.2),
        # a training step at the layer's geometry, long histories
        _window("window_train_layer", "bf16", 32, "powerlaw", 64, 4096, 4, 128, 512, 32, True, True,
                True, p=1.1),
        # prompts of up to 8192 tokens, position bias alone
        _window("window_prompts_zipf", "bf16", 128, "powerlaw", 1, 8192, 4, 64, 1024, 64, True, False,
                False, p=1.05),
        # fp32 training with odd sizes: a window that is no multiple of a tile
        _window("window_train_f32", "f32", 24, "uniform", 5, 300, 2, 32, 50, 3, True, True, True,
                nb=32),
        # four users' next token: latency
        _decode("decode_small", "bf16", 4, "uniform", 1, 300, 4, 64, 16, True, True),
        # a serving batch at the layer's geometry
        _decode("decode_batch", "bf16", 128, "powerlaw", 64, 4096, 4, 128, 64, True, True, p=1.1),
        # lifelong histories, wide heads: bandwidth
        _decode("decode_long", "bf16", 32, "uniform", 20000, 65536, 8, 128, 128, True, True),
        # fp32, most of the cache out of sight
        _decode("decode_window_f32", "f32", 64, "powerlaw", 100, 8192, 4, 64, 32, True, False, 1000, 7,
                p=1.05),
        # eight prompts of four beams each
        _cache("cache_beams", "beams", "bf16", 8, "uniform", 30, 2000, 4, 64, 16, beams=4),
        # a batch of prompts enters
        _cache("cache_fill", "fill", "bf16", 64, "powerlaw", 16, 4096, 4, 128, 64, p=1.1),
        # half the sequences have left, the rest move together
        _cache("cache_compact", "compact", "bf16", 96, "uniform", 100, 1000, 8, 128, 16),
    ]


def _odd(rng, lo, hi):
    """A whole number spread over the logarithm of the range."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["window", "window", "decode", "decode", "beams", "fill", "compact"])
    lens = rng.randrange(1 << 16)
    f32 = rng.random() < 0.25
    dtype = "f32" if f32 else "bf16"
    d = rng.choice([32, 64, 128] if f32 else [64, 128])
    H = rng.choice([1, 2, 3, 4, 6, 8])
    if kind == "window":
        hi = _odd(rng, 8, 4000)
        B = _odd(rng, 1, max(1, min(200, 24000 // hi)))
        dist = rng.choice(["uniform", "powerlaw"])
        pos, time = rng.choice([(True, True), (True, True), (True, False), (False, True),
                                (False, False)])
        return dict(kind=kind, dtype=dtype, B=B, dist=dist, p=1.1, lo=max(1, hi // 20), hi=hi,
                    H=min(H, 4), d=d, window=_odd(rng, 1, min(hi, 700)),
                    sinks=rng.choice([0, 1, 5, 40, 130]), pos=pos, time=time,
                    nb=rng.choice([32, 128]), bwd=rng.random() < 0.6, lens=lens)
    page = rng.choice([8, 16, 32, 64, 128])
    if kind == "decode":
        hi = _odd(rng, 10, 60000)
        B = _odd(rng, 1, max(1, min(256, 400000 // hi)))
        some = rng.random() < 0.4
        return dict(kind=kind, dtype=dtype, B=B, dist=rng.choice(["uniform", "powerlaw"]), p=1.1,
                    lo=max(1, hi // 30), hi=hi, H=H, d=d, page=page,
                    window=_odd(rng, 1, hi) if some else 0,
                    sinks=rng.choice([0, 3, 50]) if some else 0, pos=rng.random() < 0.8,
                    time=rng.random() < 0.6, nb=rng.choice([32, 128]), lens=lens)
    hi = _odd(rng, 20, 2000)
    return dict(kind=kind, dtype=dtype, B=_odd(rng, 1, max(1, min(64, 40000 // hi))),
                dist="uniform", p=0.0, lo=max(1, hi // 10), hi=hi, H=H, d=d, page=page,
                beams=rng.choice([1, 2, 4, 5]) if kind == "beams" else 1, lens=lens)


def _lengths(case):
    rng = np.random.default_rng(case["lens"])
    lo, hi, B = case["lo"], case["hi"], case["B"]
    if case["dist"] == "uniform":
        return rng.integers(lo, hi + 1, B)
    x = np.arange(lo, hi + 1, dtype=np.float64)
    w = x ** -case["p"]
    return rng.choice(np.arange(lo, hi + 1), size=B, p=w / w.sum())


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _clock(lens, gen):
    """Timestamps of the sequences, one after the other, each from 0 on."""
    T = int(sum(lens))
    gaps = 1 + torch.floor(-TS_GAP_MEAN * torch.log1p(
        -torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)))
    at = torch.cumsum(gaps, 0).to(torch.int64)
    first = torch.tensor(np.concatenate([[0], np.cumsum(lens)[:-1]]), device=DEV)
    return at - torch.repeat_interleave(at[first], torch.tensor(lens, device=DEV))


def _tables(case, N, gen):
    H = case["H"]
    pos = time = None
    if case["pos"]:
        pos = RAB_STD * torch.randn(H, 2 * N - 1, generator=gen, device=DEV)
    if case["time"]:
        time = RAB_STD * torch.randn(H, case["nb"], generator=gen, device=DEV)
    return pos, time


# ----------------------------------------------------------------- prepare
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"window": _prepare_window, "decode": _prepare_decode, "beams": _prepare_beams,
            "fill": _prepare_fill, "compact": _prepare_compact}[case["kind"]](case, gen)


def _randn(case, gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV).to(_dtype(case))


def _prepare_window(case, gen):
    lens = _lengths(case)
    T, H, d, N = int(lens.sum()), case["H"], case["d"], case["hi"]
    s = dict(case=case, lens=[int(x) for x in lens], N=N)
    s["off"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int64, device=DEV)
    for n in ("q", "k", "v", "u"):
        s[n] = _randn(case, gen, T, H, d)
    s["u"] = s["u"].view(T, H * d)
    if case["bwd"]:
        s["dy"] = _randn(case, gen, T, H * d)
    s["ts"] = _clock(lens, gen) if case["time"] else None
    s["pos"], s["time"] = _tables(case, N, gen)
    if own:
        from paper_2605_13433_amd import hstu
        s["plan"] = hstu.Plan(s["q"], s["off"], N, s["pos"], s["time"], s["ts"], case["nb"],
                              backward=case["bwd"], window=case["window"], sinks=case["sinks"])
    return s


def _pools(case, gen, layers, num_pages, max_pages, slots, tables, lens, ts, timestamps=True):
    """A cache's tensors, and (own) the framework's cache that holds them.
    tables: [slots][max_pages] pages (numpy), lens [slots]; refs follow."""
    H, d, P = case["H"], case["d"], case["page"]
    s = dict(case=case)
    refs = np.zeros(num_pages, np.int32)
    used = tables[tables >= 0]
    np.add.at(refs, used, 1)
    if own:
        from paper_2605_13433_amd import paged
        c = paged.Cache(num_pages, P, H, d, slots, max_pages, layers=layers, dtype=_dtype(case),
                        timestamps=timestamps, device=DEV)
        s["cache"] = c
        k, v = c.k, c.v
        s["ts"], s["tables"], s["lens"], s["refs"] = c.ts, c.tables, c.lens, c.refs
    else:
        k, v = (torch.empty(layers, num_pages, P, H, d, dtype=_dtype(case), device=DEV)
                for _ in range(2))
        s["ts"] = torch.empty(num_pages, P, dtype=torch.int64, device=DEV) if timestamps else None
        s["tables"] = torch.empty(slots, max_pages, dtype=torch.int32, device=DEV)
        s["lens"] = torch.empty(slots, dtype=torch.int32, device=DEV)
        s["refs"] = torch.empty(num_pages, dtype=torch.int32, device=DEV)
    s["k"], s["v"] = k, v
    for pool in (k, v):
        flat = pool.view(-1)
        for a in range(0, flat.numel(), 1 << 27):
            n = min(1 << 27, flat.numel() - a)
            flat[a:a + n] = torch.randn(n, generator=gen, device=DEV)
    if timestamps:
        s["ts"].zero_()
        if ts is not None:
            at, b = 0, 0
            page, row = [], []
            for b in range(slots):
                n = int(lens[b])
                x = np.arange(n)
                page.append(tables[b][x // P] if n else x)
                row.append(x % P)
            page, row = np.concatenate(page), np.concatenate(row)
            s["ts"][torch.tensor(page, device=DEV, dtype=torch.int64),
                    torch.tensor(row, device=DEV, dtype=torch.int64)] = ts
    s["tables"].copy_(torch.tensor(tables, dtype=torch.int32))
    s["lens"].copy_(torch.tensor(np.asarray(lens), dtype=torch.int32))
    s["refs"].copy_(torch.tensor(refs))
    return s


def _shuffled(case, lens, num_pages, max_pages):
    """Tables of `lens` tokens whose pages lie anywhere in the pool."""
    P = case["page"]
    order = np.random.default_rng(case["lens"] + 1).permutation(num_pages)
    tables = np.full((len(lens), max_pages), -1, np.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-int(n) // P)
        tables[b, :m] = order[at:at + m]
        at += m
    return tables


def _prepare_decode(case, gen):
    lens = _lengths(case)
    B, P, N = case["B"], case["page"], case["hi"]
    max_pages = -(-N // P)
    num_pages = int(sum(-(-int(n) // P) for n in lens)) + 3
    tables = _shuffled(case, lens, num_pages, max_pages)
    ts = _clock(lens, gen) if case["time"] else None
    s = _pools(case, gen, 1, num_pages, max_pages, B, tables, lens, ts, timestamps=case["time"])
    H, d = case["H"], case["d"]
    s["N"], s["host_lens"] = N, [int(x) for x in lens]
    s["slots"] = torch.tensor(np.random.default_rng(case["lens"] + 2).permutation(B),
                              dtype=torch.int32, device=DEV)
    s["q"] = _randn(case, gen, B, H, d)
    s["u"] = _randn(case, gen, B, H * d)
    s["pos"], s["time"] = _tables(case, N, gen)
    if own:
        from paper_2605_13433_amd import paged
        s["plan"] = paged.DecodePlan(s["cache"], B, N, s["pos"], s["time"], case["nb"],
                                     window=case["window"] or None, sinks=case["sinks"])
    return s


def _prepare_beams(case, gen):
    lens = _lengths(case)
    B, P, W, N = case["B"], case["page"], case["beams"], case["hi"] + 8
    max_pages = -(-N // P)
    prompts = int(sum(-(-int(n) // P) for n in lens))
    num_pages = prompts + B * W + 5
    slots = B * (1 + W)
    tables = np.full((slots, max_pages), -1, np.int32)
    tables[:B] = _shuffled(case, lens, num_pages, max_pages)
    all_lens = np.concatenate([lens, np.zeros(B * W, np.int64)])
    s = _pools(case, gen, 2, num_pages, max_pages, slots, tables, all_lens, _clock(lens, gen))
    s["src"] = torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(W)
    s["dst"] = torch.arange(B, slots, dtype=torch.int32, device=DEV)
    n, H, d = B * W, case["H"], case["d"]
    s["counts"] = torch.ones(n, dtype=torch.int32, device=DEV)
    s["rows"] = torch.arange(n + 1, dtype=torch.int64, device=DEV)
    s["new"] = [(_randn(case, gen, n, H, d), _randn(case, gen, n, H, d)) for _ in range(2)]
    s["new_ts"] = torch.randint(1 << 40, (n,), generator=gen, device=DEV)
    s["max_new"] = 1
    return s


def _prepare_fill(case, gen):
    lens = _lengths(case)
    B, P, N = case["B"], case["page"], case["hi"]
    max_pages = -(-N // P)
    num_pages = int(sum(-(-int(n) // P) for n in lens)) + 3
    s = _pools(case, gen, 1, num_pages, max_pages, B, np.full((B, max_pages), -1, np.int32),
               np.zeros(B, np.int64), None)
    T, H, d = int(lens.sum()), case["H"], case["d"]
    s["dst"] = torch.tensor(np.random.default_rng(case["lens"] + 2).permutation(B),
                            dtype=torch.int32, device=DEV)
    s["counts"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["rows"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int64, device=DEV)
    s["new"] = [(_randn(case, gen, T, H, d), _randn(case, gen, T, H, d))]
    s["new_ts"] = _clock(lens, gen)
    s["max_new"] = int(lens.max())
    return s


def _prepare_compact(case, gen):
    lens = _lengths(case)
    B, P, N = case["B"], case["page"], case["hi"]
    max_pages = -(-N // P)
    num_pages = int(sum(-(-int(n) // P) for n in lens)) + 3
    tables = _shuffled(case, lens, num_pages, max_pages)
    gone = np.random.default_rng(case["lens"] + 2).permutation(B)[:B // 2]
    tables[gone] = -1
    lens[gone] = 0
    s = _pools(case, gen, 1, num_pages, max_pages, B, tables, lens, _clock(lens[lens > 0], gen))
    # the bookkeeping as it stands, so that a pass begins where the last one did:
    # the pages that moved are still where they were
    s["tables0"], s["refs0"] = s["tables"].clone(), s["refs"].clone()
    return s


# --------------------------------------------------------------------- run
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"window": _own_window, "decode": _own_decode, "beams": _own_beams,
                "fill": _own_fill, "compact": _own_compact}[kind](s)
    return {"window": _plain_window, "decode": _plain_decode, "beams": _plain_beams,
            "fill": _plain_fill, "compact": _plain_compact}[kind](s)


def _own_window(s):
    f = s["plan"].forward(s["q"], s["k"], s["v"], s["u"], s["off"])
    out = dict(y=f.y, o=f.o)
    if s["case"]["bwd"]:
        g = s["plan"].backward(s["q"], s["k"], s["v"], s["u"], s["off"], s["dy"])
        out.update(dq=g.dq, dk=g.dk, dv=g.dv, du=g.du)
        if s["pos"] is not None:
            out["d_pos"] = g.d_pos_w
        if s["time"] is not None:
            out["d_time"] = g.d_time_w
    return out


def _own_decode(s):
    r = s["plan"].forward(s["q"], s["u"], s["slots"])
    return dict(y=r.y, o=r.o)


def _held(s, **more):
    return dict(tables=s["tables"], lens=s["lens"], refs=s["refs"], k=s["k"], v=s["v"], ts=s["ts"],
                **more)


def _own_beams(s):
    c = s["cache"]
    c.free(s["dst"])
    c.fork(s["src"], s["dst"])
    start = c.extend(s["dst"], s["counts"])
    c.write(0, *s["new"][0], s["dst"], start, s["rows"], s["max_new"], s["new_ts"])
    c.write(1, *s["new"][1], s["dst"], start, s["rows"], s["max_new"])
    return _held(s, start=start)


def _own_fill(s):
    c = s["cache"]
    c.free(s["dst"])
    start = c.extend(s["dst"], s["counts"])
    c.write(0, *s["new"][0], s["dst"], start, s["rows"], s["max_new"], s["new_ts"])
    return _held(s, start=start)


def _own_compact(s):
    s["tables"].copy_(s["tables0"])
    s["refs"].copy_(s["refs0"])
    live = s["cache"].compact()
    return _held(s, live=live)


# ------------------------------------------------------------- plain forms
def _bucket(delta, nb):
    """|x| < 4 -> |x|, else 4 (e - 1) + the two bits under the leading one."""
    x = delta.abs()
    e = (torch.frexp(x.clamp(min=1).double())[1] - 1).to(torch.int64)
    m = (x >> (e - 2).clamp(min=0)) & 3
    return torch.where(x < 4, x, 4 * (e - 1) + m).clamp(max=nb - 1)


def _gate(o, u):
    mean = o.mean(-1, keepdim=True)
    var = ((o - mean) ** 2).mean(-1, keepdim=True)
    rstd = torch.rsqrt(var + LN_EPS)
    n = (o - mean) * rstd
    return n * u, n, rstd


def _plain_window(s):
    """Blocks of queries against the keys that any of them sees, the sequences
    padded side by side (longest first, so that a block takes a prefix)."""
    case, lens, N = s["case"], s["lens"], s["N"]
    H, d, W, S, bwd = case["H"], case["d"], case["window"], case["sinks"], case["bwd"]
    order = sorted(range(len(lens)), key=lambda b: -lens[b])
    order_t = torch.tensor(order, device=DEV)
    L = torch.tensor([lens[b] for b in order], device=DEV)
    longest = lens[order[0]]
    at = torch.arange(longest, device=DEV)
    have = at[None, :] < L[:, None]                                        # [B][longest]
    row = torch.where(have, s["off"][order_t][:, None] + at[None, :], 0)

    def pad(x):
        return x.float()[row].permute(0, 2, 1, 3).contiguous()              # [B][H][longest][d]

    q, k, v = pad(s["q"]), pad(s["k"]), pad(s["v"])
    ts = s["ts"][row] if s["time"] is not None else None
    block = 256

    def blocks():
        for a in range(0, longest, block):
            e = min(longest, a + block)
            n = sum(1 for b in order if lens[b] > a)
            lo = max(0, a - W + 1)
            cols = torch.cat([at[:min(S, lo)], at[lo:e]])
            i = at[a:e]
            seen = (cols[None, :] <= i[:, None]) & ((i[:, None] - cols[None, :] < W) |
                                                   (cols[None, :] < S))
            seen = seen[None, None] & have[:n, a:e][:, None, :, None]
            x = torch.matmul(q[:n, :, a:e], k[:n][:, :, cols].transpose(-1, -2).contiguous())
            delta = cols[None, :] - i[:, None] + N - 1
            if s["pos"] is not None:
                x = x + s["pos"][:, delta]
            bk = None
            if ts is not None:
                bk = _bucket(ts[:n, a:e][:, :, None] - ts[:n][:, cols][:, None, :], case["nb"])
                x = x + s["time"][:, bk].permute(1, 0, 2, 3)
            yield a, e, n, cols, delta, bk, seen, x, torch.sigmoid(x)

    o = torch.zeros_like(q)
    for a, e, n, cols, _, _, seen, x, sg in blocks():
        p = torch.where(seen, x * sg / N, 0.0)
        o[:n, :, a:e] = torch.matmul(p, v[:n][:, :, cols])

    T = s["q"].shape[0]

    def back(x):                                                            # [T][H][d]
        return x.permute(0, 2, 1, 3)[have].view(-1, H, d)[inverse]

    # rows in the padded order -> their places
    inverse = torch.empty(T, dtype=torch.int64, device=DEV)
    inverse[row[have]] = torch.arange(T, device=DEV)
    of = back(o)
    u = s["u"].float()
    y, nrm, rstd = _gate(of.reshape(T, H * d), u)
    dt = _dtype(case)
    out = dict(y=y.to(dt), o=of.to(dt))
    if not bwd:
        return out
    dy = s["dy"].float()
    g = dy * u
    dO = rstd * (g - g.mean(-1, keepdim=True) - nrm * (g * nrm).mean(-1, keepdim=True))
    dO = pad(dO.view(T, H, d))
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    d_pos = torch.zeros(H, 2 * N - 1, dtype=torch.float64, device=DEV)
    d_time = torch.zeros(H, case["nb"], dtype=torch.float64, device=DEV)
    for a, e, n, cols, delta, bk, seen, x, sg in blocks():
        p = torch.where(seen, x * sg / N, 0.0)
        da = torch.matmul(dO[:n, :, a:e], v[:n][:, :, cols].transpose(-1, -2).contiguous())
        ds = torch.where(seen, da * sg * (1 + x * (1 - sg)) / N, 0.0)
        dq[:n, :, a:e] = torch.matmul(ds, k[:n][:, :, cols])
        dk[:n, :, cols] += torch.matmul(ds.transpose(-1, -2).contiguous(), q[:n, :, a:e])
        dv[:n, :, cols] += torch.matmul(p.transpose(-1, -2).contiguous(), dO[:n, :, a:e])
        if s["pos"] is not None:
            some = seen.any(0)[0]
            d_pos.index_add_(1, delta[some], ds.double().sum(0)[:, some])
        if bk is not None:
            rows = torch.zeros(n, H, e - a, case["nb"], device=DEV)
            rows.scatter_add_(3, bk[:, None].expand(n, H, -1, -1).contiguous(), ds)
            d_time += rows.double().sum((0, 2))
    out.update(dq=back(dq).to(dt), dk=back(dk).to(dt), dv=back(dv).to(dt),
               du=(nrm * dy).to(dt))
    if s["pos"] is not None:
        out["d_pos"] = d_pos.float()
    if s["time"] is not None:
        out["d_time"] = d_time.float()
    return out


def _plain_decode(s):
    case, N = s["case"], s["N"]
    H, d, P, B = case["H"], case["d"], case["page"], case["B"]
    W, S = case["window"] or N, case["sinks"]
    o = torch.zeros(B, H, d, device=DEV)
    slots = s["slots"].long()
    lens = s["lens"].long()[slots]
    longest = max(s["host_lens"])
    at = torch.arange(longest, device=DEV)
    step = max(1, (1 << 28) // (longest * H * d))                 # sequences at a time
    for b in range(0, B, step):
        n = lens[b:b + step]
        last = n - 1
        seen = (at[None] < n[:, None]) & ((last[:, None] - at[None] < W) | (at[None] < S))
        page = s["tables"].long()[slots[b:b + step]][:, at // P]
        rows = torch.where(seen, page * P + at[None] % P, 0)
        k = s["k"][0].view(-1, H, d)[rows].float()                 # [b][longest][H][d]
        x = (k * s["q"][b:b + step].float()[:, None]).sum(-1)       # [b][longest][H]
        if s["pos"] is not None:
            x = x + s["pos"].t()[(at[None] - last[:, None] + N - 1).clamp(min=0, max=2 * N - 2)]
        if s["time"] is not None:
            t = s["ts"].view(-1)[rows]
            mine = torch.gather(t, 1, last[:, None])
            x = x + s["time"].t()[_bucket(mine - t, case["nb"])]
        p = torch.where(seen[..., None], x * torch.sigmoid(x) / N, 0.0)
        v = s["v"][0].view(-1, H, d)[rows].float()
        o[b:b + step] = (p[..., None] * v).sum(1)
    y = _gate(o.view(B, H * d), s["u"].float())[0]
    dt = _dtype(case)
    return dict(y=y.to(dt), o=o.to(dt))


def _count_pages(s, tables, sign):
    """refs += sign, once for every entry of `tables`."""
    e = tables.reshape(-1).long()
    n = s["refs"].numel()
    s["refs"] += sign * torch.zeros(n + 1, dtype=torch.int32, device=DEV).index_add_(
        0, torch.where(e < 0, n, e), torch.ones_like(e, dtype=torch.int32))[:n]


def _plain_free(s, slots):
    slots = slots.long()
    _count_pages(s, s["tables"][slots], -1)
    s["tables"][slots] = -1
    s["lens"][slots] = 0


def _plain_fork(s, src, dst):
    src, dst = src.long(), dst.long()
    _count_pages(s, s["tables"][src], 1)
    _count_pages(s, s["tables"][dst], -1)
    s["tables"][dst] = s["tables"][src]
    s["lens"][dst] = s["lens"][src]


def _plain_extend(s, slots, counts):
    """Room for counts[r] more tokens of sequence slots[r]: pages from the lowest
    free one on, row by row; a last page that others share too is copied first."""
    P, tables, refs = s["case"]["page"], s["tables"], s["refs"]
    slots, counts = slots.long(), counts.long()
    start = s["lens"][slots].long()
    had, want = (start + P - 1) // P, (start + counts + P - 1) // P
    last = (had - 1).clamp(min=0)
    old = tables[slots, last].long()
    cow = (start % P != 0) & (counts > 0) & (refs[old.clamp(min=0)] > 1)
    need = want - had + cow
    base = torch.cumsum(need, 0) - need
    total, widest = int(need.sum()), int(need.max())
    fresh = torch.nonzero(refs == 0).view(-1)[:total]
    x = torch.arange(widest, device=DEV)
    mine = x[None] < need[:, None]
    r = torch.arange(len(slots), device=DEV)[:, None].expand_as(mine)[mine]
    col = ((had - cow.long())[:, None] + x[None])[mine]
    page = fresh[(base[:, None] + x[None])[mine]]
    to = fresh[base[cow]]
    row = torch.arange(P, device=DEV)
    keep = row[None] < (start[cow] % P)[:, None]
    a, b = (old[cow][:, None] * P + row[None])[keep], (to[:, None] * P + row[None])[keep]
    for pool in (s["k"], s["v"]):
        for layer in range(pool.shape[0]):
            flat = pool[layer].view(-1, pool.shape[3] * pool.shape[4])
            flat[b] = flat[a]
    s["ts"].view(-1)[b] = s["ts"].view(-1)[a]
    refs.index_add_(0, old[cow], torch.full_like(old[cow], -1, dtype=torch.int32))
    refs[page] = 1
    tables[slots[r], col] = page.int()
    s["lens"][slots] += counts.int()
    return start.int()


def _plain_write(s, layer, k, v, slots, start, rows, ts=None):
    P = s["case"]["page"]
    T = k.shape[0]
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(rows, t, right=True) - 1
    pos = start.long()[r] + t - rows[r]
    at = s["tables"][slots.long()[r], pos // P].long() * P + pos % P
    F = k.shape[1] * k.shape[2]
    s["k"][layer].view(-1, F)[at] = k.view(T, F)
    s["v"][layer].view(-1, F)[at] = v.view(T, F)
    if ts is not None:
        s["ts"].view(-1)[at] = ts


def _plain_beams(s):
    _plain_free(s, s["dst"])
    _plain_fork(s, s["src"], s["dst"])
    start = _plain_extend(s, s["dst"], s["counts"])
    _plain_write(s, 0, *s["new"][0], s["dst"], start, s["rows"], s["new_ts"])
    _plain_write(s, 1, *s["new"][1], s["dst"], start, s["rows"])
    return _held(s, start=start)


def _plain_fill(s):
    _plain_free(s, s["dst"])
    start = _plain_extend(s, s["dst"], s["counts"])
    _plain_write(s, 0, *s["new"][0], s["dst"], start, s["rows"], s["new_ts"])
    return _held(s, start=start)


def _plain_compact(s):
    s["tables"].copy_(s["tables0"])
    s["refs"].copy_(s["refs0"])
    refs, tables = s["refs"], s["tables"]
    n = refs.numel()
    used = refs > 0
    live = used.sum()
    ids = torch.arange(n, device=DEV)
    src = ids[used & (ids >= live)]
    dst = ids[~used & (ids < live)]
    to = ids.clone()
    to[src] = dst
    for pool in (s["k"], s["v"]):
        for layer in range(pool.shape[0]):
            pool[layer][dst] = pool[layer][src]
    s["ts"][dst] = s["ts"][src]
    refs[dst] = refs[src]
    refs[src] = 0
    tables.copy_(torch.where(tables >= 0, to[tables.clamp(min=0).long()].int(), tables))
    return _held(s, live=live.int().view(1))


# -------------------------------------------------------------------- work
def _seen_pairs(lens, W, S):
    """Pairs (i, j <= i) with i - j < W or j < S."""
    n = 0
    for L in lens:
        i = np.arange(int(L), dtype=np.int64)
        lo = np.maximum(0, i - W + 1)
        n += int((i + 1 - lo + np.minimum(lo, S)).sum())
    return n


def work(case):
    lens = _lengths(case)
    H, d = case["H"], case["d"]
    F, es = H * d, 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind == "window":
        T, N = int(lens.sum()), case["hi"]
        pairs = _seen_pairs(lens, case["window"], case["sinks"])
        tab = 4 * H * ((2 * N - 1 if case["pos"] else 0) + (case["nb"] if case["time"] else 0))
        ts = 8 * T if case["time"] else 0
        # q, k, v, u in, y and o out; backward: dy in, dq, dk, dv, du out too
        rows = 11 if case["bwd"] else 6
        return dict(bytes=rows * T * F * es + ts + tab * (2 if case["bwd"] else 1),
                    flops=pairs * F * (12 if case["bwd"] else 4))
    if kind == "decode":
        N = case["hi"]
        n = sum(_decode_seen(int(L), case["window"] or N, case["sinks"]) for L in lens)
        return dict(bytes=2 * n * F * es + (8 * n if case["time"] else 0) +
                    4 * n * H * bool(case["pos"]) + 4 * case["B"] * F * es, flops=4 * n * F)
    P = case["page"]
    if kind == "compact":
        s = _compact_moves(case)
        return dict(bytes=2 * s * P * (2 * F * es + 8), flops=0)
    new = case["B"] * case["beams"] if kind == "beams" else int(lens.sum())
    layers = 2 if kind == "beams" else 1
    copied = 0
    if kind == "beams":
        copied = case["beams"] * sum(int(L) % P for L in lens)
    return dict(bytes=2 * (new + copied) * (2 * layers * F * es + 8), flops=0)


def _decode_seen(L, W, S):
    lo = max(0, L - W)
    return L - lo + min(lo, S)


def _compact_moves(case):
    lens = _lengths(case)
    P = case["page"]
    num_pages = int(sum(-(-int(n) // P) for n in lens)) + 3
    tables = _shuffled(case, lens, num_pages, -(-case["hi"] // P))
    tables[np.random.default_rng(case["lens"] + 2).permutation(case["B"])[:case["B"] // 2]] = -1
    used = tables[tables >= 0]
    return int((used >= len(used)).sum())


# ------------------------------------------------------------------- exact
def _edges(nb):
    """The smallest distance of every bucket from 1 on."""
    out = [1, 2, 3]
    e = 2
    while len(out) < nb and e < 62:
        out += [(4 + m) << (e - 2) for m in range(4)]
        e += 1
    return torch.tensor(out[:nb - 1], dtype=torch.int64, device=DEV)


def exact(case, seed):
    kind = case["kind"]
    if kind == "window":
        return _exact_window(case, seed)
    if kind == "decode":
        return _exact_decode(case, seed)
    # whole numbers and copies: nothing that 64 bits would make better
    return None


def _exact_window(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    H, d, N, T = case["H"], case["d"], s["N"], s["q"].shape[0]
    edges = _edges(case["nb"])
    out = dict(y=torch.zeros(T, H * d), o=torch.zeros(T, H, d))
    out = {n: t.double().to(DEV) for n, t in out.items()}
    if case["bwd"]:
        for n in ("dq", "dk", "dv"):
            out[n] = torch.zeros(T, H, d, dtype=torch.float64, device=DEV)
        out["du"] = torch.zeros(T, H * d, dtype=torch.float64, device=DEV)
        if case["pos"]:
            out["d_pos"] = torch.zeros(H, 2 * N - 1, dtype=torch.float64, device=DEV)
        if case["time"]:
            out["d_time"] = torch.zeros(H, case["nb"], dtype=torch.float64, device=DEV)
    at = 0
    for L in s["lens"]:
        if L == 0:
            continue
        rows = slice(at, at + L)
        at += L
        q, k, v = (s[n][rows].double().transpose(0, 1).contiguous().requires_grad_(case["bwd"])
                   for n in ("q", "k", "v"))
        u = s["u"][rows].double().requires_grad_(case["bwd"])
        gap = torch.arange(L, device=DEV)[:, None] - torch.arange(L, device=DEV)[None, :]
        first = torch.arange(L, device=DEV)[None, :] < case["sinks"]
        hide = (gap < 0) | ((gap >= case["window"]) & ~first)
        bias = torch.zeros(H, L, L, dtype=torch.float64, device=DEV)
        bk = None
        if case["pos"]:
            bias += s["pos"].double()[:, N - 1 - gap]
        if case["time"]:
            t = s["ts"][rows]
            bk = torch.searchsorted(edges, (t[:, None] - t[None, :]).abs(), right=True)
            bias += s["time"].double()[:, bk]
        bias.requires_grad_(case["bwd"])
        with torch.set_grad_enabled(case["bwd"]):
            x = torch.matmul(q, k.transpose(1, 2)) + bias
            p = (x / (1 + torch.exp(-x)) / N).masked_fill(hide, 0.0)
            o = torch.matmul(p, v).transpose(0, 1)
            flat = o.reshape(L, H * d)
            c = flat - flat.mean(1, keepdim=True)
            y = c / torch.sqrt((c * c).mean(1, keepdim=True) + LN_EPS) * u
            if case["bwd"]:
                (y * s["dy"][rows].double()).sum().backward()
        out["y"][rows], out["o"][rows] = y.detach(), o.detach()
        if case["bwd"]:
            for n, x in (("dq", q), ("dk", k), ("dv", v)):
                out[n][rows] = x.grad.transpose(0, 1)
            out["du"][rows] = u.grad
            ds = bias.grad
            if case["pos"]:
                # rows upside down, each one place further right: diagonals in columns
                wide = torch.nn.functional.pad(ds.flip(1), (0, L)).view(H, -1)[:, :-L]
                out["d_pos"][:, N - L:N + L - 1] += wide.view(H, L, 2 * L - 1).sum(1)
            if case["time"]:
                per = torch.zeros(H * L, case["nb"], dtype=torch.float64, device=DEV)
                per.scatter_add_(1, bk.repeat(H, 1), ds.view(H * L, L))
                out["d_time"] += per.view(H, L, -1).sum(1)
    return out


def _exact_decode(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    H, d, P, B, N = case["H"], case["d"], case["page"], case["B"], s["N"]
    W, S = case["window"] or N, case["sinks"]
    edges = _edges(case["nb"])
    o = torch.zeros(B, H, d, dtype=torch.float64, device=DEV)
    slots = s["slots"].tolist()
    for b, slot in enumerate(slots):
        L = s["host_lens"][slot]
        if L == 0:
            continue
        j = list(range(min(S, max(0, L - W)))) + list(range(max(0, L - W), L))
        j = torch.tensor(j, device=DEV)
        page = s["tables"][slot].long()[torch.div(j, P, rounding_mode="floor")]
        k, v = (s[n][0][page, j % P].double() for n in ("k", "v"))
        x = torch.matmul(k.transpose(0, 1), s["q"][b].double()[:, :, None])[:, :, 0]   # [H][n]
        if case["pos"]:
            x = x + s["pos"].double()[:, j - (L - 1) + N - 1]
        if case["time"]:
            t = s["ts"][page, j % P]
            x = x + s["time"].double()[:, torch.searchsorted(edges, (t[-1] - t).abs(), right=True)]
        p = x / (1 + torch.exp(-x)) / N
        o[b] = torch.matmul(p[:, None], v.transpose(0, 1).contiguous())[:, 0]
    flat = o.view(B, H * d)
    c = flat - flat.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + LN_EPS) * s["u"].double()
    return dict(y=y, o=o)
