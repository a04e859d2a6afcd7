"""Performance cases of the attention operators, through their public entry points.

Between the product that makes queries, keys and values and the one that reads attention's
output, a transformer block runs

* ``rotate``  the root-mean-square norm of each head of the queries and keys, and the rotation
              by the token's position in the same pass;
* ``write``   the same with the keys and the values written into the pages of a cache, as E4M3
              codes with one scale for each token and head, or in 16 bits;
* ``read``    sequences of a cache brought back into packed rows;
* ``attend``  attention over whole prompts: packed sequences of different lengths, grouped
              heads, causal (aligned at the sequences' ends) or not;
* ``cached``  attention of each sequence's new tokens, one or a chunk, over its pages.

A cache holds [pages][heads][tokens of a page][D]; E4M3: s = max |y| / 448, floored at 2^-126.
Sizes are those of the SDXL-like and PixArt-like blocks (heads of 64 and 72, 2 x 4096 tokens,
texts of 120 tokens at 64 heads of 64), and generic grouped heads of 128.  The plain form is
elementary torch in 32 bits; ``exact`` redoes a case in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6
TINY = 2.0 ** -126


# ---------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a decoder with 32 query and 8 key heads: latency alone
        dict(name="rotate_token", kind="rotate", T=1, Hq=32, Hk=8, D=128, R=128, x="bf16", pairs=False, far=131072, norm=True),
        # queries and keys of DiT tokens (2 x 4096, 16 heads of 72), two thirds of each head rotated
        dict(name="rotate_dit", kind="rotate", T=8192, Hq=16, Hk=16, D=72, R=48, x="bf16", pairs=True, far=4096, norm=True),
        # one new token of each of 64 sequences: norm, rotation, and an 8-bit cache written in one call
        dict(name="write_tokens", kind="write", T=64, Hq=32, Hk=8, D=128, R=128, x="bf16", pairs=False, far=131072, norm=True,
             page=64, cache="e4m3"),
        # a prompt's keys and values written as they are, one token in twenty left out (padding)
        dict(name="write_prompt", kind="write", T=8100, Hq=0, Hk=8, D=128, R=0, x="f16", pairs=False, far=0, norm=False,
             page=32, cache="e4m3"),
        # two short texts out of a 16-bit cache
        dict(name="read_text", kind="read", B=2, total=240, Hk=20, D=64, page=16, x="f16", cache="f16"),
        # long contexts out of an 8-bit cache
        dict(name="read_long", kind="read", B=3, total=30001, Hk=8, D=128, page=64, x="bf16", cache="e4m3"),
        # text tokens through a causal text encoder, 64 heads of 64
        dict(name="attend_text", kind="attend", B=2, nq=240, nk=240, equal=True, Hq=64, Hk=64, D=64, x="f16", causal=True),
        # DiT tokens: two images of 4096, 16 heads of 72, every token sees every one of its image
        dict(name="attend_dit", kind="attend", B=2, nq=8192, nk=8192, equal=True, Hq=16, Hk=16, D=72, x="bf16", causal=False),
        # prompts of different lengths packed one after another, grouped heads
        dict(name="attend_packed", kind="attend", B=7, nq=8101, nk=8101, equal=False, Hq=32, Hk=8, D=128, x="bf16", causal=True),
        # one sequence that takes its next token: latency
        dict(name="cached_token", kind="cached", B=1, nq=1, total=700, Hq=32, Hk=8, D=128, page=16, x="bf16", cache="bf16"),
        # 48 sequences of up to thousands of tokens that take their next token each, 8-bit cache
        dict(name="cached_batch", kind="cached", B=48, nq=48, total=200000, Hq=32, Hk=8, D=128, page=64, x="bf16", cache="e4m3"),
        # chunks of new tokens over long 8-bit caches
        dict(name="cached_chunk", kind="cached", B=3, nq=1100, total=36000, Hq=32, Hk=8, D=128, page=64, x="bf16", cache="e4m3"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "write", "read", "attend", "attend", "cached", "cached"])
    x = rng.choice(["f16", "bf16"])
    G, Hk, D = rng.choice([1, 1, 2, 3, 4, 5, 8]), rng.choice([1, 2, 4, 5, 8, 10, 16]), rng.choice([64, 64, 80, 96, 128, 128])
    if kind in ("rotate", "write"):
        norm = rng.random() < 0.7
        R = 2 * rng.randint(4, D // 2) if rng.random() < 0.8 or not norm else 0
        c = dict(kind=kind, T=_logint(rng, 1, 16384), Hq=G * Hk, Hk=Hk, D=D, R=R, x=rng.choice([x, "f32"]),
                 pairs=rng.random() < 0.5, far=_logint(rng, 100, 1000000), norm=norm)
        while c["T"] * c["Hq"] * D > 8192 * 16 * 72:
            c["T"] = _logint(rng, 1, 16384)
        if kind == "write":
            c.update(page=rng.choice([16, 32, 64, 128]), cache="e4m3" if rng.random() < 0.6 else x)
        return c
    if kind == "read":
        B = _logint(rng, 1, 64)
        return dict(kind=kind, B=B, total=max(B, _logint(rng, 30, 30000)), Hk=min(Hk, 8), D=D, page=rng.choice([16, 32, 64, 128]),
                    x=x, cache="e4m3" if rng.random() < 0.6 else x)
    while True:
        B = _logint(rng, 1, 64)
        if kind == "attend":
            nq = max(B, _logint(rng, 16, 8192))
            nk = nq if rng.random() < 0.7 else max(B, _logint(rng, 16, 8192))
            c = dict(kind=kind, B=B, nq=nq, nk=nk, equal=False, Hq=G * Hk, Hk=Hk, D=D if rng.random() < 0.8 else 72, x=x,
                     causal=nq == nk and rng.random() < 0.7)
            lq, lk = _lengths(B, nq, False), _lengths(B, nk, False)
        else:
            nq = B if rng.random() < 0.6 else max(B, _logint(rng, 2, 2000))
            c = dict(kind=kind, B=B, nq=nq, total=max(4 * nq, _logint(rng, 100, 200000)), Hq=G * Hk, Hk=Hk, D=D,
                     page=rng.choice([16, 32, 64, 128]), x=x, cache="e4m3" if rng.random() < 0.6 else x)
            lq, lk = _new(c)
        # the plain form's scores of all sequences, padded to the longest
        if B * max(lq) * max(lk) * c["Hq"] <= 1 << 30 and B * max(lk) * Hk * D <= 1 << 28 and work(c)["flops"] <= 2.2e11:
            return c


def _lengths(B, total, equal):
    """B lengths that add up to total: equal, or spread over a factor of about thirty."""
    if equal or B == 1:
        return [total // B + (i < total % B) for i in range(B)]
    r = random.Random(B * 1000003 + total)
    w = [math.exp(r.uniform(0.0, 3.4)) for _ in range(B)]
    n = [1 + int((total - B) * v / sum(w)) for v in w]
    n[n.index(max(n))] += total - sum(n)
    return n


def _new(c):
    """Of a cached case: new tokens of each sequence, and its length with them."""
    lq = _lengths(c["B"], c["nq"], False)
    past = _lengths(c["B"], c["total"] - c["nq"], False)
    return lq, [a + b for a, b in zip(lq, past)]


def _pages(lens, page):
    return [-(-n // page) for n in lens]


def work(c):
    k, p, D = c["kind"], SIZE[c["x"]], c["D"]
    if k in ("rotate", "write"):
        q, kv = c["T"] * c["Hq"] * D, c["T"] * c["Hk"] * D
        if k == "rotate":
            return {"bytes": 2 * p * (q + kv), "flops": 10 * (q + kv)}
        out = 2 * kv * SIZE[c["cache"]] + (8 * c["T"] * c["Hk"] if c["cache"] == "e4m3" else 0)
        return {"bytes": 2 * p * q + 2 * p * kv + out, "flops": 10 * (q + kv) + 3 * kv}
    token = 2 * c["Hk"] * (D * SIZE[c["cache"]] + (4 if c["cache"] == "e4m3" else 0)) if "cache" in c else 2 * c["Hk"] * D * p
    if k == "read":
        return {"bytes": c["total"] * (token + 2 * c["Hk"] * D * p), "flops": 2 * c["total"] * c["Hk"] * D}
    if k == "attend":
        lq, lk = _lengths(c["B"], c["nq"], c["equal"]), _lengths(c["B"], c["nk"], c["equal"])
        pairs = sum(a * (a + 1) // 2 if c["causal"] else a * b for a, b in zip(lq, lk))
    else:
        lq, lk = _new(c)
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(lq, lk))
    return {"bytes": sum(lk) * token + 2 * sum(lq) * c["Hq"] * D * p, "flops": 4 * D * c["Hq"] * pairs}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _heads(g, T, H, D, dt, spread=1.0):
    """Rows as the products before attention give them: heads of different sizes, a few large columns."""
    z = torch.randn((T, H, D), generator=g, device=DEV)
    z *= spread * torch.exp(0.3 * torch.randn((1, H, 1), generator=g, device=DEV))
    z *= torch.where(torch.rand((1, 1, D), generator=g, device=DEV) < 0.03, 3.0, 1.0)
    return z.to(dt)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(lens):
    n = [0]
    for v in lens:
        n.append(n[-1] + v)
    return _ints(n)


def _cached(g, pages, c):
    """The pages of a cache: codes and scales, or 16-bit rows."""
    def one():
        z = _heads(g, pages * c["Hk"] * c["page"], 1, c["D"], torch.float32)
        if c["cache"] != "e4m3":
            return z.view(pages, c["Hk"], c["page"], c["D"]).to(DT[c["cache"]]), None
        s = (z.abs().amax(2, keepdim=True) / 448.0).clamp(min=TINY)
        codes = (z * (1.0 / s)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        return codes.view(pages, c["Hk"], c["page"], c["D"]), s.view(pages, c["Hk"], c["page"])
    (k, ks), (v, vs) = one(), one()
    return dict(k=k, ks=ks, v=v, vs=vs)


def _table(g, lens, page):
    """Each sequence's pages, in no order; places behind its last page hold none."""
    need = _pages(lens, page)
    order = torch.randperm(sum(need), generator=g, device=DEV).to(torch.int32)
    rows = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device=DEV)
    rows[torch.arange(max(need), device=DEV)[None, :] < _ints(need)[:, None]] = order
    return rows, sum(need)


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c)
    k, D = c["kind"], c["D"]
    if k in ("rotate", "write"):
        T, Hq, Hk = c["T"], c["Hq"], c["Hk"]
        # slices of one matrix, as the product in front of them writes it
        qkv = _heads(g, T, Hq + 2 * Hk, D, DT[c["x"]])
        s["q"], s["k_rows"], s["v_rows"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        s["qw"] = torch.rand(D, generator=g, device=DEV) + 0.5
        s["kw"] = torch.rand(D, generator=g, device=DEV) + 0.5
        s["pos"] = torch.randint(0, max(1, c["far"]), (T,), generator=g, device=DEV, dtype=torch.int32)
        s["freq"] = 10000.0 ** (-torch.arange(c["R"] // 2, dtype=torch.float64, device=DEV) / max(1, c["R"] // 2))
        if k == "write":
            pages = -(-T // c["page"]) + 3
            s.update(_cached(g, pages, c))
            slots = torch.randperm(pages * c["page"], generator=g, device=DEV)[:T].to(torch.int32)
            if not c["Hq"]:
                slots[torch.rand(T, generator=g, device=DEV) < 0.05] = -1
            s["slots"] = slots
        return s
    if k == "read":
        lens = _lengths(c["B"], c["total"], False)
        s["table"], pages = _table(g, lens, c["page"])
        s.update(_cached(g, pages, c))
        s["cu"], s["most"] = _starts(lens), max(lens)
        return s
    if k == "attend":
        lq, lk = _lengths(c["B"], c["nq"], c["equal"]), _lengths(c["B"], c["nk"], c["equal"])
        s["q"] = _heads(g, c["nq"], c["Hq"], D, DT[c["x"]], 1.5)
        kv = _heads(g, c["nk"], 2 * c["Hk"], D, DT[c["x"]])
        s["k_rows"], s["v_rows"] = kv[:, :c["Hk"]], kv[:, c["Hk"]:]
        s["cu_k"] = _starts(lk)
    else:
        lq, lk = _new(c)
        s["q"] = _heads(g, c["nq"], c["Hq"], D, DT[c["x"]], 1.5)
        s["table"], pages = _table(g, lk, c["page"])
        s.update(_cached(g, pages, c))
        s["lens"] = _ints(lk)
    s["cu_q"], s["most_q"], s["most_k"] = _starts(lq), max(lq), max(lk)
    return s


# ---------------------------------------------------------------------------------------------
# one pass: the plain form
# ---------------------------------------------------------------------------------------------
def _rotated(x, w, s):
    """The norm and the rotation of rows [T, H, D], in 32 bits (angles in 64)."""
    y = x.float()
    if s["norm"]:
        y = y / torch.sqrt((y * y).mean(2, keepdim=True) + EPS) * w
    R = s["R"]
    if not R:
        return y
    t = s["pos"].double()[:, None] * s["freq"]
    cos, sin = torch.cos(t).float()[:, None], torch.sin(t).float()[:, None]
    if s["pairs"]:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), 3).flatten(2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), 2)
    return torch.cat((r, y[..., R:]), 2)


def _put(rows, cache, scale, slots, page):
    """Rows [T, H, D] in 32 bits into the slots of a cache; negative slots take none."""
    keep = slots >= 0
    at, rows = slots[keep].long(), rows[keep]
    page_of, in_page = at // page, at % page
    if scale is None:
        cache[page_of, :, in_page] = rows.to(cache.dtype)
        return
    sc = (rows.abs().amax(2) / 448.0).clamp(min=TINY)
    cache.view(torch.uint8)[page_of, :, in_page] = (rows * (1.0 / sc)[..., None]).clamp(-448.0, 448.0).to(cache.dtype).view(torch.uint8)
    scale[page_of, :, in_page] = sc


def _sequences(s, lens, most):
    """Cached keys and values of every sequence, [B, H, most, D] in 32 bits."""
    at = torch.arange(most, device=DEV)
    page_of = s["table"][:, at // s["page"]].clamp(min=0).long()
    k, v = s["k"].float(), s["v"].float()
    if s["ks"] is not None:
        k, v = k * s["ks"][..., None], v * s["vs"][..., None]
    return [t[page_of, :, at % s["page"]].transpose(1, 2) for t in (k, v)]


def _padded(rows, cu, most):
    """Packed rows [T, H, D] as [B, H, most, D] in 32 bits, zeros behind each sequence."""
    at = cu[:-1, None].long() + torch.arange(most, device=DEV)
    inside = at < cu[1:, None]
    x = rows.float()[at.clamp(max=len(rows) - 1)]
    return torch.where(inside[..., None, None], x, 0.0).transpose(1, 2)


def _attended(s, k, v, lens, causal):
    """Attention of the padded sequences, packed again."""
    cu, D, x = s["cu_q"], s["D"], s["q"]
    q = _padded(x, cu, s["most_q"])
    B, Hq, nq, nk = q.shape[0], q.shape[1], q.shape[2], k.shape[2]
    q = q.reshape(B, k.shape[1], -1, D)
    t = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hq, nq, nk) * (1.0 / math.sqrt(D))
    last = lens[:, None]
    if causal:
        last = last - (cu[1:] - cu[:-1])[:, None] + torch.arange(1, nq + 1, device=DEV)
    seen = torch.arange(nk, device=DEV) < last[..., None]
    t = torch.where(seen[:, None], t, -math.inf)
    top = t.amax(3, keepdim=True)
    p = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p.view(B, k.shape[1], -1, nk), v.contiguous()).view(B, Hq, nq, D) / torch.where(total == 0, 1.0, total)
    at = torch.arange(nq, device=DEV)
    return o.transpose(1, 2)[at < (cu[1:] - cu[:-1])[:, None]].to(x.dtype)


def run(s):
    if own:
        return _call(s)
    k = s["kind"]
    if k in ("rotate", "write"):
        q = _rotated(s["q"], s["qw"], s).to(s["q"].dtype) if s["Hq"] else None
        kr = _rotated(s["k_rows"], s["kw"], s)
        if k == "rotate":
            return [q, kr.to(q.dtype)]
        _put(kr, s["k"], s["ks"], s["slots"], s["page"])
        _put(s["v_rows"].float(), s["v"], s["vs"], s["slots"], s["page"])
        return [q, s["k"], s["ks"], s["v"], s["vs"]]
    if k == "read":
        lens = s["cu"][1:] - s["cu"][:-1]
        inside = torch.arange(s["most"], device=DEV) < lens[:, None]
        return [t.transpose(1, 2)[inside].to(DT[s["x"]]) for t in _sequences(s, lens, s["most"])]
    if k == "attend":
        kk, vv = _padded(s["k_rows"], s["cu_k"], s["most_k"]), _padded(s["v_rows"], s["cu_k"], s["most_k"])
        return _attended(s, kk, vv, s["cu_k"][1:] - s["cu_k"][:-1], s["causal"])
    kk, vv = _sequences(s, s["lens"], s["most_k"])
    return _attended(s, kk, vv, s["lens"], True)


# ---------------------------------------------------------------------------------------------
# one pass: the framework's operators
# ---------------------------------------------------------------------------------------------
def _call(s):
    from paper_2609_33496_amd import cham
    k = s["kind"]
    if k in ("rotate", "write"):
        how = dict(norm=s["norm"], eps=EPS, layout=cham.ROT_PAIRS if s["pairs"] else cham.ROT_HALF)
        if s["norm"]:
            how.update(q_weight=s["qw"] if s["Hq"] else None, k_weight=s["kw"])
        if s["R"]:
            how.update(positions=s["pos"], freq=s["freq"])
        if k == "rotate":
            return cham.norm_rotate(s["q"], s["k_rows"], **how)
        cache = cham.Cache(s["k"], s["v"], s["ks"], s["vs"])
        q = cham.cache_write(cache, s["slots"], s["k_rows"], s["v_rows"], q=s["q"] if s["Hq"] else None, **how)
        return [q, s["k"], s["ks"], s["v"], s["vs"]]
    if k == "read":
        return cham.cache_read(cham.Cache(s["k"], s["v"], s["ks"], s["vs"]), s["table"], s["cu"], s["total"], dtype=DT[s["x"]])
    if k == "attend":
        if s["equal"]:
            return cham.attention(s["q"], s["k_rows"], s["v_rows"], batch=s["B"], causal=s["causal"])
        return cham.attention(s["q"], s["k_rows"], s["v_rows"], cu_q=s["cu_q"], cu_k=s["cu_k"], causal=s["causal"])
    return cham.cache_attention(s["q"], cham.Cache(s["k"], s["v"], s["ks"], s["vs"]), s["table"], s["lens"],
                                cu_q=s["cu_q"] if s["nq"] > s["B"] else None)


# ---------------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    k, D = c["kind"], c["D"]
    if k in ("rotate", "write"):
        q = _exact_rows(s["q"], s["qw"], c, s) if c["Hq"] else None
        kr = _exact_rows(s["k_rows"], s["kw"], c, s)
        if k == "rotate":
            return [q, kr]
        out = [q]
        for rows, cache, scale in ((kr, s["k"], s["ks"]), (s["v_rows"].double(), s["v"], s["vs"])):
            # codes: the values that they round, so that a side's distance from them is its rounding's
            held, sc = cache.double(), scale.double() if scale is not None else None
            for t, at in enumerate(s["slots"].tolist()):
                if at >= 0:
                    if sc is None:
                        held[at // c["page"], :, at % c["page"]] = rows[t]
                    else:
                        one = torch.clamp(rows[t].abs().max(1).values / 448, min=TINY)
                        held[at // c["page"], :, at % c["page"]] = rows[t] / one[:, None]
                        sc[at // c["page"], :, at % c["page"]] = one
            out += [held, sc]
        return out
    if k == "read":
        lens = _lengths(c["B"], c["total"], False)
        return [torch.cat([_exact_gather(s, key, b, n) for b, n in enumerate(lens)]) for key in ("k", "v")]
    if k == "attend":
        lq, lk = _lengths(c["B"], c["nq"], c["equal"]), _lengths(c["B"], c["nk"], c["equal"])
    else:
        lq, lk = _new(c)
    out, tq, tk = [], 0, 0
    for b, (nq, nk) in enumerate(zip(lq, lk)):
        q = s["q"][tq:tq + nq].double()
        if k == "attend":
            kk, vv = s["k_rows"][tk:tk + nk].double(), s["v_rows"][tk:tk + nk].double()
        else:
            kk, vv = _exact_gather(s, "k", b, nk), _exact_gather(s, "v", b, nk)
        o = torch.empty_like(q)
        hidden = None
        if k == "cached" or c["causal"]:  # query i of the last nq positions sees keys up to its own
            hidden = torch.ones(nq, nk, dtype=torch.bool, device=DEV).triu(nk - nq + 1)
        for h in range(c["Hq"]):
            j = h // (c["Hq"] // c["Hk"])
            t = q[:, h] @ kk[:, j].t() / math.sqrt(D)
            if hidden is not None:
                t.masked_fill_(hidden, -math.inf)
            o[:, h] = torch.softmax(t, 1) @ vv[:, j]
        out.append(o)
        tq, tk = tq + nq, tk + nk
    return torch.cat(out)


def _exact_rows(x, w, c, s):
    y = x.double()
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(2, keepdim=True) + EPS) * w.double()
    n = c["R"] // 2
    if n:
        y = y.clone()
        first, step = (1, 2) if c["pairs"] else (n, 1)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"][:, None, None].double() * s["freq"])
        z = torch.complex(y[..., 0:n * step:step].clone(), y[..., first:first + n * step:step].clone()) * turn
        y[..., 0:n * step:step], y[..., first:first + n * step:step] = z.real, z.imag
    return y


def _exact_gather(s, key, b, n):
    rows, scale = s[key], s[key + "s"]
    at = s["table"][b][:-(-n // s["page"])].long()
    x = rows[at].double()
    if scale is not None:
        x = x * scale[at].double()[..., None]
    return x.transpose(1, 2).reshape(-1, s["Hk"], s["D"])[:n]
