"""Serving operators over the shared paged cache: appending any number of tokens with the rotary positions applied on the
way (to a bf16 cache and to one held in 8 bits), and decode attention over the 8-bit cache.

The 8-bit cache: K and V as e4m3 numbers, with one scale for each block of 16 tokens and KV head, a power of two 2^e kept as
a byte e + 127.  e is the smallest integer, at least -100, with amax <= 448 * 2^e over the tokens of the block; where tokens
join a block that older ones began, e does not fall, and if it grows the older numbers are multiplied by the power of two
between and rounded again.

  append   new tokens of every sequence (one each, or ragged runs) go into the pages of the owner layers, K rotated by the
           token's position; the queries of all layers are rotated by the same positions into a buffer of their own
  decode8  one query token a sequence over the 8-bit cache, donor and consumer layers, outputs and log-sum-exp
  step8    both, as a serving step makes them

Sizes come from paper_2608_15943_b200/workloads.py, bench.py and the tests, or are generic.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
THETA = 10000.0
BLOCK = 16                  # tokens that share a scale
LEAST = -100                # smallest exponent of a scale


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def _append(name, L, B, new_lo, new_hi, old_lo, old_hi, Hq, Hkv, dh, page, pairs, bits):
    """new_lo..new_hi new tokens a sequence behind old_lo..old_hi older ones; the last 2 * pairs layers share in pairs (an even
    layer's K/V serves the odd layer above it); bits of a cached number: 16 or 8."""
    return dict(name=name, kind="append", L=L, B=B, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, Hq=Hq, Hkv=Hkv, dh=dh,
                page=page, pairs=pairs, bits=bits)


def _decode(name, L, B, lo, hi, Hq, Hkv, dh, page, pairs, empty=0, kind="decode8"):
    """Contexts of lo..hi tokens; the first `empty` places of the batch hold no sequence."""
    return dict(name=name, kind=kind, L=L, B=B, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, dh=dh, page=page, pairs=pairs, empty=empty)


def listed():
    return [
        # a token for each of two sequences of the tiny stack that an integration is checked with
        _append("append-token-tiny", 4, 2, 1, 1, 100, 140, 4, 2, 64, 16, 2, 16),
        # a serving batch's token step, eight layers at once
        _append("append-token-batch", 8, 32, 1, 1, 300, 1500, 32, 8, 128, 128, 2, 16),
        # prompts of no round length enter the cache behind the forward pass
        _append("append-prompts", 4, 5, 700, 4100, 0, 0, 32, 8, 128, 128, 1, 16),
        # the same token step into the 8-bit cache
        _append("append8-token-batch", 8, 32, 1, 1, 300, 1500, 32, 8, 128, 128, 2, 8),
        # drafted tokens of 13 sequences, which join begun blocks; small heads, small pages
        _append("append8-drafts", 6, 13, 1, 9, 40, 900, 16, 4, 64, 48, 1, 8),
        # long prompts continue behind a cached prefix, the largest call
        _append("append8-prompts-long", 4, 4, 7000, 8192, 1, 999, 32, 8, 128, 128, 1, 8),
        # the smallest decode call
        _decode("decode8-tiny", 4, 2, 129, 144, 4, 2, 64, 16, 2),
        # many short sequences of a padded batch, small heads
        _decode("decode8-short-padded", 6, 61, 1, 700, 12, 4, 64, 32, 2, empty=3),
        # a small batch at moderate context
        _decode("decode8-small", 4, 8, 8192, 16384, 32, 8, 128, 128, 2),
        # the serving batch at long context (a quarter of the 32-layer stack)
        _decode("decode8-batch-long", 8, 32, 16384, 32768, 32, 8, 128, 128, 2),
        # few sequences at the longest context, one KV head per query head
        _decode("decode8-mha-128k", 2, 4, 122880, 131072, 32, 32, 128, 128, 1),
        # a serving step, layer groups of two: append, then attend
        _decode("step8-batch", 4, 16, 3000, 5000, 32, 8, 128, 64, 2, kind="step8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "append", "decode8", "decode8", "step8"))
    dh, Hkv, G = rng.choice((64, 128, 128)), rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 8))
    L, page = rng.randint(1, 8), rng.choice((16, 32, 48, 64, 128))
    pairs = rng.randint(0, L // 2)
    if kind == "append":
        hi = rng.choice((1, 1, _log_int(rng, 2, 4096)))
        old = rng.choice((0, _log_int(rng, 1, 1500)))
        c = _append("", L, _log_int(rng, 1, 48), rng.randint((hi + 1) // 2, hi), hi, old // 2, old, Hkv * G, Hkv, dh, page, pairs, rng.choice((8, 8, 16)))
        while work(c)["bytes"] > 1e9 or _pool_bytes(c) > 4e9:
            c["B"] = max(1, c["B"] // 2)
            for k in ("new_lo", "new_hi", "old_lo", "old_hi"):
                c[k] = max(1 if k.startswith("new") else 0, c[k] * 3 // 4)
    else:
        lo = _log_int(rng, 1 if kind == "decode8" else 16, 65536)
        c = _decode("", L, _log_int(rng, 1, 64), lo, int(lo * rng.uniform(1.0, 2.0)), Hkv * G, Hkv, dh, page, pairs, 0, kind)
        c["empty"] = rng.choice((0, 0, c["B"] // 4))
        while _pool_bytes(c) > 3e9:
            c["lo"], c["hi"] = max(1, c["lo"] * 2 // 3), max(1, c["hi"] * 2 // 3)
    del c["name"]
    return c


def _donors(c):
    first = c["L"] - 2 * c["pairs"]
    return [l if l < first or (l - first) % 2 == 0 else l - 1 for l in range(c["L"])]


def _owners(c):
    return [l for l, d in enumerate(_donors(c)) if d == l]


def _longest(c):
    return c["new_hi"] + c["old_hi"] if c["kind"] == "append" else c["hi"]


def _spread(host, n, lo, hi):
    """n numbers from lo to hi, any of them, whose sum is always the same."""
    x = [host.randint(lo, hi) for _ in range(n)]
    off = n * (lo + hi) // 2 - sum(x)
    for i in host.sample(range(n), n):
        step = max(lo, min(hi, x[i] + off)) - x[i]
        x[i], off = x[i] + step, off - step
    return x


def _pool_bytes(c):
    tokens = c["B"] * (_longest(c) + c["page"])
    return len(_owners(c)) * tokens * 2 * c["Hkv"] * c["dh"] * (2 if c.get("bits") == 16 else 1)


# ---------------------------------------------------------------------------------------------
# states
# ---------------------------------------------------------------------------------------------
def prepare(case, seed):
    c, host = case, random.Random(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    L, B, Hq, Hkv, dh, page = (c[k] for k in ("L", "B", "Hq", "Hkv", "dh", "page"))
    owners, bits = _owners(c), c.get("bits", 8)
    if c["kind"] == "append":
        new = _spread(host, B, c["new_lo"], c["new_hi"])
        lengths = [n + host.randint(c["old_lo"], c["old_hi"]) for n in new]
    else:
        lengths = [0 if b < c["empty"] else host.randint(c["lo"], c["hi"]) for b in range(B)]
        new = [min(1, n) for n in lengths]
    one_each = c["kind"] != "append" or c["new_hi"] == 1
    # the pages of the sequences lie scattered over the pool; the table has room for them to grow
    need = [(n + page - 1) // page for n in lengths]
    most = (_longest(c) + page - 1) // page
    n_pages, max_pages = B * most + 1, most + 2
    order = list(range(n_pages))
    host.shuffle(order)
    table, at = torch.full((B, max_pages), order[-1], dtype=torch.int32), 0      # (a page that no sequence has)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s = dict(case=c, donor=_donors(c), owners=owners, n_pages=n_pages, max_pages=max_pages, one_each=one_each, table=table.to(DEV),
             lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))

    def normal(*shape, dtype=BF):
        return torch.randn(*shape, device=DEV, dtype=dtype, generator=g)

    def pool():
        """Numbers ~ N(0, 1): in 8 bits, blocks whose largest is about 4 have the scale 2^-6."""
        p = torch.empty(len(owners), n_pages, Hkv, page, dh, dtype=BF if bits == 16 else E4M3, device=DEV)
        for layer in p:
            layer.copy_(normal(n_pages, Hkv, page, dh) * (1.0 if bits == 16 else 64.0))
        return p

    s["k_cache"], s["v_cache"] = pool(), pool()
    if bits == 8:
        s["k_scale"], s["v_scale"] = (torch.randint(120, 123, (len(owners), n_pages, Hkv, page // BLOCK), device=DEV, dtype=torch.uint8, generator=g)
                                      for _ in range(2))
    T = B if one_each else sum(new)
    if c["kind"] != "decode8":
        first = [0]
        for n in (new if not one_each else [1] * B):
            first.append(first[-1] + n)
        s["first"] = torch.tensor(first, dtype=torch.int32, device=DEV)
        s["k_new"], s["v_new"] = (normal(len(owners), T, Hkv, dh) for _ in range(2))
    s["q"] = normal(L, T, Hq, dh)
    s["q_out"] = torch.zeros_like(s["q"])
    if c["kind"] != "append":
        s["o"] = torch.empty(L, B, Hq, dh, dtype=BF, device=DEV)
        s["lse"] = torch.empty(L, B, Hq, dtype=F32, device=DEV)
    return s


def run(state):
    kind, out = state["case"]["kind"], {}
    if kind != "decode8":
        (_own_append if own else _plain_append)(state)
        out.update(q=state["q_out"], k=state["k_cache"], v=state["v_cache"])
        if "k_scale" in state:
            out.update(k_scale=state["k_scale"].view(E8M0), v_scale=state["v_scale"].view(E8M0))
    if kind != "append":
        (_own_decode if own else _plain_decode)(state, state["q"] if kind == "decode8" else state["q_out"])
        out.update(o=state["o"], lse=state["lse"])
    return out


# ---------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------
def _handle(s):
    """What a serving program keeps from step to step: the description of its cache, the workspace, the lists of layers."""
    if "handle" not in s:
        from paper_2608_15943_b200 import kvp
        c, own_at = s["case"], {l: i for i, l in enumerate(s["owners"])}
        desc = kvp.DecodeDesc(c["L"], c["B"], c["Hq"], c["Hkv"], c["dh"], c["page"], s["max_pages"], s["n_pages"])
        per_layer = {k: [s[k][own_at[l]] if l in own_at else None for l in range(c["L"])]
                     for k in ("k_new", "v_new", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}
        per_layer.update({k: list(s[k]) for k in ("q", "q_out", "o", "lse") if k in s})
        ws = None
        if c["kind"] != "append":
            ws = torch.empty(max(256, kvp.decode8_workspace_bytes(desc, s["donor"])), dtype=torch.uint8, device=DEV)
        s["handle"] = (kvp, desc, per_layer, ws, None if s["one_each"] else s["first"])
    return s["handle"]


def _own_append(s):
    kvp, desc, at, _, first = _handle(s)
    kvp.cache_append_tokens(desc, s["donor"], at["k_new"], at["v_new"], at["k_cache"], at["v_cache"], s["table"], s["lengths"], first=first, theta=THETA,
                            q=at["q"], q_out=at["q_out"], k_scale=at.get("k_scale"), v_scale=at.get("v_scale"))


def _own_decode(s, q):
    kvp, desc, at, ws, _ = _handle(s)
    kvp.decode8(desc, s["donor"], at["q" if q is s["q"] else "q_out"], at["k_cache"], at["v_cache"], at["k_scale"], at["v_scale"], s["table"], s["lengths"],
                at["o"], at["lse"], ws)


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _places(s):
    """Sequence, position and validity of every token row, its page, and its place in the page."""
    first, lengths, page = s["first"].long(), s["lengths"].long(), s["case"]["page"]
    row = torch.arange(s["q"].shape[1], device=DEV)
    b = torch.bucketize(row, first[1:], right=True)
    pos = lengths[b] - first[b + 1] + row
    there = pos >= 0
    at = pos.clamp(min=0)
    return b, pos, there, s["table"].long()[b, at // page], at % page


def _rotate(x, pos):
    """Pairs of x [..., T, H, dh] turned by pos * THETA^(-2i/dh), angles in 64 bits, in 32 otherwise."""
    half = x.shape[-1] // 2
    freq = THETA ** (-torch.arange(half, device=DEV, dtype=F64) / half)
    angle = pos.double()[:, None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = x.float().unflatten(-1, (half, 2)).unbind(-1)
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)


def _power(byte):
    """2^(byte - 127), exactly."""
    return (byte.int() << 23).view(F32)


def _exponent(amax):
    mantissa, exponent = torch.frexp(amax)
    e = exponent - 9 + (mantissa > 0.875)          # 448 = 0.875 * 2^9
    return torch.where(amax > 0, e, LEAST).clamp(min=LEAST)


def _store8(cache, scale, x, s, places):
    """x [n_own, T, Hkv, dh] into the 8-bit cache [n_own, n_pages, Hkv, page, dh]."""
    b, pos, there, page, slot = places
    n_own, n_pages, Hkv, per_page = scale.shape
    block = page * per_page + slot // BLOCK
    amax = x.abs().amax(-1) * there[:, None]
    most = torch.zeros(n_own, n_pages * per_page, Hkv, device=DEV)
    most.scatter_reduce_(1, block[None, :, None].expand(n_own, -1, Hkv), amax, "amax")
    need = _exponent(most)                                               # [n_own, blocks, Hkv]
    # blocks that older tokens began: those of each sequence's first new token
    start = s["first"].long()[:-1]
    begun, older = block[start], torch.where(there[start], slot[start] % BLOCK, 0)
    by_block = scale.transpose(2, 3).reshape(n_own, -1, Hkv)
    before = by_block[:, begun].int() - 127
    after = torch.where((older > 0)[:, None], torch.maximum(before, need[:, begun]), need[:, begun])
    exponent = need.index_copy(1, begun, after.int())
    rows = cache.unflatten(3, (per_page, BLOCK)).transpose(2, 3)         # [n_own, n_pages, per_page, Hkv, 16, dh]
    bytes_ = rows.view(torch.uint8)
    at = (slice(None), page[start], slot[start] // BLOCK)
    held = bytes_[at].view(E4M3)
    again = (held.float() * _power((before - after.int()).clamp(max=0) + 127)[..., None, None]).to(E4M3).view(torch.uint8)
    is_older = torch.arange(BLOCK, device=DEV) < older[:, None]
    bytes_[at] = torch.where(is_older[:, None, :, None], again, held.view(torch.uint8))
    # the new rows and their scales (padding goes nowhere: its place gets what it has)
    e = exponent[:, block]
    new = (x * _power(127 - e)[..., None]).to(E4M3).view(torch.uint8)
    at = (slice(None), page, slice(None), slot)
    raw = cache.view(torch.uint8)
    raw[at] = torch.where(there[:, None, None, None], new.transpose(0, 1), raw[at])
    at = (slice(None), page, slice(None), slot // BLOCK)
    scale[at] = torch.where(there[:, None, None], (e + 127).to(torch.uint8).transpose(0, 1), scale[at])


def _store16(cache, x, places):
    _, _, there, page, slot = places
    at = (slice(None), page, slice(None), slot)
    cache[at] = torch.where(there[:, None, None, None], x.to(BF).transpose(0, 1), cache[at])


def _plain_append(s):
    places = _places(s)
    pos, there = places[1], places[2]
    s["q_out"].copy_(torch.where(there[:, None, None], _rotate(s["q"], pos).to(BF), s["q_out"]))
    k, v = _rotate(s["k_new"], pos), s["v_new"].float()
    if "k_scale" in s:
        _store8(s["k_cache"], s["k_scale"], k, s, places)
        _store8(s["v_cache"], s["v_scale"], v, s, places)
    else:
        _store16(s["k_cache"], k, places)
        _store16(s["v_cache"], v, places)


def _dequantised(cache, scale, pages, dtype):
    """[..., Hkv, tokens, dh] from the pages [..., P] of one layer's pool."""
    x = cache.view(torch.uint8)[pages].view(E4M3).to(dtype).unflatten(-2, (-1, BLOCK))
    x = x * _power(scale[pages]).to(dtype)[..., None, None]              # [..., P, Hkv, blocks, 16, dh]
    return x.movedim(-4, -5).flatten(-4, -2)


def _plain_decode(s, q):
    c = s["case"]
    B, Hkv, G, dh = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["dh"]
    lengths, pages = s["lengths"].long(), s["table"][:, :s["max_pages"] - 2].long()
    for i, l in enumerate(s["owners"]):
        members = [m for m, d in enumerate(s["donor"]) if d == l]
        k = _dequantised(s["k_cache"][i], s["k_scale"][i], pages, F32)  # [B, Hkv, N, dh]
        rows = q[members].float().unflatten(2, (Hkv, G)).permute(1, 2, 0, 3, 4).flatten(2, 3)
        x = (rows @ k.transpose(-1, -2)) * dh ** -0.5
        del k
        unseen = torch.arange(x.shape[-1], device=DEV) >= lengths[:, None]
        x = x.masked_fill(unseen[:, None, None], -math.inf)
        most = x.amax(-1, keepdim=True)
        p = (x - most.clamp(min=-1e30)).exp()
        total = p.sum(-1, keepdim=True)
        v = _dequantised(s["v_cache"][i], s["v_scale"][i], pages, F32).masked_fill(unseen[:, None, :, None], 0.0)
        o = (p @ v) / torch.where(total > 0, total, 1.0)
        lse = (most + total.log()).squeeze(-1)
        s["o"][members] = o.unflatten(2, (len(members), G)).permute(2, 0, 1, 3, 4).reshape(len(members), B, Hkv * G, dh).to(BF)
        s["lse"][members] = lse.unflatten(2, (len(members), G)).permute(2, 0, 1, 3).reshape(len(members), B, Hkv * G)


# ---------------------------------------------------------------------------------------------
# work and 64-bit values
# ---------------------------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once: new tokens and queries in, cached numbers and rotated queries out;
    attention reads the cached numbers and scales of its sequences once for a donor and all its consumers."""
    c = case
    n_own, nkv, nq, e = len(_owners(c)), c["Hkv"] * c["dh"], c["Hq"] * c["dh"], 2
    cached = 2.0 if c.get("bits") == 16 else 1.0 + 1.0 / (BLOCK * c["dh"])
    nbytes = flops = 0.0
    live = c["B"] - c.get("empty", 0)
    if c["kind"] != "decode8":
        T = c["B"] * (c["new_lo"] + c["new_hi"]) // 2 if c["kind"] == "append" else live
        nbytes += T * (c["L"] * 2 * nq * e + n_own * 2 * nkv * (e + cached))
        flops += T * 3 * (c["L"] * nq + n_own * nkv)
    if c["kind"] != "append":
        tokens = live * (c["lo"] + c["hi"]) / 2
        nbytes += n_own * tokens * 2 * nkv * cached + c["L"] * live * nq * e + c["L"] * c["B"] * (nq * e + c["Hq"] * 4)
        flops += c["L"] * tokens * 4 * nq
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    """From the definitions in 64 bits, sequence by sequence.  Cached 8-bit numbers are given before their rounding, so that
    their half step is in what either side is off by; scales are whole powers and given as they are."""
    c, s, out = case, prepare(case, seed), {}
    first = s["first"].tolist() if "first" in s else None
    lengths, table, page = s["lengths"].tolist(), s["table"].tolist(), c["page"]
    q, half = s["q"].double(), c["dh"] // 2
    if c["kind"] != "decode8":
        turned = s["q_out"].double()
        k, v = s["k_cache"].double(), s["v_cache"].double()
        scales = [s[n].long() for n in ("k_scale", "v_scale")] if "k_scale" in s else None
        for b in range(c["B"]):
            n = first[b + 1] - first[b]
            start = lengths[b] - n
            if start < 0:
                continue
            z = torch.arange(start, start + n, device=DEV, dtype=F64)[:, None, None] * torch.tensor([THETA ** (-i / half) for i in range(half)], device=DEV, dtype=F64)
            z = torch.polar(torch.ones_like(z), z)

            def turn(x):
                return torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous()) * z).flatten(-2)
            span = slice(first[b], first[b + 1])
            turned[:, span] = turn(q[:, span])
            for which, (cache, x) in enumerate(((k, turn(s["k_new"][:, span].double())), (v, s["v_new"][:, span].double()))):
                for lo in range(start // BLOCK * BLOCK, lengths[b], BLOCK):
                    p, i = table[b][lo // page], lo % page
                    rows = x[:, max(0, lo - start):max(0, lo - start) + min(BLOCK, lengths[b] - max(lo, start), lo + BLOCK - max(lo, start))]
                    at = max(lo, start) - lo
                    held = cache[:, p, :, i:i + BLOCK]
                    if scales is not None:
                        e = torch.ceil(torch.log2(rows.abs().amax((1, 3)) / 448.0)).clamp(min=LEAST)
                        if at:
                            was = scales[which][:, p, :, i // BLOCK] - 127
                            e = torch.maximum(e, was.double())
                            held[:, :, :at] *= torch.exp2(was - e)[..., None, None]
                        scales[which][:, p, :, i // BLOCK] = (e + 127).long()
                        rows = rows * torch.exp2(-e)[:, None, :, None]
                    held[:, :, at:at + rows.shape[1]] = rows.transpose(1, 2)
        out.update(q=turned, k=k, v=v)
        if scales is not None:
            out.update(k_scale=torch.exp2(scales[0].double() - 127), v_scale=torch.exp2(scales[1].double() - 127))
    if c["kind"] != "append":
        if c["kind"] == "step8":
            # attention reads what the append leaves: queries and cached numbers rounded to their types
            q = turned.to(BF).double()
            for n in ("k", "v"):
                s[n + "_cache"] = out[n].float().to(E4M3)
            s["k_scale"], s["v_scale"] = (x.to(torch.uint8) for x in scales)
        o = torch.zeros(s["o"].shape, dtype=F64, device=DEV)
        lse = torch.full(s["lse"].shape, -math.inf, dtype=F64, device=DEV)
        G = c["Hq"] // c["Hkv"]
        for l, d in enumerate(s["donor"]):
            i = s["owners"].index(d)
            for b, n in enumerate(lengths):
                if n == 0:
                    continue
                pages = torch.tensor(table[b][:(n + page - 1) // page], device=DEV)
                kv = []
                for name in ("k", "v"):
                    x = s[name + "_cache"][i].view(torch.uint8)[pages].view(E4M3).double()
                    x *= torch.exp2(s[name + "_scale"][i][pages].double() - 127).repeat_interleave(BLOCK, 2)[..., None]
                    kv.append(x.transpose(0, 1).flatten(1, 2)[:, :n])
                x = torch.einsum("hgd,hnd->hgn", q[l, b].unflatten(0, (c["Hkv"], G)), kv[0]) / math.sqrt(c["dh"])
                o[l, b] = torch.einsum("hgn,hnd->hgd", torch.softmax(x, -1), kv[1]).flatten(0, 1)
                lse[l, b] = torch.logsumexp(x, -1).flatten()
        out.update(o=o, lse=lse)
    return out
