"""Serving operators over the shared paged cache: attention of any number of new tokens a sequence (chunks of prompts, drafted
tokens, single tokens), with or without a sliding window and first tokens that stay visible, and the cache's pages: copied,
shared between sequences, handed out and taken back, freed behind a window, moved together.

  attend   the queries of new tokens, which are in the cache already, over all older tokens and the new ones up to their own:
           bf16 cache or 8 bits with a power of two for 16 tokens and KV head; a consumer layer reads its donor's pages
  window   the same where a token sees the last `window` tokens, its own among them, and the first `sinks`
  pages    refs[page] counts the places of the block table that hold a page; a page with 0 is free and pages are taken from
           the lowest number up, row by row.  Sequences fork by sharing pages; a row that grows inside a shared page gets a
           copy of it (but for the lowest of the rows that grow, where all that hold the page grow)

Sizes come from paper_2608_15943_b200/workloads.py, bench.py and the tests, or are generic.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 16                  # tokens that share a scale


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def _attend(name, L, B, new_lo, new_hi, old_lo, old_hi, Hq, Hkv, dh, page, pairs, bits=16, window=0, sinks=0, empty=0, pad=0):
    """new_lo..new_hi new tokens a sequence behind old_lo..old_hi older ones; the first `empty` places of the batch hold no
    sequence, `pad` rows stand behind the last one; the last 2 * pairs layers share in pairs (an even layer's K/V serves the
    odd layer above it); bits of a cached number: 16 or 8; window 0: everything older is seen."""
    return dict(name=name, kind="attend", L=L, B=B, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, Hq=Hq, Hkv=Hkv, dh=dh,
                page=page, pairs=pairs, bits=bits, window=window, sinks=sinks, empty=empty, pad=pad)


def _pages(name, kind, L, B, lo, hi, Hkv, dh, page, pairs, bits=16, width=1, kept=1, more=1):
    """B sequences of lo..hi tokens.
      copy      the pages of every sequence are copied to free ones, by a list
      beams     groups of `width` sequences that share their first half; each goes on from one of `kept` of its group, grows
                by `more` tokens and gives them back
      grow      every sequence grows by `more` tokens and gives them back
      turnover  half of the sequences end, the others' pages move together, new ones of the same lengths begin; then the
                other half"""
    return dict(name=name, kind=kind, L=L, B=B, lo=lo, hi=hi, Hkv=Hkv, dh=dh, page=page, pairs=pairs, bits=bits, width=width, kept=kept, more=more)


def listed():
    return [
        # a few tokens for each of two sequences of the tiny stack that an integration is checked with
        _attend("attend-tiny", 4, 2, 3, 5, 100, 140, 4, 2, 64, 16, 2),
        # drafted tokens of a serving batch are verified
        _attend("attend-drafts", 4, 16, 2, 8, 4000, 16000, 32, 8, 128, 64, 2),
        # the same over the 8-bit cache, in a padded batch
        _attend("attend8-drafts", 4, 19, 2, 8, 4000, 16000, 32, 8, 128, 64, 2, bits=8, empty=3, pad=37),
        # pieces of prompts of no round length behind what is cached of them
        _attend("attend-chunks", 4, 4, 900, 2200, 2000, 8000, 32, 8, 128, 128, 1),
        # the same over the 8-bit cache, small heads, small pages
        _attend("attend8-chunks", 4, 5, 700, 1500, 1000, 5000, 24, 8, 64, 48, 1, bits=8),
        # the last piece of a very long prompt, the largest call
        _attend("attend-chunk-64k", 2, 1, 8192, 8192, 65536, 65536, 32, 8, 128, 128, 1),
        # a token step of long sequences that see a window and a few first tokens
        _attend("window-tokens", 8, 32, 1, 1, 16384, 32767, 32, 8, 128, 128, 2, window=4096, sinks=4),
        # the same in 8 bits: a smaller model, contexts on both sides of the window
        _attend("window8-tokens", 6, 58, 1, 1, 1, 3000, 12, 4, 64, 32, 2, bits=8, window=1000, sinks=8, empty=3),
        # long prompts under a window
        _attend("window-prompts", 4, 3, 4000, 7000, 0, 0, 32, 8, 128, 128, 2, window=2048, sinks=16),
        # beam search: beams fork within their request, and the forks' last pages are copied as they grow
        _pages("pages-beams", "beams", 8, 64, 1500, 3000, 8, 128, 128, 2, width=4, kept=2),
        # a token step of a serving batch asks for room, and drafts are given back
        _pages("pages-grow", "grow", 4, 32, 300, 1500, 2, 64, 16, 2, bits=8, more=5),
        # sequences end and begin, the pool is kept dense
        _pages("pages-turnover", "turnover", 6, 24, 500, 3000, 8, 128, 64, 1, bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "window", "window", "copy", "beams", "grow", "turnover"))
    dh, Hkv, G = rng.choice((64, 128, 128)), rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 7, 8))
    L, page, bits = rng.randint(1, 8), rng.choice((16, 32, 48, 64, 128)), rng.choice((16, 16, 8))
    pairs = rng.randint(0, L // 2)
    if kind in ("attend", "window"):
        hi, old = rng.choice((1, _log_int(rng, 2, 16), _log_int(rng, 16, 8192))), rng.choice((0, _log_int(rng, 1, 70000)))
        c = _attend("", L, _log_int(rng, 1, 64), (hi + 1) // 2, hi, old // 2, old, Hkv * G, Hkv, dh, page, pairs, bits,
                    pad=rng.choice((0, 0, rng.randint(1, 300))) if hi > 1 else 0)
        if kind == "window":
            c["window"], c["sinks"] = _log_int(rng, 1, 8192), rng.choice((0, 1, 4, rng.randint(5, 200)))
        c["empty"] = rng.choice((0, 0, c["B"] // 4))
        while work(c)["flops"] > 4e12 or work(c)["bytes"] > 8e9 or _pool_bytes(c) > 4e9:
            c["B"] = max(1, c["B"] // 2)
            c["empty"] = min(c["empty"], c["B"] // 4)
            for k in ("new_lo", "new_hi", "old_lo", "old_hi"):
                c[k] = max(1 if k.startswith("new") else 0, c[k] * 3 // 4)
    else:
        lo = _log_int(rng, 2 * page, 6000)
        width = rng.choice((2, 3, 4, 8)) if kind == "beams" else 1
        c = _pages("", kind, L, width * _log_int(rng, 1 if kind == "beams" else 2, 64), lo, int(lo * rng.uniform(1.0, 2.0)), Hkv, dh, page, pairs, bits,
                   width, rng.randint(1, width), rng.choice((1, 1, rng.randint(2, 3 * page))))
        while _pool_bytes(c) > 1.5e9:
            c["B"] = max(2, c["width"], c["B"] // 2 // c["width"] * c["width"])
            c["lo"], c["hi"] = max(2 * page, c["lo"] * 3 // 4), max(2 * page, c["hi"] * 3 // 4)
    del c["name"]
    return c


def _donors(c):
    first = c["L"] - 2 * c["pairs"]
    return [l if l < first or (l - first) % 2 == 0 else l - 1 for l in range(c["L"])]


def _owners(c):
    return [l for l, d in enumerate(_donors(c)) if d == l]


def _pool_bytes(c):
    longest = c["new_hi"] + c["old_hi"] if c["kind"] == "attend" else c["hi"] + c["more"]
    copies = 2 if c["kind"] == "copy" else 1
    return len(_owners(c)) * copies * c["B"] * (longest + c["page"]) * 2 * c["Hkv"] * c["dh"] * c["bits"] // 8


def _spread(host, n, lo, hi):
    """n numbers from lo to hi, any of them, whose sum is always the same."""
    x = [host.randint(lo, hi) for _ in range(n)]
    off = n * (lo + hi) // 2 - sum(x)
    for i in host.sample(range(n), n):
        step = max(lo, min(hi, x[i] + off)) - x[i]
        x[i], off = x[i] + step, off - step
    return x


# ---------------------------------------------------------------------------------------------
# states
# ---------------------------------------------------------------------------------------------
def _pool(c, n_pages, g):
    """Pools of all owners, numbers ~ N(0, 1): in 8 bits, blocks whose largest is about 4 have the scale 2^-6."""
    n_own, bits = len(_owners(c)), c["bits"]
    s = {}
    for name in ("k", "v"):
        p = torch.empty(n_own, n_pages, c["Hkv"], c["page"], c["dh"], dtype=BF if bits == 16 else E4M3, device=DEV)
        for layer in p:
            layer.copy_(torch.randn(n_pages, c["Hkv"], c["page"], c["dh"], device=DEV, dtype=BF, generator=g) * (1.0 if bits == 16 else 64.0))
        s[name + "_cache"] = p
    if bits == 8:
        for name in ("k", "v"):
            s[name + "_scale"] = torch.randint(120, 123, (n_own, n_pages, c["Hkv"], c["page"] // BLOCK), device=DEV, dtype=torch.uint8, generator=g)
    return s


def prepare(case, seed):
    host, g = random.Random(seed), torch.Generator(device=DEV).manual_seed(seed)
    return (_prepare_attend if case["kind"] == "attend" else _prepare_pages)(case, host, g)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_attend(c, host, g):
    L, B, Hq, dh, page, empty = (c[k] for k in ("L", "B", "Hq", "dh", "page", "empty"))
    live = B - empty
    new = [0] * empty + _spread(host, live, c["new_lo"], c["new_hi"])
    lengths = [n + o for n, o in zip(new, [0] * empty + _spread(host, live, c["old_lo"], c["old_hi"]))]
    one_each = c["new_hi"] == 1
    # the pages of the sequences lie scattered over the pool; the table has room for them to grow
    most = max(1, (c["new_hi"] + c["old_hi"] + page - 1) // page)
    n_pages, max_pages = B * most + 1, most + 2
    order = list(range(n_pages))
    host.shuffle(order)
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate((x + page - 1) // page for x in lengths):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    first = [0]
    for n in ([1] * B if one_each else new):
        first.append(first[-1] + n)
    T = first[-1] + c["pad"]
    s = dict(case=c, donor=_donors(c), owners=_owners(c), n_pages=n_pages, max_pages=max_pages, one_each=one_each, table=table.to(DEV),
             lengths=_int32(lengths), first=_int32(first), spans=[(first[b] + (1 - n if one_each else 0), n, lengths[b]) for b, n in enumerate(new)],
             **_pool(c, n_pages, g))
    s["q"] = torch.randn(L, T, Hq, dh, device=DEV, dtype=BF, generator=g)
    s["o"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(L, T, Hq, dtype=F32, device=DEV)
    return s


def _prepare_pages(c, host, g):
    kind, B, page, width = c["kind"], c["B"], c["page"], c["width"]
    groups = B // width
    lengths = [n for n in _spread(host, groups, c["lo"], c["hi"]) for _ in range(width)]
    if kind == "beams":                                   # (the last page is neither full nor empty)
        lengths = [n if n % page else n + 1 for n in lengths]
    max_pages = (c["hi"] + c["more"] + page) // page + 2
    need = [(n + page - 1) // page for n in lengths]
    shared = [n // 2 // page if kind == "beams" else 0 for n in lengths]
    used = sum(need) - sum(shared) + sum(shared[::width])
    most, half = (c["hi"] + page) // page, c["hi"] // 2 // page if kind == "beams" else 0
    n_pages = groups * (half + width * (most - half + 1))                   # (by the longest sequences: the same for any seed)
    n_pages += {"copy": n_pages, "beams": B * (2 + c["more"] // page), "grow": B * (2 + c["more"] // page), "turnover": 3}[kind]
    order = list(range(n_pages))
    rows = list(range(B))
    if kind == "turnover":                                # (as the last turn left it: dense, the first half's pages in front)
        rows = rows[::2] + rows[1::2]
    else:
        host.shuffle(order)
    table, refs, at = [[-1] * max_pages for _ in range(B)], [0] * n_pages, 0
    for b in rows:
        for i in range(need[b]):
            if i < shared[b] and b % width:
                table[b][i] = table[b - b % width][i]
            else:
                table[b][i], at = order[at], at + 1
            refs[table[b][i]] += 1
    s = dict(case=c, donor=_donors(c), owners=_owners(c), n_pages=n_pages, max_pages=max_pages, table=_int32(table), refs=_int32(refs),
             lengths=_int32(lengths), count=_int32([0]), **_pool(c, n_pages, g))
    stay = list(range(B))
    if kind == "copy":
        s["src"], s["dst"] = _int32(order[:used]), _int32(order[used:2 * used])
    else:
        s["back"], s["grown"] = _int32(lengths), _int32([n + c["more"] for n in lengths])
    if kind == "beams":
        parent = []
        for first in range(0, B, width):
            kept = host.sample(range(first, first + width), c["kept"])
            kept += [host.choice(kept) for _ in range(width - len(kept))]
            host.shuffle(kept)
            parent += kept
        s["parent"] = _int32(parent)
    if kind == "turnover":
        s["parent"] = [_int32([-1 if b % 2 == half else b for b in stay]) for half in (0, 1)]
    return s


def run(state):
    kind = state["case"]["kind"]
    if kind == "attend":
        (_own_attend if own else _plain_attend)(state)
        return dict(o=state["o"], lse=state["lse"])
    do = _Own(state) if own else _Plain(state)
    if kind == "copy":
        do.copy(state["src"], state["dst"])
    elif kind == "turnover":
        for parent in state["parent"]:
            do.fork(parent)
            do.compact()
            do.resize(state["back"])
    else:
        if kind == "beams":
            do.fork(state["parent"])
        do.resize(state["grown"])
        do.resize(state["back"])
    out = dict(refs=state["refs"], table=state["table"], lengths=state["lengths"], count=state["count"], k=state["k_cache"], v=state["v_cache"])
    if "k_scale" in state:
        out.update(k_scale=state["k_scale"].view(E8M0), v_scale=state["v_scale"].view(E8M0))
    return out


# ---------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------
def _handle(s):
    """What a serving program keeps from step to step: the description of its cache, the workspace, the lists of layers."""
    if "handle" not in s:
        from paper_2608_15943_b200 import kvp
        c, own_at = s["case"], {l: i for i, l in enumerate(s["owners"])}
        desc = kvp.DecodeDesc(c["L"], s["table"].shape[0], c.get("Hq", c["Hkv"]), c["Hkv"], c["dh"], c["page"], s["max_pages"], s["n_pages"])
        at = {k: [s[k][own_at[l]] if l in own_at else None for l in range(c["L"])] for k in ("k_cache", "v_cache", "k_scale", "v_scale") if k in s}
        at.update({k: list(s[k]) for k in ("q", "o", "lse") if k in s})
        size = kvp.attn_chunk_workspace_bytes(desc, s["donor"], s["q"].shape[1]) if c["kind"] == "attend" else kvp.pages_workspace_bytes(desc)
        s["handle"] = (kvp, desc, at, torch.empty(max(256, size), dtype=torch.uint8, device=DEV))
    return s["handle"]


def _own_attend(s):
    kvp, desc, at, ws = _handle(s)
    c = s["case"]
    kvp.attn_chunk(desc, s["donor"], at["q"], at["k_cache"], at["v_cache"], s["table"], s["lengths"], at["o"], at["lse"], ws,
                   first=None if s["one_each"] else s["first"], window=c["window"], sinks=c["sinks"], k_scale=at.get("k_scale"), v_scale=at.get("v_scale"))


class _Own:
    def __init__(self, s):
        self.kvp, self.desc, at, self.ws = _handle(s)
        self.s, self.pools = s, (at["k_cache"], at["v_cache"], at.get("k_scale"), at.get("v_scale"))

    def copy(self, src, dst):
        self.kvp.pages_copy(self.desc, self.s["donor"], src, dst, *self.pools)

    def fork(self, parent):
        s = self.s
        self.kvp.pages_fork(self.desc, parent, s["refs"], s["table"], s["lengths"], self.ws)

    def resize(self, lengths):
        s = self.s
        self.kvp.pages_resize(self.desc, s["donor"], lengths, s["refs"], s["table"], s["lengths"], s["count"], self.ws, *self.pools)

    def compact(self):
        s = self.s
        self.kvp.pages_compact(self.desc, s["donor"], s["refs"], s["table"], s["lengths"], s["count"], self.ws, *self.pools)


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _power(byte):
    """2^(byte - 127), exactly."""
    return (byte.int() << 23).view(F32)


def _rows(s, name, i, pages):
    """[Hkv, tokens, dh] in 32 bits from the pages [P] of owner i's pool."""
    x = s[name + "_cache"][i]
    if name + "_scale" in s:
        x = x.view(torch.uint8)[pages].view(E4M3).float().unflatten(-2, (-1, BLOCK)) * _power(s[name + "_scale"][i][pages])[..., None, None]
        x = x.flatten(-3, -2)
    else:
        x = x[pages].float()
    return x.transpose(0, 1).flatten(1, 2)


def _plain_attend(s):
    c = s["case"]
    Hkv, G, dh, page = c["Hkv"], c["Hq"] // c["Hkv"], c["dh"], c["page"]
    for i, l in enumerate(s["owners"]):
        members = [m for m, d in enumerate(s["donor"]) if d == l]
        for b, (at, n, length) in enumerate(s["spans"]):
            if n == 0:
                continue
            old = length - n
            pages = s["table"][b, :(length + page - 1) // page].long()
            if c["window"]:
                # the pages that some row sees: the first tokens', and from the first row's window on
                lo = max(0, old - c["window"] + 1) // page
                which = torch.arange(len(pages), device=DEV)
                which = torch.cat((which[:min(lo, (c["sinks"] + page - 1) // page)], which[lo:]))
                pages, key = pages[which], (which[:, None] * page + torch.arange(page, device=DEV)).flatten()
            else:
                key = torch.arange(len(pages) * page, device=DEV)
            k, v = _rows(s, "k", i, pages), _rows(s, "v", i, pages)
            step = max(1, 2 ** 28 // (len(members) * c["Hq"] * len(key)))
            for r in range(0, n, step):
                m = min(step, n - r)
                pos = torch.arange(old + r, old + r + m, device=DEV)[:, None]
                unseen = key > pos
                if c["window"]:
                    unseen |= (key <= pos - c["window"]) & (key >= c["sinks"])
                q = s["q"][members, at + r:at + r + m].float().unflatten(2, (Hkv, G)).permute(2, 0, 3, 1, 4)      # [Hkv, members, G, m, dh]
                x = (q.flatten(1, 3) @ k.transpose(1, 2)).unflatten(1, (-1, m)).mul_(dh ** -0.5).masked_fill_(unseen, -math.inf)
                most = x.amax(-1, keepdim=True)
                p = x.sub_(most).exp_()
                total = p.sum(-1, keepdim=True)
                o = (p.flatten(1, 2) @ v).unflatten(1, (-1, m)) / total
                s["o"][members, at + r:at + r + m] = o.unflatten(1, (-1, G)).permute(1, 3, 0, 2, 4).flatten(2, 3).to(BF)
                s["lse"][members, at + r:at + r + m] = (most + total.log()).squeeze(-1).unflatten(1, (-1, G)).permute(1, 3, 0, 2).flatten(2, 3)


class _Plain:
    def __init__(self, s):
        self.s, self.page = s, s["case"]["page"]
        self.place = torch.arange(s["max_pages"], device=DEV)

    def _count(self, lengths):
        return (lengths.long() + self.page - 1) // self.page

    def _refs(self, held):
        """How often each page is held, of the places [B, max_pages] with -1 where there is none."""
        n = self.s["n_pages"]
        return torch.zeros(n + 1, dtype=torch.int32, device=DEV).index_add_(0, torch.where(held < 0, n, held).flatten().long(),
                                                                            torch.ones(held.numel(), dtype=torch.int32, device=DEV))[:n]

    def _held(self, table, lengths):
        return torch.where(self.place < self._count(lengths)[:, None], table, -1)

    def copy(self, src, dst):
        src, dst = src.long(), dst.long()
        for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
            if name in self.s:
                pool = self.s[name].view(torch.uint8) if self.s[name].dtype == E4M3 else self.s[name]
                for layer in pool:
                    layer[dst] = layer[src]

    def fork(self, parent):
        s = self.s
        row = torch.arange(len(parent), device=DEV)
        src = torch.where((parent >= 0) & (parent < len(parent)), parent.long(), row)
        before = self._held(s["table"], s["lengths"])
        lengths = torch.where(parent == -1, 0, s["lengths"][src])
        after = torch.where(self.place < self._count(lengths)[:, None], before[src], -1)
        table = torch.where(self.place < torch.maximum(self._count(s["lengths"]), self._count(lengths))[:, None], after, s["table"])
        s["refs"] += self._refs(after) - self._refs(before)
        s["table"].copy_(table)
        s["lengths"].copy_(lengths)

    def resize(self, lengths):
        s, page = self.s, self.page
        refs, table = s["refs"], s["table"]
        B, row = len(lengths), torch.arange(len(lengths), device=DEV)
        had, have = self._count(s["lengths"]), self._count(lengths)
        last = table[row, (had - 1).clamp(min=0)].long()
        inside = (lengths > s["lengths"]) & (s["lengths"] % page != 0) & (last >= 0)           # grows in a page that it has
        same = (last[:, None] == last) & inside[:, None] & inside
        keeps = (same.sum(1) == refs[last.clamp(min=0)]) & (torch.where(same, row, B).amin(1) == row)
        copies = inside & (refs[last.clamp(min=0)] > 1) & ~keeps
        need = (have - had).clamp(min=0) + copies
        begin = need.cumsum(0) - need
        free = refs == 0
        lacking = (need.sum() - free.sum()).clamp(min=0)
        s["count"].copy_(lacking)
        if lacking:
            return
        order = torch.argsort((~free).int(), stable=True).int()                                # free pages, lowest first
        # the place of each row's i-th new page: the copy's, then those behind its last
        new = order[(begin[:, None] + copies[:, None] + self.place - had[:, None]).clamp(0, len(order) - 1)]
        held = self._held(table, s["lengths"])
        after = torch.where((self.place >= had[:, None]) & (self.place < have[:, None]), new, held)
        to = order[begin.clamp(max=len(order) - 1)]
        after = torch.where(copies[:, None] & (self.place == had[:, None] - 1), to[:, None], after)
        after = torch.where(self.place < have[:, None], after, -1)
        self.copy(last[copies], to[copies])
        refs += self._refs(after) - self._refs(held)
        s["table"].copy_(torch.where(self.place < torch.maximum(had, have)[:, None], after, table))
        s["lengths"].copy_(lengths)

    def compact(self):
        s = self.s
        refs, table, number = s["refs"], s["table"], torch.arange(s["n_pages"], device=DEV)
        used = (refs > 0).sum()
        s["count"].copy_(used)
        src, dst = number[(refs > 0) & (number >= used)], number[(refs == 0) & (number < used)]
        to = number.index_copy(0, src, dst)
        self.copy(src, dst)
        held = self._held(table, s["lengths"])
        s["table"].copy_(torch.where(held >= 0, to[held.clamp(min=0).long()].int(), table))
        refs[dst] = refs[src]
        refs[src] = 0


# ---------------------------------------------------------------------------------------------
# work and 64-bit values
# ---------------------------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once.  Attention reads the cached numbers and scales that some row of a
    sequence sees once for a donor and all its consumers, and queries; pages that move are read and written once."""
    c = case
    n_own, nkv = len(_owners(c)), c["Hkv"] * c["dh"]
    cached = 2.0 if c["bits"] == 16 else 1.0 + 1.0 / (BLOCK * c["dh"])
    if c["kind"] == "attend":
        live, nq = c["B"] - c["empty"], c["Hq"] * c["dh"]
        n, old = (c["new_lo"] + c["new_hi"]) / 2, (c["old_lo"] + c["old_hi"]) / 2
        W, sinks = c["window"], c["sinks"]
        if W:
            free = min(n, max(0.0, W + sinks - old))             # rows that see everything older
            seen = free * (old + (free + 1) / 2) + (n - free) * (W + sinks)
            tokens = min(old + n, W + n - 1 + sinks)
        else:
            seen, tokens = n * (old + (n + 1) / 2), old + n
        nbytes = live * (n_own * tokens * 2 * nkv * cached + c["L"] * n * (2 * nq * 2 + c["Hq"] * 4))
        return {"bytes": nbytes, "flops": c["L"] * live * seen * 4 * nq}
    page = c["page"]
    mean = (c["lo"] + c["hi"]) / 2
    per_row = (mean + page / 2) / page
    moved = {"copy": c["B"] * per_row, "beams": c["B"] / c["width"] * (c["width"] - c["kept"]), "grow": 0.0, "turnover": 2 * (c["B"] // 2) * per_row}[c["kind"]]
    table = {"copy": 0.0, "beams": 2 * per_row, "grow": 2 * c["more"] / page + 2, "turnover": 3 * per_row}[c["kind"]]
    return {"bytes": 2 * moved * n_own * 2 * page * nkv * cached + 4 * c["B"] * (table + 4), "flops": 0.0}


def exact(case, seed):
    """From the definitions in 64 bits, sequence by sequence and head by head; the pages' bookkeeping in Python's numbers."""
    c, s = case, prepare(case, seed)
    return (_exact_attend if c["kind"] == "attend" else _exact_pages)(c, s)


def _exact_attend(c, s):
    o, lse = s["o"].double(), s["lse"].double()
    G, page, table = c["Hq"] // c["Hkv"], c["page"], s["table"].tolist()
    for l, d in enumerate(s["donor"]):
        i = s["owners"].index(d)
        for b, (at, n, length) in enumerate(s["spans"]):
            for h in range(c["Hkv"] if n else 0):
                kv = []
                for name in ("k", "v"):
                    x = torch.cat([s[name + "_cache"][i, p, h].double() for p in table[b][:(length + page - 1) // page]])
                    if name + "_scale" in s:
                        e = torch.cat([s[name + "_scale"][i, p, h].double() for p in table[b][:(length + page - 1) // page]])
                        x *= torch.exp2(e - 127.0).repeat_interleave(BLOCK)[:, None]
                    kv.append(x[:length])
                for r in range(0, n, 4096):
                    m = min(4096, n - r)
                    pos, key = torch.arange(length - n + r, length - n + r + m, device=DEV), torch.arange(length, device=DEV)
                    seen = key[None, :] <= pos[:, None]
                    if c["window"]:
                        seen &= (pos[:, None] - key[None, :] < c["window"]) | (key < c["sinks"])
                    span = slice(at + r, at + r + m)
                    for g in range(h * G, h * G + G):
                        x = torch.where(seen, s["q"][l, span, g].double() @ kv[0].T / math.sqrt(c["dh"]), -math.inf)
                        o[l, span, g] = torch.softmax(x, -1) @ kv[1]
                        lse[l, span, g] = torch.logsumexp(x, -1)
    return dict(o=o, lse=lse)


def _exact_pages(c, s):
    page, n_pages = c["page"], s["n_pages"]
    refs, table, lengths = s["refs"].tolist(), s["table"].tolist(), s["lengths"].tolist()
    content = list(range(n_pages))                         # whose first content a page has now
    count = 0

    def places(n):
        return -(-n // page)

    def fork(parent):
        nonlocal table, lengths
        then, was = [list(t) for t in table], list(lengths)
        for b, p in enumerate(parent):
            if p == b:
                continue
            for i in range(places(was[b])):
                if then[b][i] >= 0:
                    refs[then[b][i]] -= 1
                table[b][i] = -1
            lengths[b] = was[p] if p >= 0 else 0
            for i in range(places(lengths[b])):
                table[b][i] = then[p][i]
                if then[p][i] >= 0:
                    refs[then[p][i]] += 1

    def resize(to):
        nonlocal count
        free = [p for p in range(n_pages) if refs[p] == 0]
        holds = list(refs)
        ends = [table[b][places(n) - 1] if n % page and to[b] > n else -1 for b, n in enumerate(lengths)]
        copies = [p >= 0 and holds[p] > 1 and not (ends.count(p) == holds[p] and ends.index(p) == b) for b, p in enumerate(ends)]
        need = sum(copies) + sum(max(0, places(to[b]) - places(n)) for b, n in enumerate(lengths))
        count = max(0, need - len(free))
        if count:
            return
        for b, n in enumerate(lengths):
            if copies[b]:
                p = free.pop(0)
                content[p] = content[ends[b]]
                refs[ends[b]] -= 1
                refs[p], table[b][places(n) - 1] = 1, p
            for i in range(places(n), places(to[b])):
                table[b][i] = free.pop(0)
                refs[table[b][i]] = 1
            for i in range(places(to[b]), places(n)):
                if table[b][i] >= 0:
                    refs[table[b][i]] -= 1
                table[b][i] = -1
            lengths[b] = to[b]

    def compact():
        nonlocal count
        count = sum(r > 0 for r in refs)
        holes = [p for p in range(count) if refs[p] == 0]
        to = {p: holes.pop(0) for p in range(count, n_pages) if refs[p]}
        for p, h in to.items():
            content[h], refs[h], refs[p] = content[p], refs[p], 0
        for b, n in enumerate(lengths):
            for i in range(places(n)):
                table[b][i] = to.get(table[b][i], table[b][i])

    if c["kind"] == "copy":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            content[b] = a
    elif c["kind"] == "turnover":
        for parent in s["parent"]:
            fork(parent.tolist())
            compact()
            resize(s["back"].tolist())
    else:
        if c["kind"] == "beams":
            fork(s["parent"].tolist())
        resize(s["grown"].tolist())
        resize(s["back"].tolist())
    at = torch.tensor(content, device=DEV)
    out = {n: _int32(x) for n, x in (("refs", refs), ("table", table), ("lengths", lengths), ("count", [count]))}
    for n in ("k", "v"):
        pool = s[n + "_cache"]
        out[n] = (pool.view(torch.uint8)[:, at].view(E4M3) if pool.dtype == E4M3 else pool[:, at]).double()
        if n + "_scale" in s:
            out[n + "_scale"] = torch.exp2(s[n + "_scale"][:, at].double() - 127)
    return out
