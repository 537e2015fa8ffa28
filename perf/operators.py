"""Cases of the cache operators: windowed attention for prompts, and a paged cache with what writes it, reads it and
evicts from it.

A case has a "kind":

  window     mone_window_attention: a prompt's tokens over the first n_sink positions (a memory's tokens, say) and a
             sliding window of the positions up to their own, in a dense cache.
  attention  mone_cache_attention: one or a few new tokens over a paged cache, with the weights that each position gets
             added up for a later eviction, or without.
  evict      mone_cache_evict: a cache cut down to its first positions, its last ones and those of the highest weights,
             compacted into fresh pages.
  append     mone_cache_append: new tokens' keys and values into the pages.

Sizes are those of the repository's workloads (16 layers with 8 KV heads of 64, 28 layers with 8 of 128, 8 contexts, a
memory of 64 tokens, contexts of 32K and 128K) and generic ones around them.  `run` computes them with elementary torch
operations in 32 bits, or, where `own` is true, through the library.
"""
import math

import torch

own = False
DEV = "cuda"
ALL = 1 << 30  # a window that hides nothing
BASE = dict(n_ctx=1, n_layers=1, n_kv=8, n_q=32, hd=64, dtype="bf16")
PAGED = dict(BASE, page=64, order="head", n_sink=0, window=ALL)


def listed():
    return [
        # the smallest prompt: a chat turn of 64 tokens behind a memory of 64, one layer of a backbone that runs layer by layer
        dict(BASE, name="window_turn", kind="window", Lq=64, n_past=64, n_sink=64, window=128),
        # a 2K prompt behind a memory, every layer at once
        dict(BASE, name="window_l16_2k", kind="window", n_layers=16, Lq=2048, n_past=64, n_sink=64, window=512),
        # the last chunk of a long document, odd lengths, one layer with heads of 128: the largest prompt
        dict(BASE, name="window_16k_chunk", kind="window", hd=128, Lq=16001, n_past=5003, n_sink=4, window=4096),
        # fp32, as a run that checks numerics has it
        dict(BASE, name="window_f32", kind="window", n_layers=2, n_kv=4, n_q=8, Lq=700, n_past=33, n_sink=16, window=200, dtype="f32"),
        # the first token after a short prompt, one layer: latency
        dict(PAGED, name="token_first", kind="attention", n_tok=1, length=150, page=16, score=False),
        # decode over 1K positions, every layer, weights added up
        dict(PAGED, name="token_l16_1k", kind="attention", n_layers=16, n_tok=1, length=1151, score=True),
        # a batch of 16 conversations of very unequal length, one layer, pages of 32, weights added up
        dict(PAGED, name="token_batch16", kind="attention", n_ctx=16, hd=128, n_tok=1, length=32768, page=32, score=True),
        # a context of 128K in four layers, two new tokens: the most that is read
        dict(PAGED, name="token_128k", kind="attention", n_layers=4, hd=128, n_tok=2, length=131072, score=False),
        # half of a 2K cache goes, every layer
        dict(PAGED, name="evict_l16_2k", kind="evict", n_layers=16, length=2048, keep=1024, n_sink=4, n_recent=128),
        # eight contexts of up to 32K cut to 8K, one layer
        dict(PAGED, name="evict_ctx8_32k", kind="evict", n_ctx=8, hd=128, page=32, length=32768, keep=8192, n_sink=64, n_recent=1000),
        # one new token for each of eight contexts, one layer: latency
        dict(PAGED, name="append_token", kind="append", n_ctx=8, page=16, length=3000, n_tok=1),
        # a 2K prompt into the pages of 16 layers
        dict(PAGED, name="append_l16_2k", kind="append", n_layers=16, length=64, n_tok=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window", "window", "attention", "attention", "attention", "evict", "append"])
    n_kv = rng.choice([1, 2, 4, 8])
    c = dict(kind=kind, n_ctx=rng.choice([1, 1, 2, 5, 16]), n_layers=rng.choice([1, 1, 2, 16]), n_kv=n_kv,
             n_q=n_kv * rng.choice([1, 2, 4, 5, 8]), hd=rng.choice([64, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if kind == "window":
        c.update(Lq=_log(rng, 2, 8000), n_past=_log(rng, 1, 6000), n_sink=rng.choice([0, 4, 64, 300]), window=_log(rng, 1, 5000))
        if c["dtype"] == "f32":
            c.update(Lq=min(c["Lq"], 1500), window=min(c["window"], 600), n_layers=1)
        most = ("Lq", dict(flops=2e10 if c["dtype"] == "f32" else 4e11, bytes=1e9))
    else:
        c.update(page=rng.choice([8, 16, 32, 64, 128]), order=rng.choice(["head", "position"]), n_sink=rng.choice([0, 4, 64]),
                 length=_log(rng, 40, 60000))
        most = ("length", dict(flops=4e10, bytes=1.2e9))
        if kind == "attention":
            c.update(n_tok=rng.choice([1, 1, 1, 2, 5]), score=rng.random() < 0.5, window=rng.choice([ALL, ALL, _log(rng, 1, 20000)]))
        elif kind == "evict":
            c.update(keep=max(1, int(c["length"] * rng.uniform(0.1, 0.9))), window=ALL)
            c["n_sink"] = min(c["n_sink"], c["keep"] // 2)
            c["n_recent"] = rng.randint(0, c["keep"] - c["n_sink"])
        else:
            c.update(n_tok=_log(rng, 1, 4000), window=ALL)
            c["length"] = min(c["length"], 8000)
    while any(work(c)[k] > v for k, v in most[1].items()) or _pool_bytes(c) > 3e9:
        c[most[0]] = c[most[0]] // 2 + 1
        for k in ("keep", "n_recent", "n_sink"):
            if kind == "evict":
                c[k] = c[k] // 2 + (k == "keep")
        if kind == "append":
            c["n_tok"] = c["n_tok"] // 2 + 1
    return c


# ------------------------------------------------------------------ sizes and work

def lengths(c):
    """Positions that each context holds before the call: `length` alone, or a spread up to it."""
    n = c["n_ctx"]
    return [max(1, int(c["length"] * ((i * 7 + n - 1) % n + 1) ** 2 / n ** 2)) for i in range(n)] if n > 1 else [c["length"]]


def _width(c):
    """Entries of a context's page table: what the longest needs, and one spare."""
    return -(-(c["length"] + (c["n_tok"] if c["kind"] == "append" else 0)) // c["page"]) + 1


def _pages(c):
    """Pages of a layer's pool: every context's own, fresh ones for the survivors of an eviction, and some that nobody has."""
    return c["n_ctx"] * (_width(c) + (-(-c["keep"] // c["page"]) if c["kind"] == "evict" else 0)) + 5


def _pool_bytes(c):
    el = 4 if c["dtype"] == "f32" else 2
    return 0 if c["kind"] == "window" else 2 * el * c["n_layers"] * _pages(c) * c["page"] * c["n_kv"] * c["hd"]


def _seen(t, c):
    """Positions that the token at position t sees."""
    lo = max(0, t - c["window"] + 1)
    return t + 1 - lo + min(lo, c["n_sink"]) if t >= 0 else 0


def _union(t0, t1, c):
    """Positions that some token at t0 .. t1 sees."""
    lo = max(0, t0 - c["window"] + 1)
    return t1 + 1 - lo + min(lo, c["n_sink"]) if t1 >= 0 else 0


def work(c):
    el, hd, L = 4 if c["dtype"] == "f32" else 2, c["hd"], c["n_layers"]
    if c["kind"] == "window":
        pairs = sum(_seen(c["n_past"] + i, c) for i in range(c["Lq"]))
        read = _union(c["n_past"], c["n_past"] + c["Lq"] - 1, c)
        return {"bytes": el * hd * (2 * c["n_q"] * c["Lq"] + 2 * c["n_kv"] * read) * L * c["n_ctx"],
                "flops": 4 * hd * c["n_q"] * pairs * L * c["n_ctx"]}
    if c["kind"] == "append":
        return {"bytes": c["n_ctx"] * L * c["n_kv"] * c["n_tok"] * (4 * el * hd + 4), "flops": 0}
    if c["kind"] == "evict":
        kept = [min(n, c["keep"]) for n in lengths(c)]
        return {"bytes": L * c["n_kv"] * (4 * sum(lengths(c)) + sum(kept) * (4 * el * hd + 8)), "flops": 0}
    read = sum(_union(n - c["n_tok"], n - 1, c) for n in lengths(c))
    pairs = sum(_seen(n - 1 - i, c) for n in lengths(c) for i in range(c["n_tok"]))
    per = 2 * el * hd + (8 if c["score"] else 0)
    return {"bytes": L * (c["n_kv"] * read * per + 2 * el * hd * c["n_ctx"] * c["n_q"] * c["n_tok"]),
            "flops": 4 * hd * c["n_q"] * pairs * L}


# ------------------------------------------------------------------ what a program has in hand

def _inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    B, L, n_kv, n_q, hd = c["n_ctx"], c["n_layers"], c["n_kv"], c["n_q"], c["hd"]
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    if c["kind"] == "window":
        S = c["n_past"] + c["Lq"]
        return {"q": 2 * rn(B, L, n_q, c["Lq"], hd), "k": rn(B, L, n_kv, S, hd), "v": rn(B, L, n_kv, S, hd)}
    P, page, W = _pages(c), c["page"], _width(c)
    lens = torch.tensor(lengths(c), dtype=torch.int32, device=DEV)
    if c["order"] == "head":  # a page holds its heads' positions one head after the other
        K, V = (rn(L, P, n_kv, page, hd) for _ in range(2))
    else:                     # position after position
        K, V = (rn(L, P, page, n_kv, hd).transpose(2, 3) for _ in range(2))
    order = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    held = lens + (c["n_tok"] if c["kind"] == "append" else 0)
    table = order[:B * W].view(B, W).clone()
    table[torch.arange(W, device=DEV)[None, :] * page >= held[:, None]] = -1  # no page yet
    d = {"K": K, "V": V, "table": table, "lens": lens}
    if c["kind"] == "attention":
        d["q"] = 2 * rn(B, L, n_q, c["n_tok"], hd)
    if c["kind"] == "append":
        d["k"], d["v"] = (rn(B, L, n_kv, c["n_tok"], hd) for _ in range(2))
    if c["kind"] == "evict" or c.get("score"):  # weights as a softmax over the cache leaves them: a few large, most small
        w = torch.randn(B, L, n_kv, W * page, generator=g, device=DEV)
        d["score"] = torch.exp(2 * w) / c["length"]
    if c["kind"] == "evict":
        n = -(-c["keep"] // page)
        d["to"] = order[B * W:B * W + B * n].view(B, n).clone()
        d["to_score"] = torch.zeros(B, L, n_kv, n * page, device=DEV)
    return d


class Program:
    """Inputs, and for the library a handle and the buffers that a program keeps."""

    def __init__(self, c, seed):
        self.c, self.h = c, None
        self.d = _inputs(c, seed)
        if not own:
            return
        import paper_2608_17616_gb300 as mone
        self.mone = mone
        B, L, n_kv, hd = c["n_ctx"], c["n_layers"], c["n_kv"], c["hd"]
        d_out, dt = 2 * n_kv * hd, mone.MONE_FP32 if c["dtype"] == "f32" else mone.MONE_BF16
        if d_out >= 256 or c["dtype"] == "f32":  # the memory's own widths play no part here
            cfg = mone.make_config(B, L, 128, 256, d_out, n_kv, hd, 128, dt, mone.MONE_PLAIN, 1e-2)
            W = torch.zeros(B * L, 256, 128, device=DEV), torch.zeros(B * L, 256, d_out, device=DEV)
        else:  # one head of 64: a two-head SwiGLU memory's handle
            cfg = mone.make_config(B, L, d_out, 64, d_out, n_kv, hd, 128, dt, mone.MONE_PLAIN, 1e-2,
                                   memory=mone.MONE_MEM_SWIGLU, mem_heads=2)
            W = torch.zeros(B * L, 2, 128, 64, device=DEV), torch.zeros(B * L, 2, 64, 64, device=DEV)
        self.h = mone.mone_mem_init(cfg, *W)
        d = self.d
        self.lens_out = torch.empty_like(d["lens"]) if "lens" in d else None
        self.out = torch.empty_like(d["q"]) if "q" in d else None
        if c["kind"] != "window":
            self.cache = mone.make_cache(d["K"], d["V"], d["table"], d["lens"], d.get("score"))
        if c["kind"] == "evict":
            self.kept = torch.empty(B, L, n_kv, c["keep"], dtype=torch.int32, device=DEV)

    def __del__(self):
        if self.h:
            self.mone.mone_mem_free(self.h)


def prepare(c, seed):
    return Program(c, seed)


# ------------------------------------------------------------------ the library's calls

def _run_own(p):
    c, d, mone, h = p.c, p.d, p.mone, p.h
    every = mone.MONE_ALL_LAYERS
    if c["kind"] == "window":
        mone.mone_window_attention(h, every, d["q"], c["n_q"], c["Lq"], d["k"], d["v"], d["k"].stride()[:4], c["n_past"],
                                   c["n_sink"], c["window"], p.out)
        return {"out": p.out}
    if c["kind"] == "attention":
        mone.mone_cache_attention(h, every, p.cache, d["q"], c["n_q"], c["n_tok"], c["n_sink"], c["window"], p.out)
        return {"out": p.out, "score": d["score"]} if c["score"] else {"out": p.out}
    if c["kind"] == "append":
        mone.mone_cache_append(h, every, p.cache, d["k"], d["v"], d["k"].stride()[:4], c["n_tok"], p.lens_out)
        return {"K": d["K"], "V": d["V"], "lens": p.lens_out}
    mone.mone_cache_evict(h, every, p.cache, c["keep"], c["n_sink"], c["n_recent"], d["to"], d["to_score"], p.kept, p.lens_out)
    return {"K": d["K"], "V": d["V"], "score": d["to_score"], "kept": p.kept, "lens": p.lens_out}


# ------------------------------------------------------------------ plain form

def _attend(q, k, v, hidden):
    """q [.., rows, hd], k and v [.., keys, hd], hidden [.., rows, keys]: outputs and weights, 0 where all is hidden."""
    z = (q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1])).masked_fill_(hidden, -math.inf)
    e = (z - z.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    w = e / e.sum(-1, keepdim=True).clamp(min=1e-38)
    return w @ v, w


def _window_plain(c, d):
    """Blocks of B tokens over the first positions and the band of B + window - 1 positions that the block's tokens see."""
    B, L, n_q, Lq, hd = d["q"].shape
    n_kv, group, S = c["n_kv"], c["n_q"] // c["n_kv"], c["n_past"] + c["Lq"]
    W = min(c["window"], S)
    blk = min(Lq, max(64, min(1024, W)))
    nb = -(-Lq // blk)
    t = c["n_past"] + torch.arange(nb * blk, device=DEV).view(nb, blk, 1)
    band = c["n_past"] + torch.arange(nb, device=DEV)[:, None] * blk + torch.arange(1 - W, blk, device=DEV)
    sink = torch.arange(min(c["n_sink"], S), device=DEV).expand(nb, -1)
    pos = torch.cat([sink, band], 1)[:, None, :]                      # [blocks, 1, keys]
    of_sink = torch.arange(pos.shape[-1], device=DEV) < sink.shape[1]
    hidden = (pos < 0) | (pos > t) | torch.where(of_sink, pos > t - W, pos <= t - W)
    at = pos.clamp(0, S - 1)[:, 0].reshape(-1)
    q = torch.nn.functional.pad(d["q"].float(), (0, 0, 0, nb * blk - Lq))
    q = q.view(B, L, n_kv, group, nb, blk, hd).transpose(3, 4).reshape(B, L, n_kv, nb, group * blk, hd)
    k, v = (x[:, :, :, at].float().view(B, L, n_kv, nb, -1, hd) for x in (d["k"], d["v"]))
    out, _ = _attend(q, k, v, hidden.repeat(1, group, 1))
    out = out.view(B, L, n_kv, nb, group, blk, hd).transpose(3, 4).reshape(B, L, n_q, nb * blk, hd)[:, :, :, :Lq]
    return {"out": out.to(d["q"].dtype)}


def _rows(c, table, pos):
    """Page and place of positions [contexts, n] (a page that is not there: page 0)."""
    return table.gather(1, (pos // c["page"]).clamp(max=table.shape[1] - 1)).clamp(min=0).long(), pos % c["page"]


def _attention_plain(c, d):
    B, L, n_q, n_tok, hd = d["q"].shape
    n_kv, group, S = c["n_kv"], c["n_q"] // c["n_kv"], c["length"]
    pos = torch.arange(S, device=DEV)
    pages, place = _rows(c, d["table"], pos.expand(B, S))
    there = pos < d["lens"][:, None]
    k, v = (x[:, pages, :, place].masked_fill(~there[:, :, None, None, None], 0).permute(0, 2, 3, 1, 4).float()
            for x in (d["K"], d["V"]))                              # [contexts, layers, heads, positions, hd]
    t = (d["lens"][:, None] - n_tok + torch.arange(n_tok, device=DEV))[:, :, None]
    hidden = (pos > t) | ((pos >= c["n_sink"]) & (pos <= t - c["window"]))  # [contexts, tokens, positions]
    q = d["q"].float().reshape(B, L, n_kv, group * n_tok, hd)
    out, w = _attend(q, k, v, hidden.repeat(1, group, 1)[:, None, None])
    out = out.view(B, L, n_q, n_tok, hd).to(d["q"].dtype)
    if not c["score"]:
        return {"out": out}
    d["score"][..., :S] += w.sum(-2)
    return {"out": out, "score": d["score"]}


def _append_plain(c, d):
    B, L, n_kv, n, hd = d["k"].shape
    pages, place = _rows(c, d["table"], d["lens"][:, None] + torch.arange(n, device=DEV))
    for pool, new in ((d["K"], d["k"]), (d["V"], d["v"])):
        pool[:, pages, :, place] = new.permute(0, 3, 1, 2, 4)
    return {"K": d["K"], "V": d["V"], "lens": d["lens"] + n}


def _evict_plain(c, d):
    B, L, n_kv, cap = d["score"].shape
    keep, N = c["keep"], d["lens"][:, None, None, None]
    pos = torch.arange(cap, device=DEV).expand(B, L, n_kv, cap)
    rank = torch.where((pos < c["n_sink"]) | (pos >= N - c["n_recent"]), 2, 1).masked_fill_(pos >= N, 0)
    by_score = d["score"].nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).sort(dim=-1, descending=True, stable=True).indices
    best = by_score.gather(-1, rank.gather(-1, by_score).sort(dim=-1, descending=True, stable=True).indices)
    kept = best[..., :keep].masked_fill(torch.arange(keep, device=DEV) >= N, cap).sort(-1).values  # cap: nothing there
    is_in = kept < cap
    of, layer, head, slot = is_in.nonzero(as_tuple=True)
    src = kept[is_in]
    page = c["page"]
    old, new = d["table"][of, src // page].long(), d["to"][of, slot // page].long()
    for pool in (d["K"], d["V"]):
        pool[layer, new, head, slot % page] = pool[layer, old, head, src % page]
    d["to_score"][of, layer, head, slot] = d["score"][of, layer, head, src]
    return {"K": d["K"], "V": d["V"], "score": d["to_score"], "kept": kept.masked_fill(~is_in, -1).int(),
            "lens": d["lens"].clamp(max=keep)}


def run(p):
    if own:
        return _run_own(p)
    c, d = p.c, p.d
    if c["kind"] == "window":
        return _window_plain(c, d)
    if c["kind"] == "attention":
        return _attention_plain(c, d)
    return _append_plain(c, d) if c["kind"] == "append" else _evict_plain(c, d)


# ------------------------------------------------------------------ from the definitions, in 64 bits

def _one(q, k, v, t, c):
    """Tokens q [rows, hd] at positions t [rows] over k, v [positions, hd] of one head: outputs and weights."""
    j = torch.arange(k.shape[0], device=DEV)
    sees = (j[None] <= t[:, None]) & ((j[None] < c["n_sink"]) | (j[None] > t[:, None] - c["window"]))
    z = torch.where(sees, q @ k.T / math.sqrt(q.shape[-1]), torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
    w = torch.where(sees.any(-1, keepdim=True), torch.softmax(z, -1), torch.zeros_like(z))
    return w @ v, w


def exact(c, seed):
    d = _inputs(c, seed)
    B, L, n_kv, group = c["n_ctx"], c["n_layers"], c["n_kv"], c["n_q"] // c["n_kv"]
    if c["kind"] == "window":
        out = torch.empty(d["q"].shape, dtype=torch.float64, device=DEV)
        for b in range(B):
            for l in range(L):
                for h in range(c["n_q"]):
                    k, v = d["k"][b, l, h // group].double(), d["v"][b, l, h // group].double()
                    for i in range(0, c["Lq"], 2048):
                        q = d["q"][b, l, h, i:i + 2048].double()
                        t = c["n_past"] + i + torch.arange(len(q), device=DEV)
                        end = int(t[-1]) + 1
                        out[b, l, h, i:i + 2048] = _one(q, k[:end], v[:end], t, c)[0]
        return {"out": out}
    K, V = d["K"], d["V"]
    page, lens = c["page"], lengths(c)
    table = d["table"].tolist()

    def held(pool, b, l, g, n):
        """The rows of one head at positions 0 .. n - 1."""
        return torch.cat([pool[l, p, g] for p in table[b][:-(-n // page)]])[:n]

    if c["kind"] == "attention":
        out = torch.empty(d["q"].shape, dtype=torch.float64, device=DEV)
        score = d["score"].double() if c["score"] else None
        for b in range(B):
            t = lens[b] - c["n_tok"] + torch.arange(c["n_tok"], device=DEV)
            for l in range(L):
                for g in range(n_kv):
                    k, v = held(K, b, l, g, lens[b]).double(), held(V, b, l, g, lens[b]).double()
                    for h in range(g * group, (g + 1) * group):
                        out[b, l, h], w = _one(d["q"][b, l, h].double(), k, v, t, c)
                        if score is not None:
                            score[b, l, g, :lens[b]] += w.sum(0)
        return {"out": out, "score": score} if c["score"] else {"out": out}
    K, V = K.double(), V.double()
    if c["kind"] == "append":
        for b in range(B):
            for i0 in range(0, c["n_tok"] + page, page):  # page by page
                lo = max(lens[b], (lens[b] + i0) // page * page)
                hi = min(lens[b] + c["n_tok"], lo // page * page + page)
                if lo < hi:
                    p, s = table[b][lo // page], slice(lo % page, lo % page + hi - lo)
                    K[:, p, :, s] = d["k"][b, :, :, lo - lens[b]:hi - lens[b]].double()
                    V[:, p, :, s] = d["v"][b, :, :, lo - lens[b]:hi - lens[b]].double()
        return {"K": K, "V": V, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV) + c["n_tok"]}
    keep, score, to = c["keep"], d["to_score"].double(), d["to"].tolist()
    kept = torch.full((B, L, n_kv, keep), -1, dtype=torch.int32, device=DEV)
    for b in range(B):
        N = lens[b]
        for l in range(L):
            for g in range(n_kv):
                s = d["score"][b, l, g, :N].double()
                if N <= keep:
                    at = torch.arange(N, device=DEV)
                else:
                    lo, hi = c["n_sink"], N - c["n_recent"]
                    mid = lo + torch.sort(-s[lo:hi], stable=True).indices[:keep - c["n_sink"] - c["n_recent"]]
                    at = torch.cat([torch.arange(lo, device=DEV), mid.sort().values, torch.arange(hi, N, device=DEV)])
                n = len(at)
                kept[b, l, g, :n] = at.int()
                score[b, l, g, :n] = s[at]
                for pool in (K, V):
                    rows = held(pool, b, l, g, N)[at]
                    for i in range(0, n, page):
                        pool[l, to[b][i // page], g, :min(page, n - i)] = rows[i:i + page]
    return {"K": K, "V": V, "score": score, "kept": kept,
            "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device=DEV)}
