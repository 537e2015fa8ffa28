"""Cases of the serving operators around a cache held in 4 bits: queries and keys normalised and rotated, pages taken and given
back on the GPU, and the cache's own append, read, attention and eviction.

A case has a "kind":

  rotate     mone_norm_rotate: every head's queries and keys divided by their root mean square, scaled and rotated by their
             position, in one pass.
  pages      mone_cache_reserve and mone_cache_release: pages for new tokens from the list of free ones, the tokens' slots, and
             the pages back again, as where a draft is rejected or a request is cancelled.
  append     mone_cache4_append and mone_cache4_read: new tokens' keys and values into 4-bit pages, and a context's positions
             back as dense keys and values, as a prompt's next chunk attends over them.
  attention  mone_cache4_attention: one or a few new tokens over a 4-bit cache, with the weights that each position gets
             added up for a later eviction, or without.
  evict      mone_cache4_evict: a 4-bit cache cut down to its first positions, its last ones and those of the highest weights;
             the survivors are read back.

A row of the cache is cut into groups of 16 values: an element is 2^exp x scale x code, the scale an e4m3 number of its group, the
code one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, two to a byte.

Sizes are those of the repository's workloads (16 layers with 8 KV heads of 64, heads of 128, 8 contexts, a memory of 64 tokens,
contexts of 32K and 128K) and generic ones around them.  `run` computes them with elementary torch operations in 32 bits
(angles and what lies next to a border in 64), or, where `own` is true, through the library.
"""
import math

import torch

own = False
DEV = "cuda"
ALL = 1 << 30  # a window that hides nothing
BASE = dict(n_ctx=1, n_layers=1, n_kv=8, n_q=32, hd=64, dtype="bf16")
ROTATE = dict(BASE, kind="rotate", rot=64, pairs="halves", period=0, base=10000.0, keys_only=False, norm=True, first=3000)
PAGED = dict(BASE, page=64, order="head", n_sink=0, window=ALL, k_exp=0, v_exp=0)


def listed():
    return [
        # a decode step's projections: one token of each of eight contexts, one layer of a backbone that runs layer by layer
        dict(ROTATE, name="rotate_token", n_ctx=8, n_tok=1),
        # a 2K prompt's queries and keys behind a memory of 64 tokens, every layer
        dict(ROTATE, name="rotate_l16_2k", n_layers=16, n_tok=2048, first=64),
        # a speculative step of 256 conversations: pages for up to five draft tokens each, all rejected
        dict(BASE, name="pages_step", kind="pages", n_ctx=256, n_kv=2, n_q=8, page=16, length=8192, n_tok=5, spare=3000),
        # sixteen long prompts are admitted, and cancelled
        dict(BASE, name="pages_admit", kind="pages", n_ctx=16, n_kv=2, n_q=8, page=16, length=300, n_tok=32768, spare=50000),
        # one new token for each of eight contexts, one layer: latency
        dict(PAGED, name="append_token", kind="append", n_ctx=8, page=16, length=3000, n_tok=1, whole=False),
        # a 2K prompt into the pages of 16 layers, and the context back for the next chunk
        dict(PAGED, name="append_l16_2k", kind="append", n_layers=16, length=64, n_tok=2048, whole=True),
        # the first token after a short prompt, one layer: latency
        dict(PAGED, name="token_first", kind="attention", n_tok=1, length=150, page=16, score=False),
        # decode over 1K positions, every layer, weights added up
        dict(PAGED, name="token_l16_1k", kind="attention", n_layers=16, n_tok=1, length=1151, score=True),
        # a batch of 16 conversations of very unequal length, one layer in fp32, pages of 32, weights added up
        dict(PAGED, name="token_batch16_f32", kind="attention", n_ctx=16, hd=128, n_tok=1, length=32768, page=32, score=True, dtype="f32"),
        # a context of 128K in four layers, two new tokens: the most that is read
        dict(PAGED, name="token_128k", kind="attention", n_layers=4, hd=128, n_tok=2, length=131072, score=False),
        # half of a 2K cache goes, every layer
        dict(PAGED, name="evict_l16_2k", kind="evict", n_layers=16, length=2048, keep=1024, n_sink=4, n_recent=128),
        # eight contexts of up to 32K cut to 8K, one layer
        dict(PAGED, name="evict_ctx8_32k", kind="evict", n_ctx=8, hd=128, page=32, length=32768, keep=8192, n_sink=64, n_recent=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "pages", "append", "append", "attention", "attention", "attention", "evict"])
    n_kv = rng.choice([1, 2, 4, 8])
    c = dict(kind=kind, n_ctx=rng.choice([1, 1, 2, 5, 16]), n_layers=rng.choice([1, 1, 2, 16]), n_kv=n_kv,
             n_q=n_kv * rng.choice([1, 2, 4, 5, 8]), hd=rng.choice([64, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if kind == "rotate":
        c.update(n_tok=_log(rng, 1, 20000), first=_log(rng, 1, 1000000), pairs=rng.choice(["halves", "halves", "neighbours"]),
                 base=rng.choice([10000.0, 500000.0]), period=rng.choice([0, 0, 512, 1000]), keys_only=rng.random() < 0.3,
                 norm=rng.random() < 0.7, rot=rng.choice([c["hd"], c["hd"], c["hd"] // 2, 48]))
        most = ("n_tok", 6e8)
    elif kind == "pages":
        c.update(n_ctx=_log(rng, 1, 300), n_layers=1, n_kv=2, n_q=8, hd=64, dtype="bf16", page=rng.choice([8, 16, 32, 64, 128]),
                 length=_log(rng, 1, 20000), n_tok=_log(rng, 1, 20000), spare=_log(rng, 1, 60000))
        most = ("n_tok", 5e6)
    else:
        c.update(page=rng.choice([8, 16, 32, 64, 128]), order=rng.choice(["head", "position"]), n_sink=rng.choice([0, 4, 64]),
                 length=_log(rng, 40, 60000), window=ALL, k_exp=rng.choice([0, 0, 1, -2]), v_exp=rng.choice([0, 0, -1, 3]))
        most = ("length", 6e8)
        if kind == "attention":
            c.update(n_tok=rng.choice([1, 1, 1, 2, 5]), score=rng.random() < 0.5, window=rng.choice([ALL, ALL, _log(rng, 1, 20000)]))
        elif kind == "evict":
            c.update(keep=max(1, int(c["length"] * rng.uniform(0.1, 0.9))))
            c["n_sink"] = min(c["n_sink"], c["keep"] // 2)
            c["n_recent"] = rng.randint(0, c["keep"] - c["n_sink"])
        else:
            c.update(n_tok=_log(rng, 1, 4000), whole=rng.random() < 0.5)
            c["length"] = min(c["length"], 8000)
    while work(c)["bytes"] > most[1] or work(c)["flops"] > 2e10:
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


def _counts(c):
    """New tokens of each context: `n_tok` alone, or a spread from none to it."""
    n, t = c["n_ctx"], c["n_tok"]
    return [t * ((i * 5 + 3) % n + 1) // n for i in range(n)] if n > 1 else [t]


def _width(c):
    """Entries of a context's page table: what the longest needs, and one spare."""
    return -(-(c["length"] + (c["n_tok"] if c["kind"] in ("append", "pages") else 0)) // c["page"]) + 1


def _pages(c):
    """Pages of a layer's pool: every context's own, fresh ones for the survivors of an eviction, and some that nobody has."""
    if c["kind"] == "pages":
        return sum(-(-n // c["page"]) for n in lengths(c)) + c["spare"]
    return c["n_ctx"] * (_width(c) + (-(-c["keep"] // c["page"]) if c["kind"] == "evict" else 0)) + 5


def _seen(t, c):
    """Positions that the token at position t sees."""
    lo = max(0, t - c["window"] + 1)
    return t + 1 - lo + min(lo, c["n_sink"]) if t >= 0 else 0


def _union(t0, t1, c):
    """Positions that some token at t0 .. t1 sees."""
    lo = max(0, t0 - c["window"] + 1)
    return t1 + 1 - lo + min(lo, c["n_sink"]) if t1 >= 0 else 0


def _back(c):
    """Positions of each context that are read back after an append: its new ones, or all."""
    return c["length"] + c["n_tok"] if c["whole"] else c["n_tok"]


def work(c):
    el, hd, L, n_kv, B = 4 if c["dtype"] == "f32" else 2, c["hd"], c["n_layers"], c["n_kv"], c["n_ctx"]
    four = hd * 9 // 16  # bytes of a row in 4 bits, its scales among them
    if c["kind"] == "rotate":
        n = B * L * (n_kv + (0 if c["keys_only"] else c["n_q"])) * c["n_tok"] * hd
        return {"bytes": 2 * el * n, "flops": (8 if c["norm"] else 4) * n}
    if c["kind"] == "pages":
        page = c["page"]
        new = min(c["spare"], sum(-(-(n + k) // page) - -(-n // page) for n, k in zip(lengths(c), _counts(c))))
        return {"bytes": 20 * B + 20 * new + 8 * B * c["n_tok"], "flops": 0}
    if c["kind"] == "append":
        rows = B * L * n_kv
        read = sum(n + c["n_tok"] for n in lengths(c)) * L * n_kv if c["whole"] else rows * c["n_tok"]
        return {"bytes": rows * c["n_tok"] * 2 * (el * hd + four) + read * 2 * (el * hd + (four if c["whole"] else 0)), "flops": 0}
    if c["kind"] == "evict":
        kept = sum(min(n, c["keep"]) for n in lengths(c))
        return {"bytes": L * n_kv * (4 * sum(lengths(c)) + kept * (4 * four + 8 + 2 * el * hd)), "flops": 0}
    read = sum(_union(n - c["n_tok"], n - 1, c) for n in lengths(c))
    pairs = sum(_seen(n - 1 - i, c) for n in lengths(c) for i in range(c["n_tok"]))
    return {"bytes": L * (n_kv * read * (2 * four + (8 if c["score"] else 0)) + 2 * el * hd * B * c["n_q"] * c["n_tok"]),
            "flops": 4 * hd * c["n_q"] * pairs * L}


# ------------------------------------------------------------------ a row in 4 bits: codes and scales as the plain form has them

def _encode(x, exp):
    """x [.., hd] as codes [.., hd / 2] (two to a byte, the even element low) and e4m3 scales [.., hd / 16]: both to nearest, ties to
    even, in 64 bits."""
    g = x.double().unflatten(-1, (-1, 16)) * 2.0 ** -exp
    big = g.abs().amax(-1, keepdim=True).clamp(max=2688) / 6
    step = torch.exp2(torch.frexp(big).exponent.clamp(min=-5).double() - 4)  # of e4m3 numbers around it: four bits, 2^-9 at least
    scale = torch.round(big / step) * step
    r = (g.abs() / scale).nan_to_num(nan=0.0).clamp(max=6)
    unit = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0))
    v = torch.round(r / unit) * unit
    code = torch.where(v < 2, 2 * v, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8) | (torch.signbit(g).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., ::2] | (code[..., 1::2] << 4), scale[..., 0].float().to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(code, scale, exp):
    """Codes [.., hd / 2] and scales [.., hd / 16] as fp32 values [.., hd]."""
    c = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    m = (c & 7).float()
    v = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8))
    v = torch.where(c >= 8, -v, v).unflatten(-1, (-1, 16))
    return (v * (scale.view(torch.float8_e4m3fn).float() * 2.0 ** exp)[..., None]).flatten(-2)


# ------------------------------------------------------------------ what a program has in hand

def _inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    B, L, n_kv, n_q, hd = c["n_ctx"], c["n_layers"], c["n_kv"], c["n_q"], c["hd"]
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    if c["kind"] == "rotate":
        heads = n_kv + (0 if c["keys_only"] else n_q)
        x = 3 * rn(B, L, c["n_tok"], heads, hd).transpose(2, 3)  # as a projection leaves them: token after token, all its heads
        d = {"k": x[:, :, :n_kv], "first": torch.tensor([c["first"] * (i + 1) // B for i in range(B)], dtype=torch.int32, device=DEV)}
        if not c["keys_only"]:
            d["q"] = x[:, :, n_kv:]
        if c["norm"]:
            d["wq"], d["wk"] = (1 + 0.2 * torch.randn(L, hd, generator=g, device=DEV) for _ in range(2))
        return d
    page, W, P = c["page"], _width(c), _pages(c)
    lens = torch.tensor(lengths(c), dtype=torch.int32, device=DEV)
    order = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    at = torch.arange(W, device=DEV)[None, :]
    if c["kind"] == "pages":
        held = (lens + page - 1) // page
        before = torch.cumsum(held, 0) - held
        table = torch.where(at < held[:, None], order[(before[:, None] + at).clamp(max=P - 1)], -1)
        used = int(held.sum())
        free = torch.cat([order[used:], torch.full((used,), -1, dtype=torch.int32, device=DEV)])  # room for every page
        return {"table": table, "lens": lens, "free": free, "n_free": torch.tensor([P - used], dtype=torch.int32, device=DEV),
                "counts": torch.tensor(_counts(c), dtype=torch.int32, device=DEV)}
    d = {"lens": lens}
    for name, exp in (("K", c["k_exp"]), ("V", c["v_exp"])):
        shape = (P, n_kv, page, hd) if c["order"] == "head" else (P, page, n_kv, hd)
        rows = [_encode(2.0 ** exp * torch.randn(*shape, generator=g, device=DEV), exp) for _ in range(L)]
        d[name], d[name + "s"] = (torch.stack(x) if c["order"] == "head" else torch.stack(x).transpose(2, 3) for x in zip(*rows))
    held = lens + (c["n_tok"] if c["kind"] == "append" else 0)
    d["table"] = order[:B * W].view(B, W).masked_fill(at * page >= held[:, None], -1)  # past them, no page yet
    if c["kind"] == "attention":
        d["q"] = 2 * rn(B, L, n_q, c["n_tok"], hd)
    if c["kind"] == "append":
        d["k"], d["v"] = (2.0 ** exp * rn(B, L, n_kv, c["n_tok"], hd) for exp in (c["k_exp"], c["v_exp"]))
    if c["kind"] == "evict" or c.get("score"):  # weights as a softmax over the cache leaves them: a few large, most small
        w = torch.randn(B, L, n_kv, W * page, generator=g, device=DEV)
        d["score"] = torch.exp(2 * w) / c["length"]
    if c["kind"] == "evict":
        n = -(-c["keep"] // page)
        d["to"] = order[B * W:B * W + B * n].view(B, n).clone()
        d["to_score"] = torch.zeros(B, L, n_kv, n * page, device=DEV)
    return d


def _frequencies(c):
    return [c["base"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]


class Program:
    """Inputs, the buffers of the outputs, and for the library a handle and what else a program keeps."""

    def __init__(self, c, seed):
        self.c, self.h = c, None
        self.d = d = _inputs(c, seed)
        B, L, n_kv, hd, dt = c["n_ctx"], c["n_layers"], c["n_kv"], c["hd"], torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        if c["kind"] in ("append", "evict"):
            n = _back(c) if c["kind"] == "append" else c["keep"]
            self.K, self.V = (torch.zeros(B, L, n_kv, n, hd, dtype=dt, device=DEV) for _ in range(2))
        if not own:
            return
        import paper_2608_17616_gb300 as mone
        self.mone = mone
        d_out, kind = 2 * n_kv * hd, mone.MONE_FP32 if c["dtype"] == "f32" else mone.MONE_BF16
        if d_out >= 256 or c["dtype"] == "f32":  # the memory's own widths play no part here
            cfg = mone.make_config(B, L, 128, 256, d_out, n_kv, hd, 128, kind, mone.MONE_PLAIN, 1e-2)
            W = torch.zeros(B * L, 256, 128, device=DEV), torch.zeros(B * L, 256, d_out, device=DEV)
        else:  # one head of 64: a two-head SwiGLU memory's handle
            cfg = mone.make_config(B, L, d_out, 64, d_out, n_kv, hd, 128, kind, mone.MONE_PLAIN, 1e-2,
                                   memory=mone.MONE_MEM_SWIGLU, mem_heads=2)
            W = torch.zeros(B * L, 2, 128, 64, device=DEV), torch.zeros(B * L, 2, 64, 64, device=DEV)
        self.h = mone.mone_mem_init(cfg, *W)
        self.lens_out = torch.empty_like(d["lens"]) if "lens" in d else None
        if c["kind"] == "rotate":
            pairing = mone.MONE_ROTATE_HALVES if c["pairs"] == "halves" else mone.MONE_ROTATE_NEIGHBOURS
            self.rotary = mone.make_rotary(c["rot"], pairing, freq=_frequencies(c), period=c["period"], eps=1e-6)
            self.k = torch.empty(d["k"].shape, dtype=dt, device=DEV)
            self.heads = [None, mone.make_heads(d["k"], self.k, d.get("wk"))]
            if not c["keys_only"]:
                self.q = torch.empty(d["q"].shape, dtype=dt, device=DEV)
                self.heads[0] = mone.make_heads(d["q"], self.q, d.get("wq"))
            return
        if c["kind"] == "pages":
            self.granted, self.n_free = torch.empty_like(d["counts"]), [torch.empty_like(d["n_free"]) for _ in range(2)]
            self.slots = torch.empty(B, c["n_tok"], dtype=torch.int64, device=DEV)
            self.back = torch.empty_like(d["lens"])
            self.pages = mone.make_pages(d["free"], d["n_free"], d["table"], d["lens"], c["page"])
            self.grown = mone.make_pages(d["free"], self.n_free[0], d["table"], self.lens_out, c["page"])
            return
        exps = dict(k_exp=c["k_exp"], v_exp=c["v_exp"])
        pools = d["K"], d["V"], d["Ks"], d["Vs"]
        self.cache = mone.make_cache4(*pools, d["table"], d["lens"], d.get("score"), **exps)
        if c["kind"] == "attention":
            self.out = torch.empty_like(d["q"])
        if c["kind"] == "append":
            self.after = mone.make_cache4(*pools, d["table"], self.lens_out, **exps)
        if c["kind"] == "evict":
            self.kept = torch.empty(B, L, n_kv, c["keep"], dtype=torch.int32, device=DEV)
            self.after = mone.make_cache4(*pools, d["to"], self.lens_out, d["to_score"], **exps)

    def __del__(self):
        if self.h:
            self.mone.mone_mem_free(self.h)


def prepare(c, seed):
    return Program(c, seed)


# ------------------------------------------------------------------ the library's calls

def _run_own(p):
    c, d, mone, h = p.c, p.d, p.mone, p.h
    every = mone.MONE_ALL_LAYERS
    if c["kind"] == "rotate":
        mone.mone_norm_rotate(h, every, p.rotary, d["first"], c["n_tok"], *p.heads)
        return {"k": p.k} if c["keys_only"] else {"k": p.k, "q": p.q}
    if c["kind"] == "pages":
        mone.mone_cache_reserve(h, p.pages, c["n_tok"], p.n_free[0], p.lens_out, p.granted, p.slots, d["counts"])
        mone.mone_cache_release(h, p.grown, p.n_free[1], d["lens"], p.back)
        return {"granted": p.granted, "slots": p.slots, "lens": p.lens_out, "left": p.n_free[0], "table": d["table"], "free": d["free"],
                "n_free": p.n_free[1], "back": p.back}
    if c["kind"] == "attention":
        mone.mone_cache4_attention(h, every, p.cache, d["q"], c["n_q"], c["n_tok"], c["n_sink"], c["window"], p.out)
        return {"out": p.out, "score": d["score"]} if c["score"] else {"out": p.out}
    if c["kind"] == "append":
        mone.mone_cache4_append(h, every, p.cache, d["k"], d["v"], d["k"].stride()[:4], c["n_tok"], p.lens_out)
        mone.mone_cache4_read(h, every, p.after, None if c["whole"] else d["lens"], _back(c), p.K, p.V, p.K.stride()[:4])
        return {"K": p.K, "V": p.V, "lens": p.lens_out}
    mone.mone_cache4_evict(h, every, p.cache, c["keep"], c["n_sink"], c["n_recent"], d["to"], d["to_score"], p.kept, p.lens_out)
    mone.mone_cache4_read(h, every, p.after, None, c["keep"], p.K, p.V, p.K.stride()[:4])
    return {"K": p.K, "V": p.V, "score": d["to_score"], "kept": p.kept, "lens": p.lens_out}


# ------------------------------------------------------------------ plain form

def _rotate_plain(c, d):
    pos = d["first"][:, None].double() + torch.arange(c["n_tok"], device=DEV)
    if c["period"]:
        pos = pos % c["period"]
    angle = pos[..., None] * torch.tensor(_frequencies(c), dtype=torch.float64, device=DEV)
    cos, sin = (f(angle).float()[:, None, None] for f in (torch.cos, torch.sin))  # [contexts, 1, 1, tokens, pairs]
    n = c["rot"] // 2

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w[None, :, None, None]
        a, b = (y[..., :n], y[..., n:2 * n]) if c["pairs"] == "halves" else (y[..., 0:2 * n:2], y[..., 1:2 * n:2])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.cat([a, b], -1) if c["pairs"] == "halves" else torch.stack([a, b], -1).flatten(-2)
        return torch.cat([turned, y[..., 2 * n:]], -1).to(x.dtype)

    k = one(d["k"], d.get("wk"))
    return {"k": k} if c["keys_only"] else {"k": k, "q": one(d["q"], d.get("wq"))}


def _pages_plain(c, d):
    page, table, free, n_free, lens = c["page"], d["table"], d["free"], d["n_free"], d["lens"]
    held = (lens + page - 1) // page
    need = (lens + d["counts"] + page - 1) // page - held
    fits = (need == 0) | (torch.cumsum(need, 0) <= n_free)
    new = torch.where(fits, need, 0)
    granted, total = torch.where(fits, d["counts"], 0), new.sum()
    upto = torch.cumsum(new, 0)
    at = torch.arange(table.shape[1], device=DEV)
    fresh = (at >= held[:, None]) & (at < (held + new)[:, None])
    from_top = (n_free - total + (upto - new)[:, None] + at - held[:, None]).clamp(0, len(free) - 1)
    grown = torch.where(fresh, free[from_top], table)
    tok = torch.arange(c["n_tok"], device=DEV)
    pos = lens[:, None] + tok
    slots = grown.gather(1, (pos // page).clamp(max=table.shape[1] - 1).long()).long() * page + pos % page
    slots = torch.where(tok < granted[:, None], slots, -1)
    back = torch.where((torch.arange(len(free), device=DEV) >= n_free - total) & (torch.arange(len(free), device=DEV) < n_free), 1, 0)
    again = free.clone()
    again[back.bool()] = grown[fresh]  # context after context, as they came
    return {"granted": granted.int(), "slots": slots, "lens": lens + granted.int(), "left": (n_free - total).int(),
            "table": torch.where(fresh, -1, grown).int(), "free": again, "n_free": n_free, "back": lens}


def _attend(q, k, v, hidden):
    """q [.., rows, hd], k and v [.., keys, hd], hidden [.., rows, keys]: outputs and weights, 0 where all is hidden."""
    z = (q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1])).masked_fill_(hidden, -math.inf)
    e = (z - z.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    w = e / e.sum(-1, keepdim=True).clamp(min=1e-38)
    return w @ v, w


def _rows(c, table, pos):
    """Page and place of positions [contexts, n] (a page that is not there: page 0)."""
    return table.gather(1, (pos // c["page"]).clamp(max=table.shape[1] - 1)).clamp(min=0).long(), pos % c["page"]


def _held(c, d, table, lens, pos):
    """Keys and values at positions [contexts, n], 0 where none is held: [contexts, layers, heads, n, hd] fp32."""
    pages, place = _rows(c, table, pos)
    there = (pos < lens[:, None])[:, None, None, :, None]
    return [torch.where(there, _decode(*(d[name + s][:, pages, :, place].permute(0, 2, 3, 1, 4) for s in ("", "s")), exp), 0)
            for name, exp in (("K", c["k_exp"]), ("V", c["v_exp"]))]


def _attention_plain(c, d):
    B, L, n_q, n_tok, hd = d["q"].shape
    n_kv, group, S = c["n_kv"], c["n_q"] // c["n_kv"], c["length"]
    pos = torch.arange(S, device=DEV)
    k, v = _held(c, d, d["table"], d["lens"], pos.expand(B, S))
    t = (d["lens"][:, None] - n_tok + torch.arange(n_tok, device=DEV))[:, :, None]
    hidden = (pos > t) | ((pos >= c["n_sink"]) & (pos <= t - c["window"]))  # [contexts, tokens, positions]
    q = d["q"].float().reshape(B, L, n_kv, group * n_tok, hd)
    out, w = _attend(q, k, v, hidden.repeat(1, group, 1)[:, None, None])
    out = out.view(B, L, n_q, n_tok, hd).to(d["q"].dtype)
    if not c["score"]:
        return {"out": out}
    d["score"][..., :S] += w.sum(-2)
    return {"out": out, "score": d["score"]}


def _append_plain(p):
    c, d = p.c, p.d
    n = c["n_tok"]
    new = d["lens"][:, None] + torch.arange(n, device=DEV)
    pages, place = _rows(c, d["table"], new)
    for name, x, exp in (("K", d["k"], c["k_exp"]), ("V", d["v"], c["v_exp"])):
        code, scale = _encode(x, exp)
        d[name][:, pages, :, place] = code.permute(0, 3, 1, 2, 4)
        d[name + "s"][:, pages, :, place] = scale.permute(0, 3, 1, 2, 4)
    lens = d["lens"] + n
    K, V = _held(c, d, d["table"], lens, torch.arange(_back(c), device=DEV).expand(len(lens), -1) if c["whole"] else new)
    return {"K": K.to(p.K.dtype), "V": V.to(p.V.dtype), "lens": lens}


def _evict_plain(p):
    c, d = p.c, p.d
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
    for pool in (d["K"], d["V"], d["Ks"], d["Vs"]):
        pool[layer, new, head, slot % page] = pool[layer, old, head, src % page]
    d["to_score"][of, layer, head, slot] = d["score"][of, layer, head, src]
    lens = d["lens"].clamp(max=keep)
    K, V = _held(c, d, d["to"], lens, torch.arange(keep, device=DEV).expand(B, keep))
    return {"K": K.to(p.K.dtype), "V": V.to(p.V.dtype), "score": d["to_score"], "kept": kept.masked_fill(~is_in, -1).int(), "lens": lens}


def run(p):
    if own:
        return _run_own(p)
    c, d = p.c, p.d
    if c["kind"] == "rotate":
        return _rotate_plain(c, d)
    if c["kind"] == "pages":
        return _pages_plain(c, d)
    if c["kind"] == "attention":
        return _attention_plain(c, d)
    return _append_plain(p) if c["kind"] == "append" else _evict_plain(p)


# ------------------------------------------------------------------ from the definitions, in 64 bits

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_E4M3 = [m / 512 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119]


def _nearest(x, numbers):
    """The index of the number nearest to x >= 0, ties to the even index, the last one from there on."""
    mid = torch.tensor([(a + b) / 2 for a, b in zip(numbers, numbers[1:])], dtype=torch.float64, device=DEV)
    below, upto = torch.searchsorted(mid, x), torch.searchsorted(mid, x, right=True)  # midpoints below x, and up to it
    return torch.where((below != upto) & (below % 2 == 1), upto, below)


def _rounded(x, exp):
    """What x [.., hd] becomes in the cache."""
    codes, scales = (torch.tensor(t, dtype=torch.float64, device=DEV) for t in (_E2M1, _E4M3))
    g = x.double().reshape(*x.shape[:-1], -1, 16) / 2.0 ** exp
    s = scales[_nearest((g.abs().max(-1, keepdim=True).values / 6).contiguous(), _E4M3)]
    v = codes[_nearest(torch.where(s > 0, g.abs() / torch.where(s > 0, s, 1), 0).contiguous(), _E2M1)]
    return (torch.sign(g) * v * s * 2.0 ** exp).reshape(x.shape)


def _values(code, scale, exp):
    """Codes and scales of rows [n, hd / 2], [n, hd / 16] in 64 bits."""
    table = torch.tensor([s * v for s in (1.0, -1.0) for v in _E2M1], dtype=torch.float64, device=DEV)
    both = torch.empty(code.shape[0], 2 * code.shape[1], dtype=torch.float64, device=DEV)
    both[:, 0::2], both[:, 1::2] = table[(code % 16).long()], table[(code // 16).long()]
    s = torch.tensor(_E4M3, dtype=torch.float64, device=DEV)[(scale & 127).long()]
    return both * s.repeat_interleave(16, 1) * 2.0 ** exp


def _one(q, k, v, t, c):
    """Tokens q [rows, hd] at positions t [rows] over k, v [positions, hd] of one head: outputs and weights."""
    j = torch.arange(k.shape[0], device=DEV)
    sees = (j[None] <= t[:, None]) & ((j[None] < c["n_sink"]) | (j[None] > t[:, None] - c["window"]))
    z = torch.where(sees, q @ k.T / math.sqrt(q.shape[-1]), torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
    w = torch.where(sees.any(-1, keepdim=True), torch.softmax(z, -1), torch.zeros_like(z))
    return w @ v, w


def _exact_rotate(c, d):
    out = {}
    for name, w in (("k", d.get("wk")), ("q", d.get("wq"))):
        if name not in d:
            continue
        x = d[name].double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["hd"] + 1e-6) * w.double()[None, :, None, None, :]
        y = x.clone()
        for i, f in enumerate(_frequencies(c)):
            a, b = (i, i + c["rot"] // 2) if c["pairs"] == "halves" else (2 * i, 2 * i + 1)
            for ctx in range(c["n_ctx"]):
                p = [int(d["first"][ctx]) + j for j in range(c["n_tok"])] if ctx == 0 or i == 0 else None
                if i == 0:
                    p = [j % c["period"] for j in p] if c["period"] else p
                    out.setdefault(("p", name), []).append(torch.tensor(p, dtype=torch.float64, device=DEV))
                turn = out["p", name][ctx] * f
                y[ctx, ..., a] = x[ctx, ..., a] * torch.cos(turn) - x[ctx, ..., b] * torch.sin(turn)
                y[ctx, ..., b] = x[ctx, ..., b] * torch.cos(turn) + x[ctx, ..., a] * torch.sin(turn)
        out[name] = y
    return {k: v for k, v in out.items() if isinstance(k, str)}


def _exact_pages(c, d):
    page, lens, counts = c["page"], lengths(c), _counts(c)
    table, free, left = d["table"].tolist(), d["free"].tolist(), int(d["n_free"])
    need = [-(-(n + k) // page) - -(-n // page) for n, k in zip(lens, counts)]
    asked, fits = 0, []
    for n in need:
        asked += n
        fits.append(n == 0 or asked <= left)
    new = [n if f else 0 for n, f in zip(need, fits)]
    granted, top = [k if f else 0 for k, f in zip(counts, fits)], left - sum(new)
    slots = torch.full((len(lens), c["n_tok"]), -1, dtype=torch.int64)
    taken = top
    for b, n in enumerate(lens):
        own_pages = table[b][:-(-n // page)] + free[taken:taken + new[b]]
        taken += new[b]
        if granted[b]:
            at = torch.arange(n, n + granted[b])
            slots[b, :granted[b]] = torch.tensor(own_pages)[at // page] * page + at % page
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"granted": t(granted), "slots": slots.to(DEV), "lens": t([n + g for n, g in zip(lens, granted)]), "left": t([top]),
            "table": d["table"], "free": d["free"], "n_free": d["n_free"], "back": t(lens)}


def exact(c, seed):
    d = _inputs(c, seed)
    if c["kind"] == "rotate":
        return _exact_rotate(c, d)
    if c["kind"] == "pages":
        return _exact_pages(c, d)
    B, L, n_kv, group = c["n_ctx"], c["n_layers"], c["n_kv"], c["n_q"] // c["n_kv"]
    page, lens, table, hd = c["page"], lengths(c), d["table"].tolist(), c["hd"]

    def held(name, b, l, g, n):
        """The rows of one head at positions 0 .. n - 1."""
        code, scale = (torch.cat([d[name + s][l, p, g] for p in table[b][:-(-n // page)]])[:n] for s in ("", "s"))
        return _values(code, scale, c["k_exp"] if name == "K" else c["v_exp"])

    if c["kind"] == "attention":
        out = torch.empty(d["q"].shape, dtype=torch.float64, device=DEV)
        score = d["score"].double() if c["score"] else None
        for b in range(B):
            t = lens[b] - c["n_tok"] + torch.arange(c["n_tok"], device=DEV)
            for l in range(L):
                for g in range(n_kv):
                    k, v = held("K", b, l, g, lens[b]), held("V", b, l, g, lens[b])
                    for h in range(g * group, (g + 1) * group):
                        out[b, l, h], w = _one(d["q"][b, l, h].double(), k, v, t, c)
                        if score is not None:
                            score[b, l, g, :lens[b]] += w.sum(0)
        return {"out": out, "score": score} if c["score"] else {"out": out}
    n = _back(c) if c["kind"] == "append" else c["keep"]
    K, V = (torch.zeros(B, L, n_kv, n, hd, dtype=torch.float64, device=DEV) for _ in range(2))
    if c["kind"] == "append":
        for to, name, x, exp in ((K, "K", d["k"], c["k_exp"]), (V, "V", d["v"], c["v_exp"])):
            new = _rounded(x, exp)
            for b in range(B):
                at = lens[b] if c["whole"] else 0
                to[b, :, :, at:at + c["n_tok"]] = new[b]
                if c["whole"]:
                    for l in range(L):
                        for g in range(n_kv):
                            to[b, l, g, :at] = held(name, b, l, g, at)
        return {"K": K, "V": V, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV) + c["n_tok"]}
    keep, score = c["keep"], d["to_score"].double()
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
                kept[b, l, g, :len(at)] = at.int()
                score[b, l, g, :len(at)] = s[at]
                K[b, l, g, :len(at)], V[b, l, g, :len(at)] = held("K", b, l, g, N)[at], held("V", b, l, g, N)[at]
    return {"K": K, "V": V, "score": score, "kept": kept,
            "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device=DEV)}
