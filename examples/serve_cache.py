"""Serving with a learned memory: a context is learned into the fast weights, the memory's tokens open the cache, the prompt
attends over them and a sliding window, and new tokens are decoded over a paged cache that is cut down when it has grown.

    python examples/serve_cache.py [--check]

What a program around the library keeps is here in its smallest form: a free list of pages, the lengths, the scores.  The
backbone is not part of the library, so its per-layer activations and projections are random numbers here; --check
recomputes the prompt's and the last tokens' outputs in 64 bits.
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2608_17616_gb300 as mone  # noqa: E402

ALL = 1 << 30  # a window that hides nothing


class Pages:
    """The pages of a pool that nobody holds, and the tables of those that a context holds (the same in every layer)."""

    def __init__(self, n_ctx, width, count, page):
        self.page, self.free = page, list(range(count))
        self.table = torch.full((n_ctx, width), -1, dtype=torch.int32)
        self.held = [0] * n_ctx

    def grow(self, ctx, positions):
        """Pages for a context's first `positions` positions; True if its table changed."""
        need = -(-positions // self.page)
        for b in range(self.held[ctx], need):
            self.table[ctx, b] = self.free.pop()
        grown, self.held[ctx] = need > self.held[ctx], max(need, self.held[ctx])
        return grown

    def replace(self, new):
        """The survivors' pages in place of the old ones, which are free again."""
        for ctx, n in enumerate(self.held):
            self.free += self.table[ctx, :n].tolist()
        self.table, self.held = new.table, new.held


def serve(n_ctx=2, n_layers=3, n_kv=2, group=4, hd=64, n_mem=16, prompt=150, window=64, tokens=60, most=192, keep=96, recent=32,
          page=16, check=False, seed=0):
    """Learn, read, prefill and decode; returns how often the cache was cut, and with check the largest relative error."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf = lambda *s: rn(*s).bfloat16()  # noqa: E731
    d_in, d_hid, d_out, n_q, C = 256, 256, 2 * n_kv * hd, group * n_kv, n_ctx * n_layers

    # the memory learns a context and gives its tokens for the prompt
    cfg = mone.make_config(n_ctx, n_layers, d_in, d_hid, d_out, n_kv, hd, 128, mone.MONE_BF16, mone.MONE_PLAIN, 1e-2)
    h = mone.mone_mem_init(cfg, rn(C, d_hid, d_in) / d_in ** 0.5, rn(C, d_hid, d_out) / d_hid ** 0.5)
    mone.mone_ttl_context(h, bf(n_ctx, n_layers, 300, d_in), bf(n_ctx, n_layers, 300, d_out // 2), bf(n_ctx, n_layers, 300, d_out // 2), 300)
    K, V = bf(n_ctx, n_layers, n_kv, n_mem + prompt, hd), bf(n_ctx, n_layers, n_kv, n_mem + prompt, hd)
    mone.mone_mem_generate_kv(h, bf(n_ctx, n_layers, n_mem, d_in), n_mem, K, V, K.stride()[:4])  # positions 0 .. n_mem - 1

    # the prompt: every token sees the memory and the last `window` tokens
    Q = bf(n_ctx, n_layers, n_q, prompt, hd)
    out = torch.empty_like(Q)
    mone.mone_window_attention(h, mone.MONE_ALL_LAYERS, Q, n_q, prompt, K, V, K.stride()[:4], n_mem, n_mem, window, out)
    worst = _prompt_error(Q, K, V, out, n_mem, window) if check else 0.0

    # memory and prompt into the pages of the cache
    width = -(-most // page) + 1
    pages = Pages(n_ctx, width, 3 * n_ctx * width, page)
    pool = [torch.empty(n_layers, 3 * n_ctx * width, n_kv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    score, lens = torch.zeros(n_ctx, n_layers, n_kv, width * page, device="cuda"), torch.zeros(n_ctx, dtype=torch.int32, device="cuda")
    new_lens, length = torch.empty_like(lens), n_mem + prompt
    for ctx in range(n_ctx):
        pages.grow(ctx, length)
    table = pages.table.cuda()
    mone.mone_cache_append(h, mone.MONE_ALL_LAYERS, mone.make_cache(*pool, table, lens, score), K, V, K.stride()[:4], length, new_lens)
    lens, new_lens = new_lens, lens
    # the last prompt tokens say which positions matter: their weights open the scores
    last = Q[..., -8:, :].contiguous()
    mone.mone_cache_attention(h, mone.MONE_ALL_LAYERS, mone.make_cache(*pool, table, lens, score), last, n_q, 8, n_mem, ALL, torch.empty_like(last))

    cuts, held = 0, [K, V]  # held: what the cache should hold, for the check
    for step in range(tokens):
        if length == most:  # the cache is full: keep the memory, the recent tokens and those of the highest weights
            fresh = Pages(n_ctx, width, 0, page)
            fresh.free = pages.free
            for ctx in range(n_ctx):
                fresh.grow(ctx, keep)
            to, to_score = fresh.table.cuda(), torch.zeros_like(score)
            kept = torch.empty(n_ctx, n_layers, n_kv, keep, dtype=torch.int32, device="cuda")
            mone.mone_cache_evict(h, mone.MONE_ALL_LAYERS, mone.make_cache(*pool, table, lens, score), keep, n_mem, recent, to, to_score, kept,
                                  new_lens)
            pages.replace(fresh)
            table, score, lens, new_lens, length, cuts = to, to_score, new_lens, lens, keep, cuts + 1
            if check:
                at = kept.long()[..., None].expand(-1, -1, -1, -1, hd)
                held = [x.gather(3, at) for x in held]
        length += 1
        if any([pages.grow(ctx, length) for ctx in range(n_ctx)]):
            table.copy_(pages.table)
        k, v, q = bf(n_ctx, n_layers, n_kv, 1, hd), bf(n_ctx, n_layers, n_kv, 1, hd), bf(n_ctx, n_layers, n_q, 1, hd)
        y = torch.empty_like(q)
        before, after = mone.make_cache(*pool, table, lens, score), mone.make_cache(*pool, table, new_lens, score)
        for layer in range(n_layers):  # as a backbone runs: a layer's projections need the layer before
            kl, vl, ql, yl = (x[:, layer].contiguous() for x in (k, v, q, y))
            mone.mone_cache_append(h, layer, before, kl, vl, (kl.stride(0), 0, kl.stride(1), kl.stride(2)), 1, new_lens)
            mone.mone_cache_attention(h, layer, after, ql, n_q, 1, n_mem, ALL, yl)
            y[:, layer] = yl
        lens, new_lens = new_lens, lens
        if check:
            held = [torch.cat([x, n], 3) for x, n in zip(held, (k, v))]
            worst = max(worst, _token_error(q, *held, y))
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    return cuts, worst


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def _softmax(q, k, v, hidden=None):
    """q [.., heads, rows, hd] over k, v [.., KV heads, positions, hd] in 64 bits."""
    group = q.shape[2] // k.shape[2]
    k, v = (x.double().repeat_interleave(group, 2) for x in (k, v))
    z = q.double() @ k.transpose(-1, -2) / q.shape[-1] ** 0.5
    return torch.softmax(z if hidden is None else z.masked_fill(hidden, -float("inf")), -1) @ v


def _prompt_error(Q, K, V, out, n_mem, window):
    t, j = n_mem + torch.arange(Q.shape[3], device="cuda")[:, None], torch.arange(K.shape[3], device="cuda")
    return _rel(out, _softmax(Q, K, V, (j > t) | ((j >= n_mem) & (j <= t - window))))


def _token_error(q, K, V, y):
    return _rel(y, _softmax(q, K, V))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--check", action="store_true", help="recompute the outputs in 64 bits")
    cuts, worst = serve(check=ap.parse_args().check)
    print(f"decoded 60 tokens over a cache cut {cuts} times" + (f"; largest relative error {worst:.1e}" if worst else ""))
