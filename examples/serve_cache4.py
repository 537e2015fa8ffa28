"""Serving with a 4-bit cache whose pages live on the GPU: a prompt's queries and keys are normalised and rotated, its keys and values go
into 4-bit pages, and a captured step decodes token after token: pages from the free list, rotation, append, attention.  When the contexts
have grown to their limit the cache is cut down into fresh pages and the old ones go back to the list.

    python examples/serve_cache4.py [--check]

Nothing that a step depends on is on the host, so one graph serves contexts that grow into new pages.  The backbone is not part of the
library, so its per-layer projections are random numbers here; --check recomputes outputs in 64 bits from what the cache holds.
"""
import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2608_17616_gb300 as mone  # noqa: E402

ALL = 1 << 30  # a window that hides nothing
EVERY = mone.MONE_ALL_LAYERS


def serve(n_ctx=2, n_layers=3, n_kv=2, group=4, hd=64, n_mem=16, prompt=150, tokens=60, most=192, keep=96, recent=32, page=16,
          check=False, seed=0):
    """Learn, read, prefill and decode; returns how often the cache was cut, the free pages at the end, and with check the largest
    relative error."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf = lambda *s: rn(*s).bfloat16()  # noqa: E731
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    d_in, d_hid, d_out, n_q, C = 256, 256, 2 * n_kv * hd, group * n_kv, n_ctx * n_layers

    # the memory learns a context and gives its tokens for the prompt
    cfg = mone.make_config(n_ctx, n_layers, d_in, d_hid, d_out, n_kv, hd, 128, mone.MONE_BF16, mone.MONE_PLAIN, 1e-2)
    h = mone.mone_mem_init(cfg, rn(C, d_hid, d_in) / d_in ** 0.5, rn(C, d_hid, d_out) / d_hid ** 0.5)
    mone.mone_ttl_context(h, bf(n_ctx, n_layers, 300, d_in), bf(n_ctx, n_layers, 300, d_out // 2), bf(n_ctx, n_layers, 300, d_out // 2), 300)
    first = n_mem + prompt
    K, V = bf(n_ctx, n_layers, n_kv, first, hd), bf(n_ctx, n_layers, n_kv, first, hd)
    mone.mone_mem_generate_kv(h, bf(n_ctx, n_layers, n_mem, d_in), n_mem, K, V, K.stride()[:4])  # positions 0 .. n_mem - 1, not rotated

    # the prompt's queries and keys, as the projections leave them (token after token), normalised and rotated: keys to their place
    rotary = mone.make_rotary(hd, mone.MONE_ROTATE_HALVES, base=10000.0)
    wq, wk = (1 + 0.1 * rn(n_layers, hd) for _ in range(2))
    x = bf(n_ctx, n_layers, prompt, n_q + n_kv, hd).transpose(2, 3)
    Q, lens = torch.empty(n_ctx, n_layers, n_q, prompt, hd, dtype=torch.bfloat16, device="cuda"), ints(n_ctx)
    mone.mone_norm_rotate(h, EVERY, rotary, lens + n_mem, prompt, mone.make_heads(x[:, :, :n_q], Q, wq),
                          mone.make_heads(x[:, :, n_q:], K[..., n_mem:, :], wk))
    out = torch.empty_like(Q)
    mone.mone_window_attention(h, EVERY, Q, n_q, prompt, K, V, K.stride()[:4], n_mem, n_mem, ALL, out)

    # pages for them, from the list of free ones
    width = -(-most // page) + 1
    n_pages = n_ctx * (width + -(-keep // page))
    pools = [torch.zeros(n_layers, n_pages, n_kv, page, n, dtype=torch.uint8, device="cuda") for n in (hd // 2, hd // 2, hd // 16, hd // 16)]
    free, n_free, left = torch.arange(n_pages, dtype=torch.int32, device="cuda"), ints(1) + n_pages, ints(1)
    table, longer, granted = ints(n_ctx, width) - 1, ints(n_ctx), ints(n_ctx)
    score = torch.zeros(n_ctx, n_layers, n_kv, width * page, device="cuda")
    pages = mone.make_pages(free, n_free, table, lens, page)
    before, after = (mone.make_cache4(*pools, table, n, score) for n in (lens, longer))
    mone.mone_cache_reserve(h, pages, first, left, None, granted)
    mone.mone_cache4_append(h, EVERY, before, K, V, K.stride()[:4], first, longer, granted)
    # the last prompt tokens say which positions matter: their weights open the scores
    last = Q[..., -8:, :].contiguous()
    mone.mone_cache4_attention(h, EVERY, after, last, n_q, 8, n_mem, ALL, torch.empty_like(last))
    lens.copy_(longer)
    n_free.copy_(left)

    # a decode step of every context and layer, captured
    q, k, v, y = (torch.zeros(n_ctx, n_layers, n, 1, hd, dtype=torch.bfloat16, device="cuda") for n in (n_q, n_kv, n_kv, n_q))
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    rows = mone.make_heads(q, qr, wq), mone.make_heads(k, kr, wk)

    def step():
        mone.mone_cache_reserve(h, pages, 1, left, None, granted)
        mone.mone_norm_rotate(h, EVERY, rotary, lens, 1, *rows)
        mone.mone_cache4_append(h, EVERY, before, kr, v, kr.stride()[:4], 1, longer, granted)
        mone.mone_cache4_attention(h, EVERY, after, qr, n_q, 1, n_mem, ALL, y)
        lens.copy_(longer)
        n_free.copy_(left)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # (the call above has made the workspace)
        step()

    def cut():
        """Down to `keep` positions, in fresh pages; the old ones go back."""
        to, none, to_score = ints(n_ctx, width) - 1, ints(n_ctx), torch.zeros_like(score)
        kept = ints(n_ctx, n_layers, n_kv, keep)
        mone.mone_cache_reserve(h, mone.make_pages(free, n_free, to, none, page), keep, left)
        n_free.copy_(left)
        mone.mone_cache4_evict(h, EVERY, before, keep, n_mem, recent, to, to_score, kept, longer)
        mone.mone_cache_release(h, pages, left)
        n_free.copy_(left)
        for to_, x in ((table, to), (score, to_score), (lens, longer)):
            to_.copy_(x)

    cuts, length, worst = 0, first, 0.0
    for _ in range(tokens):
        if length == most:
            cut()
            cuts, length = cuts + 1, keep
        for x in (q, k, v):
            x.copy_(bf(*x.shape))
        graph.replay()
        length += 1
        if check:
            worst = max(worst, _step_error(h, after, length, q, k, qr, kr, (wq, wk), y, n_kv, hd))
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    return cuts, int(n_free), worst


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def _rotated(x, w, position):
    """One token's rows in 64 bits."""
    x, n = x.double(), x.shape[-1] // 2
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double()[None, :, None, None]
    f = position * 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    a, b = x[..., :n], x[..., n:]
    return torch.cat([a * f.cos() - b * f.sin(), b * f.cos() + a * f.sin()], -1)


def _step_error(h, cache, length, q, k, qr, kr, weights, y, n_kv, hd):
    """Of the rotated rows, and of the outputs over what the cache holds."""
    held = [torch.zeros(*q.shape[:2], n_kv, length, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    mone.mone_cache4_read(h, EVERY, cache, None, length, *held, held[0].stride()[:4])
    keys, values = (t.double().repeat_interleave(q.shape[2] // n_kv, 2) for t in held)
    p = torch.softmax(qr.double() @ keys.transpose(-1, -2) / math.sqrt(hd), -1)
    return max(_rel(qr, _rotated(q, weights[0], length - 1)), _rel(kr, _rotated(k, weights[1], length - 1)), _rel(y, p @ values))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--check", action="store_true", help="recompute the outputs in 64 bits")
    cuts, left, worst = serve(check=ap.parse_args().check)
    print(f"decoded 60 tokens over a 4-bit cache cut {cuts} times, {left} pages free" + (f"; largest relative error {worst:.1e}" if worst else ""))
