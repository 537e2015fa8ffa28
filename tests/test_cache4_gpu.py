"""GPU parity of the 4-bit paged cache's operators against their definitions in 64 bits.

Every position that an operator must not read holds a NaN (the scale 127): pages that no context has, the places of a page past its
context's last position, and table entries past it name no page.

Codes, scales, values read back, positions, lengths and moved rows are exact.  Attention (relative 2-norm): the cache's elements are
exact in the products.  bf16 outputs 4.4e-3: an output is off by half a step, 2^-8 of it at most, and by what its probabilities are, which
are rounded to 11 bits, 2^-11 of themselves at most.  fp32 outputs and all weights 1e-5: the score of a key is a sum of 64 or
128 products in 32 bits of queries rounded to 22, off by about 2^-22 |z| with |z| up to 15, and the weight is off by as much of itself.
"""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2608_17616_gb300 as mone
from harness import rel_fro, record

pytestmark = pytest.mark.gpu
ALL = 1 << 30
TOL = {torch.bfloat16: 4.4e-3, torch.float32: 1e-5}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_17616_gb300 import build
    build.build()
    assert torch.cuda.is_available()
    mone.lib()


def handle(n_ctx, n_layers, n_kv, hd, dtype=torch.bfloat16):
    d_out = 2 * n_kv * hd
    if dtype is torch.float32 or d_out >= 256:
        cfg = mone.make_config(n_ctx, n_layers, 128, 256, d_out, n_kv, hd, 128,
                               mone.MONE_FP32 if dtype is torch.float32 else mone.MONE_BF16, mone.MONE_PLAIN, 1e-2)
        W = torch.zeros(n_ctx * n_layers, 256, 128, device="cuda"), torch.zeros(n_ctx * n_layers, 256, d_out, device="cuda")
    else:
        cfg = mone.make_config(n_ctx, n_layers, 128, 64, 128, 1, 64, 128, mone.MONE_BF16, mone.MONE_PLAIN, 1e-2,
                               memory=mone.MONE_MEM_SWIGLU, mem_heads=2)
        W = torch.zeros(n_ctx * n_layers, 2, 128, 64, device="cuda"), torch.zeros(n_ctx * n_layers, 2, 64, 64, device="cuda")
    return mone.mone_mem_init(cfg, *W)


def packed(code):
    return (code[..., ::2] | code[..., 1::2] << 4).astype(np.uint8)


class Cache4:
    """Contexts of given lengths over scattered pages, NaN wherever nothing is held."""

    def __init__(self, lens, n_layers=2, n_kv=2, hd=64, page=16, dtype=torch.bfloat16, order="head", spare=3, seed=0, pad=0, score=True,
                 exps=(0, 0)):
        self.lens, self.L, self.n_kv, self.hd, self.page, self.dtype, self.exps = list(lens), n_layers, n_kv, hd, page, dtype, exps
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        n_ctx = len(self.lens)
        width = -(-max(max(lens), 1) // page) + spare
        P = n_ctx * width * 2 + 3
        perm = {"head": (0, 1, 2, 3, 4), "position": (0, 1, 3, 2, 4), "layers inner": (3, 0, 1, 2, 4)}[order]

        def pool(row, fill, pad):
            shape = {"head": (n_layers, P, n_kv, page, row + pad), "position": (n_layers, P, page, n_kv, row + pad),
                     "layers inner": (P, n_kv, page, n_layers, row + pad)}[order]
            return torch.full(shape, fill, dtype=torch.uint8, device="cuda").permute(*perm)[..., :row]

        self.pools = [pool(hd // 2, 0xb7, 16 * pad) for _ in range(2)] + [pool(hd // 16, 127, hd // 16 * pad) for _ in range(2)]
        pages = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        self.table = pages[:n_ctx * width].view(n_ctx, width).clone()
        self.fresh = pages[n_ctx * width:2 * n_ctx * width].view(n_ctx, width).clone()
        self.len_t = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.k, self.v = [], []  # values [layers, heads, n, hd] in 64 bits
        self.rows = []           # of each context: codes and scales of its keys and values
        for c, n in enumerate(self.lens):
            both = [O.four_bits(torch.randn(n_layers, n_kv, n, hd, generator=g, device="cuda").double().cpu().numpy() * 2.0 ** e, e) for e in exps]
            self.k.append(O.four_bit_values(*both[0], exps[0]))
            self.v.append(O.four_bit_values(*both[1], exps[1]))
            self.rows.append([packed(both[0][0]), packed(both[1][0]), both[0][1], both[1][1]])
            for p, r in zip(self.pools, self.rows[c]):
                self.put(p, c, torch.from_numpy(r).cuda())
        self.score = torch.rand(n_ctx, n_layers, n_kv, width * page, generator=g, device="cuda") if score else None
        self.h = handle(n_ctx, n_layers, n_kv, hd, dtype)
        self.tbl = self.table.clone()
        self.trim(self.tbl, self.lens)
        self.c = self.cache(self.tbl, self.len_t, self.score)

    def cache(self, table, lens, score=None):
        return mone.make_cache4(*self.pools, table, lens, score, *self.exps)

    def trim(self, table, lens):
        for c, n in enumerate(lens):
            table[c, -(-n // self.page):] = -7

    def put(self, pool, c, rows):
        for i in range(0, rows.shape[2], self.page):
            r = rows[:, :, i:i + self.page]
            pool[:, self.table[c, i // self.page].item(), :, :r.shape[2]] = r

    def held(self, pool, c, n, table=None):
        t = (self.table if table is None else table)[c].tolist()
        return torch.cat([pool[:, p] for p in t[:max(1, -(-n // self.page))]], 2)[:, :, :n]

    def values(self, c, n, table=None):
        """Keys and values of a context's first n positions, from the pools, in 64 bits."""
        out = []
        for i, e in enumerate(self.exps):
            code, scale = (self.held(self.pools[i + j], c, n, table).cpu().numpy() for j in (0, 2))
            out.append(O.four_bit_values(np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], self.hd), scale, e))
        return out

    def done(self):
        mone.mone_mem_sync(self.h)

    def __del__(self):
        if getattr(self, "h", None):
            mone.mone_mem_free(self.h)


def attend(x, group, n_tok, n_sink, window, layer=-1, scale=1.0, k=None, v=None):
    layers = range(x.L) if layer < 0 else [layer]
    n_q, B = group * x.n_kv, len(x.lens)
    Q = (scale * torch.randn(B, len(layers), n_q, n_tok, x.hd, generator=x.g, device="cuda")).to(x.dtype)
    out = torch.full_like(Q, 7.0)
    before = None if x.score is None else x.score.clone()
    mone.mone_cache4_attention(x.h, layer, x.c, Q, n_q, n_tok, n_sink, window, out)
    x.done()
    want = None if before is None else before.double().cpu()
    for c, n in enumerate(x.lens):
        ref = torch.zeros(out[c].shape, dtype=torch.float64)
        for i, l in enumerate(layers):
            o, w = O.window_attention(Q[c, i].float().cpu(), x.k[c][l], x.v[c][l], n - n_tok, n_sink, window)
            ref[i] = torch.from_numpy(o)
            if want is not None and n:
                want[c, l, :, :n] += torch.from_numpy(w)
        if ref.any():
            assert record("4-bit cache attention", f"out {str(x.dtype)[6:]}", rel_fro(out[c].float().cpu(), ref), TOL[x.dtype]) <= TOL[x.dtype], c
        assert not out[c].float().cpu()[ref.abs().amax(-1) == 0].any(), c  # tokens that see nothing
    if want is not None:
        assert record("4-bit cache attention", "weights", rel_fro(x.score.cpu(), want), 1e-5) <= 1e-5
        same = want == before.double().cpu()
        assert torch.equal(x.score.cpu()[same], before.cpu()[same])  # positions that no token sees
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,group,n_tok,hd,page,n_sink,window", [
    ([1], 1, 1, 64, 16, 0, ALL),                 # one position
    ([0, 1, 2, 0, 300], 4, 1, 64, 16, 0, ALL),     # contexts that hold nothing
    ([31, 32, 33, 63, 64, 65], 4, 1, 64, 32, 0, ALL),
    ([15, 16, 17, 47, 48, 49], 4, 1, 128, 8, 0, ALL),
    ([255, 256, 257, 600], 2, 1, 128, 64, 0, ALL),
    ([4000], 8, 1, 64, 16, 0, ALL),              # one item over many CTAs
    ([3001, 17, 900], 5, 3, 128, 8, 0, ALL),        # 15 rows, causal among the new tokens
    ([5, 2, 700], 3, 6, 64, 16, 0, ALL),           # 18 rows; contexts with fewer positions than new tokens
    ([400, 90], 7, 16, 64, 16, 0, ALL),            # 112 rows
    ([33, 200], 64, 1, 64, 16, 0, ALL),           # the most heads a KV head has
    ([700, 35, 4], 4, 1, 64, 16, 4, 50),          # first positions and a window, a gap between them
    ([700, 64, 130], 4, 2, 128, 64, 33, 70),        # first positions past a block, two tokens
    ([500, 20], 2, 4, 64, 16, 0, 1),              # a window of one: every token its own position
    ([500, 20], 2, 2, 64, 16, 5, 0),              # first positions alone
    ([500, 20], 2, 2, 64, 16, 0, 0),              # nothing to see
    ([90, 10], 2, 1, 64, 16, 1000, 3),            # more first positions than there are
    ([300, 77], 4, 1, 64, 1, 0, ALL),              # pages of one position
    ([300, 2100], 4, 2, 64, 1024, 8, 999),          # pages of 1024
    ([130, 61], 4, 1, 128, 4, 3, 40),              # pages that an instruction's rows do not fit
    ([130, 61], 4, 1, 64, 8, 0, ALL),
    ([200, 64, 5], 1, 4, 128, 32, 0, ALL),          # four rows
    ([200, 64, 5], 4, 2, 64, 16, 70, 20),           # eight; first positions that end inside a block
    ([500, 96], 8, 2, 128, 32, 32, 64),             # sixteen; a window that begins where a block does
    ([97], 3, 3, 64, 2, 32, 1),                    # nine
])
def test_attention(lens, group, n_tok, hd, page, n_sink, window, dtype):
    x = Cache4(lens, hd=hd, page=page, dtype=dtype, seed=sum(lens) + group)
    attend(x, group, n_tok, n_sink, window)
    attend(x, group, n_tok, n_sink, window, scale=4.0)  # again on the same workspace, with steeper softmaxes


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,group,n_tok,hd,page,n_sink,window", [
    ([0, 1, 2, 0, 300], 4, 1, 64, 16, 0, ALL),
    ([255, 256, 257, 600], 2, 1, 128, 64, 0, ALL),
    ([3001, 17, 900], 5, 3, 128, 8, 0, ALL),
    ([400, 90], 7, 16, 64, 16, 0, ALL),
    ([9000, 30], 4, 1, 64, 16, 100, 7000),
    ([9000, 500, 6700], 4, 3, 128, 64, 33, 6500),
    ([300, 77], 4, 1, 64, 1, 0, ALL),
])
def test_attention_where_tables_could_hold_much(lens, group, n_tok, hd, page, n_sink, window, dtype):
    """A call goes by what its tables and its window allow: dealt out here, though the contexts are short."""
    x = Cache4(lens, hd=hd, page=page, dtype=dtype, seed=sum(lens) + group, spare=16384 // page)
    attend(x, group, n_tok, n_sink, window)
    attend(x, group, n_tok, n_sink, window, scale=4.0)


@pytest.mark.parametrize("n_layers,lens", [(10, [700, 1500, 90]), (20, [300, 0, 77, 130, 1, 200]), (1, [1000]), (20, [33, 32, 31, 64, 65, 1])])
@pytest.mark.parametrize("group,n_tok,hd,n_sink,window", [(4, 1, 64, 0, ALL), (4, 1, 128, 40, 300), (3, 5, 64, 0, ALL), (2, 4, 64, 3, 33)])
def test_attention_by_clusters_of_every_size(n_layers, lens, group, n_tok, hd, n_sink, window):
    attend(Cache4(lens, n_layers=n_layers, hd=hd, page=32, seed=n_layers), group, n_tok, n_sink, window)


@pytest.mark.parametrize("n_layers,n_kv,lens,group,n_tok,page,spare", [
    (16, 8, [700, 3, 33, 0, 1, 200], 4, 1, 16, 0),     # two layers a group
    (7, 6, [700, 2100], 4, 1, 16, 600),                # an item a group
    (25, 10, [90, 600, 5], 2, 1, 32, 0),               # five layers a group
    (2, 6, [1200, 0, 31], 3, 7, 16, 1000),             # row tiles
    (1, 8, [300], 20, 16, 16, 2000),                   # more row tiles than a group could have a CTA each
    (19, 4, [40] * 5 + [0] * 9 + [1500], 4, 2, 64, 0),
])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["head", "position"])
def test_attention_dealt_out_in_groups(n_layers, n_kv, lens, group, n_tok, page, spare, order, dtype):
    attend(Cache4(lens, n_layers=n_layers, n_kv=n_kv, hd=64, page=page, dtype=dtype, order=order, spare=spare, seed=n_kv), group, n_tok, 0, ALL)


@pytest.mark.parametrize("length,window", [(17000, ALL), (17000, 16500), (300, ALL)])
@pytest.mark.parametrize("dtype,n_tok", [(torch.bfloat16, 1), (torch.bfloat16, 4), (torch.float32, 2)])
def test_one_context_whose_clusters_would_leave_the_gpu_idle(length, window, dtype, n_tok):
    attend(Cache4([length], n_layers=5, n_kv=8, hd=64, page=64, dtype=dtype, spare=(17000 - length) // 64, score=n_tok != 4), 2, n_tok, 5, window)


@pytest.mark.parametrize("order,pad", [("position", 0), ("layers inner", 0), ("head", 1), ("position", 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_over_other_strides(order, pad, dtype, hd):
    x = Cache4([70, 513], n_layers=3, hd=hd, dtype=dtype, order=order, pad=pad)
    attend(x, 4, 2, 3, 200)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("exps,scale", [((3, -4), 1.0), ((-20, 20), 2.0 ** 20), ((60, -60), 2.0 ** -60), ((30, 30), 2.0 ** -30), ((-64, 64), 2.0 ** 64)])
def test_attention_of_other_ranges(exps, scale, dtype):
    """Powers of two on keys, values and queries that leave the scores where they are."""
    x = Cache4([130, 600], dtype=dtype, exps=exps, seed=2)
    attend(x, 4, 2, 0, ALL, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_queries_of_unequal_sizes(dtype):
    """Rows of very different sizes, zeros, and elements of very different sizes in a row: each by its own range."""
    x = Cache4([300, 70], dtype=dtype, seed=4)
    Q = torch.randn(2, 2, 8, 2, 64, generator=x.g, device="cuda")
    Q *= 2.0 ** torch.randint(-130, 4, (2, 2, 8, 2, 1), generator=x.g, device="cuda").float()
    Q[:, :, 3] = 0
    Q[:, :, 5, :, ::3] *= 2.0 ** -25
    Q = Q.to(dtype)
    out = torch.full_like(Q, 7.0)
    mone.mone_cache4_attention(x.h, -1, x.c, Q, 8, 2, 0, ALL, out)
    x.done()
    for c, n in enumerate(x.lens):
        for l in range(2):
            ref, _ = O.window_attention(Q[c, l].double().cpu(), x.k[c][l], x.v[c][l], n - 2, 0, ALL)
            for r in range(8):
                assert rel_fro(out[c, l, r].float().cpu(), ref[r]) <= TOL[dtype]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_small_weights_beside_a_large_one(dtype):
    """One key takes 1 - 2^-3 of the weight, 20000 others 2^-17 of it each: less than fp16 holds next to 1."""
    x = Cache4([20001], n_layers=1, n_kv=2, dtype=dtype, score=True, seed=8)
    hot = 7777
    key = np.zeros((1, 2, 20001, 64))
    key[:, :, hot, 0] = 6.0
    val = np.ones((1, 2, 20001, 64)) * 6.0
    val[:, :, hot] = 0.75
    for i, t in ((0, key), (1, val)):
        code, scale = O.four_bits(t)
        x.put(x.pools[i], 0, torch.from_numpy(packed(code)).cuda())
        x.put(x.pools[i + 2], 0, torch.from_numpy(scale).cuda())
        assert np.array_equal(O.four_bit_values(code, scale), t)
    x.k, x.v = [key], [val]
    Q = torch.zeros(1, 1, 4, 1, 64, device="cuda")
    Q[..., 0] = 8 * np.log(20000 * 7) / 6.0
    Q = Q.to(dtype)
    out, before = torch.empty_like(Q), x.score.double().cpu()
    mone.mone_cache4_attention(x.h, 0, x.c, Q, 4, 1, 0, ALL, out)
    x.done()
    ref, w = O.window_attention(Q[0, 0].float().cpu(), key[0], val[0], 20000, 0, ALL)
    assert rel_fro(out[0, 0].float().cpu(), ref) <= TOL[dtype]
    assert rel_fro(x.score[0, 0, :, :20001].cpu(), before[0, 0, :, :20001] + torch.from_numpy(w)) <= 1e-5


@pytest.mark.parametrize("layer", [0, 2])
def test_one_layer(layer):
    attend(Cache4([70, 513, 4], n_layers=3), 4, 1, 0, ALL, layer=layer)


def test_one_head_of_64_and_no_weights():
    attend(Cache4([700, 3], n_kv=1, score=False), 5, 1, 2, 300)


def test_more_contexts_than_a_warp_and_a_long_one():
    attend(Cache4([(37 * i) % 90 for i in range(70)] + [20000], n_layers=1, page=32), 4, 1, 0, ALL)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_non_finite_values_reach_only_the_tokens_that_see_them(dtype):
    x = Cache4([200], dtype=dtype, score=False)
    n_tok, window = 4, 50
    Q = torch.randn(1, 2, 4, n_tok, 64, generator=x.g, device="cuda").to(dtype)
    for pos in (199, 198, 147, 148):  # the last tokens' own positions, and the two that only the older tokens see
        scale, v = x.rows[0][3].copy(), x.v[0].copy()
        scale[:, :, pos, 1], v[:, :, pos, 16:32] = 127, np.nan
        x.put(x.pools[3], 0, torch.from_numpy(scale).cuda())
        out = torch.full_like(Q, 7.0)
        mone.mone_cache4_attention(x.h, -1, x.c, Q, 4, n_tok, 3, window, out)
        x.done()
        for l in range(2):
            ref, _ = O.window_attention(Q[0, l].float().cpu(), x.k[0][l], v[l], 196, 3, window)
            ref = torch.from_numpy(ref)
            fine, got = ref.isfinite(), out[0, l].float().cpu()
            assert fine.any() and not fine.all()
            assert torch.equal(got.isfinite(), fine)
            assert rel_fro(got[fine], ref[fine]) <= TOL[dtype]
        x.put(x.pools[3], 0, torch.from_numpy(x.rows[0][3]).cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,spare,n_tok,bad", [
    ([200], 3, 4, slice(199, 200)),        # the newest token's key alone
    ([300, 40], 3, 3, slice(2, 3)),        # one that all see
    ([9000], 1024, 1, slice(1024, 8064)),   # dealt out: parts that hold no other score
    ([900], 3, 1, slice(100, 800)),        # a cluster's
])
def test_weights_of_tokens_whose_scores_are_not_numbers(lens, spare, n_tok, bad, dtype):
    x = Cache4(lens, dtype=dtype, spare=spare, seed=len(lens))
    window = 50 if n_tok > 1 else ALL
    scale = x.rows[0][2].copy()
    scale[:, :, bad], x.k[0][:, :, bad] = 127, np.nan
    x.put(x.pools[2], 0, torch.from_numpy(scale).cuda())
    Q = torch.randn(len(lens), 2, 8, n_tok, 64, generator=x.g, device="cuda").to(dtype)
    out, want = torch.full_like(Q, 7.0), x.score.double().cpu()
    mone.mone_cache4_attention(x.h, -1, x.c, Q, 8, n_tok, 3, window, out)
    x.done()
    for c, n in enumerate(lens):
        for l in range(2):
            ref, w = O.window_attention(Q[c, l].float().cpu(), x.k[c][l], x.v[c][l], n - n_tok, 3, window)
            want[c, l, :, :n] += torch.from_numpy(w)
            assert torch.equal(out[c, l].isnan().cpu(), torch.from_numpy(ref).isnan())
    got = x.score.cpu()
    assert torch.equal(got.isnan(), want.isnan()) and want.isnan().any()
    assert rel_fro(got.nan_to_num(), want.nan_to_num()) <= 1e-5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group,spare", [(4, 3), (8, 3), (4, 2000)])
def test_a_row_does_not_hang_on_the_others(group, spare, dtype):
    """The bits of a head's output and no other's sizes, nor whether they are numbers."""
    x = Cache4([900, 77], dtype=dtype, score=False, spare=spare, seed=3)
    Q = torch.randn(2, 2, 2 * group, 1, 64, generator=x.g, device="cuda").to(dtype)
    other, outs = Q.clone(), []
    other[:, :, 1] *= 100
    other[:, :, 2] = float("nan")
    other[:, :, group - 1] = float("inf")
    other[:, :, group + 1] = 0
    for q in (Q, other):
        outs.append(torch.empty_like(q))
        mone.mone_cache4_attention(x.h, -1, x.c, q, 2 * group, 1, 0, ALL, outs[-1])
    x.done()
    same = [i for i in range(2 * group) if i not in (1, 2, group - 1, group + 1)]
    assert torch.equal(outs[0][:, :, same], outs[1][:, :, same])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_that_are_not_finite(dtype):
    """A NaN's row is NaN; an infinity's is what the formula gives: NaN, or where every seen key's score is -inf, 0."""
    x = Cache4([150], n_layers=1, dtype=dtype, score=False, seed=1)
    code, scale = O.four_bits(np.where(np.abs(x.k[0]) < 0.3, 0.5, np.abs(x.k[0])))  # keys without a zero, all positive
    x.k[0] = O.four_bit_values(code, scale)
    x.put(x.pools[0], 0, torch.from_numpy(packed(code)).cuda())
    x.put(x.pools[2], 0, torch.from_numpy(scale).cuda())
    seen = (x.k[0] > 0).all()
    Q = torch.randn(1, 1, 8, 1, 64, generator=x.g, device="cuda")
    Q[0, 0, 1, 0, 5], Q[0, 0, 2, 0, 9], Q[0, 0, 6, 0, 9] = float("nan"), float("inf"), -float("inf")
    Q = Q.to(dtype)
    out = torch.full_like(Q, 7.0)
    mone.mone_cache4_attention(x.h, 0, x.c, Q, 8, 1, 0, ALL, out)
    x.done()
    got = out[0, 0, :, 0].float().cpu()
    assert seen
    assert got[1].isnan().all() and got[2].isnan().all() and not got[6].any()
    ref, _ = O.window_attention(Q[0, 0].float().cpu(), x.k[0][0], x.v[0][0], 149, 0, ALL)
    rest = [0, 3, 4, 5, 7]
    assert rel_fro(got[rest], ref[rest, 0]) <= TOL[dtype]


def test_pages_and_lengths_out_of_range_are_latched_and_skipped():
    x = Cache4([100, 60])
    Q = torch.randn(2, 2, 4, 1, 64, generator=x.g, device="cuda").bfloat16()
    out, K = torch.empty_like(Q), torch.zeros(2, 2, 2, 120, 64, dtype=torch.bfloat16, device="cuda")

    def fails(what, call):
        call()
        with pytest.raises(mone.MoneError) as e:
            x.done()
        assert e.value.code == 8 and what in str(e.value)

    def attention():
        mone.mone_cache4_attention(x.h, -1, x.c, Q, 4, 1, 0, ALL, out)

    def read():
        mone.mone_cache4_read(x.h, -1, x.c, None, 120, K, K.clone(), K.stride()[:4])

    for bad in (-1, x.pools[0].shape[1], 1 << 30):
        keep = x.tbl.clone()
        x.tbl[0, 2] = bad
        fails("page", attention)
        fails("page", read)
        x.tbl.copy_(keep)
    for bad in (-1, x.tbl.shape[1] * x.page + 1):
        x.tbl.copy_(x.table)
        x.len_t[0] = bad
        fails("length", attention)
        fails("length", read)
    x.len_t[0] = 100
    k = torch.randn(2, 2, 2, 200, 64, device="cuda").bfloat16()
    fails("length", lambda: mone.mone_cache4_append(x.h, -1, x.c, k, k, k.stride()[:4], 200))  # past the table's end


def test_calls_of_changing_sizes_and_of_both_caches_share_a_workspace_and_repeat_bit_for_bit():
    x = Cache4([5000, 130, 1], n_layers=1, score=False)
    P, width = x.pools[0].shape[1], x.tbl.shape[1]
    dense = [torch.randn(1, P, 2, 16, 64, generator=x.g, device="cuda").bfloat16() for _ in range(2)]
    score = torch.zeros(3, 1, 2, width * 16, device="cuda")
    both = mone.make_cache(*dense, x.tbl, x.len_t, score)
    q1, q2 = (torch.randn(3, 1, 8, n, 64, generator=x.g, device="cuda").bfloat16() for n in (1, 5))
    outs = [[], [], []]
    for _ in range(4):
        for q, o in ((q1, outs[0]), (q2, outs[1])):
            o.append(torch.empty_like(q))
            mone.mone_cache4_attention(x.h, 0, x.c, q, 8, q.shape[3], 0, ALL, o[-1])
            outs[2].append(torch.empty_like(q1))
            mone.mone_cache_attention(x.h, 0, both, q1, 8, 1, 0, ALL, outs[2][-1])
    x.done()
    for o in outs:
        assert all(torch.equal(o[0], y) for y in o[1:])
    ref, _ = O.window_attention(q1[0, 0].float().cpu(), x.k[0][0], x.v[0][0], 4999, 0, ALL)
    assert rel_fro(outs[0][0][0, 0].float().cpu(), ref) <= TOL[torch.bfloat16]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_graph_is_replayed_after_larger_calls(dtype):
    """The workspace that a graph holds stays when the handle's grows; two graphs of one handle, replayed in turn, do not disturb each other."""
    x = Cache4([300, 40], spare=40, seed=6, dtype=dtype)
    rn = lambda n_tok: torch.randn(2, 2, 8, n_tok, 64, generator=x.g, device="cuda").to(dtype)  # noqa: E731
    qs, big = [rn(1), rn(4)], rn(16)
    outs, want, graphs, score = [torch.empty_like(q) for q in qs], [], [], x.score.clone()
    for q in qs:
        want.append(torch.empty_like(q))
        mone.mone_cache4_attention(x.h, -1, x.c, q, 8, q.shape[3], 2, 100, want[-1])
    want_score = x.score.clone()
    torch.cuda.synchronize()
    for q, o in zip(qs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            mone.mone_cache4_attention(x.h, -1, x.c, q, 8, q.shape[3], 2, 100, o)
    mone.mone_cache4_attention(x.h, -1, x.c, big, 8, 16, 2, 100, torch.empty_like(big))
    junk = [torch.full((1 << 22,), float("nan"), device="cuda") for _ in range(8)]  # what would lie where the old one was
    for _ in range(3):
        x.score.copy_(score)
        for g, o in zip(graphs, outs):
            o.zero_()
            g.replay()
    x.done()
    assert all(torch.equal(a, b) for a, b in zip(outs, want)) and torch.equal(x.score, want_score) and all(j.isnan().all() for j in junk)


def test_on_another_stream():
    x = Cache4([900, 40])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        attend(x, 4, 1, 0, ALL)


# ----------------------------------------------------------------- append and read

def rows_for_rounding(shape, g, exp):
    """Rows of many sizes: normal ones, zeros, ties of codes and of scales, tiny and huge ones, infinities and NaN."""
    x = torch.randn(*shape, generator=g, device="cuda")
    x *= 2.0 ** torch.randint(-14, 14, (*shape[:-1], 1), generator=g, device="cuda").float()
    pick = torch.randint(0, 9, shape[:-1], generator=g, device="cuda")
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0], device="cuda")
    x[pick == 1] = 0.0
    x[pick == 2] = ties.repeat(shape[-1] // 16)
    # scales halfway between two e4m3 numbers: 6 x (1 + (2 m + 1) / 16)
    x[pick == 3] = (6 * (1 + (2 * torch.arange(shape[-1] // 16, device="cuda") + 1) / 16)).repeat_interleave(16) * ties.repeat(shape[-1] // 16).sign()
    x[pick == 4] *= 1e-5
    x[pick == 5] *= 1e4
    x[pick == 6, 3] = float("inf")
    x[pick == 7, -1] = float("nan")
    return x * 2.0 ** exp


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,n_tok,page,order,pad,counts,layer,hd,exps", [
    ([0], 1, 16, "head", 0, None, -1, 64, (0, 0)),
    ([15, 16, 17, 0], 1, 16, "head", 0, None, -1, 128, (0, 0)),
    ([15, 16, 17, 0], 33, 16, "position", 0, None, 1, 64, (3, -5)),
    ([100, 7], 500, 64, "head", 0, [500, 0], -1, 64, (0, 0)),       # a prompt for one context, nothing for the other
    ([9, 30], 10001, 64, "head", 0, [10001, 9000], -1, 128, (0, 2)),  # many
    ([100, 7, 9], 5, 1, "head", 0, [2, 9, -3], -1, 64, (0, 64)),      # counts past the tokens that there are, pages of one
    ([100, 7], 20, 16, "head", 3, None, -1, 128, (-64, 0)),
    ([3], 20, 8, "layers inner", 1, None, 0, 64, (0, 0)),
])
@pytest.mark.parametrize("skew", [0, 1])  # rows of the tokens that are not aligned to 16 bytes
def test_append_and_read(lens, n_tok, page, order, pad, counts, layer, hd, exps, skew, dtype):
    x = Cache4(lens, page=page, hd=hd, dtype=dtype, order=order, pad=pad, spare=-(-n_tok // page) + 1, exps=exps)
    count = [n_tok if counts is None else min(max(counts[c], 0), n_tok) for c in range(len(lens))]
    after = [n + k for n, k in zip(lens, count)]
    x.tbl.copy_(x.table)
    x.trim(x.tbl, after)
    layers = list(range(x.L)) if layer < 0 else [layer]
    # tokens with the heads inside, a strided view
    k, v = (rows_for_rounding((len(lens), len(layers), n_tok, x.n_kv, hd + 16), x.g, e).to(dtype)[..., skew:hd + skew].transpose(2, 3) for e in exps)
    out = torch.full_like(x.len_t, -5)
    before, s0 = [p.clone() for p in x.pools], x.score.clone()
    mone.mone_cache4_append(x.h, layer, x.c, k, v, k.stride()[:4], n_tok, out,
                            None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    x.done()
    assert out.tolist() == after
    new = [O.four_bits(t.double().cpu().numpy(), e) for t, e in zip((k, v), exps)]
    for i, pool in enumerate(x.pools):
        rows = packed(new[i][0]) if i < 2 else new[i - 2][1]
        want = before[i].cpu().numpy()
        for c, n in enumerate(lens):
            for j in range(count[c]):
                for a, l in enumerate(layers):
                    want[l, x.table[c, (n + j) // page].item(), :, (n + j) % page] = rows[c, a, :, j]
        got = pool.cpu().numpy()
        if i < 2:  # codes of groups that are NaN say nothing
            nan = np.repeat(x.pools[i + 2].cpu().numpy() == 127, 8, -1)
            got, want = np.where(nan, 0, got), np.where(nan, 0, want)
        assert np.array_equal(got, want), i
    for c, n in enumerate(lens):
        for l in layers:
            s0[c, l, :, n:n + count[c]] = 0
    assert torch.equal(x.score, s0)
    # back: from the middle of what was held, past the end
    at = [max(0, n - 3) for n in lens]
    n_pos = n_tok + 7
    K, V = (torch.full((len(lens), len(layers), n_pos, x.n_kv, hd + 16), 7.0, device="cuda").to(dtype)[..., skew:hd + skew].transpose(2, 3) for _ in range(2))
    mone.mone_cache4_read(x.h, layer, x.cache(x.tbl, out), torch.tensor(at, dtype=torch.int32, device="cuda"), n_pos, K, V, K.stride()[:4])
    x.done()
    for c in range(len(lens)):
        got, held = [t[c].double().cpu().numpy() for t in (K, V)], x.values(c, after[c])
        for g, w in zip(got, held):
            m = min(after[c] - at[c], n_pos)
            assert np.array_equal(g[:, :, :m], w[layers][:, :, at[c]:at[c] + m], equal_nan=True)
            assert (g[:, :, m:] == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rounding_next_to_every_tie(dtype):
    """Of every scale: groups whose largest element makes it, and elements on the ties between codes and up to three steps of the type beside
    them; and groups whose largest element lies on the ties between two scales and beside them."""
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    info, bits = (np.int32, 0) if dtype is torch.float32 else (np.int32, 16)

    def steps(v, k):  # k steps of the type away from zero
        return (v.astype(np.float32).view(info) + (k << bits)).view(np.float32)

    rows = []
    for s in O.E4M3[1:]:
        for k in range(-3, 4):
            for sign in (1.0, -1.0):
                g = np.full(16, 6.0 * s, dtype=np.float32)
                g[1:8], g[8:15] = steps(ties * s, k), steps(ties * s, -k)
                rows.append(np.float32(sign) * g)
    for lo, hi in zip(O.E4M3[1:], O.E4M3[2:]):
        for k in range(-3, 4):
            rows.append(np.full(16, 1.0, dtype=np.float32) * steps(np.array([6 * (lo + hi) / 2]), k))
    x = np.concatenate(rows)
    n = len(x) // 64
    x = x[:n * 64].reshape(1, 1, 1, n, 64)
    h = handle(1, 1, 2, 64, dtype)
    pages = -(-n // 16)
    pools = [torch.zeros(1, pages, 2, 16, w, dtype=torch.uint8, device="cuda") for w in (32, 32, 4, 4)]
    table, lens = torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.zeros(1, dtype=torch.int32, device="cuda")
    k = torch.from_numpy(x.copy()).cuda().to(dtype).expand(1, 1, 2, n, 64).contiguous()
    v = -k.flip(-1)
    mone.mone_cache4_append(h, -1, mone.make_cache4(*pools, table, lens), k, v, k.stride()[:4], n)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    for i, t in enumerate((k, v)):
        code, scale = O.four_bits(t[0, 0].double().cpu().numpy())
        for pool, want in ((pools[i], packed(code)), (pools[i + 2], scale)):
            got = pool[0].transpose(0, 1).reshape(2, pages * 16, -1)[:, :n].cpu().numpy()
            assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def test_read_of_everything_and_of_nothing():
    x = Cache4([90, 0, 33], n_layers=3)
    K, V = (torch.full((3, 3, 2, 100, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mone.mone_cache4_read(x.h, -1, x.c, None, 100, K, V, K.stride()[:4])
    x.done()
    for c, n in enumerate(x.lens):
        assert np.array_equal(K[c, :, :, :n].double().cpu().numpy(), x.k[c]) and np.array_equal(V[c, :, :, :n].double().cpu().numpy(), x.v[c])
        assert (K[c, :, :, n:] == 7).all() and (V[c, :, :, n:] == 7).all()
    mone.mone_cache4_read(x.h, -1, x.c, torch.full((3,), 2 ** 31 - 1, dtype=torch.int32, device="cuda"), 100, K, V, K.stride()[:4])
    x.done()
    assert np.array_equal(K[0, :, :, :90].double().cpu().numpy(), x.k[0])


# ----------------------------------------------------------------- eviction

@pytest.mark.parametrize("lens,keep,n_sink,n_recent,page,hd,order,pad,layer", [
    ([1, 0, 2], 1, 0, 0, 16, 64, "head", 0, -1),
    ([50, 51, 100, 3], 50, 4, 10, 16, 64, "head", 0, -1),     # all kept; one goes; half goes
    ([3000, 700, 1], 333, 0, 0, 8, 128, "position", 0, -1),
    ([2000], 1999, 1, 1, 16, 64, "head", 0, -1),
    ([500, 40], 37, 5, 7, 1, 128, "head", 3, -1),
    ([300, 20, 90], 80, 4, 8, 16, 64, "layers inner", 0, 1),
])
def test_evict(lens, keep, n_sink, n_recent, page, hd, order, pad, layer):
    x = Cache4(lens, page=page, hd=hd, order=order, pad=pad, seed=keep)
    layers = list(range(x.L)) if layer < 0 else [layer]
    B, n_to = len(lens), -(-keep // page)
    to = x.fresh[:, :n_to].contiguous()
    x.trim(to, [min(n, keep) for n in lens])  # entries past the survivors name no page
    to_score = torch.full((B, x.L, x.n_kv, n_to * page), -3.0, device="cuda")
    kept = torch.full((B, len(layers), x.n_kv, keep), -9, dtype=torch.int32, device="cuda")
    out = torch.full_like(x.len_t, -5)
    mone.mone_cache4_evict(x.h, layer, x.c, keep, n_sink, n_recent, to, to_score, kept, out)
    x.done()
    assert out.tolist() == [min(n, keep) for n in lens]
    for c, n in enumerate(lens):
        m = min(n, keep)
        for a, l in enumerate(layers):
            for g in range(x.n_kv):
                at = O.cache_keep(x.score[c, l, g, :n].cpu(), keep, n_sink, n_recent)
                assert kept[c, a, g].tolist() == at.tolist() + [-1] * (keep - m)
                assert to_score[c, l, g].tolist() == x.score[c, l, g, torch.from_numpy(at).cuda()].tolist() + [-3.0] * (n_to * page - m)
                for i, p in enumerate(x.pools):
                    if m:
                        assert np.array_equal(x.held(p, c, m, to)[l, g].cpu().numpy(), x.rows[c][i][l, g, at])
        for i, p in enumerate(x.pools):
            assert np.array_equal(x.held(p, c, n).cpu().numpy(), x.rows[c][i])  # the old pages
    for l in set(range(x.L)) - set(layers):
        assert (to_score[:, l] == -3.0).all()


# ----------------------------------------------------------------- offsets past 32 bits

@pytest.mark.parametrize("hd", [64, 128])
def test_pools_and_offsets_past_32_bits(hd):
    page, n_kv = 64, 2
    n_pages = (1 << 32) // (page * n_kv * hd // 2) + 40
    pools = [torch.empty(1, n_pages, n_kv, page, w, dtype=torch.uint8, device="cuda") for w in (hd // 2, hd // 2, hd // 16, hd // 16)]
    h = handle(1, 1, n_kv, hd)
    g = torch.Generator(device="cuda").manual_seed(5)
    n = 300
    far = torch.tensor([[n_pages - 1, n_pages - 2, n_pages - 30, 3, n_pages - 7, n_pages - 9]], dtype=torch.int32, device="cuda")
    lens, out_lens = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    score = torch.zeros(1, 1, n_kv, 6 * page, device="cuda")
    k, v = (torch.randn(1, 1, n_kv, n, hd, generator=g, device="cuda").bfloat16() for _ in range(2))
    mone.mone_cache4_append(h, -1, mone.make_cache4(*pools, far, lens, score), k, v, k.stride()[:4], n, out_lens)
    q = torch.randn(1, 1, 4 * n_kv, 1, hd, generator=g, device="cuda").bfloat16()
    out, c = torch.empty_like(q), mone.make_cache4(*pools, far, out_lens, score)
    mone.mone_cache4_attention(h, -1, c, q, 4 * n_kv, 1, 0, ALL, out)
    kq, vq = (O.four_bit_values(*O.four_bits(t[0, 0].double().cpu().numpy())) for t in (k, v))
    ref, w = O.window_attention(q[0, 0].float().cpu(), kq, vq, n - 1, 0, ALL)
    to = torch.tensor([[n_pages - 3, n_pages - 5]], dtype=torch.int32, device="cuda")
    to_score, kept = torch.zeros(1, 1, n_kv, 2 * page, device="cuda"), torch.empty(1, 1, n_kv, 100, dtype=torch.int32, device="cuda")
    lens2 = torch.zeros_like(lens)
    mone.mone_cache4_evict(h, -1, c, 100, 4, 20, to, to_score, kept, lens2)
    K, V = (torch.empty(1, 1, n_kv, 100, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mone.mone_cache4_read(h, -1, mone.make_cache4(*pools, to, lens2, to_score), None, 100, K, V, K.stride()[:4])
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    assert rel_fro(out[0, 0].float().cpu(), ref) <= TOL[torch.bfloat16]
    assert rel_fro(score[0, 0, :, :n].cpu(), w) <= 1e-5
    for a in range(n_kv):
        at = O.cache_keep(score[0, 0, a, :n].cpu(), 100, 4, 20)
        assert kept[0, 0, a].tolist() == at.tolist()
        assert np.array_equal(K[0, 0, a].double().cpu().numpy(), kq[a, at]) and np.array_equal(V[0, 0, a].double().cpu().numpy(), vq[a, at])


@pytest.mark.parametrize("dtype,group", [(torch.float32, 4), (torch.float32, 8), (torch.float32, 12), (torch.bfloat16, 4), (torch.bfloat16, 8), (torch.bfloat16, 16)])
def test_small_weights_behind_a_large_one_of_value_zero(dtype, group):
    """More items than warps, so that a warp goes through most of a context behind its first key, whose value is 0: the output is what the small
    weights give, 2^-14 to 2^-28 of the largest (2^-24 with a bf16 handle).  The queries are exact in 8 bits.  fp32: scores of up to 20, each three roundings
    of 2^-24 off, 3.6e-6 of a weight; the exponential 2^-22; a probability 2^-47 of the largest, 2^-19 of the smallest here: 5.8e-6.  bf16: as above."""
    n, B, L, n_kv, hd, page = 2048, 64, 20, 2, 64, 32
    key, val = np.zeros((1, n, hd)), np.zeros((1, n, hd))
    key[0, 0, 0] = 6.0
    val[0, 1:] = 6.0 * np.sign(np.arange(hd) - 20.5)
    pools = []
    for t in (key, val):
        code, scale = O.four_bits(t)
        assert np.array_equal(O.four_bit_values(code, scale), t)
        pools.append([torch.from_numpy(x).cuda().view(n // page, 1, page, -1).expand(L, -1, n_kv, -1, -1) for x in (packed(code), scale.astype(np.uint8))])
    (K, Ks), (V, Vs) = pools
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(B, 1)  # the contexts share their pages, layers and heads their rows
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    z = [13.25, 18.5, 22.25, 26.0 if dtype is torch.float32 else 20.0]  # 8 / 6 of the largest score: weights of 2^-14.3, 2^-20.0, 2^-24.1 and 2^-28.1
    Q = torch.zeros(B, L, n_kv * group, 1, hd, device="cuda")
    Q[:, :, :, 0, 0] = torch.tensor([z[i % 4] for i in range(n_kv * group)], device="cuda")
    Q = Q.to(dtype)
    h, out = handle(B, L, n_kv, hd, dtype), torch.full_like(Q, 7.0)
    mone.mone_cache4_attention(h, -1, mone.make_cache4(K, V, Ks, Vs, table, lens), Q, n_kv * group, 1, 0, ALL, out)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    for i in range(4):
        ref, _ = O.window_attention(Q[0, 0, i:i + 1].double().cpu(), key, val, n - 1, 0, ALL)
        got = out[:, :, i::4, 0].double().cpu()
        err = max(rel_fro(x, ref[0, 0]) for x in got.reshape(-1, hd).unique(dim=0))
        record("cache4 attention", f"weights of 2^-{z[i] * 0.75 / np.log(2):.0f} {str(dtype)[6:]} group {group}", err, TOL[dtype])
        assert err <= TOL[dtype], (i, err)


@pytest.mark.parametrize("group", [4, 8])
@pytest.mark.parametrize("hd", [64, 128])
def test_sums_of_one_sign_over_a_long_walk(hd, group):
    """More items than warps and values of one sign, so that a sum that is cut off rather than rounded shows: 512 blocks of a warp, each of 2^-20 of itself at
    most, added up with a rounding of 2^-24 of either sign each, 1.4e-6 of the sum; weights as above."""
    n, B, L, n_kv, page = 16384, 64, 20, 2, 32
    g = np.random.default_rng(hd + group)
    codes, values = [], []
    for t in (g.standard_normal((1, n, hd)), 0.5 + np.abs(g.standard_normal((1, n, hd)))):
        code, scale = O.four_bits(t)
        values.append(O.four_bit_values(code, scale))
        codes.append([torch.from_numpy(x).cuda().view(n // page, 1, page, -1).expand(L, -1, n_kv, -1, -1) for x in (packed(code), scale.astype(np.uint8))])
    (K, Ks), (V, Vs) = codes
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(B, 1)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    Q = torch.from_numpy(g.standard_normal((n_kv * group, 1, hd))).float().cuda().expand(B, L, -1, -1, -1).contiguous()
    h, out = handle(B, L, n_kv, hd, torch.float32), torch.full_like(Q, 7.0)
    mone.mone_cache4_attention(h, -1, mone.make_cache4(K, V, Ks, Vs, table, lens), Q, n_kv * group, 1, 0, ALL, out)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    ref, _ = O.window_attention(Q[0, 0].double().cpu(), *values, n - 1, 0, ALL)
    ref = torch.from_numpy(ref).cuda()
    err = ((out.double() - ref).square().sum((-1, -2, -3)) / ref.square().sum()).sqrt().max().item()
    record("cache4 attention", f"long walk hd {hd} group {group}", err, TOL[torch.float32])
    assert err <= TOL[torch.float32]
