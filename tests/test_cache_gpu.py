"""GPU parity of the paged cache's operators against the oracle's definitions in 64 bits.

Every position that an operator must not read holds NaN: pages that no context has, the places of a page past its
context's last position, and table entries past it name no page.

Tolerances (relative 2-norm).  bf16 outputs 5e-3: probabilities and outputs are rounded to 8 bits once each, at most
2^-9 of themselves and 2^-9 / sqrt(3) in the mean, 1.6e-3 together, times three.  fp32 outputs and all weights 1e-5: the
score of a key is a sum of 64 or 128 products in 32 bits, off by about 2^-24 sqrt(128) |z| with |z| up to 15, and the
weight is off by as much of itself.  Positions, lengths and moved rows are exact.
"""
import pytest
import torch

import oracle as O
import paper_2608_17616_gb300 as mone
from harness import rel_fro, record

pytestmark = pytest.mark.gpu
ALL = 1 << 30
TOL = {torch.bfloat16: 5e-3, torch.float32: 1e-5}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_17616_gb300 import build
    build.build()
    assert torch.cuda.is_available()
    mone.lib()


class Cache:
    """Contexts of given lengths over scattered pages, NaN wherever nothing is held."""

    def __init__(self, lens, n_layers=2, n_kv=2, hd=64, page=16, dtype=torch.bfloat16, order="head", spare=3, seed=0, pad=0, score=True):
        self.lens, self.L, self.n_kv, self.hd, self.page, self.dtype = list(lens), n_layers, n_kv, hd, page, dtype
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        n_ctx = len(self.lens)
        width = -(-max(max(lens), 1) // page) + spare
        P = n_ctx * width * 2 + 3
        shape = {"head": (n_layers, P, n_kv, page, hd + pad), "position": (n_layers, P, page, n_kv, hd + pad),
                 "layers inner": (P, n_kv, page, n_layers, hd + pad)}[order]
        perm = {"head": (0, 1, 2, 3, 4), "position": (0, 1, 3, 2, 4), "layers inner": (3, 0, 1, 2, 4)}[order]
        self.K, self.V = (torch.full(shape, float("nan"), dtype=dtype, device="cuda").permute(*perm)[..., :hd] for _ in range(2))
        pages = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        self.table = pages[:n_ctx * width].view(n_ctx, width).clone()
        self.fresh = pages[n_ctx * width:2 * n_ctx * width].view(n_ctx, width).clone()
        self.len_t = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        self.k, self.v = ([rn(n_layers, n_kv, n, hd) for n in self.lens] for _ in range(2))
        for c, n in enumerate(self.lens):
            self.put(self.K, c, self.k[c])
            self.put(self.V, c, self.v[c])
        self.score = torch.rand(n_ctx, n_layers, n_kv, width * page, generator=g, device="cuda") if score else None
        d_out = 2 * n_kv * hd
        if dtype is torch.float32 or d_out >= 256:
            cfg = mone.make_config(n_ctx, n_layers, 128, 256, d_out, n_kv, hd, 128,
                                   mone.MONE_FP32 if dtype is torch.float32 else mone.MONE_BF16, mone.MONE_PLAIN, 1e-2)
            W = torch.zeros(n_ctx * n_layers, 256, 128, device="cuda"), torch.zeros(n_ctx * n_layers, 256, d_out, device="cuda")
        else:
            cfg = mone.make_config(n_ctx, n_layers, 128, 64, 128, 1, 64, 128, mone.MONE_BF16, mone.MONE_PLAIN, 1e-2,
                                   memory=mone.MONE_MEM_SWIGLU, mem_heads=2)
            W = torch.zeros(n_ctx * n_layers, 2, 128, 64, device="cuda"), torch.zeros(n_ctx * n_layers, 2, 64, 64, device="cuda")
        self.h = mone.mone_mem_init(cfg, *W)
        # table entries that name no page of a context's positions are not valid page numbers
        self.tbl = self.table.clone()
        self.trim(self.tbl, self.lens)
        self.c = mone.make_cache(self.K, self.V, self.tbl, self.len_t, self.score)

    def trim(self, table, lens):
        for c, n in enumerate(lens):
            table[c, -(-n // self.page):] = -7

    def put(self, pool, c, rows):
        for i in range(0, rows.shape[2], self.page):
            r = rows[:, :, i:i + self.page]
            pool[:, self.table[c, i // self.page].item(), :, :r.shape[2]] = r

    def held(self, pool, c, n, table=None):
        """[layers, heads, n, hd] of a context's first n positions."""
        t = (self.table if table is None else table)[c].tolist()
        return torch.cat([pool[:, p] for p in t[:max(1, -(-n // self.page))]], 2)[:, :, :n]

    def done(self):
        mone.mone_mem_sync(self.h)

    def __del__(self):
        if getattr(self, "h", None):
            mone.mone_mem_free(self.h)


def attend(x, group, n_tok, n_sink, window, layer=-1, scale=1.0, what="cache attention"):
    layers = range(x.L) if layer < 0 else [layer]
    n_q, B = group * x.n_kv, len(x.lens)
    Q = (scale * torch.randn(B, len(layers), n_q, n_tok, x.hd, generator=x.g, device="cuda")).to(x.dtype)
    out = torch.full_like(Q, 7.0)
    before = None if x.score is None else x.score.clone()
    mone.mone_cache_attention(x.h, layer, x.c, Q, n_q, n_tok, n_sink, window, out)
    x.done()
    want = None if before is None else before.double().cpu()
    for c, n in enumerate(x.lens):
        ref = torch.zeros(out[c].shape, dtype=torch.float64)
        for i, l in enumerate(layers):
            o, w = O.window_attention(Q[c, i].float().cpu(), x.k[c][l].float().cpu(), x.v[c][l].float().cpu(), n - n_tok, n_sink, window)
            ref[i] = torch.from_numpy(o)
            if want is not None and n:
                want[c, l, :, :n] += torch.from_numpy(w)
        if ref.any():
            assert record(what, f"out {str(x.dtype)[6:]}", rel_fro(out[c].float().cpu(), ref), TOL[x.dtype]) <= TOL[x.dtype], c
        assert not out[c].float().cpu()[ref.abs().amax(-1) == 0].any(), c  # tokens that see nothing
    if want is not None:
        assert record(what, "weights", rel_fro(x.score.cpu(), want), 1e-5) <= 1e-5
        same = want == before.double().cpu()
        assert torch.equal(x.score.cpu()[same], before.cpu()[same])  # positions that no token sees
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,group,n_tok,hd,page,n_sink,window", [
    ([1], 1, 1, 64, 16, 0, ALL),                 # one position
    ([0, 1, 2, 0, 300], 4, 1, 64, 16, 0, ALL),     # contexts that hold nothing
    ([31, 32, 33, 63, 64, 65], 4, 1, 64, 32, 0, ALL),
    ([255, 256, 257, 600], 2, 1, 128, 64, 0, ALL),   # items that stay whole, and split ones
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
])
def test_attention(lens, group, n_tok, hd, page, n_sink, window, dtype):
    x = Cache(lens, hd=hd, page=page, dtype=dtype, seed=sum(lens) + group)
    attend(x, group, n_tok, n_sink, window)
    attend(x, group, n_tok, n_sink, window, scale=4.0)  # again on the same workspace, with steeper softmaxes


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,group,n_tok,hd,page,n_sink,window", [
    ([0, 1, 2, 0, 300], 4, 1, 64, 16, 0, ALL),
    ([31, 32, 33, 63, 64, 65], 4, 1, 64, 32, 0, ALL),
    ([255, 256, 257, 600], 2, 1, 128, 64, 0, ALL),
    ([4000], 8, 1, 64, 16, 0, ALL),
    ([3001, 17, 900], 5, 3, 128, 8, 0, ALL),
    ([400, 90], 7, 16, 64, 16, 0, ALL),
    ([9000, 30], 4, 1, 64, 16, 100, 7000),
    ([9000, 500, 6700], 4, 3, 128, 64, 33, 6500),
    ([300, 77], 4, 1, 64, 1, 0, ALL),
])
def test_attention_where_tables_could_hold_much(lens, group, n_tok, hd, page, n_sink, window, dtype):
    """A call goes by what its tables and its window allow: dealt out here, though the contexts are short."""
    x = Cache(lens, hd=hd, page=page, dtype=dtype, seed=sum(lens) + group, spare=16384 // page)
    attend(x, group, n_tok, n_sink, window)
    attend(x, group, n_tok, n_sink, window, scale=4.0)


@pytest.mark.parametrize("n_layers,lens", [
    (10, [700, 1500, 90]), (20, [700, 1500, 90]), (20, [300, 0, 77, 130, 1, 200]), (1, [1000]), (20, [33, 32, 31, 64, 65, 1])])
@pytest.mark.parametrize("group,n_tok,hd,n_sink,window", [(4, 1, 64, 0, ALL), (4, 1, 128, 40, 300), (3, 5, 64, 0, ALL), (2, 4, 64, 3, 33)])
def test_attention_by_clusters_of_every_size(n_layers, lens, group, n_tok, hd, n_sink, window):
    attend(Cache(lens, n_layers=n_layers, hd=hd, page=32, seed=n_layers), group, n_tok, n_sink, window)


@pytest.mark.parametrize("order,pad", [("position", 0), ("layers inner", 0), ("head", 8), ("head", 3), ("position", 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_over_other_strides(order, pad, dtype, hd):
    """Paddings of 3 and 1 elements leave rows that are not aligned to 16 bytes."""
    x = Cache([70, 513], n_layers=3, hd=hd, dtype=dtype, order=order, pad=pad)
    attend(x, 4, 2, 3, 200)


@pytest.mark.parametrize("layer", [0, 2])
def test_one_layer(layer):
    x = Cache([70, 513, 4], n_layers=3)
    attend(x, 4, 1, 0, ALL, layer=layer)


def test_one_head_of_64_and_no_weights():
    x = Cache([700, 3], n_kv=1, score=False)
    attend(x, 5, 1, 2, 300)


def test_more_contexts_than_a_warp_and_a_long_one():
    x = Cache([(37 * i) % 90 for i in range(70)] + [20000], n_layers=1, page=32)
    attend(x, 4, 1, 0, ALL)


def test_calls_of_changing_sizes_share_a_workspace_and_repeat_bit_for_bit():
    x = Cache([5000, 130, 1], n_layers=1, score=False)
    q1, q2 = (torch.randn(3, 1, 8, n, 64, generator=x.g, device="cuda").bfloat16() for n in (1, 5))
    outs = [[], []]
    for _ in range(4):
        for q, o in ((q1, outs[0]), (q2, outs[1])):
            o.append(torch.empty_like(q))
            mone.mone_cache_attention(x.h, 0, x.c, q, 8, q.shape[3], 0, ALL, o[-1])
    x.done()
    for o in outs:
        assert all(torch.equal(o[0], y) for y in o[1:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_non_finite_values_reach_only_the_tokens_that_see_them(dtype):
    x = Cache([200], dtype=dtype, score=False)
    n_tok, window = 4, 50
    Q = torch.randn(1, 2, 4, n_tok, 64, generator=x.g, device="cuda").to(dtype)
    for bad in (float("nan"), float("inf")):
        for pos in (199, 198, 147, 148):  # the last tokens' own positions, and the two that only the older tokens see
            keep = x.v[0].clone()
            x.v[0][:, :, pos] = bad
            x.put(x.V, 0, x.v[0])
            out = torch.full_like(Q, 7.0)
            mone.mone_cache_attention(x.h, -1, x.c, Q, 4, n_tok, 3, window, out)
            x.done()
            for l in range(2):
                ref, _ = O.window_attention(Q[0, l].float().cpu(), x.k[0][l].float().cpu(), x.v[0][l].float().cpu(), 196, 3, window)
                ref = torch.from_numpy(ref)
                fine = ref.isfinite()
                got = out[0, l].float().cpu()
                assert fine.any() and not fine.all()
                assert torch.equal(got.isfinite(), fine)
                assert rel_fro(got[fine], ref[fine]) <= TOL[dtype]
            x.v[0] = keep
            x.put(x.V, 0, keep)


def test_keys_at_minus_infinity_count_for_nothing():
    x = Cache([300, 40])
    for c, n in enumerate(x.lens):
        x.k[c][..., 0] = 0
        x.k[c][:, :, :n // 2, 0] = -1e25
        x.put(x.K, c, x.k[c])
    Q = torch.randn(2, 2, 8, 1, 64, generator=x.g, device="cuda").bfloat16()
    Q[..., 0] = 1e25
    out = torch.full_like(Q, 7.0)
    before = x.score.clone()
    mone.mone_cache_attention(x.h, -1, x.c, Q, 8, 1, 0, ALL, out)
    x.done()
    for c, n in enumerate(x.lens):
        for l in range(2):
            ref, w = O.window_attention(Q[c, l].float().cpu(), x.k[c][l].float().cpu(), x.v[c][l].float().cpu(), n - 1, 0, ALL)
            assert rel_fro(out[c, l].float().cpu(), ref) <= 5e-3
            assert rel_fro(x.score[c, l, :, :n].cpu(), before[c, l, :, :n].double().cpu() + torch.from_numpy(w)) <= 1e-5


def test_pages_and_lengths_out_of_range_are_latched_and_skipped():
    x = Cache([100, 60])
    Q = torch.randn(2, 2, 4, 1, 64, generator=x.g, device="cuda").bfloat16()
    out = torch.empty_like(Q)
    for bad in (-1, x.K.shape[1], 1 << 30):
        keep = x.tbl.clone()
        x.tbl[0, 2] = bad
        mone.mone_cache_attention(x.h, -1, x.c, Q, 4, 1, 0, ALL, out)
        with pytest.raises(mone.MoneError) as e:
            x.done()
        assert e.value.code == 8 and "page" in str(e.value)
        x.tbl.copy_(keep)
    for bad in (-1, x.tbl.shape[1] * x.page + 1):
        x.tbl.copy_(x.table)
        x.len_t[0] = bad
        mone.mone_cache_attention(x.h, -1, x.c, Q, 4, 1, 0, ALL, out)
        with pytest.raises(mone.MoneError) as e:
            x.done()
        assert e.value.code == 8 and "length" in str(e.value)
    x.len_t[0] = 100
    k = torch.randn(2, 2, 2, 200, 64, device="cuda").bfloat16()
    mone.mone_cache_append(x.h, -1, x.c, k, k, k.stride()[:4], 200)  # past the table's end
    with pytest.raises(mone.MoneError) as e:
        x.done()
    assert e.value.code == 8 and "length" in str(e.value)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,spare,n_tok,bad", [
    ([200], 3, 4, slice(199, 200)),        # the newest token's key alone: the older tokens' windows begin where its own does not
    ([300, 40], 3, 3, slice(2, 3)),        # one that all see
    ([9000], 1024, 1, slice(1024, 8064)),   # dealt out: parts of 128 positions that hold no other score
    ([9000], 1024, 4, slice(8999, 9000)),
    ([900], 3, 1, slice(100, 800)),        # a cluster's
])
def test_weights_of_tokens_whose_scores_are_not_numbers(lens, spare, n_tok, bad, dtype):
    """Such a token's weights are not numbers where it sees, and nothing where it does not."""
    x = Cache(lens, dtype=dtype, spare=spare, seed=len(lens))
    window = 50 if n_tok > 1 else ALL
    x.k[0][:, :, bad] = float("nan")
    x.put(x.K, 0, x.k[0])
    Q = torch.randn(len(lens), 2, 8, n_tok, 64, generator=x.g, device="cuda").to(dtype)
    out, want = torch.full_like(Q, 7.0), x.score.double().cpu()
    mone.mone_cache_attention(x.h, -1, x.c, Q, 8, n_tok, 3, window, out)
    x.done()
    for c, n in enumerate(lens):
        for l in range(2):
            ref, w = O.window_attention(Q[c, l].float().cpu(), x.k[c][l].float().cpu(), x.v[c][l].float().cpu(), n - n_tok, 3, window)
            want[c, l, :, :n] += torch.from_numpy(w)
            assert torch.equal(out[c, l].isnan().cpu(), torch.from_numpy(ref).isnan())
    got = x.score.cpu()
    assert torch.equal(got.isnan(), want.isnan()) and want.isnan().any()
    assert rel_fro(got.nan_to_num(), want.nan_to_num()) <= 1e-5


# ----------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,n_tok,page,order,pad,counts,layer", [
    ([0], 1, 16, "head", 0, None, -1),
    ([15, 16, 17, 0], 1, 16, "head", 0, None, -1),
    ([15, 16, 17, 0], 33, 16, "position", 0, None, 1),
    ([100, 7], 500, 64, "head", 0, [500, 0], -1),       # a prompt for one context, nothing for the other
    ([100, 7, 9], 5, 1, "head", 0, [2, 9, -3], -1),       # counts past the tokens that there are, pages of one
    ([100, 7], 20, 16, "head", 3, None, -1),             # rows that are not aligned
    ([3], 20, 8, "layers inner", 1, None, 0),
])
def test_append(lens, n_tok, page, order, pad, counts, layer, dtype):
    x = Cache(lens, page=page, dtype=dtype, order=order, pad=pad, spare=-(-n_tok // page) + 1)
    count = [n_tok if counts is None else min(max(counts[c], 0), n_tok) for c in range(len(lens))]
    x.tbl.copy_(x.table)
    x.trim(x.tbl, [n + k for n, k in zip(lens, count)])
    layers = list(range(x.L)) if layer < 0 else [layer]
    # tokens with the heads inside, a strided view
    k, v = (torch.randn(len(lens), len(layers), n_tok, x.n_kv, x.hd + pad, generator=x.g, device="cuda").to(dtype)[..., :x.hd].transpose(2, 3)
            for _ in range(2))
    out = torch.full_like(x.len_t, -5)
    K0, V0, s0 = x.K.clone(), x.V.clone(), x.score.clone()
    mone.mone_cache_append(x.h, layer, x.c, k, v, k.stride()[:4], n_tok, out,
                           None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    x.done()
    assert out.tolist() == [n + k for n, k in zip(lens, count)]
    for pool, pool0, new, old in ((x.K, K0, k, x.k), (x.V, V0, v, x.v)):
        want = pool0.clone()
        for c, n in enumerate(lens):
            for i in range(count[c]):
                for a, l in enumerate(layers):
                    want[l, x.table[c, (n + i) // page].item(), :, (n + i) % page] = new[c, a, :, i]
        assert torch.equal(pool.view(torch.int16 if dtype is torch.bfloat16 else torch.int32),
                           want.view(torch.int16 if dtype is torch.bfloat16 else torch.int32))  # NaN and all
    for c, n in enumerate(lens):
        for l in layers:
            s0[c, l, :, n:n + count[c]] = 0
    assert torch.equal(x.score, s0)


# ----------------------------------------------------------------- eviction

def evict(x, keep, n_sink, n_recent, layer=-1):
    layers = list(range(x.L)) if layer < 0 else [layer]
    B, n_to = len(x.lens), -(-keep // x.page)
    to = x.fresh[:, :n_to].contiguous()
    to_score = torch.full((B, x.L, x.n_kv, n_to * x.page), -3.0, device="cuda")
    kept = torch.full((B, len(layers), x.n_kv, keep), -9, dtype=torch.int32, device="cuda")
    out = torch.full_like(x.len_t, -5)
    s0 = x.score.clone()
    mone.mone_cache_evict(x.h, layer, x.c, keep, n_sink, n_recent, to, to_score, kept, out)
    x.done()
    assert out.tolist() == [min(n, keep) for n in x.lens]
    assert torch.equal(x.score.view(torch.int32), s0.view(torch.int32))
    want_score = torch.full_like(to_score, -3.0).cpu()
    for c, n in enumerate(x.lens):
        assert torch.equal(x.held(x.K, c, n), x.k[c]) and torch.equal(x.held(x.V, c, n), x.v[c])  # the old pages
        newK, newV = (x.held(p, c, min(n, keep), to) for p in (x.K, x.V))
        for a, l in enumerate(layers):
            for g in range(x.n_kv):
                at = torch.from_numpy(O.cache_keep(s0[c, l, g, :n].cpu(), keep, n_sink, n_recent))
                assert kept[c, a, g].tolist() == at.tolist() + [-1] * (keep - len(at)), (c, l, g)
                want_score[c, l, g, :len(at)] = s0[c, l, g, at.cuda()].cpu()
                assert torch.equal(newK[l, g], x.k[c][l, g, at.cuda()]) and torch.equal(newV[l, g], x.v[c][l, g, at.cuda()])
    assert torch.equal(to_score.cpu().nan_to_num(nan=-77.0), want_score.nan_to_num(nan=-77.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,keep,n_sink,n_recent,page,hd,order,pad", [
    ([1, 0, 2], 1, 0, 0, 16, 64, "head", 0),
    ([50, 51, 100, 3], 50, 4, 10, 16, 64, "head", 0),     # all kept; one goes; half goes
    ([3000, 700, 1], 333, 0, 0, 8, 128, "position", 0),
    ([3000, 1025], 1024, 500, 524, 64, 64, "head", 0),    # no choice among the others
    ([2000], 1999, 1, 1, 16, 64, "head", 0),
    ([500, 40], 37, 5, 7, 1, 64, "head", 3),
    ([20000], 5000, 64, 1000, 64, 64, "layers inner", 0),
])
def test_evict(lens, keep, n_sink, n_recent, page, hd, order, pad, dtype):
    evict(Cache(lens, page=page, hd=hd, dtype=dtype, order=order, pad=pad, seed=keep), keep, n_sink, n_recent)


@pytest.mark.parametrize("kind", ["equal", "few values", "nan", "infinite", "negative", "zeros of both signs", "one digit apart"])
def test_evict_by_scores_that_tie_or_are_not_finite(kind):
    x = Cache([1500, 900, 31], n_layers=1)
    s = x.score
    if kind == "equal":
        s.fill_(0.25)
    elif kind == "few values":
        s.copy_((s * 4).floor())
    elif kind == "nan":
        s[s > 0.6] = float("nan")
        s[s < 0.2] = -float("nan")
    elif kind == "infinite":
        s[s > 0.8] = float("inf")
        s[s < 0.5] = -float("inf")
    elif kind == "negative":
        s.sub_(0.5)
    elif kind == "zeros of both signs":
        s.copy_(torch.where(s > 0.5, 0.0, -0.0))
    else:
        s.copy_((torch.full_like(s, 1.0).view(torch.int32) + (s * 5).int()).view(torch.float32))
    evict(x, 400, 7, 90)


def test_evict_one_layer():
    evict(Cache([300, 90], n_layers=3), 80, 4, 8, layer=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_evict_reads_the_target_pages_of_survivors_only(dtype):
    """Contexts that hold fewer positions than are kept have target pages for what they hold; the entries past them name no page."""
    x = Cache([300, 20, 0, 90, 80, 81], dtype=dtype)
    x.trim(x.fresh, [min(n, 80) for n in x.lens])
    evict(x, 80, 4, 8)


@pytest.mark.parametrize("lens,n_layers,n_kv,keep", [
    ([16385, 20001, 40000], 14, 4, 9001),     # more rows than the SMs hold twice: a CTA has a row, past what it keeps on chip
    ([140001, 131080], 1, 1, 50000),          # eight CTAs a row, whose slices are longer than that too
])
@pytest.mark.parametrize("levels", [None, 7])  # scores that differ, and ties at every value
def test_evict_from_slices_longer_than_a_cta_holds(lens, n_layers, n_kv, keep, levels):
    n_sink, n_recent, page, B = 5, 300, 64, len(lens)
    x = Cache(lens, n_layers=n_layers, n_kv=n_kv, page=page, seed=7)
    if levels:
        x.score.mul_(levels).floor_()
    n_to = -(-keep // page)
    to = x.fresh[:, :n_to].contiguous()
    to_score = torch.zeros(B, n_layers, n_kv, n_to * page, device="cuda")
    kept = torch.full((B, n_layers, n_kv, keep), -9, dtype=torch.int32, device="cuda")
    mone.mone_cache_evict(x.h, -1, x.c, keep, n_sink, n_recent, to, to_score, kept)
    x.done()
    for c, n in enumerate(lens):
        score = x.score[c, :, :, :n].cpu()
        newK = x.held(x.K, c, keep, to)
        for l in range(n_layers):
            for g in range(n_kv):
                mid = score[l, g, n_sink:n - n_recent]
                best = torch.sort(mid, descending=True, stable=True).indices[:keep - n_sink - n_recent]  # ties by position
                at = torch.cat([torch.arange(n_sink), n_sink + best.sort().values, torch.arange(n - n_recent, n)])
                assert torch.equal(kept[c, l, g].cpu().long(), at), (c, l, g)
                assert torch.equal(to_score[c, l, g, :keep].cpu(), score[l, g, at])
                assert torch.equal(newK[l, g], x.k[c][l, g, at.cuda()])


# ----------------------------------------------------------------- together, as a serving program uses them

def test_append_attend_evict_attend():
    x = Cache([0, 0], n_layers=2, spare=20)
    B, L, n_kv, hd, group = 2, 2, x.n_kv, x.hd, 4
    k, v = (torch.randn(B, L, n_kv, 200, hd, generator=x.g, device="cuda").bfloat16() for _ in range(2))
    x.tbl.copy_(x.table)
    lens = torch.zeros_like(x.len_t)
    mone.mone_cache_append(x.h, -1, x.c, k, v, k.stride()[:4], 200, lens, torch.tensor([200, 120], dtype=torch.int32, device="cuda"))
    q = torch.randn(B, L, group * n_kv, 3, hd, generator=x.g, device="cuda").bfloat16()
    out, c2 = torch.empty_like(q), mone.make_cache(x.K, x.V, x.tbl, lens, x.score)
    mone.mone_cache_attention(x.h, -1, c2, q, group * n_kv, 3, 0, ALL, out)
    keep = 64
    to, to_score = x.fresh, torch.zeros_like(x.score)
    kept, lens2 = torch.empty(B, L, n_kv, keep, dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    mone.mone_cache_evict(x.h, -1, c2, keep, 4, 8, to, to_score, kept, lens2)
    c3 = mone.make_cache(x.K, x.V, to, lens2, to_score)
    o1 = q[..., :1, :].contiguous()
    res = torch.empty_like(o1)
    mone.mone_cache_attention(x.h, -1, c3, o1, group * n_kv, 1, 0, ALL, res)
    x.done()
    for c, n in enumerate((200, 120)):
        for l in range(L):
            ref, w = O.window_attention(q[c, l].float().cpu(), k[c, l, :, :n].float().cpu(), v[c, l, :, :n].float().cpu(), n - 3, 0, ALL)
            assert rel_fro(out[c, l].float().cpu(), ref) <= 5e-3
            assert rel_fro(x.score[c, l, :, :n].cpu(), w) <= 1e-5
            for g in range(n_kv):
                at = O.cache_keep(x.score[c, l, g, :n].cpu(), keep, 4, 8)
                assert kept[c, l, g].tolist() == at.tolist()
                one, _ = O.window_attention(o1[c, l, g * group:(g + 1) * group].float().cpu(), k[c, l, g:g + 1, at].float().cpu(),
                                            v[c, l, g:g + 1, at].float().cpu(), keep - 1, 0, ALL)
                assert rel_fro(res[c, l, g * group:(g + 1) * group].float().cpu(), one) <= 5e-3


@pytest.mark.parametrize("hd,dtype", [(64, torch.bfloat16), (128, torch.bfloat16), (64, torch.float32)])
def test_calls_in_a_row_read_what_the_kernels_ahead_wrote(hd, dtype):
    """Nothing between the calls waits: the same bits as with a synchronisation after each, whatever runs ahead of what."""
    n_kv, group, steps, keep = 2, 4, 24, 40
    results = []
    for wait in (True, False, False):
        x = Cache([70, 0, 33], n_layers=2, n_kv=n_kv, hd=hd, page=16, dtype=dtype, spare=4, seed=5)
        B, L = len(x.lens), x.L
        g = torch.Generator(device="cuda").manual_seed(9)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        Q, K, V = rn(steps, B, L, group * n_kv, 1, hd), rn(steps, B, L, n_kv, 1, hd), rn(steps, B, L, n_kv, 1, hd)
        WQ, WK, WV = rn(steps, B, L, group * n_kv, 40, hd), rn(steps, B, L, n_kv, 90, hd), rn(steps, B, L, n_kv, 90, hd)
        q, k, v, wq, wk, wv = (torch.zeros_like(t[0]) for t in (Q, K, V, WQ, WK, WV))
        out, few, w_out, longer = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(wq), torch.zeros_like(x.len_t)
        got = []
        x.tbl.copy_(x.table)
        sync = torch.cuda.synchronize if wait else lambda: None
        sync()
        for i in range(steps):
            for t, bank in ((q, Q), (k, K), (v, V), (wq, WQ), (wk, WK), (wv, WV)):
                t.copy_(bank[i])
            mone.mone_cache_append(x.h, -1, x.c, k, v, k.stride()[:4], 1, longer)
            sync()
            x.len_t.copy_(longer)
            mone.mone_cache_attention(x.h, -1, x.c, q, group * n_kv, 1, 3, 50, out)
            sync()
            mone.mone_window_attention(x.h, -1, wq, group * n_kv, 40, wk, wv, wk.stride()[:4], 50, 4, 30, w_out)  # many rows
            sync()
            mone.mone_window_attention(x.h, -1, out, group * n_kv, 1, wk, wv, wk.stride()[:4], 50, 4, 30, few)
            sync()
            got += [out.clone(), w_out.clone(), few.clone()]
        to_score = torch.zeros(B, L, n_kv, x.fresh.shape[1] * x.page, device="cuda")
        kept = torch.zeros(B, L, n_kv, keep, dtype=torch.int32, device="cuda")
        mone.mone_cache_evict(x.h, -1, x.c, keep, 4, 8, x.fresh, to_score, kept, longer)
        sync()
        x.len_t.copy_(longer)
        x.tbl[:, :x.fresh.shape[1]].copy_(x.fresh)
        x.score.copy_(to_score)
        mone.mone_cache_attention(x.h, -1, x.c, q, group * n_kv, 1, 0, ALL, out)
        got += [out.clone(), kept, to_score, x.score.clone()]
        x.done()
        results.append(got)
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("hd,spare", [(64, 4), (128, 4), (64, 1024)])
def test_a_captured_step_serves_growing_contexts(hd, spare):
    """A graph of append and attention, replayed, gives the bits of the calls; lengths grow over pages' ends in device memory."""
    n_kv, group, steps = 2, 4, 40
    results = []
    for graph in (False, True):
        x = Cache([30, 0, 500], n_kv=n_kv, hd=hd, page=16, spare=spare, seed=3)
        B, L = len(x.lens), x.L
        g = torch.Generator(device="cuda").manual_seed(4)
        Q, K, V = (torch.randn(steps, B, L, n, 1, hd, generator=g, device="cuda").bfloat16() for n in (group * n_kv, n_kv, n_kv))
        q, k, v = Q[0].clone(), K[0].clone(), V[0].clone()
        out, longer, got = torch.zeros_like(q), torch.zeros_like(x.len_t), []
        x.tbl.copy_(x.table)

        def step():
            mone.mone_cache_append(x.h, -1, x.c, k, v, k.stride()[:4], 1, longer)
            x.len_t.copy_(longer)
            mone.mone_cache_attention(x.h, -1, x.c, q, group * n_kv, 1, 2, 200, out)

        lens, score = x.len_t.clone(), x.score.clone()
        step()  # the workspace, before a capture
        x.len_t.copy_(lens)
        x.score.copy_(score)
        torch.cuda.synchronize()
        if graph:
            G = torch.cuda.CUDAGraph()
            with torch.cuda.graph(G):
                step()
        for i in range(steps):
            q.copy_(Q[i]), k.copy_(K[i]), v.copy_(V[i])
            G.replay() if graph else step()
            got.append(out.clone())
        x.done()
        assert x.len_t.tolist() == [n + steps for n in x.lens]
        results.append(got + [x.score.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_graph_is_replayed_after_larger_calls():
    """The workspace that a graph holds stays when the handle's grows, which it does not during a capture."""
    x = Cache([300, 40], spare=40, seed=6)
    n_kv, group = x.n_kv, 4
    rn = lambda n_tok: torch.randn(2, 2, group * n_kv, n_tok, 64, generator=x.g, device="cuda").bfloat16()  # noqa: E731
    q, big = rn(1), rn(16)
    out, want, score = torch.empty_like(q), torch.empty_like(q), x.score.clone()
    mone.mone_cache_attention(x.h, -1, x.c, q, group * n_kv, 1, 2, 100, want)
    want_score = x.score.clone()
    torch.cuda.synchronize()
    G = torch.cuda.CUDAGraph()
    with torch.cuda.graph(G):
        with pytest.raises(mone.MoneError) as e:
            mone.mone_cache_attention(x.h, -1, x.c, big, group * n_kv, 16, 2, 100, torch.empty_like(big))
        mone.mone_cache_attention(x.h, -1, x.c, q, group * n_kv, 1, 2, 100, out)
    assert e.value.code == 3 and "capture" in str(e.value)
    mone.mone_cache_attention(x.h, -1, x.c, big, group * n_kv, 16, 2, 100, torch.empty_like(big))
    junk = [torch.full((1 << 22,), float("nan"), device="cuda") for _ in range(8)]  # what would lie where the old one was
    for _ in range(3):
        x.score.copy_(score)
        out.zero_()
        G.replay()
    x.done()
    assert torch.equal(out, want) and torch.equal(x.score, want_score) and all(j.isnan().all() for j in junk)


def test_on_another_stream():
    x = Cache([900, 40])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        attend(x, 4, 1, 0, ALL)


# ----------------------------------------------------------------- offsets past 32 bits

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pools_and_offsets_past_32_bits(dtype):
    """Pages whose elements lie more than 2^31 from the pool's first, in a cache longer than its heads' first 2^31 bytes."""
    hd, page, n_kv, n_pages = 64, 64, 2, (1 << 31) // (64 * 64 * 2) + 40
    K, V = (torch.empty(1, n_pages, n_kv, page, hd, dtype=dtype, device="cuda") for _ in range(2))
    x = Cache([1], n_layers=1, page=page, dtype=dtype)  # a handle
    g = torch.Generator(device="cuda").manual_seed(5)
    n, extra = 300, 20
    far = torch.tensor([[n_pages - 1, n_pages - 2, n_pages - 30, 3, n_pages - 7, n_pages - 9]], dtype=torch.int32, device="cuda")
    lens, out_lens = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    score = torch.zeros(1, 1, n_kv, 6 * page, device="cuda")
    k, v = (torch.randn(1, 1, n_kv, n, hd, generator=g, device="cuda").to(dtype) for _ in range(2))
    mone.mone_cache_append(x.h, -1, mone.make_cache(K, V, far, lens, score), k, v, k.stride()[:4], n, out_lens)
    q = torch.randn(1, 1, 4 * n_kv, 1, hd, generator=g, device="cuda").to(dtype)
    out, c = torch.empty_like(q), mone.make_cache(K, V, far, out_lens, score)
    mone.mone_cache_attention(x.h, -1, c, q, 4 * n_kv, 1, 0, ALL, out)
    ref, w = O.window_attention(q[0, 0].float().cpu(), k[0, 0].float().cpu(), v[0, 0].float().cpu(), n - 1, 0, ALL)
    to = torch.tensor([[n_pages - 3, n_pages - 5]], dtype=torch.int32, device="cuda")
    to_score, kept = torch.zeros(1, 1, n_kv, 2 * page, device="cuda"), torch.empty(1, 1, n_kv, 100, dtype=torch.int32, device="cuda")
    mone.mone_cache_evict(x.h, -1, c, 100, 4, extra, to, to_score, kept)
    x.done()
    assert rel_fro(out[0, 0].float().cpu(), ref) <= TOL[dtype]
    assert rel_fro(score[0, 0, :, :n].cpu(), w) <= 1e-5
    for h in range(n_kv):
        at = O.cache_keep(score[0, 0, h, :n].cpu(), 100, 4, extra)
        assert kept[0, 0, h].tolist() == at.tolist()
        got = torch.cat([K[0, p, h] for p in to[0].tolist()])[:100]
        assert torch.equal(got, k[0, 0, h, at])
