"""GPU parity of the windowed attention against the oracle's definition in 64 bits, in each of its forms: many rows on the
tensor cores (128-row tiles, chunks of 64 keys), few rows (16-row tiles, the keys split), and the CUDA cores (fp32, and bf16
rows that are not aligned).

Tolerances (relative 2-norm).  bf16 5e-3: probabilities and outputs are rounded to 8 bits once each, at most 2^-9 of
themselves and 2^-9 / sqrt(3) in the mean, 1.6e-3 together, times three.  fp32 1e-5: the score of a key is a sum of up to
128 products in 32 bits, off by about 2^-24 sqrt(128) |z| with |z| up to 15.
"""
import pytest
import torch

import oracle as O
import paper_2608_17616_gb300 as mone
import workloads as wk
from harness import DeviceRun, record, rel_fro

pytestmark = pytest.mark.gpu
ALL = 1 << 30
TOL = {torch.bfloat16: 5e-3, torch.float32: 1e-5}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_17616_gb300 import build
    build.build()
    assert torch.cuda.is_available()
    mone.lib()


def handle(n_layers, n_kv, hd, dtype, n_ctx=1):
    return DeviceRun(wk.Workload("window", 51, n_ctx, n_layers, 256, 256, 2 * n_kv * hd, n_kv, hd, 128, 128, 8,
                                 "f32" if dtype is torch.float32 else "bf16", wk.PLAIN))


def case(group, Lq, n_past, n_sink, window, hd=64, n_layers=2, dtype=torch.bfloat16, pad=0, layer=-1, n_ctx=1, late=1.0, kind=None):
    n_kv = 2
    run = handle(n_layers, n_kv, hd, dtype, n_ctx)
    g = torch.Generator(device="cuda").manual_seed(group * 1000 + Lq + n_past + window % 97)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    S = n_past + Lq
    K, V = (rn(n_ctx, n_layers, n_kv, S + 5, hd + pad) for _ in range(2))  # spare rows that nobody may read
    K[..., 2 * S // 3:, :] *= late
    K[..., S:, :], V[..., S:, :] = float("nan"), float("nan")
    K, V = (x.to(dtype)[..., :hd] for x in (K, V))
    if kind == "heads inner":
        K, V = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (K, V))
    layers = list(range(n_layers)) if layer < 0 else [layer]
    Q = rn(n_ctx, len(layers), group * n_kv, Lq, hd).to(dtype)
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, layer, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, n_sink, window, out)
    mone.mone_mem_sync(run.h)
    run.close()
    for c in sorted({0, n_ctx - 1}):
        for a in sorted({0, len(layers) - 1}):
            ref, _ = O.window_attention(Q[c, a].float().cpu(), K[c, layers[a], :, :S].float().cpu(), V[c, layers[a], :, :S].float().cpu(),
                                        n_past, n_sink, window)
            got = out[c, a].float().cpu()
            if not ref.any():
                assert not got.any()
            else:
                assert record("window attention", f"out {str(dtype)[6:]}", rel_fro(got, ref), TOL[dtype]) <= TOL[dtype], (c, a)


MANY = [  # rows past the few-rows form: 20 layers x 2 KV heads
    (4, 200, 70, 64, 40, 64),      # first positions, then a gap that grows along the tile
    (4, 200, 70, 0, 40, 64),       # a window alone
    (4, 200, 70, 0, ALL, 64),      # everything
    (1, 300, 0, 0, 1, 64),         # a window of one
    (1, 300, 0, 4, 1, 64),
    (1, 300, 513, 100, 96, 64),    # a window of a chunk, first positions past a chunk
    (2, 133, 1000, 96, 192, 64),   # whole chunks exactly
    (2, 133, 1000, 97, 193, 64),   # one past
    (2, 133, 1000, 5000, 7, 64),   # more first positions than there are
    (2, 133, 100, 150, 30, 64),    # first positions that reach into the prompt
    (64, 3, 94, 10, 20, 64),       # the most heads a KV head has
    (3, 150, 0, 2, 64, 128),       # padded rows
    (4, 129, 383, 64, 64, 128),
    (4, 129, 383, 65, 129, 128),
    (2, 140, 200, 9, 0, 128),      # first positions alone
    (5, 77, 20, 0, 0, 64),         # nothing to see
]


@pytest.mark.parametrize("group,Lq,n_past,n_sink,window,hd", MANY)
def test_many_rows(group, Lq, n_past, n_sink, window, hd):
    case(group, Lq, n_past, n_sink, window, hd, n_layers=20)


@pytest.mark.parametrize("group,Lq,n_past,n_sink,window,hd", MANY)
@pytest.mark.parametrize("dtype,pad", [(torch.float32, 0), (torch.float32, 1), (torch.bfloat16, 4)])
def test_cuda_cores(group, Lq, n_past, n_sink, window, hd, dtype, pad):
    case(group, Lq, n_past, n_sink, window, hd, n_layers=2, dtype=dtype, pad=pad)


@pytest.mark.parametrize("group,Lq,n_past,n_sink,window,hd", [
    (1, 1, 0, 0, 1, 64),
    (1, 1, 0, 1, 0, 64),
    (4, 1, 31, 0, 32, 64),
    (4, 1, 32, 0, 32, 64),
    (4, 1, 500, 4, 100, 64),
    (7, 2, 5000, 64, 1000, 64),
    (8, 3, 700, 33, 40, 64),
    (16, 32, 100, 20, 30, 64),     # 32 row tiles of two heads
    (4, 1, 15, 3, 5, 128),
    (5, 5, 3000, 100, 200, 128),
    (5, 5, 3000, 0, ALL, 128),
    (5, 5, 3000, 100, 900, 128),   # few rows over many keys, hidden ones between
    (4, 3, 2000, 4, 801, 128),
    (1, 16, 1500, 700, 130, 128),
    (1, 90, 50, 7, 3, 64),         # row tiles of 16 tokens with windows of 3
])
def test_few_rows(group, Lq, n_past, n_sink, window, hd):
    case(group, Lq, n_past, n_sink, window, hd, n_layers=1, late=3.0)


def test_the_row_max_grows_late():
    case(4, 100, 300, 16, 250, n_layers=20, late=9.0)
    case(2, 140, 200, 16, 250, hd=128, n_layers=20, late=9.0)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("top,size", [(88.5, 1.0), (88.5, 2.0 ** -10), (60.0, 1.0), (200.0, 1.0)])
def test_scores_far_above_the_first_keys(hd, top, size):
    """Two keys in the middle whose exponentials, against the first keys', add up past 32 bits, or are past them."""
    L, group, Lq, n_past = 20, 4, 150, 300
    run = handle(L, 2, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(hd)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    K, V, Q = rn(1, L, 2, n_past + Lq, hd), size * rn(1, L, 2, n_past + Lq, hd), rn(1, L, 2 * group, Lq, hd)
    Q[..., 0], K[..., 0] = hd ** 0.5 if hd == 64 else 11.3125, 0
    Q[..., 1:] *= 0.5
    K[..., 200, 0] = K[..., 203, 0] = top
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, 2 * group, Lq, K, V, K.stride()[:4], n_past, 16, ALL, out)
    mone.mone_mem_sync(run.h)
    run.close()
    for layer in (0, L - 1):
        ref, _ = O.window_attention(Q[0, layer].float().cpu(), K[0, layer].float().cpu(), V[0, layer].float().cpu(), n_past, 16, ALL)
        assert rel_fro(out[0, layer].float().cpu(), ref) <= 5e-3


@pytest.mark.parametrize("layer", [0, 7, 19])
def test_one_layer_of_a_cache(layer):
    case(4, 400, 70, 64, 40, n_layers=20, layer=layer, n_ctx=3)


@pytest.mark.parametrize("Lq", [1, 150])
def test_heads_inside_the_positions(Lq):
    case(4, Lq, 70, 64, 40, n_layers=20, n_ctx=2, kind="heads inner")


@pytest.mark.parametrize("group,Lq,n_past,hd,n_layers,dtype,pad", [
    (4, 200, 70, 64, 20, torch.bfloat16, 0),     # many rows
    (3, 150, 0, 128, 20, torch.bfloat16, 0),
    (4, 20, 300, 64, 1, torch.bfloat16, 0),      # few rows
    (3, 50, 70, 64, 2, torch.float32, 0),        # CUDA cores
    (3, 50, 70, 64, 2, torch.bfloat16, 4),
])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_values_reach_only_the_tokens_that_see_them(group, Lq, n_past, hd, n_layers, dtype, pad, bad):
    n_kv, n_sink, window = 2, 2, 30
    run = handle(n_layers, n_kv, hd, dtype)
    g = torch.Generator(device="cuda").manual_seed(Lq)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    S = n_past + Lq
    K, V = (rn(1, n_layers, n_kv, S, hd + pad)[..., :hd] for _ in range(2))
    Q = rn(1, n_layers, group * n_kv, Lq, hd)
    V[..., n_past + Lq // 2, :] = bad
    K[..., S - 1, ::2] = bad
    V[..., S - 1, :] = bad
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, n_sink, window, out)
    mone.mone_mem_sync(run.h)
    run.close()
    ok = torch.ones(Lq, dtype=torch.bool)
    ok[Lq // 2:Lq // 2 + window] = False
    ok[-1] = False
    for layer in {0, n_layers - 1}:
        ref, _ = O.window_attention(Q[0, layer, :, :-1].float().cpu(), K[0, layer, :, :-1].float().cpu(), V[0, layer, :, :-1].float().cpu(),
                                    n_past, n_sink, window)
        got = out[0, layer].float().cpu()
        assert not got[:, ~ok].isfinite().any()
        assert rel_fro(got[:, :-1][:, ok[:-1]], ref[:, ok[:-1].numpy()]) <= TOL[dtype]


def test_keys_at_minus_infinity_count_for_nothing():
    for L, Lq in ((20, 150), (1, 4)):
        run = handle(L, 2, 64, torch.bfloat16)
        g = torch.Generator(device="cuda").manual_seed(Lq)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
        n_past = 200
        K, V, Q = rn(1, L, 2, n_past + Lq, 64), rn(1, L, 2, n_past + Lq, 64), rn(1, L, 4, Lq, 64)
        K[..., 0] = 0
        K[..., :n_past, 0] = -1e25
        Q[..., 0] = 1e25
        out = torch.full_like(Q, 7.0)
        mone.mone_window_attention(run.h, -1, Q, 4, Lq, K, V, K.stride()[:4], n_past, 50, 100, out)
        mone.mone_mem_sync(run.h)
        run.close()
        ref, _ = O.window_attention(Q[0, 0].float().cpu(), K[0, 0].float().cpu(), V[0, 0].float().cpu(), n_past, 50, 100)
        assert rel_fro(out[0, 0].float().cpu(), ref) <= 5e-3


@pytest.mark.parametrize("hd,n_sink,window", [(64, 64, 100), (128, 64, 100), (64, 0, 7), (128, 130, 300)])
def test_many_tiles_of_a_cta(hd, n_sink, window):
    """Five tiles and more for each CTA of the many-rows form: right, and the same bits again."""
    n_kv, group, Lq, n_past, L = 8, 4, 400, 64, 16
    run = handle(L, n_kv, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.randn(1, L, n_kv, n_past + Lq, hd, generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn(1, L, group * n_kv, Lq, hd, generator=g, device="cuda").bfloat16()
    outs = [torch.full_like(Q, 7.0) for _ in range(2)]
    for i in range(40):
        mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, n_sink, window, outs[i % 2])
    mone.mone_mem_sync(run.h)
    run.close()
    assert torch.equal(*outs)
    for layer in (0, 9, L - 1):
        ref, _ = O.window_attention(Q[0, layer].float().cpu(), K[0, layer].float().cpu(), V[0, layer].float().cpu(), n_past, n_sink, window)
        assert rel_fro(outs[0][0, layer].float().cpu(), ref) <= 5e-3, layer


@pytest.mark.parametrize("L,Lq", [(1, 280), (2, 280), (5, 280), (8, 280), (20, 90), (7, 500), (19, 33)])
@pytest.mark.parametrize("hd", [64, 128])
def test_every_tile_of_uneven_shares(L, Lq, hd):
    """Odd numbers of tiles of 32 tokens, over fewer CTAs than there are, over all, and with some left over: every row."""
    n_kv, group, n_past, n_sink, window = 8, 4, 20, 9, 50
    run = handle(L, n_kv, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(L)
    K, V = (torch.randn(1, L, n_kv, n_past + Lq, hd, generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn(1, L, group * n_kv, Lq, hd, generator=g, device="cuda").bfloat16()
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, n_sink, window, out)
    mone.mone_mem_sync(run.h)
    run.close()
    t, j = n_past + torch.arange(Lq, device="cuda")[:, None], torch.arange(n_past + Lq, device="cuda")[None]
    hidden = (j > t) | ((j >= n_sink) & (j <= t - window))
    k, v = (x.repeat_interleave(group, 2).double() for x in (K, V))
    z = (Q.double() @ k.transpose(-1, -2) / hd ** 0.5).masked_fill(hidden, float("-inf"))
    ref = torch.softmax(z, -1) @ v
    far = (out.double() - ref).norm(dim=-1) / ref.norm(dim=-1)
    assert (out.double() - ref).norm() / ref.norm() <= 5e-3
    assert far.max() <= 2e-2  # no row is another's: the rounding of one row's probabilities, at most 2^-8 of each, and the output's


@pytest.mark.parametrize("Lq", [3, 140])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_past_32_bits(Lq, dtype):
    """A cache whose second layer and later positions lie more than 2^31 elements from its first."""
    L, n_kv, hd, group, n_past = 20, 2, 64, 2, 500
    run = handle(L, n_kv, hd, dtype)
    g = torch.Generator(device="cuda").manual_seed(Lq)
    S, pos = n_past + Lq, 1 << 16
    size = L * n_kv * hd + (S - 1) * (1 << 22) + pos
    buf = [torch.empty(size, dtype=dtype, device="cuda") for _ in range(2)]
    K, V = (b.as_strided((1, L, n_kv, S, hd), (0, n_kv * hd, hd, 1 << 22, 1)) for b in buf)
    for x in (K, V):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    Q = torch.randn(1, L, group * n_kv, Lq, hd, generator=g, device="cuda").to(dtype)
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, 10, 490, out)
    mone.mone_mem_sync(run.h)
    run.close()
    for layer in (0, L - 1):
        ref, _ = O.window_attention(Q[0, layer].float().cpu(), K[0, layer].float().cpu(), V[0, layer].float().cpu(), n_past, 10, 490)
        assert rel_fro(out[0, layer].float().cpu(), ref) <= TOL[dtype], layer


# ----------------------------------------------------------------- what rows of padding, equal values and long recomputations show

@pytest.mark.parametrize("group,hd", [(7, 64), (7, 128), (3, 64), (5, 128)])
def test_rows_of_padding_have_no_say(group, hd):
    """A group that does not divide the tile's 128 rows leaves some that no copy fills: what a kernel before left in shared memory
    there changes no bit.  Scores grow by half a unit a position, so that every row is rescaled several times."""
    n_kv, L, n_past, Lq = 2, 20, 300, 150
    runs = handle(L, n_kv, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(group)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    K, V, Q = rn(1, L, n_kv, n_past + Lq, hd), rn(1, L, n_kv, n_past + Lq, hd), rn(1, L, group * n_kv, Lq, hd)
    Q[..., 0] = hd ** 0.5 if hd == 64 else 11.3125
    K[..., 0] = torch.arange(n_past + Lq, device="cuda") * 0.5
    K2, V2 = rn(1, L, n_kv, 2000, hd), rn(1, L, n_kv, 2000, hd)
    outs = []
    for left in (0.0, float("nan"), 1e30, float("inf")):  # queries of a call that fills all rows of every tile
        q2 = torch.full((1, L, 4 * n_kv, 2000, hd), left, dtype=torch.bfloat16, device="cuda")
        mone.mone_window_attention(runs.h, -1, q2, 4 * n_kv, 2000, K2, V2, K2.stride()[:4], 0, 0, 64, torch.empty_like(q2))
        torch.cuda.synchronize()
        out = torch.full_like(Q, 7.0)
        mone.mone_window_attention(runs.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, 16, ALL, out)
        outs.append(out)
    mone.mone_mem_sync(runs.h)
    runs.close()
    ref, _ = O.window_attention(Q[0, 3].float().cpu(), K[0, 3].float().cpu(), V[0, 3].float().cpu(), n_past, 16, ALL)
    assert rel_fro(outs[0][0, 3].float().cpu(), ref) <= 5e-3
    for out in outs[1:]:
        assert torch.equal(outs[0], out)


@pytest.mark.parametrize("hd", [64, 128])
def test_a_token_that_is_not_a_number_leaves_the_others_as_they_are(hd):
    """Its row shares a warp with other tokens', which are rescaled, as above, whatever it holds: not a bit of theirs changes."""
    n_kv, group, L, n_past, Lq = 2, 4, 20, 300, 150
    run = handle(L, n_kv, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(hd)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    K, V, Q = rn(1, L, n_kv, n_past + Lq, hd), rn(1, L, n_kv, n_past + Lq, hd), rn(1, L, group * n_kv, Lq, hd)
    Q[..., 0] = hd ** 0.5 if hd == 64 else 11.3125
    K[..., 0] = torch.arange(n_past + Lq, device="cuda") * 0.5
    outs = [torch.full_like(Q, 7.0) for _ in range(2)]
    for out in outs:
        mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, 16, ALL, out)
        Q[..., 40, :] = float("nan")
    mone.mone_mem_sync(run.h)
    run.close()
    assert outs[1][..., 40, :].isnan().all()
    outs[1][..., 40, :] = outs[0][..., 40, :]
    assert torch.equal(*outs)


@pytest.mark.parametrize("L,Lq,hd,late", [(20, 300, 64, 1.0), (20, 300, 128, 1.0), (20, 300, 64, 6.0), (1, 5, 64, 1.0), (1, 5, 128, 6.0)])
def test_values_that_are_all_the_same_come_out_as_they_are(L, Lq, hd, late):
    """The weights that a bf16 output is made of add up to 1: 32-bit sums of some hundred terms are off by 2^-16 at most, which is far
    below half of a bf16 place, so the output is the value exactly."""
    n_kv, group, n_past = 2, 4, 500
    run = handle(L, n_kv, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(Lq + hd)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    K, V, Q = rn(1, L, n_kv, n_past + Lq, hd), rn(1, L, n_kv, 1, hd).repeat(1, 1, 1, n_past + Lq, 1), 2 * rn(1, L, group * n_kv, Lq, hd)
    K[..., n_past // 2:, :] *= late
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, group * n_kv, Lq, K, V, K.stride()[:4], n_past, 7, 333, out)
    mone.mone_mem_sync(run.h)
    run.close()
    assert torch.equal(out, V[..., :1, :].repeat_interleave(group, 2).expand_as(out))


def test_rows_that_take_seconds_to_compute_again_do_not_time_out():
    """A value of the first position is infinite in one dimension: every row is computed again over all of its 450,000 positions, which
    takes a warp more than the 2 s of a wait for its 32, while the others wait for its next tile."""
    group, hd, Lq, S = 4, 128, 6000, 450000  # more pairs of tiles than CTAs
    run = handle(1, 2, hd, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(hd)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    K, V, Q = rn(1, 1, 1, S, hd), rn(1, 1, 1, S, hd), rn(1, 1, 2 * group, Lq, hd)  # both KV heads read the same: stride 0
    V[0, 0, 0, 0, 5] = float("inf")
    out = torch.full_like(Q, 7.0)
    mone.mone_window_attention(run.h, -1, Q, 2 * group, Lq, K, V, (S * hd, S * hd, 0, hd), S - Lq, 0, ALL, out)
    mone.mone_mem_sync(run.h)
    run.close()
    assert out[..., 5].isposinf().all()
    rest = [d for d in range(hd) if d != 5]
    k, v = K[0, 0, 0].float(), V[0, 0, 0, :, rest].double()
    for i in (0, 1, 37, Lq // 2, Lq - 1):
        n = S - Lq + i + 1
        ref = torch.softmax((Q[0, 0, :, i].float() @ k[:n].T).double() / hd ** 0.5, -1) @ v[:n]
        assert rel_fro(out[0, 0, :, i][:, rest].double().cpu(), ref.cpu()) <= 5e-3, i


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_past", [0, 1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 65])
def test_last_chunks_of_every_width(n_past, hd):
    """Chunks of 64 keys, tiles of 32 tokens: a pair of tiles whose last chunk ends with n_past % 64 of its keys in the second tile and
    with half a chunk less or more in the first, in sixteens and one more or less."""
    case(4, 64, n_past, 0, ALL, hd, n_layers=20)
    case(4, 41, n_past, 3, 70, hd, n_layers=20)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_sink,window", [(0, 63), (0, 64), (0, 65), (63, 64), (64, 63), (64, 64), (65, 65), (127, 64), (128, 128),
                                           (129, 127), (64, 129), (65, 1), (128, 0), (127, 0)])
def test_first_positions_and_windows_at_the_ends_of_chunks(n_sink, window, hd):
    case(4, 133, 300, n_sink, window, hd, n_layers=20)
