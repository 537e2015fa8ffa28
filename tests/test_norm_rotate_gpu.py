"""GPU parity of the heads' normalisation and rotation against the formula in 64 bits.

Tolerances, per row relative to its largest pair: an angle of 32 bits of a turn is off by 2^-32 turns, 1.5e-9; cosine and sine by 2^-22
at most; norm, scale and the two products by 2^-23 each: 6 x 2^-23 = 7e-7 for fp32, and half a step more for bf16, whose 8 bits are
2^-7 apart at 1: 2^-8 of an element.
"""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2608_17616_gb300 as mone
from test_cache4_gpu import handle

pytestmark = pytest.mark.gpu
TOL = 6 * 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_17616_gb300 import build
    build.build()
    mone.lib()


def layout(order, B, L, H, n, hd, dtype, pad=0):
    """A tensor [contexts, layers, heads, tokens, hd] of that memory order."""
    shape = {"head": (B, L, H, n), "token": (B, L, n, H), "layers inner": (B, n, H, L)}[order]
    perm = {"head": (0, 1, 2, 3, 4), "token": (0, 1, 3, 2, 4), "layers inner": (0, 3, 2, 1, 4)}[order]
    return torch.full((*shape, hd + pad), 7.0, dtype=dtype, device="cuda").permute(*perm)[..., :hd]


def check(got, x, w, pos, rotary_freq, halves, eps):
    """One head's rows."""
    ref = O.norm_rotate(x.double().cpu().numpy(), w, pos, rotary_freq, halves, eps)
    got, tol = got.double().cpu().numpy(), TOL * np.abs(ref).max(-1, keepdims=True)
    if x.dtype is torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(got - ref) <= tol * 1.01 + 1e-37).all(), np.abs(got - ref).max()


def run(B=2, L=2, n_q=4, n_kv=2, n_tok=5, hd=64, dtype=torch.bfloat16, rot=None, halves=True, period=0, base=10000.0, norm=True, first=(0, 100),
        order="token", to="head", pad=0, layer=-1, in_place=False, sides="qk", scale=1.0, eps=1e-6, freq=None, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rot = hd if rot is None else rot
    h = handle(B, L, n_kv, hd, dtype)
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)] if freq is None else freq
    rotary = mone.make_rotary(rot, mone.MONE_ROTATE_HALVES if halves else mone.MONE_ROTATE_NEIGHBOURS, base=base or 1.0, period=period, eps=eps,
                              freq=freq if base is None else None)
    first_t = None if first is None else torch.tensor(first[:B], dtype=torch.int32, device="cuda")
    heads, kept, alive = [], [], []
    for side, H in (("q", n_q), ("k", n_kv)):
        if side not in sides:
            heads.append(None)
            continue
        x = layout(order, B, L, H, n_tok, hd, dtype, pad)
        x.copy_((scale * torch.randn(x.shape, generator=g, device="cuda")).to(dtype))
        out = x if in_place else layout(to, B, L, H, n_tok, hd, dtype, pad)
        w = 1 + 0.3 * torch.randn(L, hd, generator=g, device="cuda") if norm else None
        kept.append((x.clone(), out, w))
        alive.append(x)
        heads.append(mone.make_heads(x, out, w))
    mone.mone_norm_rotate(h, layer, rotary, first_t, n_tok, *heads)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    for x, out, w in kept:
        for c in range(B):
            p = (0 if first is None else first[c]) + np.arange(n_tok, dtype=np.int64)
            p = p % period if period else p
            for l in range(L):
                for a in range(x.shape[2]):
                    if layer < 0 or l == 0:
                        check(out[c, l, a], x[c, l, a], None if w is None else w[max(layer, l)].cpu().numpy(), p, freq, halves, eps)
                    else:
                        assert torch.equal(out[c, l, a], x[c, l, a] if in_place else torch.full_like(x[c, l, a], 7.0))
    return kept


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("hd,rot", [(64, 64), (128, 128), (64, 32), (128, 48), (128, 16), (64, 0)])
@pytest.mark.parametrize("norm", [True, False])
def test_sizes_and_pairings(hd, rot, halves, norm, dtype):
    run(hd=hd, rot=rot, halves=halves, norm=norm, dtype=dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kw", [
    dict(n_tok=1), dict(n_tok=1, B=1, L=1, sides="k"), dict(sides="q"), dict(sides="k", n_tok=33),
    dict(n_tok=301, L=3, n_q=10, n_kv=2),                  # a job of several rows, the last one short
    dict(n_tok=2000, L=2, n_q=7, n_kv=1, hd=64), dict(B=1, first=(9,), n_tok=700, n_q=24, n_kv=3, hd=128),
    dict(order="head", to="token"), dict(order="layers inner", to="head"), dict(order="token", to="layers inner"),
    dict(pad=8), dict(pad=1), dict(pad=3, order="head", n_tok=65, hd=128), dict(in_place=True), dict(in_place=True, pad=5, order="layers inner"),
    dict(layer=1), dict(layer=0, in_place=True), dict(first=None), dict(period=16, n_tok=100), dict(period=1), dict(period=1000, first=(999, 123456)),
    dict(first=(2 ** 31 - 70, 2 ** 31 - 6)),               # the last positions that there are
    dict(first=(1000000, 16777217), base=500000.0), dict(base=1.0, first=(12345, 7)),  # whole radians a position
    dict(base=None, freq=[0.0, -1.0, 3.0, 100.25, 1e-9, 6.25, 2e5, 0.5], rot=16, first=(70000, 3)),
    dict(eps=0.0), dict(eps=1.0), dict(scale=1e-3),
])
def test_orders_positions_and_ranges(kw, dtype):
    run(**dict(dict(dtype=dtype), **kw))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_whose_squares_leave_the_range(dtype):
    """Squares past 2^128 and below 2^-126: the norm is the row's all the same.  Zeros stay zeros; NaN and infinity make their row NaN."""
    run(scale=1e25, dtype=dtype)
    run(scale=1e37, dtype=dtype)
    run(scale=1e-25, eps=0.0, dtype=dtype)
    h = handle(1, 1, 2, 64, dtype)
    x = torch.randn(1, 1, 2, 4, 64, device="cuda").to(dtype)
    x[0, 0, 0, 0] = 0
    x[0, 0, 0, 2, 5] = float("nan")
    x[0, 0, 1, 1, 9] = float("inf")
    out, w = torch.empty_like(x), torch.ones(1, 64, device="cuda")
    mone.mone_norm_rotate(h, -1, mone.make_rotary(64), None, 4, mone.make_heads(x, out, w), None)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    assert not out[0, 0, 0, 0].any() and out[0, 0, 0, 2].isnan().all()
    assert not out[0, 0, 1, 1].isfinite().any() or out[0, 0, 1, 1].isnan().any()
    fine = [(0, 1), (0, 3), (1, 0), (1, 2), (1, 3)]
    for a, i in fine:
        check(out[0, 0, a, i:i + 1], x[0, 0, a, i:i + 1], np.ones(64), [i], [10000.0 ** (-2.0 * j / 64) for j in range(32)], True, 1e-6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 112])
def test_what_is_not_finite_reaches_its_pair_alone(rot, halves, dtype):
    """Without a norm, an element is turned with its partner or left as it is, whatever the others of its row are."""
    h, hd, n_tok = handle(1, 1, 1, 128, dtype), 128, 128
    x = torch.randn(1, 1, 1, n_tok, hd, device="cuda").to(dtype)
    for t in range(n_tok):
        x[0, 0, 0, t, t] = [float("inf"), -float("inf"), float("nan")][t % 3]
    out = torch.empty_like(x)
    rotary = mone.make_rotary(rot, mone.MONE_ROTATE_HALVES if halves else mone.MONE_ROTATE_NEIGHBOURS, base=100.0)
    mone.mone_norm_rotate(h, -1, rotary, None, n_tok, None, mone.make_heads(x, out))
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    fine = x.clone()
    fine[~x.isfinite()] = 1.0
    ref = O.norm_rotate(fine[0, 0, 0].double().cpu().numpy(), None, np.arange(n_tok), [100.0 ** (-2.0 * i / max(rot, 1)) for i in range(rot // 2)], halves, 0.0)
    got = out[0, 0, 0].double().cpu().numpy()
    for t in range(n_tok):
        mate = t if t >= rot else (t + rot // 2) % rot if halves else t ^ 1
        if t >= rot:
            assert np.array_equal(got[t, t], x[0, 0, 0, t, t].item(), equal_nan=True)
        rest = np.array([i not in (t, mate) for i in range(hd)])
        tol = TOL * np.abs(ref[t]).max() + (2.0 ** -8 * np.abs(ref[t]) if dtype is torch.bfloat16 else 0)
        assert (np.abs(got[t] - ref[t]) <= tol * 1.01)[rest].all()


def test_a_layer_by_itself():
    """One layer's tensors, as a backbone that runs layer by layer has them, and the weights of all."""
    B, L, n_tok = 2, 3, 4
    h, w = handle(B, L, 2, 64), 1 + 0.3 * torch.randn(L, 64, device="cuda")
    x = torch.randn(B, 1, n_tok, 2, 64, device="cuda").bfloat16().transpose(2, 3)
    first = torch.tensor([7, 30], dtype=torch.int32, device="cuda")
    for l in range(L):
        out = torch.empty(B, 1, 2, n_tok, 64, dtype=x.dtype, device="cuda")
        mone.mone_norm_rotate(h, l, mone.make_rotary(64), first, n_tok, None, mone.make_heads(x, out, w))
        mone.mone_mem_sync(h)
        for c in range(B):
            for a in range(2):
                check(out[c, 0, a], x[c, 0, a], w[l].cpu().numpy(), [7, 30][c] + np.arange(n_tok), [10000.0 ** (-i / 32) for i in range(32)], True, 1e-6)
    mone.mone_mem_free(h)


def test_offsets_past_32_bits():
    """A strided view whose last rows lie more than 2^32 bytes from its first."""
    n_tok, stride = 9, (1 << 31) // 8 + 64
    buf = torch.empty(n_tok * stride, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((1, 1, 2, n_tok, 64), (0, 0, 64, stride, 1))
    x.copy_(torch.randn(x.shape, device="cuda"))
    h = handle(1, 1, 2, 64)
    before = x.clone()
    mone.mone_norm_rotate(h, -1, mone.make_rotary(64), None, n_tok, mone.make_heads(x, x), None)
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    for a in range(2):
        check(x[0, 0, a], before[0, 0, a], None, np.arange(n_tok), [10000.0 ** (-i / 32) for i in range(32)], True, 1e-6)


@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("base,rot", [(500000.0, 128), (1000000.0, 128), (10000.0, 64)])
def test_slow_pairs_turn_by_angles_of_full_precision(base, rot, halves):
    """(0, 1) becomes (-sin, cos), each to bits of its own however small the angle is.  The angle is off by 2^-23 of itself at most, and sine and
    cosine by 2^-22 of themselves: 2^-21 in all."""
    hd, first = rot, [1, 1000]
    h, n_tok = handle(2, 1, 2, hd, torch.float32), 9
    x = torch.zeros(2, 1, 2, n_tok, hd, device="cuda")
    b = slice(rot // 2, rot) if halves else slice(1, rot, 2)
    a = slice(0, rot // 2) if halves else slice(0, rot, 2)
    x[..., b] = 1.0
    out = torch.empty_like(x)
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    rotary = mone.make_rotary(rot, mone.MONE_ROTATE_HALVES if halves else mone.MONE_ROTATE_NEIGHBOURS, freq=freq)
    mone.mone_norm_rotate(h, -1, rotary, torch.tensor(first, dtype=torch.int32, device="cuda"), n_tok, None, mone.make_heads(x, out))
    mone.mone_mem_sync(h)
    mone.mone_mem_free(h)
    for c in range(2):
        angle = (first[c] + np.arange(n_tok))[:, None] * np.array(freq)
        for got, ref in ((out[c, 0, :, :, a], -np.sin(angle)), (out[c, 0, :, :, b], np.cos(angle))):
            err = np.abs(got.double().cpu().numpy() - ref) / np.abs(ref)
            assert err.max() <= 2.0 ** -21, err.max()
