"""The 4-bit cache, the pages and the rotation without a GPU: the oracle's definitions pinned by special cases, refused arguments, and
the host code of the launches."""
import ctypes
import shutil
from fractions import Fraction

import numpy as np
import pytest

import oracle as O
import paper_2608_17616_gb300 as mone
from fakert import Fake, build_fake

P = 1 << 30  # a made-up, aligned device address


# ----------------------------------------------------------------- the oracle

def test_every_4_bit_number_comes_back():
    for s in range(1, 127):
        code = np.arange(16)
        x = O.four_bit_values(code, np.array([s]))
        got, scale = O.four_bits(x)
        assert scale.tolist() == [s] and np.array_equal(got, code)  # the largest code is 6, so the scale is the group's own
    assert O.E4M3[:9].tolist() == [0, 2 ** -9, 2 ** -8, 3 * 2 ** -9, 2 ** -7, 5 * 2 ** -9, 6 * 2 ** -9, 7 * 2 ** -9, 2 ** -6]
    assert O.E4M3[-1] == 448 and len(O.E4M3) == 127


def test_rounding_to_4_bits_by_hand():
    x = np.array([6.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -0.74, -6.0, 0.0, -0.0, 2.51, -3.49])
    code, scale = O.four_bits(x)
    assert O.E4M3[scale[0]] == 1.0
    assert O.four_bit_values(code, scale).tolist() == [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -0.5, -6, 0, 0, 3, -3]
    tie = np.full(16, 6 * (1 + 1 / 16))  # halfway between the scales 1 and 1 + 1/8: the even one
    assert O.E4M3[O.four_bits(tie)[1][0]] == 1.0 and O.E4M3[O.four_bits(np.full(16, 6 * (1 + 3 / 16)))[1][0]] == 1.25
    assert O.four_bit_values(*O.four_bits(np.full(16, 1e9)))[0] == 2688 and O.four_bit_values(*O.four_bits(np.full(16, np.inf)))[0] == 2688
    assert O.four_bits(np.full(16, 1e-4))[1][0] == 0 and np.isnan(O.four_bit_values(*O.four_bits(np.array([np.nan] + [1.0] * 15)))).all()
    assert O.four_bit_values(*O.four_bits(x * 8, 3), 3).tolist() == (8 * O.four_bit_values(code, scale)).tolist()


def test_rotation_by_hand():
    x, quarter = np.array([[1.0, 2.0, 3.0, 4.0, 9.0]]), [np.pi / 2, np.pi]
    assert np.allclose(O.norm_rotate(x, None, [1], quarter, True, 0.0), [[-3, -2, 1, -4, 9]])
    assert np.allclose(O.norm_rotate(x, None, [1], quarter, False, 0.0), [[-2, 1, -3, -4, 9]])
    assert np.allclose(O.norm_rotate(x, None, [0], quarter, True, 0.0), x)
    y = O.norm_rotate(x, [2.0] * 5, [3], quarter, True, 0.0)
    assert np.isclose((y * y).mean(), 4.0)


def test_rotated_products_go_by_the_distance():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 16)), rng.standard_normal((1, 16))
    freq = [100.0 ** (-i / 8) for i in range(8)]
    dots = [(O.norm_rotate(q, None, [p + 5], freq, h, 0) * O.norm_rotate(k, None, [p], freq, h, 0)).sum() for p in (0, 3, 77) for h in (True, False)]
    assert np.allclose(dots[::2], dots[0]) and np.allclose(dots[1::2], dots[1])


def test_pages_by_hand():
    free, tables, granted, slots = O.cache_reserve([7, 8, 9], [[3], []], [3, 0], [2, 5], 4, 4)
    assert (free, tables, granted) == ([], [[3, 7], [8, 9]], [2, 5])
    assert slots == [[15, 28], [32, 33, 34, 35, 36]]
    assert O.cache_release(free, tables, [5, 5], [3, 0], 4) == ([7, 8, 9], [[3], []])
    assert O.cache_reserve([7], [[3], [], [1]], [3, 0, 2], [2, 5, 2], 4, 4)[1:3] == ([[3, 7], [], [1]], [2, 0, 2])
    assert O.cache_reserve([7, 8], [[], []], [0, 0], [9, 1], 4, 2)[1:3] == ([[], [8]], [0, 1])  # too wide for its table


# ----------------------------------------------------------------- the library's host code

@pytest.fixture(scope="module")
def built(tmp_path_factory):
    return build_fake(tmp_path_factory.mktemp("fakert"))


@pytest.fixture()
def fake(tmp_path, monkeypatch, built):
    path = shutil.copy(built, tmp_path / "libmone_fakert.so")
    f = Fake(str(path))
    monkeypatch.setattr(mone, "_lib", mone.lib(str(path)))
    return f


def init(n_ctx=2, L=3, n_kv=2, hd=64, dtype=mone.MONE_BF16):
    cfg = mone.make_config(n_ctx, L, 256, 256, 2 * n_kv * hd, n_kv, hd, 128, dtype, mone.MONE_PLAIN, 1e-2)
    return mone.mone_mem_init(cfg, P, P, None, 0)


def strides(*s):
    return (ctypes.c_longlong * 4)(*s)


def cache(n_kv=2, hd=64, page=16, n_pages=40, width=10, score=P, **kw):
    row = [hd // 2, hd // 16]
    c = mone.mone_cache4(P, P, P, P, *(strides(n_pages * n_kv * page * r, n_kv * page * r, page * r, r) for r in row), 0, 0, n_pages, page, P,
                         width, P + 4096, score)
    for k, v in kw.items():
        setattr(c, k, strides(*v) if "strides" in k else v)
    return c


def refused(code, fn, *a):
    with pytest.raises(mone.MoneError) as e:
        fn(*a, stream=0)
    assert e.value.code == code, e.value


def tensor(ptr, *shape):
    return type("T", (), dict(shape=shape, data_ptr=lambda self: ptr))()


ST = (10 ** 6, 10 ** 4, 640, 64)
BAD_CACHE = [(1, dict(K=None)), (1, dict(V=P + 8)), (1, dict(K_scale=None)), (1, dict(V_scale=P + 2)), (1, dict(table=None)), (1, dict(lens=None)),
             (1, dict(lens=P + 2)), (1, dict(n_pages=0)), (1, dict(page_size=0)), (2, dict(page_size=24)), (2, dict(page_size=2048)),
             (1, dict(table_width=0)), (1, dict(table_width=1 << 27)), (1, dict(strides=(1024, 1024, -32, 32))), (1, dict(strides=(1024, 1024, 512, 16))),
             (1, dict(strides=(1024, 1024, 512, 40))), (1, dict(strides=(1000, 1024, 512, 32))), (1, dict(strides=(1024, 0, 512, 32))),
             (1, dict(scale_strides=(128, 128, 64, 2))), (1, dict(scale_strides=(128, 130, 64, 4))), (1, dict(scale_strides=(128, 0, 64, 4))),
             (1, dict(scale_strides=(128, 128, -64, 4))), (1, dict(k_exp=65)), (1, dict(v_exp=-65))]


@pytest.mark.parametrize("code,kw", BAD_CACHE)
def test_a_bad_cache_is_refused_by_every_operator(fake, code, kw):
    h, c = init(), cache(**kw)
    refused(code, mone.mone_cache4_append, h, -1, c, P, P, ST, 3)
    refused(code, mone.mone_cache4_read, h, -1, c, None, 5, P, P, ST)
    refused(code, mone.mone_cache4_attention, h, -1, c, P, 4, 1, 0, 100, P)
    refused(code, mone.mone_cache4_evict, h, -1, c, 50, 2, 3, tensor(P + 64, 2, 10), P + 128, P)
    assert not [x for x in fake.drain()[0] if "cache" in x["name"]]


def each_bad(fn, good, bads):
    for i, bad in bads:
        refused(1, fn, *[bad if k == i else x for k, x in enumerate(good)])


def test_cache_operator_refusals(fake):
    h, c = init(), cache()
    n0 = mone.mone_mem_launch_count(h)
    each_bad(mone.mone_cache4_append, [h, -1, c, P, P, ST, 3, P, P],
             ((0, 0x1234), (1, 3), (1, -2), (3, None), (4, P + 1), (5, (1, 1, 1, -1)), (6, 0), (6, (1 << 20) + 1), (7, P + 4096), (7, P + 1), (8, P + 2)))
    each_bad(mone.mone_cache4_read, [h, -1, c, P, 5, P, P, ST],
             ((0, 0x1234), (1, 3), (3, P + 1), (4, 0), (4, (1 << 20) + 1), (5, None), (6, P + 1), (7, (1, 1, 1, -1)), (7, (10 ** 6, 10 ** 4, 640, 63)),
              (7, (10 ** 6, 10 ** 4, 0, 64)), (7, (10 ** 6, 0, 640, 64)), (7, (0, 10 ** 4, 640, 64))))
    mone.mone_cache4_read(h, 1, c, P, 1, P, P, (10 ** 6, 0, 640, 0), stream=0)  # one layer, one place
    each_bad(mone.mone_cache4_attention, [h, -1, c, P, 4, 1, 0, 100, P],
             ((0, 0x1234), (1, 3), (3, None), (3, P + 8), (4, 3), (4, 130), (5, 0), (5, 17), (6, -1), (7, -1), (8, None)))
    each_bad(mone.mone_cache4_evict, [h, -1, c, 50, 2, 3, tensor(P + 64, 2, 10), P + 128, P, P],
             ((0, 0x1234), (1, 3), (2, cache(score=None)), (3, 0), (3, 4), (4, -1), (5, -1), (6, tensor(P, 2, 10)), (6, tensor(P + 64, 2, 3)),
              (6, tensor(P + 65, 2, 10)), (7, None), (7, P), (8, None), (9, P + 4096)))
    assert mone.mone_mem_launch_count(h) == n0 + 1


def pages(**kw):
    p = mone.mone_pages(P, P + 64, 40, 16, P + 128, 10, P + 4096)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("code,kw", [(1, dict(free=None)), (1, dict(n_free=None)), (1, dict(table=None)), (1, dict(lens=None)), (1, dict(free=P + 1)),
                                     (1, dict(table=P + 2)), (1, dict(n_pages=0)), (1, dict(page_size=0)), (2, dict(page_size=24)),
                                     (2, dict(page_size=2048)), (1, dict(table_width=0)), (1, dict(table_width=1 << 27))])
def test_bad_pages_are_refused(fake, code, kw):
    h, p = init(), pages(**kw)
    refused(code, mone.mone_cache_reserve, h, p, 3, P + 8)
    refused(code, mone.mone_cache_release, h, p, P + 8)
    assert not [x for x in fake.drain()[0] if "cache" in x["name"]]


def test_page_operator_refusals(fake):
    h, p = init(), pages()
    n0 = mone.mone_mem_launch_count(h)
    each_bad(mone.mone_cache_reserve, [h, p, 3, P + 8, P + 16, P + 32, P + 48, P + 96],
             ((0, 0x1234), (2, 0), (2, (1 << 20) + 1), (3, None), (3, P + 64), (3, P + 9), (4, P + 4096), (4, P + 17), (5, P + 96), (5, P + 4096),
              (5, P + 16), (5, P + 33), (6, P + 52), (7, P + 97)))
    each_bad(mone.mone_cache_release, [h, p, P + 8, P + 16, P + 32],
             ((0, 0x1234), (2, None), (2, P + 64), (2, P + 9), (3, P + 17), (4, P + 4096), (4, P + 16), (4, P + 33)))
    assert mone.mone_mem_launch_count(h) == n0


def heads(**kw):
    s = mone.mone_heads(P, P + 65536, P, strides(*ST), strides(*ST), 4)
    for k, v in kw.items():
        setattr(s, k, strides(*v) if "strides" in k else v)
    return s


def test_rotation_refusals(fake):
    h, r, s = init(), mone.make_rotary(64), heads()
    good = [h, -1, r, P, 3, s, s]
    mone.mone_norm_rotate(*good, stream=0)
    n0 = mone.mone_mem_launch_count(h)
    bad = [heads(x=None), heads(out=None), heads(n_heads=0), heads(n_heads=4097), heads(x=P + 1), heads(weight=P + 2),
           heads(strides=(1, 1, -1, 64)), heads(out_strides=(10 ** 6, 10 ** 4, 640, 63)), heads(out_strides=(10 ** 6, 10 ** 4, 0, 64)),
           heads(out_strides=(10 ** 6, 0, 640, 64)), heads(out_strides=(0, 10 ** 4, 640, 64)), heads(out=P, out_strides=(10 ** 6, 10 ** 4, 640, 128))]
    each_bad(mone.mone_norm_rotate, good, ((0, 0x1234), (1, 3), (1, -2), (3, P + 1), (4, 0), (4, (1 << 24) + 1), (2, mone.make_rotary(128)),
                                           *((5, b) for b in bad), *((6, b) for b in bad)))
    refused(1, mone.mone_norm_rotate, h, -1, r, P, 3, None, None)
    for field, v in (("rot_dim", 24), ("rot_dim", -16), ("pairing", 2), ("period", -1), ("eps", -1.0), ("eps", float("nan"))):
        other = mone.make_rotary(64)
        setattr(other, field, v)
        refused(1, mone.mone_norm_rotate, h, -1, other, P, 3, s, s)
    assert mone.mone_mem_launch_count(h) == n0
    mone.mone_norm_rotate(h, 2, r, None, 3, None, heads(out=P, out_strides=ST), stream=0)  # in place


def test_rotary_make_refusals():
    for a, kw in (((8,), {}), ((144,), {}), ((-16,), {}), ((64, 2), {}), ((64,), dict(period=-1)), ((64,), dict(eps=-1.0)),
                  ((64,), dict(eps=float("inf"))), ((64,), dict(base=0.0)), ((64,), dict(base=float("nan"))), ((16,), dict(freq=[float("inf")] * 8)),
                  ((16,), dict(freq=[0.0] * 7 + [-2.0 ** 31]))):
        with pytest.raises(mone.MoneError) as e:
            mone.make_rotary(*a, **kw)
        assert e.value.code == 1
    with pytest.raises(ValueError):
        mone.make_rotary(16, freq=[1.0] * 7)
    raw = mone.lib().mone_rotary_make
    assert raw(None, 16, 0, None, 10.0, 0, 0.0) == 1


def test_turns_are_the_frequencies_in_turns():
    """To 64 bits: of exact fractions, rounding is off by a few at most."""
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899, 10 ** 80)
    some = [0.0, -1.0, 2 * np.pi, 100.0, 1e-9, np.pi, 2e5, 0.5, -3e-20, 2.0 ** 31 - 1, 1e-300, -12345.678]
    for freq in ([10000.0 ** (-i / 32) for i in range(32)], [500000.0 ** (-i / 64) for i in range(64)], some * 2):
        r = mone.make_rotary(2 * len(freq), freq=freq)
        for t, f in zip(r.turns, freq):
            d = (t - int(Fraction(f) / (2 * pi) * 2 ** 64)) % 2 ** 64
            assert min(d, 2 ** 64 - d) <= 3, f
        assert list(r.turns[len(freq):]) == [0] * (64 - len(freq))
    assert all(a == b for a, b in zip(mone.make_rotary(64, base=500000.0).turns, mone.make_rotary(64, freq=[500000.0 ** (-2.0 * i / 64) for i in range(32)]).turns))


@pytest.mark.parametrize("dtype", [mone.MONE_BF16, mone.MONE_FP32])
def test_launches_and_counts_on_either_device(fake, dtype):
    for dev, sms in ((0, 152), (1, 100), (0, 152)):
        fake.device(dev)
        h, c, wide = init(dtype=dtype), cache(), cache(width=2000)
        fake.drain()
        n0 = mone.mone_mem_launch_count(h)
        for layer in (-1, 2):
            for call in (lambda: mone.mone_cache4_append(h, layer, c, P, P, ST, 3, stream=0),
                         lambda: mone.mone_cache4_read(h, layer, c, None, 3, P, P, ST, stream=0),
                         lambda: mone.mone_cache4_attention(h, layer, c, P, 4, 2, 1, 100, P, stream=0),
                         lambda: mone.mone_cache4_attention(h, layer, wide, P, 4, 2, 1, 1 << 30, P, stream=0),
                         lambda: mone.mone_cache4_evict(h, layer, c, 50, 2, 3, tensor(P + 64, 2, 10), P + 128, P, stream=0),
                         lambda: mone.mone_cache_reserve(h, pages(), 3, P + 8, stream=0),
                         lambda: mone.mone_cache_release(h, pages(), P + 8, stream=0),
                         lambda: mone.mone_norm_rotate(h, layer, mone.make_rotary(64), P, 3, heads(), heads(), stream=0)):
                call()
                n, launches = mone.mone_mem_launch_count(h), fake.drain()[0]
                assert n - n0 == len(launches) > 0 and {x["dev"] for x in launches} == {dev}
                n0 = n
        mone.mone_cache4_attention(h, -1, wide, P, 4, 2, 1, 1 << 30, P, stream=0)
        attention, finish = fake.drain()[0]
        assert attention["grid"][0] % sms == 0 and "finish" in finish["name"]
        mone.mone_mem_free(h)


def test_the_attentions_share_a_workspace_that_does_not_grow_during_a_capture(fake):
    h, c = init(), cache()
    mone.mone_cache4_attention(h, 0, c, P, 4, 1, 1, 100, P, stream=0)
    n0 = mone.mone_mem_launch_count(h)
    fake.capturing(True)
    with pytest.raises(mone.MoneError) as e:
        mone.mone_cache4_attention(h, -1, c, P, 4, 16, 1, 100, P, stream=0)
    assert e.value.code == 3 and "mone_cache4_attention" in str(e.value) and "capture" in str(e.value)
    mone.mone_cache4_attention(h, 0, c, P, 4, 1, 1, 100, P, stream=0)  # what fits goes on, and stays from now on
    fake.capturing(False)
    assert mone.mone_mem_launch_count(h) == n0 + 1
    fake.frees()
    mone.mone_cache4_attention(h, -1, c, P, 4, 16, 1, 100, P, stream=0)
    assert fake.frees() == []
    mone.mone_mem_free(h)


# ----------------------------------------------------------------- the binding's checks

def tensors(L=3, n_ctx=2, n_kv=2, hd=64, page=16, width=10, score=True):
    import torch
    pools = [torch.zeros(L, 40, n_kv, page, w, dtype=torch.uint8) for w in (hd // 2, hd // 2, hd // 16, hd // 16)]
    return [*pools, torch.zeros(n_ctx, width, dtype=torch.int32), torch.zeros(n_ctx, dtype=torch.int32),
            torch.zeros(n_ctx, L, n_kv, width * page) if score else None]


def test_make_cache4_takes_strides_and_refuses_what_does_not_go_together(fake):
    import torch
    K, V = (torch.zeros(2, 3, 16, 4, 32, dtype=torch.uint8).transpose(2, 3) for _ in range(2))
    Ks, Vs = (torch.zeros(2, 3, 16, 4, 4, dtype=torch.float8_e4m3fn).transpose(2, 3) for _ in range(2))
    t, n = torch.zeros(5, 7, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    c = mone.make_cache4(K, V, Ks, Vs, t, n, k_exp=3, v_exp=-2)
    assert tuple(c.strides) == (3 * 16 * 128, 16 * 128, 32, 128) and tuple(c.scale_strides) == (3 * 16 * 16, 16 * 16, 4, 16)
    assert (c.n_pages, c.page_size, c.table_width, c.k_exp, c.v_exp) == (3, 16, 7, 3, -2) and c.score is None
    good = tensors()
    mone.make_cache4(*good)
    for i, bad in ((0, good[0][:, :2]), (0, good[0].int()), (1, good[1].transpose(1, 2)), (2, good[2].int()), (2, torch.zeros(3, 40, 2, 16, 8, dtype=torch.uint8)),
                   (3, good[3][..., :3]), (4, torch.zeros(2, 10)), (5, torch.zeros(1, dtype=torch.int32)), (6, torch.zeros(2, 3, 2, 159)),
                   (6, torch.zeros(1, 3, 2, 160))):
        with pytest.raises(ValueError):
            mone.make_cache4(*[bad if k == i else x for k, x in enumerate(good)])
    h = init()
    to, to_score, kept = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 3, 2, 64), torch.zeros(2, 3, 2, 50, dtype=torch.int32)
    mone.mone_cache4_evict(h, -1, mone.make_cache4(*good), 50, 2, 3, to, to_score, kept, stream=0)
    for kw in (dict(L=2), dict(n_ctx=1), dict(n_kv=1), dict(hd=32), dict(L=4)):
        keep = tensors(**kw)
        c = mone.make_cache4(*keep)
        for call in (lambda: mone.mone_cache4_append(h, -1, c, P, P, ST, 3, stream=0), lambda: mone.mone_cache4_read(h, -1, c, None, 3, P, P, ST, stream=0),
                     lambda: mone.mone_cache4_attention(h, -1, c, P, 4, 1, 0, 100, P, stream=0),
                     lambda: mone.mone_cache4_evict(h, -1, c, 50, 2, 3, to, to_score, kept, stream=0)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        mone.mone_cache4_evict(h, -1, mone.make_cache4(*good), 50, 2, 3, to, to_score[..., :63], kept, stream=0)


def test_pages_and_heads_of_tensors(fake):
    import torch
    h = init()
    z = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    good = [z(40), z(1), z(2, 10), z(2)]
    p = mone.make_pages(*good, 16)
    mone.mone_cache_reserve(h, p, 3, z(1), z(2), z(2), torch.zeros(2, 3, dtype=torch.int64), z(2), stream=0)
    mone.mone_cache_release(h, p, z(1), z(2), z(2), stream=0)
    for i, bad in ((0, z(40).long()), (1, z(1, 1)), (2, z(10, 2).T), (3, z(1))):
        with pytest.raises(ValueError):
            mone.make_pages(*[bad if k == i else x for k, x in enumerate(good)], 16)
    for a in ([z(0)], [z(1), z(1)], [z(1), None, z(1)], [z(1), None, None, torch.zeros(2, 2, dtype=torch.int64)], [z(1), None, None, z(2, 3)],
              [z(1), None, None, None, z(1)], [torch.zeros(1)]):
        with pytest.raises(ValueError):
            mone.mone_cache_reserve(h, p, 3, *a, stream=0)
    for a in ([z(0)], [z(1), z(1)], [z(1), None, z(1)]):
        with pytest.raises(ValueError):
            mone.mone_cache_release(h, p, *a, stream=0)
    with pytest.raises(ValueError):
        mone.mone_cache_release(h, mone.make_pages(z(40), z(1), z(1, 10), z(1), 16), z(1), stream=0)

    def x(B=2, L=3, H=4, n=5, hd=64, dtype=torch.bfloat16):
        return torch.zeros(B, L, n, H, hd, dtype=dtype).transpose(2, 3)

    r, w = mone.make_rotary(64), torch.zeros(3, 64)
    s = mone.make_heads(x(), x(), w)
    assert tuple(s.strides) == (3 * 5 * 256, 5 * 256, 64, 256) and s.n_heads == 4
    mone.mone_norm_rotate(h, -1, r, z(2), 5, s, None, stream=0)
    mone.mone_norm_rotate(h, 2, r, None, 5, None, mone.make_heads(x(L=1), x(L=1), w), stream=0)
    for a in ((x(), x(H=3)), (x(), x().float()), (x().half(), x().half()), (x(), x().contiguous()[..., ::2]), (x(), x(), w.bfloat16()), (x(), x(), w[:, :32]),
              (x(), x(), torch.zeros(64))):
        with pytest.raises(ValueError):
            mone.make_heads(*a)
    for side in (mone.make_heads(x(B=1), x(B=1)), mone.make_heads(x(L=2), x(L=2)), mone.make_heads(x(n=4), x(n=4)), mone.make_heads(x(hd=128), x(hd=128)),
                 mone.make_heads(x(dtype=torch.float32), x(dtype=torch.float32)), mone.make_heads(x(), x(), w[:2].contiguous())):
        for q, k in ((side, None), (s, side)):
            with pytest.raises(ValueError):
                mone.mone_norm_rotate(h, -1, r, None, 5, q, k, stream=0)
    with pytest.raises(ValueError):
        mone.mone_norm_rotate(h, -1, r, z(1), 5, s, None, stream=0)


def test_outputs_that_overlap_what_a_call_reads_are_refused(fake):
    """A call's CTAs read the lengths and counts of other contexts than their own, and write without waiting for one another."""
    h, c, p = init(), cache(), pages()
    n0, a, lens, n_free = mone.mone_mem_launch_count(h), P + (1 << 16), P + 4096, P + 64
    for d in (-4, 0, 4):  # of two contexts' 8 bytes
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, a + d, None, None, a)          # lens_out on counts
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, lens + d)                      # on lens
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, None, a + d, None, a)          # granted on counts
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, None, lens + d)
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, a + d, a)                      # on lens_out
        refused(1, mone.mone_cache_release, h, p, P + 8, a, a + d)                         # lens_out on keep
        refused(1, mone.mone_cache_release, h, p, P + 8, None, lens + d)
        refused(1, mone.mone_cache4_append, h, -1, c, P, P, ST, 3, a + d, a)
        refused(1, mone.mone_cache4_append, h, -1, c, P, P, ST, 3, lens + d)
        refused(1, mone.mone_cache4_evict, h, -1, c, 50, 2, 3, tensor(P + 64, 2, 10), P + 128, P, lens + d)
    for d in (0, 4):
        refused(1, mone.mone_cache_reserve, h, p, 3, a + d, None, None, None, a)           # n_free_out in counts
        refused(1, mone.mone_cache_reserve, h, p, 3, lens + d)
        refused(1, mone.mone_cache_reserve, h, p, 3, a + d, a)
        refused(1, mone.mone_cache_reserve, h, p, 3, a + d, None, a)
        refused(1, mone.mone_cache_release, h, p, a + d, a)
        refused(1, mone.mone_cache_release, h, p, lens + d)
    for d in (-40, 0):  # two contexts' three slots of 8 bytes each
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, None, None, a + d, a)
        refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, a, None, a + d)
        refused(1, mone.mone_cache_reserve, h, p, 3, a, None, None, a + d)
    refused(1, mone.mone_cache_reserve, h, p, 3, P + 8, n_free)
    refused(1, mone.mone_cache4_append, h, -1, c, P, P, ST, 3, P + 76)                     # the last entry of the table
    assert mone.mone_mem_launch_count(h) == n0
    mone.mone_cache_reserve(h, p, 3, P + 8, a, a + 8, a + 16, a + 64, stream=0)            # side by side
    mone.mone_cache_release(h, p, P + 8, a, a + 8, stream=0)
    mone.mone_cache4_append(h, -1, c, P, P, ST, 3, a, a + 8, stream=0)
    assert mone.mone_mem_launch_count(h) == n0 + 3


def test_structs_of_another_kind_are_refused(fake):
    """They go to the library by address, which would read past the end of a smaller one."""
    dense = mone.mone_cache(P, P, strides(10 ** 5, 2048, 1024, 64), 40, 16, P, 10, P + 4096, P)
    h, r, s = init(), mone.make_rotary(64), heads()
    n0 = mone.mone_mem_launch_count(h)
    others = [dense, cache(), pages(), r, s, ctypes.byref(cache()), ctypes.addressof(cache()), (ctypes.c_char * 8)()]
    calls = {mone.mone_cache4: [lambda x: mone.mone_cache4_append(h, -1, x, P, P, ST, 3, stream=0),
                                lambda x: mone.mone_cache4_read(h, -1, x, None, 3, P, P, ST, stream=0),
                                lambda x: mone.mone_cache4_attention(h, -1, x, P, 4, 2, 1, 100, P, stream=0),
                                lambda x: mone.mone_cache4_evict(h, -1, x, 50, 2, 3, tensor(P + 64, 2, 10), P + 128, P, stream=0)],
             mone.mone_pages: [lambda x: mone.mone_cache_reserve(h, x, 3, P + 8, stream=0), lambda x: mone.mone_cache_release(h, x, P + 8, stream=0)],
             mone.mone_rotary: [lambda x: mone.mone_norm_rotate(h, -1, x, P, 3, s, None, stream=0)],
             mone.mone_heads: [lambda x: mone.mone_norm_rotate(h, -1, r, P, 3, x, None, stream=0), lambda x: mone.mone_norm_rotate(h, -1, r, P, 3, s, x, stream=0)],
             mone.mone_cache: [lambda x: mone.mone_cache_append(h, -1, x, P, P, ST, 3, stream=0),
                               lambda x: mone.mone_cache_attention(h, -1, x, P, 4, 2, 1, 100, P, stream=0)]}
    for cls, fns in calls.items():
        for x in others:
            for call in fns if not isinstance(x, cls) else ():
                with pytest.raises((ctypes.ArgumentError, AttributeError)):
                    call(x)
    assert mone.mone_mem_launch_count(h) == n0
    with pytest.raises(ctypes.ArgumentError, match="mone_cache4"):
        mone.mone_cache4_attention(h, -1, dense, P, 4, 2, 1, 100, P, stream=0)
    mine = type("mine", (mone.mone_cache4,), {})
    mone.mone_cache4_append(h, -1, mine.from_buffer_copy(cache()), P, P, ST, 3, stream=0)
    assert mone.mone_mem_launch_count(h) == n0 + 1


def test_addresses_of_any_integer_class(fake):
    class Address(int):
        pass

    at, h = Address(P), init()
    n0 = mone.mone_mem_launch_count(h)
    mone.mone_cache4_append(h, -1, cache(), at, at, ST, 3, Address(P + 65536), Address(P + 65600), stream=0)
    mone.mone_cache4_attention(h, -1, cache(), at, 4, 2, 1, 100, at, stream=0)
    mone.mone_cache_reserve(h, pages(), 3, Address(P + 8), Address(P + 65536), stream=0)
    mone.mone_norm_rotate(h, -1, mone.make_rotary(64), at, 3, heads(), None, stream=0)
    dense = mone.mone_cache(P, P, strides(10 ** 5, 2048, 1024, 64), 40, 16, P, 10, P + 4096, P)
    mone.mone_cache_attention(h, -1, dense, at, 4, 2, 1, 100, at, stream=0)
    assert mone.mone_mem_launch_count(h) == n0 + 5
