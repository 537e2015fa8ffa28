"""The cache operators without a GPU: the oracle's definitions pinned by special cases, refused arguments, and the host code
of the launches."""
import ctypes
import shutil

import numpy as np
import pytest

import oracle as O
import paper_2608_17616_gb300 as mone
from fakert import Fake, build_fake

P = 1 << 30  # a made-up, aligned device address


# ----------------------------------------------------------------- the oracle

def rand(rng, *s):
    return rng.standard_normal(s)


def test_a_window_of_everything_is_the_consumer_attention():
    rng = np.random.default_rng(0)
    Q, K, V = rand(rng, 4, 6, 8), rand(rng, 2, 11, 8), rand(rng, 2, 11, 8)
    for sink, window in ((0, 100), (11, 0), (5, 6)):
        out, w = O.window_attention(Q, K, V, 5, sink, window)
        assert np.allclose(out, O.attention(Q, K, V, 5), atol=1e-14)
        assert np.isclose(w.sum(), 4 * 6)


def test_unseen_positions_have_no_effect_whatever_they_hold():
    rng = np.random.default_rng(1)
    Q, K, V = rand(rng, 2, 1, 8), rand(rng, 1, 20, 8), rand(rng, 1, 20, 8)
    base, w = O.window_attention(Q, K, V, 14, 3, 4)
    seen = [0, 1, 2, 11, 12, 13, 14]
    assert np.flatnonzero(w[0]).tolist() == seen
    K2, V2 = np.full_like(K, np.nan), np.full_like(V, np.inf)
    K2[:, seen], V2[:, seen] = K[:, seen], V[:, seen]
    assert np.array_equal(O.window_attention(Q, K2, V2, 14, 3, 4)[0], base)


def test_a_token_that_sees_nothing_is_zero_and_one_that_sees_one_key_is_its_value():
    rng = np.random.default_rng(2)
    Q, K, V = rand(rng, 1, 3, 8), rand(rng, 1, 9, 8), rand(rng, 1, 9, 8)
    assert not O.window_attention(Q, K, V, 4, 0, 0)[0].any()
    assert np.allclose(O.window_attention(Q, K, V, 4, 0, 1)[0][0], V[0, 4:7])
    assert not O.window_attention(Q, K, V, -2, 5, 5)[0][0, :2].any()


def test_weights_by_hand():
    # scores 0 and ln 3 at the two visible positions: weights 1/4 and 3/4, for both heads of the KV head
    Q, K = np.array([[[1.0]], [[1.0]]]), np.array([[[0.0], [7.0], [np.log(3.0)]]])
    out, w = O.window_attention(Q, K, np.array([[[4.0], [100.0], [8.0]]]), 2, 1, 1)
    assert np.allclose(out, 7.0) and np.allclose(w, [[0.5, 0.0, 1.5]])


def test_which_positions_stay():
    s = [5, 1, 9, 9, np.nan, 9, -np.inf, 2, 0, 7]
    assert O.cache_keep(s, 10, 2, 2).tolist() == list(range(10))
    assert O.cache_keep(s, 5, 1, 2).tolist() == [0, 2, 3, 8, 9]      # two of the three nines: the lower positions
    assert O.cache_keep(s, 9, 0, 0).tolist() == [0, 1, 2, 3, 4, 5, 7, 8, 9]  # a NaN is as low as -inf, and lower in place
    assert O.cache_keep(s, 4, 2, 2).tolist() == [0, 1, 8, 9]
    assert O.cache_keep([-0.0, 0.0, 1.0], 2, 0, 0).tolist() == [0, 2]


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


def cache(n_kv=2, hd=64, page=16, n_pages=40, width=10, score=P, **kw):
    c = mone.mone_cache(P, P, (ctypes.c_longlong * 4)(n_pages * n_kv * page * hd, n_kv * page * hd, page * hd, hd), n_pages, page, P,
                        width, P + 4096, score)
    for k, v in kw.items():
        setattr(c, k, (ctypes.c_longlong * 4)(*v) if k == "strides" else v)
    return c


def refused(code, fn, *a):
    with pytest.raises(mone.MoneError) as e:
        fn(*a, stream=0)
    assert e.value.code == code, e.value


ST = (10 ** 6, 10 ** 4, 640, 64)


def test_window_attention_refusals(fake):
    h = init()
    f = mone.mone_window_attention
    good = [h, -1, P, 4, 10, P, P, ST, 5, 2, 3, P]
    f(*good, stream=0)
    n0 = mone.mone_mem_launch_count(h)
    for i, bad in ((0, 0x1234), (1, 3), (1, -2), (2, None), (2, P + 1), (3, 3), (3, 0), (3, 130), (4, 0), (5, None), (6, None),
                   (7, (1, 1, -1, 64)), (7, (1, 1, 1, 63)), (8, -1), (8, 1 << 20), (9, -1), (10, -1), (11, None)):
        refused(1, f, *[bad if k == i else x for k, x in enumerate(good)])
    assert mone.mone_mem_launch_count(h) == n0


BAD_CACHE = [(1, dict(K=None)), (1, dict(V=P + 8)), (1, dict(table=None)), (1, dict(lens=None)), (1, dict(lens=P + 2)),
             (1, dict(n_pages=0)), (1, dict(page_size=0)), (2, dict(page_size=24)), (2, dict(page_size=2048)),
             (1, dict(table_width=0)), (1, dict(table_width=1 << 27)), (1, dict(strides=(1, 1, -64, 64))),
             (1, dict(strides=(10 ** 6, 10 ** 4, 640, 32))), (1, dict(strides=(10 ** 6, 0, 640, 64)))]


@pytest.mark.parametrize("code,kw", BAD_CACHE)
def test_a_bad_cache_is_refused_by_every_operator(fake, code, kw):
    h, c = init(), cache(**kw)
    refused(code, mone.mone_cache_append, h, -1, c, P, P, ST, 3)
    refused(code, mone.mone_cache_attention, h, -1, c, P, 4, 1, 0, 100, P)
    to = type("T", (), dict(shape=(2, 10), data_ptr=lambda self: P + 64))()
    refused(code, mone.mone_cache_evict, h, -1, c, 50, 2, 3, to, P + 128, P)
    assert not [x for x in fake.drain()[0] if "kernel" in x["name"] and "cache" in x["name"]]


def test_cache_operator_refusals(fake):
    h, c = init(), cache()
    n0 = mone.mone_mem_launch_count(h)
    append = [h, -1, c, P, P, ST, 3, P, P]
    for i, bad in ((0, 0x1234), (1, 3), (3, None), (4, P + 1), (5, (1, 1, 1, -1)), (6, 0), (6, (1 << 20) + 1), (7, P + 4096), (7, P + 1),
                   (8, P + 2)):
        refused(1, mone.mone_cache_append, *[bad if k == i else x for k, x in enumerate(append)])
    att = [h, -1, c, P, 4, 1, 0, 100, P]
    for i, bad in ((0, 0x1234), (1, 3), (3, None), (3, P + 8), (4, 3), (4, 130), (5, 0), (5, 17), (6, -1), (7, -1), (8, None)):
        refused(1, mone.mone_cache_attention, *[bad if k == i else x for k, x in enumerate(att)])

    def to(ptr, width=10):
        return type("T", (), dict(shape=(2, width), data_ptr=lambda self: ptr))()

    ev = [h, -1, c, 50, 2, 3, to(P + 64), P + 128, P, P]
    for i, bad in ((0, 0x1234), (1, 3), (2, cache(score=None)), (3, 0), (3, 4), (4, -1), (5, -1), (6, to(P)), (6, to(P + 64, 3)),
                   (6, to(P + 65)), (7, None), (7, P), (8, None), (9, P + 4096)):
        refused(1, mone.mone_cache_evict, *[bad if k == i else x for k, x in enumerate(ev)])
    assert mone.mone_mem_launch_count(h) == n0


@pytest.mark.parametrize("dtype", [mone.MONE_BF16, mone.MONE_FP32])
def test_launches_on_either_device(fake, dtype):
    for dev, sms in ((0, 152), (1, 100), (0, 152)):
        fake.device(dev)
        h, c = init(dtype=dtype), cache()
        c.table_width = 2000  # more than a cluster takes
        fake.drain()
        for layer in (-1, 2):
            mone.mone_cache_append(h, layer, c, P, P, ST, 3, stream=0)
            for score in (P, None):
                c.score = score
                mone.mone_cache_attention(h, layer, c, P, 4, 2, 1, 1 << 30, P, stream=0)
            c.score = P
            to = type("T", (), dict(shape=(2, 10), data_ptr=lambda self: P + 64))()
            mone.mone_cache_evict(h, layer, c, 50, 2, 3, to, P + 128, P, stream=0)
            launches, _ = fake.drain()
            assert {x["dev"] for x in launches} == {dev}
            assert [x["grid"][0] % sms for x in launches if "attention_kernel" in x["name"]] == [0, 0]
            assert sum("finish_kernel" in x["name"] for x in launches) == 2
        mone.mone_mem_free(h)


@pytest.mark.parametrize("width,window,ctas", [(10, 1 << 30, 1), (22, 1 << 30, 1), (23, 1 << 30, 2), (50, 1 << 30, 4), (128, 1 << 30, 8),
                                               (382, 1 << 30, 8), (383, 1 << 30, 0), (5000, 300, 1), (5000, 400, 2)])
def test_few_and_short_items_take_a_cluster_each(fake, width, window, ctas):
    """Pages of 16: blocks of 32 positions, one more for the window's start, over warps with at most three of them, or two, or six."""
    h, c = init(), cache()
    c.table_width, c.score = width, None
    fake.drain()
    mone.mone_cache_attention(h, 0, c, P, 4, 1, 0, window, P, stream=0)
    (x, *more), _ = fake.drain()
    if ctas:
        assert not more and x["grid"][0] % ctas == 0 and x["grid"][0] // ctas < 20 and max(x["cluster"], 1) == ctas
    else:
        assert len(more) == 1 and x["grid"][0] % 152 == 0


def test_launch_counts_are_the_kernels_launched(fake):
    h, c = init(), cache()
    wide = cache()
    wide.table_width = 2000
    fake.drain()
    n0 = mone.mone_mem_launch_count(h)
    to = type("T", (), dict(shape=(2, 10), data_ptr=lambda self: P + 64))()
    for call in (lambda: mone.mone_cache_append(h, 0, c, P, P, ST, 3, stream=0),
                 lambda: mone.mone_cache_attention(h, 0, c, P, 4, 2, 1, 100, P, stream=0),
                 lambda: mone.mone_cache_attention(h, 0, wide, P, 4, 2, 1, 1 << 30, P, stream=0),
                 lambda: mone.mone_cache_evict(h, 0, c, 50, 2, 3, to, P + 128, P, stream=0),
                 lambda: mone.mone_window_attention(h, 0, P, 4, 10, P, P, ST, 5, 2, 3, P, stream=0)):
        call()
        n = mone.mone_mem_launch_count(h)
        assert n - n0 == len(fake.drain()[0])
        n0 = n


def attend(h, n_tok, layer=0, score=P):
    c = cache(score=score)
    mone.mone_cache_attention(h, layer, c, P, 4, n_tok, 1, 100, P, stream=0)


def test_a_workspace_that_a_capture_has_seen_outlives_larger_calls(fake):
    h = init()
    fake.frees()
    attend(h, 1)
    assert fake.frees() == []
    attend(h, 2)  # no graph can hold the first
    first, = [f for f in fake.frees() if f != "wait"]
    fake.capturing(True)
    attend(h, 2)
    attend(h, 1)
    fake.capturing(False)
    attend(h, 8)  # a graph holds the last one: it stays
    assert fake.frees() == []
    attend(h, 8, layer=-1)  # no graph holds this one
    grown, = [f for f in fake.frees() if f != "wait"]
    assert grown > first
    fake.capturing(True)
    attend(h, 8, layer=-1)
    fake.capturing(False)
    attend(h, 16, layer=-1)
    assert fake.frees() == []
    mone.mone_mem_free(h)
    last = [f for f in fake.frees() if f != "wait"]
    assert first not in last and grown not in last
    assert sum(f > grown for f in last) == 2 and sum(first < f < grown for f in last) == 1  # the two that graphs held, and the newest


def test_a_workspace_does_not_grow_during_a_capture(fake):
    h = init()
    attend(h, 1)
    fake.frees()
    n0 = mone.mone_mem_launch_count(h)
    fake.capturing(True)
    with pytest.raises(mone.MoneError) as e:
        attend(h, 16, layer=-1)
    assert e.value.code == 3 and "capture" in str(e.value)
    assert fake.frees() == [] and mone.mone_mem_launch_count(h) == n0
    attend(h, 1)  # what fits goes on
    fake.capturing(False)
    attend(h, 16, layer=-1)
    mone.mone_mem_free(h)


def test_make_cache_takes_the_tensors_strides():
    import torch
    K, V = torch.zeros(2, 3, 16, 4, 64).transpose(2, 3), torch.zeros(2, 3, 16, 4, 64).transpose(2, 3)
    t, n = torch.zeros(5, 7, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    c = mone.make_cache(K, V, t, n)
    assert tuple(c.strides) == (3 * 16 * 256, 16 * 256, 64, 256) and (c.n_pages, c.page_size, c.table_width) == (3, 16, 7)
    assert c.score is None and c.table == t.data_ptr()
    for bad in (lambda: mone.make_cache(K, V[:, :2], t, n), lambda: mone.make_cache(K, V, t.long(), n),
                lambda: mone.make_cache(K, V, t.T, n), lambda: mone.make_cache(K.transpose(3, 4), V.transpose(3, 4), t, n)):
        with pytest.raises(ValueError):
            bad()


def tensors(L=3, n_ctx=2, n_kv=2, hd=64, page=16, width=10, dtype="bfloat16", score=True):
    import torch
    pool = [torch.zeros(L, 40, n_kv, page, hd, dtype=getattr(torch, dtype)) for _ in range(2)]
    return [*pool, torch.zeros(n_ctx, width, dtype=torch.int32), torch.zeros(n_ctx, dtype=torch.int32),
            torch.zeros(n_ctx, L, n_kv, width * page) if score else None]


def test_make_cache_refuses_tensors_that_do_not_go_together():
    import torch
    good = tensors()
    mone.make_cache(*good)
    for i, bad in ((2, torch.zeros(2, 10)), (2, torch.zeros(2, 10, dtype=torch.uint32)), (2, torch.zeros(3, 10, dtype=torch.int32)),
                   (3, torch.zeros(1, dtype=torch.int32)), (3, torch.zeros(2)), (4, torch.zeros(2, 3, 2, 159)), (4, torch.zeros(2, 3, 2, 161)),
                   (4, torch.zeros(1, 3, 2, 160)), (4, torch.zeros(2, 3, 2, 160, dtype=torch.int32)), (4, torch.zeros(2, 3, 2, 320)[..., ::2]),
                   (1, good[0].half()), (1, good[0].float())):
        with pytest.raises(ValueError):
            mone.make_cache(*[bad if k == i else x for k, x in enumerate(good)])
    with pytest.raises(ValueError):
        mone.make_cache(*[x.half() for x in good[:2]], *good[2:])


@pytest.mark.parametrize("kw", [dict(L=2), dict(n_ctx=1), dict(n_kv=1), dict(hd=32), dict(dtype="float32"), dict(L=4), dict(n_kv=4)])
def test_a_cache_of_another_handle_is_refused(fake, kw):
    """Too little of anything, and scores that lie otherwise."""
    h, keep = init(), tensors(**kw)
    n0 = mone.mone_mem_launch_count(h)
    c, to = mone.make_cache(*keep), tensors()[2]
    for call in (lambda: mone.mone_cache_append(h, -1, c, P, P, ST, 3, stream=0),
                 lambda: mone.mone_cache_attention(h, -1, c, P, 4, 1, 0, 100, P, stream=0),
                 lambda: mone.mone_cache_evict(h, -1, c, 50, 2, 3, to, P + 128, P, stream=0)):
        with pytest.raises(ValueError):
            call()
    assert mone.mone_mem_launch_count(h) == n0


def test_a_cache_with_room_for_more_than_the_handle_has_is_taken(fake):
    h, keep, exact = init(), tensors(L=4, n_ctx=3, n_kv=4, score=False), tensors()
    for t in (keep, exact):
        c = mone.make_cache(*t)
        for _ in range(2):
            mone.mone_cache_attention(h, -1, c, P, 4, 1, 0, 100, P, stream=0)
    mone.mone_mem_free(h)
    refused(1, mone.mone_cache_attention, h, -1, c, P, 4, 1, 0, 100, P)
    h = init(n_ctx=3)  # perhaps at the same address
    with pytest.raises(ValueError):
        mone.mone_cache_attention(h, -1, c, P, 4, 1, 0, 100, P, stream=0)


def test_evict_refuses_targets_that_are_too_small_or_lie_otherwise(fake):
    import torch
    h, keep = init(), tensors()
    c = mone.make_cache(*keep)
    good = [torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 3, 2, 64), torch.zeros(2, 3, 2, 50, dtype=torch.int32)]
    mone.mone_cache_evict(h, -1, c, 50, 2, 3, *good, stream=0)
    mone.mone_cache_evict(h, 1, c, 50, 2, 3, *good[:2], good[2][:, 0].contiguous(), stream=0)
    n0 = mone.mone_mem_launch_count(h)
    for i, bad in ((0, torch.zeros(2, 8, dtype=torch.int32)[:, :4]), (0, good[0].long()), (0, good[0][:1]), (1, torch.zeros(2, 3, 2, 63)),
                   (1, torch.zeros(2, 3, 2, 160)), (1, good[1].double()), (1, good[1][:1]), (2, torch.zeros(2, 3, 2, 49, dtype=torch.int32)),
                   (2, good[2].long()), (2, good[2].transpose(1, 2))):
        with pytest.raises(ValueError):
            mone.mone_cache_evict(h, -1, c, 50, 2, 3, *[bad if k == i else x for k, x in enumerate(good)], stream=0)
    assert mone.mone_mem_launch_count(h) == n0
