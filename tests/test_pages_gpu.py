"""The pages of the caches on the GPU: taken and given back as the definition says, entry by entry; and the serving operators
together, in a captured step whose contexts grow into new pages."""
import random

import numpy as np
import pytest
import torch

import oracle as O
import paper_2608_17616_gb300 as mone
from harness import rel_fro
from test_cache4_gpu import ALL, TOL, handle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_17616_gb300 import build
    build.build()
    mone.lib()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """Contexts of given lengths over a shuffled pool, with `spare` free pages."""

    def __init__(self, lens, page, width, spare, seed=0):
        rng = random.Random(seed)
        self.page, self.width, self.lens = page, width, list(lens)
        held = [-(-n // page) for n in lens]
        self.n_pages = sum(held) + spare + 2
        pages = rng.sample(range(self.n_pages), self.n_pages)
        self.tables = [[pages.pop() for _ in range(n)] for n in held]
        self.free = [pages.pop() for _ in range(spare)]
        self.h = handle(len(lens), 1, 2, 64)
        self.free_t = ints(self.free + [-9] * (self.n_pages - spare))
        self.n_free, self.lens_t = ints([spare]), ints(self.lens)
        self.table_t = ints([t + [-7] * (width - len(t)) for t in self.tables])

    def view(self, n_free=None, lens=None):
        return mone.make_pages(self.free_t, self.n_free if n_free is None else n_free, self.table_t, self.lens_t if lens is None else lens, self.page)

    def __del__(self):
        if getattr(self, "h", None):
            mone.mone_mem_free(self.h)


def reserve(p, n_tok, counts, slots=True, granted=True):
    B = len(p.lens)
    asked = [n_tok if counts is None else min(max(k, 0), n_tok) for k in (counts or [0] * B)]
    free, tables, want, at = O.cache_reserve(p.free, p.tables, p.lens, asked, p.page, p.width)
    g, s = (torch.full((B,), -5, dtype=torch.int32, device="cuda") if granted else None), None
    if slots:
        s = torch.full((B, n_tok), -5, dtype=torch.int64, device="cuda")
    left, lens = ints([-5]), torch.full_like(p.lens_t, -5)
    before_free = p.free_t.clone()
    mone.mone_cache_reserve(p.h, p.view(), n_tok, left, lens, g, s, None if counts is None else ints(counts))
    mone.mone_mem_sync(p.h)
    assert left.tolist() == [len(free)] and lens.tolist() == [n + k for n, k in zip(p.lens, want)]
    assert torch.equal(p.free_t, before_free)
    if granted:
        assert g.tolist() == want
    if slots:
        assert s.tolist() == [a + [-1] * (n_tok - len(a)) for a in at]
    assert p.table_t.tolist() == [t + [-7] * (p.width - len(t)) for t in tables]
    return left, lens, free, tables, want


def release(p, n_free, lens_t, lens, free, tables, keep):
    out, left = torch.full_like(lens_t, -5), ints([-5])
    free, tables = O.cache_release(free, tables, lens, [0] * len(lens) if keep is None else keep, p.page)
    held = p.table_t.clone().tolist()
    mone.mone_cache_release(p.h, p.view(n_free, lens_t), left, None if keep is None else ints(keep), out)
    mone.mone_mem_sync(p.h)
    assert left.tolist() == [len(free)] and p.free_t[:len(free)].tolist() == free
    assert out.tolist() == [min(max(0 if keep is None else keep[c], 0), n) for c, n in enumerate(lens)]
    for c, t in enumerate(tables):
        was = -(-lens[c] // p.page)
        assert p.table_t[c].tolist() == t + [-1] * (was - len(t)) + held[c][was:]
    return left, out, free, tables


CASES = [
    ([0], 16, 4, 3, 1, None),                              # a first token
    ([15, 16, 17, 0], 16, 5, 9, 1, None),                     # a page full to the last place, and one over it
    ([15, 16, 17, 0], 16, 5, 2, 1, None),                     # too few pages: the last context gets none
    ([30, 31, 32, 33], 32, 5, 1, 2, [2, 2, 1, 2]),              # the second takes the only page; the third gets nothing; the fourth needs none
    ([5, 0, 9], 8, 40, 100, 300, [300, 0, 77]),
    ([5, 0, 9], 8, 10, 100, 300, [300, 3, 20]),                # one whose table is too narrow
    ([100, 7], 1, 200, 60, 50, [-3, 90]),                     # pages of one position; counts outside 0 .. n_tok
    ([1, 2, 3], 1024, 2, 0, 5, None),                         # nothing free, nothing needed
    ([1000] * 3, 8, 200, 0, 5, None),                         # nothing free
    ([(37 * i) % 90 for i in range(300)], 16, 12, 500, 60, None),  # more contexts than a CTA's threads, too few pages for all
    ([(37 * i) % 90 for i in range(700)], 16, 12, 5000, 5, [i % 6 for i in range(700)]),
    ([0, 3], 16, 700, 1300, 9001, None),                      # tokens over several CTAs
]


@pytest.mark.parametrize("lens,page,width,spare,n_tok,counts", CASES)
def test_reserve_and_back(lens, page, width, spare, n_tok, counts):
    p = Pool(lens, page, width, spare, seed=len(lens))
    before = p.free_t.clone()
    left, lens_t, free, tables, granted = reserve(p, n_tok, counts)
    # what was taken goes back: the list and the lengths of before
    after = [n + k for n, k in zip(lens, granted)]
    left, out, free, tables = release(p, left, lens_t, after, free, tables, lens)
    assert torch.equal(p.free_t, before) and out.tolist() == lens and tables == p.tables
    # and then everything
    release(p, left, out, lens, free, tables, None)


@pytest.mark.parametrize("slots,granted", [(False, True), (True, False), (False, False)])
def test_outputs_that_are_left_out(slots, granted):
    reserve(Pool([5, 70, 0], 16, 30, 40), 300, [300, 1, 17], slots, granted)


@pytest.mark.parametrize("keep", [[0, 33, 90], [90, 1000, -4], [16, 17, 15], [1, 0, 64]])
def test_release_of_a_part(keep):
    p = Pool([64, 65, 90], 16, 9, 4)
    release(p, p.n_free, p.lens_t, p.lens, p.free, p.tables, keep)


def test_steps_at_random():
    """Contexts that grow, shrink and end, over many steps; no page is ever in two places."""
    rng = random.Random(3)
    p = Pool([0] * 9, 8, 30, 120)
    for _ in range(60):
        counts = [rng.choice([0, 1, 1, 5, 40]) for _ in p.lens]
        left, lens_t, free, tables, granted = reserve(p, 40, counts)
        lens = [n + k for n, k in zip(p.lens, granted)]
        keep = [n if rng.random() < 0.8 else rng.randint(0, n) for n in lens]
        p.n_free, p.lens_t, p.free, p.tables = release(p, left, lens_t, lens, free, tables, keep)
        p.lens = [min(n, k) for n, k in zip(lens, keep)]
        everywhere = p.free + [x for t in p.tables for x in t]
        assert len(set(everywhere)) == len(everywhere) == 120
        p.table_t.masked_fill_(p.table_t == -1, -7)


def test_what_is_out_of_range_is_latched():
    p = Pool([20, 30], 16, 6, 5)
    left, slots, g = ints([0]), torch.zeros(2, 20, dtype=torch.int64, device="cuda"), ints([0, 0])

    def fails(what, n_free=None, lens=None):
        for call in (lambda v: mone.mone_cache_reserve(p.h, v, 20, left, None, g, slots), lambda v: mone.mone_cache_release(p.h, v, left)):
            table, free = p.table_t.clone(), p.free_t.clone()
            call(p.view(n_free, lens))
            with pytest.raises(mone.MoneError) as e:
                mone.mone_mem_sync(p.h)
            assert e.value.code == 8 and what in str(e.value)
            p.table_t.copy_(table)
            p.free_t.copy_(free)

    fails("free pages", n_free=ints([-1]))
    fails("free pages", n_free=ints([p.n_pages + 1]))
    fails("length", lens=ints([-1, 3]))
    fails("length", lens=ints([3, 6 * 16 + 1]))
    p.free_t[4] = p.n_pages
    p.table_t[0, 0] = -1
    fails("page")
    mone.mone_cache_release(p.h, p.view(ints([p.n_pages])), left)  # more pages than there are
    with pytest.raises(mone.MoneError) as e:
        mone.mone_mem_sync(p.h)
    assert e.value.code == 8 and left.tolist() == [p.n_pages]


# ----------------------------------------------------------------- together, as a serving program uses them

class Step:
    """A decode step of every context: pages, rotation, append, attention; everything in device memory."""

    def __init__(self, hd, dtype, n_kv=2, group=4, page=8, B=3, L=2, steps=40):
        self.B, self.L, self.n_kv, self.group, self.hd, self.page, self.steps = B, L, n_kv, group, hd, page, steps
        g = torch.Generator(device="cuda").manual_seed(4)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        self.Q, self.K, self.V = (rn(steps, B, L, n, 1, hd) for n in (group * n_kv, n_kv, n_kv))
        self.q, self.k, self.v = (torch.zeros_like(t[0]) for t in (self.Q, self.K, self.V))
        self.qr, self.kr = torch.zeros_like(self.q), torch.zeros_like(self.k)
        self.w = [1 + 0.2 * torch.randn(L, hd, generator=g, device="cuda") for _ in range(2)]
        n_pages, width = B * 8 + 1, 8
        self.pools = [torch.full((L, n_pages, n_kv, page, w), f, dtype=torch.uint8, device="cuda")
                      for w, f in ((hd // 2, 0xb7), (hd // 2, 0xb7), (hd // 16, 127), (hd // 16, 127))]
        self.free, self.n_free, self.left = ints(list(range(n_pages))), ints([n_pages]), ints([0])
        self.table, self.lens, self.longer = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), ints([0] * B), ints([0] * B)
        self.granted, self.counts = ints([0] * B), ints([1] * B)
        self.score, self.out = torch.zeros(B, L, n_kv, width * page, device="cuda"), torch.zeros_like(self.q)
        self.h = handle(B, L, n_kv, hd, dtype)
        self.rotary = mone.make_rotary(hd)
        self.heads = mone.make_heads(self.q, self.qr, self.w[0]), mone.make_heads(self.k, self.kr, self.w[1])
        self.pages = mone.make_pages(self.free, self.n_free, self.table, self.lens, page)
        self.before, self.after = (mone.make_cache4(*self.pools, self.table, n, self.score) for n in (self.lens, self.longer))

    def __call__(self):
        h, n_q = self.h, self.group * self.n_kv
        mone.mone_cache_reserve(h, self.pages, 1, self.left, None, self.granted, None, self.counts)
        mone.mone_norm_rotate(h, -1, self.rotary, self.lens, 1, *self.heads)
        mone.mone_cache4_append(h, -1, self.before, self.kr, self.v, self.kr.stride()[:4], 1, self.longer, self.granted)
        mone.mone_cache4_attention(h, -1, self.after, self.qr, n_q, 1, 2, 30, self.out)
        self.lens.copy_(self.longer)
        self.n_free.copy_(self.left)

    def reset(self):
        for t, x in ((self.lens, 0), (self.score, 0), (self.table, -1), (self.n_free, len(self.free))):
            t.fill_(x)
        for p, x in zip(self.pools, (0xb7, 0xb7, 127, 127)):
            p.fill_(x)

    def __del__(self):
        if getattr(self, "h", None):
            mone.mone_mem_free(self.h)


@pytest.mark.parametrize("hd,dtype", [(64, torch.bfloat16), (128, torch.bfloat16), (64, torch.float32)])
def test_a_captured_step_takes_its_pages_as_it_grows(hd, dtype):
    """Replays give the bits of the calls, and with a wait after each call the same; the outputs are those of 64 bits."""
    results = []
    for how in ("calls", "graph", "waits"):
        s = Step(hd, dtype)
        s()  # the workspace, before a capture
        torch.cuda.synchronize()
        if how == "graph":
            G = torch.cuda.CUDAGraph()
            with torch.cuda.graph(G):
                s()
        s.reset()
        got = []
        for i in range(s.steps):
            s.q.copy_(s.Q[i]), s.k.copy_(s.K[i]), s.v.copy_(s.V[i])
            s.counts.copy_(ints([1, i % 2, int(i < 5)]))
            G.replay() if how == "graph" else s()
            if how == "waits":
                torch.cuda.synchronize()
            got += [s.out.clone(), s.granted.clone()]
        mone.mone_mem_sync(s.h)
        assert s.lens.tolist() == [40, 20, 5]
        results.append(got + [s.score.clone(), s.table.clone(), s.n_free.clone()])
    assert all(torch.equal(a, b) for other in results[1:] for a, b in zip(results[0], other))
    # context 0 by the definitions: every token is there
    freq, n_kv, group = [10000.0 ** (-2.0 * i / hd) for i in range(hd // 2)], s.n_kv, s.group

    def bits(x):
        return torch.from_numpy(x).to(dtype).double().numpy()

    for l in range(s.L):
        kq, vq = [], []
        for a in range(n_kv):
            k = bits(O.norm_rotate(s.K[:, 0, l, a, 0].double().cpu().numpy(), s.w[1][l].cpu().numpy(), np.arange(40), freq, True, 1e-6))
            kq.append(O.four_bit_values(*O.four_bits(k)))
            vq.append(O.four_bit_values(*O.four_bits(s.V[:, 0, l, a, 0].double().cpu().numpy())))
        # codes next to a border may fall on its other side where the rotated key's last bit differs: take what the cache holds
        held = [[torch.cat([s.pools[j][l, p, a] for p in s.table[0, :5].tolist()])[:40].cpu().numpy() for j in (0, 2)] for a in range(n_kv)]
        got = np.stack([O.four_bit_values(np.stack([c & 15, c >> 4], -1).reshape(40, hd), sc) for c, sc in held])
        assert rel_fro(got, np.stack(kq)) <= 2e-2
        for i in (0, 1, 7, 8, 25, 39):
            q = np.stack([bits(O.norm_rotate(s.Q[i, 0, l, a].double().cpu().numpy(), s.w[0][l].cpu().numpy(), [i], freq, True, 1e-6))
                          for a in range(n_kv * group)])
            ref, _ = O.window_attention(q, got, np.stack(vq), i, 2, 30)
            tol = 6e-3 if dtype is torch.bfloat16 else TOL[dtype]  # bf16: the rotated query's last bit may differ too
            assert rel_fro(results[0][2 * i][0, l].float().cpu(), ref) <= tol


def test_two_handles_on_two_streams():
    """Steps of two handles at once, each on a stream of its own, give what they give alone."""
    want = []
    for hd in (64, 128):
        s = Step(hd, torch.bfloat16, steps=20)
        for i in range(20):
            s.q.copy_(s.Q[i]), s.k.copy_(s.K[i]), s.v.copy_(s.V[i])
            s()
        mone.mone_mem_sync(s.h)
        want.append((s.out.clone(), s.score.clone(), s.table.clone()))
    both = [Step(hd, torch.bfloat16, steps=20) for hd in (64, 128)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for i in range(20):
        for s, st in zip(both, streams):
            with torch.cuda.stream(st):
                s.q.copy_(s.Q[i]), s.k.copy_(s.K[i]), s.v.copy_(s.V[i])
                s()
    torch.cuda.synchronize()
    for s, w in zip(both, want):
        mone.mone_mem_sync(s.h)
        assert all(torch.equal(a, b) for a, b in zip((s.out, s.score, s.table), w))
