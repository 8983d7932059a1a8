"""Page tables and slot maps, the paged 16-bit cache and the attention of prompts on the GPU, against their definitions.

Pages, slots, positions, states and what an append leaves are exact.  A score whose products' magnitudes sum to S = scale * sum |q k| + |bias| is off by at
most (d + 8) roundings of binary32 relative to S (d products into a binary32 accumulator, then factor, cap, bias, reference); a softmax weight by twice
that, and by its numerator's rounding to the 16-bit type, half a step E of it (fp16 2^-11, or half of its smallest step where the largest numerator is
2^11: 2^-36 of that; bf16 2^-8).  n weights are summed in binary32: n 2^-24 of the sum of magnitudes at most.  The output's own rounding is E again.
The log-sum-exp takes no rounded numerators: the scores' error, n 2^-24, and 2^-22 of itself for the exponentials and the logarithm.
"""
import math
import random

import numpy as np
import pytest

import kv16_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2510_05176_amd import patternkv
    return patternkv


EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float16, torch.bfloat16]


def code(pk, dtype):
    return pk.DTYPE_BF16 if dtype == torch.bfloat16 else pk.DTYPE_FP16


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- pages -------------------------------------------------------------------------------------------------------------------

class Paged:
    """A pool on the GPU and the same one as lists."""

    def __init__(self, pk, n_seq, page, n_pages, per_seq, seed=0):
        rng = random.Random(seed)
        order = rng.sample(range(n_pages), n_pages)
        self.pk, self.cfg, self.ref = pk, pk.PagesConfig(n_seq=n_seq, page_tokens=page, n_pages=n_pages, pages_per_seq=per_seq), ref.Pool(n_seq, page, n_pages, per_seq, order)
        # what is not written stays: entries that nobody needs hold something else
        self.table = torch.full((n_seq, per_seq), -7, dtype=torch.int32, device="cuda")
        self.pool = pk.PagePool(self.cfg, table=self.table, free=ints(order), n_free=ints([n_pages, 0, 0, 0]))
        self.states = torch.zeros((n_seq, 4), dtype=torch.int32, device="cuda")

    def update(self, counts, n_tokens, states=None, **kw):
        plan = self.pk.pk_pages_update(self.cfg, self.pool, self.states if states is None else states, ints(counts), n_tokens, **kw)
        return plan, self.ref.update(counts, n_tokens)

    def check(self, plan, want, states=None, n_free=None):
        starts, slots, positions, taken = want
        assert plan.starts.tolist() == starts and plan.taken.tolist() == taken
        assert plan.slots.tolist() == slots
        if plan.positions is not None:
            assert plan.positions.tolist() == positions
        states, n_free = self.states if states is None else states, self.pool.n_free if n_free is None else n_free
        assert states.tolist() == [[n, p, 0, 0] for n, p in zip(self.ref.length, self.ref.next)]
        assert n_free.tolist() == [len(self.ref.free), 0, 0, 0] and self.pool.free.tolist()[:len(self.ref.free)] == self.ref.free
        table = self.table.tolist()
        assert [row[:len(p)] for row, p in zip(table, self.ref.pages)] == self.ref.pages


@pytest.mark.parametrize("n_seq,page,n_pages,per_seq,most", [
    (1, 1, 1, 1, 3), (1, 16, 40, 40, 300), (3, 4, 9, 5, 14), (64, 16, 500, 12, 70), (65, 2, 300, 9, 9), (200, 16, 4000, 40, 3), (1000, 8, 2500, 6, 20),
    (1024, 32, 1030, 3, 40), (1025, 16, 5000, 7, 40), (2500, 1, 6000, 5, 4), (5, 256, 400, 100, 9000)])
def test_steps_of_a_pool(pk, n_seq, page, n_pages, per_seq, most):
    """Steps in a row, in place: growing, giving back, empty pools, full rows, packed tensors that are too short or longer than needed."""
    rng = random.Random(n_seq * 31 + page)
    p = Paged(pk, n_seq, page, n_pages, per_seq, seed=n_seq)
    for step in range(7):
        kind = rng.random()
        counts = [rng.choice([0, 1, 1, rng.randint(0, most), -rng.randint(1, most), -(1 << 31) if rng.random() < 0.1 else 1]) if kind < 0.7 else
                  rng.randint(0, most) if kind < 0.9 else -rng.randint(0, most) for _ in range(n_seq)]
        n_tokens = max(sum(max(c, 0) for c in counts) + rng.choice([0, 0, 5, 300, -1, -most]), 0)
        before = p.table.clone()
        plan, want = p.update(counts, n_tokens)
        p.check(plan, want)
        # entries of logical pages that no sequence has now and that were not written before are as they were
        live = torch.arange(per_seq)[None] < torch.tensor([len(x) for x in p.ref.pages])[:, None]
        assert torch.equal(p.table.cpu()[~live], before.cpu()[~live])
    everything, want = p.update([-(1 << 31)] * n_seq, 0)
    p.check(everything, want)
    assert p.pool.n_free[0] == n_pages and sorted(p.pool.free.tolist()) == list(range(n_pages))


def test_a_step_can_be_taken_back(pk):
    """States and the number of free pages of their own: the old ones and all that belongs to them stay valid, and the step repeats."""
    p = Paged(pk, 6, 16, 60, 20)
    plan, want = p.update([100, 3, 0, 200, 16, 40], 400)
    p.check(plan, want)
    old = [p.states.clone(), p.pool.n_free.clone(), p.table.clone(), p.pool.free.clone()]
    import copy
    saved = copy.deepcopy(p.ref)
    for counts in ([5, -3, 70, -200, 1, 100], [300, 300, 300, 300, 300, 300], [-1, -1, 0, 0, 0, 9]):
        for _ in range(2):
            after, n_free = torch.full_like(p.states, 9), torch.full_like(p.pool.n_free, 9)
            p.ref = copy.deepcopy(saved)
            plan, want = p.update(counts, 512, states_out=after, n_free_out=n_free)
            p.check(plan, want, after, n_free)
            assert torch.equal(p.states, old[0]) and torch.equal(p.pool.n_free, old[1])
            free = int(old[1][0])
            assert torch.equal(p.pool.free[:free], old[3][:free])
            for row, was, pages in zip(p.table.tolist(), old[2].tolist(), saved.pages):
                assert row[:len(pages)] == was[:len(pages)]


def test_pages_take_whatever_is_there(pk):
    """Numbers out of range in the states, the table and the stack: every entry and slot that comes out lies in the pool."""
    n_seq, page, n_pages, per_seq = 40, 16, 50, 8
    cfg = pk.PagesConfig(n_seq=n_seq, page_tokens=page, n_pages=n_pages, pages_per_seq=per_seq)
    g = torch.Generator().manual_seed(3)
    wild = lambda *shape: torch.randint(-(1 << 31), (1 << 31) - 1, shape, generator=g).int().cuda()   # noqa: E731
    for n_free in (-5, 0, 20, 1 << 30):
        pool = pk.PagePool(cfg, table=wild(n_seq, per_seq), free=wild(n_pages), n_free=ints([n_free, 0, 0, 0]))
        states = wild(n_seq, 4)
        plan = pk.pk_pages_update(cfg, pool, states, ints([random.Random(i).randint(-300, 300) for i in range(n_seq)]), 1000)
        assert (plan.slots >= -1).all() and (plan.slots < n_pages * page).all()
        assert (plan.starts.diff() >= 0).all() and plan.starts[0] == 0 and plan.starts[-1] <= 1000
        assert (states[:, 0] >= 0).all() and (states[:, 0] <= per_seq * page).all() and 0 <= int(pool.n_free[0]) <= n_pages
        assert (plan.taken >= 0).all() and (plan.taken <= per_seq * page).all()


@pytest.mark.parametrize("n_seq,n_tokens", [(6, 400), (6, 5000), (1100, 3000)])
def test_steps_without_positions(pk, n_seq, n_tokens):
    """A plan of the caller's that has none, in one launch and in two."""
    p = Paged(pk, n_seq, 16, 60 + n_seq, 20)
    out = pk.pk_pages_plan(p.cfg, n_tokens)
    out.positions = None
    for counts in ([100, 3, 0, 200, 16, 40], [5, -3, 70, -200, 1, 100]):
        plan, want = p.update(counts + [1] * (n_seq - 6), n_tokens, out=out)
        p.check(plan, want)


# ---- append ------------------------------------------------------------------------------------------------------------------

def packed(n, heads, d, dtype, seed, parts=1, extra=8):
    """[n][heads][d] views of wider tensors with every bit pattern"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randint(-32768, 32768, (n, heads * parts + 1, d + extra), generator=g, device="cuda", dtype=torch.int16).view(dtype)
    return [wide[:, i * heads:(i + 1) * heads, :d] for i in range(parts)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,hkv,page,n", [(64, 1, 16, 1), (96, 3, 32, 77), (128, 8, 16, 200), (256, 2, 128, 1), (128, 1, 64, 5000), (96, 8, 256, 1031), (256, 5, 16, 333), (64, 17, 16, 40)])
def test_append(pk, dtype, d, hkv, page, n):
    n_pages = -(-n // page) * 2 + 3
    cfg = pk.Kv16Config(n_seq=1, n_kv_heads=hkv, n_q_heads=hkv, head_dim=d, t_capacity=page, dtype=code(pk, dtype), page_tokens=page, n_pages=n_pages)
    cache = pk.Kv16Cache(cfg)
    for t in (cache.k, cache.v):
        t.view(torch.int16).copy_(torch.randint(-32768, 32768, t.shape, device="cuda", dtype=torch.int16))
    want = {name: getattr(cache, name).clone() for name in "kv"}
    rng = random.Random(n)
    slots = rng.sample(range(n_pages * page), n)
    for i in range(0, n, 7):   # no place, and places that are not the pool's
        slots[i] = rng.choice([-1, -(1 << 31), n_pages * page, (1 << 31) - 1])
    k, v = packed(n, hkv, d, dtype, n, parts=2)
    pk.pk_kv16_append(cfg, cache, k, v, ints(slots))
    at = [i for i, s in enumerate(slots) if 0 <= s < n_pages * page]
    to = torch.tensor([slots[i] for i in at], dtype=torch.long, device="cuda")
    for name, new in (("k", k), ("v", v)):
        w = want[name].view(torch.int16)
        w[to // page, :, to % page] = new.contiguous().view(torch.int16)[at]
        assert torch.equal(getattr(cache, name).view(torch.int16), w)


def test_append_strides(pk):
    """Heads before tokens, a vector for all tokens or heads (stride 0), strides that run backwards' worth of room apart."""
    cfg = pk.Kv16Config(n_seq=1, n_kv_heads=4, n_q_heads=4, t_capacity=64, page_tokens=16, n_pages=8)
    cache = pk.Kv16Cache(cfg)
    slots = ints([5, 100, 17, 0, 127])
    x = torch.randn(4, 5, 128, device="cuda").half()
    for k, v in ((x.transpose(0, 1), x[:, :1].transpose(0, 1).expand(5, 4, 128)), (x[:1].transpose(0, 1).expand(5, 4, 128), x.transpose(0, 1))):
        pk.pk_kv16_append(cfg, cache, k, v, slots)
        at = slots.long()
        assert torch.equal(cache.k[at // 16, :, at % 16], k) and torch.equal(cache.v[at // 16, :, at % 16], v)
    pk.pk_kv16_append(cfg, cache, k[:0], v[:0], slots[:0])


# ---- attention ---------------------------------------------------------------------------------------------------------------

def check(got, got_lse, want, want_lse, mag, size, weak, n, d, dtype, vmax):
    """got [heads][rows][d] against the definition; n: keys of a row at most"""
    E = EPS[dtype]
    off = (d + 8) * 2.0 ** -24 * size
    tol = E * np.abs(want) + (E + 2 * off + n * 2.0 ** -24)[..., None] * mag + n * 2.0 ** -36 * 2 * vmax + 2.0 ** -25
    # An infinite value gives NaN where its numerator rounds to 0.  fp16: below half of its smallest step, 2^-25, where the largest is 2^11, 2^-36 of that.
    # bf16: below binary32's smallest normal number, 2^-126, where the largest is 2^-29 at the least (2^-25 where the reference's room is used up), 2^-97 of that.
    lost = np.isinf(want) & (weak < 2.0 ** (-35.9 if dtype == torch.float16 else -96.9))[..., None] & np.isnan(got)
    want = np.where(lost, np.nan, want)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), np.argwhere(np.isnan(got) != np.isnan(want))[:4]
    assert np.array_equal(got[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)])
    with np.errstate(invalid="ignore"):
        bad = ~odd & ~(np.abs(got - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:4], (np.abs(got - want) / tol)[bad][:4])
        empty = want_lse == -np.inf
        assert np.array_equal(got_lse == -np.inf, empty) and (got[empty] == 0).all()
        assert np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
        ok = np.isfinite(want_lse)
        far = np.abs(got_lse - want_lse)
        assert (far[ok] <= (off + n * 2.0 ** -24 + 2.0 ** -22 * (np.abs(want_lse) + 2))[ok]).all(), far[ok].max()


def vectors(rng, n, heads, d, dtype, spread=1.0, keys=False):
    """[n][heads][d], a view of a wider tensor; and in 64 bits"""
    x = rng.standard_normal((n, heads, d))
    if keys:
        x = x * 1.3 + rng.standard_normal((1, heads, d))
    else:
        x *= np.exp(spread * rng.standard_normal((n, 1, 1)))
    wide = torch.zeros((n, heads + 1, d + 8), dtype=dtype, device="cuda")
    t = wide[:, :heads, :d]
    t.copy_(torch.from_numpy(x).to(dtype))
    return t, t.double().cpu().numpy()


class Step:
    """Sequences of a 16-bit cache with tables in any order, and their vectors in 64 bits."""

    def __init__(self, pk, lens, seed=0, hkv=2, r=4, d=128, page=16, dtype=torch.float16, cap=None, k=None, v=None, fill=math.nan):
        self.pk, self.lens, self.rng, self.dtype = pk, lens, np.random.default_rng(seed), dtype
        cap = cap or max(-(-max(lens) // page), 1) * page + page
        n_seq, per_seq = len(lens), cap // page
        n_pages = n_seq * per_seq + 3 if n_seq * per_seq < 3000 else sum(-(-n // page) for n in lens) + 3
        self.cfg = pk.Kv16Config(n_seq=n_seq, n_kv_heads=hkv, n_q_heads=hkv * r, head_dim=d, t_capacity=cap, dtype=code(pk, dtype), page_tokens=page, n_pages=n_pages)
        # pages of nobody and entries that are not needed hold anything
        table = self.rng.integers(-(1 << 31), 1 << 31, (n_seq, per_seq)).astype(np.int32)
        order = list(self.rng.permutation(n_pages))
        for i, n in enumerate(lens):
            for l in range(-(-n // page)):
                table[i, l] = order.pop()
        self.cache = pk.Kv16Cache(self.cfg, page_table=torch.from_numpy(table).cuda())
        self.cache.k.fill_(fill), self.cache.v.fill_(fill)
        self.k, self.v = [], []
        for i, n in enumerate(lens):
            kt, kn = vectors(self.rng, n, hkv, d, dtype, keys=True) if k is None else k(i, n)
            vt, vn = vectors(self.rng, n, hkv, d, dtype) if v is None else v(i, n)
            t = np.arange(n)
            slots = torch.from_numpy((table[i, t // page].astype(np.int64) * page + t % page).astype(np.int32)).cuda()
            pk.pk_kv16_append(self.cfg, self.cache, kt, vt, slots)
            self.k.append(kn), self.v.append(vn)
            self.cache.states[i, 0] = n
            self.cache.states[i, 1] = 12345   # not looked at

    def attend(self, scale=None, cap=0.0, window=0, slopes=False, q=None, checked=True, **kw):
        cfg, d = self.cfg, self.cfg.head_dim
        scale = d ** -0.5 if scale is None else scale
        qt, qn = q or vectors(self.rng, cfg.n_seq, cfg.n_q_heads, d, self.dtype)
        sl = torch.exp2(-torch.arange(1, cfg.n_q_heads + 1, device="cuda") / cfg.n_q_heads * 6).float() if slopes else None
        out = torch.full((cfg.n_seq, cfg.n_q_heads + 1, d), 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full((cfg.n_seq, cfg.n_q_heads), 7.0, device="cuda")
        got = self.pk.pk_kv16_attention(cfg, self.cache, qt, scale, cap=cap, window=window, slopes=sl, out=out[:, :-1], lse=lse, **kw)
        assert got.data_ptr() == out.data_ptr() and (out[:, -1] == 7.0).all()
        got, got_lse = out[:, :-1].double().cpu().numpy(), lse.double().cpu().numpy()
        if not checked:
            return got, got_lse
        r = cfg.n_q_heads // cfg.n_kv_heads
        for i, n in enumerate(self.lens):
            for h in range(cfg.n_kv_heads):
                hs = slice(h * r, (h + 1) * r)
                slope = None if sl is None else sl.double().cpu().numpy()[hs]
                want, want_lse, mag, size, weak = ref.attention(qn[i, hs, None], self.k[i][:, h], self.v[i][:, h], np.array([n - 1]), scale, cap, window, slope)
                vmax = np.abs(np.nan_to_num(self.v[i], posinf=0.0, neginf=0.0)).max(initial=0.0)
                check(got[i, hs, None], got_lse[i, hs, None], want, want_lse, mag, size, weak, n, d, self.dtype, vmax)
        return got, got_lse


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("hkv,r,page", [(1, 1, 16), (2, 4, 32), (3, 17, 16), (1, 64, 128), (2, 33, 64), (1, 24, 16), (8, 1, 256)])
def test_attention_of_one_token(pk, dtype, d, hkv, r, page):
    """Lengths around tiles, waves and pages; what lies behind them in the pages is NaN."""
    s = Step(pk, [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300, 511], seed=d + r, hkv=hkv, r=r, d=d, page=page, dtype=dtype)
    s.attend()
    s.attend(scale=-0.3)
    s.attend(bound=511)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,r", [(64, 2), (96, 5), (128, 4), (128, 20), (256, 3)])
@pytest.mark.parametrize("how", [dict(cap=5.0), dict(cap=300.0), dict(window=1), dict(window=37), dict(window=200), dict(slopes=True), dict(slopes=True, window=70, cap=20.0),
                                 dict(window=100000), dict(scale=0.0), dict(scale=0.0, cap=1.0)])
def test_attention_with_options(pk, dtype, d, r, how):
    Step(pk, [0, 1, 36, 37, 38, 64, 101, 700, 1300], seed=r, r=r, d=d, dtype=dtype).attend(**how)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,lens", [(128, [40000]), (64, [9000, 3]), (256, [5000]), (96, [20000, 1, 8000]), (128, [2500] * 7)])
def test_attention_over_long_caches(pk, dtype, d, lens):
    """Split over workgroups, and the pieces joined; more of them than a wave has lanes."""
    s = Step(pk, lens, seed=1, hkv=1 if max(lens) > 9000 else 2, r=8, d=d, dtype=dtype, page=64)
    s.attend()
    s.attend(window=max(lens) // 2 + 5)
    s.attend(slopes=True, cap=30.0)
    a, al = s.attend(checked=False, q=(torch.ones(len(lens), s.cfg.n_q_heads, d, dtype=dtype, device="cuda"), None))
    b, bl = s.attend(checked=False, bound=0, q=(torch.ones(len(lens), s.cfg.n_q_heads, d, dtype=dtype, device="cuda"), None))   # the bound only sizes the launch
    assert np.abs(a - b).max() <= 4 * EPS[dtype] * np.abs(a).max() and np.abs(al - bl).max() <= 1e-4


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hkv,r", [(1, 17), (2, 24), (1, 33), (2, 64)])
def test_attention_of_many_heads_of_256_channels(pk, dtype, hkv, r):
    """More than 16 heads per KV head with a large bound, which takes them in pairs of row tiles, and a small one."""
    s = Step(pk, [0, 1, 33, 300, 2100], seed=r, hkv=hkv, r=r, d=256, page=64, dtype=dtype, cap=1 << 17)
    s.attend()
    s.attend(slopes=True, cap=20.0, window=290)
    s.attend(scale=-0.05, bound=1 << 16)
    s.attend(bound=2100)


def test_attention_of_many_sequences(pk):
    """More sequences than the keys are dealt out over, and one for each; unequal lengths."""
    rng = random.Random(2)
    for n_seq, most in ((256, 700), (300, 200), (700, 40)):
        lens = [rng.choice([0, 1, 2, rng.randint(1, most)]) for _ in range(n_seq)]
        Step(pk, lens, hkv=1, r=2, d=64, page=16).attend()


@pytest.mark.parametrize("hkv,n_seq,n", [(1, 257, 6000), (16, 130, 2500), (32, 64, 2100), (8, 256, 1500)])
def test_a_long_sequence_among_many(pk, hkv, n_seq, n):
    """More (sequence, KV head) pairs than the keys are dealt out over: one workgroup each, whatever its length."""
    rng = random.Random(hkv)
    lens = [rng.choice([0, 1, rng.randint(1, 60)]) for _ in range(n_seq)]
    lens[n_seq // 3] = n
    s = Step(pk, lens, hkv=hkv, r=1, d=64, page=32)
    s.attend()
    s.attend(window=n - 77, slopes=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_large_and_small_scores(pk, dtype):
    """Scores of 2^20 and more (rounded ones; results stay finite and are some token's value), of no size at all, and values near the type's largest."""
    d, n = 128, 500
    for size in (2.0 ** 14, 2.0 ** 22, 2.0 ** 29):
        s = Step(pk, [n, 3], d=d, dtype=dtype)
        q = torch.randn(2, 8, d, device="cuda").to(dtype)
        got, lse = s.attend(scale=size, q=(q, None), checked=False)
        top = max(np.abs(v).max() for v in s.v)
        # numerators off by E of themselves each, so that weights add up to 1 + E at most, and the result's rounding
        assert np.isfinite(got).all() and np.isfinite(lse).all() and np.abs(got).max() <= top * (1 + EPS[dtype]) ** 2 * (1 + n * 2.0 ** -24)
    big = torch.finfo(dtype).max
    v = lambda i, n: (torch.full((n, 2, d), big, dtype=dtype, device="cuda"), np.full((n, 2, d), float(big)))   # noqa: E731
    got, _ = Step(pk, [5000, 70], d=d, dtype=dtype, v=v).attend(checked=False)
    # weights off by E each and a sum rounded n times: no further than 2 E from 1 in all, and the type's largest is not passed
    assert (got >= big * (1 - 2 * EPS[dtype])).all() and (got <= big).all()


def test_attention_where_many_tokens_have_little_weight(pk):
    """One token with a score of 0 and 30000 with 2^-20 of its weight each, two hundredths of the result: they are not lost in fp16 numerators."""
    d, n = 64, 30001
    x = np.zeros((n, 1, d))
    x[1:, 0, 0] = -20 * math.log(2.0)
    k = lambda i, n: (torch.from_numpy(x).half().cuda(), x.astype(np.float16).astype(np.float64))   # noqa: E731
    vn = np.ones((n, 1, d))
    vn[0] = 0.0
    v = lambda i, n: (torch.from_numpy(vn).half().cuda(), vn)   # noqa: E731
    q = np.zeros((1, 2, d))
    q[..., 0] = 1.0
    s = Step(pk, [n], hkv=1, r=2, d=d, k=k, v=v)
    s.attend(scale=1.0, q=(torch.from_numpy(q).half().cuda(), q))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 256])
def test_attention_of_values_that_are_not_finite(pk, dtype, d):
    """NaN and infinities in tokens that the window masks do not reach the result; in tokens that are seen they do."""
    hkv, n = 2, 200

    def odd(at, what):
        def make(i, n):
            t, x = vectors(np.random.default_rng(i), n, hkv, d, dtype)
            for a in at:
                if a < n:
                    t[a, 0, 3] = what
            return t, t.double().cpu().numpy()
        return make
    for what in (math.nan, math.inf, -math.inf):
        for at in ([0, 60, 130], [149], [150], [199, 170]):
            Step(pk, [n, n - 1], hkv=hkv, d=d, dtype=dtype, v=odd(at, what), fill=math.inf).attend(window=50)
        Step(pk, [n], hkv=hkv, d=d, dtype=dtype, k=odd([0, 149], what)).attend(window=50)
    Step(pk, [n], hkv=hkv, d=d, dtype=dtype, k=odd([170], math.nan)).attend(window=50)


def test_attention_layouts(pk):
    """Queries of heads before sequences, one query for all; results laid out like dense queries; one head; a workspace of the caller's."""
    s = Step(pk, [70, 1500, 3], hkv=2, r=2, d=96)
    cfg = s.cfg
    q = torch.randn(cfg.n_q_heads, cfg.n_seq, 96, device="cuda").half()
    want = s.pk.pk_kv16_attention(cfg, s.cache, q.transpose(0, 1).contiguous(), 0.1)
    got = s.pk.pk_kv16_attention(cfg, s.cache, q.transpose(0, 1), 0.1)
    assert torch.equal(got, want) and got.stride() == q.transpose(0, 1).stride()
    one = s.pk.pk_kv16_attention(cfg, s.cache, q[:1, :1].expand(3, 4, 96), 0.1)
    assert torch.equal(one, s.pk.pk_kv16_attention(cfg, s.cache, q[:1, :1].expand(3, 4, 96).contiguous(), 0.1))
    ws = torch.empty(s.pk.pk_kv16_workspace_bytes(cfg, 1500) + 64, dtype=torch.uint8, device="cuda")
    assert torch.equal(s.pk.pk_kv16_attention(cfg, s.cache, q.transpose(0, 1), 0.1, bound=1500, workspace=ws), s.pk.pk_kv16_attention(cfg, s.cache, q.transpose(0, 1), 0.1, bound=1500))
    with pytest.raises(s.pk.PkError):
        s.pk.pk_kv16_attention(cfg, s.cache, q.transpose(0, 1), 0.1, bound=1500, workspace=ws[:100])


def test_a_workspace_for_the_capacity_serves_smaller_bounds(pk):
    """Also where calls with a smaller bound take another form of the kernel, whose runs are more."""
    s = Step(pk, [random.Random(i).randint(0, 300) for i in range(86)], hkv=1, r=33, d=256, page=64, cap=4096)
    ws = torch.empty(pk.pk_kv16_workspace_bytes(s.cfg, 4096), dtype=torch.uint8, device="cuda")
    for bound in (4096, 3049, 3048, 2000, 300):
        s.attend(bound=bound, workspace=ws)


# ---- prompts -----------------------------------------------------------------------------------------------------------------

def run_prompts(pk, lens, hkv=2, r=4, d=128, dtype=torch.float16, scale=None, cap=0.0, window=0, slopes=False, seed=0, before=0, behind=0, spoil=None, q=None):
    """A packed call against the definition; before, behind: rows of no sequence."""
    rng = np.random.default_rng(seed)
    scale = d ** -0.5 if scale is None else scale
    hq, n = hkv * r, sum(lens) + before + behind
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32) + before
    wide = torch.zeros((n, hq + 2 * hkv + 1, d + 8), dtype=dtype, device="cuda")   # q, k and v of a token next to each other
    x = np.concatenate([vectors(rng, n, hq, d, dtype)[1], vectors(rng, n, hkv, d, dtype, keys=True)[1], vectors(rng, n, hkv, d, dtype)[1]], 1)
    wide[:, :-1, :d] = torch.from_numpy(x).to(dtype)
    qt, kt, vt = wide[:, :hq, :d], wide[:, hq:hq + hkv, :d], wide[:, hq + hkv:-1, :d]
    # rows of no sequence hold anything
    for t in (kt, vt):
        t[:before] = math.nan
        t[n - behind:] = math.nan
    if spoil:
        spoil(kt, vt, starts)
    cfg = pk.PromptConfig(n_seq=len(lens), n_kv_heads=hkv, n_q_heads=hq, head_dim=d, dtype=code(pk, dtype))
    sl = torch.exp2(-torch.arange(1, hq + 1, device="cuda") / hq * 6).float() if slopes else None
    out = torch.full((n, hq + 1, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((hq, n), 7.0, device="cuda")
    pk.pk_prompt_attention(cfg, qt, kt, vt, torch.from_numpy(starts).cuda(), scale, cap=cap, window=window, slopes=sl, out=out[:, :-1], lse=lse)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (got[:, -1] == 7.0).all()
    for a in (slice(0, before), slice(n - behind, n)):
        assert (got[a] == 7.0).all() and (got_lse[:, a] == 7.0).all()
    qn, kn, vn = (t.double().cpu().numpy() for t in (qt, kt, vt))
    for i, length in enumerate(lens):
        at = slice(starts[i], starts[i] + length)
        for h in range(hkv):
            hs = slice(h * r, (h + 1) * r)
            want, want_lse, mag, size, weak = ref.attention(qn[at, hs].transpose(1, 0, 2), kn[at, h], vn[at, h], np.arange(length), scale, cap, window,
                                                      None if sl is None else sl.double().cpu().numpy()[hs])
            vmax = np.abs(np.nan_to_num(vn[at], posinf=0.0, neginf=0.0)).max(initial=0.0)
            check(got[at, hs].transpose(1, 0, 2), got_lse[hs, at], want, want_lse, mag, size, weak, length, d, dtype, vmax)
    return got[:, :-1], got_lse


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("lens,hkv,r", [([1], 1, 1), ([61], 2, 4), ([63, 64, 65, 0, 1, 2, 0, 300], 2, 4), ([257, 130], 1, 1), ([33, 5], 1, 64), ([129, 1], 1, 33), ([200, 90], 3, 7),
                                        ([0, 0], 1, 2), ([700], 2, 2)])
def test_prompts(pk, dtype, d, lens, hkv, r):
    run_prompts(pk, lens, hkv=hkv, r=r, d=d, dtype=dtype, before=3 * (len(lens) % 2), behind=len(lens), seed=d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,r", [(64, 7), (96, 2), (128, 4), (256, 3)])
@pytest.mark.parametrize("how", [dict(cap=5.0), dict(cap=300.0), dict(window=1), dict(window=37), dict(window=64), dict(window=130), dict(slopes=True),
                                 dict(slopes=True, window=70, cap=20.0), dict(window=100000), dict(scale=-0.2), dict(scale=0.0), dict(scale=0.0, cap=1.0)])
def test_prompts_with_options(pk, dtype, d, r, how):
    run_prompts(pk, [1, 300, 64, 37], r=r, d=d, dtype=dtype, hkv=1, **how)


@pytest.mark.parametrize("n_seq,most", [(64, 40), (65, 40), (200, 9), (700, 5), (90, 170)])
def test_many_prompts(pk, n_seq, most):
    rng = random.Random(n_seq)
    lens = [rng.choice([0, 1, rng.randint(1, most), rng.randint(1, most)]) for _ in range(n_seq)]
    lens[rng.randrange(n_seq)] = 310
    run_prompts(pk, lens, hkv=1, r=3, d=64, behind=2, dtype=torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("how", [dict(), dict(window=50), dict(scale=-0.1)])
def test_prompts_of_many_rows(pk, dtype, d, how):
    """Rows enough (160000) for workgroups of two groups of waves where the rule takes them; sequences around their 16 tokens and around tiles of 64 keys, one that ends
    inside of both, and values that are not finite."""
    lens = [1, 15, 16, 17, 0, 63, 64, 65, 127, 129, 640] + [61] * 23

    def spoil(kt, vt, starts):
        for i, t in ((9, 100), (10, 0), (10, 333), (10, 639), (11, 60)):
            vt[starts[i] + t, t % 4, 7] = (math.nan, math.inf, -math.inf)[t % 3]
    run_prompts(pk, lens, hkv=4, r=16, d=d, dtype=dtype, behind=5, spoil=spoil, **how)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [96, 128])
@pytest.mark.parametrize("n_seq,most,r", [(300, 25, 4), (70, 120, 4), (2100, 3, 8)])
def test_many_short_prompts_of_many_rows(pk, dtype, d, n_seq, most, r):
    """Rows enough in all for workgroups of two groups of waves, few of them in a sequence: most of a workgroup's waves have none."""
    rng = random.Random(n_seq)
    lens = [rng.choice([0, 1, rng.randint(1, most), most]) for _ in range(n_seq)]
    hkv = -(-512 * 256 // (sum(lens) * r))
    run_prompts(pk, lens, hkv=hkv, r=r, d=d, dtype=dtype, behind=3)


def test_a_long_prompt(pk):
    for dtype, d, kw in ((torch.float16, 64, {}), (torch.bfloat16, 128, {}), (torch.bfloat16, 64, dict(window=500, slopes=True))):
        run_prompts(pk, [2500, 40], hkv=1, r=2, d=d, dtype=dtype, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_prompts_with_values_that_are_not_finite(pk, dtype, d, what):
    """What is not finite in K or V of a token reaches the rows that see it and no others: earlier ones, those whose window has passed it, other sequences."""
    def spoil(kt, vt, starts):
        for i, t in ((0, 0), (0, 100), (0, 101), (1, 70), (2, 39)):
            vt[starts[i] + t, 0, 5 + t % 7] = what
        vt[starts[0] + 130, 0, d - 1] = -what
    for window in (0, 20):
        run_prompts(pk, [150, 90, 40, 64], hkv=2, r=3, d=d, dtype=dtype, window=window, spoil=spoil)

    def spoil_keys(kt, vt, starts):
        kt[starts[0] + 77, 1, 3] = math.nan
        kt[starts[1] + 89, 0, 3] = math.nan
        vt[starts[1] + 5, 1] = what
    run_prompts(pk, [150, 90], hkv=2, r=3, d=d, dtype=dtype, window=30, spoil=spoil_keys)


def test_prompts_of_large_scores_and_values(pk):
    for dtype in TYPES:
        d, n = 128, 300
        cfg = pk.PromptConfig(n_seq=1, n_kv_heads=1, n_q_heads=2, head_dim=d, dtype=code(pk, dtype))
        q, k, v = (torch.randn(n, h, d, device="cuda").to(dtype) for h in (2, 1, 1))
        for size in (2.0 ** 14, 2.0 ** 22, 2.0 ** 29):
            got = pk.pk_prompt_attention(cfg, q, k, v, ints([0, n]), size)
            # numerators off by E of themselves each, so that weights add up to 1 + E at most, and the result's rounding
            assert torch.isfinite(got).all() and got.abs().max().double() <= v.abs().max().double() * (1 + EPS[dtype]) ** 2 * (1 + n * 2.0 ** -24)
            assert torch.equal(got[0, 0], v[0, 0])
        big = torch.finfo(dtype).max
        got = pk.pk_prompt_attention(cfg, q, k, torch.full_like(v, big), ints([0, n]), d ** -0.5).double()
        # weights off by E each and a sum rounded n times: no further than 2 E from 1 in all, and the type's largest is not passed
        assert (got >= big * (1 - 2 * EPS[dtype])).all() and (got <= big).all()


def test_starts_of_any_kind(pk):
    """Values outside the tensors are clamped, sequences that end before they begin are empty; rows of no sequence are left as they were."""
    n, d = 200, 64
    cfg = pk.PromptConfig(n_seq=4, n_kv_heads=1, n_q_heads=2, head_dim=d)
    q, k, v = (torch.randn(n, h, d, device="cuda").half() for h in (2, 1, 1))
    one = pk.PromptConfig(n_seq=1, n_kv_heads=1, n_q_heads=2, head_dim=d)
    for starts, parts in (([-50, 40, 40, 90, 1 << 30], [(0, 40), (40, 90), (90, 200)]), ([10, 5, 60, 60, 61], [(5, 60), (60, 61)]), ([300, 400, 500, 600, 700], [])):
        out = torch.full((n, 2, d), 7.0, dtype=torch.float16, device="cuda")
        pk.pk_prompt_attention(cfg, q, k, v, ints(starts), 0.2, out=out)
        want = torch.full_like(out, 7.0)
        for a, b in parts:
            pk.pk_prompt_attention(one, q, k, v, ints([a, b]), 0.2, out=want)
        assert torch.equal(out, want)


def test_prompt_layouts(pk):
    """Heads before tokens, one key head for all tokens' heads (stride 0), a result in place of another layout."""
    n, d, hq, hkv = 130, 128, 8, 4
    cfg = pk.PromptConfig(n_seq=2, n_kv_heads=hkv, n_q_heads=hq, head_dim=d)
    q, k, v = (torch.randn(h, n, d, device="cuda").half().transpose(0, 1) for h in (hq, 1, hkv))
    k = k.expand(n, hkv, d)
    starts = ints([0, 61, n])
    want = pk.pk_prompt_attention(cfg, q.contiguous(), k.contiguous(), v.contiguous(), starts, 0.1)
    assert torch.equal(pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1), want)
    out = torch.zeros(hq, n, d + 16, device="cuda").half().transpose(0, 1)[:, :, 8:-8]
    pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1, out=out)
    assert torch.equal(out, want)
    assert pk.pk_prompt_attention(cfg, q[:0], k[:0], v[:0], ints([0, 0, 0]), 0.1).shape == (0, hq, d)


def test_prompts_of_one_key_and_of_tokens_far_apart(pk):
    """Strides of 0 and of more than 2^24 elements, with offsets beyond 2^32 bytes."""
    n, d, stride = 140, 64, (1 << 24) + 8
    cfg = pk.PromptConfig(n_seq=2, n_kv_heads=1, n_q_heads=2, head_dim=d)
    q, k, v = (torch.randn(n, h, d, device="cuda").half() for h in (2, 1, 1))
    starts = ints([0, 71, n])
    one = k[:1].expand(n, 1, d)
    assert torch.equal(pk.pk_prompt_attention(cfg, q, one, v, starts, 0.1), pk.pk_prompt_attention(cfg, q, one.contiguous(), v, starts, 0.1))
    assert torch.equal(pk.pk_prompt_attention(cfg, q, k, one, starts, 0.1), pk.pk_prompt_attention(cfg, q, k, one.contiguous(), starts, 0.1))
    want = pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1)
    far = torch.empty((n - 1) * stride + 4 * d, dtype=torch.float16, device="cuda")
    fk, fv = (far.as_strided((n, 1, d), (stride, d, 1), at) for at in (0, 64))
    fk.copy_(k)
    fv.copy_(v)
    assert torch.equal(pk.pk_prompt_attention(cfg, q, fk, fv, starts, 0.1), want)
    fq, fo = (far.as_strided((n, 2, d), (stride, d, 1), at) for at in (0, 128))   # (the keys' place is free now)
    fq.copy_(q)
    pk.pk_prompt_attention(cfg, fq, k, v, starts, 0.1, out=fo)
    assert torch.equal(fo, want)


def test_many_starts_that_fall(pk):
    """More than 64 sequences, every other one of all rows: the launch has workgroups for a few of them; a row is as it was or right."""
    n, d, n_seq = 200, 64, 100
    cfg = pk.PromptConfig(n_seq=n_seq, n_kv_heads=1, n_q_heads=2, head_dim=d)
    q, k, v = (torch.randn(n, h, d, device="cuda").half() for h in (2, 1, 1))
    out = torch.full((n, 2, d), 7.0, dtype=torch.float16, device="cuda")
    pk.pk_prompt_attention(cfg, q, k, v, ints([n * (i % 2) for i in range(n_seq + 1)]), 0.2, out=out)
    want = pk.pk_prompt_attention(pk.PromptConfig(n_seq=1, n_kv_heads=1, n_q_heads=2, head_dim=d), q, k, v, ints([0, n]), 0.2)
    assert ((out == want).all(-1) | (out == 7.0).all(-1)).all()


def test_as_many_sequences_as_there_may_be(pk):
    rng = random.Random(5)
    run_prompts(pk, [rng.choice([0, 1, 2, 3, 40]) for _ in range(4096)], hkv=1, r=2, d=64)
    p = Paged(pk, 65535, 1, 70000, 2, seed=1)
    for counts in ([rng.choice([0, 1, 1, 2]) for _ in range(65535)], [rng.choice([-1, 0, 1]) for _ in range(65535)]):
        plan, want = p.update(counts, 65000)
        p.check(plan, want)
    # a token or none each: the result is its value
    n = 65535
    cfg = pk.Kv16Config(n_seq=n, n_kv_heads=1, n_q_heads=1, head_dim=64, t_capacity=16, page_tokens=16, n_pages=n)
    order = torch.randperm(n, device="cuda").to(torch.int32)
    cache = pk.Kv16Cache(cfg, page_table=order[:, None])
    cache.k.fill_(0.5), cache.v.copy_(torch.randn(cache.v.shape, device="cuda"))
    cache.states[:, 0] = torch.randint(0, 2, (n,), device="cuda")
    out = pk.pk_kv16_attention(cfg, cache, torch.randn(n, 1, 64, device="cuda").half(), 0.1)
    assert torch.equal(out[:, 0], cache.v[order.long(), 0, 0] * cache.states[:, :1])


# ---- together ----------------------------------------------------------------------------------------------------------------

class Loop:
    """A serving loop as a user writes it: requests come with prompts, get a token per step, finish; one layer."""

    def __init__(self, pk, n_seq=5, hkv=2, r=4, d=128, page=16, dtype=torch.bfloat16, rows=256):
        self.pk, self.rows, self.dtype = pk, rows, dtype
        self.pages = pk.PagesConfig(n_seq=n_seq, page_tokens=page, n_pages=60, pages_per_seq=20)
        self.cfg = pk.Kv16Config(n_seq=n_seq, n_kv_heads=hkv, n_q_heads=hkv * r, head_dim=d, t_capacity=20 * page, dtype=code(pk, dtype), page_tokens=page, n_pages=60)
        self.prompts = pk.PromptConfig(n_seq=n_seq, n_kv_heads=hkv, n_q_heads=hkv * r, head_dim=d, dtype=code(pk, dtype))
        self.pool = pk.PagePool(self.pages)
        self.cache = pk.Kv16Cache(self.cfg, page_table=self.pool.table)
        self.counts = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.plan, self.ws = pk.pk_pages_plan(self.pages, rows), torch.empty(self.pages.workspace_bytes, dtype=torch.uint8, device="cuda")
        self.decode_ws = torch.empty(max(pk.pk_kv16_workspace_bytes(self.cfg, self.cfg.t_capacity), 16), dtype=torch.uint8, device="cuda")
        self.k, self.v = (torch.zeros(rows, hkv, d, dtype=dtype, device="cuda") for _ in range(2))
        self.q = torch.zeros(n_seq, hkv * r, d, dtype=dtype, device="cuda")
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(n_seq, hkv * r, device="cuda")

    def step(self):
        self.pk.pk_pages_update(self.pages, self.pool, self.cache.states, self.counts, self.rows, out=self.plan, workspace=self.ws)
        self.pk.pk_kv16_append(self.cfg, self.cache, self.k, self.v, self.plan.slots)
        self.pk.pk_kv16_attention(self.cfg, self.cache, self.q, 0.1, out=self.out, lse=self.lse, workspace=self.decode_ws)

    def fill(self, counts, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.counts.copy_(torch.tensor(counts, dtype=torch.int32))
        for t in (self.k, self.v, self.q):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    def everything(self):
        return [t.clone() for t in (self.out, self.lse, self.cache.states, self.pool.table, self.pool.free, self.pool.n_free, self.cache.k, self.cache.v,
                                    self.plan.slots, self.plan.starts, self.plan.positions, self.plan.taken)]


STEPS = [[100, 3, 0, 47, 16], [1, 1, 30, 1, 1], [1, 1, 1, 1, 1], [-(1 << 31), 1, 1, 1, 1], [1, 1, 1, -5, 1], [80, 1, 1, 1, 1], [1, 0, -1, 1, 100]]


def test_the_last_token_of_a_prompt_attends_like_a_step(pk):
    """Prompts through the pages into the cache, their attention on the exact vectors; the cache's attention of the last token is the same row."""
    loop = Loop(pk)
    lens = [100, 3, 0, 47, 16]
    loop.fill(lens, 1)
    q = torch.randn(loop.rows, loop.cfg.n_q_heads, 128, device="cuda").to(loop.dtype)
    plan = pk.pk_pages_update(loop.pages, loop.pool, loop.cache.states, loop.counts, loop.rows)
    pk.pk_kv16_append(loop.cfg, loop.cache, loop.k, loop.v, plan.slots)
    lse = torch.zeros(loop.cfg.n_q_heads, loop.rows, device="cuda")
    out = pk.pk_prompt_attention(loop.prompts, q, loop.k, loop.v, plan.starts, 0.1, lse=lse)
    last = (plan.starts[1:] - 1).clamp(min=0).long()
    step_lse = torch.zeros(5, loop.cfg.n_q_heads, device="cuda")
    step = pk.pk_kv16_attention(loop.cfg, loop.cache, q[last], 0.1, lse=step_lse)
    for i, n in enumerate(lens):
        if n == 0:
            assert (step[i] == 0).all() and (step_lse[i] == -math.inf).all()
            continue
        assert torch.allclose(step_lse[i], lse[:, last[i]], atol=1e-4)
        assert (step[i].float() - out[last[i]].float()).abs().max() <= 4 * EPS[loop.dtype] * loop.v.float().abs().max()
    # the same tables serve the 8-bit cache: its append takes `taken` as counts, and moves its own states
    cfg8 = pk.Fp8Config(n_seq=5, n_kv_heads=2, n_q_heads=8, head_dim=128, block=64, t_capacity=1024, dtype=pk.DTYPE_BF16, page_tokens=128, n_pages=30)
    pages = pk.PagesConfig(n_seq=5, page_tokens=128, n_pages=30, pages_per_seq=8)
    pool = pk.PagePool(pages)
    cache8 = pk.Fp8Cache(cfg8, page_table=pool.table)
    after = torch.zeros_like(cache8.states)
    plan = pk.pk_pages_update(pages, pool, cache8.states, loop.counts, loop.rows, states_out=after)
    rows = (plan.starts[:-1, None].long() + torch.arange(100, device="cuda")).clamp(max=loop.rows - 1)
    pk.pk_fp8_append(cfg8, cache8, loop.k[rows].transpose(1, 2), loop.v[rows].transpose(1, 2), counts=plan.taken)
    assert torch.equal(cache8.states, after) and after[:, 0].tolist() == lens
    got = pk.pk_fp8_attention(cfg8, cache8, q[last], 0.1)
    live = torch.tensor(lens) > 0
    far = (got.float() - step.float())[live.cuda()].abs().max()
    assert far <= 0.25 * loop.v.float().abs().max()   # codes of K and V are off by 2^-4 of themselves: another softmax, the same tokens


def test_a_captured_step_replays_while_sequences_come_and_go(pk):
    """Pages, append and attention in one graph; every replay against the eager calls, with eager work of its own between them."""
    eager, graphed = Loop(pk), Loop(pk)
    side = torch.cuda.Stream()
    graphed.fill([0] * 5, 0)
    with torch.cuda.stream(side):
        graphed.step()   # (no counts: nothing changes)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    for i, counts in enumerate(STEPS):
        eager.fill(counts, i)
        graphed.fill(counts, i)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.everything(), graphed.everything()):
            assert torch.equal(a, b), i
        torch.randn(1000, device="cuda").sum().item()


def test_two_graphs_side_by_side(pk):
    """Two captured loops with memory of their own, replayed on two streams at once."""
    loops, want, graphs, streams = [Loop(pk), Loop(pk, dtype=torch.float16)], [Loop(pk), Loop(pk, dtype=torch.float16)], [], []
    for loop in loops:
        loop.fill([0] * 5, 0)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            loop.step()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            loop.step()
        graphs.append(g), streams.append(s)
    for i, counts in enumerate(STEPS):
        for loop in loops + want:
            loop.fill(counts, i)
        for loop in want:
            loop.step()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(loops, want):
            for x, y in zip(a.everything(), b.everything()):
                assert torch.equal(x, y)


def test_prompts_on_another_stream_and_in_a_graph(pk):
    cfg = pk.PromptConfig(n_seq=3, n_kv_heads=2, n_q_heads=8)
    q, k, v = (torch.randn(400, h, 128, device="cuda").half() for h in (8, 2, 2))
    starts, out = ints([0, 0, 0, 0]), torch.zeros(400, 8, 128, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1, out=out)
    for s in ([0, 100, 101, 400], [0, 400, 400, 400], [5, 6, 200, 300]):
        starts.copy_(torch.tensor(s))
        q.normal_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = pk.pk_prompt_attention(cfg, q, k, v, starts, 0.1, out=torch.zeros_like(out))
        assert torch.equal(out, want)


def test_results_repeat(pk):
    """No atomics: the same call gives the same bits."""
    s = Step(pk, [3000, 17, 900], hkv=2, r=5, d=128, dtype=torch.bfloat16)
    q = torch.randn(3, 10, 128, device="cuda").bfloat16()
    want = pk.pk_kv16_attention(s.cfg, s.cache, q, 0.1)
    cfg = pk.PromptConfig(n_seq=2, n_kv_heads=1, n_q_heads=4)
    x = [torch.randn(900, h, 128, device="cuda").half() for h in (4, 1, 1)]
    first = pk.pk_prompt_attention(cfg, *x, ints([0, 333, 900]), 0.1)
    for _ in range(4):
        assert torch.equal(pk.pk_kv16_attention(s.cfg, s.cache, q, 0.1), want)
        assert torch.equal(pk.pk_prompt_attention(cfg, *x, ints([0, 333, 900]), 0.1), first)


def test_calls_check_the_device(pk):
    s = Step(pk, [20])
    q = torch.zeros(1, 8, 128, dtype=torch.float16)
    with pytest.raises(ValueError):
        pk.pk_kv16_attention(s.cfg, s.cache, q, 0.1)
    cfg = pk.PromptConfig(n_seq=1, n_kv_heads=8, n_q_heads=8)
    with pytest.raises(ValueError):
        pk.pk_prompt_attention(cfg, q, q, q, torch.zeros(2, dtype=torch.int32), 0.1)


# ---- large scores by their values ----------------------------------------------------------------------------------------------

def chosen_scores(n, d, dtype, seed):
    """Keys whose element h % 4 is a head's whole score (its query is 1 there, 0 elsewhere), whole numbers that both types hold: the largest one once; at four tokens; at every token; at the
    last one, behind a row that grows.  Values are multiples of 4, so that means of 1, 2 or 4 of them are held too."""
    rng = np.random.default_rng(seed)
    k, v = rng.integers(-40, 41, (n, 1, d)).astype(np.float64), 4.0 * rng.integers(-16, 17, (n, 1, d))
    k[rng.integers(n), 0, 0] = 41
    k[rng.choice(n, min(n, 4), replace=False), 0, 1] = 41
    k[:, 0, 2] = 7
    k[:, 0, 3] = np.arange(n) * 250 // n - 100
    k[n - 1, 0, 3] = 200
    return k, v


def one_hot(n, heads, d):
    q = np.zeros((n, heads, d))
    for h in range(heads):
        q[:, h, h % 4] = 1.0
    return q


def check_chosen(got, got_lse, x, v, scale, dtype):
    """got [rows][d] for scores x [rows][keys] (-inf: not seen), whole numbers times a scale that leaves e^0 and nothing else.  A single largest score above 0, or two or four equal ones, give the
    mean exactly: numerators are powers of two.  Below 0 the reference may be rounded, which moves every numerator alike, by its rounding to the 16-bit type.  The log-sum-exp: six roundings (log2 e, its
    product, the score, the reference, ln 2, the last product) and 2^-20 for the logarithm."""
    E = EPS[dtype]
    s = np.where(x == -math.inf, -math.inf, x * scale)   # (0 times -inf, and a scale below 0)
    top = s.max(1, keepdims=True)
    tied = s == top
    n = tied.sum(1, keepdims=True)
    want, mag = tied @ v / n, tied @ np.abs(v) / n
    exact = np.isin(n, (1, 2, 4)) & (top > 0)
    tol = np.where(exact, np.where(want == 0, 2.0 ** -20 * mag, 0.0), E * np.abs(want) + (E + n * 2.0 ** -24) * mag)
    assert (np.abs(got - want) <= tol).all(), np.argwhere(~(np.abs(got - want) <= tol))[:4]
    want_lse = (top + np.log(n))[:, 0]
    assert (np.abs(got_lse - want_lse) <= 6 * 2.0 ** -24 * np.abs(want_lse) + 2.0 ** -20).all()


LARGE = [2.0 ** 14, -2.0 ** 14, 2.0 ** 22, 2.0 ** 29, -2.0 ** 29, 2.0 ** 40, 2.0 ** 100]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", LARGE)
@pytest.mark.parametrize("d,lens", [(128, [1, 2, 33, 500, 5000]), (256, [3, 700]), (64, [64] * 300)])
def test_attention_of_large_scores_by_value(pk, dtype, scale, d, lens):
    """The values of the largest score's tokens and no others, wherever they lie among tiles, waves and pieces."""
    made = [chosen_scores(n, d, dtype, i) for i, n in enumerate(lens)]
    on = lambda x: (torch.from_numpy(x).to(dtype).cuda(), x)   # noqa: E731
    s = Step(pk, lens, hkv=1, r=4, d=d, dtype=dtype, k=lambda i, n: on(made[i][0]), v=lambda i, n: on(made[i][1]))
    got, lse = s.attend(scale=scale, q=on(one_hot(len(lens), 4, d)), checked=False)
    for i in range(len(lens)):
        k, v = made[i]
        check_chosen(got[i], lse[i], k[:, 0, :4].T, v[:, 0], scale, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", LARGE)
@pytest.mark.parametrize("d,r,lens", [(128, 4, [1, 70, 300]), (256, 4, [150, 33]), (64, 8, [200]), (128, 64, [640, 500, 300, 640])])
def test_prompts_of_large_scores_by_value(pk, dtype, scale, d, r, lens):
    made = [chosen_scores(n, d, dtype, i) for i, n in enumerate(lens)]
    k, v = (torch.from_numpy(np.concatenate([m[i] for m in made])).to(dtype).cuda() for i in range(2))
    n, starts = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    q = torch.from_numpy(one_hot(n, r, d)).to(dtype).cuda()
    lse = torch.zeros(r, n, device="cuda")
    cfg = pk.PromptConfig(n_seq=len(lens), n_kv_heads=1, n_q_heads=r, head_dim=d, dtype=code(pk, dtype))
    got = pk.pk_prompt_attention(cfg, q, k, v, ints(starts.tolist()), scale, lse=lse).double().cpu().numpy()
    lse = lse.double().cpu().numpy()
    for i, (kn, vn) in enumerate(made):
        at = slice(starts[i], starts[i + 1])
        behind = np.triu(np.ones((lens[i], lens[i]), bool), 1)
        for h in range(r):
            x = np.where(behind, -math.inf, kn[None, :, 0, h % 4])
            check_chosen(got[at, h], lse[h, at], x, vn[:, 0], scale, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [2.0 ** 14, 2.0 ** 21, 2.0 ** 22, 2.0 ** 23, 2.0 ** 40, -2.0 ** 14, -2.0 ** 22, -2.0 ** 40])
def test_the_largest_values_under_large_scores(pk, dtype, scale):
    """Equal scores of every size over values of the type's largest: their mean is that value, and the sums that lead to it stay finite."""
    d, lens, big = 128, [1, 2, 70, 700, 5000], torch.finfo(dtype).max
    ones = lambda i, n: (torch.ones(n, 1, d, dtype=dtype, device="cuda"), None)   # noqa: E731
    most = lambda i, n: (torch.full((n, 1, d), big, dtype=dtype, device="cuda"), None)   # noqa: E731
    got, lse = Step(pk, lens, hkv=1, r=4, d=d, dtype=dtype, k=ones, v=most).attend(scale=scale, q=(torch.ones(len(lens), 4, d, device="cuda").to(dtype), None), checked=False)
    # weights off by E each and a sum rounded n times: no further than 2 E from 1 in all, and the type's largest is not passed
    assert (got >= big * (1 - 2 * EPS[dtype])).all() and (got <= big).all()
    want = d * scale + np.log(lens)[:, None]
    assert (np.abs(lse - want) <= 6 * 2.0 ** -24 * np.abs(want) + 2.0 ** -20).all()
    for r, n in ((2, 300), (64, 2100)):
        cfg = pk.PromptConfig(n_seq=1, n_kv_heads=1, n_q_heads=r, head_dim=d, dtype=code(pk, dtype))
        x = [torch.full((n, h, d), y, device="cuda", dtype=dtype) for h, y in ((r, 1.0), (1, 1.0), (1, big))]
        lse = torch.zeros(r, n, device="cuda")
        got = pk.pk_prompt_attention(cfg, *x, ints([0, n]), scale, lse=lse).double()
        assert (got >= big * (1 - 2 * EPS[dtype])).all() and (got <= big).all()
        want = d * scale + np.log(1 + np.arange(n))[None]
        assert (np.abs(lse.double().cpu().numpy() - want) <= 6 * 2.0 ** -24 * np.abs(want) + 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [300, 3000])
def test_scores_on_both_sides_of_a_large_one(pk, dtype, sign, n):
    """Scores, in units of the exponent, of 2^29 and of its neighbour 32 below in binary32 (or their negatives): the smaller one's tokens come first and have 2^-32 of the weight each."""
    d = 64
    scale = np.float32(22.1808)   # 2^5 / log2 e and a little
    x = 2.0 ** 24 - np.arange(0, 130)
    y = (x.astype(np.float32) * np.float32(scale * np.float32(math.log2(math.e)))).astype(np.float64)
    above, below = x[y >= 2.0 ** 29].min(), x[y < 2.0 ** 29].max()
    less, more = (below, above) if sign > 0 else (above, below)
    kn, vn = np.zeros((n, 1, d)), np.full((n, 1, d), 100.0)
    kn[:, 0, 0], kn[:, 0, 1] = 4096.0, less - 2.0 ** 24
    kn[n - 3, 0, 1] = more - 2.0 ** 24
    vn[n - 3] = 1.0
    kn[n - 2:], vn[n - 2:] = (0.0 if sign > 0 else 2 * 4096.0), 50.0
    if sign < 0:
        kn[n - 2:, 0, 1:] = 0.0
    q = np.zeros((1, 2, d))
    q[..., 0], q[..., 1] = 4096.0, 1.0
    on = lambda t: torch.from_numpy(t).to(dtype).cuda()   # noqa: E731
    for t in (kn, vn, q):
        assert (on(t).double().cpu().numpy() == t).all()
    # numerators of 2^-29 and less beside sums of 100 * 3000 * 2^-32 of the winner's 1: half a step of the result covers them
    got, lse = Step(pk, [n], hkv=1, r=2, d=d, dtype=dtype, k=lambda i, n: (on(kn), kn), v=lambda i, n: (on(vn), vn)).attend(
        scale=sign * float(scale), q=(on(q), q), checked=False)
    assert (np.abs(got - 1.0) <= EPS[dtype]).all()
    cfg = pk.PromptConfig(n_seq=1, n_kv_heads=1, n_q_heads=2, head_dim=d, dtype=code(pk, dtype))
    got = pk.pk_prompt_attention(cfg, on(np.repeat(q, n, 0)), on(kn), on(vn), ints([0, n]), sign * float(scale)).double()
    assert ((got[n - 3:] - 1.0).abs() <= EPS[dtype]).all() and (got[:n - 3] == 100.0).all()
