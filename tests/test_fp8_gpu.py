"""The 8-bit cache on the GPU against its definition in 64 bits.

Codes, scales, positions and the choice of an eviction are exact.  A score of magnitude sum S = scale * sum |q k| + |bias| is off by at most
(d + 8) roundings of binary32 relative to S (d products into a binary32 accumulator, then factor, cap, bias, reference);
a softmax weight by twice that, its numerator by fp16's half step 2^-11 on top, and by half of fp16's smallest step, 2^-25, relative to the largest
numerator (kept up to 2^6 smaller where V scales differ); an output by half a step of its own type on top.
"""
import math

import numpy as np
import pytest

import fp8_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2510_05176_amd import patternkv
    return patternkv


EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


class Pair:
    """A cache on the GPU and the same sequences in 64 bits."""

    def __init__(self, pk, seed, n_seq=2, hkv=2, r=4, d=128, block=64, cap=1024, bf16=False, page=0, extra_pages=3, spread=1.0):
        self.pk, self.rng, self.spread = pk, np.random.default_rng(seed), spread
        n_pages = n_seq * (cap // page) + extra_pages if page else 0
        self.cfg = pk.Fp8Config(n_seq=n_seq, n_kv_heads=hkv, n_q_heads=hkv * r, head_dim=d, block=block, t_capacity=cap,
                                dtype=pk.DTYPE_BF16 if bf16 else pk.DTYPE_FP16, page_tokens=page, n_pages=n_pages)
        self.cache = self.new_cache(self.cfg)
        self.seqs = [ref.Sequence(hkv, block, d) for _ in range(n_seq)]
        self.dtype = self.cfg.torch_dtype

    def new_cache(self, cfg):
        cache = self.pk.Fp8Cache(cfg)
        for n in ("k_codes", "v_codes"):   # what lies behind the tokens held is anything, NaN codes included
            noise = torch.from_numpy(self.rng.integers(0, 256, 65521).astype(np.uint8)).cuda()
            cache.buf[n].copy_(noise.repeat(-(-cache.buf[n].numel() // 65521))[:cache.buf[n].numel()])
        for n in ("k_scale", "v_scale", "weight"):
            cache.buf[n].fill_(math.nan)
        if cfg.page_tokens:
            cache.page_table.copy_(torch.from_numpy(self.rng.permutation(cfg.n_pages)[:cache.page_table.numel()].astype(np.int32)).view(cache.page_table.shape))
        return cache

    def rows(self, cfg, cache, seq, head):
        cap, page = cfg.t_capacity, cfg.page_tokens
        t = np.arange(cap)
        if page:
            table = cache.page_table[seq].cpu().numpy().astype(np.int64)
            return (table[t // page] * cfg.n_kv_heads + head) * page + t % page
        return (seq * cfg.n_kv_heads + head) * cap + t

    def vectors(self, n, heads, scale=1.0):
        """[n_seq][heads][n][d] of the 16-bit type, a view of a wider tensor; and in 64 bits"""
        cfg = self.cfg
        x = self.rng.standard_normal((cfg.n_seq, n, heads, cfg.head_dim)) * scale
        x *= np.exp(self.spread * self.rng.standard_normal((cfg.n_seq, n, 1, 1)))
        wide = torch.zeros((cfg.n_seq, n, heads + 1, cfg.head_dim + 8), dtype=self.dtype, device="cuda")
        t = wide[:, :, :heads, :cfg.head_dim].transpose(1, 2)
        t.copy_(torch.from_numpy(x).transpose(1, 2).to(self.dtype))
        return t, t.double().cpu().numpy()

    def append(self, n, counts=None, k=None, v=None, **kw):
        (kt, kn), (vt, vn) = k or self.vectors(n, self.cfg.n_kv_heads), v or self.vectors(n, self.cfg.n_kv_heads)
        c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        got = self.pk.pk_fp8_append(self.cfg, self.cache, kt, vt, counts=c, **kw)
        for b, s in enumerate(self.seqs):
            m = n if counts is None else counts[b]
            m = min(m, self.cfg.t_capacity - s.length)
            s.append(kn[b][:, :m], vn[b][:, :m])
        return got

    def check(self, cfg=None, cache=None, seqs=None, weights=True):
        cfg, cache, seqs = cfg or self.cfg, cache or self.cache, seqs or self.seqs
        d, B = cfg.head_dim, cfg.block
        codes = {n: cache.buf[n + "_codes"].cpu().numpy().reshape(-1, d) for n in "kv"}
        scale = {n: cache.buf[n + "_scale"].cpu().numpy() for n in "kv"}
        pos = cache.buf["pos"].cpu().numpy().reshape(cfg.n_seq, cfg.n_kv_heads, -1)
        weight = cache.buf["weight"].cpu().numpy().reshape(pos.shape)
        states = cache.states.cpu().numpy()
        for b, s in enumerate(seqs):
            assert list(states[b]) == [s.length, s.next, 0, 0], b
            for h in range(cfg.n_kv_heads):
                at = self.rows(cfg, cache, b, h)[:s.length]
                assert np.array_equal(pos[b, h, :s.length], s.pos[h])
                if weights:
                    assert np.array_equal(weight[b, h, :s.length], s.weight[h].astype(np.float32), equal_nan=True)
                for n, want in (("k", s.k[h]), ("v", s.v[h])):
                    nan = np.isnan(ref.VALUES[want.codes])
                    have = codes[n][at]
                    assert np.array_equal((have & 127) == 127, nan), (b, h, n)
                    assert np.array_equal(np.where(nan, 0, have), np.where(nan, 0, want.codes)), (b, h, n)
                    sc = scale[n][at[::B] // B]
                    assert np.array_equal(np.abs(sc), 2.0 ** np.array(want.exp, float)), (b, h, n)
                    assert np.array_equal(np.signbit(sc), np.array(want.flag, bool)), (b, h, n)

    def attend(self, n, counts=None, scale=None, cap=0.0, window=0, slopes=False, weights=None, bound=None, q=None, **kw):
        """A call against the definition; weights: None, or whether they accumulate"""
        cfg = self.cfg
        scale = cfg.head_dim ** -0.5 if scale is None else scale
        qt, qn = q or self.vectors(n, cfg.n_q_heads)
        c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        sl = torch.exp2(-torch.arange(1, cfg.n_q_heads + 1, device="cuda").float()) if slopes else None
        lse = torch.full((cfg.n_seq, cfg.n_q_heads, n), 7.0, device="cuda")
        out = torch.full((cfg.n_seq, cfg.n_q_heads, n, cfg.head_dim), 7.0, dtype=self.dtype, device="cuda")
        self.pk.pk_fp8_attention(cfg, self.cache, qt, scale, cap=cap, window=window, slopes=sl, counts=c, bound=bound, out=out, lse=lse, **kw)
        before = self.cache.buf["weight"].cpu().numpy().reshape(cfg.n_seq, cfg.n_kv_heads, -1).copy()
        if weights is not None:
            self.pk.pk_fp8_weights(cfg, self.cache, qt, lse, scale, cap=cap, window=window, slopes=sl, counts=c, bound=bound, accumulate=weights)
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        after = self.cache.buf["weight"].cpu().numpy().reshape(before.shape)
        r = cfg.n_q_heads // cfg.n_kv_heads
        for b, s in enumerate(self.seqs):
            m = n if counts is None else counts[b]
            assert (got[b, :, m:] == 7.0).all() and (got_lse[b, :, m:] == 7.0).all()   # rows behind the sequence's
            if m:
                want, want_lse, soft, mag, size = s.attention(qn[b][:, :m], scale, cap=cap, window=window, slopes=None if sl is None else sl.double().cpu().numpy())
                off = (cfg.head_dim + 8) * 2.0 ** -24 * size          # of a score
                nan = np.isnan(want)
                top = max([np.nanmax(np.abs(x.values()), initial=0.0) for x in s.v] + [0.0])
                tol = EPS[self.dtype] * np.abs(want) + (2.0 ** -11 + 2 * off[..., None]) * mag + s.length * 2.0 ** -25 * 2 * top + 2.0 ** -25
                assert np.array_equal(np.isnan(got[b, :, :m]), nan), b
                bad = ~nan & ~(np.abs(got[b, :, :m] - want) <= tol)
                assert not bad.any(), (b, np.argwhere(bad)[:4], (np.abs(got[b, :, :m] - want) / tol)[bad][:4])
                empty = want_lse == -np.inf
                assert np.array_equal(got_lse[b, :, :m] == -np.inf, empty) and (got[b, :, :m][empty] == 0).all()
                ok = ~empty & ~np.isnan(want_lse)
                assert np.array_equal(np.isnan(got_lse[b, :, :m]), np.isnan(want_lse))
                far = np.abs(got_lse[b, :, :m][ok] - want_lse[ok])
                assert (far <= (off + s.length * 2.0 ** -24 + 2.0 ** -22 * (np.abs(want_lse) + 2))[ok]).all()
            if weights is not None:
                soft = soft if m else np.zeros((cfg.n_q_heads, 0, s.length))
                rel = (2 * off + s.length * 2.0 ** -24 + 2.0 ** -21 * (np.abs(np.where(empty, 0.0, want_lse)) + 4))[..., None] if m else 0.0
                for h in range(cfg.n_kv_heads):
                    mine = soft[h * r:(h + 1) * r]
                    want_w, tol_w = mine.sum((0, 1)), (mine * rel[h * r:(h + 1) * r]).sum((0, 1)) if m else 0.0
                    old = before[b, h, :s.length].astype(np.float64) if weights else 0.0
                    total = want_w + old
                    room = tol_w + 2.0 ** -24 * (np.abs(total) + (r * m + 4) * want_w) + 1e-37
                    assert (np.abs(after[b, h, :s.length] - total) <= room).all(), (b, h)
                    assert np.array_equal(after[b, h, s.length:], before[b, h, s.length:], equal_nan=True)
                    s.weight[h] = after[b, h, :s.length].astype(np.float64)
        return out, lse


APPENDS = [  # d, block, bf16, page
    (128, 64, False, 0), (128, 64, True, 128), (64, 32, True, 0), (96, 32, False, 256), (96, 64, True, 0), (256, 128, False, 0), (256, 32, True, 128), (64, 128, False, 0)]


@pytest.mark.parametrize("d,block,bf16,page", APPENDS)
def test_append(pk, d, block, bf16, page):
    """In pieces of every kind: prompts, single tokens into begun blocks, unequal counts, nothing; vectors grow, so that begun blocks get
    larger scales."""
    p = Pair(pk, 1, n_seq=3, hkv=2, d=d, block=block, cap=512, bf16=bf16, page=page)
    p.append(70, counts=[70, 1, 0])
    p.check()
    for step in range(4):
        big = 4.0 ** step
        p.append(1, k=p.vectors(1, 2, big), v=p.vectors(1, 2, big))
    p.check()
    p.append(130, counts=[0, 130, 65])
    p.append(33)
    p.append(3, counts=[3, 2, 1], k=p.vectors(3, 2, 2.0 ** -14), v=p.vectors(3, 2, 0.0))
    p.check()


def test_append_stops_at_the_capacity(pk):
    p = Pair(pk, 2, n_seq=2, cap=128, block=64)
    p.append(100, counts=[100, 60])
    p.append(50)
    p.check()
    assert p.cache.lengths.tolist() == [128, 110]
    p.append(1)
    p.append(128)
    p.check()
    assert p.cache.lengths.tolist() == [128, 128]


@pytest.mark.parametrize("bf16", [False, True])
def test_append_of_extreme_values(pk, bf16):
    """Zeros, the type's largest and smallest values, infinities and NaN, which leave the rest of their block alone."""
    p = Pair(pk, 3, n_seq=1, hkv=2, d=64, block=32, cap=256, bf16=bf16)
    info = torch.finfo(p.dtype)
    x = p.rng.standard_normal((1, 100, 2, 64))
    x[0, :5] = 0.0
    x[0, 33, 0, 3], x[0, 34, 1, 0] = math.inf, math.nan
    x[0, 64:96, 1] = -math.inf
    x[0, 40:64, 1] *= info.max / 8
    x[0, 70, 0] = info.smallest_normal
    x[0, 96:, 0] = info.tiny / 4
    x[0, 96:, 1] = info.max
    x = np.clip(x, -info.max, info.max, out=x, where=np.isfinite(x))
    t = torch.from_numpy(x).to(p.dtype).cuda().transpose(1, 2)
    n = t.double().cpu().numpy()
    half = (t[:, :, :50], n[:, :, :50])
    rest = (t[:, :, 50:], n[:, :, 50:])
    p.append(50, k=half, v=half)
    p.append(50, k=rest, v=rest)
    p.check()


def test_append_beside_the_old_states(pk):
    """states_out leaves the cache's own states: drafts are appended, dropped, and others take their place."""
    p = Pair(pk, 4, n_seq=2, d=128, cap=256)
    p.append(61)
    old = p.cache.states.clone()
    out = torch.full_like(old, 9)
    k, v = p.vectors(5, 2), p.vectors(5, 2)
    assert p.pk.pk_fp8_append(p.cfg, p.cache, k[0], v[0], states_out=out) is out
    assert torch.equal(p.cache.states, old) and out.tolist() == [[66, 66, 0, 0]] * 2
    p.append(5, k=k, v=v)     # the same ones again, for good: the begun block's scale is there already
    p.check()
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    p.pk.pk_fp8_append(p.cfg, p.cache, k[0], v[0], counts=none, states_out=out)
    assert torch.equal(out, p.cache.states)
    p.check()


@pytest.mark.parametrize("d,block", [(128, 64), (96, 32), (256, 128), (64, 128)])
def test_append_leaves_pages_behind_the_tokens_alone(pk, d, block):
    """Appends in place whose launch has workgroups without a block of vectors; the entries of the page table behind a sequence's last page
    name pages of its neighbour, as a table does where pages are given out on demand.  The neighbours' codes, scales, positions and
    weights stay as they are."""
    page, n_seq, hkv = 128, 16, 2
    p = Pair(pk, 25, n_seq=n_seq, hkv=hkv, d=d, block=block, cap=1024, page=page)
    own = torch.arange(n_seq * 2, dtype=torch.int32, device="cuda").view(n_seq, 2)         # two pages of its own each
    p.cache.page_table.copy_(torch.cat([own, own.roll(-1, 0).repeat(1, 3)], 1))
    rng = np.random.default_rng(7)
    start = [int(x) for x in rng.integers(0, 2 * block, n_seq)]
    p.append(max(start), counts=start)
    for n in (2, 3, 5, 17, block // 2 + 1, block - 2):
        room = [2 * page - s.length for s in p.seqs]
        p.append(n, counts=[min(int(x), r) for x, r in zip(rng.integers(0, n + 1, n_seq), room)])
        p.check()
    p.append(150, counts=[min(int(x), 2 * page - s.length) for x, s in zip(rng.integers(0, 30, n_seq), p.seqs)])
    p.check()


ATTENDS = [
    # lengths, n, r, d, block, bf16, page, options
    ([1, 5, 64, 65], 1, 4, 128, 64, False, 0, {}),
    ([1, 333, 1000, 517], 1, 1, 128, 32, True, 128, {}),
    ([130, 700, 2, 1024], 1, 7, 256, 128, True, 0, {}),
    ([130, 700, 2, 1024], 1, 16, 96, 64, False, 256, {}),
    ([130, 700, 25, 1024], 1, 24, 64, 32, True, 0, {}),
    ([130, 700, 25, 1024], 1, 64, 128, 64, False, 0, {}),
    ([9, 700, 64, 1000], 5, 4, 128, 32, False, 128, {}),
    ([9, 700, 64, 1000], 5, 5, 128, 64, True, 0, dict(cap=20.0)),
    ([100, 333, 65, 1000], 37, 2, 64, 64, False, 0, {}),
    ([100, 333, 65, 1000], 65, 3, 96, 32, True, 128, dict(cap=5.0)),
    ([200, 333, 129, 1000], 129, 4, 128, 64, True, 0, {}),
    ([200, 333, 129, 1000], 129, 2, 256, 64, False, 0, {}),
    ([9, 700, 64, 1000], 3, 4, 128, 64, False, 0, dict(window=1)),
    ([9, 700, 64, 1000], 3, 4, 128, 64, False, 256, dict(window=100, slopes=True)),
    ([200, 333, 129, 1000], 100, 4, 64, 128, True, 0, dict(window=90)),
    ([200, 333, 129, 1000], 100, 1, 128, 64, False, 0, dict(window=64, slopes=True, cap=10.0)),
    ([9, 700, 64, 1000], 1, 4, 256, 32, True, 128, dict(slopes=True)),
    ([9, 700, 64, 1000], 2, 4, 96, 64, True, 0, dict(window=33, cap=30.0)),
]


# What the capacity decides: short caches are taken whole, longer ones in runs whose pieces are merged, and very long ones in long runs.
CAPS = [1024, 4096, 1 << 19]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("lengths,n,r,d,block,bf16,page,how", ATTENDS)
def test_attention_and_weights(pk, lengths, n, r, d, block, bf16, page, how, cap):
    p = Pair(pk, 5, n_seq=4, hkv=2, r=r, d=d, block=block, cap=cap, bf16=bf16, page=page, spread=0.5)
    p.append(max(lengths), counts=lengths)
    p.attend(n, weights=False, **how)
    p.attend(n, weights=True, **how)
    p.attend(n, counts=[n, n // 2, 0, max(n - 1, 0)], weights=True, bound=64, **how)   # a bound below the lengths costs time only


@pytest.mark.parametrize("cap", [1024, 4096])
@pytest.mark.parametrize("n,r,d,block,bf16,page,how", [
    (90, 3, 96, 32, True, 128, dict(cap=5.0)), (100, 3, 96, 64, False, 0, {}), (300, 1, 64, 64, False, 128, {}), (131, 2, 128, 32, True, 128, dict(window=100, slopes=True)),
    (65, 5, 128, 128, False, 0, {}), (65, 4, 128, 64, True, 0, dict(window=1)), (9, 2, 256, 32, True, 128, {}), (33, 2, 256, 128, False, 0, dict(window=50, cap=10.0))])
def test_many_rows_share_the_keys(pk, n, r, d, block, bf16, page, how, cap):
    """Waves with rows of their own over tiles in LDS: some of the waves without rows or keys, more queries than tokens, one tile and
    several, NaN in a tile that only some rows see, and counts that leave whole workgroups nothing."""
    lengths = [1, 333, 64, 1000]
    p = Pair(pk, 23, n_seq=4, hkv=2, r=r, d=d, block=block, cap=cap, bf16=bf16, page=page, spread=0.5)
    k, v = p.vectors(1000, 2), p.vectors(1000, 2)
    v[0][1, 1, 330, 7] = v[0][3, 0, 995, d - 1] = v[0][3, 1, 500, 3] = math.nan
    k, v = (k[0], k[0].double().cpu().numpy()), (v[0], v[0].double().cpu().numpy())
    p.append(1000, counts=lengths, k=k, v=v)
    p.attend(n, weights=False, **how)
    p.attend(n, weights=False, counts=[n, 1, 0, max(n - 1, 0)], **how)


def test_lse_in_another_order(pk):
    """A log-sum-exp that lies query by query, as a softmax over the heads of one KV head leaves it, gives the same weights."""
    p = Pair(pk, 24, n_seq=2, hkv=1, r=16, cap=512)
    p.append(300, counts=[300, 77])
    q, _ = p.vectors(9, 16)
    lse = torch.empty(2, 16, 9, device="cuda")
    pk.pk_fp8_attention(p.cfg, p.cache, q, 0.1, lse=lse)
    pk.pk_fp8_weights(p.cfg, p.cache, q, lse, 0.1, accumulate=False)
    want = p.cache.buf["weight"].clone()
    turned = lse.transpose(1, 2).contiguous().transpose(1, 2)
    assert not turned.is_contiguous()
    pk.pk_fp8_weights(p.cfg, p.cache, q, turned, 0.1, accumulate=False)
    held = [want.view(2, -1)[b, :n] for b, n in enumerate((300, 77))]
    assert all(torch.equal(x, p.cache.buf["weight"].view(2, -1)[b, :len(x)]) for b, x in enumerate(held))
    with pytest.raises(ValueError):
        pk.pk_fp8_weights(p.cfg, p.cache, q, lse.transpose(1, 2), 0.1)


def nan_rows(pk, seed, n, d, bf16, cap, n_seq=2):
    """Sequences of 300 and 290 tokens; of the queries one is NaN, one infinite; a key that only the last queries see is NaN."""
    p = Pair(pk, seed, n_seq=n_seq, hkv=2, r=2, d=d, cap=cap, bf16=bf16, spread=0.3)
    k, v = p.vectors(300, 2), p.vectors(300, 2)
    k[0][1, 1, 288, 5] = math.nan
    p.append(300, counts=[300, 290], k=(k[0], k[0].double().cpu().numpy()), v=v)
    q, _ = p.vectors(n, 4)
    q[0, 1, 1, 3], q[1, 0, 0, d - 1], q[0, 2, n // 2, :] = math.nan, math.nan, math.inf
    return p, q, q.double().cpu().numpy()


@pytest.mark.parametrize("cap", [512, 4096])
@pytest.mark.parametrize("n,how", [(5, {}), (5, dict(window=40)), (80, {}), (80, dict(window=100, slopes=True)), (80, dict(cap=20.0))])
@pytest.mark.parametrize("d,bf16", [(128, False), (96, True)])
def test_weights_of_rows_without_a_result(pk, n, how, d, bf16, cap):
    """A row whose log-sum-exp is NaN (its query, or a key that it sees, is) gives NaN to the tokens that it sees, and nothing to the others."""
    p, q, qn = nan_rows(pk, 26, n, d, bf16, cap)
    how = dict(how)
    slopes = torch.exp2(-torch.arange(1, 5, device="cuda").float()) if how.pop("slopes", False) else None
    lse = torch.empty(2, 4, n, device="cuda")
    pk.pk_fp8_attention(p.cfg, p.cache, q, 0.1, lse=lse, slopes=slopes, **how)
    for add in (False, True):
        pk.pk_fp8_weights(p.cfg, p.cache, q, lse, 0.1, slopes=slopes, accumulate=add, **how)
    got = p.cache.buf["weight"].double().cpu().numpy().reshape(2, 2, -1)
    partly = 0
    for b, s in enumerate(p.seqs):
        with np.errstate(invalid="ignore"):
            x, size = s.scores(qn[b], 0.1, slopes=None if slopes is None else slopes.double().cpu().numpy(), **how)
        for h in range(2):
            want, room = np.zeros(s.length), np.zeros(s.length)
            for row in range(2 * h, 2 * h + 2):
                for i in range(n):
                    seen = x[row, i] != -np.inf
                    if np.isnan(lse[b, row, i].item()):
                        assert not np.isfinite(x[row, i][seen]).all()
                        want[seen] = math.nan
                        continue
                    assert np.isfinite(x[row, i][seen]).all()
                    top = x[row, i][seen].max()
                    total = top + np.log(np.exp(x[row, i][seen] - top).sum())
                    w = np.exp(x[row, i] - total)
                    want += 2 * w
                    # the scores' roundings in the weight and in the sum, the log-sum-exp's own
                    room += 2 * w * (2 * (d + 8) * 2.0 ** -24 * size[row, i] + s.length * 2.0 ** -24 + 2.0 ** -21 * (abs(total) + 4) + 2.0 ** -24 * (4 * n + 8))
            have = got[b, h, :s.length]
            assert np.isnan(want).any()
            partly += not np.isnan(want).all()
            assert np.array_equal(np.isnan(have), np.isnan(want)), (b, h, np.argwhere(np.isnan(have) != np.isnan(want))[:4])
            ok = ~np.isnan(want)
            assert (np.abs(have - want)[ok] <= room[ok] + 1e-37).all(), (b, h)
    assert partly >= 3


@pytest.mark.parametrize("cap", [256, 4096])
def test_empty_sequences(pk, cap):
    """Nothing held, and more queries than tokens: no row sees anything, or only the last do.  No queries, no new vectors."""
    p = Pair(pk, 6, n_seq=3, cap=cap)
    p.attend(0)
    p.append(0)
    p.check()
    assert p.append(0, states_out=torch.full_like(p.cache.states, 5)).tolist() == [[0, 0, 0, 0]] * 3
    p.attend(1, weights=True)
    p.attend(4, weights=False)
    p.append(3, counts=[0, 3, 1])
    for n in (1, 2, 5, 70):
        p.attend(n, weights=False)
        p.attend(n, weights=False, counts=[n, 0, min(n, 2)], window=2)


@pytest.mark.parametrize("cap", [320, 2240, 1 << 21])
def test_few_heads_and_queries_share_tiles(pk, cap):
    """Every number of rows around the tile sizes."""
    p = Pair(pk, 7, n_seq=1, hkv=1, r=1, d=64, cap=cap)
    p.append(300)
    for n in (15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300):
        p.attend(n, weights=False)


@pytest.mark.parametrize("n_seq,hkv,r,n,window", [(70, 1, 1, 1, 0), (200, 1, 3, 2, 0), (256, 1, 1, 1, 50), (257, 1, 1, 1, 0), (65, 2, 2, 1, 100), (33, 4, 40, 1, 0)])
def test_many_sequences_of_unequal_lengths(pk, n_seq, hkv, r, n, window):
    """Runs that begin and end anywhere in the batch, several sequences in one run and several runs in one sequence, empty ones among
    them; more sequences than one wave has lanes, and more than are dealt out."""
    rng = np.random.default_rng(n_seq)
    p = Pair(pk, 19, n_seq=n_seq, hkv=hkv, r=r, d=64, cap=2176, spread=0.3)
    lengths = [0, 2100, 1] + [int(x) for x in rng.integers(0, 150, n_seq - 4)] + [1300]
    p.append(150, counts=[min(x, 150) for x in lengths])
    rest = [x - min(x, 150) for x in lengths]
    p.append(max(rest), counts=rest)
    p.attend(n, weights=False, window=window)
    p.attend(n, weights=True, counts=[int(x) for x in rng.integers(0, n + 1, n_seq)], window=window)


@pytest.mark.parametrize("cap", [512, 4096])
@pytest.mark.parametrize("n,how", [(1, {}), (1, dict(window=40)), (6, {}), (6, dict(window=40)), (150, {}), (150, dict(window=100))])
@pytest.mark.parametrize("d,block", [(128, 64), (96, 32), (256, 128)])
def test_masked_values_do_not_reach_a_row(pk, n, how, d, block, cap):
    """NaN in K and V at tokens that some rows see and others do not, and in whole blocks; and behind the tokens held (every
    cache of these tests starts with NaN codes and scales there)."""
    p = Pair(pk, 8, n_seq=2, hkv=1, r=2, d=d, block=block, cap=cap)
    k, v = p.vectors(300, 1), p.vectors(300, 1)
    for t, c in ((298, 5), (297, 70 % d), (220, d - 1), (150, 0)):
        v[0][0, 0, t, c] = math.nan
    v[0][1, 0, 10:90] = math.inf
    k[0][1, 0, 20, 3] = math.nan
    k[0][0, 0, 170, 1] = -math.inf
    k, v = (k[0], k[0].double().cpu().numpy()), (v[0], v[0].double().cpu().numpy())
    p.append(300, counts=[300, 299], k=k, v=v)
    p.check()
    p.attend(n, **how)


def test_scores_of_any_size(pk):
    """Queries and keys that make scores of thousands, of nothing, and of both signs; negative scale."""
    p = Pair(pk, 9, n_seq=1, hkv=1, r=4, d=128, cap=512)
    p.append(400, k=p.vectors(400, 1, 30.0))
    q = p.vectors(2, 4, 60.0)
    p.attend(2, q=q)
    p.attend(2, q=q, scale=-0.01, weights=False)
    p.attend(2, q=q, cap=40.0)
    p.attend(2, q=q, scale=0.0, weights=False)
    q[0].zero_()
    p.attend(2, q=(q[0], q[1] * 0.0), weights=False)


@pytest.mark.parametrize("cap", [512, 4096])
@pytest.mark.parametrize("bf16", [False, True])
def test_value_scales_of_every_size(pk, bf16, cap):
    """Blocks whose V scales differ by up to 2^24 (bfloat16: 2^70) in both orders, the large ones with little softmax weight: the rest of
    the result keeps its precision."""
    p = Pair(pk, 10, n_seq=1, hkv=1, r=2, d=64, block=32, cap=cap, bf16=bf16, spread=0.0)
    k, v = p.vectors(512, 1), p.vectors(512, 1)
    sizes = [0, 3, -4, 10, 2, -9, 12, 1, 0, 5, -3, 8, 4, 0, 11, 2] if not bf16 else [0, 3, -40, 30, 2, -9, 12, 1, 0, 25, -35, 8, 4, 0, 11, 2]
    for i, e in enumerate(sizes):
        v[0][0, 0, 32 * i:32 * i + 32] *= 2.0 ** e
    q = p.vectors(1, 2, 4.0)
    for i in (3, 6, 9, 14):       # the keys of the large blocks point away from both queries
        k[0][0, 0, 32 * i:32 * i + 32] -= (q[0][0, 0, 0] + q[0][0, 1, 0]) * 0.5
    p.append(512, k=(k[0], k[0].double().cpu().numpy()), v=(v[0], v[0].double().cpu().numpy()))
    p.attend(1, q=q)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,r,n,how", [(64, 1, 1, {}), (64, 4, 1, dict(cap=1e6)), (128, 1, 1, dict(window=1 << 20)), (64, 3, 9, {}), (64, 1, 300, {}), (256, 2, 9, {}), (64, 64, 512, {})])
def test_many_tokens_of_little_weight(pk, d, r, n, how, bf16):
    """One token with all but the weight of 2^19 others, each 2^-26 of it: in channels where that token has nothing the result is theirs.  A
    numerator is off by 2^-11 of itself, or by half of fp16's smallest step, 2^-36 of the largest numerator."""
    T, count = (1 << 19) + 70, (1 << 19)
    cfg = pk.Fp8Config(n_seq=1, n_kv_heads=1, n_q_heads=r, head_dim=d, t_capacity=(1 << 19) + 128, dtype=pk.DTYPE_BF16 if bf16 else pk.DTYPE_FP16)
    cache = pk.Fp8Cache(cfg, track_weight=False)
    for first in (0, 64 * 5000 + 7):      # where the token is
        cache.states.zero_()
        k = torch.zeros((1, 1, T, d), dtype=cfg.torch_dtype, device="cuda")
        v = torch.ones_like(k)
        k[0, 0, first, 0] = 18.0
        v[0, 0, first, : d // 2] = 0.0
        v[0, 0, :, 1] *= 208.0
        pk.pk_fp8_append(cfg, cache, k, v)
        q = torch.zeros((1, r, n, d), dtype=cfg.torch_dtype, device="cuda")
        q[..., 0] = 1.0
        out = pk.pk_fp8_attention(cfg, cache, q, 1.0, **how).double().cpu().numpy()[0]
        # the capped score: 18 - 18^3 / 3e12 and less
        for i in range(n):
            small = (T - n + i) * math.exp(-18.0)
            want = np.ones(d)
            want[:d // 2] = small / (1 + small)
            want[1] *= 208.0
            # bounds: the score's rounding (18 in units of log2 e: 26, three roundings), the numerators', the sum's over runs of at most
            # 2^13 tokens, the result's
            rel = EPS[cfg.torch_dtype] + 26 * 3 * 2.0 ** -24 + 2.0 ** -11 + 2.0 ** -36 * math.exp(18.0) + 2.0 ** -11
            bad = np.abs(out[:, i] - want) > rel * want
            assert not bad.any(), (i, np.argwhere(bad)[:3], out[0, i, :3], want[:3])



def attend_closely(p, n, q, scale=None, **how):
    """The attention against the definition where a bound by the largest value would say nothing: a numerator is off by 2^-11 of itself or by
    2^-36 of the row's largest (2^6 more where its block's scale of V is up to 2^6 smaller), sums by the roundings of 1024 additions."""
    scale = p.cfg.head_dim ** -0.5 if scale is None else scale
    sl = torch.exp2(-torch.arange(1, p.cfg.n_q_heads + 1, device="cuda").float()) if how.pop("slopes", False) else None
    lse = torch.empty(p.cfg.n_seq, p.cfg.n_q_heads, n, device="cuda")
    got = p.pk.pk_fp8_attention(p.cfg, p.cache, q[0], scale, lse=lse, slopes=sl, **how).double().cpu().numpy()
    lse = lse.double().cpu().numpy()
    r = p.cfg.n_q_heads // p.cfg.n_kv_heads
    for b, s in enumerate(p.seqs):
        want, want_lse, soft, mag, size = s.attention(q[1][b], scale, slopes=None if sl is None else sl.double().cpu().numpy(), **how)
        off = (p.cfg.head_dim + 8) * 2.0 ** -24 * size
        small = np.minimum(soft, 2.0 ** -30 * soft.max(2, keepdims=True))
        lost = np.stack([small[h] @ np.abs(s.v[h // r].values()) for h in range(p.cfg.n_q_heads)])
        tol = EPS[p.dtype] * np.abs(want) + (2.0 ** -11 + 2.0 ** -14 + 2 * off[..., None]) * mag + lost + 2.0 ** -25 * (p.dtype == torch.float16)
        # a bound that could fail: a hundredth of the result in most places
        assert np.median(tol / np.abs(want)) < 0.01, np.median(tol / np.abs(want))
        bad = ~(np.abs(got[b] - want) <= tol)
        assert not bad.any(), (b, np.argwhere(bad)[:4], (np.abs(got[b] - want) / tol)[bad][:4])
        assert (np.abs(lse[b] - want_lse) <= off + 2.0 ** -14 + 2.0 ** -22 * (np.abs(want_lse) + 2)).all(), b


@pytest.mark.parametrize("cap", [512, 4096])
@pytest.mark.parametrize("d,n", [(64, 1), (128, 9), (96, 200), (64, 200), (256, 100)])
@pytest.mark.parametrize("bf16", [False, True])
def test_value_scales_of_every_size_closely(pk, bf16, d, n, cap):
    """Blocks whose V scales differ by up to 2^24 (bfloat16: 2^70) in both orders, the large ones with little softmax weight, against bounds of
    the rest's size: one row and many."""
    p = Pair(pk, 27, n_seq=1, hkv=1, r=2, d=d, block=32, cap=cap, bf16=bf16, spread=0.0)
    k, v = p.vectors(512, 1, 0.25), p.vectors(512, 1)
    v[0].abs_()
    sizes = [0, 3, -4, 10, 2, -9, 12, 1, 0, 5, -3, 8, 4, 0, 11, 2] if not bf16 else [0, 3, -40, 30, 2, -9, 12, 1, 0, 25, -35, 8, 4, 0, 11, 2]
    far = [i for i, e in enumerate(sizes) if e >= 8]
    for i, e in enumerate(sizes):
        v[0][0, 0, 32 * i:32 * i + 32] *= 2.0 ** e
    q, _ = p.vectors(1, 2, 4.0)
    for i in far:       # the keys of the large blocks point away from both queries
        k[0][0, 0, 32 * i:32 * i + 32] -= (q[0, 0, 0] + q[0, 1, 0]) * (40.0 * d ** -0.5 / 4.0 / 4.0)
    p.append(512, k=(k[0], k[0].double().cpu().numpy()), v=(v[0], v[0].double().cpu().numpy()))
    q = q.expand(-1, -1, n, -1)
    attend_closely(p, n, (q, q.double().cpu().numpy()))


@pytest.mark.parametrize("d,r,n,bf16,page,how", [
    (64, 1, 1, False, 0, {}), (64, 8, 1, True, 256, {}), (128, 8, 3, False, 0, dict(cap=30.0)), (64, 1, 300, False, 0, {}), (96, 5, 3, True, 0, dict(window=30000)),
    (256, 8, 1, False, 128, {}), (256, 8, 4, True, 0, dict(window=20000))])
@pytest.mark.parametrize("at", [700, 32900])
def test_more_pieces_than_lanes(pk, d, r, n, bf16, page, how, at):
    """One KV head over 33k tokens: more runs of its keys than a wave that merges them has lanes; the largest score in one of the first of
    them, or of the last."""
    p = Pair(pk, 28, n_seq=1, hkv=1, r=r, d=d, block=128, cap=33280, bf16=bf16, page=page, spread=0.3)
    k, v = p.vectors(33100, 1), p.vectors(33100, 1)
    v[0].add_(2.0)
    q = p.vectors(n, r)
    k[0][0, 0, at] = q[0][0, 0, 0] * 1.5
    p.append(33100, k=(k[0], k[0].double().cpu().numpy()), v=(v[0], v[0].double().cpu().numpy()))
    attend_closely(p, n, q, **how)


@pytest.mark.parametrize("d,n", [(64, 1), (128, 200), (256, 3)])
def test_values_near_the_largest(pk, d, n):
    """Values up to a quarter of bfloat16's largest: the weighted mean of many of them is finite, though their sum is not."""
    p = Pair(pk, 29, n_seq=1, hkv=1, r=2, d=d, cap=8192, bf16=True, spread=0.0)
    k, v = p.vectors(8000, 1), p.vectors(8000, 1)
    v[0].abs_().clamp_(max=3.0).add_(1.0).mul_(2.0 ** 124)
    p.append(8000, k=k, v=(v[0], v[0].double().cpu().numpy()))
    attend_closely(p, n, p.vectors(n, 2))


@pytest.mark.parametrize("d,r,n,cap", [(64, 1, 1, 1024), (128, 4, 1, 8192), (64, 2, 200, 1024), (256, 1, 20, 1024), (128, 20, 1, 1024)])
@pytest.mark.parametrize("how", [{}, dict(window=1 << 20)])
def test_scores_whose_steps_are_large(pk, d, r, n, cap, how):
    """Scores around 2^18 to 2^40 of both signs, whose own binary32 steps are up to 2^17: results are means of the values and the log-sum-exp is the
    largest score's, whatever the order of the scores."""
    cfg = pk.Fp8Config(n_seq=4, n_kv_heads=1, n_q_heads=r, head_dim=d, t_capacity=cap, dtype=pk.DTYPE_BF16)
    g = torch.Generator().manual_seed(31)
    for e in range(18, 41, 2):
        cache = pk.Fp8Cache(cfg, track_weight=False)
        k = torch.zeros(4, 1, 900, d)
        k[:2, 0, :, 0], k[2:, 0, :, 0] = 1.0, -1.0
        rise = torch.randint(0, 16, (900,), generator=g).float() / 16            # 1 .. 1.9 in steps that e4m3 has
        k[:, 0, :, 0] *= 1 + (rise * 8).floor() / 8
        k[1::2, 0] = k[1::2, 0].flip(1).sort(1).values                           # every second sequence in order
        v = torch.rand(4, 1, 900, d, generator=g) + 1.0
        pk.pk_fp8_append(cfg, cache, k.bfloat16().cuda(), v.bfloat16().cuda())
        q = torch.zeros(4, r, n, d)
        q[..., 0] = 1.37 * 2.0 ** e
        q[..., 1] = 1.0
        lse = torch.empty(4, r, n, device="cuda")
        out = pk.pk_fp8_attention(cfg, cache, q.bfloat16().cuda(), 1.0, lse=lse, **how).float().cpu()
        assert torch.isfinite(out).all() and (out >= 1 - 2.0 ** -4).all() and (out <= 2 + 2.0 ** -3).all(), (e, out.min(), out.max())
        top = torch.stack([k[..., : 900 - n + i + 1, 0].amax(-1).expand(-1, r) for i in range(n)], 2) * q[..., 0].bfloat16().float()
        # e4m3 and the values' own rounding aside, a row's mean lies among its largest scores' values; the sum of up to 900 of them adds 10
        assert ((lse.cpu() - top).abs() <= 10 + top.abs() * 2.0 ** -20).all(), e


EVICTS = [(128, 64, 0, 0, 100, 4, 16), (64, 32, 128, 0, 64, 0, 0), (96, 32, 0, 128, 77, 0, 77), (256, 128, 256, 128, 129, 1, 0), (128, 64, 0, 0, 1, 0, 0), (64, 64, 0, 0, 63, 31, 32)]


@pytest.mark.parametrize("d,block,page,to_page,budget,first,last", EVICTS)
def test_evict(pk, d, block, page, to_page, budget, first, last):
    """Unequal lengths on both sides of the budget; equal weights, zeros of both signs, infinite and NaN ones; NaN codes move along."""
    p = Pair(pk, 11, n_seq=4, hkv=2, d=d, block=block, cap=512, page=page)
    k = p.vectors(500, 2)
    k[0][1, 0, 450, 2] = math.nan
    p.append(500, counts=[500, 499, 0, budget], k=(k[0], k[0].double().cpu().numpy()))
    w = p.cache.buf["weight"].view(4, 2, -1)
    for b, s in enumerate(p.seqs):
        for h in range(2):
            x = p.rng.random(s.length).astype(np.float32) ** 4
            if h == 1:
                x = np.float32(p.rng.integers(0, 3, s.length))   # many ties
                x[x == 0] *= np.float32(-1.0) ** np.arange((x == 0).sum())
            if b == 1 and s.length > 60:
                x[20:40], x[50] = math.nan, math.inf
            s.weight[h] = x.astype(np.float64)
            w[b, h, :s.length] = torch.from_numpy(x).cuda()
    n_pages = 4 * (256 // to_page) + 2 if to_page else 0
    to_cfg = pk.Fp8Config(n_seq=4, n_kv_heads=2, n_q_heads=8, head_dim=d, block=block, t_capacity=256, page_tokens=to_page, n_pages=n_pages)
    to = p.new_cache(to_cfg)
    before = {n: t.clone() for n, t in p.cache.buf.items()}
    pk.pk_fp8_evict(p.cfg, p.cache, to_cfg, to, budget, keep_first=first, keep_last=last)
    p.check(to_cfg, to, [s.evict(budget, first, last) for s in p.seqs])
    assert all(torch.equal(before[n].view(torch.uint8), p.cache.buf[n].view(torch.uint8)) for n in before)


def test_evict_larger_budget_than_the_cache(pk):
    p = Pair(pk, 12, n_seq=2, cap=128)
    p.append(128, counts=[128, 5])
    to_cfg = pk.Fp8Config(n_seq=2, n_kv_heads=2, n_q_heads=8, t_capacity=1024)
    to = p.new_cache(to_cfg)
    pk.pk_fp8_evict(p.cfg, p.cache, to_cfg, to, 1024)
    p.check(to_cfg, to, [s.evict(1024, 0, 0) for s in p.seqs])


def test_evict_long(pk):
    """More tokens than the selection's workgroup has threads, every weight from few values."""
    p = Pair(pk, 13, n_seq=1, hkv=1, r=1, d=64, block=128, cap=8192)
    p.append(8191)
    x = np.float32(p.rng.integers(0, 50, 8191) / 7.0)
    p.seqs[0].weight[0] = x.astype(np.float64)
    p.cache.buf["weight"][:8191] = torch.from_numpy(x).cuda()
    to_cfg = pk.Fp8Config(n_seq=1, n_kv_heads=1, n_q_heads=1, head_dim=64, block=128, t_capacity=4096)
    to = p.new_cache(to_cfg)
    pk.pk_fp8_evict(p.cfg, p.cache, to_cfg, to, 3001, keep_first=3, keep_last=100)
    p.check(to_cfg, to, [p.seqs[0].evict(3001, 3, 100)])


@pytest.mark.parametrize("cap,held,budget,first,last", [
    (4096, 4000, 1000, 0, 0), (4224, 4223, 4000, 100, 60), (16384, 16380, 64, 1, 1), (32768, 32768, 20000, 0, 5), (32832, 32832, 32000, 40, 24), (65536, 40000, 333, 0, 0)])
@pytest.mark.parametrize("kind", ["distinct", "few", "equal"])
def test_evict_chooses_the_largest(pk, cap, held, budget, first, last, kind):
    """Every way of choosing, by the capacity; weights that are all different, from few values, all the same."""
    p = Pair(pk, 18, n_seq=1, hkv=2, r=1, d=64, block=64, cap=cap)
    p.cache.states.copy_(torch.tensor([[held, held, 0, 0]]))
    p.cache.buf["k_codes"].fill_(8)      # what the tokens hold is not looked at here
    p.cache.buf["v_codes"].fill_(8)
    p.cache.buf["k_scale"].fill_(1.0)
    p.cache.buf["v_scale"].fill_(1.0)
    pos = np.arange(cap, dtype=np.int32)
    p.cache.buf["pos"].copy_(torch.from_numpy(np.concatenate([pos, pos])))
    w = np.stack([np.float32(p.rng.permutation(cap) + 1) * 1e-3, np.float32(p.rng.permutation(cap) + 1) * -1e20])
    w = w if kind == "distinct" else np.float32(p.rng.integers(0, 4, (2, cap)) * 0.1) if kind == "few" else np.full((2, cap), 0.7, np.float32)
    p.cache.buf["weight"].copy_(torch.from_numpy(w.reshape(-1)))
    to_cap = -(-budget // 64) * 64
    to_cfg = pk.Fp8Config(n_seq=1, n_kv_heads=2, n_q_heads=2, head_dim=64, t_capacity=to_cap)
    to = p.new_cache(to_cfg)
    pk.pk_fp8_evict(p.cfg, p.cache, to_cfg, to, budget, keep_first=first, keep_last=last)
    got = to.buf["pos"].cpu().numpy().reshape(2, -1)[:, :budget]
    for h in range(2):
        middle = np.arange(first, held - last)
        order = middle[np.argsort(-w[h, middle].astype(np.float64), kind="stable")][:budget - first - last]
        assert np.array_equal(got[h], np.sort(np.concatenate([np.arange(first), order, np.arange(held - last, held)])))
    assert to.states.tolist() == [[budget, held, 0, 0]]


@pytest.mark.parametrize("bf16,page", [(False, 0), (True, 128)])
def test_a_serving_loop(pk, bf16, page):
    """Prompts, generation steps with weights, eviction, further steps with window and distance bias over the gaps, drafts, eviction
    back."""
    p = Pair(pk, 14, n_seq=2, hkv=2, r=4, d=128, block=32, cap=512, bf16=bf16, page=page, spread=0.5)
    p.append(300, counts=[300, 170])
    p.attend(32, weights=False)
    for _ in range(3):
        p.append(1)
        p.attend(1, weights=True)
    first_cfg, first = p.cfg, p.cache
    to_cfg = pk.Fp8Config(n_seq=2, n_kv_heads=2, n_q_heads=8, head_dim=128, block=32, t_capacity=256, dtype=p.cfg.dtype)
    to = p.new_cache(to_cfg)
    pk.pk_fp8_evict(p.cfg, p.cache, to_cfg, to, 150, keep_first=4, keep_last=20)
    p.cfg, p.cache, p.seqs = to_cfg, to, [s.evict(150, 4, 20) for s in p.seqs]
    p.check()
    for _ in range(3):
        p.append(1)
        p.attend(1, weights=True, window=60, slopes=True)
    p.append(5)
    p.attend(5, weights=True, window=200, slopes=True, cap=20.0)
    p.check()
    first.states.zero_()
    pk.pk_fp8_evict(p.cfg, p.cache, first_cfg, first, 64, keep_first=1, keep_last=30)
    p.cfg, p.cache, p.seqs = first_cfg, first, [s.evict(64, 1, 30) for s in p.seqs]
    p.append(1)
    p.attend(1, slopes=True)
    p.check()


@pytest.mark.parametrize("cap", [1024, 4096])
def test_replayed_graph_grows_the_sequences(pk, cap):
    """A generation step (append in place, attention, weights) captured once and replayed with new tokens, eager work and waits in
    between, against the same steps without a graph."""
    a, b = (Pair(pk, 15, n_seq=3, hkv=2, r=4, cap=cap) for _ in range(2))
    a.append(200, counts=[200, 63, 0])
    b.append(200, counts=[200, 63, 0])
    new = [(a.vectors(1, 2)[0], a.vectors(1, 2)[0], a.vectors(1, 8)[0]) for _ in range(6)]
    k, v, q = (t.clone() for t in new[0])
    out, lse = torch.zeros(3, 8, 1, 128, dtype=torch.float16, device="cuda"), torch.zeros(3, 8, 1, device="cuda")

    def step(p, k, v, q, out, lse):
        pk.pk_fp8_append(p.cfg, p.cache, k, v)
        pk.pk_fp8_attention(p.cfg, p.cache, q, 0.09, out=out, lse=lse)
        pk.pk_fp8_weights(p.cfg, p.cache, q, lse, 0.09)

    step(a, k, v, q, out, lse)       # everything the launches need is loaded before the capture
    step(b, k, v, q, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, k, v, q, out, lse)
    for kk, vv, qq in new[1:]:
        k.copy_(kk), v.copy_(vv), q.copy_(qq)
        graph.replay()
        out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
        step(b, kk, vv, qq, out2, lse2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(a.cache.states, b.cache.states)
        held = b.cache.lengths.max().item()
        for n in ("pos", "weight"):
            for s, have in enumerate(b.cache.lengths.tolist()):
                assert torch.equal(a.cache.buf[n].view(3, 2, -1)[s, :, :have], b.cache.buf[n].view(3, 2, -1)[s, :, :have])
        assert held > 200


def test_another_stream(pk):
    p = Pair(pk, 16, n_seq=2, cap=1024)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.append(700)
        p.attend(1, weights=False)
    s.synchronize()
    p.check()


def test_many_appends_in_place_count_once(pk):
    """The state moves once per call, however many workgroups an append has."""
    p = Pair(pk, 17, n_seq=1, hkv=4, r=1, d=64, block=32, cap=8192)
    t = torch.randn(1, 4, 1000, 64, device="cuda").half()
    for i in range(1, 9):
        pk.pk_fp8_append(p.cfg, p.cache, t, t)
        assert p.cache.states.tolist() == [[min(1000 * i, 8192), min(1000 * i, 8192), 0, 0]]


def test_a_stream_of_more_than_4_gib(pk):
    """Byte offsets inside a stream that need more than 32 bits: the same tokens at the end of a long stream and in a short one."""
    cap = 1 << 25
    long_cfg = pk.Fp8Config(n_seq=1, n_kv_heads=1, n_q_heads=4, head_dim=256, t_capacity=cap)
    short_cfg = pk.Fp8Config(n_seq=1, n_kv_heads=1, n_q_heads=4, head_dim=256, t_capacity=512)
    long, short = pk.Fp8Cache(long_cfg), pk.Fp8Cache(short_cfg)
    start = cap - 448
    long.states.copy_(torch.tensor([[start, start, 0, 0]]))
    g = torch.Generator().manual_seed(3)
    k, v, q = (torch.randn(1, h, n, 256, generator=g).half().cuda() for h, n in ((1, 448), (1, 448), (4, 2)))
    got = []
    for cfg, cache in ((long_cfg, long), (short_cfg, short)):
        pk.pk_fp8_append(cfg, cache, k, v)
        lse = torch.zeros(1, 4, 2, device="cuda")
        out = pk.pk_fp8_attention(cfg, cache, q, 0.1, window=440, lse=lse, bound=512)
        pk.pk_fp8_weights(cfg, cache, q, lse, 0.1, window=440, accumulate=False)
        got.append((out, lse))
    assert long.states.tolist() == [[cap, cap, 0, 0]]
    assert torch.equal(long.buf["k_codes"][start * 256:], short.buf["k_codes"][:448 * 256])
    assert torch.equal(long.buf["v_codes"][start * 256:], short.buf["v_codes"][:448 * 256])
    assert torch.equal(long.buf["weight"][start:], short.buf["weight"][:448])
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][0], got[1][0])
