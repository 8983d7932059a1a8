"""The paged 16-bit cache, its pages and the attention of prompts without a GPU: sizes, refusals (every one before a launch, so that fake pointers do),
what the binding looks at, and that the reference that the GPU tests compare with keeps its pages in order."""
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

import kv16_reference as ref

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2510_05176_amd", "libpatternkv.so")), reason="libpatternkv.so not built")

OK, INVALID, UNSUPPORTED, SHAPE, ALIGNMENT, CAPACITY, STATE, WORKSPACE = range(8)
P = 0x10000000   # never dereferenced


@pytest.fixture(scope="module")
def pk():
    from paper_2510_05176_amd import patternkv
    return patternkv


BASE = dict(n_seq=2, n_kv_heads=2, n_q_heads=8, head_dim=128, t_capacity=1024, page_tokens=16, n_pages=200)


@pytest.mark.parametrize("change", [dict(), dict(n_kv_heads=1, n_q_heads=24, head_dim=256), dict(n_seq=5, n_q_heads=128, head_dim=256), dict(n_seq=250, n_q_heads=40), dict(n_seq=300)])
def test_workspaces_grow_with_the_bound(pk, change):
    cfg = pk.Kv16Config(**{**BASE, "t_capacity": 1 << 20, **change})
    bounds = sorted({b for i in range(4, 21) for b in ((1 << i) - 1, 1 << i, (1 << i) + 1, 3 << (i - 1), 5 << (i - 2)) if b <= 1 << 20})
    needs = [pk.pk_kv16_workspace_bytes(cfg, b) for b in bounds]
    assert needs == sorted(needs) and (needs[-1] > 0 or cfg.n_seq == 300)


def test_workspaces_for_a_larger_bound_serve_every_smaller_one(pk):
    """Whichever form the kernel takes (256 channels with more than 16 heads per KV head have two, by sequences * KV heads * bound), and wherever the keys stop being dealt out."""
    for hkv in (1, 2, 3, 4, 8):
        for r in (1, 16, 17, 20, 33, 40, 48, 49, 64):
            for n_seq in (1, 2, 26, 31, 32, 46, 61, 64, 85, 86, 100, 127, 128, 170, 171, 255, 256, 257):
                cfg = pk.Kv16Config(**{**BASE, "t_capacity": 1 << 20, "n_seq": n_seq, "n_kv_heads": hkv, "n_q_heads": hkv * r, "head_dim": 256})
                turn = (1 << 18) // (n_seq * hkv)
                bounds = sorted({b for b in (0, 1, 256, 257, 1000, turn - 1, turn, turn + 1, turn + 100, 2 * turn, 1 << 20) if 0 <= b <= 1 << 20})
                needs = [pk.pk_kv16_workspace_bytes(cfg, b) for b in bounds]
                assert needs == sorted(needs), (hkv, r, n_seq, bounds, needs)


def test_sizes(pk):
    cfg = pk.Kv16Config(**BASE)
    assert pk.pk_kv16_cache_bytes(cfg) == 200 * 2 * 16 * 128 * 2
    last = 0
    for bound in range(0, 1025, 16):
        need = pk.pk_kv16_workspace_bytes(cfg, bound)
        assert need >= last
        last = need
    assert last > 0 and pk.pk_kv16_workspace_bytes(cfg, -1) == 0 and pk.pk_kv16_workspace_bytes(cfg, 1025) == 0
    assert pk.PagesConfig(n_seq=1000, page_tokens=1, n_pages=5, pages_per_seq=3).workspace_bytes >= 4000
    big = pk.Kv16Config(n_seq=65535, n_kv_heads=1, n_q_heads=64, head_dim=256, t_capacity=1 << 25, page_tokens=1 << 25, n_pages=63)
    assert pk.pk_kv16_cache_bytes(big) == 63 * (1 << 25) * 512


@pytest.mark.parametrize("change", [
    dict(head_dim=80), dict(n_q_heads=7), dict(n_q_heads=130), dict(t_capacity=1000), dict(t_capacity=0), dict(t_capacity=1 << 26), dict(dtype=2),
    dict(n_seq=0), dict(n_seq=40000), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=0), dict(page_tokens=2048), dict(n_pages=0),
    dict(n_pages=1 << 27), dict(n_kv_heads=0)])
def test_bad_configurations(pk, change):
    cfg = pk.Kv16Config(**{**BASE, **change})
    assert pk.pk_kv16_cache_bytes(cfg) == 0 and pk.pk_kv16_workspace_bytes(cfg, 16) == 0
    with pytest.raises(ValueError):
        pk.Kv16Cache(cfg, device="cpu")


@pytest.mark.parametrize("change", [dict(n_seq=0), dict(n_seq=65536), dict(page_tokens=0), dict(page_tokens=24), dict(n_pages=0), dict(n_pages=1 << 27),
                                    dict(pages_per_seq=0), dict(pages_per_seq=(1 << 21) + 1)])
def test_bad_pages(pk, change):
    assert pk.PagesConfig(**{**dict(n_seq=4, page_tokens=16, n_pages=9, pages_per_seq=3), **change}).workspace_bytes == 0


def pages_update(pk, table=P, free=P + 0x1000, n_free=P + 0x2000, n_free_out=0, states=P + 0x3000, states_out=0, counts=P + 0x4000, n=8, starts=P + 0x5000,
                 slots=P + 0x6000, positions=P + 0x7000, taken=P + 0x8000, ws=P + 0x9000, size=1 << 20, cfg=None):
    cfg = cfg or pk._pack_pages_config(4, 16, 9, 3)
    return pk._lib.pk_pages_update(cfg, pk._pack_pages(table, free, n_free, n_free_out), states, states_out, counts, n, starts, slots, positions, taken, ws, size, None)


def test_pages_refuse(pk):
    for want, kw in [(INVALID, dict(table=0)), (INVALID, dict(free=0)), (INVALID, dict(n_free=0)), (INVALID, dict(states=0)), (INVALID, dict(counts=0)),
                     (INVALID, dict(starts=0)), (INVALID, dict(slots=0)), (INVALID, dict(taken=0)), (INVALID, dict(n=-1)), (WORKSPACE, dict(ws=0)),
                     (WORKSPACE, dict(size=15)), (ALIGNMENT, dict(table=P + 4)), (ALIGNMENT, dict(free=P + 0x1008)), (ALIGNMENT, dict(n_free=P + 0x2004)),
                     (ALIGNMENT, dict(n_free_out=P + 0xa004)), (ALIGNMENT, dict(states=P + 0x3004)), (ALIGNMENT, dict(states_out=P + 0xb004)),
                     (ALIGNMENT, dict(counts=P + 0x4004)), (ALIGNMENT, dict(starts=P + 0x5004)), (ALIGNMENT, dict(slots=P + 0x6004)),
                     (ALIGNMENT, dict(positions=P + 0x7004)), (ALIGNMENT, dict(taken=P + 0x8004)), (ALIGNMENT, dict(ws=P + 0x9004)),
                     # one array within another
                     (INVALID, dict(states_out=P + 0x3010)), (INVALID, dict(taken=P + 0x5010)), (INVALID, dict(slots=P + 0x7010)), (INVALID, dict(counts=P + 0x8000)),
                     (INVALID, dict(starts=P + 0x4000)), (INVALID, dict(n_free_out=P + 0x1010)), (INVALID, dict(ws=P)),
                     (UNSUPPORTED, dict(cfg=pk._pack_pages_config(4, 24, 9, 3))), (INVALID, dict(cfg=pk._pack_pages_config(0, 16, 9, 3))),
                     (UNSUPPORTED, dict(cfg=pk._pack_pages_config(65536, 16, 9, 3))), (UNSUPPORTED, dict(cfg=pk._pack_pages_config(4, 16, 1 << 27, 3))),
                     (UNSUPPORTED, dict(cfg=pk._pack_pages_config(4, 16, 9, (1 << 21) + 1)))]:
        assert pages_update(pk, **kw) == want, kw


def strides(pk, *s):
    return pk._pack_strides(*(s or (1024, 1024, 128)))


def scores(pk, scale=1.0, cap=0.0, window=0, slopes=0):
    return pk._pack_fp8_scores(scale, cap, window, slopes)


def append(pk, cfg=None, k=P, v=P, k_new=P, v_new=P, ks=None, vs=None, slots=P, n=4):
    return pk._lib.pk_kv16_append(cfg or pk.Kv16Config(**BASE).packed, pk._pack_kv16_cache(k, v, 0), k_new, v_new, ks or strides(pk), vs or strides(pk), slots, n, None)


def attention(pk, cfg=None, k=P, v=P, table=P, states=P, bound=1024, q=P, qs=None, sc=None, out=P, os_=None, lse=0, ws=P, size=1 << 40):
    return pk._lib.pk_kv16_attention(cfg or pk.Kv16Config(**BASE).packed, pk._pack_kv16_cache(k, v, table), states, bound, q, qs or strides(pk), sc or scores(pk),
                                     out, os_ or strides(pk), lse, ws, size, None)


def prompt(pk, n_seq=2, hkv=2, hq=8, d=128, dtype=0, q=P, k=P, v=P, qs=None, ks=None, vs=None, starts=P, n=4, sc=None, out=P, os_=None, lse=0):
    return pk._lib.pk_prompt_attention(pk._pack_prompt_config(n_seq, hkv, hq, d, dtype), q, k, v, qs or strides(pk), ks or strides(pk), vs or strides(pk), starts, n,
                                       sc or scores(pk), out, os_ or strides(pk), lse, None)


BAD_SCORES = [dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=1e-38), dict(cap=float("inf")), dict(window=-1)]


def test_append_refuses(pk):
    assert append(pk, n=0) == OK and append(pk, n=0, k_new=0, v_new=0, slots=0) == OK
    bad = pk.Kv16Config(**{**BASE, "page_tokens": 8}).packed
    for want, kw in [(INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(k_new=0)), (INVALID, dict(v_new=0)), (INVALID, dict(slots=0)), (INVALID, dict(n=-1)),
                     (UNSUPPORTED, dict(cfg=bad)), (ALIGNMENT, dict(k=P + 8)), (ALIGNMENT, dict(v=P + 2)), (ALIGNMENT, dict(k_new=P + 8)), (ALIGNMENT, dict(v_new=P + 2)),
                     (ALIGNMENT, dict(slots=P + 4)), (ALIGNMENT, dict(ks=strides(pk, 0, 4, 128))), (ALIGNMENT, dict(vs=strides(pk, 0, 1024, 129)))]:
        assert append(pk, **kw) == want, kw


def test_attention_refuses(pk):
    for want, kw in [(INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(table=0)), (INVALID, dict(states=0)), (INVALID, dict(q=0)), (INVALID, dict(out=0)),
                     (INVALID, dict(bound=-1)), (CAPACITY, dict(bound=1025)), (ALIGNMENT, dict(table=P + 4)), (ALIGNMENT, dict(states=P + 8)), (ALIGNMENT, dict(q=P + 8)),
                     (ALIGNMENT, dict(out=P + 8)), (ALIGNMENT, dict(lse=P + 4)), (ALIGNMENT, dict(ws=P + 4)), (ALIGNMENT, dict(sc=scores(pk, slopes=P + 4))),
                     (ALIGNMENT, dict(qs=strides(pk, 4, 0, 128))), (ALIGNMENT, dict(os_=strides(pk, 1024, 0, 132))), (SHAPE, dict(os_=strides(pk, 0, 0, 128))),
                     (SHAPE, dict(os_=strides(pk, 1024, 0, 0))), (SHAPE, dict(os_=strides(pk, 1024, 0, -120))), (SHAPE, dict(os_=strides(pk, 64, 0, 2048))),
                     (WORKSPACE, dict(ws=0)), (WORKSPACE, dict(size=255))] + [(INVALID, dict(sc=scores(pk, **b))) for b in BAD_SCORES]:
        assert attention(pk, **kw) == want, kw


def test_prompt_refuses(pk):
    assert prompt(pk, n=0) == OK and prompt(pk, n=0, q=0, k=0, v=0, out=0) == OK
    for want, kw in [(INVALID, dict(q=0)), (INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(out=0)), (INVALID, dict(starts=0)), (INVALID, dict(n=-1)),
                     (INVALID, dict(n_seq=0)), (UNSUPPORTED, dict(n_seq=4097)), (UNSUPPORTED, dict(d=80)), (SHAPE, dict(hq=7)), (UNSUPPORTED, dict(hq=130)),
                     (INVALID, dict(dtype=2)), (UNSUPPORTED, dict(n=(1 << 25) + 1)), (UNSUPPORTED, dict(hkv=1, hq=64, n=(1 << 22) + 1)),
                     (UNSUPPORTED, dict(hkv=60000, hq=60000, n=1 << 20)), (ALIGNMENT, dict(q=P + 8)), (ALIGNMENT, dict(k=P + 8)),
                     (ALIGNMENT, dict(v=P + 8)), (ALIGNMENT, dict(out=P + 8)), (ALIGNMENT, dict(starts=P + 4)), (ALIGNMENT, dict(lse=P + 4)),
                     (ALIGNMENT, dict(sc=scores(pk, slopes=P + 4))), (ALIGNMENT, dict(qs=strides(pk, 0, 12, 128))), (ALIGNMENT, dict(ks=strides(pk, 0, 1024, 4))),
                     (ALIGNMENT, dict(vs=strides(pk, 0, 1, 8))), (ALIGNMENT, dict(os_=strides(pk, 0, 1024, 129))), (SHAPE, dict(os_=strides(pk, 0, 0, 128))),
                     (SHAPE, dict(os_=strides(pk, 0, 1024, 64)))] + [(INVALID, dict(sc=scores(pk, **b))) for b in BAD_SCORES]:
        assert prompt(pk, **kw) == want, kw


def test_binding_refuses(pk):
    """What the binding looks at before it calls the library."""
    cfg = pk.Kv16Config(**BASE)
    cache = pk.Kv16Cache(cfg, device="cpu")
    k, q, slots = torch.zeros(4, 2, 128, dtype=torch.float16), torch.zeros(2, 8, 128, dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
    for t in (k.float(), k[:, :1], k[..., :64], k.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            pk.pk_kv16_append(cfg, cache, t, t, slots)
    for bad in (slots[:3], slots.long(), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="slots"):
            pk.pk_kv16_append(cfg, cache, k, k, bad)
    with pytest.raises(ValueError):
        pk.pk_kv16_append(cfg, cache, k, k[:3], slots)
    with pytest.raises(ValueError, match="current device"):
        pk._stream_of(torch.device("cpu"))
    with pytest.raises(ValueError, match="another configuration"):
        pk.pk_kv16_append(pk.Kv16Config(**{**BASE, "n_pages": 201}), cache, k, k, slots)
    for kw in (dict(out=q[:, :4]), dict(out=q.float()), dict(slopes=torch.zeros(2)), dict(lse=torch.zeros(2, 8, 1)), dict(bound=1 << 31), dict(window=1 << 31),
               dict(workspace=torch.zeros(8))):
        with pytest.raises(ValueError):
            pk.pk_kv16_attention(cfg, cache, q, 1.0, **kw)
    with pytest.raises(ValueError):
        pk.pk_kv16_attention(cfg, cache, q[:1], 1.0)
    for kw in (dict(k=cache.k[:-1]), dict(v=cache.v.float()), dict(states=torch.zeros(2, 4)), dict(page_table=cache.page_table[:1]),
               dict(page_table=cache.page_table.long()), dict(states=cache.states.to("meta"))):
        with pytest.raises(ValueError):
            pk.Kv16Cache(cfg, device="cpu", **kw)
    pc = pk.PromptConfig(n_seq=2, n_kv_heads=2, n_q_heads=8)
    q, starts = torch.zeros(4, 8, 128, dtype=torch.float16), torch.zeros(3, dtype=torch.int32)
    for args, kw in (((q, k[:3], k, starts), {}), ((q, k, k.float(), starts), {}), ((q[:, :4], k, k, starts), {}), ((q, k, k, starts[:2]), {}),
                     ((q, k, k, starts.long()), {}), ((q, k, k, starts), dict(out=q[:3])), ((q, k, k, starts), dict(lse=torch.zeros(4, 8))),
                     ((q, k, k, starts), dict(slopes=torch.zeros(4))), ((q, k, k, starts), dict(window=1 << 40))):
        with pytest.raises(ValueError):
            pk.pk_prompt_attention(pc, *args, 1.0, **kw)
    gc = pk.PagesConfig(n_seq=4, page_tokens=16, n_pages=9, pages_per_seq=3)
    pool = pk.PagePool(gc, device="cpu")
    assert pool.free.tolist() == list(range(8, -1, -1)) and pool.n_free.tolist() == [9, 0, 0, 0]
    states, counts = torch.zeros(4, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for args, kw in (((states[:3], counts, 4), {}), ((states.long(), counts, 4), {}), ((states, counts[:3], 4), {}), ((states, counts, -1), {}), ((states, counts, 1 << 31), {}),
                     ((states, counts, 4), dict(states_out=counts)), ((states, counts, 4), dict(n_free_out=counts[:1])), ((states, counts, 4), dict(out=pk.pk_pages_plan(gc, 5, "cpu")))):
        with pytest.raises(ValueError):
            pk.pk_pages_update(gc, pool, *args, **kw)
    with pytest.raises(ValueError):
        pk.PagePool(gc, device="cpu", free=pool.free)
    with pytest.raises(ValueError):
        pk.PagePool(gc, device="cpu", table=pool.table[:, :2])
    plan = pk.pk_pages_plan(gc, 5, "cpu")
    parts = sorted((t.data_ptr(), t.numel() * 4) for t in (plan.starts, plan.slots, plan.positions, plan.taken))
    assert all(p % 16 == parts[0][0] % 16 for p, _ in parts) and all(a + n <= b for (a, n), (b, _) in zip(parts, parts[1:]))


@pytest.mark.parametrize("change", [dict(n_seq=0), dict(n_seq=65536), dict(page_tokens=24), dict(n_pages=0), dict(n_pages=1 << 27), dict(pages_per_seq=0)])
def test_binding_refuses_bad_pages(pk, change, monkeypatch):
    """A configuration that the library refuses makes no pool and no plan, as it makes no cache; a step with memory of the caller's comes to an error of the binding's own."""
    cfg = pk.PagesConfig(**{**dict(n_seq=4, page_tokens=16, n_pages=9, pages_per_seq=3), **change})
    monkeypatch.setattr(pk, "_stream_of", lambda device: None)
    n = cfg.n_seq
    states, counts, starts = (torch.zeros(shape, dtype=torch.int32) for shape in ((n, 4), n, n + 1))
    rows = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="not a configuration"):
        pk.pk_pages_update(cfg, pk.PagePool(cfg, device="cpu"), states, counts, 4, out=pk.PagesPlan(starts, rows, rows.clone(), counts.clone()))
    with pytest.raises(ValueError, match="not a configuration"):
        pk.pk_pages_plan(cfg, 4, "cpu")


def test_binding_passes_a_plan_without_positions(pk, monkeypatch):
    """The C call takes none; so does the binding, where the caller's plan has none."""
    cfg = pk.PagesConfig(n_seq=4, page_tokens=16, n_pages=9, pages_per_seq=3)
    calls = []

    class Lib:
        def pk_pages_update(self, *args):
            calls.append(args)
            return OK
    pool, states, counts, plan = pk.PagePool(cfg, device="cpu"), torch.zeros(4, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), pk.pk_pages_plan(cfg, 5, "cpu")
    plan.positions = None
    monkeypatch.setattr(pk, "_stream_of", lambda device: None)
    monkeypatch.setattr(pk, "_lib", Lib())
    assert pk.pk_pages_update(cfg, pool, states, counts, 5, out=plan) is plan
    assert calls[0][6:10] == (plan.starts.data_ptr(), plan.slots.data_ptr(), None, plan.taken.data_ptr())


def test_reference_pages_belong_to_one_sequence():
    rng = random.Random(5)
    for _ in range(40):
        n_seq, page, n_pages, per_seq = rng.randint(1, 6), rng.choice([1, 4, 16]), rng.randint(1, 40), rng.randint(1, 9)
        pool = ref.Pool(n_seq, page, n_pages, per_seq, rng.sample(range(n_pages), n_pages))
        for _ in range(6):
            counts = [rng.randint(-2 * page, 4 * page) for _ in range(n_seq)]
            n_tokens = max(sum(max(c, 0) for c in counts) + rng.randint(-3, 3), 0)
            starts, slots, positions, taken = pool.update(counts, n_tokens)
            used = sum(pool.pages, pool.free[:])
            assert sorted(used) == list(range(n_pages))
            live = [s for s in slots if s >= 0]
            assert len(set(live)) == len(live) == sum(taken) and starts[-1] <= n_tokens
            assert all(len(p) == -(-n // page) and len(p) <= per_seq for p, n in zip(pool.pages, pool.length))


def test_reference_attention_is_a_softmax():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 5, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    place = np.array([0, 2, 4, 8, 8])
    got, lse, mag, _, _ = ref.attention(q, k, v, place, 0.3, window=4)
    want = torch.from_numpy(q @ k.T * 0.3)
    back = torch.from_numpy(place)[:, None] - torch.arange(9)
    want = want.masked_fill((back < 0) | (back >= 4), -float("inf"))
    assert np.allclose(got, (want.softmax(-1) @ torch.from_numpy(v)).numpy()) and np.allclose(lse, want.logsumexp(-1).numpy())
    assert (np.abs(got) <= mag + 1e-15).all()


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_host_checks_under_asan_ubsan(tmp_path):
    """The host side with its launches replaced by stubs; the sanitizer flags go to the host pass only."""
    csrc, driver, exe = os.path.join(ROOT, "paper_2510_05176_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize", "kv16_api_driver.cpp"), str(tmp_path / "kv16_san")
    san = [x for f in ("-fsanitize=address,undefined", "-fno-sanitize-recover=undefined") for x in ("-Xarch_host", f)]
    cmd = [shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "-x", "hip", "-std=c++17", "--offload-arch=gfx950", "-O1", "-g", "-fno-omit-frame-pointer"] + san + [
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "pk_kv16_api.hip"), driver, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.returncode, r.stdout[-2000:], r.stderr[-4000:])
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
