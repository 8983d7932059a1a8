"""The 8-bit cache's entry points without a GPU: sizes, refusals (every one before a launch, so that fake pointers do), and the
64-bit reference that the GPU tests compare with against torch's own e4m3 type."""
import os
import shutil
import subprocess
import sys

import numpy as np
import pytest

import fp8_reference as ref

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2510_05176_amd", "libpatternkv.so")), reason="libpatternkv.so not built")

OK, INVALID, UNSUPPORTED, SHAPE, ALIGNMENT, CAPACITY, STATE, WORKSPACE = range(8)


@pytest.fixture(scope="module")
def pk():
    from paper_2510_05176_amd import patternkv
    return patternkv


BASE = dict(n_seq=2, n_kv_heads=2, n_q_heads=8, head_dim=128, block=64, t_capacity=1024)


def test_sizes(pk):
    lay = pk.pk_fp8_cache_layout(pk.Fp8Config(**BASE))
    assert lay["k_codes"] == lay["v_codes"] == 4 * 1024 * 128
    assert lay["k_scale"] == lay["v_scale"] == 4 * 16 * 4 and lay["pos"] == lay["weight"] == 4 * 1024 * 4
    assert lay["align"] == 16 and lay["total"] == sum(lay[n] for n in ("k_codes", "v_codes", "k_scale", "v_scale", "pos", "weight"))
    paged = pk.pk_fp8_cache_layout(pk.Fp8Config(**BASE, page_tokens=128, n_pages=40))
    assert paged["k_codes"] == 40 * 2 * 128 * 128 and paged["k_scale"] == 40 * 2 * 2 * 4 and paged["pos"] == lay["pos"]
    cfg = pk.Fp8Config(**BASE)
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_EVICT, 100) >= 4 * 100 * 4
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_EVICT, 1024) == 0 and pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_ATTENTION, -1, 5) == 0
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_ATTENTION, 1, 0) == 0 and pk.pk_fp8_workspace_bytes(cfg, 7, 1, 1) == 0
    last = 0
    for bound in range(0, 1025, 64):   # a longer cache never needs less
        need = pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_ATTENTION, 1, bound)
        assert need >= last
        last = need


@pytest.mark.parametrize("field,value,status", [
    ("head_dim", 80, UNSUPPORTED), ("head_dim", 512, UNSUPPORTED), ("block", 16, UNSUPPORTED), ("block", 0, UNSUPPORTED), ("n_q_heads", 7, SHAPE),
    ("n_q_heads", 130, UNSUPPORTED), ("t_capacity", 1000, SHAPE), ("t_capacity", 0, INVALID), ("t_capacity", 1 << 26, UNSUPPORTED),
    ("dtype", 2, INVALID), ("n_seq", 0, INVALID), ("n_seq", 40000, UNSUPPORTED), ("page_tokens", 64, UNSUPPORTED), ("page_tokens", 192, UNSUPPORTED),
    ("page_tokens", 2048, SHAPE), ("page_tokens", 128, INVALID), ("page_tokens", -1, INVALID)])
def test_bad_configurations(pk, field, value, status):
    kw = dict(BASE)
    kw[field] = value
    cfg = pk.Fp8Config(**kw)
    with pytest.raises(pk.PkError) as e:
        pk.pk_fp8_cache_layout(cfg)
    assert e.value.status == status
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_ATTENTION, 1, 64) == 0


P = 0x10000000   # never dereferenced


def cache_of(pk, at=P, **change):
    """fake arrays, far enough apart for the sizes of BASE"""
    a = dict(k_codes=at, v_codes=at + 0x100000, k_scale=at + 0x200000, v_scale=at + 0x300000, pos=at + 0x400000, weight=at + 0x500000, page_table=0)
    a.update(change)
    return pk._pack_fp8_cache(*a.values())


def strides(pk, *s):
    return pk._pack_strides(*(s or (8192, 256, 128)))


def append(pk, cfg=None, cache=None, states=P, out=0, k=P, v=P, ks=None, vs=None, n=4, counts=0):
    return pk._lib.pk_fp8_append(cfg or pk.Fp8Config(**BASE).packed, cache or cache_of(pk), states, out, k, v, ks or strides(pk), vs or strides(pk), n, counts, None)


def attention(pk, cfg=None, cache=None, states=P, bound=1024, q=P, qs=None, n=1, counts=0, scores=None, out=P, os_=None, lse=0, ws=P, size=1 << 40):
    return pk._lib.pk_fp8_attention(cfg or pk.Fp8Config(**BASE).packed, cache or cache_of(pk), states, bound, q, qs or strides(pk), n, counts,
                                    scores or pk._pack_fp8_scores(1.0, 0.0, 0, 0), out, os_ or strides(pk), lse, ws, size, None)


def weights(pk, cache=None, states=P, bound=1024, q=P, n=1, lse=P, scores=None, add=1):
    return pk._lib.pk_fp8_weights(pk.Fp8Config(**BASE).packed, cache or cache_of(pk), states, bound, q, strides(pk), n, 0,
                                  scores or pk._pack_fp8_scores(1.0, 0.0, 0, 0), lse, add, None)


def evict(pk, cfg=None, cache=None, states=P + 0x600000, to_cfg=None, to=None, to_states=P + 0x700000, budget=128, first=4, last=32, ws=P, size=1 << 40):
    return pk._lib.pk_fp8_evict(cfg or pk.Fp8Config(**BASE).packed, cache or cache_of(pk), states, to_cfg or pk.Fp8Config(**BASE).packed,
                                to or cache_of(pk, 0x40000000), to_states, budget, first, last, ws, size, None)


def test_append_refuses(pk):
    paged = pk.Fp8Config(**BASE, page_tokens=128, n_pages=16).packed
    wide = pk.Fp8Config(n_seq=1, n_kv_heads=65535, n_q_heads=65535, block=32, t_capacity=1 << 25).packed
    assert append(pk, n=0) == OK                                     # nothing to do, nothing launched
    for want, kw in [(INVALID, dict(cache=cache_of(pk, k_codes=0))), (INVALID, dict(cache=cache_of(pk, pos=0))), (INVALID, dict(states=0)),
                     (INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(n=-1)), (INVALID, dict(out=P + 16)), (INVALID, dict(cfg=paged)),
                     (ALIGNMENT, dict(cache=cache_of(pk, v_codes=P + 8))), (ALIGNMENT, dict(cache=cache_of(pk, weight=P + 4))),
                     (ALIGNMENT, dict(cfg=paged, cache=cache_of(pk, page_table=P + 4))), (ALIGNMENT, dict(states=P + 4)), (ALIGNMENT, dict(k=P + 2)),
                     (ALIGNMENT, dict(counts=P + 4)), (ALIGNMENT, dict(ks=strides(pk, 8192, 4, 128))), (ALIGNMENT, dict(vs=strides(pk, 8192, 256, 130))),
                     (CAPACITY, dict(n=1025)), (UNSUPPORTED, dict(cfg=wide, n=1 << 25))]:
        assert append(pk, **kw) == want, kw


def test_attention_and_weights_refuse(pk):
    bad = pk._pack_fp8_scores
    long = pk.Fp8Config(**{**BASE, "t_capacity": 8192}).packed   # split over workgroups, so that there is something to merge
    wide = pk.Fp8Config(n_seq=1, n_kv_heads=1, n_q_heads=64, t_capacity=1 << 25).packed
    assert attention(pk, n=0) == OK and attention(pk, n=0, q=0, out=0) == OK
    for want, kw in [(INVALID, dict(states=0)), (INVALID, dict(q=0)), (INVALID, dict(out=0)), (INVALID, dict(n=-1)), (INVALID, dict(bound=-1)),
                     (INVALID, dict(scores=bad(1.0, -1.0, 0, 0))), (INVALID, dict(scores=bad(1.0, float("nan"), 0, 0))),
                     (INVALID, dict(scores=bad(1.0, 0.0, -1, 0))), (INVALID, dict(scores=bad(float("nan"), 0.0, 0, 0))), (INVALID, dict(scores=bad(float("-inf"), 0.0, 0, 0))),
                     (UNSUPPORTED, dict(cfg=wide, bound=64, n=(1 << 22) + 1)), (INVALID, dict(scores=bad(1.0, float("inf"), 0, 0))), (INVALID, dict(scores=bad(1.0, 1e-38, 0, 0))),
                     (SHAPE, dict(os_=strides(pk, 0, 256, 128))), (SHAPE, dict(os_=strides(pk, 8192, 256, 0))), (SHAPE, dict(n=2, os_=strides(pk, 8192, 0, 128))),
                     (ALIGNMENT, dict(scores=bad(1.0, 0.0, 0, P + 4))), (ALIGNMENT, dict(q=P + 8)),
                     (ALIGNMENT, dict(out=P + 8)), (ALIGNMENT, dict(lse=P + 4)), (ALIGNMENT, dict(ws=P + 4)), (ALIGNMENT, dict(qs=strides(pk, 8, 9, 8))),
                     (ALIGNMENT, dict(os_=strides(pk, 8, 8, 12))), (CAPACITY, dict(bound=1025)), (CAPACITY, dict(n=1025)),
                     (WORKSPACE, dict(cfg=long, bound=8192, ws=0)), (WORKSPACE, dict(cfg=long, bound=8192, size=255))]:
        assert attention(pk, **kw) == want, kw
    assert weights(pk, n=0) == OK and weights(pk, n=0, q=0, lse=0) == OK
    for want, kw in [(INVALID, dict(lse=0)), (INVALID, dict(cache=cache_of(pk, weight=0))), (INVALID, dict(q=0)), (ALIGNMENT, dict(lse=P + 8)),
                     (CAPACITY, dict(bound=2000)), (INVALID, dict(scores=bad(1.0, 0.0, -5, 0)))]:
        assert weights(pk, **kw) == want, kw


def test_evict_refuses(pk):
    other = dict(BASE)
    for want, kw in [(INVALID, dict(budget=0)), (INVALID, dict(first=-1)), (INVALID, dict(last=-1)), (INVALID, dict(states=0)), (INVALID, dict(to_states=0)),
                     (INVALID, dict(cache=cache_of(pk, weight=0))), (INVALID, dict(to=cache_of(pk))), (INVALID, dict(to=cache_of(pk, 0x40000000, pos=P + 0x1000))),
                     (INVALID, dict(to_states=P + 0x600010)), (SHAPE, dict(first=100, last=29)), (CAPACITY, dict(budget=1025)),
                     (SHAPE, dict(to_cfg=pk.Fp8Config(**{**other, "block": 32}).packed)), (SHAPE, dict(to_cfg=pk.Fp8Config(**{**other, "head_dim": 64}).packed)),
                     (SHAPE, dict(to_cfg=pk.Fp8Config(**{**other, "n_seq": 1}).packed)), (ALIGNMENT, dict(to_states=P + 0x700004)),
                     (WORKSPACE, dict(ws=0)), (WORKSPACE, dict(size=4 * 128 * 4 - 1))]:
        assert evict(pk, **kw) == want, kw


def test_binding_refuses(pk):
    """What the binding looks at before it calls the library."""
    cfg = pk.Fp8Config(**BASE)
    cache = pk.Fp8Cache(cfg, device="cpu")
    k = torch.zeros(2, 2, 4, 128, dtype=torch.float16)
    q = torch.zeros(2, 8, 1, 128, dtype=torch.float16)
    for t in (k.float(), k[:1], k[:, :1], k[..., :64], k.transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(ValueError):
            pk.pk_fp8_append(cfg, cache, t, t)
    with pytest.raises(ValueError):
        pk.pk_fp8_append(cfg, cache, k, k[:, :, :3])
    with pytest.raises(ValueError):
        pk.pk_fp8_append(cfg, cache, k, k, states_out=torch.zeros(2, 4))
    with pytest.raises(ValueError):
        pk.pk_fp8_attention(cfg, cache, q, 1.0, counts=None, out=q[:, :4])
    with pytest.raises(ValueError):
        pk.pk_fp8_attention(cfg, cache, q, 1.0, counts=torch.zeros(2))
    with pytest.raises(ValueError):
        pk.pk_fp8_attention(cfg, cache, q, 1.0, slopes=torch.zeros(2))
    with pytest.raises(ValueError):
        pk.pk_fp8_weights(cfg, cache, q, torch.zeros(2, 8), 1.0)
    with pytest.raises(ValueError):
        pk._fp8_stream(pk.Fp8Config(**{**BASE, "t_capacity": 2048}), cache)     # another configuration's cache
    with pytest.raises(ValueError):
        pk._fp8_stream(cfg, cache)                                              # not on the current device
    with pytest.raises(AssertionError):
        pk.Fp8Cache(cfg, device="cpu", arrays={**cache.buf, "pos": cache.buf["pos"][:-1]})
    with pytest.raises(AssertionError):
        pk.Fp8Cache(cfg, device="cpu", states=torch.zeros(2, 4))


def test_workspace_size_while_another_thread_forgets_it(pk):
    """The sizes that a configuration remembers may be cleared by another thread at any point."""
    class Racing(dict):
        def __contains__(self, key):
            there = dict.__contains__(self, key)
            self.clear()
            return there

        def __len__(self):
            return 1 << 20

        def __setitem__(self, key, value):
            pass

    cfg = pk.Fp8Config(**BASE)
    need = pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_EVICT, 100)
    racing = Racing({(pk.FP8_OP_EVICT, 100, 0): need})
    object.__setattr__(cfg, "_workspaces", racing)
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_EVICT, 100) == need
    racing.clear()
    assert pk.pk_fp8_workspace_bytes(cfg, pk.FP8_OP_EVICT, 100) == need


def test_cache_is_checked_under_optimization():
    """`python -O` drops assert statements, and a cache whose arrays are too small is written out of bounds: its checks are none."""
    code = """
import torch
from paper_2510_05176_amd import patternkv as pk
cfg = pk.Fp8Config(n_seq=2, n_kv_heads=2, n_q_heads=8, t_capacity=1024)
paged = pk.Fp8Config(n_seq=2, n_kv_heads=2, n_q_heads=8, t_capacity=1024, page_tokens=128, n_pages=16)
good = pk.Fp8Cache(cfg, device="cpu")
table = pk.Fp8Cache(paged, device="cpu").page_table
bad = [(cfg, dict(arrays={**good.buf, "pos": good.buf["pos"][:-1]})), (cfg, dict(arrays={k: v for k, v in good.buf.items() if k != "k_scale"})),
       (cfg, dict(arrays={**good.buf, "weight": good.buf["weight"].double()})), (cfg, dict(states=torch.zeros(2, 4))),
       (cfg, dict(states=torch.zeros(2, 8, dtype=torch.int32)[:, ::2])), (paged, dict(page_table=table[:1])), (paged, dict(page_table=table.long())),
       (cfg, dict(states=good.states.to("meta")))]
for c, kw in bad:
    try:
        pk.Fp8Cache(c, device="cpu", **kw)
    except AssertionError:
        continue
    raise SystemExit(str(list(kw)))
print("ok", __debug__)
"""
    for flag, debug in (("-O", "False"), ("-B", "True")):
        r = subprocess.run([sys.executable, flag, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
        assert r.returncode == 0 and r.stdout.split() == ["ok", debug], (flag, r.stdout, r.stderr[-2000:])


def test_evict_refuses_numbers_of_more_than_32_bits(pk):
    """ctypes would cut them off: 2^32 + 64 tokens to 64."""
    cfg = pk.Fp8Config(**BASE)
    a, b = pk.Fp8Cache(cfg, device="cpu"), pk.Fp8Cache(cfg, device="cpu")
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for name in ("budget", "keep_first", "keep_last"):
        for value in ((1 << 32) + 64, 1 << 31, -(1 << 32)):
            with pytest.raises(ValueError, match=name):
                pk.pk_fp8_evict(cfg, a, cfg, b, **{"budget": 64, name: value}, workspace=ws)
    for kw in (dict(bound=(1 << 32) + 64), dict(window=1 << 31)):
        q = torch.zeros(2, 8, 1, 128, dtype=torch.float16)
        with pytest.raises(ValueError, match=list(kw)[0]):
            pk.pk_fp8_attention(cfg, a, q, 1.0, **kw)
        with pytest.raises(ValueError, match=list(kw)[0]):
            pk.pk_fp8_weights(cfg, a, q, torch.zeros(2, 8, 1), 1.0, **kw)


def test_attention_refuses_rows_of_the_output_within_each_other(pk):
    """Strides of the output shorter than a vector, where there is more than one: whichever row is written last would win."""
    for s, n in (((8192, 256, 64), 1), ((8192, 120, 2048), 2), ((64, 1024, 128), 1), ((-64, 1024, 128), 1), ((8192, 1024, -120), 1)):
        assert attention(pk, n=n, os_=strides(pk, *s)) == SHAPE, (s, n)


def test_reference_codes_are_e4m3():
    x = torch.arange(256, dtype=torch.uint8)
    got = x.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref.VALUES)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(ref.VALUES))
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 6, 20000), (ref.GRID[1:] + ref.GRID[:-1]) / 2, [0.0, -0.0, 448.0]])
    y = np.float32(y).astype(np.float64)
    y = y[np.abs(y) <= 448]
    want = torch.from_numpy(np.float32(y)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.nearest_codes(y), want)


def test_reference_exponents():
    for top, e in [(448.0, 0), (448.25, 1), (447.0, 0), (224.0, -1), (224.5, 0), (0.0, -126), (1.0, -8), (65504.0, 8), (2.0 ** -140, -126)]:
        assert ref.block_exponent(np.array([0.0, -top, np.inf, np.nan])) == e, top


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_host_checks_under_asan_ubsan(tmp_path):
    """The host side with its launches replaced by stubs; the sanitizer flags go to the host pass only."""
    csrc, driver, exe = os.path.join(ROOT, "paper_2510_05176_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize", "fp8_api_driver.cpp"), str(tmp_path / "fp8_san")
    san = [x for f in ("-fsanitize=address,undefined", "-fno-sanitize-recover=undefined") for x in ("-Xarch_host", f)]
    cmd = [shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "-x", "hip", "-std=c++17", "--offload-arch=gfx950", "-O1", "-g", "-fno-omit-frame-pointer"] + san + [
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "pk_fp8_api.hip"), driver, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.returncode, r.stdout[-2000:], r.stderr[-4000:])
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
