"""Operators of a layer in 8 bits, what needs no GPU: sizes, refusals, the frequencies of a rotary plan, and the oracle against itself."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import layer8 as O


@pytest.fixture(scope="module")
def P():
    import paper_2408_15766_amd as pkg
    return pkg


def test_oracle_rounds_to_the_grid_of_e4m3():
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    grid = np.unique(codes[np.isfinite(codes)])
    assert np.array_equal(O.e4m3(grid), grid) and grid.max() == 448
    mid = (grid[1:] + grid[:-1]) / 2
    for x in (mid, mid * (1 + 1e-12), mid * (1 - 1e-12)):
        want = np.array([min(grid, key=lambda g: abs(g - v)) for v in x])
        near = np.abs(x - O.e4m3(x))
        assert np.all(near <= np.abs(x - want) * (1 + 1e-9) + 1e-300)
    assert np.array_equal(O.e4m3(mid), torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy())   # ties to even
    assert np.isnan(O.e4m3(np.array([np.inf, -np.inf, np.nan]))).all()


def test_oracle_exponent_is_the_least():
    for amax in (448.0, 449.0, 1.0, 3.5, 3.5000001, 1e-30, 1e30, 2.0 ** -92 * 1.75, 0.0):
        e = O.exponent(np.array([amax, np.nan, -np.inf]))
        assert amax <= 448 * 2.0 ** e and (e == -100 or amax > 448 * 2.0 ** (e - 1))


def test_sizes(P):
    assert P.spec_packed8_bytes(1, 1) >= 2048 + 64 and P.spec_packed8_bytes(0, 5) == 0 and P.spec_packed8_bytes(5, -1) == 0
    assert P.spec_packed8_bytes(4096, 4096) == 4096 * 4096 + 256 * 8 * 64
    assert P.spec_packed8_bytes(128256, 32768) == 128256 * 32768 + 8016 * 64 * 64   # (over 2^31)
    assert P.spec_k_gemm8_scratch_bytes(0, 128, 16) == 0 and P.spec_k_gemm8_scratch_bytes((1 << 20) + 1, 128, 16) == 0
    assert P.spec_kv8_bytes(1, 8, 128) % 256 == 0 and P.spec_kv8_bytes(3, 8, 128) == 3 * P.spec_kv8_bytes(1, 8, 128)
    assert P.spec_kv8_bytes(1, 8, 96) == 0 and P.spec_kv8_bytes(1, 129, 64) == 0 and P.spec_kv8_bytes(0, 8, 64) == 0
    assert P.spec_kv8_bytes(100000, 32, 128) > 1 << 35
    for bad in ((0, 8, 8, 64, 1, 1), (1, 12, 4, 64, 1, 1), (1, 8, 8, 64, -1, 1), (1, 8, 8, 64, 1, 0), (1, 7, 2, 64, 1, 1), (1, 8, 8, 80, 1, 1)):
        assert P.spec_k_attention8_scratch_bytes(*bad) == 0
    assert P.spec_k_attention8_scratch_bytes(60, 32, 8, 128, 64, 100) > 0 and P.spec_k_attention8_scratch_bytes(1, 32, 8, 128, 4, 40) == 0


X = 4096   # an address that is aligned and never read: every call below is refused first


def refused(rc):
    assert rc == -1


def test_gemm8_refusals(P):
    f = P.lib.spec_k_gemm8
    good = dict(dtype=1, x=X, ldx=256, m=40, k=256, w8=2 * X, rows=32, out=1, y=3 * X, ldy=32, scratch=4 * X, nbytes=1 << 30)
    for kw in (dict(dtype=2), dict(x=None), dict(ldx=255), dict(m=0), dict(m=-1), dict(m=(1 << 20) + 1), dict(k=0), dict(k=(1 << 20) + 1, ldx=1 << 21),
               dict(w8=None), dict(w8=X + 128), dict(rows=0), dict(out=3), dict(y=None), dict(y=X + 1), dict(x=X + 1), dict(ldy=31), dict(scratch=None),
               dict(scratch=X + 16), dict(nbytes=10), dict(y=X), dict(y=2 * X), dict(y=4 * X)):
        a = {**good, **kw}
        refused(f(a["dtype"], a["x"], a["ldx"], a["m"], a["k"], a["w8"], a["rows"], a["out"], a["y"], a["ldy"], a["scratch"], a["nbytes"], None))
    g = P.lib.spec_pack_weight8
    for a in ((2, X, 4, 4, X), (1, None, 4, 4, X), (1, X, 0, 4, X), (1, X, 4, 0, X), (1, X, 4, 4, X + 16), (0, X + 2, 4, 4, X), (1, X, 4, 4, None)):
        refused(g(*a, None))


def test_kv8_refusals(P):
    good = dict(k=2 * X, v=3 * X, ld=512, n=1, hkv=8, hd=64, c=X, first=0)
    for kw in (dict(k=None), dict(v=None), dict(ld=511), dict(n=-1), dict(hkv=0), dict(hkv=129, ld=1 << 20), dict(hd=32), dict(c=None), dict(c=X + 16),
               dict(first=-1), dict(first=1 << 24), dict(k=X + 1)):
        a = {**good, **kw}
        refused(P.lib.spec_k_kv8_store(a["k"], a["v"], a["ld"], a["n"], a["hkv"], a["hd"], a["c"], a["first"], None))
        refused(P.lib.spec_k_kv8_load(a["c"], a["first"], a["n"], a["hkv"], a["hd"], a["k"], a["v"], a["ld"], None))
    refused(P.lib.spec_k_kv8_load(X, 0, 1, 8, 64, 2 * X, 2 * X, 512, None))


def test_attention8_refusals(P):
    good = dict(q=X, c=2 * X, nb=20, kw=3 * X, vw=4 * X, win=8, rows=4, hq=8, hkv=2, hd=64, base=1280, depth=X, anc=X, md=3, scratch=5 * X, nbytes=1 << 40, out=6 * X)
    for kw in (dict(q=None), dict(q=X + 4), dict(c=None), dict(c=X + 16), dict(nb=-1), dict(kw=None), dict(vw=None), dict(kw=X + 2), dict(win=0), dict(win=2 ** 31 - 1), dict(rows=0),
               dict(hq=9), dict(hq=32), dict(hq=1), dict(hkv=0), dict(hd=80), dict(base=1279), dict(base=-1, nb=0), dict(depth=None), dict(md=-1), dict(md=16),
               dict(anc=None, md=2 ** 31 - 1), dict(scratch=None), dict(scratch=X + 64), dict(nbytes=0), dict(out=None), dict(out=X + 2), dict(anc=X + 1),
               dict(out=X), dict(out=2 * X), dict(out=3 * X), dict(out=4 * X), dict(out=5 * X)):
        a = {**good, **kw}
        refused(P.lib.spec_k_attention8(a["q"], a["c"], a["nb"], a["kw"], a["vw"], a["win"], a["rows"], a["hq"], a["hkv"], a["hd"], a["base"], a["depth"],
                                        a["anc"], a["md"], a["scratch"], a["nbytes"], a["out"], None))


@pytest.mark.parametrize("rot,theta,kw", [
    (128, 1e4, {}), (2, 10.0, {}), (64, 5e5, dict(scaling="linear", factor=8.0)),
    (128, 5e5, dict(scaling="llama3", factor=8.0, trained_len=8192, low_freq=1.0, high_freq=4.0)),
    (128, 1e4, dict(scaling="yarn", factor=16.0, trained_len=4096)), (32, 1e4, dict(scaling="yarn", factor=2.5, trained_len=512, beta_fast=20.0, beta_slow=2.0)),
    (6, 1e4, dict(scaling="yarn", factor=4.0, trained_len=1)), (0, 1e4, {})])
def test_rotary_plan_has_the_frequencies(P, rot, theta, kw):
    plan = P.spec_rotary_plan(rot, theta, layout="interleaved", **kw)
    f, m = O.rope_frequencies(rot, theta, **kw) if rot else (np.zeros(0), 1.0)
    got = np.array(plan.freq[:rot // 2])
    assert plan.rot == rot and plan.layout == 1 and np.allclose(got, f, rtol=1e-14, atol=0) and math.isclose(plan.mscale, m, rel_tol=1e-15)
    assert all(x == 0.0 for x in plan.freq[rot // 2:])


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=258), dict(rot=-2), dict(theta=1.0), dict(theta=float("nan")), dict(layout="third"), dict(scaling="more"),
                                dict(scaling="linear", factor=0.5), dict(scaling="llama3", factor=8.0), dict(scaling="llama3", factor=8.0, trained_len=8192, high_freq=1.0),
                                dict(scaling="yarn", factor=float("inf"), trained_len=4096), dict(scaling="yarn", factor=2.0, trained_len=4096, beta_slow=0.0)])
def test_rotary_plan_refusals(P, kw):
    with pytest.raises(P.SpecError) as e:
        P.spec_rotary_plan(**{**dict(rot=64, theta=1e4), **kw})
    assert e.value.code == -1


def test_rotary_refusals(P):
    b = P.binding
    plan = P.spec_rotary_plan(64, 1e4)

    def call(hd=64, rows=4, n=1, pos=X, plan=plan, **kw):
        p = {**dict(x=X, out=X, ldx=256, hsx=64, ldo=256, hso=64, heads=4, dtype=1, out_dtype=1, turn=1), **kw}
        return P.lib.spec_k_rotary(plan and C.byref(plan), n, bytes((b.spec_rotary_part * 3)(b.spec_rotary_part(**p))), hd, rows, pos, 0, 0, None)

    for kw in (dict(hd=0), dict(hd=62), dict(hd=257), dict(rows=0), dict(rows=(1 << 24) + 1), dict(n=0), dict(n=4), dict(n=2), dict(pos=X + 2), dict(plan=None),
               dict(x=None), dict(out=None), dict(x=X + 1, out=X + 1), dict(ldx=63), dict(ldo=10), dict(hsx=63), dict(hso=0), dict(heads=0), dict(heads=1025),
               dict(dtype=5), dict(out_dtype=-1), dict(ldx=-256), dict(out_dtype=0), dict(ldo=512)):
        assert call(**kw) == -1, kw
    part = dict(ldx=256, hsx=64, ldo=256, hso=64, heads=4, dtype=1, out_dtype=1, turn=1)
    for x, out, x2, out2 in ((X, X, X, X), (X, 2 * X, 3 * X, 2 * X), (X, 2 * X, 2 * X, 3 * X), (X, 2 * X, 3 * X, X)):   # one tensor written twice, or read and written
        two = bytes((b.spec_rotary_part * 2)(b.spec_rotary_part(x=x, out=out, **part), b.spec_rotary_part(x=x2, out=out2, **part)))
        assert P.lib.spec_k_rotary(C.byref(plan), 2, two, 64, 4, X, 0, 0, None) == -1
    odd = b.spec_rotary_plan_t(63, 0, 1.0)
    assert call(plan=odd) == -1
    odd = b.spec_rotary_plan_t(64, 7, 1.0)
    assert call(plan=odd) == -1


def test_binding_refuses_host_tensors(P):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("host-only check")
    w = torch.zeros(4, 128)
    for call in (lambda: P.spec_pack_weight8(w), lambda: P.spec_k_rotary(P.spec_rotary_plan(64, 1e4), [torch.zeros(2, 1, 64)], 0),
                 lambda: P.spec_k_kv8_load(torch.zeros(1, 16640, dtype=torch.uint8), 0, 1, 1, 128)):
        with pytest.raises(P.SpecError):
            call()


def test_attention8_plan(P):
    """Ranges are at most as many as the blocks; sizes that a call refuses are refused."""
    for a in ((1, 8, 8, 128, 4, 40), (60, 64, 8, 128, 512, 60), (1024, 32, 8, 64, 128, 1024), (2, 2, 1, 64, 0, 5000)):
        waves, query_blocks, block_parts, win_parts = P.spec_k_attention8_plan(*a)
        assert waves in (0, 2, 4, 8) and query_blocks == -(-a[0] * a[1] // a[2] // (32 * max(waves, 1))) and block_parts <= a[4] and block_parts + win_parts >= 1
    for a in ((0, 8, 8, 64, 1, 1), (1, 12, 4, 64, 1, 1), (1, 8, 8, 64, 1, 0)):
        with pytest.raises(P.SpecError):
            P.spec_k_attention8_plan(*a)
    assert P.lib.spec_k_attention8_plan(1, 8, 8, 64, 1, 1, None, None, None, None) == -1


@pytest.mark.parametrize("rows,hq,hkv,hd,blocks,win", [(3, 1, 1, 128, 1000, 5), (1, 1, 1, 64, 1000, 1), (33, 1, 1, 64, 500, 40), (2, 1, 1, 128, 1000, 5), (5, 3, 3, 128, 700, 9)])
def test_attention8_scratch_keeps_its_parts_aligned(P, rows, hq, hkv, hd, blocks, win):
    """Every part is statistics (two floats a query) and outputs, both beginning at multiples of 16 bytes, for odd numbers of queries too."""
    _, _, block_parts, win_parts = P.spec_k_attention8_plan(rows, hq, hkv, hd, blocks, win)
    of_part = -(-8 * rows * hq // 16) * 16 + 4 * rows * hq * hd
    assert block_parts + win_parts > 32
    assert P.spec_k_attention8_scratch_bytes(rows, hq, hkv, hd, blocks, win) == -(-(block_parts + win_parts) * of_part // 256) * 256


def test_sizes_beyond_32_bits_are_no_sizes(P):
    """2^32 + n is not n."""
    far = 2 ** 32
    assert P.spec_packed8_bytes(far + 16, 1) == P.spec_packed8_bytes(16, far + 128) == P.spec_packed8_bytes(16, -far + 128) == 0
    assert P.spec_k_gemm8_scratch_bytes(far + 40, 128, 16) == P.spec_k_gemm8_scratch_bytes(40, far + 128, 16) == P.spec_k_gemm8_scratch_bytes(40, 128, far + 16) == 0
    assert P.spec_kv8_bytes(far + 1, 8, 128) == P.spec_kv8_bytes(1, far + 8, 128) == P.spec_kv8_bytes(1, 8, far + 128) == 0
    good = (60, 32, 8, 128, 64, 100)
    for i in range(6):
        a = tuple(n + far * (j == i) for j, n in enumerate(good))
        assert P.spec_k_attention8_scratch_bytes(*a) == 0
        with pytest.raises(P.SpecError):
            P.spec_k_attention8_plan(*a)
    for kw in (dict(rot=far + 64), dict(rot=64 - far), dict(rot=64, scaling="yarn", factor=4.0, trained_len=far + 4096)):
        with pytest.raises(P.SpecError):
            P.spec_rotary_plan(**{**dict(theta=1e4), **kw})
    for kw in (dict(hkv=far + 8, hd=128), dict(hkv=8, hd=far + 128)):
        with pytest.raises(P.SpecError):
            P.spec_kv8_alloc(1, **kw, device="cpu")
