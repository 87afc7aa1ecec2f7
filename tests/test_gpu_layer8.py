"""Operators of a layer in 8 bits on the GPU, against their definitions in 64 bits (oracle/layer8.py).

Tolerances.  u32 = 2^-24, u16 = 2^-8 (bf16), h = 2^-11 (fp16): the largest relative error of a rounding.
* gemm8, fp32 results: products are exact, a sum of n terms is off by at most n u32 sum|x w|.
* gemm8, bf16 results: in addition u16 of the result, and what the 8-bit matrix instruction drops: products of 128 k are lined up 2^-13 below
  the largest, so that those from 2^-6 of it on are exact (a product has 8 bits) and smaller ones lose at most that step (one more bit allowed here).
* attention8: u16 of the result; queries in fp16 move a score by at most d = h sum|q k| / sqrt(hd) + 2^-24 max|q| sum|k| / sqrt(hd) (elements below
  fp16's normal range beside the row's largest), weights by e^(2 d) - 1 in all, and weights in fp16 by at most 2 h (cut off and centred; rounded: h);
  2^-17 + 1e-6 for the window's and fp32 arithmetic.
* kv8: exact.  rotary: angles below 2^-22 off, so 2^-21 mscale (|a| + |b|), and the output's rounding.
"""
import math

import numpy as np
import pytest

from oracle import layer8 as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U32, U16, H = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def P():
    import paper_2408_15766_amd as pkg
    assert torch.cuda.is_available()
    return pkg


def rand(seed, *shape, scale=1.0):
    return torch.from_numpy((np.random.default_rng(seed).standard_normal(shape) * scale).astype(np.float32))


def f64(t):
    return t.detach().double().cpu().numpy()


# ---- gemm8 --------------------------------------------------------------------------------------

def gemm_bound(xq, wq, bf16):
    """(exact result, largest error allowed)"""
    y = xq @ wq.T
    tol = (xq.shape[1] + 8) * U32 * (np.abs(xq) @ np.abs(wq).T)
    if bf16:
        for c in range(0, xq.shape[1], 128):
            p = np.abs(xq[:, None, c:c + 128] * wq[None, :, c:c + 128])
            top = p.max(2, keepdims=True)
            tol += np.where(p < top * 2.0 ** -5, np.minimum(p, top * 2.0 ** -12), 0.0).sum(2)
        tol += U16 * (np.abs(y) + tol)
    return y, tol + 1e-37


def check_gemm(P, x, w, kind, **kw):
    xq, wq = O.held_rows(f64(x)), O.held_rows(f64(w))
    want, tol = gemm_bound(xq, wq, kind == torch.bfloat16)
    y = P.spec_k_gemm8(x, P.spec_pack_weight8(w), out_dtype=kind, **kw)
    assert y.dtype == kind and tuple(y.shape) == want.shape
    bad = ~(np.abs(f64(y) - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], f64(y)[bad][:5], want[bad][:5], tol[bad][:5])
    return y


SIZES = [(1, 1, 1), (1, 128, 16), (1, 4096, 48), (2, 130, 33), (7, 256, 100), (16, 640, 31), (17, 513, 70), (33, 1000, 65), (64, 384, 129), (65, 96, 200),
         (128, 260, 300), (129, 129, 257), (200, 1024, 520), (333, 250, 150), (520, 128, 600)]


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("m,k,rows", SIZES)
def test_gemm8_sizes(P, m, k, rows, dtype, out):
    gain = torch.exp(rand(3, k))
    x = (rand(m * 7 + k, m, k) * gain).to(DT[dtype]).cuda()
    w = rand(rows, rows, k, scale=0.02).to(DT[dtype]).cuda()
    check_gemm(P, x, w, DT[out])


def held_gpu(x):
    """O.held_rows on the device, in float64."""
    r, k = x.shape
    y = torch.nn.functional.pad(x.double(), (0, -k % 128)).view(r, -1, 128)
    m, e = torch.frexp(y.abs().amax(2, keepdim=True) / 448)
    e = torch.where(m > 0, torch.where(m > 0.5, e, e - 1), -100).clamp(min=-100).double()
    t = y * torch.exp2(-e)
    step = torch.exp2((torch.frexp(t)[1] - 1).clamp(min=-6).double() - 3)
    return torch.round(t / step) * step * torch.exp2(e)


@pytest.mark.parametrize("m,k,rows", [(40, 300, 20001), (64, 700, 12290), (300, 130, 12000), (90, 256, 20480), (2047, 130, 28671), (2048, 384, 12288), (2000, 129, 12289),
                                      (1024, 200, 4100), (600, 512, 4097), (513, 256, 28600), (4096, 256, 4096), (200, 600, 3000)])
def test_gemm8_launches_of_many_tiles(P, m, k, rows):
    """Every shape of tile, whole and ragged, and launches in two parts.  (The 8-bit instruction's loss is bounded by 128 times 2^-12 of the largest product of a block.)"""
    g = torch.Generator(device="cuda").manual_seed(m + rows)
    x, w = (torch.randn(n, k, generator=g, device="cuda") for n in (m, rows))
    assert np.array_equal(f64(held_gpu(x[:5])).reshape(5, -1)[:, :k], O.held_rows(f64(x[:5])))
    xq, wq = held_gpu(x), held_gpu(w)
    ref, size = xq.flatten(1) @ wq.flatten(1).t(), xq.flatten(1).abs() @ wq.flatten(1).abs().t()
    lost = 2.0 ** -5 * (xq.abs().amax(2) @ wq.abs().amax(2).t())
    w8 = P.spec_pack_weight8(w)
    tol = (k + 8) * U32 * size
    for out, bound in ((torch.float32, tol), (torch.bfloat16, tol + lost + U16 * (ref.abs() + tol + lost))):
        wide = torch.full((m, rows + 3), 7.0, dtype=out, device="cuda")
        for y in (wide[:, 3:], torch.empty(m, rows, dtype=out, device="cuda")):
            P.spec_k_gemm8(x, w8, out=y)
            assert bool(((y.double() - ref).abs() <= bound).all())
        assert bool((wide[:, :3] == 7).all())


@pytest.mark.parametrize("m", [1, 5, 40, 300])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_gemm8_strides_alignment_and_what_lies_beside(P, m, out):
    k, rows = 272, 77
    big = rand(1, m + 2, k + 35).to(torch.bfloat16).cuda()
    w = rand(2, rows, k, scale=0.1).to(torch.bfloat16).cuda()
    for x in (big[1:m + 1, 3:k + 3], big[1:m + 1, 8:k + 8], big[:m, :k]):
        for at, width in ((0, rows), (5, rows + 9), (4, rows + 7)):
            y = torch.full((m, width), 7.0, dtype=DT[out], device="cuda")
            view = y[:, at:at + rows]
            got = check_gemm(P, x, w, DT[out], out=view)
            assert got.data_ptr() == view.data_ptr()
            assert (y[:, :at] == 7).all() and (y[:, at + rows:] == 7).all()


@pytest.mark.parametrize("m", [1, 16, 17, 200])
def test_gemm8_holds_the_8_bit_form_of_x(P, m):
    """w = 1: y is what the codes of x stand for, exactly (one product a sum)."""
    k = 384
    x = rand(9, m, k) * torch.exp(4 * rand(10, m, k))
    x[0, :128] = 0.0
    x[0, 128:256] = torch.linspace(-448, 448, 128)                      # ties and both ends
    x[0, 256] = 1e30
    x[-1, 300:340] *= 1e-33
    for dtype in (torch.float32, torch.bfloat16):
        xd = x.to(dtype).cuda()
        y = P.spec_k_gemm8(xd, P.spec_pack_weight8(torch.eye(k, dtype=dtype, device="cuda")), out_dtype=torch.float32)
        assert np.array_equal(f64(y), O.held_rows(f64(xd)))
        wt = P.spec_k_gemm8(torch.eye(k, dtype=dtype, device="cuda"), P.spec_pack_weight8(xd), out_dtype=torch.float32)
        assert np.array_equal(f64(wt).T, O.held_rows(f64(xd)))


@pytest.mark.parametrize("m", [3, 60, 150])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_gemm8_not_finite(P, m, out):
    k, rows = 300, 90
    x, w = rand(4, m, k).cuda(), rand(5, rows, k).cuda()
    clean = P.spec_k_gemm8(x, P.spec_pack_weight8(w), out_dtype=DT[out])
    x[1, 7], x[2, 299] = float("inf"), float("nan")
    w[11, 130], w[89, 0] = float("nan"), float("-inf")
    y = P.spec_k_gemm8(x, P.spec_pack_weight8(w), out_dtype=DT[out])
    nan = torch.zeros(m, rows, dtype=torch.bool, device="cuda")
    nan[1:3], nan[:, 11], nan[:, 89] = True, True, True
    assert torch.equal(torch.isnan(y), nan)
    assert torch.equal(y[~nan], clean[~nan])
    assert clean.isfinite().all()


def test_gemm8_sums_of_cancelling_and_far_apart_values(P):
    """fp32 results keep small products beside large ones that cancel."""
    x = torch.zeros(2, 256).cuda()
    w = torch.zeros(3, 256).cuda()
    x[:, 0], x[:, 1], x[:, 5], x[:, 200] = 256, -256, 2.0 ** -3, 2.0 ** -20
    w[:, 0], w[:, 1], w[:, 5], w[:, 200] = 1, 1, 2.0 ** -4, 1
    y = P.spec_k_gemm8(x, P.spec_pack_weight8(w), out_dtype=torch.float32)
    assert (y == 2.0 ** -7 + 2.0 ** -20).all()


def test_gemm8_scratch_is_checked_and_may_be_kept(P):
    x, w = rand(1, 40, 200).cuda(), P.spec_pack_weight8(rand(2, 50, 200).cuda())
    n = P.spec_k_gemm8_scratch_bytes(40, 200, 50)
    scratch = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    want = P.spec_k_gemm8(x, w)
    for _ in range(2):
        assert torch.equal(P.spec_k_gemm8(x, w, scratch=scratch), want)
    for call in (lambda: P.spec_k_gemm8(x, w, scratch=scratch[:n - 256]), lambda: P.spec_k_gemm8(x[:, :100], w), lambda: P.spec_k_gemm8(x.half(), w),
                 lambda: P.spec_k_gemm8(x[:0], w), lambda: P.spec_k_gemm8(x, w, out_dtype=torch.float16), lambda: P.spec_k_gemm8(x.cpu(), w),
                 lambda: P.spec_k_gemm8(x, w, out=torch.empty(40, 51, device="cuda")), lambda: P.spec_k_gemm8(x.t().contiguous().t(), w),
                 lambda: P.spec_k_gemm8(x, P.spec_pack_weight(torch.zeros(50, 200, device="cuda"))), lambda: P.spec_k_gemm8(x[:1].expand(40, 200), w),
                 lambda: P.spec_k_gemm8(x, torch.empty_like(w))):
        with pytest.raises(P.SpecError):
            call()


@pytest.mark.parametrize("m", [2, 300])
def test_gemm8_weights_beyond_2_gib(P, m):
    rows, k = 135008, 16384
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randn(rows, k, generator=g, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(m, k, generator=g, device="cuda", dtype=torch.bfloat16)
    w8 = P.spec_pack_weight8(w)
    assert w8.numel() > 1 << 31
    y = P.spec_k_gemm8(x, w8)
    for at in (0, rows // 2, rows - 96):
        part = P.spec_k_gemm8(x, P.spec_pack_weight8(w[at:at + 96].contiguous()), out_dtype=torch.float32)
        ref = f64(part)
        assert np.abs(f64(y[:, at:at + 96]) - ref).max() <= 2 * U16 * np.abs(ref).max()


def test_gemm8_packs_more_than_2_to_the_36_elements(P):
    """2^24 rows of 4100 (138 GB): blocks of 16 rows at the ends and in the middle are packed as they are by themselves."""
    rows, k = 1 << 24, 4100
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 2 * rows * k + P.spec_packed8_bytes(rows, k) + (4 << 30):
        pytest.skip("not enough free memory")
    w = torch.empty(rows, k, dtype=torch.bfloat16, device="cuda")
    firsts = [0, 16, rows // 2 - 16, rows // 2, (1 << 36) // k // 16 * 16, rows - 16]
    for i, r in enumerate(firsts):
        w[r:r + 16] = rand(i, 16, k).cuda()
    w8 = P.spec_pack_weight8(w)
    tiles, quads = (k + 127) // 128, (k + 511) // 512
    for r in firsts:
        one = P.spec_pack_weight8(w[r:r + 16].contiguous())
        b = r // 16
        assert torch.equal(w8[b * tiles * 2048:(b + 1) * tiles * 2048], one[:tiles * 2048])
        exps = rows // 16 * tiles * 2048 + b * quads * 64
        assert torch.equal(w8[exps:exps + quads * 64], one[tiles * 2048:tiles * 2048 + quads * 64])
    del w, w8
    torch.cuda.empty_cache()


# ---- cache --------------------------------------------------------------------------------------

@pytest.mark.parametrize("hkv,hd", [(1, 64), (3, 128), (8, 128), (128, 64)])
def test_kv8_store_and_load(P, hkv, hd):
    n = 3
    big = rand(hkv, 64 * n, hkv * hd + 24) * torch.exp(rand(7, 64 * n, 1)) * torch.exp(2 * rand(8, 1, hkv * hd + 24))
    big[70, 5], big[71, 6], big[72, 7] = float("nan"), float("inf"), float("-inf")
    big[128:, 8:8 + hd] = 0.0
    big = big.bfloat16().cuda()
    for k in (big[:, 8:8 + hkv * hd], big[:, 3:3 + hkv * hd]):          # aligned and not
        v = (big * 3 + 1).bfloat16()[:, 1:1 + hkv * hd]
        v = torch.as_strided(v, v.shape, k.stride(), v.storage_offset())
        cache = P.spec_kv8_alloc(n + 2, hkv, hd)
        cache.fill_(77)
        P.spec_k_kv8_store(k, v, cache, 1, hkv, hd)
        assert (cache[0] == 77).all() and (cache[-1] == 77).all()
        gk, gv = P.spec_k_kv8_load(cache, 1, n, hkv, hd)
        for got, src in ((gk, k), (gv, v)):
            assert np.array_equal(f64(got), O.held_kv(f64(src), hkv, hd), equal_nan=True)
        moved = cache.clone()                                           # blocks stand by themselves
        moved[0] = cache[2]
        assert torch.equal(P.spec_k_kv8_load(moved, 0, 1, hkv, hd)[0], gk[64:128]) or bool(gk[64:128].isnan().any())


def test_kv8_refusals_and_empty(P):
    k = torch.zeros(128, 256, dtype=torch.bfloat16, device="cuda")
    c = P.spec_kv8_alloc(2, 2, 128)
    P.spec_k_kv8_store(k[:0], k[:0], c, 2, 2, 128)
    assert P.spec_k_kv8_load(c, 2, 0, 2, 128)[0].shape == (0, 256)
    for call in (lambda: P.spec_k_kv8_store(k, k, c, 1, 2, 128), lambda: P.spec_k_kv8_store(k[:100], k[:100], c, 0, 2, 128),
                 lambda: P.spec_k_kv8_store(k.float(), k.float(), c, 0, 2, 128), lambda: P.spec_k_kv8_store(k, k, c, 0, 2, 64),
                 lambda: P.spec_k_kv8_store(k, k, c, -1, 2, 128), lambda: P.spec_k_kv8_load(c, 0, 3, 2, 128), lambda: P.spec_k_kv8_load(c, 0, -1, 2, 128)):
        with pytest.raises(P.SpecError):
            call()


# ---- attention8 -----------------------------------------------------------------------------------

def tree(rows, seed, deepest=15):
    r = np.random.default_rng(seed)
    depth, anc = [0], [np.zeros(16, np.int32)]
    for i in range(1, rows):
        p = int(r.integers(max(0, i - 9), i))
        while depth[p] == deepest:
            p = anc[p][deepest - 1]
        a = anc[p].copy()
        depth.append(depth[p] + 1)
        a[depth[i]] = i
        anc.append(a)
    return np.array(depth, np.int32), np.stack(anc)


def inputs(rows, hq, hkv, hd, blocks, win, seed, sharp=1.0):
    q = rand(seed, rows, hq * hd, scale=sharp)
    k = (rand(seed + 1, 64 * blocks + win, hkv * hd) * torch.exp(0.5 * rand(seed + 2, 1, hkv * hd))).bfloat16()
    v = (rand(seed + 3, 64 * blocks + win, hkv * hd) * torch.exp(rand(seed + 4, 64 * blocks + win, 1))).bfloat16()
    return q.cuda(), k.cuda(), v.cuda()


def run8(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd, **kw):
    n = 64 * blocks
    cache = None
    if blocks:
        cache = P.spec_kv8_alloc(blocks, hkv, hd)
        P.spec_k_kv8_store(k[:n], v[:n], cache, 0, hkv, hd)
    d = torch.from_numpy(np.asarray(depth, np.int32)).cuda()
    a = None if anc is None else torch.from_numpy(np.ascontiguousarray(anc, np.int32)).cuda()
    return P.spec_k_attention8(q, cache, blocks, k[n:].contiguous(), v[n:].contiguous(), base, d, a, hq, hkv, hd, **kw)


def attention_bound(q, k, v, blocks, base, depth, anc, hq, hkv, hd):
    n = 64 * blocks
    kf, vf = f64(k), f64(v)
    k8 = O.held_kv(kf[:n], hkv, hd) if blocks else kf[:0]
    v8 = O.held_kv(vf[:n], hkv, hd) if blocks else vf[:0]
    want, spread, delta, qk = O.attention8(f64(q), k8, v8, kf[n:], vf[n:], base, depth, anc, hq, hkv, hd)
    d = H * delta + U32 * qk
    return want, U16 * np.abs(want) + (np.exp(2 * d) - 1 + 2 * H + 2.0 ** -17 + 1e-6) * spread * (1 + U16) + 1e-37


def check_attention(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd, **kw):
    got = f64(run8(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd, **kw))
    want, tol = attention_bound(q, k, v, blocks, base, depth, anc, hq, hkv, hd)
    rows = np.asarray(depth) >= 0
    bad = ~(np.abs(got - want) <= tol)[rows]
    assert not bad.any(), (np.argwhere(bad)[:5], got[rows][bad][:5], want[rows][bad][:5], tol[rows][bad][:5])
    return got


@pytest.mark.parametrize("rows,hq,hkv,hd,blocks,recent,sharp", [
    (1, 1, 1, 64, 0, 0, 1.0), (1, 8, 1, 128, 1, 0, 1.0), (1, 4, 4, 128, 3, 63, 1.0), (1, 32, 8, 128, 40, 17, 1.0), (2, 2, 2, 64, 9, 5, 3.0), (5, 8, 2, 64, 2, 1, 1.0),
    (33, 4, 1, 128, 5, 30, 1.0), (60, 4, 4, 128, 8, 21, 1.0), (17, 16, 2, 128, 70, 3, 2.0), (64, 8, 8, 64, 1, 64, 1.0), (128, 8, 1, 64, 4, 0, 1.0),
    (130, 2, 1, 128, 3, 100, 1.0), (300, 4, 2, 128, 2, 40, 1.0), (257, 8, 1, 64, 6, 9, 1.0), (3, 1, 1, 128, 130, 2, 8.0)])
def test_attention8_chain(P, rows, hq, hkv, hd, blocks, recent, sharp):
    win = recent + rows
    q, k, v = inputs(rows, hq, hkv, hd, blocks, win, rows + hd + blocks, sharp)
    check_attention(P, q, k, v, blocks, 64 * blocks + recent, np.arange(rows), None, hq, hkv, hd)


@pytest.mark.parametrize("rows,hq,hkv,hd,blocks,recent", [
    (1, 2, 1, 64, 2, 0), (10, 4, 4, 128, 1, 7), (60, 8, 1, 128, 6, 40), (60, 4, 4, 64, 0, 3), (61, 4, 2, 128, 17, 0), (100, 8, 1, 128, 3, 63), (128, 2, 1, 64, 5, 64),
    (26, 16, 4, 128, 33, 129)])
def test_attention8_tree(P, rows, hq, hkv, hd, blocks, recent):
    win = recent + rows
    q, k, v = inputs(rows, hq, hkv, hd, blocks, win, rows + 2 * hd + blocks)
    depth, anc = tree(rows, rows)
    check_attention(P, q, k, v, blocks, 64 * blocks + recent, depth, anc, hq, hkv, hd)


@pytest.mark.parametrize("hq,hkv,hd,blocks", [(4, 2, 128, 3), (2, 2, 64, 0), (8, 1, 128, 20)])
def test_attention8_rows_that_see_little_padding_and_odd_paths(P, hq, hkv, hd, blocks):
    rows, recent = 40, 6
    win = recent + rows
    q, k, v = inputs(rows, hq, hkv, hd, blocks, win, 5)
    depth, anc = tree(rows, 3)
    depth[7], depth[39], depth[20] = -1, -5, 3                            # padding rows
    anc[20, :4] = [4, 4, 4, 9]                                          # one index several times
    anc[21, :2] = [-3, 2 ** 31 - 1 - 64 * blocks - recent]               # negative: a row of the window all the same; and one far beyond it
    depth[21] = 1
    anc[22, 0], depth[22] = -1000, 0                                    # outside: left out
    base = 64 * blocks + recent
    out = torch.full((rows, hq * hd), 5.0, dtype=torch.bfloat16, device="cuda")
    got = check_attention(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd, out=out, max_depth=15)
    assert (got[7] == 5).all() and (got[39] == 5).all()


def test_attention8_row_that_sees_nothing_is_zero(P):
    q, k, v = inputs(3, 4, 2, 128, 0, 3, 1)
    anc = np.zeros((3, 16), np.int32)
    anc[1] = 1000
    got = run8(P, q, k, v, 0, 0, [0, 2, 0], anc, 4, 2, 128)
    assert (got[1] == 0).all() and (got[0] != 0).any()
    chain = run8(P, q, k, v, 0, 3, [0, 0, -1], None, 4, 2, 128)         # row 0's own position lies behind the window: it sees the three rows in it
    want, tol = attention_bound(q, k, v, 0, 3, [0, 0, -1], None, 4, 2, 128)
    assert (np.abs(f64(chain)[:2] - want[:2]) <= tol[:2]).all()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf"), 3.3e38])
@pytest.mark.parametrize("anc_used", [False, True])
@pytest.mark.parametrize("rows,blocks", [(12, 2), (90, 1)])
def test_attention8_what_a_row_does_not_see_does_not_touch_it(P, what, anc_used, rows, blocks):
    hq, hkv, hd, recent = 4, 2, 128, 5
    q, k, v = inputs(rows, hq, hkv, hd, blocks, recent + rows, 9)
    depth, anc = tree(rows, 8) if anc_used else (np.arange(rows, dtype=np.int32), None)
    base, n = 64 * blocks + recent, 64 * blocks
    clean = run8(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd)
    bad = 9
    k[n + recent + bad], v[n + recent + bad] = what, what
    got = run8(P, q, k, v, blocks, base, depth, anc, hq, hkv, hd)
    sees = np.array([bad in ([i for i in range(depth[r] + 1)] if anc is None else list(anc[r][:depth[r] + 1])) for r in range(rows)])
    assert sees.any() and not sees.all()
    assert torch.equal(got[~sees], clean[~sees])
    if not math.isfinite(what):
        assert not torch.isfinite(got[sees]).all(1).any()


def test_attention8_not_finite_where_seen(P):
    """A NaN key makes the rows that see it NaN; a NaN value its dim; an infinite value in the window stays one."""
    hq, hkv, hd, blocks, rows = 2, 1, 64, 2, 4
    q, k, v = inputs(rows, hq, hkv, hd, blocks, 3 + rows, 2)
    depth = np.arange(rows)
    for at in (30, 128 + 1):                                            # in a block, in the window
        v2 = v.clone()
        v2[at, 17] = float("nan")
        got = run8(P, q, k, v2, blocks, 131, depth, None, hq, hkv, hd).view(rows, hq, hd)
        assert got[:, :, 17].isnan().all() and got[:, :, :17].isfinite().all() and got[:, :, 18:].isfinite().all()
        k2 = k.clone()
        k2[at, 17] = float("nan")
        assert run8(P, q, k2, v, blocks, 131, depth, None, hq, hkv, hd).isnan().all()
    v[128 + 1, 17], v[128 + 2, 18] = float("inf"), float("-inf")
    got = run8(P, q, k, v, blocks, 131, depth, None, hq, hkv, hd).view(rows, hq, hd)
    assert (got[:, :, 17] == float("inf")).all() and (got[:, :, 18] == float("-inf")).all() and got[:, :, 19:].isfinite().all()


@pytest.mark.parametrize("rows,hq,hkv,hd,blocks,is_tree", [(2, 4, 2, 128, 0, False), (2, 4, 2, 128, 2, True), (40, 4, 4, 128, 3, True), (60, 2, 2, 64, 0, True), (300, 8, 2, 128, 130, False)])
@pytest.mark.parametrize("exact", [True, False])
def test_attention8_infinite_keys(P, rows, hq, hkv, hd, blocks, is_tree, exact):
    """A window key whose score is -infinity weighs nothing, whether or not the query is a bf16 value: the call without that row is the reference.  One of +infinity makes NaN."""
    recent, bad, n = 40, 33, 64 * blocks
    q, k, v = inputs(rows, hq, hkv, hd, blocks, recent + rows, 21)
    q = q.abs() + 0.01
    if exact:
        q = q.bfloat16().float()
    depth, anc = tree(rows, 8) if is_tree else (np.arange(rows, dtype=np.int32), None)
    rest = [torch.cat([t[:n + bad], t[n + bad + 1:]]) for t in (k, v)]
    for dim, what in ((17, float("-inf")), (hd - 1, float("-inf")), (slice(3, 30, 5), float("-inf"))):
        k2 = k.clone().view(-1, hkv, hd)
        k2[n + bad, :, dim] = what
        got = f64(run8(P, q, k2.view(k.shape), v, blocks, n + recent, depth, anc, hq, hkv, hd))
        some = [i for i in (0, 1, rows // 2, rows - 1) if i < rows]
        want, tol = attention_bound(q[some], *rest, blocks, n + recent - 1, depth[some], None if anc is None else anc[some], hq, hkv, hd)
        assert (np.abs(got[some] - want) <= tol).all()
        assert np.isfinite(got).all()
        k2[n + bad, :, dim] = -what
        assert run8(P, q, k2.view(k.shape), v, blocks, n + recent, depth, anc, hq, hkv, hd).isnan().all()
        assert torch.isfinite(run8(P, -q, k2.view(k.shape), v, blocks, n + recent, depth, anc, hq, hkv, hd)).all()


def test_attention8_infinite_scores(P):
    """Rows that see nothing but scores of -infinity get zeros; scores beyond fp32 are infinities; a query's own infinity stays in its row."""
    hq, hkv, hd, rows = 2, 1, 64, 3
    q, k, v = inputs(rows, hq, hkv, hd, 0, rows, 4)
    q = q.abs() + 0.01
    alone = k.clone()
    alone[0, 9] = float("-inf")
    got = run8(P, q, alone, v, 0, 0, [0, 1, 2], None, hq, hkv, hd)
    assert (got[0] == 0).all() and torch.isfinite(got).all()
    want, tol = attention_bound(q, k[1:], v[1:], 0, 0, [-1, 0, 1], None, hq, hkv, hd)
    assert (np.abs(f64(got)[1:] - want[1:]) <= tol[1:]).all()
    for far in (1.2345e30, 1e30 * (1 + 2.0 ** -9 - 2.0 ** -14)):         # (their rests have either sign)
        big, key = q.clone().view(rows, hq, hd), k.clone()
        big[:, :, 3], key[:, 3] = far, 0.0
        key[0, 3] = -1e30
        got = run8(P, big.view(rows, -1), key, v, 0, 0, [0, 1, 2], None, hq, hkv, hd)
        big[:, :, 3] = 0.0
        want, tol = attention_bound(big.view(rows, -1), key[1:], v[1:], 0, 0, [-1, 0, 1], None, hq, hkv, hd)
        assert (got[0] == 0).all() and (np.abs(f64(got)[1:] - want[1:]) <= tol[1:]).all()
    clean = run8(P, q, k, v, 0, 0, [0, 1, 2], None, hq, hkv, hd)
    for sign, check in ((-1, lambda t: (t == 0).all()), (1, lambda t: t.isnan().all())):
        key, wild = k.clone(), q.clone().view(rows, hq, hd)
        key[:, 5] = sign * (key[:, 5].abs() + 1)
        wild[1, 0, 5] = float("inf")
        same = run8(P, q, key, v, 0, 0, [0, 1, 2], None, hq, hkv, hd).view(rows, hq, hd)
        got = run8(P, wild.view(rows, -1), key, v, 0, 0, [0, 1, 2], None, hq, hkv, hd).view(rows, hq, hd)
        assert check(got[1, 0])
        same[1, 0], got[1, 0] = 0, 0
        assert torch.equal(same, got)
    assert torch.isfinite(clean).all()


def test_attention8_scales_far_apart(P):
    """Keys, values and queries whose magnitudes differ by block, head and row."""
    hq, hkv, hd, blocks, rows = 4, 2, 128, 12, 6
    q, k, v = inputs(rows, hq, hkv, hd, blocks, 4 + rows, 77)
    q *= torch.tensor([1e-6, 1.0, 30.0, 1e4, 1e-30, 0.0]).cuda()[:, None]
    for b in range(blocks):
        k[64 * b:64 * b + 64] *= 2.0 ** (b % 5 - 4)
        v[64 * b:64 * b + 64] *= 2.0 ** (3 * (b % 4) - 6)
    k[:, :hd] *= 1e-3
    check_attention(P, q, k, v, blocks, 64 * blocks + 4, np.arange(rows), None, hq, hkv, hd)


@pytest.mark.parametrize("rows", [1, 60, 200])
@pytest.mark.parametrize("large", [1e20, 1e24])
def test_attention8_blocks_without_values_beside_large_ones(P, rows, large):
    """Blocks whose values are all zero keep their share of the sum of weights, before and behind a block of values far larger than theirs."""
    hq, hkv, hd, blocks = 64, 64, 64, 24                                  # (several blocks one after the other in a workgroup)
    q, k, v = inputs(rows, hq, hkv, hd, blocks, rows, 15)
    v[:] = 0
    v[64 * 8:64 * 12] = large * (1 + torch.rand(256, hkv * hd, generator=torch.Generator().manual_seed(1)).cuda())
    check_attention(P, q, k, v.bfloat16(), blocks, 64 * blocks, np.arange(rows), None, hq, hkv, hd)


@pytest.mark.parametrize("rows,hq,hkv,hd,blocks", [(1, 2, 2, 64, 9), (1, 64, 64, 128, 100), (60, 32, 32, 64, 40), (104, 8, 8, 128, 101), (60, 64, 8, 128, 300)])
@pytest.mark.parametrize("bits", [0, 12.2, 20.6, 23.8, 25.7])
def test_attention8_small_weights_behind_a_sink(P, rows, hq, hkv, hd, blocks, bits):
    """In every block one key, whose value is zero, outweighs the others by 2^bits: the result is what the others hold, and their weights have the precision that is stated
    (2^-10 = 2 h).  Queries have one element, exact in fp16, so that scores are off by fp32's roundings only: 100 * 2^-24 in units of log2."""
    a = round(bits * 64 * math.sqrt(hd) / 192 * math.log(2)) / 64            # (192 is a code)
    q = torch.zeros(rows, hq, hd)
    q[:, :, 0] = a
    k = torch.zeros(64 * blocks + rows, hkv, hd)
    v = torch.exp(rand(3, 64 * blocks + rows, hkv, hd))
    for b in range(blocks):
        at = 64 * b + 17 * b % 64
        k[at, :, 0], v[at] = 192.0, 0.0
    q, k, v = q.view(rows, -1).cuda(), k.view(-1, hkv * hd).bfloat16().cuda(), v.view(-1, hkv * hd).bfloat16().cuda()
    n, depth = 64 * blocks, np.zeros(rows, np.int32)
    got = f64(run8(P, q, k, v, blocks, n, depth, None, hq, hkv, hd)).reshape(rows, hkv, -1)
    for h in (0, hkv - 1):
        kh, vh = (f64(t[:, h * hd:h * hd + hd]) for t in (k, v))
        want, spread, _, _ = O.attention8(f64(q).reshape(rows, hkv, -1)[:1, h], O.held_kv(kh[:n], 1, hd), O.held_kv(vh[:n], 1, hd), kh[n:], vh[n:], n, depth[:1], None, hq // hkv, 1, hd)
        tol = U16 * np.abs(want) + (2 * H + 100 * U32 + 2.0 ** -17 + 1e-6) * spread * (1 + U16)
        assert (np.abs(got[:, h] - want) <= tol).all(), float((np.abs(got[:, h] - want) / tol).max())


def test_attention8_one_key_outweighs_all(P):
    hq, hkv, hd, blocks = 2, 1, 128, 20
    q, k, v = inputs(2, hq, hkv, hd, blocks, 2, 5)
    for at in (0, 63, 64, 700, 64 * blocks - 1, 64 * blocks):
        k2 = k.clone()
        k2[at] = (q[0, :hd] * 40).bfloat16()
        got = check_attention(P, q, k2, v, blocks, 64 * blocks, np.arange(2), None, hq, hkv, hd)
        assert np.isfinite(got).all()


def test_attention8_offsets_beyond_2_gib(P):
    """A million tokens: every block the same but one, so that the exact result is that of 128 keys with their numbers of copies."""
    hq, hkv, hd = 8, 8, 128
    blocks = (1 << 31) // P.spec_kv8_bytes(1, hkv, hd) + 40
    q, k, v = inputs(1, hq, hkv, hd, 2, 1, 3)
    two = P.spec_kv8_alloc(2, hkv, hd)
    P.spec_k_kv8_store(k[:128], v[:128], two, 0, hkv, hd)
    cache = two[:1].repeat(blocks, 1)
    last = blocks - 7
    cache[last] = two[1]
    assert cache.numel() > 1 << 31
    d = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = f64(P.spec_k_attention8(q, cache, blocks, k[128:], v[128:], 64 * blocks, d, None, hq, hkv, hd, max_depth=0)).reshape(hq, hd)
    kk = np.concatenate([O.held_kv(f64(k[:128]), hkv, hd), f64(k[128:])]).reshape(-1, hkv, hd)
    vv = np.concatenate([O.held_kv(f64(v[:128]), hkv, hd), f64(v[128:])]).reshape(-1, hkv, hd)
    copies = np.array([blocks - 1] * 64 + [1] * 65, np.float64)
    for h in range(hq):
        qq = f64(q).reshape(hq, hd)[h]
        p = np.exp(kk[:, h] @ qq / math.sqrt(hd)) * copies
        p /= p.sum()
        dd = H * (np.abs(kk[:, h]) @ np.abs(qq)).max() / math.sqrt(hd)
        want, spread = p @ vv[:, h], p @ np.abs(vv[:, h])
        # (a sum of n fp32 terms that the lanes and parts share: its blocks are added up in chains of at most n / 64)
        tol = U16 * np.abs(want) + (np.exp(2 * dd) - 1 + 2 * H + 2.0 ** -17 + blocks * U32) * spread
        assert (np.abs(got[h] - want) <= tol).all()


def test_attention8_joins_the_parts_of_2_to_the_28_queries(P):
    """Rows repeat every 64, and every 64 have the bits of the first: the launch that joins two window parts has more than 2^32 threads (249 GB in all)."""
    rows, hq, hkv, hd, win = 1 << 20, 264, 33, 64, 300
    assert P.spec_k_attention8_plan(rows, hq, hkv, hd, 0, win)[2:] == (0, 2)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 6 * rows * hq * hd + P.spec_k_attention8_scratch_bytes(rows, hq, hkv, hd, 0, win) + (4 << 30):
        pytest.skip("not enough free memory")
    base, k, v = inputs(64, hq, hkv, hd, 0, win, 3)
    q = torch.empty(rows, hq * hd, device="cuda")
    q.view(-1, 64, hq * hd).copy_(base)
    out = P.spec_k_attention8(q, None, 0, k, v, win - 1, torch.zeros(rows, dtype=torch.int32, device="cuda"), None, hq, hkv, hd, max_depth=0)
    for at in range(0, rows, 1 << 17):
        assert bool((out[at:at + (1 << 17)].view(-1, 64, hq * hd) == out[:64]).all())
    assert torch.equal(out[-64:], out[:64])
    h = hkv - 1
    want, tol = attention_bound(base.view(64, hkv, -1)[:3, h], k[:, h * hd:], v[:, h * hd:], 0, win - 1, np.zeros(3, np.int32), None, hq // hkv, 1, hd)
    assert (np.abs(f64(out[-64:].view(64, hkv, -1)[:3, h]) - want) <= tol).all()
    del q, out
    torch.cuda.empty_cache()


def test_attention8_binding_refusals(P):
    hq, hkv, hd = 4, 2, 64
    q, k, v = inputs(3, hq, hkv, hd, 1, 4, 1)
    c = P.spec_kv8_alloc(1, hkv, hd)
    d = torch.zeros(3, dtype=torch.int32, device="cuda")
    ok = dict(q=q, cache8=c, n_blocks=1, kwin=k[64:].contiguous(), vwin=v[64:].contiguous(), base=65, depth=d, anc=None, hq=hq, hkv=hkv, hd=hd)
    for kw in (dict(q=q.bfloat16()), dict(q=q[:, :64]), dict(n_blocks=2), dict(cache8=None), dict(kwin=k[64:].float()), dict(vwin=v[:64]), dict(base=63), dict(depth=d.long()),
               dict(depth=d[:2]), dict(anc=torch.zeros(3, 15, dtype=torch.int32, device="cuda")), dict(hq=3), dict(hd=128), dict(max_depth=-1), dict(max_depth=2 ** 32), dict(base=2 ** 32 + 65),
               dict(out=torch.empty(3, 256, device="cuda")), dict(q=q.cpu()),
               dict(kwin=k[64:64], vwin=v[64:64]), dict(q=q[:0], depth=d[:0]), dict(anc=torch.zeros(3, 16, dtype=torch.int32, device="cuda"), max_depth=16)):
        with pytest.raises(P.SpecError):
            P.spec_k_attention8(**{**ok, **kw})
    q, k, v = inputs(60, hq, hkv, hd, 1, 60, 1)                           # a call that needs scratch: too little, and its own kept for two calls
    many = {**ok, **dict(q=q, kwin=k[64:].contiguous(), vwin=v[64:].contiguous(), base=64, depth=torch.arange(60, dtype=torch.int32, device="cuda"))}
    n = P.spec_k_attention8_scratch_bytes(60, hq, hkv, hd, 1, 60)
    P.spec_k_kv8_store(k[:64], v[:64], c, 0, hkv, hd)
    want = P.spec_k_attention8(**many)
    kept = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        assert torch.equal(P.spec_k_attention8(**many, scratch=kept), want)
    with pytest.raises(P.SpecError):
        P.spec_k_attention8(**many, scratch=kept[:n - 256])


# What large calls take: (waves, query blocks, block parts, window parts), so that a case keeps to its path.  Joined ranges that go on into the window, several blocks one after the
# other in the LDS of 2, 4 and 8 wavefronts and in the registers of few queries, query blocks dealt out in turn (hkv * parts not a multiple of 8, more than 256 workgroups).
LARGE = [
    (True, 60, 64, 8, 512, 0, (8, 2, 16, 0)), (True, 60, 64, 8, 510, 40, (8, 2, 16, 0)), (False, 1024, 32, 8, 128, 0, (8, 16, 2, 0)), (False, 300, 16, 2, 130, 40, (8, 10, 11, 1)),
    (False, 1200, 3, 3, 500, 50, (8, 5, 16, 1)), (False, 700, 16, 4, 40, 0, (8, 11, 3, 2)), (False, 1000, 72, 9, 11, 10, (8, 32, 1, 0)), (False, 1500, 9, 9, 0, 0, (8, 6, 0, 6)),
    (True, 60, 16, 2, 300, 40, (4, 4, 30, 2)), (False, 104, 8, 8, 101, 6, (4, 1, 30, 2)), (True, 60, 32, 32, 64, 21, (2, 1, 14, 2)), (False, 1, 64, 64, 100, 40, (0, 1, 3, 1)),
]


@pytest.mark.parametrize("is_tree,rows,hq,hkv,blocks,recent,plan", LARGE)
def test_attention8_large_calls(P, is_tree, rows, hq, hkv, blocks, recent, plan):
    """Some rows and kv heads of large calls.  Dim d of the values has what the 64 tokens b = d (mod 128) hold, and a hundredth of it elsewhere: a block or window row too many, too
    few or in the wrong place moves a dim by far more than roundings may."""
    hd, win = 128, recent + rows
    assert P.spec_k_attention8_plan(rows, hq, hkv, hd, blocks, win) == plan
    q, k, _ = inputs(rows, hq, hkv, hd, blocks, win, rows + blocks, 0.5)
    n = 64 * blocks
    g = torch.Generator(device="cuda").manual_seed(rows)
    v = torch.rand(n + win, hkv, hd, generator=g, device="cuda") + 0.5
    at = torch.arange(n + win, device="cuda") // 64
    v = (v * torch.where((at % hd)[:, None] == torch.arange(hd, device="cuda"), 1.0, 0.01)[:, None] * torch.exp2((at % 5).float())[:, None, None]).view(n + win, -1).bfloat16()
    depth, anc = tree(rows, rows) if is_tree else (np.arange(rows, dtype=np.int32), None)
    got = f64(run8(P, q, k, v, blocks, n + recent, depth, anc, hq, hkv, hd)).reshape(rows, hkv, -1)
    some = sorted({i for i in (0, 1, rows - 1, rows // 2, 255 * hkv // hq, 256 * hkv // hq) if i < rows})
    for h in sorted({0, hkv - 1}):
        group = hq // hkv
        want, tol = attention_bound(q.view(rows, hkv, -1)[some, h], k[:, h * hd:h * hd + hd], v[:, h * hd:h * hd + hd], blocks, n + recent, depth[some], None if anc is None else anc[some],
                                    group, 1, hd)
        bad = ~(np.abs(got[some, h] - want) <= tol)
        assert not bad.any(), (h, np.argwhere(bad)[:5], got[some, h][bad][:5], want[bad][:5], tol[bad][:5])



# ---- rotary ---------------------------------------------------------------------------------------

def check_rotary(P, plan, f, m, rot, layout, x, pos, out_dtype, adjoint=False, **kw):
    src = f64(x)                                                        # (before the call: it may be in place)
    got = P.spec_k_rotary(plan, [x], pos, out_dtypes=[out_dtype], adjoint=adjoint, **kw)[0]
    at = f64(pos) if isinstance(pos, torch.Tensor) else pos + np.arange(x.shape[0])
    # angles in 64 bits: positions up to 2^31 are off by 2^31 * 2^-53 turns, as are the oracle's
    want = O.rotary(src, at, f, m, rot, layout, adjoint)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size = np.zeros_like(src)
    size[..., a] = size[..., b] = np.abs(src[..., a]) + np.abs(src[..., b])
    tol = 2.0 ** -21 * m * size + (U16 if out_dtype == torch.bfloat16 else U32) * np.abs(want) + 1e-38
    bad = ~(np.abs(f64(got) - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], f64(got)[bad][:5], want[bad][:5])
    if out_dtype == x.dtype:
        assert np.array_equal(f64(got)[..., rot:], src[..., rot:])      # untouched dims
    return got


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,hd,rot", [(1, 1, 2, 2), (3, 5, 80, 32), (7, 2, 128, 128), (33, 40, 128, 64), (2, 3, 96, 90), (5, 1, 7, 6), (4, 6, 256, 256), (9, 3, 64, 48),
                                               (130, 1, 33, 2), (1, 1024, 64, 64), (3, 2, 16, 0), (2, 1024, 255, 254), (700, 2, 64, 64)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32")])
def test_rotary(P, rows, heads, hd, rot, layout, dtype, out):
    kw = dict(scaling="yarn", factor=4.0, trained_len=2048) if rot >= 64 else {}
    plan = P.spec_rotary_plan(rot, 1e4, layout=layout, **kw)
    f, m = O.rope_frequencies(rot, 1e4, **kw) if rot else (np.zeros(0), 1.0)
    x = rand(rows + hd, rows, heads, hd).to(DT[dtype]).cuda()
    pos = torch.from_numpy(np.random.default_rng(1).integers(0, 200000, rows).astype(np.int32)).cuda()
    for adjoint in (False, True):
        check_rotary(P, plan, f, m, rot, layout, x, pos, DT[out], adjoint)
    check_rotary(P, plan, f, m, rot, layout, x, 17, DT[out])


def test_rotary_far_and_negative_positions(P):
    plan = P.spec_rotary_plan(128, 5e5)
    f, m = O.rope_frequencies(128, 5e5)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003, 131071], dtype=torch.int32, device="cuda")
    x = rand(1, 7, 2, 128).cuda()
    check_rotary(P, plan, f, m, 128, "half", x, pos, torch.float32)
    check_rotary(P, plan, f, m, 128, "half", x, 2 ** 31 - 3, torch.float32)   # rows beyond: positions go on in 64 bits


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot,off", [(128, 128, 0), (128, 64, 8), (64, 64, 1), (80, 48, 3)])
def test_rotary_strides_orders_and_in_place(P, layout, hd, rot, off):
    rows, heads = 11, 3
    plan = P.spec_rotary_plan(rot, 1e4, layout=layout)
    f, m = O.rope_frequencies(rot, 1e4)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 37
    for dtype in (torch.bfloat16, torch.float32):
        flat = rand(5, rows, heads * hd + 40).to(dtype).cuda()
        a = flat[:, off:off + heads * hd].unflatten(1, (heads, hd))     # part of a wider row
        b = rand(6, heads, rows, hd).to(dtype).cuda().transpose(0, 1)   # heads outermost
        wide = flat.clone()
        o = wide[:, off:off + heads * hd].unflatten(1, (heads, hd))
        for x in (a, b):
            got = P.spec_k_rotary(plan, [x], pos, outs=[o])[0]
            assert got.data_ptr() == o.data_ptr()
            assert torch.equal(o, check_rotary(P, plan, f, m, rot, layout, x, pos, dtype))
        assert torch.equal(wide[:, :off], flat[:, :off]) and torch.equal(wide[:, off + heads * hd:], flat[:, off + heads * hd:])
        keep = check_rotary(P, plan, f, m, rot, layout, b, pos, dtype)
        P.spec_k_rotary(plan, [b], pos, outs=[b])                       # in place
        assert torch.equal(b, keep)


def test_rotary_three_parts_and_copies(P):
    rows, hq, hkv, hd = 60, 32, 8, 128
    plan = P.spec_rotary_plan(hd, 5e5, scaling="llama3", factor=8.0, trained_len=8192)
    f, m = O.rope_frequencies(hd, 5e5, scaling="llama3", factor=8.0, trained_len=8192)
    qkv = rand(1, rows, (hq + 2 * hkv) * hd).cuda()
    xs = [t.unflatten(1, (-1, hd)) for t in qkv.split([hq * hd, hkv * hd, hkv * hd], 1)]
    window = torch.zeros(rows + 5, hkv * hd, dtype=torch.bfloat16, device="cuda")
    outs = [torch.empty(rows, hq, hd, device="cuda"), window[5:].unflatten(1, (hkv, hd)), torch.empty(rows, hkv, hd, dtype=torch.bfloat16, device="cuda")]
    pos = torch.arange(100000, 100000 + rows, dtype=torch.int32, device="cuda")
    P.spec_k_rotary(plan, xs, pos, turned=[True, True, False], outs=outs)
    assert torch.equal(outs[0], check_rotary(P, plan, f, m, hd, "half", xs[0], pos, torch.float32))
    assert torch.equal(outs[1], check_rotary(P, plan, f, m, hd, "half", xs[1], pos, torch.bfloat16))
    assert torch.equal(outs[2], xs[2].bfloat16()) and (window[:5] == 0).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_adjoint_is_the_gradient(P, layout):
    """Against the formula's (the transpose, by the products of random vectors) and against differences."""
    rows, heads, hd, rot = 6, 2, 64, 40
    plan = P.spec_rotary_plan(rot, 1e4, layout=layout, scaling="yarn", factor=8.0, trained_len=256)
    x, g = rand(1, rows, heads, hd).cuda(), rand(2, rows, heads, hd).cuda()
    y = P.spec_k_rotary(plan, [x], 1234)[0]
    gx = P.spec_k_rotary(plan, [g], 1234, adjoint=True)[0]
    a, b = float((y.double() * g.double()).sum()), float((x.double() * gx.double()).sum())
    assert abs(a - b) <= 2.0 ** -20 * 1.3 * float((x.abs().double() * (g.abs() + g.abs().flip(-1)).double()).sum()) + 2.0 ** -20 * float((y.abs() * g.abs()).sum())
    for at in ((0, 0, 3), (5, 1, 39), (2, 0, 50)):                      # d (y . g) / d x by differences of the linear map, h = 1/4
        d = torch.zeros_like(x)
        d[at] = 0.25
        up, down = (P.spec_k_rotary(plan, [x + s * d], 1234)[0].double() for s in (1, -1))
        slope = float(((up - down) * g.double()).sum() / 0.5)
        assert abs(slope - float(gx[at])) <= 2.0 ** -18 * 2 * (float(g.abs().max()) * 4 * float(x.abs().max()) + 1)


def test_rotary_binding_refusals(P):
    plan = P.spec_rotary_plan(64, 1e4)
    x, pos = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: P.spec_k_rotary(plan, [], 0), lambda: P.spec_k_rotary(plan, [x] * 4, 0), lambda: P.spec_k_rotary(plan, [x[0]], 0), lambda: P.spec_k_rotary(plan, [x, x[:3]], 0),
                 lambda: P.spec_k_rotary(plan, [x, x[..., :32]], 0), lambda: P.spec_k_rotary(plan, [x.half()], 0), lambda: P.spec_k_rotary(plan, [x], pos.long()),
                 lambda: P.spec_k_rotary(plan, [x], pos[:3]), lambda: P.spec_k_rotary(plan, [x], 2 ** 31), lambda: P.spec_k_rotary(plan, [x], 0, outs=[x, x]),
                 lambda: P.spec_k_rotary(plan, [x], 0, outs=[x[:, :1]]), lambda: P.spec_k_rotary(plan, [x], 0, turned=[True, False]), lambda: P.spec_k_rotary(plan, [x.cpu()], 0),
                 lambda: P.spec_k_rotary(plan, [x.transpose(1, 2)], 0), lambda: P.spec_k_rotary(P.spec_rotary_plan(128, 1e4), [x], 0), lambda: P.spec_k_rotary(plan, [x[:0]], 0)):
        with pytest.raises(P.SpecError):
            call()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot", [(128, 128), (90, 66)])
@pytest.mark.parametrize("kw", [dict(), dict(scaling="yarn", factor=16.0, trained_len=4096), dict(scaling="yarn", factor=5.3, trained_len=300)])
def test_rotary_sines_and_cosines_are_rounded_once(P, layout, hd, rot, kw):
    """Planes (1, 0) and (0, 1) become mscale (cos t, sin t) and mscale (-sin t, cos t) as they are held: half a step of fp32 off (and 4 roundings of 64 bits of angles up to 5000, and
    the series' 4e-13 mscale)."""
    plan = P.spec_rotary_plan(rot, 1e4, layout=layout, **kw)
    pos = np.concatenate([np.arange(0, 200), np.random.default_rng(1).integers(-5000, 5000, 300)])
    t = pos[:, None].astype(np.float64) * np.array(plan.freq[:rot // 2])
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    x = torch.zeros(len(pos), 2, hd)
    x[:, 0, first], x[:, 1, second] = 1.0, 1.0
    for adjoint in (False, True):
        y = f64(P.spec_k_rotary(plan, [x.cuda()], torch.from_numpy(pos.astype(np.int32)).cuda(), adjoint=adjoint)[0])
        c, s = plan.mscale * np.cos(t), plan.mscale * np.sin(t) * (-1 if adjoint else 1)
        for got, want in ((y[:, 0, first], c), (y[:, 0, second], s), (y[:, 1, first], -s), (y[:, 1, second], c)):
            assert (np.abs(got - want) <= U32 * np.abs(want) + plan.mscale * (4 * 5000 * 2.0 ** -53 + 5e-13)).all()


def test_rotary_of_most_rows(P):
    """2^24 rows, each more than a workgroup's steps, in place: as the same rows by themselves."""
    rows, heads, hd = 1 << 24, 3, 96
    plan = P.spec_rotary_plan(2, 1e4, layout="interleaved")
    some = torch.tensor([0, 1, 77, rows // 2 - 1, rows // 2, rows // 2 + 1, rows - 2, rows - 1], device="cuda")
    x = torch.empty(rows, heads, hd, dtype=torch.bfloat16, device="cuda")
    x.view(-1, 64, heads, hd).copy_(rand(1, 64, heads, hd).cuda())
    want = P.spec_k_rotary(plan, [x[some]], some.to(torch.int32))[0]
    assert not torch.equal(want, x[some])
    P.spec_k_rotary(plan, [x], 0, outs=[x])
    assert torch.equal(x[some], want)


def test_rotary_not_finite_values_stay_in_their_plane(P):
    plan = P.spec_rotary_plan(64, 1e4)
    x = rand(1, 4, 2, 64).cuda()
    x[1, 0, 5], x[2, 1, 40] = float("nan"), float("inf")
    y = P.spec_k_rotary(plan, [x], 9)[0]
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 0, 5] = bad[1, 0, 37] = bad[2, 1, 40] = bad[2, 1, 8] = True
    assert torch.equal(~y.isfinite(), bad)


# ---- together -------------------------------------------------------------------------------------

def layer_pass(P, w, x, cache, blocks, window, recent, depth, anc, pos, plan, hq, hkv, hd):
    """Attention block of a layer as a program runs it: QKV, rotary into the window, attention, O."""
    rows = x.shape[0]
    qkv = P.spec_k_gemm8(x, w["qkv"], out_dtype=torch.float32)
    xs = [t.unflatten(1, (-1, hd)) for t in qkv.split([hq * hd, hkv * hd, hkv * hd], 1)]
    q = torch.empty(rows, hq, hd, device="cuda")
    kw, vw = (t[recent:recent + rows].unflatten(1, (hkv, hd)) for t in window)
    P.spec_k_rotary(plan, xs, pos, turned=[True, True, False], outs=[q, kw, vw])
    o = P.spec_k_attention8(q.view(rows, -1), cache, blocks, window[0][:recent + rows], window[1][:recent + rows], 64 * blocks + recent, depth, anc, hq, hkv, hd,
                            max_depth=15 if anc is not None else rows - 1)
    return P.spec_k_gemm8(o, w["o"])


def test_layer_prompt_then_trees(P):
    """A prompt, its whole blocks into 8 bits, then a tree's rows and their commit: every step against the oracle run on the step's own inputs."""
    hq, hkv, hd, d = 8, 2, 64, 320
    wf = {"qkv": rand(1, (hq + 2 * hkv) * hd, d, scale=0.06).bfloat16().cuda(), "o": rand(2, d, hq * hd, scale=0.06).bfloat16().cuda()}
    w = {n: P.spec_pack_weight8(t) for n, t in wf.items()}
    plan = P.spec_rotary_plan(hd, 1e4, scaling="linear", factor=2.0)
    f, m = O.rope_frequencies(hd, 1e4, scaling="linear", factor=2.0)
    window = [torch.full((256, hkv * hd), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = P.spec_kv8_alloc(8, hkv, hd)

    def oracle(x, pos, blocks, recent, depth, anc):
        qkv, tol = gemm_bound(O.held_rows(f64(x)), O.held_rows(f64(wf["qkv"])), False)
        q = O.rotary(qkv[:, :hq * hd].reshape(len(pos), hq, hd), pos, f, m, hd, "half").reshape(len(pos), -1)
        k8, v8 = (f64(t) for t in P.spec_k_kv8_load(cache, 0, blocks, hkv, hd))
        win = [f64(t[:recent + len(pos)]) for t in window]
        k = O.rotary(qkv[:, hq * hd:(hq + hkv) * hd].reshape(len(pos), hkv, hd), pos, f, m, hd, "half").reshape(len(pos), -1)
        assert np.abs(win[0][recent:] - k).max() <= 2 * U16 * np.abs(k).max()       # what the rotary wrote into the window
        out, spread, delta, qk = O.attention8(q, k8, v8, win[0], win[1], 64 * blocks + recent, depth, anc, hq, hkv, hd)
        return out

    def close(got, attn):
        # O projection of bf16 attention outputs: their rounding may move a code to its neighbour (2^-3 of it in all), the sum is of independent ones
        want = O.held_rows(attn) @ O.held_rows(f64(wf["o"])).T
        assert np.linalg.norm(f64(got) - want) <= 0.04 * np.linalg.norm(want)

    n = 150
    x = rand(3, n, d).bfloat16().cuda()
    y = layer_pass(P, w, x, cache, 0, window, 0, torch.arange(n, dtype=torch.int32, device="cuda"), None, 0, plan, hq, hkv, hd)
    close(y, oracle(x, np.arange(n), 0, 0, np.arange(n), None))
    P.spec_k_kv8_store(window[0][:128], window[1][:128], cache, 0, hkv, hd)
    for t in window:
        t[:22] = t[128:150].clone()
        t[22:] = float("nan")
    committed = 150
    for cycle in range(3):
        depth, anc = tree(26, cycle)
        blocks, recent = committed // 64, committed % 64
        pos = committed + depth
        x = rand(10 + cycle, 26, d).bfloat16().cuda()
        y = layer_pass(P, w, x, cache, blocks, window, recent, torch.from_numpy(depth).cuda(), torch.from_numpy(anc).cuda(),
                       torch.from_numpy(pos.astype(np.int32)).cuda(), plan, hq, hkv, hd)
        close(y, oracle(x, pos, blocks, recent, depth, anc))
        path = anc[int(np.argmax(depth))][:depth.max() + 1]             # the deepest path is accepted
        for t in window:
            t[recent:recent + len(path)] = t[recent + path].clone()
        recent += len(path)
        if recent >= 64:                                                # a block has filled
            P.spec_k_kv8_store(window[0][:64], window[1][:64], cache, blocks, hkv, hd)
            for t in window:
                t[:recent - 64] = t[64:recent].clone()
        committed += len(path)


def test_layer_example_of_the_readme_runs(P):
    """Its code as it stands, twice: the rows of the path are in the window, and then in a block."""
    import pathlib
    import re
    readme = (pathlib.Path(__file__).resolve().parent.parent / "README.md").read_text()
    code, = [c for c in re.findall(r"```python\n(.*?)```", readme, re.S) if "spec_k_attention8" in c]
    hq, hkv, hd, d, rows, recent = 8, 2, 128, 256, 10, 62
    depth, anc = tree(rows, 2)
    path = torch.from_numpy(anc[int(np.argmax(depth))][:depth.max() + 1].astype(np.int64)).cuda()
    w = {"qkv": P.spec_pack_weight8(rand(1, (hq + 2 * hkv) * hd, d, scale=0.05).bfloat16().cuda()), "o": P.spec_pack_weight8(rand(2, d, hq * hd, scale=0.05).bfloat16().cuda())}
    kwin, vwin = (rand(i, 128, hkv * hd).bfloat16().cuda() for i in (3, 4))
    env = dict(torch=torch, P=P, hq=hq, hkv=hkv, hd=hd, max_tokens=640, rows=rows, w=w, x=rand(5, rows, d).bfloat16().cuda(), kwin=kwin, vwin=vwin, blocks=0, recent=recent, path=path,
               depth=torch.from_numpy(depth).cuda(), anc=torch.from_numpy(anc).cuda(), deepest=int(depth.max()), pos=torch.from_numpy((recent + depth).astype(np.int32)).cuda())
    exec(code, env)
    n = recent + len(path)
    assert env["y"].shape == (rows, d) and env["y"].isfinite().all()
    kept, at = (n - 64, 64) if n >= 64 else (n, 0)
    assert (env["blocks"], env["recent"]) == (int(n >= 64), kept)
    turned = P.spec_k_rotary(env["plan"], [env["k"]], env["pos"], out_dtypes=[torch.bfloat16])[0].view(rows, -1)
    assert n >= 64 and torch.equal(kwin[:kept], turned[path][at - recent:]) and torch.equal(vwin[:kept], env["v"].reshape(rows, -1).bfloat16()[path][at - recent:])
    block = P.spec_k_kv8_load(env["cache"], 0, 1, hkv, hd)[1]
    first = torch.cat([rand(4, 128, hkv * hd).bfloat16()[:recent].cuda(), env["v"].reshape(rows, -1).bfloat16()[path]])[:64]
    assert np.array_equal(f64(block), O.held_kv(f64(first), hkv, hd))
    exec(code.split("# once per layer")[1].split("\n", 1)[1], {**env, "pos": env["pos"] + len(path)})


def test_layer_on_a_stream_and_captured(P):
    """The same calls on a stream of their own, and captured and replayed with other work between: the bits of the eager calls."""
    hq, hkv, hd, d, rows, blocks, recent = 8, 2, 128, 512, 26, 5, 9
    w = {"qkv": P.spec_pack_weight8(rand(1, (hq + 2 * hkv) * hd, d, scale=0.05).bfloat16().cuda()), "o": P.spec_pack_weight8(rand(2, d, hq * hd, scale=0.05).bfloat16().cuda())}
    plan = P.spec_rotary_plan(hd, 1e4)
    k, v = (rand(s, 64 * blocks + recent, hkv * hd).bfloat16().cuda() for s in (4, 5))
    cache = P.spec_kv8_alloc(blocks, hkv, hd)
    window = [torch.zeros(recent + rows, hkv * hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    depth, anc = (torch.from_numpy(t).cuda() for t in tree(rows, 4))
    pos = (64 * blocks + recent + depth).to(torch.int32)
    x = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")

    def whole():
        P.spec_k_kv8_store(k[:64 * blocks], v[:64 * blocks], cache, 0, hkv, hd)
        for t, s in zip(window, (k, v)):
            t[:recent] = s[64 * blocks:]
        return layer_pass(P, w, x, cache, blocks, window, recent, depth, anc, pos, plan, hq, hkv, hd)

    inputs_ = [rand(20 + i, rows, d).bfloat16().cuda() for i in range(4)]
    want = []
    for t in inputs_:
        x.copy_(t)
        want.append(whole().clone())
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        x.copy_(inputs_[0])
        got = whole()
    stream.synchronize()
    assert torch.equal(got, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = whole()
    for i in (1, 2, 0, 3, 3):
        x.copy_(inputs_[i])
        cache.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        assert torch.equal(whole(), want[i])                            # eager work between the replays
        torch.cuda.synchronize()


def test_two_calls_of_each_at_once(P):
    """Two streams, each with inputs, outputs and scratch of its own: the bits of one call after the other."""
    hq, hkv, hd, d, blocks = 8, 2, 128, 640, 6
    w = P.spec_pack_weight8(rand(1, 900, d).bfloat16().cuda())
    plan = P.spec_rotary_plan(hd, 1e4)
    sides = []
    for i in range(2):
        rows = (40, 70)[i]
        q, k, v = inputs(rows, hq, hkv, hd, blocks, rows, 30 + i)
        sides.append(dict(x=rand(10 + i, rows, d).bfloat16().cuda(), q=q, k=k, v=v, cache=P.spec_kv8_alloc(blocks, hkv, hd), depth=torch.arange(rows, dtype=torch.int32, device="cuda")))

    def run(s):
        rows, n = s["q"].shape[0], 64 * blocks
        y = P.spec_k_gemm8(s["x"], w)
        P.spec_k_kv8_store(s["k"][:n], s["v"][:n], s["cache"], 0, hkv, hd)
        q, k = P.spec_k_rotary(plan, [s["q"].view(rows, hq, hd), s["k"][n:].view(rows, hkv, hd)], n)
        return y, P.spec_k_attention8(q.view(rows, -1), s["cache"], blocks, k.view(rows, -1), s["v"][n:], n, s["depth"], None, hq, hkv, hd, max_depth=rows - 1)

    want = [run(s) for s in sides]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(5):
        got = []
        for s, stream in zip(sides, streams):
            with torch.cuda.stream(stream):
                got.append(run(s))
        torch.cuda.synchronize()
        for g, t in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, t))


def test_more_elements_than_31_bits_count(P):
    """Rows whose first element lies beyond 2^31 elements, against the same rows at the front."""
    m, k, rows = 270016, 8192, 8192
    base = rand(1, 64, k).bfloat16().cuda()
    w = P.spec_pack_weight8(rand(2, rows, k).bfloat16().cuda())
    y = P.spec_k_gemm8(base.repeat(m // 64, 1), w)
    assert torch.equal(y[-64:], y[:64]) and y[:64].isfinite().all() and float(y[:64].float().std()) > 1
    del y, w
    hq, hkv, hd, m = 128, 16, 128, 140032
    q, kv, vv = inputs(64, hq, hkv, hd, 1, 1, 7)
    cache = P.spec_kv8_alloc(1, hkv, hd)
    P.spec_k_kv8_store(kv[:64], vv[:64], cache, 0, hkv, hd)
    o = P.spec_k_attention8(q.repeat(m // 64, 1), cache, 1, kv[64:].contiguous(), vv[64:].contiguous(), 64, torch.zeros(m, dtype=torch.int32, device="cuda"), None, hq, hkv, hd, max_depth=0)
    assert torch.equal(o[-64:], o[:64])
    want, tol = attention_bound(q, kv, vv, 1, 64, np.zeros(64, np.int32), None, hq, hkv, hd)
    assert (np.abs(f64(o[:64]) - want) <= tol).all()
    del o
    x = rand(3, 64, 64, 128).bfloat16().cuda().repeat(4200, 1, 1)                       # 268800 rows
    pos = torch.arange(64, dtype=torch.int32, device="cuda").repeat(4200)
    r = P.spec_k_rotary(P.spec_rotary_plan(128, 1e4), [x], pos, outs=[x])[0]
    assert torch.equal(r[-64:], r[:64]) and not torch.equal(r[1], r[0])


def test_tensors_with_dims_beyond_32_bits_are_refused(P):
    """2^32 + n rows, dims or blocks are not n of them."""
    far = 2 ** 32
    base = torch.empty(far + 64, dtype=torch.bfloat16, device="cuda")
    one = P.spec_pack_weight8(torch.ones(1, 1, dtype=torch.bfloat16, device="cuda"))
    plan, none = P.spec_rotary_plan(64, 1e4), P.spec_rotary_plan(0, 1e4)
    q, k, v = inputs(1, 1, 1, 64, 1, 1, 1)
    cache, d = P.spec_kv8_alloc(1, 1, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in (lambda: P.spec_pack_weight8(base.view(-1, 1)), lambda: P.spec_pack_weight8(base.view(1, -1)), lambda: P.spec_k_gemm8(base.view(-1, 1), one),
                 lambda: P.spec_k_rotary(none, [base.view(-1, 1, 1)], 0, outs=[base.view(-1, 1, 1)]), lambda: P.spec_k_rotary(none, [base.view(1, -1, 1)], 0, outs=[base.view(1, -1, 1)]),
                 lambda: P.spec_k_rotary(plan, [base.view(1, 1, -1)], 0, outs=[base.view(1, 1, -1)]),
                 lambda: P.spec_k_attention8(q, cache, -far, k[:1], v[:1], 0, d, None, 1, 1, 64, max_depth=0), lambda: P.spec_k_attention8(q, cache, -1, k[:1], v[:1], 0, d, None, 1, 1, 64)):
        with pytest.raises(P.SpecError):
            call()


def test_rotary_ahead_of_and_behind_training_attention(P):
    """q and k of a training step turned ahead of spec_hca_attention; relative positions alone matter, so a shift of all positions changes nothing but roundings."""
    b, s, hq, hkv, hd = 2, 96, 4, 2, 64
    plan = P.spec_rotary_plan(hd, 1e4)
    q, k, v = (rand(i, b * s, h, hd).bfloat16().cuda() for i, h in ((1, hq), (2, hkv), (3, hkv)))
    outs = []
    for shift in (0, 50000):
        pos = (torch.arange(b * s, device="cuda") % s + shift).to(torch.int32)
        qr, kr = P.spec_k_rotary(plan, [q, k], pos)
        outs.append(P.spec_hca_attention(qr.view(b, s, hq, hd), [kr.view(b, s, hkv, hd)], [v.view(b, s, hkv, hd)]))
    # roundings of q, k (u16 each, both runs) move a score by at most 4 u16 |q| |k| / sqrt(hd), a weight by twice that
    size = float(q.float().norm(dim=-1).max() * k.float().norm(dim=-1).max()) / math.sqrt(hd)
    assert float((outs[0].float() - outs[1].float()).abs().max()) <= (8 * U16 * size + 4 * U16) * float(v.float().abs().max())
