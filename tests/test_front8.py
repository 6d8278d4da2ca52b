"""The 8-bit front end (bmlp_quantize_rows, bmlp_norm_quantize, bmlp_int8_matmul,
bmlp_int8_sign) against the formulas in 64 bits, at the sizes, strides, values and
types where it can go wrong, and its refusals.

Sums of products of codes are integers below 2^53, so the 64-bit reference has
them exactly and outputs are compared for equality: int32 sums and signs as they
are, scaled outputs after the same fp32 operations, rounded one by one."""
import numpy as np
import pytest
import torch

import oracle as O
import workloads as W
from paper_2412_00119_gb300 import bmlp as B

DEV = "cuda:0"
gpu = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-6
LEAST = 127 * 2.0 ** -126


@pytest.fixture(autouse=True)
def _device(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            pytest.skip("needs a GPU")
        torch.cuda.set_device(DEV)


def rows(n, K, dtype, pad=0, off=0, fill=0):
    """An n x K view whose rows are K + pad apart and start off elements into a buffer."""
    buf = torch.full((off + n * (K + pad) + 8,), fill, dtype=dtype, device=DEV)
    return buf, buf[off:off + n * (K + pad)].view(n, K + pad)[:, :K]


def hidden(n, K, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, K), generator=g) * torch.exp(torch.randn((n, 1), generator=g))
    x[:, torch.rand((K,), generator=g) < 0.02] *= 16
    return x.to(dtype)


def codes(n, K, seed, kind="full"):
    g = torch.Generator().manual_seed(seed)
    if kind == "low":
        return torch.full((n, K), -128, dtype=torch.int8)
    if kind == "high":
        return torch.full((n, K), 127, dtype=torch.int8)
    if kind == "ends":
        return (torch.randint(0, 2, (n, K), generator=g) * 255 - 128).to(torch.int8)
    return torch.randint(-128, 128, (n, K), generator=g).to(torch.int8)


def sums64(a, w):
    return a.to(DEV).double() @ w.to(DEV).double().t()


# -- quantisation ------------------------------------------------------------------

def plain_codes(x, res=None, gain=None):
    """Codes by the same fp32 operations one by one, on the CPU; and u in 64 bits."""
    h = x.float() if res is None else x.float() + res.float()
    u = h if gain is None else h * gain.float()
    most = u.abs().amax(1, keepdim=True)
    ok = torch.isfinite(u).all(1, keepdim=True) & (most >= LEAST)
    q = torch.round(torch.where(ok, u, 0) * (torch.full_like(most, 127.0) / torch.where(ok, most, 1)))
    return h, q.to(torch.int8)


def check_codes(q, scale, x, res, gain, norm, K):
    h64 = x.double() if res is None else x.double() + res.double()
    u64 = h64 if gain is None else h64 * gain.double()
    A = u64.abs().amax(1, keepdim=True)
    # u carries at most two fp32 roundings, A two, 127 / A one, the product one
    ideal = u64 * 127 / torch.where(A > 0, A, 1)
    assert ((q.double() - ideal).abs() <= 0.5 + 127 * 6 * 2.0 ** -24).all()
    want = A[:, 0] / 127
    if norm:
        want = want / torch.sqrt((h64 * h64).mean(1) + EPS)
    # roundings: u (2), A / 127, mean, + eps, sqrt, 1 / it, product; h^2 and its sum of
    # at most K / 256 + 16 additions in sequence, halved by the root
    tol = (10 + (K / 256 + 20) / 2) * 2.0 ** -24
    assert ((scale.double() - want).abs() <= tol * want).all()


SHAPES = [(1, 1), (1, 2), (3, 7), (2, 31), (5, 32), (4, 33), (9, 64), (3, 100), (1, 255), (2, 256), (17, 257),
          (6, 784), (3, 1000), (3, 1001), (2, 1024), (2, 2047), (300, 129), (1, 4096), (3, 5003), (1, 8192), (2, 8193),
          (2, 16384), (1, 16400), (2, 33000), (1, 70001)]


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", SHAPES)
def test_norm_quantize(n, K, dtype):
    for variant, (pad, off) in enumerate([(0, 0), (8, 8), (3, 1)]):
        x, res = hidden(n, K, 3 * n + K, dtype), hidden(n, K, n + 5 * K, dtype)
        gain = (1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to(dtype)
        use_res, use_gain, use_sum = variant != 1, variant != 2, variant != 1
        xb, xd = rows(n, K, dtype, pad, off)
        rb, rd = rows(n, K, dtype, 2 * pad, off)
        sb, sd = rows(n, K, dtype, pad, 2 * off, fill=7)
        qb, qd = rows(n, K, torch.int8, pad, off, fill=99)
        xd.copy_(x)
        rd.copy_(res)
        scale = torch.full((n,), -1.0, device=DEV)
        B.bmlp_norm_quantize(xd, gain.to(DEV) if use_gain else None, qd, scale, res=rd if use_res else None,
                             sum_out=sd if use_sum else None, eps=EPS)
        r, g = res if use_res else None, gain if use_gain else None
        h, want = plain_codes(x, r, g)
        q = qd.cpu()
        assert torch.equal(q, want)
        check_codes(q, scale.cpu(), x, r, g, True, K)
        if use_sum:
            assert torch.equal(sd.cpu(), h.to(dtype))
            assert (sb[:2 * off] == 7).all() and (sb[2 * off + n * (K + pad):] == 7).all()
            if pad:
                assert (sb[2 * off:2 * off + n * (K + pad)].view(n, -1)[:, K:] == 7).all()
        if pad:
            assert (qb[off:off + n * (K + pad)].view(n, -1)[:, K:] == 99).all()
        assert (qb[:off] == 99).all() and (qb[off + n * (K + pad):] == 99).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", SHAPES)
def test_quantize_rows(n, K, dtype):
    for pad, off in [(0, 0), (8, 8), (5, 3)]:
        x = hidden(n, K, n + K, dtype)
        _, xd = rows(n, K, dtype, pad, off)
        qb, qd = rows(n, K, torch.int8, pad, off, fill=99)
        xd.copy_(x)
        scale = torch.full((n,), -1.0, device=DEV)
        B.bmlp_quantize_rows(xd, qd, scale)
        q = qd.cpu()
        assert torch.equal(q, plain_codes(x)[1])
        check_codes(q, scale.cpu(), x, None, None, False, K)
        assert (qb[:off] == 99).all() and (qb[off + n * (K + pad):] == 99).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K", [8, 100, 1024, 5000, 40000])
def test_quantize_special_rows(K, dtype):
    """Rows of zeros, of the type's largest and least values, of one value, with infinities
    and NaNs: alone in their rows' outputs."""
    big = torch.finfo(dtype).max
    x = hidden(12, K, K, dtype)
    x[0] = 0
    x[1] = big
    x[2, :] = -big
    x[3] = 0
    x[3, K // 2] = float("nan")
    x[4, K - 1] = float("inf")
    x[5, 0] = -float("inf")
    x[6] = 0
    x[6, K - 1] = 2.0 ** -130 if dtype != torch.float16 else 2.0 ** -24
    x[7] = 3
    x[8, 0] = float("inf")
    x[8, 1] = float("nan")
    x[9] = -0.0
    x[10] = 0
    x[10, 1] = float(torch.finfo(dtype).tiny)
    for norm in (False, True):
        q = torch.full((12, K), 99, dtype=torch.int8, device=DEV)
        scale = torch.full((12,), -1.0, device=DEV)
        if norm:
            s = torch.empty((12, K), dtype=dtype, device=DEV)
            B.bmlp_norm_quantize(x.to(DEV), None, q, scale, sum_out=s, eps=EPS)
            got, raw = s.cpu(), torch.int32 if dtype == torch.float32 else torch.int16
            assert torch.equal(torch.isnan(got), torch.isnan(x))    # (a NaN's payload is free)
            assert torch.equal(got.view(raw)[~torch.isnan(x)], x.view(raw)[~torch.isnan(x)])
        else:
            B.bmlp_quantize_rows(x.to(DEV), q, scale)
        q, scale = q.cpu(), scale.cpu()
        bad = [3, 4, 5, 8]
        if norm and dtype != torch.float16:
            bad += [1, 2]   # their sum of squares is not finite
        want = plain_codes(x)[1]
        for i in range(12):
            if i in bad:
                assert torch.isnan(scale[i]) and (q[i] == 0).all(), i
            else:
                assert torch.isfinite(scale[i]) and scale[i] >= 0, i
                assert torch.equal(q[i], want[i]), i
        assert scale[0] == 0 and scale[9] == 0
        if dtype != torch.float16:
            assert scale[6] == 0 and scale[10] == 0
        else:
            assert scale[6] > 0 and (q[6, K - 1] == 127) and scale[10] > 0


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", [(1, 4097), (3, 8184), (330, 513), (2500, 517), (611, 784), (400, 1001), (701, 2047), (330, 4096),
                                 (311, 8180), (5, 16376)])
def test_norm_with_sums_that_lie_elsewhere(n, K, dtype):
    """Inputs whose rows start alike, sums that start otherwise, in some rows or in all."""
    for pad, off, spad, soff in [(1, 0, 0, 0), (3, 5, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (7, 2, 16, 2), (2, 8, 5, 3)]:
        x, res = hidden(n, K, n + K, dtype), hidden(n, K, n + 5 * K, dtype)
        xd, rd = (rows(n, K, dtype, pad, off)[1] for _ in range(2))
        sb, sd = rows(n, K, dtype, spad, soff, fill=7)
        qb, qd = rows(n, K, torch.int8, spad, soff, fill=99)
        xd.copy_(x)
        rd.copy_(res)
        scale = torch.full((n,), -1.0, device=DEV)
        B.bmlp_norm_quantize(xd, None, qd, scale, res=rd, sum_out=sd, eps=EPS)
        h, want = plain_codes(x, res)
        assert torch.equal(qd.cpu(), want)
        check_codes(qd.cpu(), scale.cpu(), x, res, None, True, K)
        assert torch.equal(sd.cpu(), h.to(dtype))
        for b, fill in ((sb, 7), (qb, 99)):
            assert (b[:soff] == fill).all() and (b[soff + n * (K + spad):] == fill).all()
            assert (b[soff:soff + n * (K + spad)].view(n, -1)[:, K:] == fill).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K", [96, 1001, 8192, 40000])
def test_norm_in_place(K, dtype):
    n = 5
    x, res = hidden(n, K, 1, dtype), hidden(n, K, 2, dtype)
    h, want = plain_codes(x, res)
    for which in (0, 1):
        xd, rd = x.to(DEV), res.to(DEV)
        q = torch.empty((n, K), dtype=torch.int8, device=DEV)
        scale = torch.empty((n,), device=DEV)
        B.bmlp_norm_quantize(xd, None, q, scale, res=rd, sum_out=(xd, rd)[which], eps=EPS)
        assert torch.equal((xd, rd)[which].cpu(), h.to(dtype)) and torch.equal(q.cpu(), want)
        assert torch.equal((rd, xd)[which].cpu(), (res, x)[which])


@gpu
def test_norm_overflow_in_the_addition():
    """fp16 inputs whose sum leaves fp16 but not fp32: coded; sum_out is infinite."""
    x = torch.full((2, 64), 60000.0, dtype=torch.float16)
    x[1] = 1
    q = torch.empty((2, 64), dtype=torch.int8, device=DEV)
    scale = torch.empty((2,), device=DEV)
    s = torch.empty((2, 64), dtype=torch.float16, device=DEV)
    B.bmlp_norm_quantize(x.to(DEV), None, q, scale, res=x.to(DEV), sum_out=s, eps=0.0)
    assert (q == 127).all() and torch.isinf(s[0]).all() and (s[1] == 2).all()
    assert ((scale.cpu() - 1 / 127).abs() < 1e-8).all()


# -- products ----------------------------------------------------------------------

def run_all(a, w, K, N, seed, pad, off, thr=None):
    """Every output type and the signs of a w^T, compared with the 64-bit sums."""
    n = a.shape[0]
    g = torch.Generator().manual_seed(seed)
    _, ad = rows(n, K, torch.int8, pad, off, fill=-77)
    _, wd = rows(N, K, torch.int8, pad, off, fill=-78)
    ad.copy_(a)
    wd.copy_(w)
    S = sums64(a, w)
    ob, od = rows(n, N, torch.int32, pad, off, fill=-5)
    B.bmlp_int8_matmul(ad, wd, od)
    assert torch.equal(od.double(), S)
    assert (ob[:off] == -5).all() and (ob[off + n * (N + pad):] == -5).all()
    if pad:
        assert (ob[off:off + n * (N + pad)].view(n, -1)[:, N:] == -5).all()
    sa = torch.exp(torch.randn((n,), generator=g)).to(DEV) / 100
    sw = torch.exp(torch.randn((N,), generator=g)).to(DEV) / 100
    bias = torch.randn((N,), generator=g).to(DEV) * 10
    y = S.float() * sa[:, None] * sw + bias       # (S exact, each step rounded to fp32)
    for dtype in TYPES:
        ob, od = rows(n, N, dtype, pad, off, fill=-5)
        B.bmlp_int8_matmul(ad, wd, od, sa, sw, bias)
        assert torch.equal(od, y.to(dtype)), dtype
        assert (ob[:off] == -5).all() and (ob[off + n * (N + pad):] == -5).all()
    out = torch.full((n, N), -1.0, device=DEV)
    B.bmlp_int8_matmul(ad, wd, out, a_scale=sa)
    assert torch.equal(out, S.float() * sa[:, None])
    B.bmlp_int8_matmul(ad, wd, out, w_scale=sw)
    assert torch.equal(out, S.float() * sw)
    thr = thr if thr is not None else S[0].to(torch.int32)    # the first row's own sums: its bits are 1
    for t in (None, thr):
        want = S >= (0 if t is None else t.double())
        words = torch.full((n, W.words(N)), -1, dtype=torch.int64, device=DEV)
        B.bmlp_int8_sign(ad, wd, words, t)
        got = words.cpu().numpy().view(np.uint64)
        assert np.array_equal(got, W.pack(np.where(want.cpu().numpy(), 1, -1)))


NS = [1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 17, 24, 31, 33, 48, 64, 65, 100, 127, 128, 129, 192, 200, 255, 257, 300, 513]
KS = [1, 2, 3, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 511, 784, 1000, 1001, 1023, 1024,
      1025, 1040, 2047, 2049, 4096, 5003]
CH = [1, 2, 7, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 525, 1024, 2050]


@gpu
@pytest.mark.parametrize("n", NS)
def test_product_over_rows(n):
    for i, (K, N) in enumerate([(129, 70), (1000, 300), (4096, 257)]):
        run_all(codes(n, K, n), codes(N, K, K), K, N, n, *[(0, 0), (16, 16), (5, 3)][(i + n) % 3])


@gpu
@pytest.mark.parametrize("K", KS)
def test_product_over_depth(K):
    for i, (n, N) in enumerate([(1, 130), (6, 65), (70, 33), (260, 300)]):
        run_all(codes(n, K, n), codes(N, K, K), K, N, n, *[(0, 0), (16, 0), (7, 1)][(i + K) % 3])


@gpu
@pytest.mark.parametrize("N", CH)
def test_product_over_channels(N):
    for i, (n, K) in enumerate([(1, 200), (3, 1040), (40, 96), (150, 784)]):
        run_all(codes(n, K, n), codes(N, K, K), K, N, n, *[(0, 0), (32, 16), (1, 7)][(i + N) % 3])


@gpu
@pytest.mark.parametrize("kinds", [("low", "low"), ("low", "high"), ("high", "high"), ("ends", "ends"), ("ends", "low")])
@pytest.mark.parametrize("n", [1, 3, 10, 40, 150, 600])
def test_product_of_extreme_codes(n, kinds):
    """Sums far past 2^24 are exact too, up to the longest rows."""
    for K, N in [(1024, 64), (1041, 70), (4100, 300), (16384, 130)]:
        run_all(codes(n, K, 1, kinds[0]), codes(N, K, 2, kinds[1]), K, N, n, 0, 0)
    if n in (1, 10, 150):
        K = B.BMLP_INT8_MAX_K
        run_all(codes(n, K, 1, kinds[0]), codes(40, K, 2, kinds[1]), K, 40, n, 1 if n == 10 else 0, 0)


@gpu
@pytest.mark.parametrize("n,K,N", [(2000, 1500, 1000), (4097, 2049, 515), (1000, 1000, 525), (700, 8192, 4100),
                                   (20000, 130, 300), (33, 4096, 20000), (1, 9000, 20011), (2, 16384, 4096), (100, 4096, 8192)])
def test_product_of_many_tiles(n, K, N):
    run_all(codes(n, K, n, "ends"), codes(N, K, K), K, N, n, 0, 0)


@gpu
def test_thresholds_at_the_ends_of_int32():
    K, N = 200, 6
    thr = torch.tensor([-2 ** 31, 2 ** 31 - 1, 0, 1, -1, 5], dtype=torch.int32, device=DEV)
    for n in (1, 20, 200):
        a, w = codes(n, K, 4), codes(N, K, 5)
        w[2] = 0          # sums of 0: bit 1 at threshold 0
        w[3] = 0
        w[4] = 0
        run_all(a, w, K, N, n, 0, 0, thr)


@gpu
@pytest.mark.parametrize("n,K,N", [(2500, 1024, 4000), (3000, 1025, 4000), (5000, 1024, 60), (9000, 300, 100), (70, 1024, 300)])
def test_thresholds_about_two_to_the_24(n, K, N):
    """Sums up to 2^24 against thresholds at and past it, in every kernel that compares them in
    fp32 or whose lanes are rows."""
    a, w = codes(n, K, 1, "ends"), codes(N, K, 2, "ends")
    a[:5], w[:5] = -128, -128
    a[5:8], w[5:8] = 127, -128
    g = torch.Generator().manual_seed(3)
    near = torch.tensor([0, 1, -1, 2 ** 24, 2 ** 24 - 1, 2 ** 24 + 1, 2 ** 24 + 2, -2 ** 24, -2 ** 24 - 1, -2 ** 24 + 1,
                         2 ** 31 - 1, -2 ** 31, 127 * -128 * K, 128 * 128 * K])
    thr = near[torch.randint(0, len(near), (N,), generator=g)].to(torch.int32).to(DEV)
    run_all(a, w, K, N, 7, 0, 0, thr)


@gpu
@pytest.mark.parametrize("n,K,N", [(1000, 64, 20), (3000, 200, 31), (17871, 646, 78), (5000, 1100, 100), (9000, 79, 129),
                                   (40000, 88, 105), (2615, 3000, 42), (700, 4096, 64), (3333, 4100, 33)])
def test_many_rows_and_few_channels(n, K, N):
    """Where rows and channels change places inside: strides, biases and thresholds too."""
    for pad, off in [(0, 0), (16, 16), (3, 1)]:
        run_all(codes(n, K, n, "ends"), codes(N, K, K), K, N, n, pad, off)


@gpu
@pytest.mark.parametrize("n", [1, 2, 20, 130, 400])
def test_scales_that_are_not_finite(n):
    """A row's NaN scale (a row that could not be coded) reaches its outputs and no others;
    products that leave the output's type become infinite."""
    K, N = 300, 140
    a, w = codes(n, K, 1).to(DEV), codes(N, K, 2).to(DEV)
    sa = torch.ones((n,), device=DEV)
    sa[n // 2] = float("nan")
    sw = torch.ones((N,), device=DEV)
    sw[3] = float("inf")
    sw[5] = 1e30
    out = torch.zeros((n, N), dtype=torch.float16, device=DEV)
    B.bmlp_int8_matmul(a, w, out, sa, sw)
    want = (sums64(a, w).float() * sa[:, None] * sw).half()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.isnan(out[n // 2]).all()
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))


@gpu
@pytest.mark.parametrize("n", [2, 20, 150])
def test_offsets_past_32_bits(n):
    """Rows 2^31 elements and more apart in every operand."""
    K, N = 70, 40
    far = (2 ** 32 // (n - 1) + 15) // 16 * 16 + 16
    abuf = torch.zeros(far * (n - 1) + K, dtype=torch.int8, device=DEV)
    a = abuf.as_strided((n, K), (far, 1))
    a.copy_(codes(n, K, 9))
    wfar = 2 ** 32 // (N - 1) + 17
    wbuf = torch.zeros(wfar * (N - 1) + K, dtype=torch.int8, device=DEV)
    w = wbuf.as_strided((N, K), (wfar, 1))
    w.copy_(codes(N, K, 8))
    obuf = torch.zeros(far * (n - 1) + N, dtype=torch.float16, device=DEV)
    out = obuf.as_strided((n, N), (far, 1))
    B.bmlp_int8_matmul(a, w, out, torch.full((n,), 1 / 512, device=DEV))
    assert torch.equal(out, (sums64(a, w).float() / 512).half())
    words = torch.zeros((n, 1), dtype=torch.int64, device=DEV)
    B.bmlp_int8_sign(a, w, words)
    assert np.array_equal(words.cpu().numpy().view(np.uint64), W.pack(np.where(sums64(a, w).cpu().numpy() >= 0, 1, -1)))
    x = obuf.as_strided((n, N), (far, 1))
    q = abuf.as_strided((n, N), (far, 1))
    scale = torch.zeros((n,), device=DEV)
    want = plain_codes(x.cpu())[1]
    B.bmlp_quantize_rows(x, q, scale)
    assert torch.equal(q.cpu(), want)


@gpu
@pytest.mark.parametrize("n,K,N", [(9000, 512, 128), (5000, 640, 96), (20000, 300, 64), (6000, 304, 48), (30000, 130, 256)])
def test_many_rows_and_few_channels_in_whole_vectors(n, K, N):
    run_all(codes(n, K, n, "ends"), codes(N, K, K), K, N, n, 0, 0)


@gpu
@pytest.mark.parametrize("n,K,N", [(5000, 300, 60), (4500, 1500, 120)])
def test_offsets_past_32_bits_of_many_rows(n, K, N):
    """Few channels: rows and channels change places; the last rows lie past 2^32 elements."""
    far = 2 ** 32 // (n - 1) + 5
    abuf = torch.zeros(far * (n - 1) + K, dtype=torch.int8, device=DEV)
    a = abuf.as_strided((n, K), (far, 1))
    a.copy_(codes(n, K, 9))
    w = codes(N, K, 8).to(DEV)
    obuf = torch.zeros(far * (n - 1) + N, dtype=torch.float16, device=DEV)
    out = obuf.as_strided((n, N), (far, 1))
    B.bmlp_int8_matmul(a, w, out, torch.full((n,), 2.0 ** -16, device=DEV))
    assert torch.equal(out, (sums64(a, w).float() * 2.0 ** -16).half())
    words = torch.zeros((n, W.words(N)), dtype=torch.int64, device=DEV)
    B.bmlp_int8_sign(a, w, words)
    assert np.array_equal(words.cpu().numpy().view(np.uint64), W.pack(np.where(sums64(a, w).cpu().numpy() >= 0, 1, -1)))


@gpu
def test_streams_and_capture():
    """On a stream of its own, and replayed from a graph on new inputs."""
    n, K, N = 37, 512, 200
    s = torch.cuda.Stream()
    x = torch.empty((n, K), dtype=torch.bfloat16, device=DEV)
    w = codes(N, K, 3).to(DEV)
    q = torch.empty((n, K), dtype=torch.int8, device=DEV)
    scale = torch.empty((n,), device=DEV)
    out = torch.empty((n, N), device=DEV)

    def call(stream=None):
        B.bmlp_norm_quantize(x, None, q, scale, eps=EPS, stream=stream)
        B.bmlp_int8_matmul(q, w, out, scale, stream=stream)

    def check():
        torch.cuda.synchronize()
        assert torch.equal(q.cpu(), plain_codes(x.cpu())[1])
        assert torch.equal(out, sums64(q, w).float() * scale[:, None])

    x.copy_(hidden(n, K, 1))
    torch.cuda.synchronize()
    call(s)
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (2, 3):
        x.copy_(hidden(n, K, seed))
        out.fill_(0)
        g.replay()
        check()


# sizes whose kernel is, in turn: the streamed one; 32-row tiles (K shared by eight, one CTA);
# 64- and 128-row tiles of ready activations (with and without sharing K; two rounds); pairs
PLANS = [(5, 300, 100), (20, 2048, 300), (31, 100, 19500), (50, 8192, 8192), (64, 8000, 7000), (100, 4096, 8192),
         (120, 8191, 4096), (300, 2300, 9000), (700, 4096, 4096), (1500, 1024, 8192), (2100, 1001, 6000)]


@gpu
@pytest.mark.parametrize("n,K,N", PLANS)
def test_every_plan(n, K, N):
    run_all(codes(n, K, n, "ends"), codes(N, K, K), K, N, n, 0, 0)


@gpu
@pytest.mark.parametrize("n,K,N", [(12, 200, 300), (20, 2048, 300), (50, 4096, 4000), (100, 2048, 4096), (300, 3000, 2000),
                                   (1500, 1024, 8192), (4000, 1500, 50), (4000, 3000, 120)])
def test_expired_waits_cost_time_only(n, K, N):
    """With every CTA's wait taken as expired the sums are made again, whole; without a
    workspace too."""
    a, w = codes(n, K, n).to(DEV), codes(N, K, K).to(DEV)
    S = sums64(a, w)
    for ws in (None, torch.empty(16, dtype=torch.uint8, device=DEV)):
        out = torch.full((n, N), -3, dtype=torch.int32, device=DEV)
        B.bmlp_int8_matmul(a, w, out, workspace=ws, expired=True)
        assert torch.equal(out.double(), S)
        out.fill_(-3)
        B.bmlp_int8_matmul(a, w, out, workspace=ws)     # the device is as it was
        assert torch.equal(out.double(), S)


# a few tiles, whose K eight CTAs share, and one tile more
SHARED = [(20, 2048, 1536), (20, 2047, 1537), (12, 9000, 40), (21, 14142, 384), (60, 4096, 700), (100, 5000, 200), (200, 8192, 128)]


@gpu
@pytest.mark.parametrize("n,K,N", SHARED)
def test_depth_shared_by_eight(n, K, N):
    run_all(codes(n, K, n, "ends"), codes(N, K, K), K, N, n, 0, 0)
    a, w = codes(n, K, n).to(DEV), codes(N, K, K).to(DEV)
    out = torch.full((n, N), -3, dtype=torch.int32, device=DEV)
    for expired in (True, False):
        B.bmlp_int8_matmul(a, w, out, expired=expired)
        assert torch.equal(out.double(), sums64(a, w))


@gpu
@pytest.mark.parametrize("n,K,N", [(40, 3000, 5000), (100, 4096, 8192), (300, 2304, 4000), (1500, 1024, 8192), (4000, 1500, 100)])
def test_workspaces(n, K, N):
    """Given, too small, misaligned, kept, on other streams: the same sums."""
    a, w = codes(n, K, n).to(DEV), codes(N, K, K).to(DEV)
    S = sums64(a, w)
    size = B.bmlp_int8_workspace(n, K, N)
    out = torch.empty((n, N), dtype=torch.int32, device=DEV)

    def check():
        torch.cuda.synchronize()
        assert torch.equal(out.double(), S)
        out.fill_(-3)

    for bytes_ in (size, max(size - 1, 16), 16):
        ws = torch.full((bytes_,), 0x7F, dtype=torch.uint8, device=DEV)     # (fp16 NaNs)
        B.bmlp_int8_matmul(a, w, out, workspace=ws)
        check()
    if size:
        with pytest.raises(B.BmlpError):
            B.bmlp_int8_matmul(a, w, out, workspace=torch.empty(size + 16, dtype=torch.uint8, device=DEV)[1:])
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty((n, N), dtype=torch.int32, device=DEV) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                B.bmlp_int8_matmul(a, w, o)
        for s, o in zip(streams, outs):
            B.bmlp_int8_matmul(a, w, o, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.double(), S)
    B.bmlp_int8_matmul(a, w, out)
    check()
    B.bmlp_release_workspaces()
    B.bmlp_int8_matmul(a, w, out)
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.bmlp_int8_matmul(a, w, out)
    B.bmlp_release_workspaces()
    junk = torch.full((max(size, 16),), 0x7F, dtype=torch.uint8, device=DEV)
    out.fill_(-3)
    g.replay()
    check()
    del junk


@gpu
def test_back_to_back_calls_do_not_mix():
    """Calls that depend on one another, with nothing between them: each kernel may start while
    the one before it ends."""
    n, K = 200, 512
    a, w1, w2 = codes(n, K, 1).to(DEV), codes(K, K, 2).to(DEV), codes(96, K, 3).to(DEV)
    y = torch.empty((n, K), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((n, K), dtype=torch.int8, device=DEV)
    q2 = torch.empty((n, K), dtype=torch.int8, device=DEV)
    s = torch.empty((n,), device=DEV)
    out = torch.empty((n, 96), dtype=torch.int32, device=DEV)
    want = None
    for rep in range(30):
        for rows in (n, 3, 20, 70):
            B.bmlp_int8_matmul(a[:rows], w1, y[:rows], None, None)
            B.bmlp_quantize_rows(y[:rows], q[:rows], s[:rows])
            B.bmlp_int8_matmul(q[:rows], w1, y[:rows])
            B.bmlp_norm_quantize(y[:rows], None, q2[:rows], s[:rows])
            B.bmlp_int8_matmul(q2[:rows], w2, out[:rows])
        torch.cuda.synchronize()
        if want is None:
            S1 = sums64(a, w1).float().bfloat16()
            c1 = plain_codes(S1.cpu())[1]
            c2 = plain_codes(sums64(c1, w1).float().bfloat16().cpu())[1]
            want = sums64(c2, w2)
        assert torch.equal(out.double(), want), rep


@gpu
def test_front_end_feeds_training():
    """Hidden states -> norm -> 8-bit product's signs -> training and prediction, equal to the
    oracle trained on the reference's words; the whole chain on one stream."""
    n, D, K = 300, 96, 130
    x, res = hidden(n, D, 1, torch.bfloat16), hidden(n, D, 2, torch.bfloat16)
    wf = 0.02 * torch.randn((K, D), generator=torch.Generator().manual_seed(3))
    q = torch.empty((n, D), dtype=torch.int8, device=DEV)
    scale = torch.empty((n,), device=DEV)
    w = torch.empty((K, D), dtype=torch.int8, device=DEV)
    w_scale = torch.empty((K,), device=DEV)
    words = torch.empty((n, W.words(K)), dtype=torch.int64, device=DEV)
    y = torch.from_numpy(np.arange(n, dtype=np.int32) % 4).to(DEV)
    B.bmlp_quantize_rows(wf.to(DEV), w, w_scale)
    B.bmlp_norm_quantize(x.to(DEV), None, q, scale, res=res.to(DEV), eps=EPS)
    B.bmlp_int8_sign(q, w, words)
    m = B.BMLP([K, 64], 4, seed=5, bs=50)
    errs = m.train(words, y, epoch_end=True, count_errors=True)
    out = torch.empty((n,), dtype=torch.int32, device=DEV)
    m.predict(words, out)
    qw = plain_codes(x, res)[1].double() @ plain_codes(wf)[1].double().t()
    pm1 = np.where(qw.numpy() >= 0, 1, -1).astype(np.int8)
    ref = O.OracleModel([K, 64], 4, seed=5, bs=50)
    assert errs == ref.train(pm1, y.cpu().numpy(), epoch_end=True)
    assert np.array_equal(out.cpu().numpy(), ref.predict(pm1))
    m.close()


# -- refusals ------------------------------------------------------------------------

def test_quantize_refusals():
    lib = B.lib()
    x = np.zeros((4, 8), np.float32)
    q = np.zeros((4, 8), np.int8)
    sc = np.zeros(4, np.float32)
    px, pq, ps = x.ctypes.data, q.ctypes.data, sc.ctypes.data

    def rows_call(ptr=px, typ=B.BMLP_F32, ldx=8, n=4, K=8, qp=pq, ldq=8, sp=ps):
        return lib.bmlp_quantize_rows(ptr, typ, ldx, n, K, qp, ldq, sp, None)

    def norm_call(ptr=px, ldx=8, res=None, ldr=0, gain=None, typ=B.BMLP_F32, n=4, K=8, eps=1e-6, sm=None, lds=0):
        return lib.bmlp_norm_quantize(ptr, ldx, res, ldr, gain, typ, n, K, eps, sm, lds, pq, 8, ps, None)

    def refused(rc, text):
        assert rc == B.BMLP_EINVAL and text in B.bmlp_last_error(), B.bmlp_last_error()

    refused(rows_call(n=-1), "n < 0")
    refused(rows_call(K=0), "K < 1")
    refused(rows_call(typ=B.BMLP_I32), "x_type")
    refused(rows_call(typ=9), "x_type")
    refused(rows_call(ldx=7), "row stride")
    refused(rows_call(ldq=7), "row stride")
    refused(rows_call(), "device pointers")        # host memory
    refused(rows_call(ptr=None), "device pointers")
    assert rows_call(ptr=None, n=0) == B.BMLP_OK
    refused(norm_call(eps=-1.0), "eps")
    refused(norm_call(eps=float("nan")), "eps")
    refused(norm_call(eps=float("inf")), "eps")
    refused(norm_call(res=px, ldr=4), "row stride")
    refused(norm_call(sm=px, lds=4), "row stride")
    refused(norm_call(sm=px, lds=9), "in place")
    refused(norm_call(res=px, ldr=8), "device pointers")
    assert norm_call(n=0) == B.BMLP_OK


def test_product_refusals():
    lib = B.lib()
    a = np.zeros((4, 8), np.int8)
    f = np.zeros(8, np.float32)
    out = np.zeros((4, 4), np.float32)
    pa, pf, po = a.ctypes.data, f.ctypes.data, out.ctypes.data

    def mm(lda=8, ldw=8, n=4, K=8, N=4, typ=B.BMLP_F32, ldo=4, sa=None, sw=None, bias=None, o=po):
        return lib.bmlp_int8_matmul(pa, lda, sa, pa, ldw, sw, bias, n, K, N, o, typ, ldo, None, 0, None)

    def refused(rc, text):
        assert rc == B.BMLP_EINVAL and text in B.bmlp_last_error(), B.bmlp_last_error()

    refused(mm(n=-1), "n < 0")
    refused(mm(K=0), "K outside")
    refused(mm(K=B.BMLP_INT8_MAX_K + 1, lda=1 << 20, ldw=1 << 20), "K outside")
    refused(mm(N=0), "N < 1")
    refused(mm(typ=4), "out_type")
    refused(mm(typ=-1), "out_type")
    for kw in (dict(sa=pf), dict(sw=pf), dict(bias=pf)):
        refused(mm(typ=B.BMLP_I32, **kw), "no scales")
    refused(mm(lda=7), "row stride")
    refused(mm(ldw=7), "row stride")
    refused(mm(ldo=3), "row stride")
    refused(mm(), "device pointers")
    refused(mm(o=None), "device pointers")
    assert mm(n=0) == B.BMLP_OK
    assert lib.bmlp_int8_sign(pa, 8, pa, 8, None, 0, 8, 4, None, None, 0, None) == B.BMLP_OK
    refused(lib.bmlp_int8_sign(pa, 8, pa, 8, None, 4, 8, 4, None, None, 0, None), "device pointers")
    refused(lib.bmlp_int8_sign(pa, 7, pa, 8, None, 4, 8, 4, po, None, 0, None), "row stride")


def test_binding_refusals():
    """Shapes, types and strides that the binding turns away before the library is called."""
    t = torch.zeros
    with pytest.raises(TypeError):
        B.bmlp_quantize_rows(t((2, 8), dtype=torch.float64), t((2, 8), dtype=torch.int8), t(2))
    with pytest.raises(TypeError):
        B.bmlp_quantize_rows(t((2, 8)), t((2, 8), dtype=torch.uint8), t(2))
    with pytest.raises(ValueError):
        B.bmlp_quantize_rows(t((2, 8)), t((2, 7), dtype=torch.int8), t(2))
    with pytest.raises(ValueError):
        B.bmlp_quantize_rows(t((8, 2)).t(), t((2, 8), dtype=torch.int8), t(2))
    with pytest.raises(ValueError):
        B.bmlp_quantize_rows(t((2, 8)), t((2, 8), dtype=torch.int8), t(3))
    i8 = lambda *s: t(s, dtype=torch.int8)   # noqa: E731
    with pytest.raises(TypeError):
        B.bmlp_norm_quantize(t((2, 8)), None, i8(2, 8), t(2), res=t((2, 8), dtype=torch.float16))
    with pytest.raises(ValueError):
        B.bmlp_norm_quantize(t((2, 8)), t(8, dtype=torch.float16), i8(2, 8), t(2))
    with pytest.raises(ValueError):
        B.bmlp_int8_matmul(i8(2, 8), i8(4, 7), t((2, 4)))
    with pytest.raises(ValueError):
        B.bmlp_int8_matmul(i8(2, 8), i8(4, 8), t((2, 5)))
    with pytest.raises(TypeError):
        B.bmlp_int8_matmul(i8(2, 8), i8(4, 8), t((2, 4), dtype=torch.float64))
    with pytest.raises(ValueError):
        B.bmlp_int8_matmul(i8(2, 8), i8(4, 8), t((2, 4)), a_scale=t(3))
    with pytest.raises(ValueError):
        B.bmlp_int8_sign(i8(2, 8), i8(4, 8), t((2, 2), dtype=torch.int64))
    with pytest.raises(B.BmlpError):
        B.bmlp_int8_sign(i8(2, 8), i8(4, 8), t((2, 1), dtype=torch.int64))   # host memory


@gpu
def test_example_runs():
    """The example program: hidden states through the front end into training and prediction."""
    import importlib.util
    import os
    from conftest import ROOT
    spec = importlib.util.spec_from_file_location("hidden_states", os.path.join(ROOT, "examples", "hidden_states.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    got = ex.main(["--n", "3000", "--dim", "512", "--width", "512", "--epochs", "4"])
    # codes of 8 bits are off by at most half a step of 1/127 of a row's largest value, here some
    # 16 times the others' size: errors of that step's uniform distribution, 16 / 127 / sqrt(12) = 0.036
    assert got["error"] < 0.1
    assert got["same"]
    # trained by the oracle on the same words
    pm1 = lambda t: W.unpack(t.cpu().numpy().view(np.uint64), 512)   # noqa: E731
    ref = O.OracleModel([512, 255, 255], 10, seed=5, bs=100)
    x, y = pm1(got["words"]), got["y"].cpu().numpy()
    for _ in range(4):
        errors = ref.train(x, y, epoch_end=True)
    assert errors == got["errors"]
    assert np.array_equal(got["labels"].cpu().numpy(), ref.predict(pm1(got["test"])))
