"""The microscaled 4-bit front end (bmlp_mx4_quantize, bmlp_mx4_norm_quantize,
bmlp_mx4_dequantize, bmlp_mx4_matmul, bmlp_mx4_matmul_grouped) against the formulas in
64 bits, at the sizes, strides, values, scales and groups where it can go wrong, and
its refusals.

Codes and scales are compared for equality: they have one rounding each after the same fp32
operations.  Products are compared for equality where every partial sum is an integer
multiple of one unit below 2^24 of them, which fp32 holds in any order; and else within a
bound on the roundings of a sum in fp32."""
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
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
U8 = torch.uint8


@pytest.fixture(autouse=True)
def _device(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            pytest.skip("needs a GPU")
        torch.cuda.set_device(DEV)


def rows(n, K, dtype, pad=0, off=0, fill=0):
    """An n x K view whose rows are K + pad apart and start off elements into a buffer (pad -1:
    at multiples of 16 elements)."""
    wide = (K + 15) // 16 * 16 if pad < 0 else K + pad
    buf = torch.full((off + n * wide + 8,), fill, dtype=dtype, device=DEV)
    return buf, buf[off:off + n * wide].view(n, wide)[:, :K]


def untouched(buf, n, K, pad, off, fill):
    wide = (K + 15) // 16 * 16 if pad < 0 else K + pad
    ok = (buf[:off] == fill).all() and (buf[off + n * wide:] == fill).all()
    return ok and (buf[off:off + n * wide].view(n, wide)[:, K:] == fill).all()


def hidden(n, K, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, K), generator=g) * torch.exp(torch.randn((n, 1), generator=g))
    x[:, torch.rand((K,), generator=g) < 0.02] *= 16
    return x.to(dtype)


def unpack(q, K):
    """The codes 0..15 of packed rows."""
    return torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :K]


def pack(c):
    c = torch.nn.functional.pad(c, (0, c.shape[-1] % 2)).to(U8)
    return c[..., 0::2] | c[..., 1::2] << 4


def decoded(q, scale, K):
    """Values of codes and scales in 64 bits."""
    v = GRID.to(q.device)[unpack(q, K).long()]
    s = scale.repeat_interleave(32, -1)[..., :K].double()
    return v * torch.where(s == 255, float("nan"), 2.0 ** (s - 127))


# -- quantisation ------------------------------------------------------------------

def plain_codes(u):
    """Codes (0..15) and scales of the rows of u (fp32, on the CPU), by counting: how many of the
    seven borders between sizes lie below, ties to the even code."""
    n, K = u.shape
    b = torch.nn.functional.pad(u.double(), (0, -K % 32)).view(n, -1, 32)
    m = b.abs().amax(2)
    finite = torch.isfinite(b).all(2)
    most = torch.where(finite, m, 1.0)
    p = torch.floor(torch.log2(torch.clamp(most, min=2.0 ** -200)))
    p = torch.where(most >= 2.0 ** (p + 1), p + 1, torch.where(most < 2.0 ** p, p - 1, p))
    s = torch.where(finite, (p - 2 + 127).clamp(min=0), 255.0)
    t = torch.where(finite[:, :, None], b, 0) / 2.0 ** (torch.where(finite, s, 127.0) - 127)[:, :, None]
    grid = GRID[:8]
    edge = (grid[1:] + grid[:-1]) / 2
    odd = torch.arange(7) % 2 == 1
    c = ((t.abs()[..., None] > edge) | ((t.abs()[..., None] == edge) & odd)).sum(-1)
    return (c + 8 * torch.signbit(t)).view(n, -1)[:, :K].to(U8), s.to(U8)


def same_codes(q, want):
    """Equal as values: a zero's sign is no matter."""
    return bool(((q == want) | ((q & 7 == 0) & (want & 7 == 0))).all())


SHAPES = [(1, 1), (1, 2), (3, 7), (2, 31), (5, 32), (4, 33), (9, 64), (3, 100), (1, 255), (2, 256), (17, 257),
          (6, 784), (3, 1000), (3, 1001), (2, 1024), (2, 2047), (300, 129), (1, 4096), (3, 5003), (1, 8192), (2, 8193),
          (2, 16384), (1, 16400), (2, 33000), (1, 70001), (700, 1024)]
PADS = [(0, 0), (-1, 0), (8, 8), (3, 1)]


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", SHAPES)
def test_quantize_and_back(n, K, dtype):
    kb, ks = (K + 1) // 2, (K + 31) // 32
    for pad, off in PADS:
        x = hidden(n, K, n + K, dtype)
        _, xd = rows(n, K, dtype, pad, off)
        qb, qd = rows(n, kb, U8, pad, off, fill=99)
        sb, sd = rows(n, ks, U8, pad, off, fill=98)
        xd.copy_(x)
        B.bmlp_mx4_quantize(xd, qd, sd)
        c, s = plain_codes(x.float())
        q = qd.cpu()
        assert torch.equal(sd.cpu(), s)
        assert same_codes(unpack(q, K), c)
        assert K % 2 == 0 or (q[:, -1] >> 4 == 0).all()
        assert untouched(qb, n, kb, pad, off, 99) and untouched(sb, n, ks, pad, off, 98)
        # and back: exact in fp32; fp16 and bf16 round to nearest, as the cast does
        want = decoded(q, s, K)
        by = torch.rand((n,), generator=torch.Generator().manual_seed(n)) + 0.5
        for out_type in TYPES:
            ob, od = rows(n, K, out_type, pad, off, fill=7)
            B.bmlp_mx4_dequantize(qd, sd, od)
            assert torch.equal(od.cpu(), want.float().to(out_type))
            B.bmlp_mx4_dequantize(qd, sd, od, row_scale=by.to(DEV))
            assert torch.equal(od.cpu(), (want.float() * by[:, None]).to(out_type))
            assert untouched(ob, n, K, pad, off, 7)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", SHAPES)
def test_norm_quantize(n, K, dtype):
    kb, ks = (K + 1) // 2, (K + 31) // 32
    for variant, (pad, off) in enumerate(PADS):
        x, res = hidden(n, K, 3 * n + K, dtype), hidden(n, K, n + 5 * K, dtype)
        gain = (1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to(dtype)
        use_res, use_gain = variant != 2, variant != 3
        _, xd = rows(n, K, dtype, pad, off)
        _, rd = rows(n, K, dtype, max(2 * pad, 0), off)
        ob, od = rows(n, K, dtype, pad, 2 * off, fill=7)
        qb, qd = rows(n, kb, U8, pad, off, fill=99)
        sb, sd = rows(n, ks, U8, pad, off, fill=98)
        xd.copy_(x)
        rd.copy_(res)
        by = torch.full((n,), -1.0, device=DEV)
        B.bmlp_mx4_norm_quantize(xd, gain.to(DEV) if use_gain else None, qd, sd, by, res=rd if use_res else None,
                                 sum_out=od if use_res else None, eps=EPS)
        h = x.float() + res.float() if use_res else x.float()
        c, s = plain_codes(h * gain.float() if use_gain else h)
        assert torch.equal(sd.cpu(), s) and same_codes(unpack(qd.cpu(), K), c)
        assert untouched(qb, n, kb, pad, off, 99) and untouched(sb, n, ks, pad, off, 98)
        if use_res:
            assert torch.equal(od.cpu(), h.to(dtype)) and untouched(ob, n, K, pad, 2 * off, 7)
        # roundings: h (1), h^2 and the sum of them, halved by the root (a thread's at most K / 32 in
        # sequence, then 10 by lanes and warps), mean, + eps, sqrt, 1 / it
        h64 = x.double() + res.double() if use_res else x.double()
        want = 1 / torch.sqrt((h64 * h64).mean(1) + EPS)
        assert ((by.cpu().double() - want).abs() <= (6 + (K / 32 + 12) / 2) * 2.0 ** -24 * want).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("K", [32, 100, 1001])
def test_special_blocks(K, dtype):
    """Zeros, the ties of every pair of neighbouring sizes, saturation, the smallest and largest numbers,
    infinities and NaNs, each in a block of its own."""
    blocks = []
    grid = GRID[:8].tolist()
    blocks.append([0.0] * 32)
    ties = [(a + b) / 2 for a, b in zip(grid[1:], grid[:-1])]
    blocks.append(([4.0] + [v for t in ties for v in (t, -t)] + [5.0, -5.0, 7.0, 7.9, 6.0, 0.25] + [0.0] * 32)[:32])
    blocks.append([7.9, -7.9] + [0.1] * 30)                                     # above 6: becomes 6
    info = torch.finfo(dtype)
    blocks.append([info.max, info.min] + [1.0] * 30)
    blocks.append([info.tiny, -info.tiny] + [info.tiny / 2] * 30)
    blocks.append([float(info.smallest_normal) * 2.0 ** -7] * 32)               # a subnormal number
    blocks.append([1.0] * 31 + [float("inf")])
    blocks.append([1.0, float("nan")] + [2.0] * 30)
    blocks.append([-float("inf"), float("nan")] + [0.0] * 30)
    x = torch.zeros((len(blocks), K), dtype=torch.float64)
    for i, b in enumerate(blocks):
        for first in range(0, K, 64):
            take = min(32, K - first)
            x[i, first:first + take] = torch.tensor(b[:take], dtype=torch.float64)
    x = x.to(dtype)
    n = len(blocks)
    c, s = plain_codes(x.float())
    for pad in (-1, 3):
        _, xd = rows(n, K, dtype, max(pad, 0))
        _, q = rows(n, (K + 1) // 2, U8, pad)
        _, sd = rows(n, (K + 31) // 32, U8, pad)
        xd.copy_(x)
        B.bmlp_mx4_quantize(xd, q, sd)
        assert torch.equal(sd.cpu(), s) and same_codes(unpack(q.cpu(), K), c)
        out = torch.empty((n, K), device=DEV)
        B.bmlp_mx4_dequantize(q, sd, out)
        assert torch.equal(out.cpu().nan_to_num(nan=-77.0), decoded(q.cpu(), s, K).float().nan_to_num(nan=-77.0))
        by = torch.empty((n,), device=DEV)
        q.fill_(0)
        sd.fill_(0)
        B.bmlp_mx4_norm_quantize(xd, None, q, sd, by, eps=EPS)
        assert torch.equal(sd.cpu(), s) and same_codes(unpack(q.cpu(), K), c)
        # a row whose sum of squares is not finite in fp32 (or could be rounded so): NaN
        sq = x.double().square().sum(1)
        assert torch.equal(by.cpu().isnan(), ~(sq < torch.finfo(torch.float32).max))


@gpu
def test_norm_at_eps_zero_and_small():
    x = torch.zeros((4, 64), device=DEV)
    x[1] = 2.0 ** -75       # squares far below fp32's least
    x[2] = 2.0 ** -100
    x[3, 0] = 2.0 ** 60
    q, s = B.bmlp_mx4_empty(4, 64)
    by = torch.empty((4,), device=DEV)
    for eps in (0.0, 1e-30, 2.0 ** -140):
        B.bmlp_mx4_norm_quantize(x, None, q, s, by, eps=eps)
        ms = (x.double() ** 2).mean(1) + float(np.float32(eps))
        want = torch.where(ms > 0, 1 / torch.sqrt(ms), 0.0)
        # roundings: the square, mean, + eps, sqrt, 1 / it, its product with a power of two
        ok = (by.double() - want).abs() <= 8 * 2.0 ** -24 * want
        assert ok.all(), (eps, by, want)


@gpu
@pytest.mark.parametrize("K", [64, 1000, 9000])
def test_norm_in_place(K):
    n = 5
    for dtype in TYPES:
        x, res = hidden(n, K, 1, dtype).to(DEV), hidden(n, K, 2, dtype).to(DEV)
        q, s = B.bmlp_mx4_empty(n, K)
        by = torch.empty((n,), device=DEV)
        want, q0 = x + res, None
        for into in (0, 1, 2):
            xi, ri = x.clone(), res.clone()
            out = (torch.empty_like(x), xi, ri)[into]
            B.bmlp_mx4_norm_quantize(xi, None, q, s, by, res=ri, sum_out=out, eps=EPS)
            assert torch.equal(out, want)
            if q0 is None:
                q0, s0, by0 = q.clone(), s.clone(), by.clone()
            assert torch.equal(q, q0) and torch.equal(s, s0) and torch.equal(by, by0)


# -- products ----------------------------------------------------------------------

def coded(n, K, seed, span=2, pad=-1, off=0, kind="any", base=127):
    """Random codes and scales (bytes base .. base + span) on the device, padding bytes 255."""
    g = torch.Generator().manual_seed(seed)
    lead = (n,) if isinstance(n, int) else tuple(n)
    m = int(np.prod(lead))
    c = torch.randint(0, 16, (m, K), generator=g).to(U8)
    if kind == "most":
        c = torch.full((m, K), 7, dtype=U8)
    s = (base + torch.randint(0, span + 1, (m, (K + 31) // 32), generator=g)).to(U8)
    _, qd = rows(m, (K + 1) // 2, U8, pad, off, fill=255)
    _, sd = rows(m, (K + 31) // 32, U8, pad, off, fill=255)
    qd.copy_(pack(c))
    sd.copy_(s)
    if len(lead) == 2:
        qd, sd = qd.unflatten(0, lead), sd.unflatten(0, lead)
    return qd, sd


def finish(S, row_scale, bias, out_type):
    """The outputs from exact sums: fp32 steps rounded one by one."""
    y = S.float()
    if row_scale is not None:
        y = y * row_scale[:, None]
    if bias is not None:
        y = y + bias
    return y.to(out_type)


def check_exact(n, K, N, pad=-1, off=0, out_type=torch.float32, extra=True, kind="any", expired=False, ldo=0, span=2):
    """Scales within a factor of 2^span: partial sums are multiples of 1/4 of at most
    K 36 4^span, below 2^24 quarters for the sizes here (for random codes they are far from it),
    so that every order gives the same."""
    a, sa = coded(n, K, 7 * n + K, pad=pad, off=off, kind=kind, span=span)
    w, sw = coded(N, K, 3 * N + K + 1, pad=pad, off=off, kind=kind, span=span)
    x, y = decoded(a, sa, K), decoded(w, sw, K)
    S = x @ y.t()
    assert (4 * (x.abs() @ y.abs().t()).max()) < 2 ** 24
    by = torch.rand((n,), generator=torch.Generator().manual_seed(n)).to(DEV) + 0.5 if extra else None
    bias = torch.randn((N,), generator=torch.Generator().manual_seed(N)).to(DEV) if extra else None
    ob, out = rows(n, N, out_type, ldo, 0, fill=-5)
    B.bmlp_mx4_matmul(a, sa, w, sw, out, row_scale=by, bias=bias, expired=expired)
    want = finish(S, by, bias, out_type)
    assert torch.equal(out, want), ((out != want).sum().item(), torch.nonzero(out != want)[:5].tolist())
    assert untouched(ob, n, N, ldo, 0, -5)


@gpu
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256,
                               257, 300, 513])
def test_product_over_rows(n):
    for pad, off in [(-1, 0), (0, 0), (5, 3)]:
        check_exact(n, 512, 130, pad, off)
        check_exact(n, 203, 70, pad, off, out_type=torch.bfloat16, ldo=3)


@gpu
@pytest.mark.parametrize("K", [1, 2, 3, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 192, 193, 255, 256, 257, 500,
                               511, 512, 513, 767, 768, 769, 1000, 1023, 1024, 1025, 1535, 1537, 2047, 2049, 4095, 4097, 5000])
def test_product_over_depth(K):
    for n in (3, 40, 150):
        for pad, off in [(-1, 0), (0, 0), (1, 7)]:
            check_exact(n, K, 140, pad, off, out_type=torch.float16 if n == 40 else torch.float32, span=1)


@gpu
@pytest.mark.parametrize("N", [1, 2, 7, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 384, 500, 525, 1001])
def test_product_over_channels(N):
    for n in (2, 50, 260):
        for pad, off in [(-1, 0), (4, 2)]:
            check_exact(n, 784, N, pad, off, extra=n != 50)


@gpu
@pytest.mark.parametrize("n,K,N", [(1, 16384, 384), (5, 8192, 2048), (100, 4096, 1024), (1000, 1000, 525), (3000, 512, 2000),
                                   (1024, 4096, 1024), (2300, 2048, 1500), (2049, 1030, 4097), (40000, 64, 48), (5000, 96, 33),
                                   (700, 8192, 700), (64, 11000, 260)])
def test_product_of_many_tiles(n, K, N):
    for pad in (-1, 0):
        check_exact(n, K, N, pad, 0, out_type=torch.bfloat16 if n > 2000 else torch.float32, span=0 if K > 4096 else 1)


@gpu
@pytest.mark.parametrize("n", [4, 100, 1000])
def test_product_of_largest_codes(n):
    check_exact(n, 3200, 256, kind="most", span=0)


def bound(x, y, K):
    """How far a sum of products in fp32 may be off: a rounding (a cut at most: 2^-23) of the running
    sum for each addition, of at most K / 32 blocks and 8 parts, none of which is larger than the sum
    of the magnitudes."""
    return (K / 32 + 16) * 2.0 ** -23 * (x.abs() @ y.abs().t())


@gpu
@pytest.mark.parametrize("n,K,N", [(1, 8192, 256), (33, 1001, 200), (130, 4096, 500), (1500, 2048, 1300), (600, 16384, 512)])
@pytest.mark.parametrize("pad", [-1, 1])
def test_product_of_any_scales(n, K, N, pad):
    a, sa = coded(n, K, 1, span=40, base=107, pad=pad)
    w, sw = coded(N, K, 2, span=40, base=87, pad=pad)
    x, y = decoded(a, sa, K), decoded(w, sw, K)
    out = torch.empty((n, N), device=DEV)
    B.bmlp_mx4_matmul(a, sa, w, sw, out)
    S = x @ y.t()
    assert ((out.double() - S).abs() <= bound(x, y, K) + 2.0 ** -24 * S.abs()).all()
    for t in (torch.float16, torch.bfloat16):
        half = torch.empty((n, N), dtype=t, device=DEV)
        B.bmlp_mx4_matmul(a, sa, w, sw, half)
        assert torch.equal(half, out.to(t))


@gpu
@pytest.mark.parametrize("n", [1, 40, 700])
def test_scales_that_are_nan_and_at_the_ends(n):
    K, N = 640, 300
    a, sa = coded(n, K, 5)
    w, sw = coded(N, K, 6)
    sa[n // 2, 3] = 255
    sw[17, 19] = 255
    sw[40] = 0          # 2^-127 with 2^127 and so on
    sa[0, 5:8] = 0
    x, y = decoded(a, sa, K), decoded(w, sw, K)
    out = torch.empty((n, N), device=DEV)
    B.bmlp_mx4_matmul(a, sa, w, sw, out)
    S = x @ y.t()
    assert torch.equal(out.isnan(), S.isnan())
    ok = ~S.isnan()
    x, y = x.nan_to_num(nan=0.0), y.nan_to_num(nan=0.0)
    # (what is below fp32's normal numbers may be lost)
    assert ((out.double() - S).abs() <= bound(x, y, K) + 2.0 ** -24 * S.abs() + K * 2.0 ** -126)[ok].all()


@gpu
def test_odd_depth_ignores_one_side():
    """The unused half of a row's last byte may be anything in one operand."""
    n, K, N = 20, 333, 140
    a, sa = coded(n, K, 1)
    w, sw = coded(N, K, 2)
    out = torch.empty((n, N), device=DEV)
    B.bmlp_mx4_matmul(a, sa, w, sw, out)
    w2 = w.clone()
    w2[:, -1] |= 0x70
    again = torch.empty((n, N), device=DEV)
    B.bmlp_mx4_matmul(a, sa, w2, sw, again)
    assert torch.equal(out, again)


@gpu
@pytest.mark.parametrize("n,K,N", [(3, 512, 200), (1, 8192, 256), (200, 1024, 520), (2100, 1024, 1100), (600, 4000, 300)])
def test_expired_waits_cost_time_only(n, K, N):
    for pad in (-1, 3):
        check_exact(n, K, N, pad, 0, expired=True, span=1)
        check_exact(n, K, N, pad, 0, span=1)


@gpu
def test_operands_of_different_alignment():
    n, K, N = 70, 1024, 150
    for pa, oa, pw, ow, ps in [(-1, 0, 3, 1, -1), (3, 1, -1, 0, 2), (16, 16, 16, 0, 1), (8, 8, 4, 4, 16)]:
        a, _ = coded(n, K, 1, pad=pa, off=oa)
        w, _ = coded(N, K, 2, pad=pw, off=ow)
        _, sa = coded(n, K, 3, pad=ps, off=oa)
        _, sw = coded(N, K, 4, pad=ps, off=ow)
        out = torch.empty((n, N), device=DEV)
        B.bmlp_mx4_matmul(a, sa, w, sw, out)
        assert torch.equal(out.double(), decoded(a, sa, K) @ decoded(w, sw, K).t())


# -- products by group ---------------------------------------------------------------

def check_groups(sizes, K, N, pad=-1, out_type=torch.float32, extra=True, before=0, after=0, expired=False, seed=0, span=1):
    E = len(sizes)
    at = torch.tensor([before] + [0] * E, dtype=torch.int64)
    at[1:] = before + torch.tensor(sizes).cumsum(0)
    n = int(at[-1]) + after
    a, sa = coded(n, K, seed + 1, pad=pad, span=span)
    w, sw = coded((E, N), K, seed + 2, pad=pad, span=span)
    if after:
        sa[n - after:] = 255     # of rows in no group nothing matters
    x, y = decoded(a, sa, K), decoded(w, sw, K)
    by = torch.rand((n,), generator=torch.Generator().manual_seed(n)).to(DEV) + 0.5 if extra else None
    bias = torch.randn((E, N), generator=torch.Generator().manual_seed(N)).to(DEV) if extra else None
    out = torch.full((n, N), -5.0, dtype=out_type, device=DEV)
    want = out.clone()
    for e in range(E):
        if sizes[e]:
            r = slice(int(at[e]), int(at[e + 1]))
            assert 4 * (x[r].abs() @ y[e].abs().t()).max() < 2 ** 24
            want[r] = finish(x[r] @ y[e].t(), by[r] if extra else None, bias[e] if extra else None, out_type)
    B.bmlp_mx4_matmul_grouped(a, sa, w, sw, at.to(torch.int32).to(DEV), out, row_scale=by, bias=bias, expired=expired)
    assert torch.equal(out, want), torch.nonzero(out != want)[:5].tolist()


GROUPS = [[1], [5], [0], [0, 0, 0], [0, 3, 0], [1, 1, 1, 1], [16, 16, 16], [17, 0, 15, 33], [0, 128, 1, 129, 0, 0, 300],
          [3] * 32, [0] * 70 + [9] + [0] * 60, list(range(40)), [257, 1, 0, 700], [1000, 0, 2], [256, 256], [200, 2, 200, 90, 411]]


@gpu
@pytest.mark.parametrize("sizes", GROUPS, ids=lambda s: "%dx%d" % (len(s), sum(s)))
def test_groups(sizes):
    check_groups(sizes, 512, 130)
    check_groups(sizes, 203, 70, pad=3, out_type=torch.bfloat16, before=3, after=40)
    check_groups(sizes, 1100, 260, out_type=torch.float16, extra=False, after=1)


@gpu
@pytest.mark.parametrize("sizes,K,N", [([500, 0, 700, 1300, 1], 1024, 1030), ([3] * 32, 4096, 512), ([90, 2000, 10], 784, 2048),
                                       ([7, 1, 3], 8192, 256), ([1, 0], 16384, 128)])
def test_groups_of_real_sizes(sizes, K, N):
    for pad in (-1, 5):
        check_groups(sizes, K, N, pad, out_type=torch.bfloat16, after=100, span=0)


@gpu
@pytest.mark.parametrize("sizes", [[40, 0, 3], [300, 500, 2], [1000, 1300]], ids=str)
def test_groups_expired(sizes):
    for pad in (-1, 3):
        check_groups(sizes, 1024, 150, pad, expired=True, after=5)


@gpu
def test_many_groups():
    E = B.BMLP_MX4_MAX_GROUPS
    g = torch.Generator().manual_seed(1)
    check_groups(torch.randint(0, 3, (E,), generator=g).tolist(), 64, 5)
    check_groups([2000] + [0] * (E - 2) + [3000], 64, 40)


@gpu
def test_offsets_out_of_order():
    """Offsets that decrease or leave 0..n are taken as the nearest that do not."""
    n, K, N, E = 50, 128, 40, 5
    a, sa = coded(n, K, 1)
    w, sw = coded((E, N), K, 2)
    x, y = decoded(a, sa, K), decoded(w, sw, K)
    for given, taken in [([-7, 10, 5, 30, 99, 20], [0, 10, 10, 30, 50, 50]),
                         ([2 ** 31 - 1] * 6, [50] * 6), ([-2 ** 31] * 6, [0] * 6),
                         ([60, 0, 10, 20, 30, 50], [50] * 6)]:
        out = torch.full((n, N), -5.0, device=DEV)
        B.bmlp_mx4_matmul_grouped(a, sa, w, sw, torch.tensor(given, dtype=torch.int32, device=DEV), out)
        want = torch.full((n, N), -5.0, device=DEV)
        for e in range(E):
            r = slice(taken[e], taken[e + 1])
            want[r] = (x[r] @ y[e].t()).float()
        assert torch.equal(out, want), given


@gpu
def test_groups_that_share_weights():
    """A group stride of zero: every group by the same matrix; and groups in steps."""
    E, K, N, n = 3, 256, 70, 90
    w, sw = coded(N, K, 2)
    a, sa = coded(n, K, 1)
    at = torch.tensor([0, 20, 50, 90], dtype=torch.int32, device=DEV)
    out = torch.empty((n, N), device=DEV)
    B.bmlp_mx4_matmul_grouped(a, sa, w.expand(E, *w.shape), sw.expand(E, *sw.shape), at, out)
    assert torch.equal(out.double(), decoded(a, sa, K) @ decoded(w, sw, K).t())
    w, sw = coded((2 * E, N), K, 3)
    B.bmlp_mx4_matmul_grouped(a, sa, w[::2], sw[::2], at, out)
    for e, (i, j) in enumerate([(0, 20), (20, 50), (50, 90)]):
        assert torch.equal(out[i:j].double(), decoded(a[i:j], sa[i:j], K) @ decoded(w[2 * e], sw[2 * e], K).t())


@gpu
@pytest.mark.parametrize("n,K,N,E", [(16, 4096, 60000, 1), (32, 2048, 60000, 1), (5000, 2048, 300, 1), (1000, 4096, 4096, 1),
                                     (3000, 2304, 3000, 1), (96, 4096, 2048, 32), (200, 1280, 4096, 30), (4000, 1536, 2048, 5)])
@pytest.mark.parametrize("pad", [-1, 0, 1])
def test_no_wait_expires(n, K, N, E, pad):
    """Several tiles, rings and units a CTA: the calls end long before a bounded wait (2 s) would, so none was
    taken as expired (an expired one costs time only)."""
    a, sa = coded(n, K, 1, pad=pad)
    w, sw = coded((E, N), K, 2, pad=pad)
    at = torch.linspace(0, n, E + 1).to(torch.int32).to(DEV)
    out = torch.empty((n, N), dtype=torch.bfloat16, device=DEV)

    def call():
        if E == 1:
            B.bmlp_mx4_matmul(a, sa, w[0], sw[0], out)
        else:
            B.bmlp_mx4_matmul_grouped(a, sa, w, sw, at, out)

    call()
    torch.cuda.synchronize()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(3):
        call()
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 1000


# -- as they are used ------------------------------------------------------------------

@gpu
def test_offsets_past_32_bits():
    """Rows of codes, of outputs, and groups whose bytes lie past 2^32."""
    n, K, N = 300, 256, 64
    far = (1 << 32) // (n - 1) + 4096 // 16 * 16
    far = far // 16 * 16
    buf = torch.zeros((n - 1) * far + K // 2, dtype=U8, device=DEV)
    a, sa = coded(n, K, 1)
    w, sw = coded(N, K, 2)
    big = buf.as_strided((n, K // 2), (far, 1))
    big.copy_(a)
    out = torch.empty((n, N), device=DEV)
    want = decoded(a, sa, K) @ decoded(w, sw, K).t()
    B.bmlp_mx4_matmul(big, sa, w, sw, out)
    assert torch.equal(out.double(), want)
    B.bmlp_mx4_matmul(w, sw, big, sa, out.view(N, n))
    assert torch.equal(out.view(N, n).double(), want.t())
    one, ones = coded((2, N), K, 4)
    group = buf[:2 * (1 << 31)].as_strided((2, N, K // 2), (1 << 31, K // 2, 1))
    group.copy_(one)
    at = torch.tensor([0, 100, 300], dtype=torch.int32, device=DEV)
    B.bmlp_mx4_matmul_grouped(a, sa, group, ones, at, out)
    for e, r in enumerate([slice(0, 100), slice(100, 300)]):
        assert torch.equal(out[r].double(), decoded(a[r], sa[r], K) @ decoded(one[e], ones[e], K).t())
    wide = torch.empty((1 << 32) // 4 + 4096, device=DEV)
    y = wide.as_strided((n, N), ((1 << 30) // (n - 1), 1))
    B.bmlp_mx4_matmul(a, sa, w, sw, y)
    assert torch.equal(y.double(), want)


@gpu
def test_streams_and_capture():
    """On another stream, captured with its offsets computed on the device, and replayed on new inputs."""
    n, K, N, E = 60, 512, 140, 4
    x = hidden(n, K, 1, torch.bfloat16).to(DEV)
    wf = 0.02 * torch.randn((E * N, K), generator=torch.Generator().manual_seed(3)).to(DEV)
    w, sw = B.bmlp_mx4_empty((E, N), K)
    q, s = B.bmlp_mx4_empty(n, K)
    by = torch.empty((n,), device=DEV)
    at = torch.tensor([0, 10, 10, 40, 55], dtype=torch.int32, device=DEV)
    outs = [torch.full((n, N), -5.0, device=DEV) for _ in range(2)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    B.bmlp_mx4_quantize(wf, w.flatten(0, 1), sw.flatten(0, 1), stream=st)

    def step():
        B.bmlp_mx4_norm_quantize(x, None, q, s, by, eps=EPS, stream=st)
        B.bmlp_mx4_matmul_grouped(q, s, w, sw, at, outs[0], row_scale=by, stream=st)
        B.bmlp_mx4_matmul(q, s, w[1], sw[1], outs[1], row_scale=by, stream=st)

    def check():
        st.synchronize()
        c, sc = plain_codes(x.cpu().float())
        want = decoded(pack(c), sc, K)
        y = decoded(w.cpu(), sw.cpu(), K)
        grouped = torch.full((n, N), -5.0, dtype=torch.float64)
        a = at.tolist()
        for e in range(E):
            r = slice(a[e], a[e + 1])
            grouped[r] = want[r] @ y[e].t() * by.cpu().double()[r, None]
        plain = want @ y[1].t() * by.cpu().double()[:, None]
        for got, ref, of in ((outs[0], grouped, None), (outs[1], plain, None)):
            lim = (K / 32 + 18) * 2.0 ** -23 * (want.abs() @ y.abs().amax(0).t() * by.cpu().double()[:, None])
            assert ((got.cpu().double() - ref).abs() <= lim).all()

    step()
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step()
    x.copy_(hidden(n, K, 9, torch.bfloat16))
    at.copy_(torch.tensor([2, 2, 30, 31, 60], dtype=torch.int32))
    outs[0].fill_(-5.0)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    check()


@gpu
def test_two_streams_at_once():
    n, K, N = 200, 4096, 1024
    a, sa = coded(n, K, 1, span=1)
    w, sw = coded(N, K, 2, span=1)
    want = (decoded(a, sa, K) @ decoded(w, sw, K).t()).float()
    sts = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty((n, N), device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, out in zip(sts, outs):
            B.bmlp_mx4_matmul(a, sa, w, sw, out, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@gpu
def test_beside_other_kernels():
    """Every plan of the products on three streams, mixed with the 8-bit product: CTAs of several of them share
    the SMs and their tensor memory."""
    jobs = []
    for n, K, N, pad in [(1, 4096, 4096, -1), (20, 2048, 3000, -1), (100, 4096, 2048, -1), (1500, 1024, 2048, -1),
                         (3000, 2048, 1024, -1), (70, 1000, 500, 1), (400, 700, 300, 0), (9, 8192, 256, -1)]:
        (a, sa), (w, sw) = coded(n, K, 1, span=0, pad=pad), coded(N, K, 2, span=0, pad=pad)
        want = (decoded(a, sa, K) @ decoded(w, sw, K).t()).float()
        jobs.append((want, [torch.empty((n, N), device=DEV) for _ in range(3)],
                     lambda st, out, a=a, sa=sa, w=w, sw=sw: B.bmlp_mx4_matmul(a, sa, w, sw, out, stream=st)))
    for n, K, N in [(40, 1024, 2048), (2000, 1024, 1024)]:
        a, w = (torch.randint(-128, 128, (m, K), dtype=torch.int8).to(DEV) for m in (n, N))
        jobs.append(((a.double() @ w.double().t()).int(), [torch.empty((n, N), dtype=torch.int32, device=DEV) for _ in range(3)],
                     lambda st, out, a=a, w=w: B.bmlp_int8_matmul(a, w, out, stream=st)))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for rep in range(6):
        for k in range(3 * len(jobs)):
            want, outs, call = jobs[(7 * k + rep) % len(jobs)]
            i = k % 3
            call(streams[i], outs[i])
        torch.cuda.synchronize()
        for want, outs, _ in jobs:
            for out in outs:
                assert torch.equal(out, want)
                out.fill_(-1)
        torch.cuda.synchronize()


@gpu
def test_back_to_back_calls_do_not_mix():
    """Calls that depend on one another, with nothing between them: each kernel may start while
    the one before it ends."""
    n, K = 2100, 512
    w1, s1 = coded(K, K, 2, span=0)
    q, s = B.bmlp_mx4_empty(n, K)
    x0 = hidden(n, K, 1, torch.bfloat16).to(DEV)
    y = torch.empty((n, K), dtype=torch.bfloat16, device=DEV)
    by = torch.empty((n,), device=DEV)
    for m in (3, 70, 2100):
        want = None
        for rep in range(12):
            B.bmlp_mx4_norm_quantize(x0[:m], None, q[:m], s[:m], by[:m], eps=EPS)
            B.bmlp_mx4_matmul(q[:m], s[:m], w1, s1, y[:m], row_scale=by[:m])
            B.bmlp_mx4_quantize(y[:m], q[:m], s[:m])
            B.bmlp_mx4_matmul(q[:m], s[:m], w1, s1, y[:m])
            got = y[:m].clone()
            if want is None:
                torch.cuda.synchronize()
                B.bmlp_mx4_norm_quantize(x0[:m], None, q[:m], s[:m], by[:m], eps=EPS)
                torch.cuda.synchronize()
                B.bmlp_mx4_matmul(q[:m], s[:m], w1, s1, y[:m], row_scale=by[:m])
                torch.cuda.synchronize()
                B.bmlp_mx4_quantize(y[:m], q[:m], s[:m])
                torch.cuda.synchronize()
                B.bmlp_mx4_matmul(q[:m], s[:m], w1, s1, y[:m])
                want = y[:m].clone()
            assert torch.equal(got, want), (m, rep)


@gpu
def test_front_end_feeds_training():
    """Hidden states -> norm -> 4-bit product -> median binarisation -> training and prediction, equal
    to the oracle trained on the words; the whole chain on one stream."""
    n, D, K = 300, 96, 130
    x, res = hidden(n, D, 1, torch.bfloat16), hidden(n, D, 2, torch.bfloat16)
    wf = 0.02 * torch.randn((K, D), generator=torch.Generator().manual_seed(3))
    q, s = B.bmlp_mx4_empty(n, D)
    w, sw = B.bmlp_mx4_empty(K, D)
    by = torch.empty((n,), device=DEV)
    z = torch.empty((n, K), device=DEV)
    words = torch.empty((n, W.words(K)), dtype=torch.int64, device=DEV)
    y = torch.from_numpy(np.arange(n, dtype=np.int32) % 4).to(DEV)
    B.bmlp_mx4_quantize(wf.to(DEV), w, sw)
    B.bmlp_mx4_norm_quantize(x.to(DEV), None, q, s, by, res=res.to(DEV), eps=EPS)
    B.bmlp_mx4_matmul(q, s, w, sw, z, row_scale=by)
    B.bmlp_binarize_median(z, words)
    m = B.BMLP([K, 64], 4, seed=5, bs=50)
    errs = m.train(words, y, epoch_end=True, count_errors=True)
    out = torch.empty((n,), dtype=torch.int32, device=DEV)
    m.predict(words, out)
    # the product is the definition's within its roundings
    cx, sx = plain_codes(x.float() + res.float())
    cw, scw = plain_codes(wf)
    X, Y = decoded(pack(cx), sx, D), decoded(pack(cw), scw, D)
    lim = (D / 32 + 18) * 2.0 ** -23 * (X.abs() @ Y.abs().t()) * by.cpu().double()[:, None]
    assert ((z.cpu().double() - X @ Y.t() * by.cpu().double()[:, None]).abs() <= lim).all()
    pm1 = W.unpack(words.cpu().numpy().view(np.uint64), K)
    ref = O.OracleModel([K, 64], 4, seed=5, bs=50)
    assert errs == ref.train(pm1, y.cpu().numpy(), epoch_end=True)
    assert np.array_equal(out.cpu().numpy(), ref.predict(pm1))
    m.close()


# -- refusals ------------------------------------------------------------------------

def test_quantize_refusals():
    lib = B.lib()
    x = np.zeros((4, 8), np.float32)
    q = np.zeros((4, 8), np.uint8)
    f = np.zeros(4, np.float32)
    px, pq, pf = x.ctypes.data, q.ctypes.data, f.ctypes.data

    def rows_call(ptr=px, typ=B.BMLP_F32, ldx=8, n=4, K=8, qp=pq, ldq=4, sp=pq, lds=1):
        return lib.bmlp_mx4_quantize(ptr, typ, ldx, n, K, qp, ldq, sp, lds, None)

    def norm_call(ptr=px, ldx=8, res=None, ldr=0, gain=None, typ=B.BMLP_F32, n=4, K=8, eps=1e-6, sm=None, lds=0, rs=pf):
        return lib.bmlp_mx4_norm_quantize(ptr, ldx, res, ldr, gain, typ, n, K, eps, sm, lds, pq, 4, pq, 1, rs, None)

    def back_call(qp=pq, ldq=4, sp=pq, lds=1, n=4, K=8, o=px, typ=B.BMLP_F32, ldo=8):
        return lib.bmlp_mx4_dequantize(qp, ldq, sp, lds, None, n, K, o, typ, ldo, None)

    def refused(rc, text):
        assert rc == B.BMLP_EINVAL and text in B.bmlp_last_error(), B.bmlp_last_error()

    for call in (rows_call, norm_call, back_call):
        refused(call(n=-1), "n outside")
        refused(call(n=B.BMLP_MX4_MAX_ROWS + 1), "n outside")
        refused(call(K=0), "K < 1")
        refused(call(typ=B.BMLP_I32), "_type")
        refused(call(typ=9), "_type")
        refused(call(), "device pointers")        # host memory
        assert call(n=0) == B.BMLP_OK
    for call in (rows_call, back_call):
        refused(call(ldq=3), "row stride")
        refused(call(lds=0), "row stride")
    refused(rows_call(ldx=7), "row stride")
    refused(back_call(ldo=7), "row stride")
    refused(rows_call(ptr=None), "device pointers")
    refused(norm_call(eps=-1.0), "eps")
    refused(norm_call(eps=float("nan")), "eps")
    refused(norm_call(eps=float("inf")), "eps")
    refused(norm_call(res=px, ldr=4), "row stride")
    refused(norm_call(sm=px, lds=4), "row stride")
    refused(norm_call(sm=px, lds=9), "in place")


def test_product_refusals():
    lib = B.lib()
    a = np.zeros((4, 8), np.uint8)
    out = np.zeros((4, 4), np.float32)
    pa, po = a.ctypes.data, out.ctypes.data

    def mm(lda=4, ldas=1, ldw=4, ldws=1, n=4, K=8, N=4, typ=B.BMLP_F32, ldo=4, o=po):
        return lib.bmlp_mx4_matmul(pa, lda, pa, ldas, None, pa, ldw, pa, ldws, None, n, K, N, o, typ, ldo, None)

    def grouped(lda=4, ldas=1, ldw=4, ldws=1, n=4, K=8, N=4, typ=B.BMLP_F32, ldo=4, o=po, E=2, gw=16, gws=4, gb=4, at=pa):
        return lib.bmlp_mx4_matmul_grouped(pa, lda, pa, ldas, None, pa, ldw, gw, pa, ldws, gws, None, gb, at, E, n, K, N, o,
                                           typ, ldo, None)

    def refused(rc, text):
        assert rc == B.BMLP_EINVAL and text in B.bmlp_last_error(), B.bmlp_last_error()

    for call in (mm, grouped):
        refused(call(n=-1), "n outside")
        refused(call(n=B.BMLP_MX4_MAX_ROWS + 1), "n outside")
        refused(call(K=0), "K < 1")
        refused(call(N=0), "N outside")
        refused(call(N=(1 << 30) + 1), "N outside")
        refused(call(typ=B.BMLP_I32), "out_type")
        refused(call(typ=-1), "out_type")
        for kw in (dict(lda=3), dict(ldas=0), dict(ldw=3), dict(ldws=0), dict(ldo=3)):
            refused(call(**kw), "row stride")
        refused(call(), "device pointers")
        refused(call(o=None), "device pointers")
        assert call(n=0) == B.BMLP_OK
    refused(grouped(E=0), "E outside")
    refused(grouped(E=B.BMLP_MX4_MAX_GROUPS + 1), "E outside")
    refused(grouped(gw=-16), "group stride")
    refused(grouped(gws=-1), "group stride")
    refused(grouped(at=None), "device pointers")


def test_binding_refusals():
    """Shapes, types and strides that the binding turns away before the library is called."""
    t = torch.zeros
    u8 = lambda *s: t(s, dtype=U8)   # noqa: E731
    i32 = lambda *s: t(s, dtype=torch.int32)   # noqa: E731
    with pytest.raises(TypeError):
        B.bmlp_mx4_quantize(t((2, 64), dtype=torch.float64), u8(2, 32), u8(2, 2))
    with pytest.raises(TypeError):
        B.bmlp_mx4_quantize(t((2, 64)), t((2, 32), dtype=torch.int8), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_quantize(t((2, 64)), u8(2, 31), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_quantize(t((2, 65)), u8(2, 33), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_quantize(t((64, 2)).t(), u8(2, 32), u8(2, 2))
    with pytest.raises(TypeError):
        B.bmlp_mx4_norm_quantize(t((2, 64)), None, u8(2, 32), u8(2, 2), t(2), res=t((2, 64), dtype=torch.float16))
    with pytest.raises(ValueError):
        B.bmlp_mx4_norm_quantize(t((2, 64)), t(64, dtype=torch.float16), u8(2, 32), u8(2, 2), t(2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_norm_quantize(t((2, 64)), None, u8(2, 32), u8(2, 2), t(3))
    with pytest.raises(ValueError):
        B.bmlp_mx4_dequantize(u8(2, 32), u8(2, 2), t((2, 63, 1)).squeeze(-1)[:, :62])
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 31), u8(4, 2), t((2, 4)))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 1), t((2, 4)))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 2), t((2, 5)))
    with pytest.raises(TypeError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 2), t((2, 4), dtype=torch.float64))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 2), t((2, 4)), row_scale=t(3))
    grouped = B.bmlp_mx4_matmul_grouped
    with pytest.raises(ValueError):
        grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(3, 4, 2), i32(3), t((2, 4)))
    with pytest.raises(ValueError):
        grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(3, 4, 2), t(4, dtype=torch.int64), t((2, 4)))
    with pytest.raises(ValueError):
        grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(2, 4, 2), i32(4), t((2, 4)))
    with pytest.raises(ValueError):
        grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(3, 4, 2), i32(4), t((2, 4)), bias=t((3, 5)))
    with pytest.raises(B.BmlpError):
        grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(3, 4, 2), i32(4), t((2, 4)))   # host memory


@gpu
def test_refusals_of_device_tensors():
    """What the native marshalling does not take comes to the same checks and errors, and the library's own
    refusals come through it."""
    t = lambda *s, d=torch.float32: torch.zeros(s, dtype=d, device=DEV)   # noqa: E731
    u8 = lambda *s: t(*s, d=U8)   # noqa: E731
    with pytest.raises(TypeError):
        B.bmlp_mx4_quantize(t(2, 64, d=torch.float64), u8(2, 32), u8(2, 2))
    with pytest.raises(TypeError):
        B.bmlp_mx4_quantize(t(2, 64), t(2, 32, d=torch.int8), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_quantize(t(2, 64), u8(2, 31), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_quantize(t(64, 2).t(), u8(2, 32), u8(2, 2))
    with pytest.raises(ValueError):
        B.bmlp_mx4_norm_quantize(t(2, 64), t(63), u8(2, 32), u8(2, 2), t(2))
    with pytest.raises(B.BmlpError):
        B.bmlp_mx4_norm_quantize(t(2, 64), None, u8(2, 32), u8(2, 2), None)
    with pytest.raises(B.BmlpError, match="eps"):
        B.bmlp_mx4_norm_quantize(t(2, 64), None, u8(2, 32), u8(2, 2), t(2), eps=-1.0)
    with pytest.raises(ValueError):
        B.bmlp_mx4_dequantize(u8(2, 32), u8(2, 2), t(2, 62))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 2), t(2, 5))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32), u8(4, 2), t(2, 4), row_scale=t(3))
    with pytest.raises(B.BmlpError, match="device pointers"):
        B.bmlp_mx4_matmul(u8(2, 32), u8(2, 2), u8(4, 32).cpu(), u8(4, 2), t(2, 4))
    with pytest.raises(ValueError):
        B.bmlp_mx4_matmul_grouped(u8(2, 32), u8(2, 2), u8(3, 4, 32), u8(3, 4, 2), t(3, d=torch.int32), t(2, 4))
    E = B.BMLP_MX4_MAX_GROUPS + 1
    with pytest.raises(B.BmlpError, match="E outside"):
        B.bmlp_mx4_matmul_grouped(u8(2, 32), u8(2, 2), u8(E, 1, 32), u8(E, 1, 2), t(E + 1, d=torch.int32), t(2, 1))
    with pytest.raises(B.BmlpError, match="row stride"):
        B.bmlp_mx4_quantize(t(1, 64).expand(2, 64), u8(2, 32), u8(2, 2))


@gpu
def test_both_ways_of_marshalling_agree():
    """On the current stream (native) and on one given by hand (the interpreter's way)."""
    n, K, N, E = 70, 1001, 130, 3
    x, res = hidden(n, K, 1, torch.bfloat16).to(DEV), hidden(n, K, 2, torch.bfloat16).to(DEV)
    w, sw = coded((E, N), 2 * ((K + 1) // 2), 3, pad=3)
    w = w.clone()
    at = torch.tensor([0, 20, 20, 60], dtype=torch.int32, device=DEV)
    bias = torch.randn((E, N), generator=torch.Generator().manual_seed(1)).to(DEV)
    st = torch.cuda.current_stream()
    got = []
    for stream in (None, st):
        q, s = B.bmlp_mx4_empty(n, K)
        q2, s2 = B.bmlp_mx4_empty(n, K)
        by, total, back = torch.empty(n, device=DEV), torch.empty_like(x), torch.empty((n, K), device=DEV)
        out, grouped = torch.zeros((n, N), device=DEV), torch.zeros((n, N), dtype=torch.float16, device=DEV)
        B.bmlp_mx4_quantize(x, q2, s2, stream=stream)
        B.bmlp_mx4_norm_quantize(x, None, q, s, by, res=res, sum_out=total, eps=EPS, stream=stream)
        B.bmlp_mx4_dequantize(q, s, back, row_scale=by, stream=stream)
        B.bmlp_mx4_matmul(q, s, w[0], sw[0], out, row_scale=by, bias=bias[0], stream=stream)
        B.bmlp_mx4_matmul_grouped(q, s, w, sw, at, grouped, row_scale=by, bias=bias, stream=stream)
        got.append([v.clone() for v in (q2, s2, q, s, by, total, back, out, grouped)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_sizes_past_31_bits_are_refused():
    x = torch.empty((1,), dtype=U8).expand(1 << 31).unsqueeze(0)
    with pytest.raises((B.BmlpError, ValueError)):
        B.bmlp_mx4_quantize(torch.empty((1,)).expand(1, 1 << 31), x, x)
    with pytest.raises(B.BmlpError, match="31 bits"):
        B.bmlp_mx4_matmul(x, x, x, x, torch.empty((1, 1)))


def test_empty_buffers_are_aligned():
    for n, K in [(3, 1), (5, 1001), ((2, 7), 64)]:
        q, s = B.bmlp_mx4_empty(n, K, device="cpu")
        lead = (n,) if isinstance(n, int) else n
        assert q.shape == (*lead, (K + 1) // 2) and s.shape == (*lead, (K + 31) // 32)
        assert all(v % 16 == 0 for t in (q, s) for v in t.stride()[:-1])
