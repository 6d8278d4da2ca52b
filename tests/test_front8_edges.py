"""The 8-bit front end past the sizes of its other tests: rows and channels that leave 31
bits or a slab, second turns of persistent kernels, rows whose squares leave fp32, and
tensors that do not belong to the call."""
import threading

import pytest
import torch

import workloads as W
from paper_2412_00119_gb300 import bmlp as B
from test_front8 import TYPES, check_codes, codes, hidden, plain_codes, rows

DEV = "cuda:0"
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            pytest.skip("needs a GPU")
        torch.cuda.set_device(DEV)


# -- refusals ------------------------------------------------------------------------

def test_sizes_past_31_bits_are_refused():
    """Sizes that the C types cannot hold: not the call of the size that is left of them."""
    def t(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="meta")   # (shapes and strides without memory)
    i8, f32 = torch.int8, torch.float32
    for big in (2 ** 31, 2 ** 32 + 8, 2 ** 33 + 1):
        calls = [lambda: B.bmlp_quantize_rows(t((1, big), f32), t((1, big), i8), t((1,), f32)),
                 lambda: B.bmlp_norm_quantize(t((1, big), f32), None, t((1, big), i8), t((1,), f32)),
                 lambda: B.bmlp_int8_matmul(t((1, big), i8), t((4, big), i8), t((1, 4), f32)),
                 lambda: B.bmlp_int8_matmul(t((1, 8), i8), t((big, 8), i8), t((1, big), f32)),
                 lambda: B.bmlp_int8_sign(t((1, big), i8), t((4, big), i8), t((1, 1), torch.int64)),
                 lambda: B.bmlp_int8_sign(t((1, 8), i8), t((big, 8), i8), t((1, (big + 63) // 64), torch.int64))]
        for call in calls:
            with pytest.raises(B.BmlpError, match="31 bits") as e:
                call()
            assert e.value.code == B.BMLP_EINVAL
        assert B.bmlp_int8_workspace(300, big, 4000) == 0
        assert B.bmlp_int8_workspace(300, 2304, big) == 0
    assert B.bmlp_int8_workspace(300, 2 - 2 ** 32, 4000) == 0


# -- many rows -------------------------------------------------------------------------

def few_workspaces(n, K, N):
    """A workspace as the size wants it, and one that is too small for any."""
    size = B.bmlp_int8_workspace(n, K, N)
    assert size > 16
    return torch.empty((size,), dtype=torch.uint8, device=DEV), torch.empty((16,), dtype=torch.uint8, device=DEV)


# (n, K, N): the pairs of both operands' blocks, whose rows come in slabs of 65,536: two and
# three slabs, the last of one row and of some; one chunk of K and two
SLABS = [(65537, 64, 700), (65536 + 300, 1100, 515), (131100, 200, 515), (131073, 64, 1024), (196608, 40, 300)]


@gpu
@pytest.mark.parametrize("n,K,N", SLABS)
def test_rows_past_a_slab(n, K, N):
    """Every output type and the signs, in rows at even and odd places, with the workspace of the
    pairs and with none, which leaves the tiles' slabs."""
    a, w = codes(n, K, n, "ends").to(DEV), codes(N, K, K).to(DEV)
    whole, small = few_workspaces(n, K, N)
    assert whole.numel() == 128 * ((K + 63) // 64) * ((N + 255) // 256 * 256 + 65536)   # (the pairs')
    S = a.double() @ w.double().t()
    g = torch.Generator(device=DEV).manual_seed(5)
    # scales of two rows a slab apart differ, as do biases and thresholds of channels
    sa = torch.exp(torch.randn((n,), generator=g, device=DEV)) / 100
    sw = torch.exp(torch.randn((N,), generator=g, device=DEV)) / 100
    bias = torch.randn((N,), generator=g, device=DEV) * 10
    thr = torch.randint(-3000, 3000, (N,), generator=g, device=DEV, dtype=torch.int32)
    y = S.float() * sa[:, None] * sw + bias
    bits = torch.zeros((n, 64 * W.words(N)), dtype=torch.bool, device=DEV)
    bits[:, :N] = S >= thr.double()
    words = (bits.view(n, -1, 64).long() << torch.arange(64, device=DEV)).sum(2)
    for pad in (0, 3):
        _, ad = rows(n, K, torch.int8, pad, pad, fill=-77)
        ad.copy_(a)
        for ws in (whole, small):
            whole.fill_(0x7F)
            for dtype in [torch.int32] + TYPES:
                buf, out = rows(n, N, dtype, pad, pad, fill=-5)
                if dtype == torch.int32:
                    B.bmlp_int8_matmul(ad, w, out, workspace=ws)
                    assert torch.equal(out.double(), S), (pad, ws.numel())
                else:
                    B.bmlp_int8_matmul(ad, w, out, sa, sw, bias, workspace=ws)
                    assert torch.equal(out, y.to(dtype)), (pad, ws.numel(), dtype)
                assert (buf[:pad] == -5).all() and (buf[pad + n * (N + pad):] == -5).all()
                if pad:
                    assert (buf[pad:pad + n * (N + pad)].view(n, -1)[:, N:] == -5).all()
            got = torch.full((n, W.words(N)), -1, dtype=torch.int64, device=DEV)
            B.bmlp_int8_sign(ad, w, got, thr, workspace=ws)
            assert torch.equal(got, words), (pad, ws.numel())


@gpu
@pytest.mark.parametrize("n,K,N", [(12, 200, 300), (20, 2048, 300), (33, 1000, 100), (50, 4096, 4000), (100, 2048, 4096),
                                   (300, 3000, 2000), (1500, 1024, 8130), (1500, 1030, 4001), (4000, 1500, 50), (4000, 3000, 120),
                                   (1000, 64, 20)])
def test_signs_after_expired_waits(n, K, N):
    """With every CTA's wait taken as expired the words are whole, their pad bits zero; with a
    workspace and without one that suffices."""
    a, w = codes(n, K, n, "ends").to(DEV), codes(N, K, K).to(DEV)
    S = a.double() @ w.double().t()
    for thr in (None, S[0].to(torch.int32)):
        bits = torch.zeros((n, 64 * W.words(N)), dtype=torch.bool, device=DEV)
        bits[:, :N] = S >= (0 if thr is None else thr.double())
        want = (bits.view(n, -1, 64).long() << torch.arange(64, device=DEV)).sum(2)
        for ws in (None, torch.empty(16, dtype=torch.uint8, device=DEV)):
            for expired in (True, False):      # (and the device is as it was)
                out = torch.full((n, W.words(N)), -1, dtype=torch.int64, device=DEV)
                B.bmlp_int8_sign(a, w, out, thr, workspace=ws, expired=expired)
                assert torch.equal(out, want), (ws is None, expired)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", [(20011, 40), (20011, 100), (10007, 255), (20011, 784), (10007, 785), (10007, 1001), (1500, 4096),
                                 (1500, 4095), (1500, 8184)])
def test_norm_of_rows_past_a_turn(n, K, dtype):
    """More rows than the kernel's warps or CTAs take at once: those that follow, with the rows loaded
    ahead of an in-place sum and the places that rows keep from turn to turn."""
    x, res = hidden(n, K, n + K, dtype), hidden(n, K, n + 5 * K, dtype)
    gain = (1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to(dtype)
    for use_res in (False, True):
        r = res if use_res else None
        for use_gain in (False, True):
            gn = gain if use_gain else None
            h, want = plain_codes(x, r, gn)
            # (pad and start of the inputs, of the sums; in place)
            for pad, off, spad, soff, place in [(0, 0, 0, 0, None), (0, 0, 0, 0, "x"), (0, 0, 0, 0, "res"), (3, 1, 0, 0, None),
                                                (3, 1, 0, 0, "x"), (1, 0, 1, 0, "res"), (0, 0, 5, 3, None), (7, 2, 2, 1, None)]:
                if place == "res" and not use_res:
                    continue
                xd, rd = rows(n, K, dtype, pad, off)[1], rows(n, K, dtype, pad, off)[1]
                sb, sd = rows(n, K, dtype, spad, soff, fill=7)
                qb, qd = rows(n, K, torch.int8, spad, soff, fill=99)
                xd.copy_(x)
                rd.copy_(res)
                scale = torch.full((n,), -1.0, device=DEV)
                out = {"x": xd, "res": rd, None: sd}[place]
                B.bmlp_norm_quantize(xd, None if gn is None else gn.to(DEV), qd, scale, res=rd if use_res else None, sum_out=out,
                                     eps=1e-6)
                assert torch.equal(qd.cpu(), want), (use_res, use_gain, pad, place)
                assert torch.equal(out.cpu(), h.to(dtype)), (use_res, use_gain, pad, place)
                assert (qb[:soff] == 99).all() and (qb[soff + n * (K + spad):] == 99).all()
                if place is None:
                    assert (sb[:soff] == 7).all() and (sb[soff + n * (K + spad):] == 7).all()
                    if spad:
                        assert (sb[soff:soff + n * (K + spad)].view(n, -1)[:, K:] == 7).all()
            check_codes(qd.cpu(), scale.cpu(), x, r, gn, True, K)
    want = plain_codes(x)[1]
    for pad, off in [(0, 0), (3, 1)]:
        xd = rows(n, K, dtype, pad, off)[1]
        xd.copy_(x)
        _, qd = rows(n, K, torch.int8, pad, off, fill=99)
        scale = torch.full((n,), -1.0, device=DEV)
        B.bmlp_quantize_rows(xd, qd, scale)
        assert torch.equal(qd.cpu(), want)
        check_codes(qd.cpu(), scale.cpu(), x, None, None, False, K)


@gpu
def test_rows_of_thousands_of_slabs():
    """157 M rows without a workspace, 2,400 launches, from a thread with a small stack: the host
    side needs no more of it than for one."""
    n, N = 65536 * 2400 + 77, 130
    g = torch.Generator(device=DEV).manual_seed(1)
    a = torch.randint(-128, 128, (n, 1), generator=g, device=DEV).to(torch.int8)
    w = torch.randint(-128, 128, (N, 1), generator=g, device=DEV).to(torch.int8)
    thr = torch.randint(-9000, 9000, (N,), generator=g, device=DEV, dtype=torch.int32)
    out = torch.full((n, 3), -1, dtype=torch.int64, device=DEV)
    _, small = few_workspaces(n, 1, N)
    torch.cuda.synchronize()
    failed = []

    def call():
        try:
            B.bmlp_int8_sign(a, w, out, thr, workspace=small)
            torch.cuda.synchronize()
        except Exception as e:      # (to be raised below)
            failed.append(e)

    B.bmlp_int8_sign(a[:70000], w, out[:70000], thr, workspace=small)
    before = threading.stack_size(512 * 1024)
    try:
        t = threading.Thread(target=call)
        t.start()
        t.join()
    finally:
        threading.stack_size(before)
    assert not failed, failed
    # the words of each of the 256 codes
    values = torch.arange(-128, 128, device=DEV)
    bits = torch.zeros((256, 192), dtype=torch.bool, device=DEV)
    bits[:, :N] = values[:, None] * w[:, 0].long() >= thr.long()
    table = (bits.view(256, 3, 64).long() << torch.arange(64, device=DEV)).sum(2)
    for first in range(0, n, 1 << 24):
        rows = slice(first, min(n, first + (1 << 24)))
        assert torch.equal(out[rows], table[a[rows, 0].long() + 128])


# -- rows whose squares leave fp32 -----------------------------------------------------

@gpu
@pytest.mark.parametrize("K", [1, 7, 64, 257, 784, 4096, 8191, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
def test_norm_of_small_rows_at_small_eps(K, dtype):
    """The scale of rows down to the type's least values, where eps does not hold their mean
    square up: finite, and as the formula in 64 bits has it."""
    sizes = [1.0, 1e-5, 1e-12, 1e-14, 1e-18, 3e-20, 1e-21, 1e-23, 1e-25, 1e-30, 1e-35, 1e-37, 1e-42, 0.0]
    if dtype == torch.float16:
        sizes = [1.0, 1e-3, 1e-6, 6e-8, 0.0]
    n = len(sizes)
    g = torch.Generator().manual_seed(K)
    size = torch.tensor(sizes, dtype=torch.float64)[:, None]
    x = (torch.randn((n, K), generator=g, dtype=torch.float64) * size).to(dtype)
    res = (torch.randn((n, K), generator=g, dtype=torch.float64) * size).to(dtype)
    x[:, 0] = size[:, 0].to(dtype)      # (no row of a size is 0)
    res[:, 0] = 0
    for gain_size in (None, 1.0, 1e20):
        if gain_size == 1e20 and dtype == torch.float16:
            continue
        gain = None if gain_size is None else ((1 + 0.3 * torch.rand((K,), generator=g)) * gain_size).to(dtype)
        for eps in (0.0, 1e-45, 1e-38, 1e-30, 7e-25, 9e-25, 1e-12):
            for use_res, place in ((False, None), (True, None), (True, "x"), (True, "res"), (False, "x")):
                xd, rd = x.to(DEV), res.to(DEV) if use_res else None
                q = torch.full((n, K), 99, dtype=torch.int8, device=DEV)
                scale = torch.full((n,), -1.0, device=DEV)
                out = {"x": xd, "res": rd, None: None}[place]
                B.bmlp_norm_quantize(xd, None if gain is None else gain.to(DEV), q, scale, res=rd, sum_out=out, eps=eps)
                h = x.float() + res.float() if use_res else x.float()
                u = h if gain is None else h * gain.float()
                A = u.abs().amax(1)
                coded = A >= 127 * 2.0 ** -126
                inv = torch.full_like(A, 127.0) / torch.where(coded, A, 1)
                want_q = torch.round(torch.where(coded[:, None], u * inv[:, None], 0)).to(torch.int8)
                assert torch.equal(q.cpu(), want_q)
                if place:
                    assert torch.equal(out.cpu(), h.to(dtype))
                # h and A as they are in fp32, everything after them in 64 bits, with eps as the call has it
                eps32 = torch.tensor(eps, dtype=torch.float32).double()
                want = torch.where(coded, A.double() / 127 / torch.sqrt(h.double().square().mean(1) + eps32), 0)
                # roundings: A / 127, mean, eps, the addition, root, 1 / it, product; h^2 and its sum of at
                # most K / 256 + 16 additions in sequence, halved by the root; a subnormal result's last place
                tol = (8 + (K / 256 + 20) / 2) * 2.0 ** -24 * want + 2.0 ** -149
                got = scale.cpu().double()
                assert torch.isfinite(got).all(), (eps, gain_size, got)
                assert ((got - want).abs() <= tol).all(), (eps, gain_size, got, want)
