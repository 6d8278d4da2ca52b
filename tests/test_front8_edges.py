"""The 8-bit front end past the sizes of its other tests: rows and channels that leave 31
bits or a slab, second turns of persistent kernels, rows whose squares leave fp32, and
tensors that do not belong to the call."""
import threading

import pytest
import torch

from paper_2412_00119_gb300 import bmlp as B

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
