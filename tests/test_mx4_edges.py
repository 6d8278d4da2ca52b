"""The 4-bit front end past its other tests: the binding's native module and the torch it belongs to, the kernel of
each instance and plan, rows at odd places, operands that tensor copies refuse, and values at
the ends of fp32."""
import os
import shutil

import pytest
import torch

from paper_2412_00119_gb300 import _build, bmlp as B
from test_mx4 import (DEV, EPS, GROUPS, TYPES, U8, bound, coded, decoded, finish, hidden, plain_codes, rows, same_codes, unpack,
                      untouched)

gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            pytest.skip("needs a GPU")
        torch.cuda.set_device(DEV)


# -- the binding's native module ---------------------------------------------------------

def own_module():
    return _build.marshal_path(torch.__version__, torch.version.git_version)


@pytest.fixture
def unloaded(monkeypatch):
    """As before the first call."""
    B._marshal()
    monkeypatch.setattr(B, "_native", None)


def test_module_of_another_torch_is_not_loaded(unloaded, monkeypatch):
    """It reads tensors as they lie in its own torch's memory."""
    names = {own_module(), _build.marshal_path("1.0", torch.version.git_version),
             _build.marshal_path(torch.__version__, "0" * 40), _build.marshal_path(torch.__version__, None)}
    assert len(names) == 4 and all(os.path.dirname(n) == _build.HERE for n in names)
    monkeypatch.setattr(torch, "__version__", "1.0")
    assert B._marshal() is B._NoMarshal
    monkeypatch.undo()


def test_module_that_the_first_call_builds_is_found(unloaded, monkeypatch, tmp_path):
    if not os.path.exists(own_module()):
        pytest.skip("built where there are torch's headers")
    real, path = own_module(), str(tmp_path / os.path.basename(own_module()))
    L = B.lib()

    def building():
        shutil.copy(real, path)
        return L

    monkeypatch.setattr(B, "lib", building)
    monkeypatch.setattr(_build, "marshal_path", lambda *_: path)
    assert B._marshal() is not B._NoMarshal


@gpu
def test_native_module_takes_calls():
    """It is there, takes what is as it should be (0), and leaves the rest to the interpreter's way (SLOW)."""
    M = B._marshal()
    if _build._marshal_job(force=True) is None:
        pytest.skip("no torch headers to build it with")
    assert M is not B._NoMarshal
    n, K, N, E = 5, 64, 8, 2
    x = torch.randn((n, K), device=DEV)
    q, s = B.bmlp_mx4_empty(n, K)
    w, ws = B.bmlp_mx4_empty((E, N), K)
    B.bmlp_mx4_quantize(torch.randn((E * N, K), device=DEV), w.flatten(0, 1), ws.flatten(0, 1))
    by, out = torch.empty(n, device=DEV), torch.empty((n, N), device=DEV)
    at = torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV)
    good = [(M.quantize, [x, q, s]), (M.norm_quantize, [x, None, q, s, by, None, None, 1e-6]),
            (M.dequantize, [q, s, torch.empty_like(x), by]), (M.matmul, [q, s, w[0], ws[0], out, by, None]),
            (M.matmul_grouped, [q, s, w, ws, at, out, None, None])]
    for call, args in good:
        assert call(*args) == 0
        for i, a in enumerate(args):
            if not isinstance(a, torch.Tensor):
                continue
            for wrong in (None, 3, a.cpu(), a.double(), a[:-1], a.unsqueeze(0)):
                if wrong is None and call in (M.dequantize, M.matmul) and a is by:
                    continue
                assert call(*args[:i], wrong, *args[i + 1:]) == M.SLOW, (call, i)
    assert M.quantize(x, q.t(), s) == M.SLOW
    with pytest.raises(TypeError):
        M.quantize(x, q)
    torch.cuda.synchronize()


# -- rows to codes and back ----------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", [(5, 1), (300, 7), (40, 129), (9, 1001), (3, 4099), (400, 4099), (5, 9001), (2, 33001)])
def test_norm_in_place_at_odd_places(n, K, dtype):
    """The sum over the rows that it is made of, where they start anywhere."""
    x, res = hidden(n, K, 1, dtype), hidden(n, K, 2, dtype)
    h = x.float() + res.float()
    want, (c, s) = h.to(dtype), plain_codes(h)
    for eps in (EPS, 0.0):
        for pad, off in ((0, 0), (3, 1)):
            for into in (0, 1):
                (xb, xd), (rb, rd) = rows(n, K, dtype, pad, off, fill=3), rows(n, K, dtype, pad, off, fill=3)
                xd.copy_(x)
                rd.copy_(res)
                q, sd = B.bmlp_mx4_empty(n, K)
                by = torch.empty((n,), device=DEV)
                B.bmlp_mx4_norm_quantize(xd, None, q, sd, by, res=rd, sum_out=(xd, rd)[into], eps=eps)
                assert torch.equal((xd, rd)[into].cpu(), want) and torch.equal((rd, xd)[into].cpu(), (res, x)[into])
                assert untouched(xb, n, K, pad, off, 3) and untouched(rb, n, K, pad, off, 3)
                assert torch.equal(sd.cpu(), s) and same_codes(unpack(q.cpu(), K), c)


@gpu
@pytest.mark.parametrize("K", [64, 1001])
def test_values_past_fp32_times_a_small_factor(K):
    """Of scales 2^126 and 2^127: the value leaves fp32, its product with the row's factor has one rounding."""
    by = torch.tensor([1.0, 0.3, 2.0 ** -10, -2.0 ** -126 * 1.7, 2.0 ** -149, 0.0, 3.0, float("inf"), float("nan"), 2.0 ** 124,
                       -2.0 ** 126, 2.0 ** 123 * 1.9, -0.7])
    n = len(by)
    for pad in (-1, 3):
        q, s = coded(n, K, 5, span=4, base=251, pad=pad)
        # (on the CPU: a device's pow in 64 bits is off by a bit at 2^122; code and factor have 27 bits together)
        value = decoded(q.cpu(), s.cpu(), K)
        for factor in (by, None):
            want = (value if factor is None else value * factor.double()[:, None]).float()
            for t in TYPES:
                _, out = rows(n, K, t, max(pad, 0))
                B.bmlp_mx4_dequantize(q, s, out, row_scale=None if factor is None else factor.to(DEV))
                got, ref = out.cpu().double(), want.to(t).double()
                bad = (got != ref) & ~(got.isnan() & ref.isnan())
                assert not bad.any(), (t, pad, torch.nonzero(bad)[:5].tolist(), got[bad][:5], ref[bad][:5])


# -- operands of products ------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("n,K,N", [(90, 256, 70), (9, 1000, 130), (300, 100, 200)])
def test_groups_in_other_orders(n, K, N):
    """Groups whose rows lie between one another's (a group stride below the row stride), and a group stride that is no multiple of the rows'."""
    E, kb, ks = 3, (K + 1) // 2, (K + 31) // 32
    a, sa = coded(n, K, 1, span=1)
    at = torch.tensor([0, n // 4, n // 4, n - 3], dtype=torch.int32, device=DEV)

    def laid(t, order):
        size = t.shape[-1]
        wide = (size + 15) // 16 * 16
        if order == "between":
            buf = torch.full((N, E, wide), 255, dtype=t.dtype, device=DEV)
            v = buf[..., :size].transpose(0, 1)
        else:
            buf = torch.full((E * (N * wide + 16),), 255, dtype=t.dtype, device=DEV)
            v = buf.as_strided((E, N, size), (N * wide + 16, wide, 1))
        v.copy_(t)
        return v

    w, sw = coded((E, N), K, 3, span=1)
    want = torch.full((n, N), -5.0, dtype=torch.float64, device=DEV)
    for e in range(E):
        r = slice(int(at[e]), int(at[e + 1]))
        want[r] = decoded(a[r], sa[r], K) @ decoded(w[e], sw[e], K).t()
    for order in ("between", "apart"):
        wl, sl = laid(w, order), laid(sw, order)
        assert (wl.shape[-1], sl.shape[-1]) == (kb, ks) and (order == "apart" or wl.stride(0) < wl.stride(1))
        out = torch.full((n, N), -5.0, device=DEV)
        B.bmlp_mx4_matmul_grouped(a, sa, wl, sl, at, out)
        assert torch.equal(out.double(), want), order


# -- products of many rows: the pairs, at sizes of any kind ------------------------------------
#
# Codes in rows at multiples of 16 bytes, scales anywhere.  As in test_mx4, sums are exact in fp32 in any order:
# multiples of a quarter, fewer than 2^24 of them.

def check_pairs(K, N, n=None, sizes=None, scale_pad=-1, out_type=torch.float32, extra=True, ldo=0, before=0, after=0,
                span=1, call=None, **kw):
    E = 1 if sizes is None else len(sizes)
    at = torch.tensor([0, n] if sizes is None else [before] + (before + torch.tensor(sizes).cumsum(0)).tolist())
    n = int(at[-1]) + after
    a, w = coded(n, K, n + K)[0], coded((E, N), K, N + K)[0]
    sa, sw = coded(n, K, n + K + 1, span=span, pad=scale_pad)[1], coded((E, N), K, N + K + 1, span=span, pad=scale_pad)[1]
    if after:
        sa[n - after:] = 255     # of rows in no group nothing matters
    by = torch.rand((n,), generator=torch.Generator().manual_seed(n)).to(DEV) + 0.5 if extra else None
    bias = torch.randn((E, N), generator=torch.Generator().manual_seed(N)).to(DEV) if extra else None
    ob, out = rows(n, N, out_type, ldo, 0, fill=-5)
    want = torch.full((n, N), -5, dtype=out_type, device=DEV)
    for e in range(E):
        r = slice(int(at[e]), int(at[e + 1]))
        if r.start < r.stop:
            x, y = decoded(a[r], sa[r], K), decoded(w[e], sw[e], K)
            assert 4 * (x.abs() @ y.abs().t()).max() < 2 ** 24
            want[r] = finish(x @ y.t(), by[r] if extra else None, bias[e] if extra else None, out_type)
    if sizes is None:
        (call or B.bmlp_debug_mx4_pairs)(a, sa, w[0], sw[0], *((None,) if call is None else ()), out, row_scale=by,
                                         bias=bias[0] if extra else None, **kw)
    else:
        (call or B.bmlp_debug_mx4_pairs)(a, sa, w, sw, at.to(torch.int32).to(DEV), out, row_scale=by, bias=bias, **kw)
    bad = out != want
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:5].tolist(), out[bad][:5], want[bad][:5])
    assert untouched(ob, n, N, ldo, 0, -5)


@gpu
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 100, 127, 128, 129, 144, 160, 161, 255, 256, 257, 300, 511, 513, 2100])
def test_pairs_over_rows(n):
    check_pairs(512, 130, n)
    check_pairs(203, 70, n, scale_pad=5, out_type=torch.bfloat16, ldo=3)
    check_pairs(1300, 300, n, scale_pad=0, out_type=torch.float16, extra=False)


@gpu
@pytest.mark.parametrize("K", [1, 2, 31, 32, 33, 63, 64, 65, 97, 127, 128, 129, 192, 255, 256, 257, 511, 512, 513, 769, 1000, 1023, 1024,
                               1025, 1281, 1536, 1793, 2047, 2048, 2049, 2305, 2561, 4095, 4097, 5000])
def test_pairs_over_depth(K):
    for n, scale_pad in ((150, -1), (290, 0), (290, 1)):
        check_pairs(K, 300, n, scale_pad=scale_pad)


@gpu
@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 127, 128, 129, 159, 255, 256, 257, 385, 511, 513, 1001])
def test_pairs_over_channels(N):
    for n, out_type in ((40, torch.float16), (260, torch.float32), (520, torch.bfloat16)):
        check_pairs(784, N, n, out_type=out_type, extra=n != 260, ldo=n % 8)


@gpu
@pytest.mark.parametrize("n,K,N", [(40000, 64, 48), (20000, 300, 1000), (60001, 33, 257), (6000, 1100, 1500), (5000, 2300, 1400),
                                   (30000, 520, 700), (3000, 4096, 2100), (600, 16384, 300)])
@pytest.mark.parametrize("scale_pad", [-1, 3])
def test_pairs_of_several_tiles(n, K, N, scale_pad):
    """Tiles one after another in a pair of CTAs, with units of one to four steps at their ends."""
    check_pairs(K, N, n, scale_pad=scale_pad, out_type=torch.bfloat16 if n > 10000 else torch.float32, span=0 if K > 4000 else 1)


@gpu
@pytest.mark.parametrize("sizes", GROUPS + [[1] * 256, [300, 0, 5] * 60], ids=lambda s: "%dx%d" % (len(s), sum(s)))
def test_pairs_by_group(sizes):
    check_pairs(512, 130, sizes=sizes)
    check_pairs(203, 70, sizes=sizes, scale_pad=3, out_type=torch.bfloat16, before=3, after=40, ldo=1)
    check_pairs(1100, 260, sizes=sizes, out_type=torch.float16, extra=False, after=1)


@gpu
def test_pairs_by_long_groups():
    check_pairs(1024, 2050, sizes=[3000, 1, 0, 2900, 513], out_type=torch.bfloat16, after=700)
    check_pairs(300, 700, sizes=[7000, 9000, 4001], scale_pad=1, before=100)


@gpu
@pytest.mark.parametrize("n,K,N", [(1, 64, 5), (100, 512, 200), (600, 1100, 300), (9000, 300, 700)])
def test_pairs_expired(n, K, N):
    for scale_pad in (-1, 3):
        check_pairs(K, N, n, scale_pad=scale_pad, expired=True)
        check_pairs(K, N, sizes=[n // 3, 0, n - n // 3], scale_pad=scale_pad, after=5, expired=True)
    check_pairs(K, N, n)


@gpu
def test_pairs_of_any_scales():
    for n, K, N in ((130, 4096, 500), (300, 1001, 200)):
        a, sa = coded(n, K, 1, span=40, base=107)
        w, sw = coded(N, K, 2, span=40, base=87)
        sa[n // 2, 3] = 255
        sw[17, 19] = 255
        sw[40] = 0          # 2^-127
        sa[0, 5:8] = 0
        x, y = decoded(a, sa, K), decoded(w, sw, K)
        out = torch.empty((n, N), device=DEV)
        B.bmlp_debug_mx4_pairs(a, sa, w, sw, None, out)
        S = x @ y.t()
        assert torch.equal(out.isnan(), S.isnan())
        x, y = x.nan_to_num(nan=0.0), y.nan_to_num(nan=0.0)
        # (what is below fp32's normal numbers may be lost)
        lim = bound(x, y, K) + 2.0 ** -24 * S.abs() + K * 2.0 ** -126
        assert ((out.double() - S).abs() <= lim)[~S.isnan()].all()


@gpu
@pytest.mark.parametrize("n,K,N,sizes", [(4096, 4096, 4100, None), (16384, 512, 4096, None), (None, 2048, 4096, [1500, 0, 2100, 1200, 3000])],
                         ids=str)
def test_products_of_many_rows(n, K, N, sizes):
    """Long prompts, by the rule: each on the kernel that it takes."""
    call = B.bmlp_mx4_matmul if sizes is None else B.bmlp_mx4_matmul_grouped
    check_pairs(K, N, n, sizes=sizes, out_type=torch.bfloat16, span=0, call=call, after=0 if sizes is None else 9)


@gpu
def test_pairs_beside_other_kernels():
    """On three streams at once with tiles of every kind, and back to back: their CTAs share SMs and tensor memory."""
    jobs = []
    for n, K, N, pad, pairs in [(600, 1024, 700, -1, True), (2000, 512, 1500, -1, True), (300, 2048, 4000, -1, True),
                                (20, 2048, 3000, -1, False), (9, 8192, 256, -1, False), (200, 1000, 500, 1, False)]:
        (a, sa), (w, sw) = coded(n, K, 1, span=0, pad=pad), coded(N, K, 2, span=0, pad=pad)
        want = (decoded(a, sa, K) @ decoded(w, sw, K).t()).float()

        def call(st, out, a=a, sa=sa, w=w, sw=sw, pairs=pairs):
            if pairs:
                B.bmlp_debug_mx4_pairs(a, sa, w, sw, None, out, stream=st)
            else:
                B.bmlp_mx4_matmul(a, sa, w, sw, out, stream=st)
        jobs.append((want, [torch.empty((n, N), device=DEV) for _ in range(3)], call))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for rep in range(10):
        for k in range(3 * len(jobs)):
            want, outs, call = jobs[(5 * k + rep) % len(jobs)]
            i = (k + k // len(jobs)) % 3     # (every job once on every stream)
            call(streams[i], outs[i])
        torch.cuda.synchronize()
        for want, outs, _ in jobs:
            for out in outs:
                assert torch.equal(out, want)
                out.fill_(-1)
        torch.cuda.synchronize()


@gpu
def test_pairs_on_what_the_kernel_before_writes():
    """Norm, product and quantisation depend on one another with nothing between; captured, and replayed on other
    inputs."""
    n, K = 700, 768
    w, sw = coded(K, K, 2, span=0)
    q, s = B.bmlp_mx4_empty(n, K)
    x, by = hidden(n, K, 1, torch.bfloat16).to(DEV), torch.empty((n,), device=DEV)
    y = torch.empty((n, K), dtype=torch.bfloat16, device=DEV)
    st = torch.cuda.Stream()

    def step(wait=lambda: None):
        B.bmlp_mx4_norm_quantize(x, None, q, s, by, eps=EPS, stream=st)
        wait()
        B.bmlp_debug_mx4_pairs(q, s, w, sw, None, y, row_scale=by, stream=st)
        wait()
        B.bmlp_mx4_quantize(y, q, s, stream=st)
        wait()
        B.bmlp_debug_mx4_pairs(q, s, w, sw, None, y, stream=st)

    torch.cuda.synchronize()
    step()
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        for _ in range(3):
            step()
    for seed in (3, 4, 5):
        x.copy_(hidden(n, K, seed, torch.bfloat16))
        torch.cuda.synchronize()
        step(st.synchronize)
        st.synchronize()
        want = y.clone()
        y.fill_(0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@gpu
def test_pairs_refuse_what_they_do_not_take():
    a, sa = coded(9, 64, 1)
    w, sw = coded((257, 5), 64, 2)
    out = torch.empty((9, 5), device=DEV)
    with pytest.raises(B.BmlpError, match="multiples of 16"):
        B.bmlp_debug_mx4_pairs(a, sa, w, sw, torch.zeros(258, dtype=torch.int32, device=DEV), out)
    odd = coded(9, 64, 1, pad=1)
    with pytest.raises(B.BmlpError, match="multiples of 16"):
        B.bmlp_debug_mx4_pairs(*odd, w[0], sw[0], None, out)


# -- instances with loads ahead -----------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,K", [(4900, 1024), (1300, 4500), (2500, 2049), (9800, 513), (5000, 1100)])
def test_many_long_rows(n, K, dtype):
    """So many that a warp has four of its loads under way (in each direction, at any place), with whole and ragged
    last parts and several rows a CTA."""
    kb, ks = (K + 1) // 2, (K + 31) // 32
    x = hidden(n, K, n + K, dtype)
    c, s = plain_codes(x.float())
    for pad, off in ((-1, 0), (3, 1)):
        _, xd = rows(n, K, dtype, pad, off)
        qb, qd = rows(n, kb, U8, pad, off, fill=99)
        sb, sd = rows(n, ks, U8, pad, off, fill=98)
        xd.copy_(x)
        B.bmlp_mx4_quantize(xd, qd, sd)
        q = qd.cpu()
        assert torch.equal(sd.cpu(), s) and same_codes(unpack(q, K), c)
        assert K % 2 == 0 or (q[:, -1] >> 4 == 0).all()
        assert untouched(qb, n, kb, pad, off, 99) and untouched(sb, n, ks, pad, off, 98)
        ob, od = rows(n, K, dtype, pad, off, fill=7)
        B.bmlp_mx4_dequantize(qd, sd, od)
        # (a value has two bits after its first, in bf16's and fp32's range)
        assert torch.equal(od, decoded(qd, sd, K).to(torch.float32).to(dtype)) and untouched(ob, n, K, pad, off, 7)
