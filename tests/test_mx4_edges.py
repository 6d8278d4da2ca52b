"""The 4-bit front end past its other tests: the binding's native module and the torch it belongs to, the kernel of
each instance and plan, rows at odd places, operands that tensor copies refuse, and values at
the ends of fp32."""
import os
import shutil

import pytest
import torch

from paper_2412_00119_gb300 import _build, bmlp as B
from test_mx4 import DEV, EPS, TYPES, coded, decoded, hidden, plain_codes, rows, same_codes, unpack, untouched

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
    by = torch.tensor([1.0, 0.3, 2.0 ** -10, -2.0 ** -126 * 1.7, 2.0 ** -149, 0.0, 3.0, float("inf"), float("nan")])
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
