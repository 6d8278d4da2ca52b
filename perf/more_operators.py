"""Measured cases of the microscaled 4-bit front end: real-valued rows -- hidden
states of a language model, channels of its projections -- as 4-bit floating-point
codes (e2m1, two per byte) with a power-of-two scale per 32 of them, and the
products of such rows, over the range of their use.

A case is a dict of plain values; ``kind`` names the call:

  quantize  bmlp_mx4_quantize, then bmlp_mx4_dequantize: n rows of K values to codes
            and scales, and the values that these stand for (bf16 holds them exactly)
  norm      bmlp_mx4_norm_quantize: root-mean-square norm of n rows, with the
            residual's addition, to codes, scales and a factor per row; then
            bmlp_mx4_dequantize with that factor: the normed rows as 4 bits hold them
  matmul    bmlp_mx4_matmul: n x K codes times (N x K)^T
  grouped   bmlp_mx4_matmul_grouped: the same with weights E x N x K, row i taking
            those of the group that offsets put it in
  linear    norm, then matmul: a projection of hidden states

``types`` is the type of the real-valued input (norm, quantize, linear) or of the
output (matmul, grouped).  Rows of codes and scales start at multiples of 16 bytes
where ``pad`` is -1, else ``pad`` bytes (of real values: elements) lie between them.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6


def listed():
    return [
        # the channels of a projection, once per model that is loaded, and what they became
        dict(name="quantize 8192x8192 bf16", kind="quantize", n=8192, K=8192, types="bf16", pad=-1),
        # odd rows of a wider buffer
        dict(name="quantize 257x1001 f16", kind="quantize", n=257, K=1001, types="f16", pad=7),
        # one token's hidden state between two layers: latency counts
        dict(name="norm 1x8192 bf16", kind="norm", n=1, K=8192, types="bf16", residual=True, pad=-1),
        # the hidden states of a long prompt
        dict(name="norm 8191x4096 bf16", kind="norm", n=8191, K=4096, types="bf16", residual=True, pad=-1),
        # one token through a projection: the weights' bytes
        dict(name="matmul 1x8192x8192", kind="matmul", n=1, K=8192, N=8192, types="bf16", bias=False, pad=-1),
        # a mini-batch of 100
        dict(name="matmul 100x4096x8192", kind="matmul", n=100, K=4096, N=8192, types="bf16", bias=False, pad=-1),
        # 1,000 features, rows of 500 bytes one after another
        dict(name="matmul 1000x1000x525 f32", kind="matmul", n=1000, K=1000, N=525, types="f32", bias=True, pad=0),
        # a long prompt through a projection: the tensor cores
        dict(name="matmul 16384x8192x8192", kind="matmul", n=16384, K=8192, N=8192, types="bf16", bias=False, pad=-1),
        # a serving step's tokens, three to an expert: the experts' bytes
        dict(name="grouped 96x4096x2048 by 32", kind="grouped", n=96, K=4096, N=2048, E=32, used=96,
             types="bf16", bias=False, pad=-1),
        # a long prompt's tokens by expert
        dict(name="grouped 16384x4096x4096 by 16", kind="grouped", n=16384, K=4096, N=4096, E=16, used=16384,
             types="bf16", bias=False, pad=-1),
        # small experts at odd sizes, some of them without rows, and a padded batch's last rows in none
        dict(name="grouped 1500x784x1001 by 40 f32", kind="grouped", n=1500, K=784, N=1001, E=40, used=1391,
             types="f32", bias=True, pad=3),
        # the whole way for the few requests of one serving step
        dict(name="linear 7x4096x8192", kind="linear", n=7, K=4096, N=8192, types="bf16", residual=True, bias=False,
             pad=-1),
    ]


# Multiply-accumulates that a drawn product may cost (the largest listed one: 1.1e12), values
# that a drawn norm or quantisation may read (the listed one: 6.7e7) and that a drawn set of
# experts may have (the listed ones: 2.7e8).
_MOST_MACS, _MOST_VALUES, _MOST_WEIGHTS = 1.0e12, 6.0e7, 2.5e8


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return max(lo, w // 64 * 64) if w >= 128 and rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "norm", "norm", "matmul", "matmul", "matmul", "grouped", "grouped",
                       "grouped", "linear"])
    K = _width(rng, 48, 16384)
    case = dict(kind=kind, K=K, pad=rng.choice([-1, -1, -1, rng.randint(0, 64)]))
    if kind in ("norm", "quantize"):
        case.update(n=_log(rng, 1, min(65536, _MOST_VALUES // K)), types=rng.choice(["bf16", "f16", "f32"]))
        if kind == "norm":
            case.update(residual=rng.random() < 0.7)
        return case
    if kind == "grouped":
        E = _log(rng, 2, 128)
        N = _width(rng, 32, max(64, min(8192, int(_MOST_WEIGHTS / (K * E)))))
        n = _log(rng, 1, min(32768, int(0.25 * _MOST_MACS / (K * N))))
        used = n if rng.random() < 0.7 else rng.randint(0, n)
        case.update(E=E, N=N, n=n, used=used, types=rng.choice(["bf16", "bf16", "f16", "f32"]), bias=rng.random() < 0.3)
        return case
    N = _width(rng, 32, 16384)
    case.update(N=N, n=_log(rng, 1, min(65536, int(_MOST_MACS / (K * N)))))
    case.update(types=rng.choice(["bf16", "bf16", "f16", "f32"]), bias=rng.random() < 0.3)
    if kind == "linear":
        case.update(residual=rng.random() < 0.7)
    return case


# -- inputs ---------------------------------------------------------------------

def _rows(n, K, pad, dtype):
    """n x K of a new buffer with that padding between its rows."""
    wide = (K + 15) // 16 * 16 if pad < 0 else K + pad
    return torch.zeros((n, wide), dtype=dtype, device="cuda")[:, :K]


def _hidden(n, K, g):
    """Hidden states as a language model has them: normal values, one channel in
    128 of 16 times the others' size, and rows of different sizes."""
    x = torch.randn((n, K), generator=g, device="cuda")
    big = torch.rand((K,), generator=g, device="cuda") < 1 / 128
    size = torch.exp(0.5 * torch.randn((n, 1), generator=g, device="cuda"))
    return x * torch.where(big, 16.0, 1.0) * size


def _coded(x, pad):
    """Codes and scales of the rows of x, in buffers of padded rows."""
    n, K = x.shape
    q, scale = _rows(n, (K + 1) // 2, pad, torch.uint8), _rows(n, (K + 31) // 32, pad, torch.uint8)
    values, s = _plain_codes(x)
    m = values.abs()
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)) + 8 * (values < 0)
    code = torch.nn.functional.pad(code, (0, K % 2)).to(torch.uint8).view(n, -1, 2)
    q.copy_(code[:, :, 0] + 16 * code[:, :, 1])
    scale.copy_(s)
    return q, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, n, K, pad = case["kind"], case["n"], case["K"], case["pad"]
    s = dict(case=case, table=torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda"))
    if kind in ("norm", "quantize", "linear"):
        dtype = _TYPES[case["types"]]
        s["x"] = _rows(n, K, max(pad, 0), dtype)
        if kind == "quantize":
            s["x"].copy_(0.02 * torch.randn((n, K), generator=g, device="cuda"))
            s["values"] = torch.empty((n, K), dtype=torch.bfloat16, device="cuda")
        else:
            s["x"].copy_(_hidden(n, K, g))
            s["gain"] = (1 + 0.2 * torch.randn((K,), generator=g, device="cuda")).to(dtype)
            s["row_scale"] = torch.empty((n,), device="cuda")
            s["values"] = torch.empty((n, K), dtype=dtype, device="cuda")
        s["res"] = s["sum"] = None
        if case.get("residual"):
            s["res"] = _rows(n, K, max(pad, 0), dtype)
            s["res"].copy_(_hidden(n, K, g))
            s["sum"] = torch.empty((n, K), dtype=dtype, device="cuda")
        s["q"], s["scale"] = _rows(n, (K + 1) // 2, pad, torch.uint8), _rows(n, (K + 31) // 32, pad, torch.uint8)
    if kind in ("matmul", "grouped", "linear"):
        N, E = case["N"], case.get("E", 1)
        w, ws = _coded(0.02 * torch.randn((E * N, K), generator=g, device="cuda"), pad)
        s["w"], s["w_scale"] = (w, ws) if kind != "grouped" else (w.unflatten(0, (E, N)), ws.unflatten(0, (E, N)))
        if kind != "linear":
            s["a"], s["a_scale"] = _coded(_hidden(n, K, g), pad)
            s["row_scale"] = torch.rand((n,), generator=g, device="cuda") + 0.5
        s["bias"] = None
        if case["bias"]:
            s["bias"] = torch.randn((E, N) if kind == "grouped" else (N,), generator=g, device="cuda")
        s["out"] = torch.zeros((n, N), dtype=_TYPES[case["types"]], device="cuda")
        if kind == "grouped":
            # sizes of groups: some experts are asked for several times as often as others
            often = torch.exp(0.7 * torch.randn((E,), generator=g, device="cuda"))
            of = torch.multinomial(often, max(1, case["used"]), replacement=True, generator=g)[:case["used"]]
            sizes = (of[:, None] == torch.arange(E, device="cuda")).sum(0)
            s["offsets"] = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).to(torch.int32)
            s["largest"] = int(sizes.max())
    return s


# -- the plain forms ------------------------------------------------------------

def _plain_codes(u):
    """What the codes of the rows of u stand for before their blocks' scales, and those scales' bytes."""
    n, K = u.shape
    blocks = torch.nn.functional.pad(u, (0, -K % 32)).view(n, -1, 32)
    most = blocks.abs().amax(2)
    s = torch.where(most > 0, (torch.frexp(most).exponent + 124).clamp(0, 254), 0)
    t = torch.ldexp(blocks, 127 - s[:, :, None])
    m = t.abs()
    m = torch.where(m < 2, torch.round(2 * m) / 2, torch.where(m < 4, torch.round(m), 2 * torch.round(m / 2))).clamp(max=6)
    return torch.where(t < 0, -m, m).view(n, -1)[:, :K], s


def _scaled(values, s):
    n, K = values.shape
    blocks = torch.nn.functional.pad(values, (0, -K % 32)).view(n, -1, 32)
    return torch.ldexp(blocks, s[:, :, None] - 127).view(n, -1)[:, :K]


def _decoded(q, scale, table, K):
    """The fp32 values of packed codes."""
    both = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1)[:, :K]
    return _scaled(table[both.long()], scale.to(torch.int32))


def _plain_norm(s):
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    values, scale = _plain_codes(h * s["gain"].float())
    total = {"sum": h.to(s["x"].dtype)} if s["res"] is not None else {}
    return _scaled(values, scale), torch.rsqrt((h * h).mean(1) + _EPS), total


def _plain_out(y, s, row_scale):
    y = y * row_scale[:, None]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y


def _plain(s):
    case = s["case"]
    kind, K = case["kind"], case["K"]
    if kind == "quantize":
        return {"values": _scaled(*_plain_codes(s["x"].float())).to(torch.bfloat16)}
    if kind == "norm":
        values, rstd, total = _plain_norm(s)
        return {"values": (values * rstd[:, None]).to(s["x"].dtype), "row_scale": rstd} | total
    if kind == "linear":
        values, rstd, total = _plain_norm(s)
        y = torch.mm(values, _decoded(s["w"], s["w_scale"], s["table"], K).t())
        return {"out": _plain_out(y, s, rstd).to(s["out"].dtype)} | total
    a = _decoded(s["a"], s["a_scale"], s["table"], K)
    w = _decoded(s["w"].flatten(0, -2), s["w_scale"].flatten(0, -2), s["table"], K)
    if kind == "matmul":
        return {"out": _plain_out(torch.mm(a, w.t()), s, s["row_scale"]).to(s["out"].dtype)}
    # groups side by side, each with room for the largest (and a place for rows of none)
    E, N, at = case["E"], case["N"], s["offsets"].long()
    i = torch.arange(case["n"], device="cuda")
    e = (i[:, None] >= at[1:]).sum(1)
    some = e < E
    e = e.clamp(max=E - 1)
    place = torch.where(some, i - at[e], s["largest"])
    side = torch.zeros((E, s["largest"] + 1, K), device="cuda")
    side[e, place] = a
    y = torch.bmm(side, w.view(E, N, K).transpose(1, 2))[e, place] * s["row_scale"][:, None]
    if s["bias"] is not None:
        y = y + s["bias"][e]
    return {"out": torch.where(some[:, None], y.to(s["out"].dtype), s["out"])}


# -- the framework's operators ----------------------------------------------------

def _operators(s):
    from paper_2412_00119_gb300 import bmlp as B
    kind = s["case"]["kind"]
    if kind == "quantize":
        B.bmlp_mx4_quantize(s["x"], s["q"], s["scale"])
        B.bmlp_mx4_dequantize(s["q"], s["scale"], s["values"])
        return {"values": s["values"]}
    if kind == "matmul":
        B.bmlp_mx4_matmul(s["a"], s["a_scale"], s["w"], s["w_scale"], s["out"], row_scale=s["row_scale"], bias=s["bias"])
        return {"out": s["out"]}
    if kind == "grouped":
        B.bmlp_mx4_matmul_grouped(s["a"], s["a_scale"], s["w"], s["w_scale"], s["offsets"], s["out"],
                                  row_scale=s["row_scale"], bias=s["bias"])
        return {"out": s["out"]}
    B.bmlp_mx4_norm_quantize(s["x"], s["gain"], s["q"], s["scale"], s["row_scale"], res=s["res"], sum_out=s["sum"], eps=_EPS)
    total = {"sum": s["sum"]} if s["sum"] is not None else {}
    if kind == "norm":
        B.bmlp_mx4_dequantize(s["q"], s["scale"], s["values"], row_scale=s["row_scale"])
        return {"values": s["values"], "row_scale": s["row_scale"]} | total
    B.bmlp_mx4_matmul(s["q"], s["scale"], s["w"], s["w_scale"], s["out"], row_scale=s["row_scale"], bias=s["bias"])
    return {"out": s["out"]} | total


def run(s):
    return _operators(s) if own else _plain(s)


# -- the definition in 64 bits ------------------------------------------------------

def _exact_values(u):
    """The values, in 64 bits, that 4 bits and a scale per 32 hold of u: of the 15 multiples of the
    scale, the nearest, of two the one whose code is even."""
    n, K = u.shape
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    edge = (grid[1:] + grid[:-1]) / 2
    odd = torch.arange(7, device="cuda") % 2 == 1      # a tie above an odd code goes up
    got = torch.zeros_like(u)
    for k in range(0, K, 32):
        b = u[:, k:k + 32]
        most = b.abs().max(1, keepdim=True).values
        # (log2's rounding is kept off the powers of two)
        p = torch.floor(torch.log2(most.clamp(min=2.0 ** -1000)))
        p = torch.where(most >= 2.0 ** (p + 1), p + 1, torch.where(most < 2.0 ** p, p - 1, p))
        unit = 2.0 ** (p - 2).clamp(min=-127.0)
        m = (b.abs() / unit)[:, :, None]
        at = ((m > edge) | ((m == edge) & odd)).sum(2)
        got[:, k:k + 32] = torch.sign(b) * grid[at] * unit
    return got


def _exact_decoded(q, scale, K):
    """Values from the fields of the codes: sign, two exponent bits, one of mantissa."""
    v = torch.zeros((q.shape[0], 2 * q.shape[1]), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (q >> (4 * half)) & 15
        e, m = ((c >> 1) & 3).double(), (c & 1).double()
        v[:, half::2] = torch.where(e > 0, 2.0 ** (e - 1) * (1 + m / 2), m / 2) * torch.where(c > 7, -1.0, 1.0)
    return v[:, :K] * (2.0 ** (scale.double() - 127)).repeat_interleave(32, dim=1)[:, :K]


def exact(case, seed):
    kind, n, K = case["kind"], case["n"], case["K"]
    s = prepare(case, seed)
    if kind == "quantize":
        return {"values": _exact_values(s["x"].double())}
    got = {}
    if kind in ("norm", "linear"):
        x = s["x"].double()
        if s["res"] is not None:
            x = x + s["res"].double()
            got["sum"] = x
        rstd = 1 / torch.sqrt(x.square().sum(1) / K + _EPS)
        a = _exact_values(x * s["gain"].double())
        if kind == "norm":
            return got | {"values": a * rstd[:, None], "row_scale": rstd}
    else:
        a, rstd = _exact_decoded(s["a"], s["a_scale"], K), s["row_scale"].double()
    if kind != "grouped":
        w = _exact_decoded(s["w"], s["w_scale"], K)
        y = (a @ w.t()) * rstd[:, None]
        return got | {"out": y if s["bias"] is None else y + s["bias"].double()}
    y, at = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), s["offsets"].tolist()
    for e in range(case["E"]):
        if at[e] < at[e + 1]:
            rows = slice(at[e], at[e + 1])
            y[rows] = (a[rows] @ _exact_decoded(s["w"][e], s["w_scale"][e], K).t()) * rstd[rows, None]
            if s["bias"] is not None:
                y[rows] += s["bias"][e].double()
    return {"out": y}


def work(case):
    kind, n, K = case["kind"], case["n"], case["K"]
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["types"]]
    coded = (K + 1) // 2 + (K + 31) // 32            # bytes of a row
    if kind == "quantize":
        # the codes and scales are written, the values too
        return {"bytes": n * K * (size + 2) + n * coded, "flops": 4 * n * K}
    real = n * K * size * (3 if case.get("residual") else 1) + K * size   # x, residual, sum; gain
    if kind == "norm":
        return {"bytes": real + n * (coded + 4) + n * K * size, "flops": 8 * n * K}
    N = case["N"]
    if kind == "grouped":
        # each expert's weights once if it has rows: all of them, or as many as there are rows
        E, used = case["E"], case["used"]
        return {"bytes": used * coded + min(E, used) * N * coded + used * N * size + 4 * used + 4 * E
                         + (4 * min(E, used) * N if case["bias"] else 0),
                "flops": 2 * used * K * N}
    bytes_ = N * coded + n * N * size + 4 * n + (4 * N if case["bias"] else 0)
    if kind == "matmul":
        return {"bytes": n * coded + bytes_, "flops": 2 * n * K * N}
    # the codes between the two need not leave the chip
    return {"bytes": real + bytes_ - 4 * n, "flops": 8 * n * K + 2 * n * K * N}
