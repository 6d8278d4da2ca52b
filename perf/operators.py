"""Measured cases of the 8-bit front end: the operators that take real-valued
rows -- hidden states of a language model, features of an encoder -- to what a
binary multi-layer perceptron reads, over the range of their use.

A case is a dict of plain values; ``kind`` names the call:

  norm      bmlp_norm_quantize: root-mean-square norm of n rows of K values, with
            the residual's addition, to 8 bits and a scale per row
  quantize  bmlp_quantize_rows: n rows of K values (the channels of a weight
            matrix, or rows that are normalised already) to 8 bits and a scale
  matmul    bmlp_int8_matmul: n x K times (N x K)^T in 8-bit integers, scaled per
            row and channel
  sign      bmlp_int8_sign: the same product's signs as packed +-1 words
  front     norm, then sign: the whole way from hidden states to a BMLP's input

``types`` is the type of the real-valued input (norm, quantize, front) or of
the output (matmul); ``pad`` elements lie between the rows of the inputs.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6


def listed():
    return [
        # one token's hidden state between two layers: latency counts
        dict(name="norm 1x8192 bf16", kind="norm", n=1, K=8192, types="bf16", residual=True, pad=0),
        # the hidden states of a long prompt
        dict(name="norm 8191x4096 bf16", kind="norm", n=8191, K=4096, types="bf16", residual=True, pad=0),
        # a training set of 784 real-valued features, no residual
        dict(name="norm 60000x784 f32", kind="norm", n=60000, K=784, types="f32", residual=False, pad=0),
        # the channels of a projection, once per model that is loaded
        dict(name="quantize 8192x8192 bf16", kind="quantize", n=8192, K=8192, types="bf16", pad=0),
        # odd rows of a wider buffer
        dict(name="quantize 257x1001 f16", kind="quantize", n=257, K=1001, types="f16", pad=7),
        # one token through a projection: the weights' bytes
        dict(name="matmul 1x8192x8192", kind="matmul", n=1, K=8192, N=8192, types="bf16", bias=False, pad=0),
        # a mini-batch of 100
        dict(name="matmul 100x4096x8192", kind="matmul", n=100, K=4096, N=8192, types="bf16", bias=False, pad=0),
        # 1,000 features, rows that start at odd multiples of 8 bytes
        dict(name="matmul 1000x1000x525 f32", kind="matmul", n=1000, K=1000, N=525, types="f32", bias=True, pad=0),
        # a long prompt through a projection: the tensor cores
        dict(name="matmul 16384x8192x8192", kind="matmul", n=16384, K=8192, N=8192, types="bf16", bias=False, pad=0),
        # a few patterns of 784 features to a 2,048-wide first layer
        dict(name="sign 20x784x2048", kind="sign", n=20, K=784, N=2048, pad=0),
        # the evaluation sweep's 65,536 patterns to an 8,192-wide first layer
        dict(name="sign 65536x4096x8192", kind="sign", n=65536, K=4096, N=8192, pad=0),
        # the whole way for the few requests of one serving step
        dict(name="front 7x4096x8192", kind="front", n=7, K=4096, N=8192, types="bf16", residual=True, pad=0),
    ]


# Multiply-accumulates that a drawn product may cost (the listed sweep: 2.2e12) and
# values that a drawn norm or quantisation may read (the listed ones: 6.7e7).
_MOST_MACS, _MOST_VALUES = 2.0e12, 6.0e7


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return max(lo, w // 64 * 64) if w >= 128 and rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["norm", "norm", "quantize", "matmul", "matmul", "matmul", "sign", "sign", "front"])
    K = _width(rng, 48, 16384)
    case = dict(kind=kind, K=K, pad=rng.choice([0, 0, 0, rng.randint(1, 64)]))
    if kind in ("norm", "quantize"):
        case.update(n=_log(rng, 1, min(65536, _MOST_VALUES // K)), types=rng.choice(["bf16", "f16", "f32"]))
        if kind == "norm":
            case.update(residual=rng.random() < 0.7)
        return case
    N = _width(rng, 32, 16384)
    case.update(N=N, n=_log(rng, 1, min(65536, int(_MOST_MACS / (K * N)))))
    if kind == "matmul":
        case.update(types=rng.choice(["bf16", "bf16", "f16", "f32"]), bias=rng.random() < 0.3)
    elif kind == "front":
        case.update(types=rng.choice(["bf16", "f16", "f32"]), residual=rng.random() < 0.7)
    return case


# -- inputs ---------------------------------------------------------------------

def _rows(n, K, pad, dtype):
    """n x K of a new buffer whose rows are K + pad elements apart."""
    return torch.empty((n, K + pad), dtype=dtype, device="cuda")[:, :K]


def _hidden(n, K, g):
    """Hidden states as a language model has them: normal values, one channel in
    128 of 16 times the others' size, and rows of different sizes."""
    x = torch.randn((n, K), generator=g, device="cuda")
    big = torch.rand((K,), generator=g, device="cuda") < 1 / 128
    size = torch.exp(0.5 * torch.randn((n, 1), generator=g, device="cuda"))
    return x * torch.where(big, 16.0, 1.0) * size


def _codes(x, pad):
    """8-bit codes and scales of the rows of x, in a buffer of padded rows."""
    q = _rows(x.shape[0], x.shape[1], pad, torch.int8)
    most = x.abs().amax(1, keepdim=True)
    q.copy_(torch.round(x * (torch.full_like(most, 127.0) / most)))
    return q, (most / 127.0).squeeze(1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, n, K, pad = case["kind"], case["n"], case["K"], case["pad"]
    s = dict(case=case)
    if kind in ("norm", "quantize", "front"):
        dtype = _TYPES[case["types"]]
        s["x"] = _rows(n, K, pad, dtype)
        if kind == "quantize":
            s["x"].copy_(0.02 * torch.randn((n, K), generator=g, device="cuda"))
        else:
            s["x"].copy_(_hidden(n, K, g))
            s["gain"] = (1 + 0.2 * torch.randn((K,), generator=g, device="cuda")).to(dtype)
        s["res"] = s["sum"] = None
        if case.get("residual"):
            s["res"] = _rows(n, K, pad, dtype)
            s["res"].copy_(_hidden(n, K, g))
            s["sum"] = torch.empty((n, K), dtype=dtype, device="cuda")
        s["q"] = torch.empty((n, K), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty((n,), dtype=torch.float32, device="cuda")
    if kind in ("matmul", "sign", "front"):
        N = case["N"]
        s["w"], s["w_scale"] = _codes(0.02 * torch.randn((N, K), generator=g, device="cuda"), pad)
        if kind != "front":
            s["a"], s["a_scale"] = _codes(_hidden(n, K, g), pad)
        if kind == "matmul":
            s["bias"] = torch.randn((N,), generator=g, device="cuda") if case["bias"] else None
            s["out"] = torch.empty((n, N), dtype=_TYPES[case["types"]], device="cuda")
        else:
            # thresholds near the middle of the sums: zero for half of the channels
            t = torch.randint(-2000, 2001, (N,), generator=g, device="cuda", dtype=torch.int32)
            s["threshold"] = torch.where(torch.rand((N,), generator=g, device="cuda") < 0.5, 0, t).to(torch.int32)
            s["words"] = torch.empty((n, (N + 63) // 64), dtype=torch.int64, device="cuda")
            s["bit"] = torch.ones((64,), dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    return s


# -- the plain forms ------------------------------------------------------------

def _plain_codes(u):
    most = u.abs().amax(1, keepdim=True)
    inv = torch.where(most > 0, torch.full_like(most, 127.0) / most, torch.zeros_like(most))
    return torch.round(u * inv).to(torch.int8), most.squeeze(1) / torch.full_like(most.squeeze(1), 127.0)


def _plain_norm(s):
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    rstd = torch.rsqrt((h * h).mean(1) + _EPS)
    q, scale = _plain_codes(h * s["gain"].float())
    return q, scale * rstd, h.to(s["x"].dtype) if s["res"] is not None else None


def _plain_sums(a, w):
    return torch.mm(a.float(), w.float().t())


def _plain_sign(a, s):
    n, N = a.shape[0], s["w"].shape[0]
    bits = _plain_sums(a, s["w"]) >= s["threshold"].float()
    full = torch.zeros((n, 64 * s["words"].shape[1]), dtype=torch.bool, device="cuda")
    full[:, :N] = bits
    return torch.where(full.view(n, -1, 64), s["bit"], 0).sum(2)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "quantize":
        q, scale = _plain_codes(s["x"].float())
        return {"q": q, "scale": scale}
    if kind == "norm":
        q, scale, total = _plain_norm(s)
        return {"q": q, "scale": scale} | ({"sum": total} if total is not None else {})
    if kind == "matmul":
        y = _plain_sums(s["a"], s["w"]) * s["a_scale"][:, None] * s["w_scale"]
        if s["bias"] is not None:
            y = y + s["bias"]
        return {"out": y.to(s["out"].dtype)}
    if kind == "sign":
        return {"words": _plain_sign(s["a"], s)}
    q, scale, total = _plain_norm(s)
    return {"words": _plain_sign(q, s), "scale": scale} | ({"sum": total} if total is not None else {})


# -- the framework's operators ----------------------------------------------------

def _operators(s):
    from paper_2412_00119_gb300 import bmlp as B
    kind = s["case"]["kind"]
    if kind == "quantize":
        B.bmlp_quantize_rows(s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if kind == "matmul":
        B.bmlp_int8_matmul(s["a"], s["w"], s["out"], s["a_scale"], s["w_scale"], s["bias"])
        return {"out": s["out"]}
    if kind == "sign":
        B.bmlp_int8_sign(s["a"], s["w"], s["words"], s["threshold"])
        return {"words": s["words"]}
    B.bmlp_norm_quantize(s["x"], s["gain"], s["q"], s["scale"], res=s["res"], sum_out=s["sum"], eps=_EPS)
    total = {"sum": s["sum"]} if s["sum"] is not None else {}
    if kind == "norm":
        return {"q": s["q"], "scale": s["scale"]} | total
    B.bmlp_int8_sign(s["q"], s["w"], s["words"], s["threshold"])
    return {"words": s["words"], "scale": s["scale"]} | total


def run(s):
    return _operators(s) if own else _plain(s)


# -- the definition in 64 bits ------------------------------------------------------

def exact(case, seed):
    """Codes and packed signs are whole numbers: None in their place."""
    kind = case["kind"]
    if kind == "sign":
        return None
    s = prepare(case, seed)
    if kind == "matmul":
        # y_ij = a_scale_i w_scale_j (sum_k a_ik w_jk) + bias_j, in blocks of rows
        wt = s["w"].double().t()
        y = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
        for i in range(0, case["n"], 4096):
            rows = slice(i, i + 4096)
            y[rows] = (s["a"][rows].double() @ wt) * torch.outer(s["a_scale"][rows].double(), s["w_scale"].double())
        if s["bias"] is not None:
            y += s["bias"].double()
        return {"out": y}
    x = s["x"].double()
    if kind == "quantize":
        return {"q": None, "scale": x.abs().max(dim=1).values / 127}
    if s["res"] is not None:
        x = x + s["res"].double()
    normed = x / torch.sqrt(x.square().sum(1, keepdim=True) / case["K"] + _EPS) * s["gain"].double()
    got = {"scale": normed.abs().max(dim=1).values / 127, "words" if kind == "front" else "q": None}
    return got | ({"sum": x} if s["res"] is not None else {})


def work(case):
    kind, n, K = case["kind"], case["n"], case["K"]
    size = {"f32": 4, "f16": 2, "bf16": 2}.get(case.get("types"), 0)
    N = case.get("N", 0)
    words = 8 * n * ((N + 63) // 64)
    rows = n * K * size * (3 if case.get("residual") else 1) + 4 * n   # x, residual, sum; scales
    if kind == "quantize":
        return {"bytes": rows + n * K, "flops": 4 * n * K}
    norm = {"bytes": rows + K * size + n * K, "flops": 7 * n * K}
    if kind == "norm":
        return norm
    if kind == "matmul":
        return {"bytes": n * K + N * K + n * N * size + 4 * n + 4 * N * (2 if case["bias"] else 1),
                "flops": 2 * n * K * N}
    if kind == "sign":
        return {"bytes": n * K + N * K + words + 4 * N, "flops": 2 * n * K * N}
    # the codes between the two need not leave the chip
    return {"bytes": norm["bytes"] - n * K + N * K + words + 4 * N, "flops": norm["flops"] + 2 * n * K * N}
