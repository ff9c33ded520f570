"""The operators of linear layers in 8-bit integers, as cases that can be timed and compared.

A matrix of bf16 rows is held as 8-bit codes with one fp32 scale a row: the rows of a weight are its output
channels, the rows of the activations are tokens.  Three operators work on that form:

* ``quant``: codes and scales of bf16 rows;
* ``norm``: RMSNorm of rows of the fp32 residual stream, its result as codes and scales;
* ``gemm``: the product of two such matrices, summed in 32-bit integers and scaled back, with one of four
  epilogues: bf16, fp32, added to an fp32 residual, or SwiGLU of a gate and an up weight.

With ``own`` false a case runs in plain torch operations, in 32 bits, rounded once at the end; with ``own``
true it makes the calls of ``paper_2505_05286_amd.hxf``.

Codes are kept in tiles of 16 rows x 64 columns, row tiles outermost, zero padded; element (r, k) of a tile is at
``k // 16 * 256 + r * 16 + k % 16``.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
TINY = 2.0 ** -119     # rows whose largest magnitude is below it are zero
EPILOGUES = ("bf16", "resid", "swiglu", "f32")


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a layer's down projection of the 8B shape, quantised when a model is loaded
        {"name": "quant_weight_down_8b", "op": "quant", "rows": 4096, "k": 14336, "pad": 0, "holes": 0},
        # the attention's output in a decode iteration of 64 sequences, before the output projection
        {"name": "quant_decode_8b", "op": "quant", "rows": 64, "k": 4096, "pad": 0, "holes": 0},
        # SwiGLU's output in a mixed iteration (a 2048-token chunk and 32 decodes) of the 70B shape
        {"name": "quant_mixed_ffn_70b", "op": "quant", "rows": 2080, "k": 28672, "pad": 0, "holes": 0},
        # a lone request's token before the QKV projection: the lowest latency
        {"name": "norm_lone_8b", "op": "norm", "rows": 1, "k": 4096, "src": 1, "gather": False},
        # a mixed iteration's rows of the 32B shape
        {"name": "norm_mixed_32b", "op": "norm", "rows": 2080, "k": 5120, "src": 2080, "gather": False},
        # the rows of a mixed iteration that need logits, some places of the batch empty
        {"name": "norm_logit_rows_70b", "op": "norm", "rows": 37, "k": 8192, "src": 2080, "gather": True},
        # a lone request's QKV projection
        {"name": "gemm_lone_qkv_8b", "op": "gemm", "m": 1, "n": 6144, "k": 4096, "epi": "bf16", "pad": 0},
        # gate and up projections of 64 decoding sequences
        {"name": "gemm_decode_ffn_8b", "op": "gemm", "m": 64, "n": 28672, "k": 4096, "epi": "swiglu", "pad": 0},
        # the down projection of 256 branches that decode together, into the residual stream
        {"name": "gemm_branches_down_70b", "op": "gemm", "m": 256, "n": 8192, "k": 28672, "epi": "resid", "pad": 0},
        # a mixed iteration's down projection
        {"name": "gemm_mixed_down_8b", "op": "gemm", "m": 2080, "n": 4096, "k": 14336, "epi": "resid", "pad": 0},
        # a mixed iteration's gate and up projections: the largest product of the step
        {"name": "gemm_mixed_ffn_70b", "op": "gemm", "m": 2080, "n": 57344, "k": 8192, "epi": "swiglu", "pad": 0},
        # logits of an odd number of rows over a vocabulary of the tiny shape, cut to an odd width
        {"name": "gemm_odd_logits", "op": "gemm", "m": 33, "n": 2045, "k": 260, "epi": "f32", "pad": 3},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant", "norm", "gemm", "gemm"])
    if op == "quant":
        k = 8 * _log_int(rng, 1, 3584)
        return {"op": op, "rows": _log_int(rng, 1, min(20000, 59_000_000 // k)), "k": k,
                "pad": rng.choice([0, 0, 8 * rng.randrange(1, 100)]), "holes": rng.choice([0, 0, 1, 2])}
    if op == "norm":
        k = 4 * _log_int(rng, 2, 4096)
        src = _log_int(rng, 1, min(8192, 30_000_000 // k))
        gather = rng.random() < 0.4
        return {"op": op, "rows": _log_int(rng, 1, src) if gather else src, "k": k, "src": src, "gather": gather}
    epi = rng.choice(EPILOGUES)
    m, k = _log_int(rng, 1, 3000), 4 * _log_int(rng, 4, 7168)
    most = max(16, min(128256, 500_000_000 // k, 900_000_000_000 // (m * k), 400_000_000 // m))
    n = _log_int(rng, 16, most)
    n += n % 2 if epi == "swiglu" else 0
    return {"op": op, "m": m, "n": n, "k": k, "epi": epi, "pad": rng.choice([0, 0, rng.randrange(1, 70)])}


# ------------------------------------------------------------------ inputs
def _up(n, to):
    return -(-n // to) * to


def _tile(codes):
    """Row-major int8 codes [rows, k] as tiles."""
    r, k = codes.shape
    x = torch.zeros(_up(r, 16), _up(k, 64), dtype=torch.int8, device=DEV)
    x[:r, :k] = codes
    return x.view(-1, 16, x.shape[1] // 64, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1)


def _untile(tiles, rows, k):
    x = tiles.view(-1, _up(k, 64) // 64, 4, 16, 16).permute(0, 3, 1, 2, 4)
    return x.reshape(_up(rows, 16), -1)[:rows, :k]


def _random_codes(g, rows, k):
    """Tiles and scales of a matrix with normal values: the largest of a row has the code 127 or -127."""
    x = torch.randn(rows, k, generator=g, device=DEV)
    m = x.abs().amax(1)
    codes = (x * (127 / m)[:, None]).round().to(torch.int8)
    return _tile(codes), m / 127


def _activations(g, rows, k):
    """Normal values, a few of the channels much larger than the others, rows of different sizes."""
    x = torch.randn(rows, k, generator=g, device=DEV)
    x *= 1 + 12 * (torch.rand(k, generator=g, device=DEV) < 0.004)
    return x * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device=DEV))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case)
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], sa = _random_codes(g, m, k)
        s["sa"] = sa * torch.exp(0.5 * torch.randn(m, generator=g, device=DEV))
        cols = n // 2 if case["epi"] == "swiglu" else n
        s["b"], sb = _random_codes(g, cols, k)
        s["sb"] = sb / math.sqrt(k)
        s["cols"], s["ldc"] = cols, cols + case["pad"]
        if case["epi"] == "swiglu":
            s["b2"], sb = _random_codes(g, cols, k)
            s["sb2"] = sb / math.sqrt(k)
        kind = torch.bfloat16 if case["epi"] in ("bf16", "swiglu") else torch.float32
        if case["epi"] == "resid":
            s["c"] = torch.randn(m, s["ldc"], generator=g, device=DEV)
        else:
            s["c"] = torch.zeros(m, s["ldc"], dtype=kind, device=DEV)
        return s
    rows, k = case["rows"], case["k"]
    s["codes"] = torch.zeros(_up(rows, 16) * _up(k, 64), dtype=torch.int8, device=DEV)
    s["scale"] = torch.zeros(rows, device=DEV)
    if case["op"] == "quant":
        x = torch.zeros(rows, k + case["pad"], dtype=torch.bfloat16, device=DEV)
        x[:, :k] = _activations(g, rows, k).to(torch.bfloat16)
        if case["holes"]:                      # empty places of a batch
            x[torch.randperm(rows, generator=g, device=DEV)[:case["holes"]]] = 0
        s["x"] = x
        return s
    s["x"] = 3 * _activations(g, case["src"], k)
    s["gain"] = (1 + torch.rand(k, generator=g, device=DEV) - 0.5).to(torch.bfloat16)
    s["at"] = None
    if case["gather"]:
        at = torch.randint(0, case["src"], (rows,), generator=g, device=DEV, dtype=torch.int32)
        at[torch.rand(rows, generator=g, device=DEV) < 0.1] = -1      # empty places
        s["at"] = at
    return s


# ------------------------------------------------------------------ the framework's calls
def _own_run(s):
    from paper_2505_05286_amd import hxf
    st = torch.cuda.current_stream().cuda_stream
    if s["op"] == "quant":
        hxf.op_quant_i8(s["x"].data_ptr(), s["x"].stride(0), s["rows"], s["k"], s["codes"].data_ptr(),
                        s["scale"].data_ptr(), stream=st)
        return {"codes": s["codes"], "scale": s["scale"]}
    if s["op"] == "norm":
        hxf.op_rmsnorm_i8(s["x"].data_ptr(), s["at"].data_ptr() if s["gather"] else 0, s["src"],
                          s["gain"].data_ptr(), s["codes"].data_ptr(), s["scale"].data_ptr(), s["rows"], s["k"], EPS,
                          stream=st)
        return {"codes": s["codes"], "scale": s["scale"]}
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, hxf.op_gemm_i8_workspace_bytes(s["m"], s["n"], s["k"])), dtype=torch.uint8,
                              device=DEV)
    gated = s["epi"] == "swiglu"
    hxf.op_gemm_i8(s["a"].data_ptr(), s["sa"].data_ptr(), s["b"].data_ptr(), s["sb"].data_ptr(),
                   s["b2"].data_ptr() if gated else 0, s["sb2"].data_ptr() if gated else 0, s["c"].data_ptr(),
                   s["ldc"], s["m"], s["n"], s["k"], EPILOGUE_CODE[s["epi"]], s["ws"].data_ptr(), s["ws"].numel(),
                   stream=st)
    return s["c"]


EPILOGUE_CODE = {"bf16": 0, "resid": 1, "swiglu": 2, "f32": 3}


# ------------------------------------------------------------------ the plain forms
def _plain_codes(t):
    """Codes [rows, k] and m / 127 of rows t; m: the largest magnitude of a row."""
    m = t.abs().amax(1)
    ok = torch.isfinite(m) & (m >= TINY)
    most = torch.full_like(m, 127)
    codes = torch.where(ok[:, None], torch.round(t * torch.where(ok, most / m, 0)[:, None]), 0)
    return codes.to(torch.int8), torch.where(torch.isfinite(m), torch.where(ok, m / most, 0), math.nan)


def _plain_quant(s):
    codes, scale = _plain_codes(s["x"][:, :s["k"]].float())
    return {"codes": _tile(codes), "scale": scale}


def _plain_norm(s):
    x = s["x"]
    if s["gather"]:
        x = torch.where((s["at"] >= 0)[:, None], x[s["at"].long().clamp(min=0)], 0)
    codes, scale = _plain_codes(x * s["gain"].float())
    return {"codes": _tile(codes), "scale": scale * torch.rsqrt((x * x).mean(1) + EPS)}


def _plain_product(s, b, sb):
    a = _untile(s["a"], s["m"], s["k"]).float()
    w = _untile(b, s["cols"], s["k"]).float()
    return (a @ w.T) * s["sa"][:, None] * sb


def _plain_gemm(s):
    y = _plain_product(s, s["b"], s["sb"])
    if s["epi"] == "swiglu":
        y = y / (1 + torch.exp(-y)) * _plain_product(s, s["b2"], s["sb2"])
    c = s["c"]
    c[:, :s["cols"]] = c[:, :s["cols"]] + y if s["epi"] == "resid" else y.to(c.dtype)
    return c


def run(state):
    if own:
        return _own_run(state)
    return {"quant": _plain_quant, "norm": _plain_norm, "gemm": _plain_gemm}[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        out = {"bf16": 2 * m * n, "resid": 8 * m * n, "swiglu": m * n, "f32": 4 * m * n}[case["epi"]]
        return {"bytes": float(m * k + n * k + 4 * (m + n) + out), "flops": 2.0 * m * n * k}
    rows, k = case["rows"], case["k"]
    if case["op"] == "quant":
        return {"bytes": float(rows * (3 * k + 4)), "flops": float(3 * rows * k)}
    read = min(rows, case["src"])
    return {"bytes": float(read * 4 * k + 2 * k + rows * (k + 4) + (4 * rows if case["gather"] else 0)),
            "flops": float(6 * rows * k)}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_matrix(tiles, rows, k):
    """The codes as a matrix, each looked up at its place."""
    r = torch.arange(rows, device=DEV)[:, None]
    c = torch.arange(k, device=DEV)
    at = (r // 16 * ((k + 63) // 64) + c // 64) * 1024 + c % 64 // 16 * 256 + r % 16 * 16 + c % 16
    return tiles[at].double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":      # the codes are whole numbers
        return {"codes": None, "scale": s["x"].double().abs().amax(1) / 127}
    if case["op"] == "norm":
        x = s["x"].double()
        if case["gather"]:
            x = torch.cat([x, torch.zeros_like(x[:1])])[s["at"].long()]     # -1: the row of zeros
        root = torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / case["k"] + EPS)
        return {"codes": None, "scale": (x * s["gain"].double()).abs().amax(1) / root / 127}
    a = _exact_matrix(s["a"], case["m"], case["k"]) * s["sa"].double()[:, None]
    cols = s["cols"]
    out = s["c"].double()
    for j in range(0, cols, 8192):
        e = min(cols, j + 8192)
        rows = torch.arange(j, e, device=DEV)
        take = lambda b: _exact_matrix(b[j * _up(case["k"], 64):], e - j, case["k"])   # noqa: E731
        y = a @ (take(s["b"]) * s["sb"].double()[rows, None]).T
        if case["epi"] == "swiglu":
            y = y * torch.sigmoid(y) * (a @ (take(s["b2"]) * s["sb2"].double()[rows, None]).T)
        out[:, j:e] = out[:, j:e] + y if case["epi"] == "resid" else y
    return out
