"""Linear layers in 8-bit integers on the GPU: codes to the bit, products against whole numbers and 64 bits."""
import numpy as np
import pytest

import synth
from paper_2505_05286_amd import hxf

from . import i8_util as U
from ._lib import ensure_built
from .gpu_util import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
GUARD = 64
U32, UB16 = 2.0 ** -24, 2.0 ** -8     # half a step of fp32 and of bf16, relative


@pytest.fixture(autouse=True)
def _built():
    ensure_built()


def _dev(a):
    return torch().from_numpy(np.ascontiguousarray(a)).to(DEV)


def _bf16(x):
    """float32 values rounded to bf16: (bits, the values)."""
    b = synth.f32_to_bf16_bits(np.asarray(x, np.float32)).reshape(np.shape(x))
    return b, synth.bf16_bits_to_f32(b).reshape(np.shape(x))


class Codes:
    """A codes buffer and its scales, filled with 0x55 and followed by guards."""

    def __init__(self, rows, k):
        t = torch()
        self.n, self.rows = hxf.i8_codes_bytes(rows, k), rows
        assert self.n == U.up(rows, 16) * U.up(k, 64)
        self.codes = t.full((self.n + GUARD,), 0x55, dtype=t.int8, device=DEV)
        self.scale = t.full((rows + GUARD,), 7.0, device=DEV)

    def ptrs(self):
        return self.codes.data_ptr(), self.scale.data_ptr()

    def get(self):
        c, s = self.codes.cpu().numpy(), self.scale.cpu().numpy()
        assert (c[self.n:] == 0x55).all() and (s[self.rows:] == 7.0).all(), "written behind the end"
        return c[:self.n], s[:self.rows]


def _rows(rng, R, K):
    """Rows of many sizes, with rows that are zero, tiny, of one value, half of their largest, and not finite."""
    x = (rng.standard_normal((R, K)) * np.exp(rng.standard_normal((R, 1)) * 3)).astype(np.float32)
    x[:, ::max(1, K // 5)] *= 20
    kinds = rng.integers(0, 12, R) if R > 4 else np.arange(R) + 8
    for r, kind in enumerate(kinds):
        if kind == 0:
            x[r] = 0
        elif kind == 1:
            x[r] *= 2.0 ** -121 / np.abs(x[r]).max()
        elif kind == 2:
            x[r] = x[r, 0]
        elif kind == 3:      # ties
            x[r] = np.where(rng.random(K) < 0.5, 0.5, -1.0) * x[r, 0]
        elif kind == 4:
            x[r, rng.integers(K)] = np.nan
        elif kind == 5:
            x[r, rng.integers(K)] = -np.inf
        elif kind == 6:
            x[r] = np.where(np.abs(x[r]) > 0, x[r] / np.abs(x[r]).max() * 3e38, 0)
        elif kind == 7:
            x[r] *= 2.0 ** -117 / np.abs(x[r]).max()
    return x


QUANT = [(1, 8, 0), (1, 64, 0), (16, 64, 8), (17, 72, 0), (5, 4096, 0), (33, 1000, 24), (64, 4096, 64), (3, 28672, 0),
         (130, 5120, 8), (2, 131064, 0), (300, 264, 0), (257, 2048, 0), (1030, 64, 0), (40, 14336, 8), (600, 8200, 0),
         (18, 33000, 0)]


@pytest.mark.parametrize("R,K,pad", QUANT)
def test_quant(R, K, pad):
    rng = np.random.default_rng(R * 131 + K)
    bits, x = _bf16(_rows(rng, R, K))
    wide = rng.integers(0, 1 << 16, (R, K + pad)).astype(np.uint16)
    wide[:, :K] = bits
    out = Codes(R, K)
    src = _dev(wide.view(np.int16))
    hxf.op_quant_i8(src.data_ptr(), K + pad, R, K, *out.ptrs())
    codes, scale = out.get()
    want, unit = U.codes_of(x)
    assert np.array_equal(codes, U.tile(want))
    assert np.array_equal(scale, unit, equal_nan=True)
    assert np.array_equal(src.cpu().numpy(), wide.view(np.int16))
    # and against 64 bits: half a step, and two roundings of a value up to 127
    ok = unit > 0
    t = x[ok].astype(np.float64)
    m = np.abs(t).max(1, keepdims=True) if len(t) else t
    assert (np.abs(want[ok] - t * 127 / m) <= 0.5 + 127 * 2.1 * U32).all()


NORM = [(1, 4, 1, False), (1, 4096, 1, False), (16, 256, 16, False), (37, 8192, 300, True), (64, 4096, 64, False),
        (5, 68, 3, True), (300, 5120, 300, False), (1000, 260, 40, True), (2, 131068, 3, True), (600, 1024, 600, False),
        (270, 14336, 270, False), (520, 8192, 520, False), (70, 20000, 70, False)]


@pytest.mark.parametrize("n,d,src,gather", NORM)
def test_norm(n, d, src, gather):
    rng = np.random.default_rng(n * 17 + d)
    x = _rows(rng, src, d)
    x = np.where(np.abs(x) > 1e18, np.sign(x) * np.float32(1e15), x).astype(np.float32)   # squares within fp32
    gb, g = _bf16(1 + rng.uniform(-0.5, 0.5, d))
    rows = None
    if gather:
        rows = rng.integers(0, src, n).astype(np.int32)
        rows[rng.random(n) < 0.2] = -1
        rows[n // 2] = src
        rows[0], rows[-1] = (-2 ** 31, 2 ** 31 - 1) if n > 2 else (0, 2 ** 31 - 1)
    out = Codes(n, d)
    xd, gd, rd = _dev(x), _dev(gb.view(np.int16)), _dev(rows) if gather else None
    eps = 1e-5
    hxf.op_rmsnorm_i8(xd.data_ptr(), rd.data_ptr() if gather else 0, src, gd.data_ptr(), *out.ptrs(), n, d, eps)
    codes, scale = out.get()
    y, r = U.norm_rows(x, rows, g, np.float32(eps))
    want, unit = U.codes_of(y)
    assert np.array_equal(codes, U.tile(want))
    assert np.array_equal(np.isnan(scale), np.isnan(unit))
    ok = np.isfinite(unit)
    # the sum of squares in fp32 over at most d / 64 + 16 terms in a chain, halved by the root; the mean, eps, the root
    # (two half steps) and three products
    tol = ((d / 64 + 16) / 2 + 8) * U32
    assert (np.abs(scale[ok] - unit[ok] * r[ok]) <= tol * np.abs(unit[ok] * r[ok]) + 2.0 ** -149).all()
    assert np.array_equal(xd.cpu().numpy(), x, equal_nan=True)


def test_norm_without_rows_takes_the_first_of_more():
    rng = np.random.default_rng(3)
    x, g = rng.standard_normal((9, 128)).astype(np.float32), np.ones(128, np.float32)
    out = Codes(4, 128)
    xd, gd = _dev(x), _dev(_bf16(g)[0].view(np.int16))
    hxf.op_rmsnorm_i8(xd.data_ptr(), 0, 9, gd.data_ptr(), *out.ptrs(), 4, 128, 1e-5)
    assert np.array_equal(out.get()[0], U.tile(U.codes_of(x[:4])[0]))


def test_norm_rows_that_are_not_finite_or_beyond_fp32():
    """Infinities, products with the gain that pass fp32, and squares that do (the scale is then 0)."""
    x = np.ones((5, 192), np.float32)
    x[0, 7], x[1, 3], x[2, 100], x[3, 5] = np.inf, -np.inf, 3e38, 1e30
    gb, g = _bf16(np.where(np.arange(192) == 100, 4.0, 1.0))
    out = Codes(5, 192)
    xd, gd = _dev(x), _dev(gb.view(np.int16))
    hxf.op_rmsnorm_i8(xd.data_ptr(), 0, 5, gd.data_ptr(), *out.ptrs(), 5, 192, 1e-5)
    codes, scale = out.get()
    y, _ = U.norm_rows(x, None, g, 1e-5)
    want, _ = U.codes_of(y)
    assert np.array_equal(codes, U.tile(want))
    assert np.isnan(scale[:3]).all() and scale[3] == 0 and scale[4] > 0
    assert want[3, 5] == 127 and not want[:3].any()


EPI = {"bf16": hxf.EPI_BF16, "resid": hxf.EPI_RESID, "swiglu": hxf.EPI_SWIGLU, "f32": hxf.EPI_F32}


def _codes(rng, rows, k):
    return rng.integers(-127, 128, (rows, k)).astype(np.int8)


class Product:
    """Operands of one product on the GPU, with what it should give."""

    def __init__(self, rng, M, N, K, epi, pad=0, shift=0):
        t = torch()
        self.M, self.N, self.K, self.epi = M, N, K, epi
        self.cols = cols = N // 2 if epi == "swiglu" else N
        self.ldc, self.shift = cols + pad, shift
        self.a, self.b = _codes(rng, M, K), _codes(rng, cols, K)
        size = 1 / (5000 * np.sqrt(K))
        self.sa = np.exp(rng.standard_normal(M)).astype(np.float32)
        self.sb = (size * np.exp(rng.standard_normal(cols))).astype(np.float32)
        self.b2, self.sb2 = _codes(rng, cols, K), (size * np.exp(rng.standard_normal(cols))).astype(np.float32)
        wide = epi in ("resid", "f32")
        self.c0 = rng.standard_normal((M, self.ldc)).astype(np.float32)
        if not wide:
            self.c0 = _bf16(self.c0)[1]
        self.dev = [_dev(v) for v in (U.tile(self.a), self.sa, U.tile(self.b), self.sb, U.tile(self.b2), self.sb2)]
        whole = t.full((M * self.ldc + shift + GUARD,), 3.0, device=DEV, dtype=t.float32 if wide else t.bfloat16)
        whole[shift:shift + M * self.ldc] = _dev(self.c0).view(-1).to(whole.dtype)
        self.c = whole
        self.ws = self.workspace()

    def workspace(self):
        t = torch()
        n = hxf.op_gemm_i8_workspace_bytes(self.M, self.N, self.K)
        return t.full((n + GUARD,), 0x5A, dtype=t.uint8, device=DEV)

    def call(self, stream=0):
        a, sa, b, sb, b2, sb2 = (v.data_ptr() for v in self.dev)
        sw = self.epi == "swiglu"
        hxf.op_gemm_i8(a, sa, b, sb, b2 if sw else 0, sb2 if sw else 0, self.c[self.shift:].data_ptr(), self.ldc,
                       self.M, self.N, self.K, EPI[self.epi], self.ws.data_ptr(), self.ws.numel() - GUARD,
                       stream=stream)

    def check(self, rows=None):
        c = self.c.float().cpu().numpy()
        n = self.M * self.ldc
        assert (c[:self.shift] == 3.0).all() and (c[self.shift + n:] == 3.0).all(), "written outside"
        assert (self.ws[-GUARD:].cpu().numpy() == 0x5A).all(), "written behind the workspace"
        c = c[self.shift:self.shift + n].reshape(self.M, self.ldc)
        assert np.array_equal(c[:, self.cols:], self.c0[:, self.cols:]), "written between rows"
        got = c[:, :self.cols].astype(np.float64)
        y = U.product(self.a, self.sa, self.b, self.sb)
        # float(acc) and two products: three half steps (and their products with each other)
        rel = 3.001 * U32
        if self.epi == "f32":
            want, tol = y, rel * np.abs(y)
        elif self.epi == "bf16":
            want, tol = y, (UB16 + 2 * rel) * np.abs(y)
        elif self.epi == "resid":
            want = y + self.c0[:, :self.cols]
            tol = rel * np.abs(y) + 1.001 * U32 * (np.abs(want) + rel * np.abs(y))
        else:
            # silu(z (1 + e)) is off by at most (1 + |z|) e of itself; e^-z from an exponent rounded in fp32, by |z| steps
            # and a few; then the sum, the quotient, the product and its rounding to bf16
            up = U.product(self.a, self.sa, self.b2, self.sb2)
            want = U.silu(y) * up
            tol = (UB16 + (6 * np.abs(y) + 16) * 2 * U32) * np.abs(want) + 1e-30
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


# one row to many, one column to many, K below, at and past a tile, widths that no tile divides
SIZES = [(1, 1, 1), (1, 64, 64), (2, 16, 4), (3, 17, 70), (16, 128, 256), (17, 130, 260), (33, 2046, 260), (31, 512, 1000),
         (64, 4096, 2048), (65, 688, 512), (100, 300, 4100), (128, 1024, 1088), (129, 512, 704), (200, 1376, 256),
         (257, 770, 640), (513, 514, 1344), (700, 260, 132), (1000, 1030, 192), (2080, 256, 320), (5, 20000, 128),
         (1, 6144, 4096), (48, 96, 20000), (300, 2048, 4096), (90, 1024, 8192), (270, 128, 14336)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("epi", list(EPI))
def test_gemm(M, N, K, epi):
    if epi == "swiglu":
        N += N % 2
    p = Product(np.random.default_rng(M + 7 * N + 31 * K), M, N, K, epi, pad=(M + N) % 3)
    p.call()
    p.check()


@pytest.mark.parametrize("epi", list(EPI))
@pytest.mark.parametrize("M,N,K,pad,shift", [(19, 64, 128, 0, 1), (40, 96, 64, 5, 3), (130, 256, 64, 2, 2), (7, 33, 64, 4, 0)])
def test_gemm_outputs_of_any_alignment(M, N, K, pad, shift, epi):
    p = Product(np.random.default_rng(M), M, N + (N % 2 if epi == "swiglu" else 0), K, epi, pad, shift)
    p.call()
    p.check()


@pytest.mark.parametrize("M,K", [(1, 131071), (40, 131071), (200, 131071)])
@pytest.mark.parametrize("sign", [1, -1])
def test_gemm_sums_up_to_the_end_of_32_bits(M, K, sign):
    """127^2 K = 2114044159; and codes of -128, which the quantisers never make, still fit: 2^14 K < 2^31."""
    rng = np.random.default_rng(5)
    for lo in (127, -128):
        p = Product(rng, M, 48, K, "f32")
        p.a[:], p.b[:] = lo, lo
        if sign < 0:
            p.b[:] = 127
            p.a[:] = -128 if lo < 0 else -127
        p.dev[0], p.dev[2] = _dev(U.tile(p.a)), _dev(U.tile(p.b))
        p.call()
        p.check()


@pytest.mark.parametrize("M", [20, 150])
@pytest.mark.parametrize("epi", list(EPI))
def test_gemm_scales_that_are_nan_or_zero_stay_in_their_rows_and_columns(M, epi):
    p = Product(np.random.default_rng(M), M, 96, 192, epi)
    cols = p.cols
    p.sa[3], p.sb[5], p.sa[7] = np.nan, np.nan, 0.0
    p.dev[1], p.dev[3] = _dev(p.sa), _dev(p.sb)
    p.call()
    got = p.c.float().cpu().numpy()[:M * p.ldc].reshape(M, p.ldc)
    nan = np.zeros((M, cols), bool)
    nan[3], nan[:, 5] = True, True
    assert np.array_equal(np.isnan(got), nan)
    assert np.array_equal(got[7][~nan[7]], (p.c0[7] if epi == "resid" else np.zeros(cols))[~nan[7]])


def test_gemm_swiglu_at_large_gates():
    """silu goes to z and to -0 without NaN."""
    p = Product(np.random.default_rng(1), 16, 64, 64, "swiglu")
    p.sa[:] = 1.0
    p.sb[:] = np.linspace(0.0, 0.1, 32, dtype=np.float32)
    p.sb2[:] = 1e-4
    p.dev[1], p.dev[3], p.dev[5] = _dev(p.sa), _dev(p.sb), _dev(p.sb2)
    p.call()
    p.check()


def _tile_dev(x):
    """Row-major int8 codes on the GPU as padded tiles."""
    t = torch()
    r, k = x.shape
    p = t.zeros(U.up(r, 16), U.up(k, 64), dtype=t.int8, device=DEV)
    p[:r, :k] = x
    return p.view(-1, 16, p.shape[1] // 64, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1)


@pytest.mark.parametrize("M,N,K", U.PLANS)
def test_gemm_in_every_plan(M, N, K):
    """Each instance of the kernels, all epilogues; the whole numbers by products in 64 bits (exact below 2^53)."""
    t = torch()
    g = t.Generator(device=DEV)
    g.manual_seed(M * 7 + N)
    rand = lambda n: t.randint(-127, 128, (n, K), generator=g, device=DEV, dtype=t.int8)   # noqa: E731
    a, b, b2 = rand(M), rand(N), rand(N)
    sa = t.rand(M, generator=g, device=DEV) + 0.5
    sb = (t.rand(N, generator=g, device=DEV) + 0.5) / (5000 * K ** 0.5)
    dev = [_tile_dev(v) for v in (a, b, b2)]
    y, up = (((a.double() @ v.double().T) * sa.double()[:, None]) * sb.double() for v in (b, b2))
    rel = 3.001 * U32
    for epi in EPI:
        cols = 2 * N if epi == "swiglu" else N
        print(epi, M, cols, K, hxf.op_gemm_i8_plan(M, cols, K, EPI[epi]), flush=True)
        wide = epi in ("resid", "f32")
        c = t.randn(M, N + 1, generator=g, device=DEV).to(t.float32 if wide else t.bfloat16)
        c0 = c.double()
        n = hxf.op_gemm_i8_workspace_bytes(M, cols, K)
        ws = t.full((n + GUARD,), 0x5A, dtype=t.uint8, device=DEV)
        hxf.op_gemm_i8(dev[0].data_ptr(), sa.data_ptr(), dev[1].data_ptr(), sb.data_ptr(), dev[2].data_ptr(),
                       sb.data_ptr(), c.data_ptr(), N + 1, M, cols, K, EPI[epi], ws.data_ptr(), n)
        t.cuda.synchronize()
        assert bool((ws[n:] == 0x5A).all()) and t.equal(c[:, N].double(), c0[:, N])
        got, old = c[:, :N].double(), c0[:, :N]
        if epi == "swiglu":
            want = y * t.sigmoid(y) * up
            tol = (UB16 + (6 * y.abs() + 16) * 2 * U32) * want.abs() + 1e-30
        elif epi == "resid":
            want = y + old
            tol = rel * y.abs() + 1.001 * U32 * (want.abs() + rel * y.abs())
        else:
            want, tol = y, (rel + (0 if wide else UB16 + rel)) * y.abs()
        bad = ~((got - want).abs() <= tol)
        assert not bool(bad.any()), (epi, int(bad.sum()), bad.nonzero()[:4].tolist())


def test_gemm_outputs_and_weights_beyond_32_bits_of_offset():
    """4.6 GB of outputs, then 4.5 GB of codes; rows and columns at the ends and around 2^31 and 2^32 bytes."""
    t = torch()
    g = t.Generator(device=DEV)
    g.manual_seed(3)
    for M, N, K, epi in ((70001, 32770, 64, "bf16"), (3, 262147, 17000, "f32")):
        a = t.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=t.int8)
        b = t.randint(-127, 128, (N, K), generator=g, device=DEV, dtype=t.int8)
        ta, tb = _tile_dev(a), _tile_dev(b)
        sa, sb = t.ones(M, device=DEV), t.ones(N, device=DEV)
        c = t.zeros(M, N, device=DEV, dtype=t.bfloat16 if epi == "bf16" else t.float32)
        ws = t.empty(hxf.op_gemm_i8_workspace_bytes(M, N, K) + 16, dtype=t.uint8, device=DEV)
        print(M, N, K, hxf.op_gemm_i8_plan(M, N, K, EPI[epi]), flush=True)
        hxf.op_gemm_i8(ta.data_ptr(), sa.data_ptr(), tb.data_ptr(), sb.data_ptr(), 0, 0, c.data_ptr(), N, M, N, K,
                       EPI[epi], ws.data_ptr(), ws.numel())
        t.cuda.synchronize()
        rows = t.tensor(sorted({0, M // 2, M - 1, min(M - 1, 2 ** 30 // N + 1), min(M - 1, 2 ** 31 // N + 1)}), device=DEV)
        for lo in (0, N // 2, N - 40, min(N - 40, 2 ** 31 // 17024), min(N - 40, 2 ** 32 // 17024)):
            want = a[rows].double() @ b[lo:lo + 40].double().T
            off = (c[rows][:, lo:lo + 40].double() - want).abs()
            assert bool((off <= (UB16 if epi == "bf16" else U32) * want.abs()).all())
        del a, b, ta, tb, c


def test_quant_beyond_32_bits_of_offset():
    t = torch()
    R, K = 140001, 16392
    x = t.randn(R, 8, device=DEV).repeat(1, K // 8).to(t.bfloat16)
    codes = t.empty(hxf.i8_codes_bytes(R, K), dtype=t.int8, device=DEV)
    scale = t.empty(R, device=DEV)
    hxf.op_quant_i8(x.data_ptr(), K, R, K, codes.data_ptr(), scale.data_ptr())
    t.cuda.synchronize()
    kt = U.up(K, 64) // 64
    for r in (0, 65537, 2 ** 31 // (2 * K) + 1, 2 ** 32 // (2 * K) + 1, 2 ** 31 // (kt * 64) + 3, R - 1):
        want, unit = U.codes_of(x[r:r + 1].float().cpu().numpy())
        tile = codes[(r // 16) * kt * 1024:(r // 16 + 1) * kt * 1024].view(kt * 4, 16, 16)[:, r % 16].reshape(-1)
        assert np.array_equal(tile.cpu().numpy()[:K], want[0]) and not bool(tile[K:].any())
        assert float(scale[r]) == float(unit[0])


def test_calls_repeat_to_the_bit():
    """Sums of whole numbers do not depend on an order."""
    t = torch()
    for M, N, K in ((33, 1024, 8192), (300, 512, 4096)):
        p = Product(np.random.default_rng(K), M, N, K, "bf16")
        p.call()
        first = p.c.clone()
        for _ in range(5):
            p.c.zero_()
            p.call()
            t.cuda.synchronize()
            assert t.equal(p.c[:M * N], first[:M * N])


class Layer:
    """The linear half of a decoder block in 8 bits: norm, gate and up, codes of their product, down into the residual."""

    def __init__(self, rng, T, d, F):
        t = torch()
        self.T, self.d, self.F = T, d, F
        self.wb, self.wv = zip(*[_bf16(rng.standard_normal(s) * 0.5 / np.sqrt(s[1])) for s in ((F, d), (F, d), (d, F))])
        self.w = []
        for bits in self.wb:
            out = Codes(*bits.shape)
            src = _dev(bits.view(np.int16))
            hxf.op_quant_i8(src.data_ptr(), bits.shape[1], *bits.shape, *out.ptrs())
            t.cuda.synchronize()
            self.w.append(out)
        gb, self.g = _bf16(1 + rng.uniform(-0.5, 0.5, d))
        self.gd = _dev(gb.view(np.int16))
        self.x = t.zeros(T, d, device=DEV)
        self.h = t.zeros(T, F, device=DEV, dtype=t.bfloat16)
        self.cx, self.ch = Codes(T, d), Codes(T, F)
        n = max(hxf.op_gemm_i8_workspace_bytes(T, 2 * F, d), hxf.op_gemm_i8_workspace_bytes(T, d, F))
        self.ws = t.empty(max(16, n), dtype=t.uint8, device=DEV)

    def run(self):
        st = torch().cuda.current_stream().cuda_stream
        T, d, F = self.T, self.d, self.F
        g, u, down = (w.ptrs() for w in self.w)
        hxf.op_rmsnorm_i8(self.x.data_ptr(), 0, T, self.gd.data_ptr(), *self.cx.ptrs(), T, d, 1e-5, stream=st)
        hxf.op_gemm_i8(*self.cx.ptrs(), *g, *u, self.h.data_ptr(), F, T, 2 * F, d, hxf.EPI_SWIGLU, self.ws.data_ptr(),
                       self.ws.numel(), stream=st)
        hxf.op_quant_i8(self.h.data_ptr(), F, T, F, *self.ch.ptrs(), stream=st)
        hxf.op_gemm_i8(*self.ch.ptrs(), *down, 0, 0, self.x.data_ptr(), d, T, d, F, hxf.EPI_RESID, self.ws.data_ptr(),
                       self.ws.numel(), stream=st)

    def want(self, x):
        """The block in 64 bits on the unrounded weights."""
        x = x.astype(np.float64)
        y = x / np.sqrt((x * x).mean(1, keepdims=True) + 1e-5) * self.g
        g, u, down = (v.astype(np.float64) for v in self.wv)
        return (U.silu(y @ g.T) * (y @ u.T)) @ down.T


@pytest.mark.parametrize("T,d,F", [(1, 256, 688), (13, 256, 688), (64, 1024, 2752), (260, 512, 1376)])
def test_a_block_of_them(T, d, F):
    """Together: what the block adds to the residual against 64 bits.  A code is off by at most half a step of its row's
    largest / 127; for normal rows (largest about 3.5 deviations) that is 0.8% of a deviation rms, in each of both
    operands of three products one after the other: below sqrt(6) * 0.8% + bf16's 0.2%, 3% allowed."""
    rng = np.random.default_rng(T + d)
    layer = Layer(rng, T, d, F)
    x = rng.standard_normal((T, d)).astype(np.float32)
    layer.x.copy_(_dev(x))
    layer.run()
    got = layer.x.cpu().numpy() - x
    want = layer.want(x)
    assert np.linalg.norm(got - want) <= 0.03 * np.linalg.norm(want)


def test_a_captured_block_replays_on_new_inputs():
    """Two graphs with a workspace each, replayed in turn, eager calls and waits between them."""
    t = torch()
    rng = np.random.default_rng(8)
    layers = [Layer(rng, 37, 512, 1376), Layer(rng, 300, 256, 688)]
    graphs = []
    for layer in layers:
        layer.run()
        t.cuda.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            layer.run()
        graphs.append(graph)
    for k in range(4):
        wants = []
        for layer, graph in zip(layers, graphs):
            x = _dev(rng.standard_normal((layer.T, layer.d)).astype(np.float32))
            layer.x.copy_(x)
            layer.run()
            t.cuda.synchronize()
            wants.append(layer.x.clone())
            layer.x.copy_(x)
            if k % 2:
                t.cuda.synchronize()
        for layer, graph in zip(layers, graphs):
            graph.replay()
        t.cuda.synchronize()
        for layer, want in zip(layers, wants):
            assert t.equal(layer.x, want)


def test_a_block_on_a_stream_of_its_own():
    """The calls go to the stream they are given: a block on a side stream gives what one on the default stream does."""
    t = torch()
    rng = np.random.default_rng(12)
    layer = Layer(rng, 50, 512, 1376)
    x = _dev(rng.standard_normal((50, 512)).astype(np.float32))
    layer.x.copy_(x)
    layer.run()
    want = layer.x.clone()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        for _ in range(3):
            layer.x.copy_(x)
            layer.run()
    t.cuda.current_stream().wait_stream(side)
    assert t.equal(layer.x, want)


def test_two_streams_at_once():
    t = torch()
    rng = np.random.default_rng(9)
    ps = [Product(rng, 64, 1024, 4096, "f32"), Product(rng, 64, 1024, 4096, "f32")]
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    t.cuda.synchronize()
    for _ in range(10):
        for p, s in zip(ps, streams):
            p.call(stream=s.cuda_stream)
    t.cuda.synchronize()
    for p in ps:
        p.check()
