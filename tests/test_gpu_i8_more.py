"""Linear layers in 8-bit integers on the GPU: values at the ends of the number formats, every instance of the product,
cut K in batches, on streams and in graphs."""
import numpy as np
import pytest

from paper_2505_05286_amd import hxf

from . import i8_instances
from . import i8_util as U
from ._lib import ensure_built
from .gpu_util import torch
from .test_gpu_i8 import DEV, GUARD, U32, UB16, Codes, Layer, Product, _bf16, _dev, _tile_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built():
    ensure_built()


# in the kernel that shares K out in a workgroup, in those with whole K and with cut K and its join
@pytest.mark.parametrize("M,F,K,thin,cut", [(20, 600, 1600, 1, False), (3, 200, 64, 0, False), (150, 202, 192, 0, False),
                                            (66, 2706, 7248, 0, True)])
def test_swiglu_at_gates_far_below_zero(M, F, K, thin, cut):
    """silu(z) is a normal bf16 value down to z = -91.9, and times a large up value further down: gates from -112 to -60
    and a few near and above zero, up values from 2^-7 to 2^100."""
    p = Product(np.random.default_rng(M), M, 2 * F, K, "swiglu")
    plan = hxf.op_gemm_i8_plan(M, 2 * F, K, hxf.EPI_SWIGLU)
    assert plan[6] == thin and (plan[4] > 1) == cut
    z = np.linspace(-112, -60, F)
    z[::17] = np.linspace(-3, 90, len(z[::17]))
    p.a[:], p.b[:], p.b2[:] = 0, 0, 0
    p.a[:, 0] = 1 + np.arange(M) % 3
    p.b[:, 0], p.b2[:, 0] = -100, 127
    p.sa[:] = 1 / (1 + np.arange(M) % 3).astype(np.float32)
    p.sb[:] = z / -100
    p.sb2[:] = np.array([2.0 ** -14, 2.0 ** -3, 2.0 ** 53, 2.0 ** 93], np.float32)[np.arange(F) % 4]
    p.dev = [_dev(v) for v in (U.tile(p.a), p.sa, U.tile(p.b), p.sb, U.tile(p.b2), p.sb2)]
    p.call()
    got = p.c.float().cpu().numpy()[:M * p.ldc].reshape(M, p.ldc)[:, :F].astype(np.float64)
    y, up = U.product(p.a, p.sa, p.b, p.sb), U.product(p.a, p.sa, p.b2, p.sb2)
    want = U.silu(y) * up
    # relative: two half steps of the gate and two of e^-z's exponent, times |z|; a few each of the exponential, the sum,
    # the reciprocal, the products and up; then bf16's.  Below the normal numbers half a step of silu (times up) and of
    # the product in fp32, and of bf16.
    tol = ((6 * np.abs(y) + 16) * U32 + UB16) * np.abs(want) + 2.0 ** -149 * (np.abs(up) + 1) + 2.0 ** -134
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), [(y[i, j], up[i, j], got[i, j], want[i, j]) for i, j in np.argwhere(bad)[:4]])


@pytest.mark.parametrize("d", [128, 1000, 3000, 8000, 20000, 33000])
def test_norm_without_eps(d):
    """eps 0: rows of zeros, and those too small for codes, have the scale 0, like rows that are quantised without a norm;
    small rows that have codes are as good as others; a row that is not finite stays NaN."""
    rng = np.random.default_rng(d)
    x = rng.standard_normal((37, d)).astype(np.float32)
    x[::5] = 0
    x[3] *= np.float32(2.0 ** -125)
    x[6] *= np.float32(2.0 ** -45)
    x[8, d // 2] = np.nan
    gb, g = _bf16(1 + rng.uniform(-0.5, 0.5, d))
    out = Codes(37, d)
    xd, gd = _dev(x), _dev(gb.view(np.int16))
    hxf.op_rmsnorm_i8(xd.data_ptr(), 0, 37, gd.data_ptr(), *out.ptrs(), 37, d, 0.0)
    codes, scale = out.get()
    y, r = U.norm_rows(x, None, g, 0.0)
    want, unit = U.codes_of(y)
    assert np.array_equal(codes, U.tile(want))
    zero = unit == 0
    assert zero[::5].all() and zero[3] and not scale[zero].any()
    assert np.isnan(scale[8]) and np.isnan(unit).sum() == 1
    ok = unit > 0
    tol = ((d / 64 + 16) / 2 + 8) * U32      # as with eps: the chain of the sum, halved by the root, and a few steps more
    assert ok[6] and (np.abs(scale[ok] - unit[ok] * r[ok]) <= tol * unit[ok] * r[ok]).all()


def test_a_workspace_for_the_largest_batch_serves_smaller_ones():
    """One buffer, sized once for a batch whose K is whole, for batches whose K is cut."""
    t = torch()
    rng = np.random.default_rng(23)
    N, K = 1024, 4096
    n = hxf.op_gemm_i8_workspace_bytes(2080, N, K)
    ws = t.full((n + GUARD,), 0x5A, dtype=t.uint8, device=DEV)
    assert hxf.op_gemm_i8_plan(2080, N, K, hxf.EPI_RESID)[4] == 1
    assert all(hxf.op_gemm_i8_plan(m, N, K, hxf.EPI_RESID)[4] > 1 for m in (300, 129))
    for m in (2080, 300, 129, 33):
        p = Product(rng, m, N, K, "resid")
        p.ws = ws
        p.call()
        p.check()


@pytest.mark.parametrize("M,N,K,epi", i8_instances.MORE)
def test_gemm_in_the_instances_of_one_epilogue(M, N, K, epi):
    """With the other list's, every compiled instance of the kernels; whole numbers by products in 64 bits (exact below
    2^53), rows of outputs a column apart, the buffers' ends guarded."""
    t = torch()
    cols, gated, wide = (2 * N if epi == "swiglu" else N), epi == "swiglu", epi in ("resid", "f32")
    print(i8_instances.instance(M, N, K, epi), flush=True)
    g = t.Generator(device=DEV)
    g.manual_seed(M * 7 + N)
    rand = lambda n: t.randint(-127, 128, (n, K), generator=g, device=DEV, dtype=t.int8)   # noqa: E731
    a, b, b2 = rand(M), rand(N), rand(N if gated else 1)
    sa = t.rand(M, generator=g, device=DEV) + 0.5
    sb, sb2 = ((t.rand(len(w), generator=g, device=DEV) + 0.5) / (5000 * K ** 0.5) for w in (b, b2))
    dev = [_tile_dev(v) for v in (a, b, b2)]
    c = t.full((M * (N + 1) + GUARD,), 3.0, device=DEV, dtype=t.float32 if wide else t.bfloat16)
    view = c[:M * (N + 1)].view(M, N + 1)
    if epi == "resid":
        view[:, :N] = t.randn(M, N, generator=g, device=DEV)
    old = view[:, :N].double()
    n = hxf.op_gemm_i8_workspace_bytes(M, cols, K)
    ws = t.full((n + GUARD,), 0x5A, dtype=t.uint8, device=DEV)
    hxf.op_gemm_i8(dev[0].data_ptr(), sa.data_ptr(), dev[1].data_ptr(), sb.data_ptr(), dev[2].data_ptr() if gated else 0,
                   sb2.data_ptr() if gated else 0, c.data_ptr(), N + 1, M, cols, K, i8_instances.EPILOGUES[epi], ws.data_ptr(), n)
    t.cuda.synchronize()
    assert bool((ws[n:] == 0x5A).all()) and bool((view[:, N] == 3.0).all()) and bool((c[M * (N + 1):] == 3.0).all())
    y = ((a.double() @ b.double().T) * sa.double()[:, None]) * sb.double()
    rel = 3.001 * U32           # float(acc) and two products
    if gated:
        want = y * t.sigmoid(y) * (((a.double() @ b2.double().T) * sa.double()[:, None]) * sb2.double())
        tol = (UB16 + (6 * y.abs() + 16) * U32) * want.abs() + 2.0 ** -134
    elif epi == "resid":
        want = y + old
        tol = rel * y.abs() + 1.001 * U32 * (want.abs() + rel * y.abs())
    else:
        want, tol = y, (rel + (0 if wide else UB16 + rel)) * y.abs()
    bad = ~((view[:, :N].double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


def _cut(m, n, k, epi):
    """The product is cut into pieces of K: partials in the workspace and a second launch."""
    assert hxf.op_gemm_i8_plan(m, n, k, i8_instances.EPILOGUES[epi])[4] > 1


def test_products_with_cut_k_on_two_streams_at_once():
    """A workspace each, other operands, outputs and workspaces filled with something else before each call."""
    t = torch()
    rng = np.random.default_rng(19)
    ps = [Product(rng, 33, 1024, 8192, "f32"), Product(rng, 300, 512, 4096, "f32")]
    for p in ps:
        _cut(p.M, p.N, p.K, p.epi)
    streams = [t.cuda.Stream() for _ in ps]
    t.cuda.synchronize()
    seen = [[], []]
    for _ in range(8):
        for p, s, out in zip(ps, streams, seen):
            with t.cuda.stream(s):
                p.c[:p.M * p.ldc].fill_(float("nan"))
                p.ws[:-GUARD].fill_(0x33)
                p.call(stream=s.cuda_stream)
                out.append(p.c.clone())
    t.cuda.synchronize()
    for p, out in zip(ps, seen):
        p.check()
        assert all(t.equal(c, p.c) for c in out)


def _layers(rng):
    """Blocks whose gate and up projections, or whose down projection, are cut."""
    _cut(70, 2 * 1408, 4096, "swiglu")
    _cut(33, 1024, 8192, "resid")
    return [Layer(rng, 70, 4096, 1408), Layer(rng, 33, 1024, 8192)]


def _eager(layer, x):
    layer.ws.fill_(0x33)
    layer.x.copy_(x)
    layer.run()
    return layer.x.clone()


def test_blocks_with_cut_k_step_by_step():
    """Each step from what the step before it left: codes to the bit, scales and products within their roundings."""
    rng = np.random.default_rng(20)
    for layer in _layers(rng):
        x = rng.standard_normal((layer.T, layer.d)).astype(np.float32)
        got = _eager(layer, _dev(x)).cpu().numpy().astype(np.float64)
        (gate, sg), (up, su), (down, sd) = (U.codes_of(w) for w in layer.wv)
        y, r = U.norm_rows(x, None, layer.g, np.float32(1e-5))
        a, unit = U.codes_of(y)
        codes, sa = layer.cx.get()
        assert np.array_equal(codes, U.tile(a))
        assert (np.abs(sa - unit * r) <= ((layer.d / 64 + 16) / 2 + 8) * U32 * unit * r).all()
        h = layer.h.float().cpu().numpy()
        z = U.product(a, sa, gate, sg)
        want = U.silu(z) * U.product(a, sa, up, su)
        assert (np.abs(h - want) <= (UB16 + (6 * np.abs(z) + 16) * U32) * np.abs(want) + 2.0 ** -134).all()
        a, unit = U.codes_of(h)
        codes, sa = layer.ch.get()
        assert np.array_equal(codes, U.tile(a)) and np.array_equal(sa, unit)
        v = U.product(a, sa, down, sd)
        rel = 3.001 * U32
        assert (np.abs(got - (x + v)) <= rel * np.abs(v) + 1.001 * U32 * (np.abs(x + v) + rel * np.abs(v))).all()


def test_blocks_with_cut_k_on_streams_of_their_own():
    t = torch()
    rng = np.random.default_rng(21)
    layers = _layers(rng)
    xs = [_dev(rng.standard_normal((v.T, v.d)).astype(np.float32)) for v in layers]
    wants = [_eager(v, x) for v, x in zip(layers, xs)]
    streams = [t.cuda.Stream() for _ in layers]
    t.cuda.synchronize()
    gots = [[], []]
    for _ in range(4):
        for layer, x, s, out in zip(layers, xs, streams, gots):
            with t.cuda.stream(s):
                layer.h.zero_()
                out.append(_eager(layer, x))
    t.cuda.synchronize()
    for want, out in zip(wants, gots):
        assert all(t.equal(v, want) for v in out)


def test_captured_blocks_with_cut_k_replay_on_new_inputs():
    """Two graphs with a workspace each, replayed at once on two streams; eager calls and waits between the replays."""
    t = torch()
    rng = np.random.default_rng(22)
    layers = _layers(rng)
    graphs, streams = [], [t.cuda.Stream() for _ in layers]
    for layer in layers:
        layer.run()
        t.cuda.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            layer.run()
        graphs.append(graph)
    for k in range(4):
        xs = [_dev(rng.standard_normal((v.T, v.d)).astype(np.float32)) for v in layers]
        wants = [_eager(v, x) for v, x in zip(layers, xs)]
        for layer, x in zip(layers, xs):
            layer.x.copy_(x)
            layer.ws.fill_(0x33)
            layer.h.zero_()
        t.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with t.cuda.stream(s):
                graph.replay()
        t.cuda.synchronize()
        for layer, want in zip(layers, wants):
            assert t.equal(layer.x, want)
