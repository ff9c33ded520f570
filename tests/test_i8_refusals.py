"""The operators of 8-bit linear layers refuse what they cannot do before anything is launched, and the model they
are tested against is right on hand values (no GPU)."""
import numpy as np
import pytest

from paper_2505_05286_amd import hxf

from . import i8_util as U
from ._lib import ensure_built


@pytest.fixture(autouse=True)
def _built():
    ensure_built()


A = 4096          # an aligned address that nothing reads


def _refused(code, f, **k):
    with pytest.raises(hxf.HxfError) as e:
        f(**k)
    assert e.value.code == code


def _quant(**k):
    d = dict(x=A, stride=128, R=3, K=128, codes=A, scale=A)
    d.update(k)
    hxf.op_quant_i8(*d.values())


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=A + 8), dict(stride=120), dict(stride=132), dict(R=-1),
                                 dict(R=(1 << 22) - 15), dict(K=0), dict(K=-8), dict(K=100), dict(K=1 << 17, stride=1 << 17),
                                 dict(codes=None), dict(codes=A + 8), dict(scale=None)])
def test_quant_refuses(bad):
    _refused(hxf.EINVAL, _quant, **bad)


def _norm(**k):
    d = dict(x=A, rows=A, x_rows=9, g=A, codes=A, scale=A, n_rows=3, d=128, eps=1e-5)
    d.update(k)
    hxf.op_rmsnorm_i8(*d.values())


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=A + 4), dict(x_rows=-1), dict(rows=0, x_rows=2), dict(g=None),
                                 dict(g=A + 2), dict(codes=None), dict(codes=A + 4), dict(scale=None), dict(n_rows=-1),
                                 dict(n_rows=(1 << 22) - 15, x_rows=1 << 23), dict(d=0), dict(d=126), dict(d=1 << 17)])
def test_norm_refuses(bad):
    _refused(hxf.EINVAL, _norm, **bad)


def _gemm(**k):
    d = dict(a=A, sa=A, b=A, sb=A, b2=0, sb2=0, c=A, ldc=64, M=3, N=64, K=100, epi=hxf.EPI_BF16, ws=A,
             ws_bytes=1 << 40)
    d.update(k)
    hxf.op_gemm_i8(*d.values())


SW = dict(epi=hxf.EPI_SWIGLU, b2=A, sb2=A, ldc=32)


@pytest.mark.parametrize("bad", [dict(a=None), dict(a=A + 8), dict(sa=None), dict(b=None), dict(b=A + 1), dict(sb=None),
                                 dict(c=None), dict(ldc=63), dict(M=-1), dict(M=(1 << 22) - 15), dict(N=0), dict(N=-64),
                                 dict(N=1 << 22, ldc=1 << 22), dict(K=0), dict(K=-1), dict(K=1 << 17), dict(epi=-1), dict(epi=4),
                                 dict(epi=hxf.EPI_BF16 | hxf.GEMM_A_PACKED), dict(c=A + 1), dict(c=A + 2, epi=hxf.EPI_F32),
                                 dict(c=A + 2, epi=hxf.EPI_RESID), dict(M=1 << 18, N=1 << 18, ldc=1 << 18),
                                 dict(SW, b2=0), dict(SW, sb2=0), dict(SW, b2=A + 8), dict(SW, N=63), dict(SW, ldc=31)])
def test_gemm_refuses(bad):
    _refused(hxf.EINVAL, _gemm, **bad)


def test_sizes_of_buffers():
    assert hxf.i8_codes_bytes(0, 64) == 0
    assert hxf.i8_codes_bytes(1, 1) == 1024 and hxf.i8_codes_bytes(16, 64) == 1024
    assert hxf.i8_codes_bytes(17, 65) == 4096
    assert hxf.i8_codes_bytes((1 << 22) - 16, (1 << 17) - 1) == (1 << 39) - (1 << 21)
    for bad in ((-1, 64), ((1 << 22) - 15, 64), (4, 0), (4, 1 << 17)):
        assert hxf.i8_codes_bytes(*bad) == -1
    for bad in ((-1, 64, 64), (4, 0, 64), (4, 64, 0), (4, 64, 1 << 17), (1 << 18, 1 << 18, 64)):
        assert hxf.op_gemm_i8_workspace_bytes(*bad) == -1


@pytest.mark.parametrize("m,n,k", [(64, 4096, 14336), (256, 8192, 28672)])
def test_a_short_workspace_is_refused(m, n, k):
    """Products whose K is cut need their partials, four bytes an output and piece."""
    need = hxf.op_gemm_i8_workspace_bytes(m, n, k)
    assert need > 0 and need % (4 * m * n) == 0
    for bad in (dict(ws_bytes=0), dict(ws=0), dict(ws=A + 8), dict(ws_bytes=4 * m * n)):
        for epi in (hxf.EPI_BF16, hxf.EPI_RESID, hxf.EPI_F32):
            _refused(hxf.ENOMEM, _gemm, M=m, N=n, K=k, ldc=n, epi=epi, **bad)


def test_empty_batches_are_done_without_a_launch():
    _quant(R=0)
    _norm(n_rows=0, x_rows=0)
    _gemm(M=0)


def test_the_model_by_hand():
    codes, scale = U.codes_of([[0.5, -1.0, 1.0, 0.25], [0, 0, 0, 0], [2.0 ** -120, 0, 0, 0], [1, np.nan, 2, 3],
                               [np.inf, 1, 0, 0]])
    # 63.5 is a tie: to the even 64; 31.75 rounds to 32
    assert codes[0].tolist() == [64, -127, 127, 32] and scale[0] == np.float32(1 / np.float32(127))
    assert not codes[1:].any() and scale[1] == 0 and scale[2] == 0 and np.isnan(scale[3:]).all()
    t = U.tile(np.arange(1, 36, dtype=np.int8)[:, None] * np.ones((1, 70), np.int8))
    assert t.size == 3 * 2 * 1024
    assert t[0] == 1 and t[16] == 2 and t[256] == 1 and t[1024] == 1 and t[2048] == 17 and t[1024 + 5] == 1
    assert t[1024 + 6] == 0 and t[2 * 2048 + 3 * 16] == 0       # column 70, row 35: padding
    # x g and the norm's factor
    y, r = U.norm_rows([[3.0, -4.0], [1.0, 1.0]], [0, 5, -1, 0], [2.0, 0.5], 0.0)
    assert y.tolist() == [[6, -2], [0, 0], [0, 0], [6, -2]] and r[0] == 1 / np.sqrt(12.5)
    p = U.product(np.array([[1, -2]], np.int8), [0.5], np.array([[3, 4], [127, -127]], np.int8), [2.0, 1.0])
    assert p.tolist() == [[-5.0, 190.5]]
    assert U.silu(np.array([0.0, 800.0, -800.0])).tolist() == [0.0, 800.0, -0.0]


def test_plans_report_what_the_shapes_of_the_gpu_test_take():
    """Every kernel instance that the table stands for is taken, whole and cut K alike, and pieces cover K."""
    seen = set()
    for m, n, k in U.PLANS:
        for epi in range(4):
            tm, nw, wv, once, splits, piece, thin = hxf.op_gemm_i8_plan(m, 2 * n if epi == hxf.EPI_SWIGLU else n, k, epi)
            kt = -(-k // 64)
            assert piece % 2 == 0 and splits == (1 if thin else -(-kt // piece)) and (thin or (splits - 1) * piece < kt)
            seen.add((tm, nw, wv, once, thin, splits > 1))
    assert len(seen) >= 80
    assert {t[4] for t in seen} == {0, 1} and {t[2] for t in seen if not t[4]} == {4, 8}
    for bad in ((0, 64, 64, 0), (4, 0, 64, 0), (4, 63, 64, hxf.EPI_SWIGLU), (4, 64, 0, 0), (4, 64, 64, 4)):
        with pytest.raises(hxf.HxfError):
            hxf.op_gemm_i8_plan(*bad)


@pytest.mark.parametrize("m,n,k", U.PLANS)
def test_workspace_covers_the_plan(m, n, k):
    for epi in range(4):
        cols = 2 * n if epi == hxf.EPI_SWIGLU else n
        splits = hxf.op_gemm_i8_plan(m, cols, k, epi)[4]
        assert hxf.op_gemm_i8_workspace_bytes(m, cols, k) >= (splits * m * cols * 4 if splits > 1 else 0)
