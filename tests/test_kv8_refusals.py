"""The operators of the 8-bit KV cache refuse what they cannot do before anything is launched, and the model
they are tested against is right on hand values (no GPU)."""
import os
import subprocess

import numpy as np
import pytest

from paper_2505_05286_amd import hxf

from . import kv8_util as U
from ._lib import ensure_built


@pytest.fixture(autouse=True)
def _built():
    ensure_built()


A = 4096          # an aligned address that nothing reads


def _refused(code, f, *a, **k):
    with pytest.raises(hxf.HxfError) as e:
        f(*a, **k)
    assert e.value.code == code


def _pool(**k):
    d = dict(k=A, v=A, k_scale=A, v_scale=A, n_blocks=8)
    d.update(k)
    return hxf.Kv8Pool(*d.values())


BAD_POOLS = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(n_blocks=0), dict(n_blocks=-1),
             dict(n_blocks=1 << 27), dict(k=A + 8), dict(v=A + 1)]


def _slot_map(**k):
    d = dict(start=A, n_new=A, S=4, free_pages=A, n_free=A, free_cap=9, bt=A, bt_stride=5, row0=A, pos=A, slot=A, T=8,
             ctx=A, status=A)
    d.update(k)
    hxf.op_slot_map(*d.values())


@pytest.mark.parametrize("bad", [dict(start=None), dict(n_new=None), dict(S=-1), dict(S=hxf.SLOT_MAP_MAX_SEQS + 1),
                                 dict(free_pages=None), dict(n_free=None), dict(free_cap=-1), dict(bt=None),
                                 dict(bt_stride=0), dict(bt_stride=1 << 26), dict(row0=None), dict(pos=None),
                                 dict(slot=None), dict(T=-1), dict(ctx=None), dict(status=None)])
def test_slot_map_refuses(bad):
    _refused(hxf.EINVAL, _slot_map, **bad)


def _write(**k):
    d = dict(qkv=A, qkv_stride=8 * 128, pos=A, slot=A, table=A, max_pos=64, q_out=A, q_stride=4 * 128, pool=_pool(),
             T=3, Hq=4, Hkv=2, dh=128)
    d.update(k)
    hxf.op_rope_kv8_write(*d.values())


@pytest.mark.parametrize("bad", [dict(qkv=None), dict(qkv=A + 2), dict(qkv_stride=8 * 128 - 8), dict(qkv_stride=1028),
                                 dict(pos=None), dict(slot=None), dict(max_pos=0), dict(q_out=A + 4),
                                 dict(q_stride=504), dict(q_stride=513), dict(table=A + 8), dict(T=-1), dict(Hq=5),
                                 dict(Hkv=0), dict(Hq=34), dict(dh=96), dict(dh=256), dict(pool=None)] +
                         [dict(pool=_pool(**p)) for p in BAD_POOLS])
def test_write_refuses(bad):
    _refused(hxf.EINVAL, _write, **bad)


@pytest.mark.parametrize("f,bad", [(_slot_map, dict(T=1 << 30)), (_slot_map, dict(T=2 ** 31 - 1)),
                                   (_slot_map, dict(free_cap=1 << 30)), (_slot_map, dict(free_cap=2 ** 31 - 1)),
                                   (_write, dict(T=1 << 30)), (_write, dict(T=2 ** 31 - 1))])
def test_counts_whose_indices_would_pass_32_bits_are_refused(f, bad):
    _refused(hxf.EINVAL, f, **bad)


def _decode(**k):
    d = dict(q=A, q_stride=512, pool=_pool(), bt=A, bt_stride=4, ctx=A, out=A, out_stride=512, B=3, Hq=4, Hkv=2,
             dh=128, ws=A, ws_bytes=1 << 40)
    d.update(k)
    hxf.op_decode_attention_kv8(*d.values())


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=A + 8), dict(q_stride=511), dict(q_stride=504), dict(bt=None),
                                 dict(bt_stride=0), dict(bt_stride=1 << 26), dict(ctx=None), dict(out=None),
                                 dict(out=A + 2), dict(out_stride=500), dict(B=-1), dict(Hq=6, Hkv=4), dict(Hkv=-2),
                                 dict(Hq=68), dict(dh=32), dict(pool=None)] + [dict(pool=_pool(**p)) for p in BAD_POOLS])
def test_decode_refuses(bad):
    _refused(hxf.EINVAL, _decode, **bad)


def test_decode_refuses_a_short_workspace():
    n = hxf.op_decode_attention_kv8_workspace_bytes(3, 4, 2, 128)
    assert n > 0
    for bad in (dict(ws_bytes=n - 1), dict(ws_bytes=0), dict(ws=None), dict(ws=A + 8, ws_bytes=n)):
        _refused(hxf.ENOMEM, _decode, **bad)
    assert hxf.op_decode_attention_kv8_workspace_bytes(-1, 4, 2, 128) == -1
    assert hxf.op_decode_attention_kv8_workspace_bytes(3, 5, 2, 128) == -1
    assert hxf.op_decode_attention_kv8_workspace_bytes(3, 4, 2, 80) == -1


def _prefill(**k):
    d = dict(q=A, q_stride=512, pool=_pool(), bt=A, bt_stride=4, row0=A, pos0=A, out=A, out_stride=512, S=2, T=9, Hq=4,
             Hkv=2, dh=128, ws=A, ws_bytes=1 << 40)
    d.update(k)
    hxf.op_prefill_attention_kv8(*d.values())


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=A + 8), dict(q_stride=511), dict(q_stride=504), dict(bt=None),
                                 dict(bt_stride=0), dict(bt_stride=1 << 26), dict(row0=None), dict(pos0=None),
                                 dict(out=None), dict(out=A + 2), dict(out_stride=500), dict(S=-1), dict(T=-1),
                                 dict(Hq=6, Hkv=4), dict(Hkv=-2), dict(Hq=68), dict(dh=32), dict(pool=None)] +
                         [dict(pool=_pool(**p)) for p in BAD_POOLS])
def test_prefill_refuses(bad):
    _refused(hxf.EINVAL, _prefill, **bad)


def test_prefill_refuses_a_short_workspace():
    n = hxf.op_prefill_attention_kv8_workspace_bytes(2, 9, 4, 2, 128)
    assert n > 0
    for bad in (dict(ws_bytes=n - 1), dict(ws_bytes=0), dict(ws=None), dict(ws=A + 8, ws_bytes=n)):
        _refused(hxf.ENOMEM, _prefill, **bad)
    for a in ((-1, 9, 4, 2, 128), (2, -1, 4, 2, 128), (2, 9, 5, 2, 128), (2, 9, 4, 2, 80)):
        assert hxf.op_prefill_attention_kv8_workspace_bytes(*a) == -1


def test_nothing_to_do_is_no_error():
    """Empty batches return without touching a device."""
    _write(T=0)
    _decode(B=0, ws=None, ws_bytes=0)
    _prefill(S=0, ws=None, ws_bytes=0)
    _prefill(T=0, ws=None, ws_bytes=0)


def test_work_splits(tmp_path):
    """tests/kv8_split.cpp: the decode and prefill splits cover everything once and fit their launches."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "kv8_split")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(root, "paper_2505_05286_amd", "csrc"),
                    os.path.join(root, "tests", "kv8_split.cpp"), "-o", exe], check=True, capture_output=True,
                   timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


# ------------------------------------------------------------------ the model
def test_codes():
    assert U.VALUES[0x7E] == 448 and U.VALUES[0x01] == 2.0 ** -9 and U.VALUES[0x38] == 1 and U.VALUES[0xB8] == -1
    assert np.isnan(U.VALUES[0x7F]) and np.isnan(U.VALUES[0xFF])
    finite = np.delete(np.arange(256), [0x7F, 0xFF])
    np.testing.assert_array_equal(U.encode(U.VALUES[finite]), finite)
    # ties to the even code; below half the smallest value to zero
    np.testing.assert_array_equal(U.encode([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 1e-9, -2.0 ** -10, 447, 432]),
                                  [U.encode(16.0), U.encode(20.0), 0, 2, 0, 0x80, 0x7E, 0x7E])


def test_scales():
    assert U.scale_for(448.0) == 1 and U.scale_for(448.01) == 2 and U.scale_for(224.0) == 0.5
    assert U.scale_for(0.0) == 2.0 ** -100 and U.scale_for(1e-38) == 2.0 ** -100
    assert U.scale_for(3.38e38) == 2.0 ** 120


def test_layouts():
    pages = np.arange(16 * 64, dtype=np.int64).reshape(1, 16, 64)
    for kind in "kv":
        raw = U.pack(pages, kind)
        np.testing.assert_array_equal(U.unpack(raw, kind, 64), pages)
        for t, d in ((0, 0), (3, 17), (15, 63), (7, 32)):
            at = ((d // 16) * 16 + t) * 16 + d % 16 if kind == "k" else ((t // 4) * 64 + d) * 4 + t % 4
            assert raw[0, at] == pages[0, t, d]


def test_a_growing_page_keeps_its_codes_up_to_the_exponent():
    c = U.Cache(1, 1, 16)
    x = np.full((1, 1, 16), 1.0, np.float32)
    c.write_run("k", 0, 0, x)
    assert c.scale["k"][0, 0] == 2.0 ** -8 and U.VALUES[c.codes["k"][0, 0, 0, 0]] == 256
    c.write_run("k", 0, 1, 100 * x)
    assert c.scale["k"][0, 0] == 0.25 and U.VALUES[c.codes["k"][0, 0, 0, 0]] == 4
    np.testing.assert_array_equal(c.values("k", 0, [0])[:2, 0], [1.0, U.VALUES[U.encode(400.0)] / 4])
    c.write_run("k", 0, 2, 0 * x)          # nothing shrinks
    assert c.scale["k"][0, 0] == 0.25


def test_attention_of_one_key_is_its_value():
    c = U.Cache(1, 2, 64)
    c.fill(np.random.default_rng(0), [0, 1])
    o, size = U.attend(np.ones((1, 2, 64)), c, [1], 1, 2)
    np.testing.assert_allclose(o[0, 1], c.values("v", 0, [1])[0], rtol=1e-15)
    o, _ = U.attend(np.ones((1, 2, 64)), c, [-1], 16, 2)
    assert np.all(o == 0)


# ------------------------------------------------------------------ launches
def test_launch_limits(tmp_path):
    """tests/kv8_limits.cpp: the batches that the operators accept are those that their launches hold."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "kv8_limits")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(root, "paper_2505_05286_amd", "csrc"),
                    os.path.join(root, "tests", "kv8_limits.cpp"), "-o", exe], check=True, capture_output=True,
                   timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_batches_whose_launch_would_pass_32_bits_of_threads_are_refused():
    """With HXF_EINVAL, before anything is enqueued, and with no size of a workspace for them."""
    wide = dict(qkv_stride=1 << 30, q_stride=1 << 30)
    for bad in (dict(T=(1 << 28) - 15), dict(T=1 << 29), dict(Hq=1 << 16, Hkv=1 << 16, **wide),
                dict(Hq=1 << 30, Hkv=1 << 30, qkv_stride=1 << 40, q_stride=1 << 40)):
        _refused(hxf.EINVAL, _write, **bad)
    one = dict(Hq=1, Hkv=1, dh=64)
    _refused(hxf.EINVAL, _decode, B=(1 << 26) - 3 * 1024, bt_stride=4, **one)
    _refused(hxf.EINVAL, _decode, B=1 << 24, bt_stride=9, **one)
    _refused(hxf.EINVAL, _prefill, S=(1 << 24) - 1, T=1, **one)
    assert hxf.op_decode_attention_kv8_workspace_bytes((1 << 26) - 3 * 1024, 1, 1, 64) == -1
    assert hxf.op_decode_attention_kv8_workspace_bytes((1 << 26) - 3 * 1024 - 1, 1, 1, 64) > 0
    assert hxf.op_prefill_attention_kv8_workspace_bytes((1 << 24) - 1, 1, 1, 1, 64) == -1
    assert hxf.op_prefill_attention_kv8_workspace_bytes((1 << 24) - 2, 1, 1, 1, 64) > 0


def test_dequantised_values_are_bf16_values_up_to_scales_of_2_119():
    """Every code times every scale that the write makes below 2^120 is a finite bf16 value; at 2^120 those of codes under 256
    are, and |x| under 1.9375 * 2^127 gets no other code."""
    v = np.delete(U.VALUES, [0x7F, 0xFF])
    for e in range(-100, 121):
        x = (v if e < 120 else v[np.abs(v) < 256]) * 2.0 ** e
        f = x.astype(np.float32)
        assert np.all(np.isfinite(f)) and np.array_equal(f.astype(np.float64), x)
        assert not np.any(f.view(np.uint32) & 0xFFFF)
    assert U.scale_for(1.75 * 2.0 ** 127) == 2.0 ** 119 and U.scale_for(1.76 * 2.0 ** 127) == 2.0 ** 120
    top = np.nextafter(np.float32(1.9375 * 2.0 ** 127), np.float32(0)).astype(np.float64)
    assert U.VALUES[U.encode(top / 2.0 ** 120)] == 240 and U.VALUES[U.encode(248.0)] == 256
