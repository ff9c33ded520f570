"""The operators of the 8-bit KV cache against a plain model in float64 (tests/kv8_util.py): tables and
codes to the last bit, attention within the roundings it makes."""
import copy

import numpy as np
import pytest

import synth
from paper_2505_05286_amd import hxf

from . import kv8_util as U
from .gpu_util import dev_bits, host_f64, i32, log, rand_bf16, torch

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (32, 8, 128), (40, 8, 128), (16, 1, 64), (3, 3, 128), (13, 1, 128), (14, 2, 64)]


class DevCache:
    """A Cache in HBM."""

    def __init__(self, c):
        t = torch()
        self.c = c
        put = lambda a: t.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
        self.k, self.v = (put(U.pack(c.codes[x], x)) for x in "kv")
        self.ks, self.vs = put(c.scale["k"]), put(c.scale["v"])
        self.pool = hxf.Kv8Pool(self.k.data_ptr(), self.v.data_ptr(), self.ks.data_ptr(), self.vs.data_ptr(), c.nb)

    def check(self, what):
        for kind, codes, scale in (("k", self.k, self.ks), ("v", self.v, self.vs)):
            got = U.unpack(codes.cpu().numpy(), kind, self.c.dh)
            np.testing.assert_array_equal(scale.cpu().numpy(), self.c.scale[kind], err_msg=f"{what}: {kind} scales")
            assert U.same_codes(got, self.c.codes[kind]), (
                f"{what}: {kind} codes differ at {np.argwhere(got != self.c.codes[kind])[:5].tolist()}")


def _dev_slot_map(start, n_new, free, n_free, bt, T, stream=0):
    t = torch()
    S, stride = bt.shape
    guard = 7                                    # words past each output that stay as they are
    new = lambda n: t.full((n + guard,), 77, dtype=t.int32, device="cuda:0")
    o = {"bt": i32(bt), "row0": new(S + 1), "pos": new(T), "slot": new(T), "ctx": new(S), "status": new(2)}
    a, b, f, nf = i32(start), i32(n_new), i32(np.append(free, [0])), i32([n_free])
    hxf.op_slot_map(a.data_ptr(), b.data_ptr(), S, f.data_ptr(), nf.data_ptr(), len(free), o["bt"].data_ptr(), stride,
                    o["row0"].data_ptr(), o["pos"].data_ptr(), o["slot"].data_ptr(), T, o["ctx"].data_ptr(),
                    o["status"].data_ptr(), stream=stream)
    t.cuda.synchronize()
    out = {k: v.cpu().numpy() for k, v in o.items()}
    for k, n in (("row0", S + 1), ("pos", T), ("slot", T), ("ctx", S), ("status", 2)):
        assert np.all(out[k][n:] == 77), k
        out[k] = out[k][:n]
    return out


def _check_slot_map(start, n_new, free, bt, T, what, n_free=None):
    start, n_new = np.asarray(start, np.int64), np.asarray(n_new, np.int64)
    n_free = len(free) if n_free is None else n_free
    log(f"slot map {what}: S={len(start)} T={T}")
    got = _dev_slot_map(start, n_new, np.asarray(free), n_free, bt, T)
    ref = U.slot_map(start, n_new, free[:max(0, min(n_free, len(free)))], bt, T)
    for k, r in zip(("bt", "row0", "pos", "slot", "ctx", "status"), ref):
        np.testing.assert_array_equal(got[k], r, err_msg=f"{what}: {k}")
    return got


def _batch(rng, S, hi_start, hi_new):
    start = rng.integers(0, hi_start + 1, S)
    n_new = rng.integers(0, hi_new + 1, S)
    old, end = -(-start // 16), -(-(start + n_new) // 16)
    stride = int(end.max(initial=0)) + 2
    order = rng.permutation(int(end.sum()) + 9)
    bt = np.full((S, stride), -5, np.int64)
    at = 0
    for s in range(S):
        bt[s, :old[s]] = order[at:at + old[s]]
        at += old[s]
    return start, n_new, order[at:], bt


@pytest.mark.parametrize("S,hi_start,hi_new", [(0, 0, 0), (1, 0, 1), (1, 100, 1), (2, 0, 40), (63, 50, 3), (64, 300, 1),
                                               (65, 31, 33), (257, 64, 17), (1000, 500, 30), (1025, 3, 2),
                                               (4096, 90, 5), (5, 3000, 5000)])
def test_slot_map(S, hi_start, hi_new):
    rng = np.random.default_rng(S * 1000 + hi_start + hi_new)
    start, n_new, free, bt = _batch(rng, S, hi_start, hi_new)
    for pad in (0, 1, 45):
        _check_slot_map(start, n_new, free, bt, int(n_new.sum()) + pad, f"pad {pad}")


def test_slot_map_page_borders():
    """Lengths on both sides of a page's end; sequences that get nothing between ones that do."""
    start = np.array([0, 15, 16, 17, 0, 31, 32, 48, 15, 16])
    n_new = np.array([16, 1, 0, 15, 17, 1, 1, 0, 2, 16])
    end = -(-(start + n_new) // 16)
    old = -(-start // 16)
    bt = np.full((10, int(end.max())), -1, np.int64)
    for s in range(10):
        bt[s, :old[s]] = 100 + 10 * s + np.arange(old[s])
    need = int((end - old).sum())
    got = _check_slot_map(start, n_new, np.arange(500, 500 + need), bt, int(n_new.sum()), "borders")
    assert got["status"][0] == need       # the last free page is taken, and no more


@pytest.mark.parametrize("why", ["pages", "n_free", "n_free negative", "rows", "stride", "held pages", "start", "new"])
def test_slot_map_that_does_not_fit_changes_nothing(why):
    rng = np.random.default_rng(7)
    start, n_new, free, bt = _batch(rng, 70, 100, 40)
    need = int((-(-(start + n_new) // 16) - -(-start // 16)).sum())
    free, T, n_free = free[:need], int(n_new.sum()), None
    if why == "pages":
        free = free[:-1]
    elif why.startswith("n_free"):
        n_free = need - 1 if why == "n_free" else -3
    elif why == "rows":
        T -= 1
    elif why == "stride":
        bt = bt[:, :int((-(-(start + n_new) // 16)).max()) - 1].copy()
    elif why == "held pages":
        start[3], n_new[3] = 16 * bt.shape[1] + 1, 0
    elif why == "start":
        start[69] = -1
    else:
        n_new[0] = -1
    got = _check_slot_map(start, n_new, free, bt, T, why, n_free)
    assert got["status"].tolist() == [-1, 0]


def test_slot_map_counts_beyond_the_free_list():
    """n_free larger than the list's capacity counts as the capacity; sums beyond 32 bits do not wrap."""
    bt = np.full((3, 5), -1, np.int64)
    _check_slot_map([0, 0, 0], [20, 1, 7], np.arange(9, 13), bt, 28, "capacity", n_free=1000)
    _check_slot_map([0, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 2], np.arange(4), bt, 10, "wrap")
    _check_slot_map([2 ** 31 - 1, 0, 0], [2 ** 31 - 1, 1, 1], np.arange(4), bt, 10, "wrap of one")


def _write(cache, dev, rng, slot, pos, hq, table, scale=1.0, bits=None, pad_cols=0, q_pad=0):
    """One call of the write against the model, q_out included; bits: the rows to take."""
    t = torch()
    T, hkv, dh = len(slot), cache.hkv, cache.dh
    width = (hq + 2 * hkv) * dh
    if bits is None:
        bits = rand_bf16(rng, (T, width), scale)[0]
    rows = np.full((T, width + pad_cols), 0x7FC0, np.uint16)
    rows[:, :width] = bits
    d_rows, d_pos, d_slot = dev_bits(rows), i32(pos), i32(slot)
    before = rows.copy()
    q = dev_bits(np.full((T, hq * dh + q_pad), 0x1234, np.uint16))
    tab = t.from_numpy(table).to("cuda:0") if table is not None else None
    hxf.op_rope_kv8_write(d_rows.data_ptr(), width + pad_cols, d_pos.data_ptr(), d_slot.data_ptr(),
                          tab.data_ptr() if tab is not None else 0, len(table) if tab is not None else 0,
                          q.data_ptr(), hq * dh + q_pad, dev.pool, T, hq, hkv, dh)
    t.cuda.synchronize()
    x = U.f32_of(bits).reshape(T, hq + 2 * hkv, dh)
    live = (slot >= 0) & (slot < cache.nb * 16)
    qk = x[:, :hq + hkv]
    if table is not None:
        live &= (pos >= 0) & (pos < len(table))
        qk = U.rotate(qk, table[np.where(live, pos, 0)])
    cache.write(qk[:, hq:], x[:, hq + hkv:], np.where(live, slot, -1))
    dev.check(f"T={T}")
    got = q.cpu().numpy().view(np.uint16)
    ref = np.full_like(got, 0x1234)
    ref[live, :hq * dh] = synth.f32_to_bf16_bits(qk[live, :hq].reshape(-1, hq * dh))
    fin = np.ones_like(got, bool)
    fin[live, :hq * dh] = np.isfinite(qk[live, :hq].reshape(-1, hq * dh))
    np.testing.assert_array_equal(np.where(fin, got, 0), np.where(fin, ref, 0))
    assert np.all(~np.isfinite(U.f32_of(got)[~fin]))
    np.testing.assert_array_equal(d_rows.cpu().numpy().view(np.uint16), before)


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_write_in_pieces(hq, hkv, dh):
    """A sequence in chunks of many lengths with values that grow and shrink: codes, scales, requantised pages
    and untouched places after every call."""
    rng = np.random.default_rng(hq * 100 + hkv + dh)
    cache = U.Cache(hkv, 23, dh)
    dev = DevCache(cache)
    blocks = rng.permutation(23)
    table = U.rope_table(400, dh)
    p = 0
    for i, n in enumerate([1, 1, 14, 5, 1, 27, 16, 33, 1, 1, 2, 64, 1, 3, 100]):
        pos = np.arange(p, p + n)
        slot = blocks[pos // 16] * 16 + pos % 16
        log(f"write {hq}/{hkv}x{dh}: {n} rows at {p}")
        _write(cache, dev, rng, slot, pos, hq, table, scale=[1.0, 6.0, 0.1, 40.0, 900.0][i % 5], pad_cols=8 * (i % 3),
               q_pad=8 * (i % 2))
        p += n


@pytest.mark.parametrize("hq,hkv,dh", [(4, 2, 64), (32, 8, 128), (5, 1, 128)])
@pytest.mark.parametrize("with_table", [True, False])
def test_write_of_many_sequences(hq, hkv, dh, with_table):
    """Decode rows, chunks that begin and continue, dead rows between them and behind them."""
    rng = np.random.default_rng(hq + dh + with_table)
    nb = 150
    cache = U.Cache(hkv, nb, dh)
    cache.fill(rng, np.arange(nb))
    order = iter(rng.permutation(nb))
    slot, pos = [], []
    for first, n in [(5, 1), (0, 1), (15, 1), (0, 16), (3, 13), (8, 30), (0, 57), (1, 1), (15, 2), (0, 200), (7, 1)]:
        p = np.arange(first, first + n)
        pages = np.array([next(order) for _ in range(p[-1] // 16 + 1)])
        slot += list(pages[p // 16] * 16 + p % 16)
        pos += list(p + 64)
        if n == 13:
            slot += [-1, nb * 16, 2 ** 31 - 1, -2 ** 31]
            pos += [1, 2, 3, 4]
    table = U.rope_table(300, dh) if with_table else None
    slot, pos = np.array(slot), np.array(pos)
    if with_table:
        pos[3], pos[-2] = -1, 300     # rows without a rotation are skipped, wherever they stand in a run
    dev = DevCache(cache)
    _write(cache, dev, rng, slot, pos, hq, table, scale=3.0)


@pytest.mark.parametrize("hq,hkv,dh", [(4, 2, 64), (8, 8, 128), (40, 8, 128)])
def test_write_of_decode_rows(hq, hkv, dh):
    """Many rows that each continue a page of their own, some of which must grow, between chunks and dead rows."""
    rng = np.random.default_rng(hq + hkv)
    nb = 130
    cache = U.Cache(hkv, nb, dh)
    cache.fill(rng, np.arange(nb), spread=8)
    dev = DevCache(cache)
    table = U.rope_table(50, dh)
    first = np.arange(100) % 16
    slot = rng.permutation(nb - 30)[:100] * 16 + first
    slot[rng.permutation(100)[:12]] = -1
    chunk = (nb - 30 + np.arange(3)) * 16
    slot = np.concatenate([slot[:37], chunk[0] + np.arange(5), slot[37:70], chunk[1] + np.arange(2), slot[70:],
                           chunk[2] + 9 + np.arange(7)])
    pos = rng.integers(0, 50, len(slot))
    for scale in (0.01, 1.0, 30.0):
        log(f"write decode rows {hq}/{hkv}x{dh} scale {scale}")
        _write(cache, dev, rng, slot, pos, hq, table, scale=scale)


@pytest.mark.parametrize("dh", [64, 128])
def test_write_values(dh):
    """Every rounding: all bf16 values near the codes and their midpoints, the ends of the range, subnormal codes,
    zeros of both signs, pages of zeros, tiny and huge pages, infinities and NaN."""
    rng = np.random.default_rng(dh)
    hkv, hq, nb = 2, 2, 40
    cache = U.Cache(hkv, nb, dh)
    dev = DevCache(cache)
    width = (hq + 2 * hkv) * dh
    for i in range(nb - 1):
        bits = rng.integers(0, 1 << 16, (16, width)).astype(np.uint16)
        x = U.f32_of(bits)
        top = [448.0, 449.0, 480.0, 1e-30, 1e-38, 3e38, 0.0, 1.0][i % 8]
        if i < 8:
            bits = np.where(np.abs(x) <= top, bits, bits & 0x8000)          # (NaN and infinity too)
        elif i < 24:
            # significands on and next to the midpoints of three-bit ones, exponents around the code's
            m = rng.choice([0, 7, 8, 9, 15, 16, 17, 24, 64, 120, 127], (16, width))
            e = rng.integers(127 - 12, 127 + 9, (16, width))
            bits = ((rng.integers(0, 2, (16, width)) << 15) | (e << 7) | m).astype(np.uint16)
        elif i < 32:
            bits = np.where(rng.random((16, width)) < 0.02, np.uint16(0x7F80 if i % 2 else 0xFFC0),
                            rand_bf16(rng, (16, width))[0])
        n = 16 if i % 3 else 9
        slot = i * 16 + np.arange(n)
        log(f"write values {i}")
        _write(cache, dev, rng, slot, slot, hq, None, bits=bits[:n].astype(np.uint16))
        if n == 9:                                                           # and the page's rest, at another size
            slot = i * 16 + np.arange(9, 16)
            _write(cache, dev, rng, slot, slot, hq, None, scale=2.0 ** rng.integers(-20, 20))


def _attention_case(rng, ctx, hq, hkv, dh, spare=5):
    """A cache with these contexts behind a permuted table: NaN past every context, unused pages and their scales
    NaN, table entries past the context out of range."""
    ctx = np.asarray(ctx)
    pages = -(-ctx // 16)
    nb = int(pages.sum()) + spare
    cache = U.Cache(hkv, nb, dh)
    order = rng.permutation(nb)
    stride = max(1, int(pages.max(initial=0)) + 2)
    bt = rng.choice([-1, nb, 2 ** 31 - 1, -2 ** 31], (len(ctx), stride))
    at = 0
    for s, n in enumerate(pages):
        bt[s, :n] = order[at:at + n]
        at += n
    cache.fill(rng, order[:at])
    for s, n in enumerate(ctx):
        if n % 16:
            cache.poison(bt[s, n // 16], n % 16)
    return cache, bt


def _decode(cache, bt, ctx, hq, rng, q_pad=0, o_pad=0, what="", ws_fill=0xFF, q_scale=1.0):
    t = torch()
    B, hkv, dh = len(ctx), cache.hkv, cache.dh
    dev = DevCache(cache)
    bits, _ = rand_bf16(rng, (B, hq * dh + q_pad), q_scale)
    if q_pad:
        bits[:, hq * dh:] = 0x7FC0
    qf = U.f32_of(bits)[:, :hq * dh].astype(np.float64).reshape(B, hq, dh)
    q, d_bt, d_ctx = dev_bits(bits), i32(bt), i32(ctx)
    out = dev_bits(np.full((B + 1, hq * dh + o_pad), 0x1234, np.uint16))
    n = hxf.op_decode_attention_kv8_workspace_bytes(B, hq, hkv, dh)
    ws = t.full((n,), ws_fill, dtype=t.uint8, device="cuda:0")
    log(f"decode kv8 {what}: B={B} {hq}/{hkv}x{dh} ctx max {int(np.max(ctx))}")
    hxf.op_decode_attention_kv8(q.data_ptr(), hq * dh + q_pad, dev.pool, d_bt.data_ptr(), bt.shape[1],
                                d_ctx.data_ptr(), out.data_ptr(), hq * dh + o_pad, B, hq, hkv, dh, ws.data_ptr(), n)
    t.cuda.synchronize()
    raw = out.cpu().numpy().view(np.uint16).reshape(B + 1, -1)
    assert np.all(raw[B] == 0x1234) and np.all(raw[:, hq * dh:] == 0x1234), what
    got = host_f64(out).reshape(B + 1, -1)[:B, :hq * dh].reshape(B, hq, dh)
    dev.check(what)
    for b in range(B):
        ref, size = U.attend(qf[b:b + 1], cache, bt[b], min(max(int(ctx[b]), 0), 16 * bt.shape[1]), hq)
        U.assert_attention(got[b:b + 1], ref, size, f"{what} sequence {b} (ctx {ctx[b]})")
    return raw


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_decode_lengths(hq, hkv, dh):
    rng = np.random.default_rng(hq + 10 * hkv + dh)
    for i, ctx in enumerate([[1], [0], [0, 5, 0, 33, 0], [15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65],
                             [127, 128, 129, 255, 256, 257, 258, 511, 513], [1000, 1, 2], [2500]]):
        cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
        _decode(cache, bt, np.array(ctx), hq, rng, q_pad=8 * (i % 3), o_pad=8 * (i % 2), what=f"lengths {i}")


@pytest.mark.parametrize("B,hi,heads", [(63, 300, (4, 2, 64)), (64, 200, (32, 8, 128)), (65, 500, (8, 8, 128)),
                                        (130, 90, (16, 1, 64)), (300, 40, (4, 2, 64)), (1100, 20, (2, 1, 64)),
                                        (2, 9000, (8, 1, 128)), (17, 3000, (4, 2, 64))])
def test_decode_batches(B, hi, heads):
    """Batches around the wavefront's width and beyond it, very uneven, some places empty."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(B + hi)
    ctx = np.rint(np.exp(rng.uniform(0, np.log(hi), B))).astype(np.int64)
    ctx[rng.random(B) < 0.1] = 0
    ctx[B // 2] = hi
    cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
    _decode(cache, bt, ctx, hq, rng, what="batch")


@pytest.mark.parametrize("B,hi,heads", [(10, 1300, (32, 8, 128)), (30, 1200, (14, 2, 64)), (300, 9000, (4, 2, 64)),
                                        (70, 12000, (16, 2, 128)), (1, 30000, (4, 2, 64)), (1, 30000, (13, 1, 128))])
def test_decode_joins_of_many_parts(B, hi, heads):
    """One context of many parts among short ones: a wavefront, a workgroup and a quarter of a head at a time."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(B + hi)
    ctx = rng.integers(1, 90, B)
    ctx[B // 3] = hi
    ctx[-1:] = hi // 2
    cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
    _decode(cache, bt, ctx, hq, rng, o_pad=8, what="joins")


def test_decode_entries_that_are_no_page():
    """Entries out of range inside a context are neither read nor weighted; a context of nothing else is empty; a
    context longer than the table's row, or negative, is cut."""
    rng = np.random.default_rng(3)
    ctx = [100, 600, 40, 33, 16]
    cache, bt = _attention_case(rng, ctx, 8, 2, 128)
    bt[0, 0], bt[0, 5], bt[0, 6] = -1, cache.nb, 2 ** 31 - 1
    bt[1, 10:30] = -7
    bt[2, :3] = [-1, cache.nb + 5, -2 ** 31]
    bt[3, 2] = -1
    _decode(cache, bt, np.array(ctx), 8, rng, what="bad entries")
    stride = bt.shape[1]
    bt[1, 38:] = bt[1, 0]
    ctx = np.array([100, 2 ** 31 - 1, -5, -2 ** 31, 16])
    cache.fill(rng, bt[1, 37:38])
    assert stride * 16 > 600
    _decode(cache, bt, ctx, 8, rng, what="cut contexts")


def test_decode_extreme_scores():
    """One key far above the others, large and tiny scales: no overflow, and the same result for any split."""
    rng = np.random.default_rng(4)
    for q_scale in (0.0, 2.0 ** -20, 6.0):
        cache, bt = _attention_case(rng, [700, 3], 8, 2, 128)
        cache.scale["k"][:] = np.minimum(cache.scale["k"], 2.0 ** -4)
        _decode(cache, bt, np.array([700, 3]), 8, rng, what=f"q {q_scale}", q_scale=q_scale)
    for s in (2.0 ** -50, 2.0 ** -66, 2.0 ** 60, 2.0 ** 110):
        cache, bt = _attention_case(rng, [90], 4, 1, 64)
        cache.scale["v"][:] *= s
        cache.scale["k"][:] *= 2.0 ** -40
        _decode(cache, bt, np.array([90]), 4, rng, what=f"v {s}")
        _prefill(cache, bt, np.array([70]), np.array([20]), 4, rng, what=f"v {s}")


def test_attention_over_pages_of_very_different_sizes():
    """Scales of V far apart in one context, pages of zeros (whose scale is the least there is) among them: zeros
    weigh in the denominator as any other value does."""
    rng = np.random.default_rng(41)
    for dh in (64, 128):
        cache, bt = _attention_case(rng, [400, 33], 4, 2, dh)
        for b in range(25):
            cache.scale["v"][:, bt[0, b]] = 2.0 ** [-6, -100, 3, -30, 10][b % 5]
            if b % 5 == 1:
                cache.codes["v"][:, bt[0, b]] = 0
        cache.scale["v"][:, bt[1, 0]] = 2.0 ** -100
        cache.codes["v"][:, bt[1, 0]] = 0
        _decode(cache, bt, np.array([400, 33]), 4, rng, what="sizes")
        _prefill(cache, bt, np.array([300, 0]), np.array([100, 33]), 4, rng, what="sizes")


def test_decode_offsets_beyond_32_bits():
    """A pool of more than 4 GiB per tensor, pages at its far end."""
    t = torch()
    rng = np.random.default_rng(5)
    hq, hkv, dh, nb = 4, 2, 128, (1 << 20) + 50_000
    small = U.Cache(hkv, 40, dh)
    small.fill(rng, np.arange(40))
    at = np.concatenate([np.arange(5), nb - 35 + np.arange(35)])
    k = t.full((hkv, nb, 16 * dh), 0x7F, dtype=t.uint8, device="cuda:0")
    v = t.full((hkv, nb, 16 * dh), 0x7F, dtype=t.uint8, device="cuda:0")
    ks = t.full((hkv, nb), float("nan"), device="cuda:0")
    vs = t.full((hkv, nb), float("nan"), device="cuda:0")
    ix = t.from_numpy(at).to("cuda:0")
    for kind, codes, scale in (("k", k, ks), ("v", v, vs)):
        codes[:, ix] = t.from_numpy(U.pack(small.codes[kind], kind)).to("cuda:0")
        scale[:, ix] = t.from_numpy(small.scale[kind]).to("cuda:0")
    pool = hxf.Kv8Pool(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), nb)
    order = rng.permutation(40)
    bits, qf = rand_bf16(rng, (1, hq, dh))
    q, bt, ctx, out = dev_bits(bits), i32(at[order][None]), i32([640]), dev_bits(np.zeros((1, hq, dh), np.uint16))
    n = hxf.op_decode_attention_kv8_workspace_bytes(1, hq, hkv, dh)
    ws = t.empty(n, dtype=t.uint8, device="cuda:0")
    hxf.op_decode_attention_kv8(q.data_ptr(), hq * dh, pool, bt.data_ptr(), 40, ctx.data_ptr(), out.data_ptr(),
                                hq * dh, 1, hq, hkv, dh, ws.data_ptr(), n)
    n = hxf.op_prefill_attention_kv8_workspace_bytes(1, 1, hq, hkv, dh)
    ws2, row0, pos0 = t.empty(n, dtype=t.uint8, device="cuda:0"), i32([0, 1]), i32([639])
    out2 = dev_bits(np.zeros((1, hq, dh), np.uint16))
    hxf.op_prefill_attention_kv8(q.data_ptr(), hq * dh, pool, bt.data_ptr(), 40, row0.data_ptr(), pos0.data_ptr(),
                                 out2.data_ptr(), hq * dh, 1, 1, hq, hkv, dh, ws2.data_ptr(), n)
    t.cuda.synchronize()
    ref, size = U.attend(qf, small, order, 640, hq)
    U.assert_attention(host_f64(out).reshape(1, hq, dh), ref, size, "decode")
    U.assert_attention(host_f64(out2).reshape(1, hq, dh), ref, size, "prefill")


def _prefill(cache, bt, pos0, n, hq, rng, pad=0, lead=0, q_pad=0, o_pad=0, what="", row0=None):
    """lead: rows before the first sequence; pad: rows behind the last one."""
    t = torch()
    S, hkv, dh = len(n), cache.hkv, cache.dh
    dev = DevCache(cache)
    if row0 is None:
        row0 = lead + np.concatenate([[0], np.cumsum(n)])
    T = int(max(row0)) + pad
    bits, _ = rand_bf16(rng, (T, hq * dh + q_pad))
    qf = U.f32_of(bits)[:, :hq * dh].astype(np.float64).reshape(T, hq, dh)
    q, d_bt, d_row0, d_pos0 = dev_bits(bits), i32(bt), i32(row0), i32(pos0)
    out = dev_bits(np.full((T + 1, hq * dh + o_pad), 0x1234, np.uint16))
    m = hxf.op_prefill_attention_kv8_workspace_bytes(S, T, hq, hkv, dh)
    ws = t.full((m,), 0xFF, dtype=t.uint8, device="cuda:0")
    log(f"prefill kv8 {what}: S={S} T={T} {hq}/{hkv}x{dh}")
    hxf.op_prefill_attention_kv8(q.data_ptr(), hq * dh + q_pad, dev.pool, d_bt.data_ptr(), bt.shape[1],
                                 d_row0.data_ptr(), d_pos0.data_ptr(), out.data_ptr(), hq * dh + o_pad, S, T, hq, hkv,
                                 dh, ws.data_ptr(), m)
    t.cuda.synchronize()
    raw = out.cpu().numpy().view(np.uint16).reshape(T + 1, -1)
    assert np.all(raw[:, hq * dh:] == 0x1234), what
    got = host_f64(out).reshape(T + 1, -1)[:T, :hq * dh].reshape(T, hq, dh)
    dev.check(what)
    seen = np.zeros(T + 1, bool)
    for s in range(S):
        r = slice(int(row0[s]), int(row0[s]) + int(n[s]))
        seen[r] = True
        ref, size = U.attend(qf[r], cache, bt[s], min(int(pos0[s] + n[s]), 16 * bt.shape[1]), hq, first=int(pos0[s]))
        U.assert_attention(got[r], ref, size, f"{what} sequence {s} (pos {pos0[s]}, {n[s]} rows)")
    assert np.all(raw[~seen] == 0x1234), f"{what}: rows of no sequence"
    return raw


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_prefill_lengths(hq, hkv, dh):
    rng = np.random.default_rng(hq + 10 * hkv + dh)
    for i, (pos0, n) in enumerate([([0], [1]), ([0], [37]), ([5, 0, 16, 31], [1, 0, 33, 1]), ([100, 15], [70, 17]),
                                   ([0, 300, 7], [129, 2, 0]), ([1000], [3]), ([2300], [40]), ([0], [257]),
                                   ([31, 32, 33, 47], [32, 31, 33, 17])]):
        cache, bt = _attention_case(rng, np.add(pos0, n), hq, hkv, dh)
        _prefill(cache, bt, np.array(pos0), np.array(n), hq, rng, pad=3 * (i % 2), lead=2 * (i % 3), q_pad=8 * (i % 2),
                 o_pad=8 * (i % 3), what=f"lengths {i}")


@pytest.mark.parametrize("S,hi_pos,hi_n,heads", [(33, 200, 20, (4, 2, 64)), (70, 60, 9, (32, 8, 128)),
                                                 (8, 700, 300, (8, 2, 128)), (300, 33, 3, (2, 1, 64)),
                                                 (2, 3000, 400, (10, 2, 128)), (1100, 9, 2, (4, 2, 64))])
def test_prefill_batches(S, hi_pos, hi_n, heads):
    hq, hkv, dh = heads
    rng = np.random.default_rng(S + hi_pos)
    pos0, n = rng.integers(0, hi_pos + 1, S), rng.integers(0, hi_n + 1, S)
    n[S // 2] = hi_n
    cache, bt = _attention_case(rng, pos0 + n, hq, hkv, dh)
    _prefill(cache, bt, pos0, n, hq, rng, pad=5, what="batch")


def test_prefill_few_chunks_among_many_places():
    """A batch of more than 1024 places of which few have queries, whose long contexts are cut."""
    rng = np.random.default_rng(15)
    S = 2300
    n, pos0 = np.zeros(S, np.int64), np.zeros(S, np.int64)
    for s, p, m in ((3, 900, 5), (1027, 1500, 2), (1028, 0, 40), (2051, 64, 1), (2299, 700, 33)):
        pos0[s], n[s] = p, m
    cache, bt = _attention_case(rng, pos0 + n, 4, 2, 64)
    _prefill(cache, bt, pos0, n, 4, rng, pad=2, what="places")


def test_prefill_entries_that_are_no_page():
    rng = np.random.default_rng(13)
    pos0, n = np.array([80, 0, 300, 0]), np.array([40, 33, 9, 16])
    cache, bt = _attention_case(rng, pos0 + n, 8, 2, 128)
    bt[0, 2], bt[0, 3], bt[0, 4] = -1, cache.nb, -2 ** 31
    bt[1, 1] = 2 ** 31 - 1
    bt[2, :12] = -1
    bt[3, 0] = -3                       # a sequence none of whose keys is there
    raw = _prefill(cache, bt, pos0, n, 8, rng, what="bad entries")
    assert np.all(raw[82:98] == 0)


def test_prefill_rows_past_the_table_and_row0_out_of_range():
    """Positions past the table's row see the keys it holds; row0 beyond T counts as T."""
    t = torch()
    rng = np.random.default_rng(14)
    cache, bt = _attention_case(rng, [64, 40], 4, 2, 64)
    bt = bt[:, :4].copy()
    cache.fill(rng, bt[0])
    _prefill(cache, bt, np.array([50, 30]), np.array([30, 10]), 4, rng, what="past the table")
    dev = DevCache(cache)
    bits, qf = rand_bf16(rng, (20, 4, 64))
    q, d_bt, row0, pos0 = dev_bits(bits), i32(bt), i32([0, 12, 50]), i32([20, 12])
    out = dev_bits(np.full((24, 4, 64), 0x1234, np.uint16))
    m = hxf.op_prefill_attention_kv8_workspace_bytes(2, 20, 4, 2, 64)
    ws = t.empty(m, dtype=t.uint8, device="cuda:0")
    hxf.op_prefill_attention_kv8(q.data_ptr(), 256, dev.pool, d_bt.data_ptr(), 4, row0.data_ptr(), pos0.data_ptr(),
                                 out.data_ptr(), 256, 2, 20, 4, 2, 64, ws.data_ptr(), m)
    t.cuda.synchronize()
    got = host_f64(out).reshape(24, 4, 64)
    for r, s, p in ((slice(0, 12), 0, 20), (slice(12, 20), 1, 12)):
        ref, size = U.attend(qf[r], cache, bt[s], p + r.stop - r.start, 4, first=p)
        U.assert_attention(got[r], ref, size, f"sequence {s}")
    assert np.all(out.cpu().numpy().view(np.uint16).reshape(24, -1)[20:] == 0x1234)


@pytest.mark.parametrize("heads,n,hi_pos,places", [
    ((32, 8, 128), [300, 250, 200, 150, 40, 33, 17, 1], 2500, 0), ((32, 8, 128), [300, 250, 200, 150, 40, 33, 17, 1], 2500, 300),
    ((16, 1, 64), [700, 450, 200, 9], 2000, 0), ((16, 1, 64), [700, 450, 200, 9], 2000, 280), ((8, 2, 64), [1, 1, 130, 1], 9000, 0),
    ((40, 8, 128), [64, 200, 256, 7, 90], 1200, 0), ((6, 6, 64), [129, 300, 20], 4000, 0)])
def test_prefill_blocks_dealt_out_in_shares(heads, n, hi_pos, places):
    """Blocks of very different lengths, cut where the workgroups' shares end, more pieces than are resident at once;
    places: empty ones among them, for the batches that a launch of its own plans."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(hi_pos + places)
    n, pos0 = np.array(n + [0] * places), rng.integers(0, hi_pos, len(n) + places)
    pos0[:3] = hi_pos, 5, hi_pos // 2
    order = rng.permutation(len(n))
    n, pos0 = n[order], pos0[order]
    pos0[n == 0] = 0
    cache, bt = _attention_case(rng, pos0 + n, hq, hkv, dh)
    _prefill(cache, bt, pos0, n, hq, rng, pad=3, what="shares")


def test_prefill_of_a_very_wide_table():
    """2^25 entries a sequence: the work split counts in coarser units."""
    rng = np.random.default_rng(21)
    pos0, n = np.array([4000]), np.array([45])
    cache, bt = _attention_case(rng, pos0 + n, 8, 2, 128)
    wide = np.full((1, 1 << 25), -1, np.int32)
    wide[:, :bt.shape[1]] = bt
    _prefill(cache, wide, pos0, n, 8, rng, what="wide table")


@pytest.mark.parametrize("S,T", [(10, 256), (401, 256), (3, 64)])
def test_prefill_row0_that_does_not_ascend_stays_in_its_buffers(S, T):
    """More rows than T in all, over contexts long enough to be cut: nothing is written past the workspace or out."""
    t = torch()
    rng = np.random.default_rng(S)
    cache, bt = _attention_case(rng, [2500] * 2, 16, 1, 64)
    bt = bt[np.arange(S) % 2]
    dev = DevCache(cache)
    row0 = np.zeros(S + 1, np.int64)
    row0[1:10:2] = T
    q, d_bt, d_row0, pos0 = dev_bits(rand_bf16(rng, (T, 1024))[0]), i32(bt), i32(row0), i32(np.full(S, 2200))
    out = dev_bits(np.full((T + 8, 1024), 0x1234, np.uint16))
    m = hxf.op_prefill_attention_kv8_workspace_bytes(S, T, 16, 1, 64)
    ws = t.full((m + (16 << 20),), 0x5A, dtype=t.uint8, device="cuda:0")
    log(f"prefill kv8 row0 that does not ascend: S={S} T={T}")
    hxf.op_prefill_attention_kv8(q.data_ptr(), 1024, dev.pool, d_bt.data_ptr(), bt.shape[1], d_row0.data_ptr(),
                                 pos0.data_ptr(), out.data_ptr(), 1024, S, T, 16, 1, 64, ws.data_ptr(), m)
    t.cuda.synchronize()
    assert bool((ws[m:] == 0x5A).all())
    assert np.all(out.cpu().numpy().view(np.uint16)[T:] == 0x1234)


def _outputs(cache, bt, pos0, n, hq, rng, decode):
    """q float64 and outputs of prefill, or of decode (n 1 everywhere), nothing checked."""
    t = torch()
    S, T, hkv, dh = len(n), int(np.sum(n)), cache.hkv, cache.dh
    dev = DevCache(cache)
    bits, _ = rand_bf16(rng, (T, hq * dh))
    q, out, d_bt = dev_bits(bits), dev_bits(np.zeros((T, hq * dh), np.uint16)), i32(bt)
    row0, d_pos0, ctx = i32(np.concatenate([[0], np.cumsum(n)])), i32(pos0), i32(np.add(pos0, n))
    m = (hxf.op_decode_attention_kv8_workspace_bytes(S, hq, hkv, dh) if decode else
         hxf.op_prefill_attention_kv8_workspace_bytes(S, T, hq, hkv, dh))
    ws = t.full((m,), 0xFF, dtype=t.uint8, device="cuda:0")
    log(f"values that are not finite: {'decode' if decode else 'prefill'} S={S} T={T} {hq}/{hkv}x{dh}")
    if decode:
        hxf.op_decode_attention_kv8(q.data_ptr(), hq * dh, dev.pool, d_bt.data_ptr(), bt.shape[1], ctx.data_ptr(),
                                    out.data_ptr(), hq * dh, S, hq, hkv, dh, ws.data_ptr(), m)
    else:
        hxf.op_prefill_attention_kv8(q.data_ptr(), hq * dh, dev.pool, d_bt.data_ptr(), bt.shape[1], row0.data_ptr(),
                                     d_pos0.data_ptr(), out.data_ptr(), hq * dh, S, T, hq, hkv, dh, ws.data_ptr(), m)
    t.cuda.synchronize()
    return U.f32_of(bits).astype(np.float64).reshape(T, hq, dh), host_f64(out).reshape(T, hq, dh)


@pytest.mark.parametrize("hq,hkv,dh", [(8, 2, 128), (4, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("decode", [False, True])
def test_nan_in_the_cache_reaches_the_queries_that_see_it(hq, hkv, dh, decode):
    """NaN of V in some dimensions of some places, and one NaN of K: exactly the outputs whose sums hold them are NaN,
    those of earlier queries of the same block are not."""
    rng = np.random.default_rng(hq + dh)
    pos0, n = np.array([100, 0, 2000, 40, 7, 0]), np.array([70, 45, 40, 1, 3, 5])
    if decode:
        pos0, n = pos0 + n - 1, np.ones(6, np.int64)
    cache, bt = _attention_case(rng, pos0 + n, hq, hkv, dh)
    clean = copy.deepcopy(cache)
    v_nan, k_nan = [], []       # (sequence, position, head, dimension or None)
    for s, p, d in ((0, 104, 3), (0, 120, dh - 1), (0, 169, 17), (1, 0, 0), (1, 31, 33), (1, 44, 2), (2, 5, 40), (2, 2001, 41),
                    (2, 2017, 42), (2, 2039, 43), (4, 9, 1)):
        h = (p + d) % hkv
        cache.codes["v"][h, bt[s, p // 16], p % 16, d] = 0x7F if p % 2 else 0xFF
        v_nan.append((s, p, h, d))
    for s, p, h in ((0, 150, 0), (1, 20, 1)):
        cache.codes["k"][h, bt[s, p // 16], p % 16, 5] = 0x7F
        k_nan.append((s, p, h))
    q, got = _outputs(cache, bt, pos0, n, hq, rng, decode)
    G, r0 = hq // hkv, 0
    for s in range(len(n)):
        r = slice(r0, r0 + n[s])
        ref, size = U.attend(q[r], clean, bt[s], int(pos0[s] + n[s]), hq, first=int(pos0[s]))
        nan = np.zeros(ref.shape, bool)
        for j, p, h, d in v_nan:
            if j == s:
                nan[max(p - pos0[s], 0):, h * G:(h + 1) * G, d] = True
        for j, p, h in k_nan:
            if j == s:
                nan[max(p - pos0[s], 0):, h * G:(h + 1) * G] = True
        what = f"sequence {s}"
        assert np.array_equal(np.isnan(got[r]), nan), what
        U.assert_attention(np.where(nan, 0, got[r]), np.where(nan, 0, ref), size, what)
        r0 += n[s]


def test_prefill_long_blocks_that_are_not_cut():
    """More blocks than CUs, each over many tables of 64 pages."""
    rng = np.random.default_rng(16)
    pos0, n = np.array([1500, 2100, 0, 1023]), np.array([300, 257, 320, 290])
    cache, bt = _attention_case(rng, pos0 + n, 32, 8, 128)
    _prefill(cache, bt, pos0, n, 32, rng, what="not cut")


def test_attention_repeats_to_the_bit():
    """The order in which work is taken up does not show in the result, whatever the workspace held before."""
    for hq, hkv, dh, ctx in ((8, 2, 128, [2000, 3, 0, 700]), (4, 2, 64, list(range(1, 150)))):
        raw = []
        for fill in (0xFF, 0, 0x7F):
            rng = np.random.default_rng(21)
            cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
            raw.append(_decode(cache, bt, np.array(ctx), hq, rng, what="again", ws_fill=fill))
        assert all(np.array_equal(r, raw[0]) for r in raw)
    raw = []
    for _ in range(3):
        rng = np.random.default_rng(22)
        pos0, n = rng.integers(0, 200, 60), rng.integers(0, 20, 60)
        cache, bt = _attention_case(rng, pos0 + n, 32, 8, 128)
        raw.append(_prefill(cache, bt, pos0, n, 32, rng, what="again"))
    assert all(np.array_equal(r, raw[0]) for r in raw)


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own, do not disturb each other."""
    t = torch()
    hq, hkv, dh = 8, 2, 128
    sides = []
    for seed in (31, 32):
        rng = np.random.default_rng(seed)
        ctx = rng.integers(1, 1500, 40)
        cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
        bits, qf = rand_bf16(rng, (40, hq, dh))
        n = hxf.op_decode_attention_kv8_workspace_bytes(40, hq, hkv, dh)
        m = hxf.op_prefill_attention_kv8_workspace_bytes(40, 40, hq, hkv, dh)
        sides.append(dict(ctx=ctx, cache=cache, bt=bt, qf=qf, dev=DevCache(cache), q=dev_bits(bits), d_bt=i32(bt),
                          d_ctx=i32(ctx), row0=i32(np.arange(41)), pos0=i32(ctx - 1), ws=t.empty(n, dtype=t.uint8, device="cuda:0"),
                          ws2=t.empty(m, dtype=t.uint8, device="cuda:0"), out=dev_bits(np.zeros((40, hq, dh), np.uint16)),
                          out2=dev_bits(np.zeros((40, hq, dh), np.uint16)), st=t.cuda.Stream()))
    t.cuda.synchronize()
    log("two streams")
    for _ in range(20):
        for s in sides:
            hxf.op_decode_attention_kv8(s["q"].data_ptr(), hq * dh, s["dev"].pool, s["d_bt"].data_ptr(),
                                        s["bt"].shape[1], s["d_ctx"].data_ptr(), s["out"].data_ptr(), hq * dh, 40, hq,
                                        hkv, dh, s["ws"].data_ptr(), s["ws"].numel(), stream=s["st"].cuda_stream)
            hxf.op_prefill_attention_kv8(s["q"].data_ptr(), hq * dh, s["dev"].pool, s["d_bt"].data_ptr(),
                                         s["bt"].shape[1], s["row0"].data_ptr(), s["pos0"].data_ptr(),
                                         s["out2"].data_ptr(), hq * dh, 40, 40, hq, hkv, dh, s["ws2"].data_ptr(),
                                         s["ws2"].numel(), stream=s["st"].cuda_stream)
    t.cuda.synchronize()
    for s in sides:
        for b in range(40):
            ref, size = U.attend(s["qf"][b:b + 1], s["cache"], s["bt"][b], int(s["ctx"][b]), hq)
            for o in ("out", "out2"):
                U.assert_attention(host_f64(s[o]).reshape(40, hq, dh)[b:b + 1], ref, size, f"{o} {b}")


@pytest.mark.parametrize("hq,hkv,dh", [(4, 2, 64), (16, 2, 128)])
def test_a_captured_step_of_all_operators(hq, hkv, dh):
    """The operators as a serving loop runs them, in one captured graph that is replayed with other lengths: tables,
    rotation and write, attention of the decode rows and of the chunks (both through one workspace).  Every
    replay is checked against the model and against the same calls made eagerly on a second cache."""
    t = torch()
    rng = np.random.default_rng(hq)
    D, P, T, stride, nb, max_pos = 5, 4, 120, 12, 160, 200
    S = D + P
    width = (hq + 2 * hkv) * dh
    table = U.rope_table(max_pos, dh)
    cache = U.Cache(hkv, nb, dh)
    order = list(rng.permutation(nb))
    start = np.concatenate([rng.integers(1, 60, D), np.zeros(P, np.int64)])
    bt = np.full((S, stride), -1, np.int64)
    for s in range(D):                                    # the decode sequences' prompts are in the cache already
        for p in range(-(-start[s] // 16)):
            bt[s, p] = order.pop()
        cache.fill(rng, bt[s, :-(-start[s] // 16)])
        if start[s] % 16:
            cache.poison(bt[s, start[s] // 16], start[s] % 16)

    def side():
        z = lambda *n: t.zeros(n, dtype=t.int32, device="cuda:0")
        ws = max(hxf.op_decode_attention_kv8_workspace_bytes(D, hq, hkv, dh),
                 hxf.op_prefill_attention_kv8_workspace_bytes(P, T, hq, hkv, dh))
        return dict(dev=DevCache(cache), bt=i32(bt), start=z(S), new=z(S), free=z(64), n_free=z(1), row0=z(S + 1), pos=z(T),
                    slot=z(T), ctx=z(S), status=z(2), qkv=t.zeros(T * width, dtype=t.int16, device="cuda:0"),
                    q=t.zeros(T * hq * dh, dtype=t.int16, device="cuda:0"),
                    out=t.zeros(T * hq * dh, dtype=t.int16, device="cuda:0"), ws=t.zeros(ws, dtype=t.uint8, device="cuda:0"),
                    table=t.from_numpy(table).to("cuda:0"))

    def step(s, stream):
        p = lambda k, at=0: s[k].data_ptr() + at
        hxf.op_slot_map(p("start"), p("new"), S, p("free"), p("n_free"), 64, p("bt"), stride, p("row0"), p("pos"),
                        p("slot"), T, p("ctx"), p("status"), stream=stream)
        hxf.op_rope_kv8_write(p("qkv"), width, p("pos"), p("slot"), p("table"), max_pos, p("q"), hq * dh, s["dev"].pool,
                              T, hq, hkv, dh, stream=stream)
        hxf.op_decode_attention_kv8(p("q"), hq * dh, s["dev"].pool, p("bt"), stride, p("ctx"), p("out"), hq * dh, D, hq,
                                    hkv, dh, p("ws"), s["ws"].numel(), stream=stream)
        hxf.op_prefill_attention_kv8(p("q"), hq * dh, s["dev"].pool, p("bt", 4 * D * stride), stride, p("row0", 4 * D),
                                     p("start", 4 * D), p("out"), hq * dh, P, T, hq, hkv, dh, p("ws"), s["ws"].numel(),
                                     stream=stream)

    cap, eager = side(), side()
    cap["n_free"].fill_(64)
    st = t.cuda.Stream()
    with t.cuda.stream(st):
        step(cap, st.cuda_stream)                          # lengths of zero: nothing is written
        st.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph, stream=st):
            step(cap, t.cuda.current_stream().cuda_stream)
    t.cuda.synchronize()
    cap["dev"].check("before the first replay")
    for it in range(7):
        new = np.concatenate([np.ones(D, np.int64), rng.integers(0, 28, P)])
        if it == 2:
            new[D:] = 0
        if it == 4:
            new[D] = 200                                   # more rows than the batch holds: nothing may happen
        free = [order.pop() for _ in range(24)]
        bits, _ = rand_bf16(rng, (T, width), [1.0, 3.0, 0.2][it % 3])
        for s in (cap, eager):
            for k, a in (("start", start), ("new", new), ("n_free", [len(free)])):
                s[k].copy_(i32(a))
            s["free"][:len(free)].copy_(i32(free))
            s["qkv"].copy_(dev_bits(bits).view(-1))
            s["out"].fill_(0x1234)
        t.cuda.synchronize()
        log(f"replay {it}: new {new.tolist()}")
        graph.replay()
        step(eager, 0)
        t.cuda.synchronize()
        bt, row0, pos, slot, ctx, status = U.slot_map(start, new, free, bt, T)
        for k, r in (("bt", bt), ("row0", row0), ("pos", pos), ("slot", slot), ("ctx", ctx), ("status", status)):
            for s in (cap, eager):
                np.testing.assert_array_equal(s[k].cpu().numpy().reshape(r.shape), r, err_msg=f"replay {it}: {k}")
        order = free[max(0, status[0]):] + order            # what was not taken goes back
        x = U.f32_of(bits).reshape(T, hq + 2 * hkv, dh)
        qk = U.rotate(x[:, :hq + hkv], table[pos])
        cache.write(qk[:, hq:], x[:, hq + hkv:], slot)
        for s in (cap, eager):
            s["dev"].check(f"replay {it}")
        assert t.equal(cap["out"], eager["out"]) and t.equal(cap["q"], eager["q"])
        got = host_f64(cap["out"]).reshape(T, hq, dh)
        qf = host_f64(cap["q"]).reshape(T, hq, dh)
        live = np.zeros(T, bool)
        for s in range(S):
            rows = slice(s, s + 1) if s < D else slice(row0[s], row0[s + 1])
            live[rows] = True
            if status[0] < 0 and s >= D:
                continue
            ref, size = U.attend(qf[rows], cache, bt[s], int(ctx[s]), hq, first=None if s < D else int(start[s]))
            U.assert_attention(got[rows], ref, size, f"replay {it} sequence {s}")
        raw = cap["out"].cpu().numpy().reshape(T, -1)
        assert np.all(raw[~live] == 0x1234)
        start = ctx


@pytest.mark.parametrize("spread", [122, -91])
@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("heads,ctx", [((8, 2, 128), [700, 3]), ((4, 2, 64), [3000, 40]), ((13, 1, 128), [30000]),
                                       ((32, 8, 128), [1300, 20, 8, 500, 1, 16, 17, 90, 30, 1200])])
def test_decode_of_the_largest_and_smallest_values_in_many_parts(heads, ctx, flat, spread):
    """V scales up to 2^119 and down to 2^-100 in contexts that are cut, by each of the joins: the sums of a part may be far
    larger than any value.  flat: all weights alike, so that they are largest."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(sum(ctx) + flat)
    cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
    cache.scale["v"][:] *= 2.0 ** spread
    if flat:
        cache.scale["k"][:] *= 2.0 ** -40
    _decode(cache, bt, np.array(ctx), hq, rng, what=f"v 2^{spread}")


@pytest.mark.parametrize("spread", [122, -91])
@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("heads,places", [((8, 2, 128), 0), ((4, 2, 64), 300), ((32, 8, 128), 300)])
def test_prefill_of_the_largest_and_smallest_values_in_many_parts(heads, places, flat, spread):
    """The same for blocks that are cut, planned by the workgroups and by a launch."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(hq + places + flat)
    pos0, n = np.array([700, 2900, 60] + [0] * places), np.array([20, 60, 9] + [0] * places)
    cache, bt = _attention_case(rng, pos0 + n, hq, hkv, dh)
    cache.scale["v"][:] *= 2.0 ** spread
    if flat:
        cache.scale["k"][:] *= 2.0 ** -40
    _prefill(cache, bt, pos0, n, hq, rng, what=f"v 2^{spread}")


@pytest.mark.parametrize("hq,hkv,dh", [(8, 2, 128), (4, 2, 64)])
def test_pages_whose_scale_is_zero(hq, hkv, dh):
    """A page whose stored scale is 0 (a pool that began as zeros) holds zeros: its keys score 0 and have their weight, its
    values add nothing.  Only an entry that is no page has no weight."""
    rng = np.random.default_rng(dh + 7)
    ctx = np.array([1300, 16, 40, 33])
    cache, bt = _attention_case(rng, ctx, hq, hkv, dh)
    for s, p, kinds in ((0, 0, "k"), (0, 3, "kv"), (0, 64, "k"), (0, 70, "v"), (0, 81, "k"), (1, 0, "k"), (2, 1, "k"),
                        (2, 2, "v"), (3, 0, "v"), (3, 1, "v"), (3, 2, "kv")):
        for kind in kinds:
            cache.scale[kind][:, bt[s, p]] = 0
    bt[0, 5], bt[2, 0] = -1, cache.nb
    _decode(cache, bt, ctx, hq, rng, what="scales of 0")
    _prefill(cache, bt, ctx - np.array([30, 16, 17, 1]), np.array([30, 16, 17, 1]), hq, rng, what="scales of 0")


@pytest.mark.parametrize("S,hi_pos,hi_n,heads", [(300, 200, 20, (32, 8, 128)), (300, 2500, 2, (4, 2, 64)),
                                                 (2, 900, 4300, (32, 8, 128))])
def test_prefill_planned_by_a_launch_repeats_to_the_bit(S, hi_pos, hi_n, heads):
    """The planning launch lists units in an order that atomics make: it does not show in the result."""
    hq, hkv, dh = heads
    rng = np.random.default_rng(S + hi_n)
    pos0, n = rng.integers(0, hi_pos + 1, S), rng.integers(0, hi_n + 1, S)
    pos0[0], n[0] = hi_pos, hi_n
    if hi_n == 2:
        pos0[5:], n[5:] = 0, 0                          # few queries over long contexts: cut
    cache, bt = _attention_case(rng, pos0 + n, hq, hkv, dh)
    out = [_outputs(cache, bt, pos0, n, hq, np.random.default_rng(5), False)[1] for _ in range(4)]
    assert all(np.array_equal(o, out[0]) for o in out)


@pytest.mark.parametrize("hi_ctx", [100, 2500])
def test_prefill_planned_blocks_of_a_row0_that_goes_up_and_down_are_bounded(hi_ctx):
    """A thousand sequences that each claim all rows: the planning launch takes no more blocks than it has units for,
    nothing is written past the workspace or out, and the next call on the same workspace is right."""
    t = torch()
    rng = np.random.default_rng(hi_ctx)
    S, T, heads = 2000, 2048, (16, 1, 64)
    cache, bt = _attention_case(rng, [hi_ctx] * 2, *heads)
    bt = bt[np.arange(S) % 2]
    dev = DevCache(cache)
    bits, qf = rand_bf16(rng, (T, 16, 64))
    q, d_bt, pos0 = dev_bits(bits), i32(bt), i32(np.full(S, hi_ctx - 90))
    out = dev_bits(np.full((T + 8, 1024), 0x1234, np.uint16))
    m = hxf.op_prefill_attention_kv8_workspace_bytes(S, T, *heads)
    ws = t.full((m + (16 << 20),), 0x5A, dtype=t.uint8, device="cuda:0")
    up_down, up = np.arange(S + 1) % 2 * T, np.minimum(np.arange(S + 1), 90)
    for row0 in (up_down, up):
        d_row0 = i32(row0)
        log(f"prefill kv8 row0 up and down: S={S} T={T} rows {row0[:3].tolist()}")
        hxf.op_prefill_attention_kv8(q.data_ptr(), 1024, dev.pool, d_bt.data_ptr(), bt.shape[1], d_row0.data_ptr(),
                                     pos0.data_ptr(), out.data_ptr(), 1024, S, T, *heads, ws.data_ptr(), m)
        t.cuda.synchronize()
    assert bool((ws[m:] == 0x5A).all())
    assert np.all(out.cpu().numpy().view(np.uint16)[T:] == 0x1234)
    got = host_f64(out).reshape(-1, 16, 64)
    for s in (0, 1, 57, 89):
        ref, size = U.attend(qf[s:s + 1], cache, bt[s], hi_ctx - 89, 16, first=hi_ctx - 90)
        U.assert_attention(got[s:s + 1], ref, size, f"sequence {s}")


@pytest.mark.parametrize("hq,hkv,dh", [(2, 1, 64), (4, 2, 128)])
def test_scores_far_beyond_the_steps_of_their_references(hq, hkv, dh):
    """Scores of 2^16 to 2^28, where fp32 counts in steps of up to 16, that climb by a few such steps from key to key: no
    weight may pass fp16.  Every value of V is 1, and so is every average of them."""
    t = torch()
    n_keys, rows = 700, 3
    cases = [(e, m, s) for e in range(16, 29) for m in (1.0, 1.25, 1.6875) for s in (1, 2, 3)]
    S = len(cases)
    pages = -(-n_keys // 16)
    cache = U.Cache(hkv, S * pages, dh)
    cache.codes["k"][:], cache.codes["v"][:] = 0, U.encode(256.0)
    cache.scale["k"][:], cache.scale["v"][:] = 1, 2.0 ** -8
    q = np.zeros((S, dh), np.float32)
    log2_unit = 1.4426950408889634 / np.sqrt(dh)
    for i, (e, m, s) in enumerate(cases):
        at = slice(i * pages, (i + 1) * pages)
        # dimension 0 makes the size, 256 q0; dimension 1 climbs, by s steps of its fp32 products in 16 keys, from 0 to 240
        q[i, 0] = m * 2.0 ** (e - 8) / log2_unit
        q[i, 1] = s * 2.0 ** (e - 24) / log2_unit
        cache.codes["k"][:, at, :, 0] = U.encode(256.0)
        climb = np.minimum(np.arange(pages * 16) // 16 + 1, 15).reshape(pages, 16) * 1.0
        cache.codes["k"][:, at, :, 1] = U.encode(climb)
    bits = synth.f32_to_bf16_bits(np.repeat(q[:, None], hq, 1).reshape(S, hq, dh)).reshape(S, hq * dh)
    dev = DevCache(cache)
    bt = i32(np.arange(S * pages).reshape(S, pages))
    ctx, dq, out = i32(np.full(S, n_keys)), dev_bits(bits), dev_bits(np.zeros((S, hq * dh), np.uint16))
    ws = t.empty(hxf.op_decode_attention_kv8_workspace_bytes(S, hq, hkv, dh), dtype=t.uint8, device="cuda:0")
    log(f"scores far beyond: {hq}/{hkv}x{dh}")
    hxf.op_decode_attention_kv8(dq.data_ptr(), hq * dh, dev.pool, bt.data_ptr(), pages, ctx.data_ptr(), out.data_ptr(),
                                hq * dh, S, hq, hkv, dh, ws.data_ptr(), ws.numel())
    T = S * rows
    dq2, out2 = dev_bits(np.repeat(bits, rows, 0)), dev_bits(np.zeros((T, hq * dh), np.uint16))
    row0, pos0 = i32(np.arange(S + 1) * rows), i32(np.full(S, n_keys - rows))
    ws2 = t.empty(hxf.op_prefill_attention_kv8_workspace_bytes(S, T, hq, hkv, dh), dtype=t.uint8, device="cuda:0")
    hxf.op_prefill_attention_kv8(dq2.data_ptr(), hq * dh, dev.pool, bt.data_ptr(), pages, row0.data_ptr(),
                                 pos0.data_ptr(), out2.data_ptr(), hq * dh, S, T, hq, hkv, dh, ws2.data_ptr(), ws2.numel())
    t.cuda.synchronize()
    for what, o in (("decode", out), ("prefill", out2)):
        got = host_f64(o).reshape(S, -1)
        # the weights' roundings to fp16 (2^-11) and the output's to bf16 (2^-8)
        bad = [cases[i] for i in range(S) if not np.all(np.abs(got[i] - 1) <= 2.0 ** -8 + 2.0 ** -10)]
        assert not bad, (what, bad)
