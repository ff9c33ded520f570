"""The operators of the 8-bit paged KV cache, as cases that can be timed and compared.

The cache holds K and V in e4m3, in pages of 16 tokens, with one power-of-two scale for each (kv-head,
page) of each pool.  Four operators work on it, all with the lengths in device memory:

* ``slot_map``: block tables, token slots and positions from the requests' lengths and a list of free pages;
* ``write``: RoPE of q and k, and the quantised write of k and v into their pages;
* ``decode``: attention of one query per sequence over the cache;
* ``prefill``: causal attention of prompt chunks over the cache.

With ``own`` false a case runs in plain torch operations, in 32 bits, rounded once at the end; with ``own``
true it makes the calls of ``paper_2505_05286_amd.hxf``.

Layouts of one page (16 tokens) of one kv-head, in bytes: K ``[dh/16][16 tokens][16 dims]``, V
``[4][dh][4 tokens]`` (token ``4 g + j`` of dimension ``d`` at ``(g * dh + d) * 4 + j``).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16
ROPE_BASE = 10000.0
HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "32b": (40, 8, 128), "70b": (64, 8, 128), "mqa64": (16, 1, 64),
         "mha": (8, 8, 128)}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the tables of a decode iteration: 64 sequences take one token each
        {"name": "slot_map_decode_64", "op": "slot_map", "decodes": 64, "prompts": 0, "new_lo": 1, "new_hi": 1,
         "ctx_lo": 1024, "ctx_hi": 8192, "pad": 0, "short": False, "lengths": 1},
        # a burst of prompts of many lengths, some of them continued, in one padded batch
        {"name": "slot_map_prompts_1000", "op": "slot_map", "decodes": 100, "prompts": 900, "new_lo": 1,
         "new_hi": 700, "ctx_lo": 1, "ctx_hi": 4096, "pad": 333, "short": False, "lengths": 2},
        # a decode iteration's write on the 8B shape: each row continues a page
        {"name": "write_decode_8b", "op": "write", "heads": "8b", "decodes": 64, "prompts": 0, "new_lo": 1,
         "new_hi": 1, "ctx_lo": 1024, "ctx_hi": 8192, "pad": 0, "lengths": 3},
        # a mixed iteration's write: a 2048-token prompt chunk and 32 decodes
        {"name": "write_mixed_8b", "op": "write", "heads": "8b", "decodes": 32, "prompts": 1, "new_lo": 2048,
         "new_hi": 2048, "ctx_lo": 1024, "ctx_hi": 8192, "pad": 0, "lengths": 4},
        # a handful of short prompts on the small shape, in a padded batch
        {"name": "write_tiny_odd", "op": "write", "heads": "tiny", "decodes": 3, "prompts": 5, "new_lo": 2,
         "new_hi": 41, "ctx_lo": 1, "ctx_hi": 200, "pad": 5, "lengths": 5},
        # a lone request with a long context: the lowest latency of a decode step's attention
        {"name": "decode_lone_8b", "op": "decode", "heads": "8b", "seqs": 1, "empty": 0, "ctx_lo": 8191,
         "ctx_hi": 8191, "lengths": 6},
        # decode attention over 64 contexts of 1k to 8k tokens
        {"name": "decode_64_8b", "op": "decode", "heads": "8b", "seqs": 64, "empty": 0, "ctx_lo": 1024,
         "ctx_hi": 8192, "lengths": 7},
        # a large batch on the 70B shape, very uneven, some of its places empty
        {"name": "decode_97_70b", "op": "decode", "heads": "70b", "seqs": 97, "empty": 3, "ctx_lo": 512,
         "ctx_hi": 16384, "lengths": 8},
        # short contexts on the small shape: launch-bound
        {"name": "decode_tiny", "op": "decode", "heads": "tiny", "seqs": 13, "empty": 2, "ctx_lo": 1, "ctx_hi": 300,
         "lengths": 9},
        # the fourth 2048-token chunk of a long prompt on the 8B shape
        {"name": "prefill_chunk_8b", "op": "prefill", "heads": "8b", "seqs": 1, "new_lo": 2048, "new_hi": 2048,
         "ctx_lo": 6144, "ctx_hi": 6144, "pad": 0, "lengths": 10},
        # candidate requests continuing 4k-token prompts, of many lengths, on the 32B shape
        {"name": "prefill_forks_32b", "op": "prefill", "heads": "32b", "seqs": 16, "new_lo": 5, "new_hi": 256,
         "ctx_lo": 3500, "ctx_hi": 4500, "pad": 7, "lengths": 11},
        # the last few tokens of a long prompt: few queries over many keys
        {"name": "prefill_tail_8b", "op": "prefill", "heads": "8b", "seqs": 1, "new_lo": 17, "new_hi": 17,
         "ctx_lo": 30001, "ctx_hi": 30001, "pad": 0, "lengths": 12},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slot_map", "write", "decode", "prefill"])
    heads = rng.choice(sorted(HEADS))
    seed = rng.randrange(1 << 30)
    if op == "slot_map":
        return {"op": op, "decodes": _log_int(rng, 1, 101) - 1, "prompts": _log_int(rng, 1, 900), "new_lo": 1,
                "new_hi": _log_int(rng, 1, 700), "ctx_lo": 1, "ctx_hi": _log_int(rng, 2, 4096),
                "pad": rng.choice([0, 0, _log_int(rng, 1, 500)]), "short": rng.random() < 0.15, "lengths": seed}
    if op == "write":
        prompts = _log_int(rng, 1, 30) - 1
        hi = _log_int(rng, 1, 1200 // max(1, prompts))
        return {"op": op, "heads": heads, "decodes": _log_int(rng, 1, 64), "prompts": prompts, "new_lo": 1,
                "new_hi": hi, "ctx_lo": 1, "ctx_hi": _log_int(rng, 2, 8192), "pad": rng.choice([0, rng.randrange(40)]),
                "lengths": seed}
    if op == "decode":
        seqs = _log_int(rng, 1, 120)
        hi = _log_int(rng, 2, min(40000, 430_000 // seqs))
        return {"op": op, "heads": heads, "seqs": seqs, "empty": rng.choice([0, 0, min(3, seqs - 1)]),
                "ctx_lo": _log_int(rng, 1, hi), "ctx_hi": hi, "lengths": seed}
    seqs = _log_int(rng, 1, 16)
    hi = _log_int(rng, 1, 2048 // seqs)
    ctx = _log_int(rng, 1, min(30000, 5_000_000 // (hi * seqs)))
    return {"op": op, "heads": heads, "seqs": seqs, "new_lo": _log_int(rng, 1, hi), "new_hi": hi, "ctx_lo": 1,
            "ctx_hi": ctx, "pad": rng.choice([0, rng.randrange(20)]), "lengths": seed}


def _spread(r, lo, hi, n):
    """n whole numbers in [lo, hi], even over their logarithm; the first is hi."""
    v = np.rint(np.exp(r.uniform(math.log(lo), math.log(hi), n))).astype(np.int64)
    v[:1] = hi
    return v


def _lengths(case):
    """(tokens in the cache, new tokens) of each sequence; they depend on the case alone."""
    r = np.random.RandomState(case["lengths"])
    if case["op"] == "decode":
        ctx = _spread(r, case["ctx_lo"], case["ctx_hi"], case["seqs"])
        if case["empty"]:
            ctx[-case["empty"]:] = 0
        return ctx, np.zeros_like(ctx)
    if case["op"] == "prefill":
        return (_spread(r, case["ctx_lo"], case["ctx_hi"], case["seqs"]),
                _spread(r, case["new_lo"], case["new_hi"], case["seqs"]))
    d, p = case["decodes"], case["prompts"]
    start = _spread(r, case["ctx_lo"], case["ctx_hi"], d + p)
    start[d:] *= r.randint(0, 2, p)   # half of the prompts begin, half are continued
    return start, np.concatenate([np.ones(d, np.int64), _spread(r, case["new_lo"], case["new_hi"], p)])


def _pages(n):
    return -(-n // PAGE)


def _scale_of(amax):
    """The least power of two s with amax <= 448 s (448: the largest e4m3 value), no less than 2^-100."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -100)).clamp(min=-100)
    return torch.ldexp(torch.ones_like(amax), e)


def _random_pool(g, hkv, nb, dh):
    """(codes, scales) of a pool whose heads have values of different sizes.  The values of a page have one
    distribution, so their order inside the page is that of either layout."""
    codes = torch.empty(hkv, nb, PAGE * dh, dtype=torch.uint8, device=DEV)
    scale = torch.empty(hkv, nb, device=DEV)
    size = torch.exp2(torch.rand(hkv, generator=g, device=DEV) * 2 - 1)
    for h in range(hkv):
        x = torch.randn(nb, PAGE * dh, generator=g, device=DEV) * size[h]
        scale[h] = _scale_of(x.abs().amax(1))
        codes[h] = (x / scale[h, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scale


def _tables(r, pages, stride, nb):
    """Block tables of sequences that hold these many pages each, and the pages left, in a random order."""
    order = r.permutation(nb).astype(np.int32)
    bt = np.full((len(pages), stride), -1, np.int32)
    at = 0
    for s, n in enumerate(pages):
        bt[s, :n] = order[at:at + n]
        at += n
    return bt, order[at:]


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def prepare(case, seed):
    r = np.random.RandomState(seed % (1 << 32))
    g = torch.Generator(device=DEV).manual_seed(seed)
    start, new = _lengths(case)
    S, T = len(start), int(new.sum()) + case.get("pad", 0)
    old, need = _pages(start), _pages(start + new) - _pages(start)
    s = {"op": case["op"], "S": S, "T": T, "ctx": _i32(start + new), "start": _i32(start), "new": _i32(new),
         "wide": int(new.max()), "row0": _i32(np.concatenate([[0], np.cumsum(new)]))}
    if case["op"] == "slot_map":
        stride = int((old + need).max()) + 3
        bt, free = _tables(r, old, stride, int(old.sum() + need.sum()) + 50)
        n_free = int(need.sum()) - 1 if case["short"] else len(free) - 10
        s |= {"bt": _i32(bt), "stride": stride, "free": _i32(free), "n_free": _i32([max(0, n_free)]),
              "row0": torch.zeros(S + 1, dtype=torch.int32, device=DEV), "status": _i32([0, 0]),
              "pos": torch.zeros(T, dtype=torch.int32, device=DEV), "slot": torch.zeros(T, dtype=torch.int32, device=DEV),
              "ctx": torch.zeros(S, dtype=torch.int32, device=DEV)}
        return s
    hq, hkv, dh = HEADS[case["heads"]]
    s |= {"hq": hq, "hkv": hkv, "dh": dh}
    if case["op"] == "write":
        # the pages that this batch touches, and as many others: what the operator's time depends on
        first = start // PAGE
        touched = np.where(new > 0, _pages(start + new) - first, 0)
        nb = 2 * int(touched.sum()) + 16
        order = r.permutation(nb).astype(np.int64)
        page0 = np.concatenate([[0], np.cumsum(touched)])
        seq = np.repeat(np.arange(S), new)
        pos = start[seq] + np.arange(len(seq)) - np.concatenate([[0], np.cumsum(new)])[seq]
        slot = order[page0[seq] + pos // PAGE - first[seq]] * PAGE + pos % PAGE
        pad = case["pad"]
        ang = (torch.arange(int(pos.max()) + 1, dtype=torch.float64, device=DEV)[:, None] *
               ROPE_BASE ** (-2 * torch.arange(dh // 2, dtype=torch.float64, device=DEV) / dh))
        x = torch.randn(T, hq + 2 * hkv, dh, generator=g, device=DEV)
        x *= torch.exp2(torch.rand(hq + 2 * hkv, 1, generator=g, device=DEV) * 3 - 1)
        s |= {"nb": nb, "qkv": x.to(torch.bfloat16).view(T, -1), "pos": _i32(np.concatenate([pos, np.zeros(pad)])),
              "slot": _i32(np.concatenate([slot, -np.ones(pad)])),
              "table": torch.stack([ang.cos(), ang.sin()], -1).float().contiguous(),
              "q": torch.zeros(T, hq, dh, dtype=torch.bfloat16, device=DEV)}
    else:
        rows = S if case["op"] == "decode" else T
        total = old + need
        nb = int(total.sum()) + 11
        stride = int(total.max()) + 2
        s |= {"nb": nb, "stride": stride, "bt": _i32(_tables(r, total, stride, nb)[0]),
              "q": torch.randn(rows, hq, dh, generator=g, device=DEV).to(torch.bfloat16),
              "out": torch.zeros(rows, hq, dh, dtype=torch.bfloat16, device=DEV)}
    s["k"], s["ks"] = _random_pool(g, hkv, s["nb"], dh)
    s["v"], s["vs"] = _random_pool(g, hkv, s["nb"], dh)
    return s


# ------------------------------------------------------------------ the framework's calls
def _own_run(s):
    from paper_2505_05286_amd import hxf
    st = torch.cuda.current_stream().cuda_stream
    if s["op"] == "slot_map":
        hxf.op_slot_map(s["start"].data_ptr(), s["new"].data_ptr(), s["S"], s["free"].data_ptr(),
                        s["n_free"].data_ptr(), s["free"].numel(), s["bt"].data_ptr(), s["stride"],
                        s["row0"].data_ptr(), s["pos"].data_ptr(), s["slot"].data_ptr(), s["T"], s["ctx"].data_ptr(),
                        s["status"].data_ptr(), stream=st)
        return {k: s[k] for k in ("bt", "row0", "pos", "slot", "ctx", "status")}
    hq, hkv, dh = s["hq"], s["hkv"], s["dh"]
    if "pool" not in s:
        s["pool"] = hxf.Kv8Pool(s["k"].data_ptr(), s["v"].data_ptr(), s["ks"].data_ptr(), s["vs"].data_ptr(), s["nb"])
    if s["op"] == "write":
        hxf.op_rope_kv8_write(s["qkv"].data_ptr(), (hq + 2 * hkv) * dh, s["pos"].data_ptr(), s["slot"].data_ptr(),
                              s["table"].data_ptr(), s["table"].shape[0], s["q"].data_ptr(), hq * dh, s["pool"],
                              s["T"], hq, hkv, dh, stream=st)
        return _write_outputs(s, s["q"])
    if s["op"] == "decode":
        if "ws" not in s:
            s["ws"] = torch.empty(hxf.op_decode_attention_kv8_workspace_bytes(s["S"], hq, hkv, dh), dtype=torch.uint8,
                                  device=DEV)
        hxf.op_decode_attention_kv8(s["q"].data_ptr(), hq * dh, s["pool"], s["bt"].data_ptr(), s["stride"],
                                    s["ctx"].data_ptr(), s["out"].data_ptr(), hq * dh, s["S"], hq, hkv, dh,
                                    s["ws"].data_ptr(), s["ws"].numel(), stream=st)
        return s["out"]
    if "ws" not in s:
        s["ws"] = torch.empty(hxf.op_prefill_attention_kv8_workspace_bytes(s["S"], s["T"], hq, hkv, dh),
                              dtype=torch.uint8, device=DEV)
    hxf.op_prefill_attention_kv8(s["q"].data_ptr(), hq * dh, s["pool"], s["bt"].data_ptr(), s["stride"],
                                 s["row0"].data_ptr(), s["start"].data_ptr(), s["out"].data_ptr(), hq * dh, s["S"],
                                 s["T"], hq, hkv, dh, s["ws"].data_ptr(), s["ws"].numel(), stream=st)
    return s["out"]


# ------------------------------------------------------------------ the plain forms
def _plain_slot_map(s):
    S, T, stride = s["S"], s["T"], s["stride"]
    start, new = s["start"].long(), s["new"].long()
    have = (start + PAGE - 1) // PAGE
    need = (start + new + PAGE - 1) // PAGE - have
    rows, taken = new.cumsum(0), need.cumsum(0)
    fits = ((taken[-1] <= s["n_free"][0].clamp(0, s["free"].numel())) & (rows[-1] <= T) &
            ((have + need).max() <= stride) & (start.min() >= 0) & (new.min() >= 0))
    j = torch.arange(stride, device=DEV)
    at = (taken - need - have)[:, None] + j
    fresh = (j >= have[:, None]) & (j < (have + need)[:, None]) & fits
    bt = torch.where(fresh, s["free"][at.clamp(0, s["free"].numel() - 1)], s["bt"])
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(rows, t, right=True).clamp(max=S - 1)
    pos = start[seq] + t - (rows - new)[seq]
    live = (t < rows[-1]) & fits
    slot = bt[seq, (pos // PAGE).clamp(0, stride - 1)].long() * PAGE + pos % PAGE
    row0 = torch.cat([torch.zeros_like(rows[:1]), rows])
    status = torch.stack([torch.where(fits, taken[-1], -1), torch.where(fits, rows[-1], 0)])
    out = {"bt": bt, "row0": torch.where(fits, row0, 0), "pos": torch.where(live, pos, 0),
           "slot": torch.where(live, slot, -1), "ctx": torch.where(fits, start + new, start), "status": status}
    return {k: v.int() for k, v in out.items()}


def _quantise(x, codes, scale, live, run, page, first, off, unpack, pack):
    """Write rows x [T, Hkv, dh] into the pages of their runs: codes [Hkv, nb, 16 dh] and scale [Hkv, nb] are
    updated.  Each row builds its run's whole page, so rows of one run write the same values."""
    T, hkv, dh = x.shape
    amax = torch.where(live[:, None], x.abs().amax(-1), 0)
    need = _scale_of(torch.zeros_like(amax).scatter_reduce(0, run[:, None].expand(-1, hkv), amax, "amax")[run])
    before = scale[:, page].T
    after = torch.where(first[:, None] > 0, torch.maximum(before, need), need)
    raw = unpack(codes[:, page]).transpose(0, 1)                                        # [T, Hkv, 16, dh]
    moved = (raw.view(torch.float8_e4m3fn).float() * (before / after)[..., None, None]).to(torch.float8_e4m3fn)
    mine = (x / after[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    to = torch.where(live, run, T)                                                      # dead rows go nowhere
    tile = torch.zeros(T + 1, PAGE, hkv, dh, dtype=torch.uint8, device=DEV)
    has = torch.zeros(T + 1, PAGE, dtype=torch.bool, device=DEV)
    tile[to, off], has[to, off] = mine, True
    kept = torch.arange(PAGE, device=DEV) < first[:, None]                              # [T, 16]
    page_new = torch.where(kept[:, None, :, None], moved.view(torch.uint8), raw)
    page_new = torch.where(has[run][:, None, :, None], tile[run].transpose(1, 2), page_new)
    codes[:, page] = pack(page_new.transpose(0, 1))
    scale[:, page] = after.T


def _plain_write(s):
    T, hq, hkv, dh = s["T"], s["hq"], s["hkv"], s["dh"]
    x = s["qkv"].float().view(T, hq + 2 * hkv, dh)
    cs = s["table"][s["pos"].long()]
    c, sn = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[:, :hq + hkv, :dh // 2], x[:, :hq + hkv, dh // 2:]
    x = torch.cat([torch.cat([a * c - b * sn, b * c + a * sn], -1), x[:, hq + hkv:]], 1)
    slot = s["slot"].long()
    live = slot >= 0
    off = slot % PAGE
    # a run: rows that go to successive places of one page
    lead = live & ((off == 0) | (slot != torch.cat([slot[:1] - 2, slot[:-1]]) + 1))
    run = (lead.cumsum(0) - 1).clamp(min=0)
    page = torch.zeros_like(run).scatter_reduce(0, run, torch.where(live, slot // PAGE, 0), "amax")[run]
    first = torch.full_like(run, PAGE).scatter_reduce(0, run, torch.where(live, off, PAGE), "amin")[run]
    hn = (hkv, T)
    _quantise(x[:, hq:hq + hkv], s["k"], s["ks"], live, run, page, first, off,
              lambda p: p.view(*hn, dh // 16, PAGE, 16).transpose(2, 3).reshape(*hn, PAGE, dh),
              lambda p: p.reshape(*hn, PAGE, dh // 16, 16).transpose(2, 3).reshape(*hn, PAGE * dh))
    _quantise(x[:, hq + hkv:], s["v"], s["vs"], live, run, page, first, off,
              lambda p: p.view(*hn, 4, dh, 4).transpose(3, 4).reshape(*hn, PAGE, dh),
              lambda p: p.reshape(*hn, 4, 4, dh).transpose(3, 4).reshape(*hn, PAGE * dh))
    return _write_outputs(s, torch.where(live[:, None, None], x[:, :hq].to(torch.bfloat16), s["q"]))


def _write_outputs(s, q):
    return {"q": q, "k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "ks": s["ks"],
            "vs": s["vs"]}


def _plain_kv(s):
    """K and V of every sequence in 32 bits, [S, Hkv, places of the block table, dh]."""
    dh, hkv, S, P = s["dh"], s["hkv"], s["S"], s["stride"]
    at = s["bt"].long().clamp(min=0)
    k = s["k"][:, at].view(torch.float8_e4m3fn).float() * s["ks"][:, at][..., None]
    k = k.view(hkv, S, P, dh // 16, PAGE, 16).transpose(3, 4).reshape(hkv, S, P * PAGE, dh)
    v = s["v"][:, at].view(torch.float8_e4m3fn).float() * s["vs"][:, at][..., None]
    v = v.view(hkv, S, P, 4, dh, 4).transpose(4, 5).reshape(hkv, S, P * PAGE, dh)
    return k.transpose(0, 1), v.transpose(0, 1)


def _plain_decode(s):
    S, hq, hkv, dh = s["S"], s["hq"], s["hkv"], s["dh"]
    k, v = _plain_kv(s)
    x = s["q"].float().view(S, hkv, hq // hkv, dh) @ k.transpose(2, 3) / math.sqrt(dh)
    ctx = s["ctx"].long()[:, None, None, None]
    seen = torch.arange(k.shape[2], device=DEV) < ctx
    p = torch.softmax(x.masked_fill(~seen, -math.inf), -1).masked_fill(~seen, 0)
    return (p @ v.masked_fill(~seen.transpose(2, 3), 0)).view(S, hq, dh).to(torch.bfloat16)


def _plain_prefill(s):
    S, T, hq, hkv, dh = s["S"], s["T"], s["hq"], s["hkv"], s["dh"]
    k, v = _plain_kv(s)
    n, start, row0 = s["new"].long(), s["start"].long(), s["row0"].long()[:-1]
    i = torch.arange(T, device=DEV)
    seq = torch.searchsorted(s["row0"][1:].long(), i, right=True)
    live, seq = seq < S, seq.clamp(max=S - 1)
    # the queries of all sequences side by side, padded to the longest
    wide = s["wide"]
    at = (row0[:, None] + torch.arange(wide, device=DEV)).clamp(max=T - 1)
    q = s["q"].float()[at].view(S, wide, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4)
    x = q.reshape(S, hkv, -1, dh) @ k.transpose(2, 3) / math.sqrt(dh)
    key = torch.arange(k.shape[2], device=DEV)
    seen = key <= (start[:, None] + torch.arange(wide, device=DEV))[..., None]            # [S, wide, keys]
    x = x.view(S, hkv, hq // hkv, wide, -1).masked_fill(~seen[:, None, None], -math.inf)
    p = torch.softmax(x, -1).view(S, hkv, -1, k.shape[2])
    o = p @ v.masked_fill((key >= (start + n)[:, None])[:, None, :, None], 0)
    o = o.view(S, hq, wide, dh).transpose(1, 2)[seq, (i - row0[seq]).clamp(0, wide - 1)]
    return torch.where(live[:, None, None], o.to(torch.bfloat16), s["out"])


def run(state):
    if own:
        return _own_run(state)
    return {"slot_map": _plain_slot_map, "write": _plain_write, "decode": _plain_decode,
            "prefill": _plain_prefill}[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    start, new = (a.astype(float) for a in _lengths(case))
    total = new.sum()
    need = (np.ceil((start + new) / PAGE) - np.ceil(start / PAGE)).sum()
    if case["op"] == "slot_map":
        # lengths and free pages read, tables, slots, positions and offsets written
        return {"bytes": float(16 * len(start) + 8 * need + 8 * (total + case["pad"])), "flops": 0.0}
    hq, hkv, dh = HEADS[case["heads"]]
    if case["op"] == "write":
        # rows read, q and codes written, a rotation's row and the scales; six operations for each rotated pair,
        # three for each quantised value
        row = (hq + 2 * hkv) * dh * 2 + hq * dh * 2 + 2 * hkv * dh + dh * 4 + 8
        runs = np.where(new > 0, np.ceil((start + new) / PAGE) - start // PAGE, 0).sum()
        return {"bytes": float(total * row + runs * hkv * 8),
                "flops": float(total * ((hq + hkv) * dh * 3 + 2 * hkv * dh * 3))}
    if case["op"] == "decode":
        return {"bytes": float(start.sum() * hkv * 2 * dh + np.ceil(start / PAGE).sum() * (hkv * 8 + 4) +
                               len(start) * hq * dh * 4),
                "flops": float(4 * dh * hq * start.sum())}
    pairs = (new * start + new * (new + 1) / 2).sum()
    ctx = start + new
    return {"bytes": float(ctx.sum() * hkv * 2 * dh + np.ceil(ctx / PAGE).sum() * (hkv * 8 + 4) + total * hq * dh * 4),
            "flops": float(4 * dh * hq * pairs)}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_page(pool, h, b, dh, kind):
    """Values of one page of one head before scaling, [16, dh]."""
    c = pool[h, b].astype(np.float64)
    return (c.reshape(dh // 16, PAGE, 16).transpose(1, 0, 2).reshape(PAGE, dh) if kind == "k"
            else c.reshape(4, dh, 4).transpose(0, 2, 1).reshape(PAGE, dh))


def _e4m3(x):
    """Nearest e4m3 value, ties to even; |x| <= 448."""
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.rint(x / step) * step


def _exact_write(s):
    hq, hkv, dh = s["hq"], s["hkv"], s["dh"]
    slot, pos = s["slot"].cpu().numpy(), s["pos"].cpu().numpy()
    x = s["qkv"].double().cpu().numpy().reshape(len(slot), -1, dh)
    cs = s["table"].double().cpu().numpy()[pos]
    z = (x[..., :dh // 2] + 1j * x[..., dh // 2:]) * (cs[..., 0] + 1j * cs[..., 1])[:, None]
    z = np.concatenate([z.real, z.imag], -1)
    rows = {"k": z[:, hq:hq + hkv], "v": x[:, hq + hkv:]}
    out = {"q": np.where((slot >= 0)[:, None, None], z[:, :hq], 0.0)}
    runs = []
    for t, at in enumerate(slot):
        if at < 0:
            continue
        if runs and at % PAGE and slot[runs[-1][-1]] == at - 1:
            runs[-1].append(t)
        else:
            runs.append([t])
    for kind in ("k", "v"):
        pool = s[kind].view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)
        scale = s[kind + "s"].double().cpu().numpy()
        for ts in runs:
            b, o = slot[ts[0]] // PAGE, slot[ts[0]] % PAGE
            new = rows[kind][ts]                                            # [n, Hkv, dh]
            for h in range(hkv):
                want = 2.0 ** np.ceil(np.log2(np.abs(new[:, h]).max() / 448.0))
                after = max(want, scale[h, b]) if o else want
                page = _exact_page(pool, h, b, dh, kind)
                page[:o] = _e4m3(page[:o] * (scale[h, b] / after))
                page[o:o + len(ts)] = _e4m3(new[:, h] / after)
                pool[h, b] = (page.reshape(PAGE, dh // 16, 16).transpose(1, 0, 2) if kind == "k"
                              else page.reshape(4, 4, dh).transpose(0, 2, 1)).reshape(-1)
                scale[h, b] = after
        out[kind], out[kind + "s"] = pool, scale
    return out


def _exact_attention(s, rows_of):
    """softmax(q k / sqrt(dh)) v of each sequence in turn; rows_of(i) gives its rows and their first position."""
    hq, hkv, dh = s["hq"], s["hkv"], s["dh"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    ctx = s["ctx"].tolist()
    for i, n in enumerate(ctx):
        r0, r1, p0 = rows_of(i)
        if n == 0 or r0 == r1:
            continue
        at = s["bt"][i, :_pages(n)].long()
        for h in range(hkv):
            k = s["k"][h, at].view(torch.float8_e4m3fn).double() * s["ks"][h, at].double()[:, None]
            v = s["v"][h, at].view(torch.float8_e4m3fn).double() * s["vs"][h, at].double()[:, None]
            k = k.view(-1, dh // 16, PAGE, 16).permute(0, 2, 1, 3).reshape(-1, dh)[:n]
            v = v.view(-1, 4, dh, 4).permute(0, 1, 3, 2).reshape(-1, dh)[:n]
            G = hq // hkv
            q = s["q"][r0:r1, h * G:(h + 1) * G].double()
            hide = torch.arange(n, device=DEV) > torch.arange(p0, p0 + r1 - r0, device=DEV)[:, None]
            x = (q.reshape(-1, dh) @ k.T).view(r1 - r0, G, n) / math.sqrt(dh)
            x = x.masked_fill(hide[:, None], -math.inf)
            w = torch.exp(x - x.amax(-1, keepdim=True))
            o = (w / w.sum(-1, keepdim=True)).view(-1, n) @ v
            out[r0:r1, h * G:(h + 1) * G] = o.view(r1 - r0, G, dh)
    return out


def exact(case, seed):
    if case["op"] == "slot_map":
        return None   # whole numbers
    s = prepare(case, seed)
    if case["op"] == "write":
        return _exact_write(s)
    if case["op"] == "decode":
        ctx = s["ctx"].tolist()
        return _exact_attention(s, lambda i: (i, i + 1, ctx[i] - 1))
    row0, start = s["row0"].tolist(), s["start"].tolist()
    return _exact_attention(s, lambda i: (row0[i], row0[i + 1], start[i]))
