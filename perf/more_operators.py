"""Performance cases of positions, per-head norms and drafted trees on the packed cache.

What stands between a layer's projection and its attention, and the check of
drafted tokens:

* ``rope``     rotary positions of queries and keys, with the RMS norm of each
               head in the same pass where the model has one;
* ``append``   the same on the way into a packed cache: keys normed, rotated,
               coded and packed, values coded, queries rotated; or, without
               queries, the accepted ones of a draft's rows;
* ``tree``     attention of the newest C tokens of every sequence, which form
               a tree (each sees its ancestors), over a prefix cache and the
               sequence's own.

With ``own`` false, ``run`` computes a case in elementary torch operations
(the packed bytes included); with it true it calls the library.  ``exact`` is
the definition in 64 bits.  The formats' rules are restated here from their
definitions in ``include/kvq.h``.
"""
import math
import random

import numpy as np
import torch

own = False

# ------------------------------------------------------------------ formats

FIELDS = ("k_bits", "v_bits", "k_mode", "v_mode", "k_axis", "v_axis", "k_group", "v_group", "residual", "flush",
          "rotate", "meta_fp16", "sink")
AFFINE, SYMMETRIC = 0, 1


def _fmt(kb, vb, kg, vg, mode=AFFINE, per_channel=0, residual=0, flush=0, rotate=0, meta_fp16=0, sink=0):
    return dict(zip(FIELDS, (kb, vb, mode, mode, per_channel, 0, kg, vg, residual, flush, rotate, meta_fp16, sink)))


# The repository's workload formats (grouped affine, KIVI, rotated symmetric K4V2) and their options.
FORMATS = {
    "affine4_g32": _fmt(4, 4, 32, 32),
    "affine4_g64": _fmt(4, 4, 64, 64),
    "affine4_g64_meta16": _fmt(4, 4, 64, 64, meta_fp16=1),
    "affine2_g32": _fmt(2, 2, 32, 32),
    "affine8_g64": _fmt(8, 8, 64, 64),
    "affine4_g64_sink": _fmt(4, 4, 64, 64, sink=128),
    "kivi2": _fmt(2, 2, 32, 32, per_channel=1, residual=128, flush=32),
    "kivi2_meta16": _fmt(2, 2, 32, 32, per_channel=1, residual=128, flush=32, meta_fp16=1),
    "had": _fmt(4, 2, 128, 32, mode=SYMMETRIC, rotate=1),
    "had_sink": _fmt(4, 2, 128, 32, mode=SYMMETRIC, rotate=1, sink=128),
}

# (D, H_q, H_kv): the repository's layers (TinyLlama-, Llama-3.1-8B- and 12B-class-shaped), and one whose
# query heads share no KV heads.
LAYERS = {"tiny": (64, 32, 4), "llama8b": (128, 32, 8), "gqa12b": (256, 16, 8), "mha": (128, 16, 16)}


def _format(case):
    f, D = dict(FORMATS[case["format"]]), LAYERS[case["layer"]][0]
    f["rotate"] = D if f["rotate"] else 0
    f["k_group"], f["v_group"] = min(D, f["k_group"]), min(D, f["v_group"])
    return f


def _coded(f, n):
    """Tokens held as codes of the n - sink tail tokens."""
    n = max(0, n - f["sink"])
    return n if not f["flush"] else max(0, n - f["residual"]) // f["flush"] * f["flush"]


# -------------------------------------------------------------------- cases

def listed():
    return [
        # One decode step of a small model: a token's queries and keys.
        dict(name="rope_tiny_b1", kind="rope", layer="tiny", B=1, n=1, rot=64, interleaved=False, norm=False,
             bands=False, start=255, depths=False),
        # Drafted trees of a batch with query and key norms: positions by depth.
        dict(name="rope_gqa12b_drafts", kind="rope", layer="gqa12b", B=8, n=24, rot=256, interleaved=False, norm=True,
             bands=False, start=6000, depths=True),
        # A ragged chunk far into a long context: half of the head, neighbouring channels, scaled frequencies.
        dict(name="rope_llama8b_333", kind="rope", layer="llama8b", B=3, n=333, rot=64, interleaved=True, norm=False,
             bands=True, start=100000, depths=False),
        # The prompt chunk of a serving batch, wide heads with norms.
        dict(name="rope_gqa12b_2048", kind="rope", layer="gqa12b", B=8, n=2048, rot=256, interleaved=False, norm=True,
             bands=False, start=4096, depths=False),
        # The smallest append: one token of one sequence.
        dict(name="append_tiny_b1", kind="append", layer="tiny", format="affine4_g32", B=1, n=1, cached=200, rot=64,
             interleaved=False, norm=False, bands=False, queries=True, drafts=0),
        # A decode step of the KIVI cache at which 32 tokens leave the window.
        dict(name="append_llama8b_kivi", kind="append", layer="llama8b", format="kivi2", B=32, n=1, cached=4127,
             rot=128, interleaved=False, norm=False, bands=True, queries=True, drafts=0),
        # Five accepted tokens of 32 drafted ones, into the committed rotated cache.
        dict(name="append_llama8b_accept", kind="append", layer="llama8b", format="had", B=16, n=5, cached=5003,
             rot=128, interleaved=False, norm=False, bands=True, queries=False, drafts=32),
        # The largest append: a prompt chunk of a batch, wide heads with norms.
        dict(name="append_gqa12b_2048", kind="append", layer="gqa12b", format="affine4_g64", B=8, n=2048, cached=4096,
             rot=256, interleaved=False, norm=True, bands=False, queries=True, drafts=0),
        # Eight drafts of one short prompt.
        dict(name="tree_tiny_b1", kind="tree", layer="tiny", format="affine4_g32", P=1, B=1, prefix=256, suffix=8, C=8,
             ragged=False),
        # A batch whose sequences have a committed KIVI cache and a draft cache each.
        dict(name="tree_llama8b_kivi", kind="tree", layer="llama8b", format="kivi2", P=8, B=8, prefix=4096, suffix=48,
             C=48, ragged=False),
        # Drafts behind the tokens of one cache, wide heads.
        dict(name="tree_gqa12b", kind="tree", layer="gqa12b", format="affine4_g64", P=1, B=2, prefix=0, suffix=8191,
             C=64, ragged=False),
        # The largest tree call: 16 users of one 32k document, their own tokens behind it, rotated cache.
        dict(name="tree_llama8b_had", kind="tree", layer="llama8b", format="had", P=1, B=16, prefix=32768, suffix=300,
             C=24, ragged=False),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "tree"])
    case = dict(kind=kind, layer=rng.choice(list(LAYERS)))
    D, H_q, H = LAYERS[case["layer"]]
    if kind != "tree":
        # tokens: at most the numbers of the largest listed call
        most = (8 * 2048 * 24 * 256) // ((H_q + H) * D)
        case["n"] = _log_int(rng, 1, 2048) if rng.random() < 0.7 else 1
        case["B"] = _log_int(rng, 1, max(1, min(64, most // case["n"])))
        case["rot"] = D if rng.random() < 0.5 else 16 * rng.randint(1, D // 16)
        case["interleaved"], case["norm"], case["bands"] = rng.random() < 0.4, rng.random() < 0.5, rng.random() < 0.4
    if kind == "rope":
        case["start"] = _log_int(rng, 1, 1000000)
        case["depths"] = case["n"] <= 256 and rng.random() < 0.4
        return case
    case["format"] = rng.choice(list(FORMATS))
    if kind == "append":
        f = _format(case)
        case["queries"] = rng.random() < 0.7
        case["drafts"] = 0
        if not case["queries"] and case["n"] <= 16 and rng.random() < 0.7:
            case["drafts"] = rng.randint(case["n"], 64)
        # (a window's slots are replaced by later tokens: a longer call on a cache of such a format starts it)
        case["cached"] = 0 if f["flush"] and case["n"] > 1 else _log_int(rng, 1, 5000)
        return case
    case["P"] = rng.choice([1, 1, 2, 8])
    case["B"] = _log_int(rng, case["P"], 16)
    case["ragged"] = rng.random() < 0.4
    if not case["ragged"]:
        case["B"] = case["B"] // case["P"] * case["P"]
    case["C"] = _log_int(rng, 2, 96)
    case["suffix"] = case["C"] + (0 if rng.random() < 0.5 else _log_int(rng, 1, 2000))
    # at most the work of the largest listed call
    most = 16 * 24 * 32 * 128 * 32768 // (case["B"] * case["C"] * H_q * D)
    most = min(32768 // case["P"], most)
    case["prefix"] = 0 if case["P"] == 1 and rng.random() < 0.3 else _log_int(rng, 64, max(65, most))
    return case


def _first(case):
    """The first sequence of each prefix's group, and B: equal groups, or growing ones (the first may be empty)."""
    P, B = case["P"], case["B"]
    return [B * g * g // (P * P) if case["ragged"] else B // P * g for g in range(P)] + [B]


def _turns(case):
    """Turns per position of every rotated pair, 64 bits; `bands` slows wavelengths of 2048 and more down by 8, those
    below 512 not at all and what is between gradually, for contexts of eight times 2048."""
    rot = case["rot"]
    f = (500000.0 if case["bands"] else 10000.0) ** (-2.0 * np.arange(rot // 2, dtype=np.float64) / rot)
    if case["bands"]:
        waves = 2048.0 / (2 * math.pi / f)  # of a pair in 2048 positions
        keep = np.clip((waves - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 8.0)
    return f / (2 * math.pi)


EPS = 1e-6

# ------------------------------------------------------------------- inputs

def _gen(seed, name):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + sum((i + 1) * ord(c) for i, c in enumerate(name)) * 7919) % (1 << 62))
    return g


def _normal(seed, name, shape):
    return torch.randn(shape, generator=_gen(seed, name), device="cuda").to(torch.bfloat16)


def _code(x, bits, mode, meta16):
    """Codes, scales and offsets (None when symmetric) of the last axis' groups."""
    if mode == AFFINE:
        lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
        s, z, shift, low, top = ((hi - lo) / (2 ** bits - 1)).clamp_min(1e-8), lo, 0, 0, 2 ** bits - 1
    else:
        top = 2 ** (bits - 1) - 1
        s, z, shift, low = (x.abs().amax(-1, keepdim=True) / top).clamp_min(1e-8), None, top + 1, -top
    if meta16:
        s = s.clamp(2.0 ** -24, 65504.0).half().float()
        z = None if z is None else z.half().float()
    c = ((x if z is None else x - z) / s).round().clamp(low, top) + shift
    return c.to(torch.uint8), s, z


def _tokens(case, f, seed, name, U, n):
    """The tokens of U sequences: codes [U, H, nq, D], scales and offsets per group, fp16 sink and window rows."""
    D, _, H = LAYERS[case["layer"]]
    nq, nsink = _coded(f, n), min(n, f["sink"])
    fac = torch.ones((H, 1, D), device="cuda")
    if not f["rotate"]:  # key outlier channels: a factor of 20 on four channels of each KV head
        order = torch.rand((H, 1, D), generator=_gen(seed, name + "outlier"), device="cuda").argsort(dim=-1)
        fac.scatter_(-1, order[..., :4], 20.0)
    K = (_normal(seed, name + "K", (U, H, n, D)) * fac).to(torch.bfloat16).float()
    V = _normal(seed, name + "V", (U, H, n, D)).float()
    t = dict(n=n, nq=nq, nsink=nsink, sinkK=K[:, :, :nsink].half(), sinkV=V[:, :, :nsink].half(),
             winK=K[:, :, nsink + nq:].half(), winV=V[:, :, nsink + nq:].half())
    K, V = K[:, :, nsink:nsink + nq], V[:, :, nsink:nsink + nq]
    m16 = f["meta_fp16"]
    if f["k_axis"]:  # groups of 32 tokens of a channel: the group axis last
        c, s, z = _code(K.reshape(U, H, nq // 32, 32, D).transpose(-1, -2), f["k_bits"], f["k_mode"], m16)
        t["kc"], t["ks"], t["kz"] = c.transpose(-1, -2).reshape(U, H, nq, D), s[..., 0], None if z is None else z[..., 0]
    else:
        c, s, z = _code(K.reshape(U, H, nq, D // f["k_group"], f["k_group"]), f["k_bits"], f["k_mode"], m16)
        t["kc"], t["ks"], t["kz"] = c.reshape(U, H, nq, D), s[..., 0], None if z is None else z[..., 0]
    c, s, z = _code(V.reshape(U, H, nq, D // f["v_group"], f["v_group"]), f["v_bits"], f["v_mode"], m16)
    t["vc"], t["vs"], t["vz"] = c.reshape(U, H, nq, D), s[..., 0], None if z is None else z[..., 0]
    return t


# ------------------------------------------------ the caches' bytes (include/kvq.h)

def _block_bytes(f, D):
    """Bytes of a (sequence, head)'s 32-token block in sections 0 to 5."""
    m = 2 if f["meta_fp16"] else 4
    km, vm = (D if f["k_axis"] else D // f["k_group"] * 32) * m, D // f["v_group"] * 32 * m
    return [4 * D * f["k_bits"], km, km if f["k_mode"] == AFFINE else 0, 4 * D * f["v_bits"], vm,
            vm if f["v_mode"] == AFFINE else 0]


def _live_bytes(f, n, H, D):
    """Bytes of one sequence's n tokens."""
    nq, nsink = _coded(f, n), min(n, f["sink"])
    return H * (sum(_block_bytes(f, D)) * -(-nq // 32) + 4 * D * (n - nq))


def _sections(f, U, H, D, T_max):
    """(offset, bytes of a (sequence, head)) of the ten sections, and the total."""
    NB = -(-max(T_max - f["sink"], 0) // 32)
    ring = 2 * D * (f["residual"] + f["flush"])
    per = [NB * b for b in _block_bytes(f, D)] + [ring, ring, 2 * D * f["sink"], 2 * D * f["sink"]]
    ends = [0]
    for p in per:
        ends.append(-(-(ends[-1] + U * H * p) // 256) * 256)
    return list(zip(ends, per)), ends[-1]


def _view(img, section, U, H):
    """A section's bytes [U, H, bytes]."""
    off, per = section
    return img[off:off + U * H * per].view(U, H, per)


def _blocks(x):
    """Tokens of axis 2 padded with zeros to whole 32-token blocks [U, H, blocks, 32, ...]."""
    U, H, n = x.shape[:3]
    out = torch.zeros((U, H, -(-n // 32) * 32) + x.shape[3:], dtype=x.dtype, device=x.device)
    out[:, :, :n] = x
    return out.view((U, H, -(-n // 32), 32) + x.shape[3:])


def _pack8(c, bits):
    """Pieces of eight codes (last axis) -> `bits` bytes, code j at bits [bits j, bits j + bits)."""
    if bits == 8:
        return c
    per = 8 // bits
    c = c.reshape(c.shape[:-1] + (bits, per)).to(torch.int32) << (torch.arange(per, device=c.device) * bits).int()
    return c.sum(-1).to(torch.uint8)


def _image(case, f, t, U, T_max):
    """The storage image of a cache that holds the tokens t (dead bytes zero)."""
    D, _, H = LAYERS[case["layer"]]
    sec, total = _sections(f, U, H, D, T_max)
    img = torch.zeros(total, dtype=torch.uint8, device="cuda")

    def put(i, x):
        if x is not None and x.numel():
            x = x.flatten(2).contiguous().view(torch.uint8)
            _view(img, sec[i], U, H)[:, :, :x.shape[2]] = x

    meta = torch.float16 if f["meta_fp16"] else torch.float32
    # key pieces: token 8 o + 4 e + w, channels 8 (4 P + p) + j  ->  [e][p][o][w][P]
    k = _blocks(t["kc"]).unflatten(4, (D // 32, 4, 8)).unflatten(3, (4, 2, 4)).permute(0, 1, 2, 4, 7, 3, 5, 6, 8)
    put(0, _pack8(k, f["k_bits"]))
    # value pieces: tokens 8 o + j, channel 16 a + b  ->  [o][b][a]
    v = _blocks(t["vc"]).unflatten(4, (D // 16, 16)).unflatten(3, (4, 8)).permute(0, 1, 2, 3, 6, 5, 4)
    put(3, _pack8(v, f["v_bits"]))
    for i, x in ((1, t["ks"]), (2, t["kz"]), (4, t["vs"]), (5, t["vz"])):
        if x is not None:
            # per token: [block][group][32 tokens]; per channel as it is: [block][channel]
            put(i, (x if f["k_axis"] and i < 3 else _blocks(x).transpose(-1, -2)).to(meta))
    ring = f["residual"] + f["flush"]
    if ring:
        slot = torch.arange(t["nq"], t["nq"] + t["winK"].shape[2], device="cuda") % ring
        for i, x in ((6, t["winK"]), (7, t["winV"])):
            _view(img, sec[i], U, H).view(torch.float16).view(U, H, ring, D)[:, :, slot] = x
    put(8, t["sinkK"])
    put(9, t["sinkV"])
    return img


def _tree(case, seed):
    """The parents of a random tree per sequence and who sees whom, [B, C, C]; the last sequences have fewer drafts,
    the rows behind them see no draft."""
    rng = np.random.default_rng([int(seed), 11])
    B, C = case["B"], case["C"]
    sees, depth = np.zeros((B, C, C), bool), np.zeros((B, C), np.int64)
    for i in range(C):
        if i:  # near the end of what is there, as trees grow by levels
            parent = np.maximum(0, i - 1 - rng.integers(0, 4, B))
            sees[:, i] = sees[np.arange(B), parent]
            depth[:, i] = depth[np.arange(B), parent] + 1
        sees[:, i, i] = True
    used = C - np.arange(B) * (C // 3) // B
    sees[np.arange(C)[None, :] >= used[:, None]] = False
    return sees, depth


def _words(sees):
    """Bit j % 32 of word j / 32 of a row: whether it sees draft j."""
    B, C, _ = sees.shape
    bits = np.zeros((B, C, -(-C // 32) * 32), np.uint64)
    bits[:, :, :C] = sees
    return (bits.reshape(B, C, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def _positions(case, seed):
    """[B, n] positions, and whether they are consecutive from the first."""
    B, n, start = case["B"], case["n"], case.get("start", case.get("cached"))
    if case.get("depths") or case.get("drafts"):
        # by depth, sequence b a little further on; accepted rows have consecutive depths, but are given as positions too
        depth = _tree(dict(B=B, C=n), seed)[1] if case.get("depths") else np.arange(n)[None, :].repeat(B, 0)
        return torch.from_numpy(start + np.arange(B)[:, None] + depth).int().cuda(), False
    return (start + torch.arange(n, device="cuda")).expand(B, n), True


def prepare(case, seed):
    D, H_q, H = LAYERS[case["layer"]]
    s = dict(case=dict(case), H=H, D=D, H_q=H_q, sm=D ** -0.5)
    if case["kind"] == "tree":
        _prepare_tree(s, case, seed)
    else:
        B, n = case["B"], case["n"]
        s["turns"], s["rot"], s["interleaved"] = _turns(case), case["rot"], case["interleaved"]
        s["turn"] = torch.from_numpy(s["turns"]).cuda()
        s["pos"], s["consecutive"] = _positions(case, seed)
        s["start"] = case.get("start", case.get("cached"))
        s["wq"] = s["wk"] = None
        if case["norm"]:  # weights near one
            s["wq"], s["wk"] = ((1 + 0.2 * _normal(seed, w, (D,)).float()).to(torch.bfloat16) for w in ("wq", "wk"))
        s["Q"] = _normal(seed, "Q", (B, n, H_q, D)) if case.get("queries", True) else None
        if case["kind"] == "rope":
            s["K"] = _normal(seed, "K", (B, n, H, D))
        else:
            _prepare_append(s, case, seed)
    if own:
        _handles(s)
    return s


def _prepare_append(s, case, seed):
    f, B, n, H, D, n0 = _format(case), case["B"], case["n"], s["H"], s["D"], case["cached"]
    s["f"], s["n0"], s["n"], s["T"] = f, n0, n, n0 + n + 64
    s["image"] = _image(case, f, _tokens(case, f, seed, "cache", B, n0), B, s["T"])
    rows = case["drafts"] or n
    fac = torch.ones((H, D), device="cuda")
    if not f["rotate"]:
        order = torch.rand((H, D), generator=_gen(seed, "outlier"), device="cuda").argsort(dim=-1)
        fac.scatter_(-1, order[..., :4], 20.0)
    s["K"], s["V"] = (_normal(seed, "K", (B, rows, H, D)) * fac).to(torch.bfloat16), _normal(seed, "V", (B, rows, H, D))
    s["rows"] = None
    if case["drafts"]:  # accepted drafts: increasing, another path in every sequence
        pick = torch.rand((B, rows), generator=_gen(seed, "rows"), device="cuda").argsort(dim=-1)[:, :n]
        s["rows"] = pick.sort(dim=-1).values.int().contiguous()
    f32 = dict(dtype=torch.float32, device="cuda")
    s["rot_c"] = torch.tensor(D ** -0.5, **f32)
    s["levels"] = {b: torch.tensor(float(b), **f32) for b in (1, 3, 7, 15, 127, 255)}


def _prepare_tree(s, case, seed):
    f, H, H_q, D = _format(case), s["H"], s["H_q"], s["D"]
    P, B, C = case["P"], case["B"], case["C"]
    s["f"], s["P"], s["B"], s["C"], s["np"], s["ns"] = f, P, B, C, case["prefix"], case["suffix"]
    s["first"] = _first(case)
    s["Tp"], s["Ts"] = max(1, s["np"]), s["ns"] + 64
    s["prefix"] = _image(case, f, _tokens(case, f, seed, "prefix", P, s["np"]), P, s["Tp"])
    s["suffix"] = _image(case, f, _tokens(case, f, seed, "suffix", B, s["ns"]), B, s["Ts"])
    s["Q"] = _normal(seed, "Q", (B, C, H_q, D))
    s["tree"] = torch.from_numpy(_words(_tree(case, seed)[0])).cuda()
    group = torch.bucketize(torch.arange(B), torch.tensor(s["first"][1:]), right=True)
    s["group"], s["slot"] = group.cuda(), (torch.arange(B) - torch.tensor(s["first"])[group]).cuda()
    s["most"] = max(b - a for a, b in zip(s["first"], s["first"][1:]))


def _handles(s):
    """The library's handles and the buffers that a serving loop keeps."""
    from paper_2609_04263_amd import kvq

    def cache(img, U, T, n):
        c = kvq.Cache(s["f"], U, s["H"], s["D"], T, storage=img)
        c.restore(n)
        return c
    kind = s["case"]["kind"]
    if kind == "tree":
        s["prefix_cache"] = cache(s["prefix"], s["P"], s["Tp"], s["np"])
        s["suffix_cache"] = cache(s["suffix"], s["B"], s["Ts"], s["ns"])
        s["ws"] = s["suffix_cache"].shared_workspace(s["prefix_cache"], s["H_q"], s["C"])
        s["O"] = torch.empty(s["Q"].shape, dtype=torch.float32, device="cuda")
        return
    s["rope"] = kvq.Rope(s["rot"], turns=s["turns"], interleaved=s["interleaved"], eps=EPS)
    s["at"] = None if s["consecutive"] else s["pos"]
    s["Qo"] = None if s["Q"] is None else torch.empty_like(s["Q"])
    if kind == "rope":
        s["Ko"] = torch.empty_like(s["K"])
    else:
        s["cache"] = cache(s["image"], s["case"]["B"], s["T"], s["n0"])


# --------------------------------------------------------------------- pass

def run(s):
    if own:
        return _own(s)
    return {"rope": _rope, "append": _append, "tree": _attention}[s["case"]["kind"]](s)


def _own(s):
    kind = s["case"]["kind"]
    if kind == "rope":
        s["rope"].qk(s["Q"], s["K"], s["Qo"], s["Ko"], q_norm=s["wq"], k_norm=s["wk"], pos=s["at"], pos0=s["start"])
        return {"Q": s["Qo"], "K": s["Ko"]}
    if kind == "append":
        s["cache"].restore(s["n0"])
        s["cache"].append_rope(s["rope"], s["K"], s["V"], s["n"], rows=s["rows"], Q=s["Q"], Qo=s["Qo"], q_norm=s["wq"],
                               k_norm=s["wk"], pos=s["at"], pos0=s["start"])
        return {"image": s["image"]} if s["Q"] is None else {"image": s["image"], "Q": s["Qo"]}
    s["suffix_cache"].tree_attn_shared(s["prefix_cache"], s["Q"], s["C"], s["H_q"], s["sm"], s["tree"], s["O"], s["ws"],
                                       first=s["first"])
    return s["O"]


def _angles(s):
    """Cosines and sines [B, n, 1, rot / 2]: the fraction of a turn in 64 bits, exact by a high part of 24 bits."""
    t, high = s["pos"].double()[..., None, None], s["turn"].float().double()
    a = t * high
    a = 2 * math.pi * ((a - a.floor()) + t * (s["turn"] - high))
    return a.cos().float(), a.sin().float()


def _turned(s, x, w, cos, sin):
    """Rows [B, n, heads, D] normed (w) and rotated, 32 bits."""
    x = x.float()
    if w is not None:
        r = (1.0 / (x.double().square().sum(-1, keepdim=True) / s["D"] + float(np.float32(EPS))).sqrt()).float()
        x = (x * r) * w.float()
    rot = s["rot"]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1).to(torch.bfloat16)


def _rope(s):
    cos, sin = _angles(s)
    return {"Q": _turned(s, s["Q"], s["wq"], cos, sin), "K": _turned(s, s["K"], s["wk"], cos, sin)}


def _butterflies(x, c):
    """The transform of a rotating format on the last axis: additions of half widths 1, 2, .., then one product."""
    D, h = x.shape[-1], 1
    while h < D:
        a, b = x.unflatten(-1, (-1, 2, h)).unbind(-2)
        x, h = torch.stack((a + b, a - b), -2).flatten(-3), 2 * h
    return x * c


def _coded_values(s, x, bits, mode, axis, group):
    """Codes (uint8), scales and offsets of [B, H, tokens, D]; groups along channels, or 32 tokens of a channel.
    (Divisors are tensors: a division by a number becomes a product with its reciprocal.)"""
    x = x.unflatten(2, (-1, 32)).transpose(-1, -2) if axis else x.unflatten(-1, (-1, group))
    if mode == AFFINE:
        z, shift, low, top = x.amin(-1, keepdim=True) + 0.0, 0, 0, 2 ** bits - 1
        sc = ((x.amax(-1, keepdim=True) - z) / s["levels"][top]).clamp_min(1e-8)
    else:
        top = 2 ** (bits - 1) - 1
        z, shift, low = None, top + 1, -top
        sc = (x.abs().amax(-1, keepdim=True) / s["levels"][top]).clamp_min(1e-8)
    if s["f"]["meta_fp16"]:
        sc = sc.clamp(2.0 ** -24, 65504.0).half().float()
        z = None if z is None else z.clamp(-65504.0, 65504.0).half().float() + 0.0
    c = (((x if z is None else x - z) / sc).round().clamp(low, top) + shift).to(torch.uint8)
    c = c.transpose(-1, -2).flatten(2, 3) if axis else c.flatten(-2)
    return c, sc[..., 0], None if z is None else z[..., 0]


def _append(s):
    """The packed bytes of n tokens behind n0: what they share a block with is unpacked and packed again."""
    f, H, D, n0, n, img = s["f"], s["H"], s["D"], s["n0"], s["n"], s["image"]
    cos, sin = _angles(s)
    K, V = s["K"], s["V"]
    if s["rows"] is not None:
        at = s["rows"].long()[..., None, None].expand(-1, -1, H, D)
        K, V = K.gather(1, at), V.gather(1, at)
    K = _turned(s, K, s["wk"], cos, sin).float().transpose(1, 2)
    V = V.float().transpose(1, 2)
    if f["rotate"]:
        K, V = _butterflies(K, s["rot_c"]), _butterflies(V, s["rot_c"])
    U, S, ring = K.shape[0], f["sink"], f["residual"] + f["flush"]
    sec, size = _sections(f, U, H, D, s["T"])[0], _block_bytes(f, D)
    sink = max(0, min(n0 + n, S) - n0)
    for i, x in ((8, K), (9, V)):
        if sink:
            _view(img, sec[i], U, H).view(torch.float16).view(U, H, S, D)[:, :, n0:n0 + sink] = x[:, :, :sink].half()
    K, V, t0 = K[:, :, sink:], V[:, :, sink:], max(0, n0 - S)  # the tail
    t1, q0, q1 = t0 + K.shape[2], _coded(f, n0), _coded(f, n0 + n)
    if ring:
        K, V = K.half().float(), V.half().float()
        slots, older = torch.arange(q0, t0, device="cuda") % ring, []
        for i, x in ((6, K), (7, V)):
            window = _view(img, sec[i], U, H).view(torch.float16).view(U, H, ring, D)
            older.append(torch.cat((window[:, :, slots].float(), x), 2)[:, :, :q1 - q0])
            lo = max(t0, t1 - ring)
            window[:, :, torch.arange(lo, t1, device="cuda") % ring] = x[:, :, lo - t0:].half()
        K, V = older
    if q1 > q0:
        b0, b1, meta = q0 // 32, -(-q1 // 32), torch.float16 if f["meta_fp16"] else torch.float32

        def part(i):
            return _view(img, sec[i], U, H)[:, :, size[i] * b0:size[i] * b1].unflatten(2, (b1 - b0, size[i]))

        def codes(c, whole):
            whole = whole.reshape(U, H, -1, D)
            whole[:, :, q0 - 32 * b0:q1 - 32 * b0] = c
            return whole.unflatten(2, (-1, 32))

        def numbers(i, x, axis):
            if x is None:
                return
            if axis:
                part(i).copy_(x.to(meta).contiguous().view(torch.uint8))
                return
            old = part(i).contiguous().view(meta).unflatten(3, (-1, 32)).transpose(-1, -2).flatten(2, 3)
            old[:, :, q0 - 32 * b0:q1 - 32 * b0] = x.to(meta)
            part(i).copy_(old.unflatten(2, (-1, 32)).transpose(-1, -2).flatten(3).contiguous().view(torch.uint8))
        for first, x, bits, mode, axis, group in (
                (0, K, f["k_bits"], f["k_mode"], f["k_axis"], f["k_group"]),
                (3, V, f["v_bits"], f["v_mode"], 0, f["v_group"])):
            c, sc, z = _coded_values(s, x, bits, mode, axis, group)
            if first:
                old = _unpack8(part(3).unflatten(3, (4, 16, D // 16, bits)), bits)
                c = codes(c, old.permute(0, 1, 2, 3, 6, 5, 4))
                c = c.unflatten(4, (D // 16, 16)).unflatten(3, (4, 8)).permute(0, 1, 2, 3, 6, 5, 4)
            else:
                old = _unpack8(part(0).unflatten(3, (2, 4, 4, 4, D // 32, bits)), bits)
                c = codes(c, old.permute(0, 1, 2, 5, 3, 6, 7, 4, 8))
                c = c.unflatten(4, (D // 32, 4, 8)).unflatten(3, (4, 2, 4)).permute(0, 1, 2, 4, 7, 3, 5, 6, 8)
            part(first).copy_(_pack8(c, bits).flatten(3))
            numbers(first + 1, sc, axis)
            numbers(first + 2, z, axis)
    return {"image": img} if s["Q"] is None else {"image": img, "Q": _turned(s, s["Q"], s["wq"], cos, sin)}


def _unpack8(x, bits):
    """Bytes [..., bits] of a piece -> its eight codes."""
    if bits == 8:
        return x
    shift = (torch.arange(8 // bits, device=x.device) * bits).to(torch.uint8)
    return ((x[..., None] >> shift) & (2 ** bits - 1)).flatten(-2)


def _reconstruct(s, img, U, T, n):
    """The stored keys and values [U, H, n, D] in 32 bits."""
    f, H, D = s["f"], s["H"], s["D"]
    nq, ring, nsink = _coded(f, n), f["residual"] + f["flush"], min(n, f["sink"])
    sec, nb = _sections(f, U, H, D, T)[0], -(-nq // 32)
    size, meta = _block_bytes(f, D), torch.float16 if f["meta_fp16"] else torch.float32

    def part(i):
        return _view(img, sec[i], U, H)[:, :, :size[i] * nb].unflatten(2, (nb, size[i]))

    def numbers(i, channel):
        x = part(i).contiguous().view(meta).float()
        if channel:
            return x[:, :, :, None, :]  # [U, H, block, 1, D]
        g = x.shape[-1] // 32
        return x.unflatten(3, (g, 32)).transpose(-1, -2).repeat_interleave(D // g, dim=-1)  # [U, H, block, 32, D]

    def values(c, i, bits, mode, channel):
        scale = numbers(i + 1, channel)
        x = c * scale + numbers(i + 2, channel) if mode == AFFINE else (c - 2 ** (bits - 1)) * scale
        return x.flatten(2, 3)[:, :, :nq]

    def whole(i, x):
        rows = _view(img, sec[i + 8], U, H)[:, :, :2 * D * nsink].reshape(U, H, nsink, 2 * D)
        parts = [rows.view(torch.float16).float(), x]
        if ring:
            slot = torch.arange(nq, n - nsink, device="cuda") % ring
            parts.append(_view(img, sec[i + 6], U, H).view(torch.float16).view(U, H, ring, D)[:, :, slot].float())
        return torch.cat(parts, 2)
    empty = torch.zeros((U, H, 0, D), device="cuda")
    if nb:
        k = _unpack8(part(0).unflatten(3, (2, 4, 4, 4, D // 32, f["k_bits"])), f["k_bits"]).float()
        k = k.permute(0, 1, 2, 5, 3, 6, 7, 4, 8).reshape(U, H, nb, 32, D)
        v = _unpack8(part(3).unflatten(3, (4, 16, D // 16, f["v_bits"])), f["v_bits"]).float()
        v = v.permute(0, 1, 2, 3, 6, 5, 4).reshape(U, H, nb, 32, D)
        k = values(k, 0, f["k_bits"], f["k_mode"], f["k_axis"])
        v = values(v, 3, f["v_bits"], f["v_mode"], 0)
    else:
        k = v = empty
    return whole(0, k), whole(1, v)


def _hadamard(D):
    """The normalized Sylvester matrix, 32 bits."""
    i = torch.arange(D, device="cuda")
    x = i[:, None] & i[None, :]
    bits = (x[..., None] >> torch.arange(8, device="cuda")) & 1
    return (1.0 - 2.0 * (bits.sum(-1) & 1).float()) * D ** -0.5


def _attention(s):
    """Softmax over a sequence's prefix and the suffix tokens that a row sees; every prefix meets the queries of all its
    sequences in one product."""
    B, P, C, H, D, G = s["B"], s["P"], s["C"], s["H"], s["D"], s["H_q"] // s["H"]
    q = s["Q"].float()
    if s["f"]["rotate"]:
        q = q @ _hadamard(D)
    q = q.view(B, C, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, C * G, D) * s["sm"]
    ks, vs = _reconstruct(s, s["suffix"], B, s["Ts"], s["ns"])

    def by_prefix(x):  # [B, H, rows, E] -> [P, H, most rows, E]
        out = torch.zeros((P, s["most"]) + x.shape[1:], device="cuda")
        out[s["group"], s["slot"]] = x
        return out.transpose(1, 2).flatten(2, 3)

    def by_sequence(x):
        return x.unflatten(2, (s["most"], C * G)).transpose(1, 2)[s["group"], s["slot"]]
    j = torch.arange(C, device="cuda")
    sees = (s["tree"][:, :, j // 32] >> (j % 32).int()) & 1  # [B, C, C]
    sees = sees.bool().repeat_interleave(G, 1)[:, None]
    suf = q @ ks.transpose(-1, -2)
    suf[..., s["ns"] - C:] = torch.where(sees, suf[..., s["ns"] - C:], -math.inf)
    top = suf.amax(-1, keepdim=True)
    if s["np"]:
        kp, vp = _reconstruct(s, s["prefix"], P, s["Tp"], s["np"])
        pre = by_prefix(q) @ kp.transpose(-1, -2)
        top = torch.maximum(top, by_sequence(pre.amax(-1, keepdim=True)))
        pre = (pre - by_prefix(top)).exp_()
    # (a row that sees no token at all is zeros)
    suf = torch.where(suf == -math.inf, 0.0, (suf - top).exp_())
    total, o = suf.sum(-1, keepdim=True), suf @ vs
    if s["np"]:
        total, o = total + by_sequence(pre.sum(-1, keepdim=True)), o + by_sequence(pre @ vp)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(B, H, C, G, D).permute(0, 2, 1, 3, 4).reshape(B, C, s["H_q"], D)
    return o @ _hadamard(D) if s["f"]["rotate"] else o


def work(case):
    D, H_q, H = LAYERS[case["layer"]]
    B = case["B"]
    if case["kind"] == "tree":
        f, C, n = _format(case), case["C"], case["suffix"]
        used = sum(b > a for a, b in zip(_first(case), _first(case)[1:]))  # prefixes that somebody reads
        seen = B * C * (case["prefix"] + n - C) + int(_tree(case, 0)[0].sum())  # (row, token) pairs of a head
        return {"bytes": used * _live_bytes(f, case["prefix"], H, D) + B * _live_bytes(f, n, H, D) + 6 * B * C * H_q * D,
                "flops": 4 * D * H_q * seen}
    heads = (H_q if case.get("queries", True) else 0) + H
    flops = B * case["n"] * heads * (3 * case["rot"] + (4 * D if case["norm"] else 0))
    if case["kind"] == "rope":
        return {"bytes": 4 * B * case["n"] * heads * D, "flops": flops}
    f, n0, n = _format(case), case["cached"], case["n"]
    q0, q1 = _coded(f, n0), _coded(f, n0 + n)
    older = max(0, min(q1, n0 - f["sink"]) - q0) if f["flush"] else 0  # tokens coded from the window
    fp16 = max(0, min(n0 + n, f["sink"]) - n0)
    if f["flush"]:
        fp16 += min(n, f["residual"] + f["flush"])
    packed = sum(_block_bytes(f, D)) * (q1 - q0) // 32 + 4 * D * (fp16 + older)
    queries = 4 * B * n * H_q * D if case["queries"] else 0
    return {"bytes": queries + B * H * (4 * D * n + packed), "flops": flops}


# ---------------------------------------------------------------------- exact

def _wide(f, t):
    """The stored keys and values in 64 bits, from the codes, scales and offsets."""
    def value(c, s, z, bits, group):
        s = s.double().repeat_interleave(group, -1) if group else s.double().repeat_interleave(32, 2)
        if z is None:
            return (c.double() - 2 ** (bits - 1)) * s
        return c.double() * s + (z.double().repeat_interleave(group, -1) if group else z.double().repeat_interleave(32, 2))
    k = value(t["kc"], t["ks"], t["kz"], f["k_bits"], 0 if f["k_axis"] else f["k_group"])
    v = value(t["vc"], t["vs"], t["vz"], f["v_bits"], f["v_group"])
    return (torch.cat([t["sinkK"].double(), k, t["winK"].double()], 2),
            torch.cat([t["sinkV"].double(), v, t["winV"].double()], 2))


def _turn(x):
    """Normalized Walsh-Hadamard transform of the last axis in 64 bits, by butterflies."""
    D, h = x.shape[-1], 1
    while h < D:
        a, b = x.reshape(x.shape[:-1] + (D // (2 * h), 2, h)).unbind(-2)
        x = torch.stack((a + b, a - b), -2).reshape(x.shape)
        h *= 2
    return x / math.sqrt(D)


def _spun(case, s, x, w):
    """Rows normed and rotated in 64 bits, as complex numbers."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
    rot = case["rot"]
    t = torch.remainder(s["pos"].double()[..., None] * torch.from_numpy(_turns(case)).cuda(), 1.0)[:, :, None, :]
    z = x[..., :rot]
    z = z.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else z.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(t), 2 * math.pi * t))
    z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat((z, x[..., rot:]), -1)


def exact(case, seed):
    D, H_q, H = LAYERS[case["layer"]]
    s = None
    if case["kind"] != "tree":
        B, n = case["B"], case["n"]
        s = dict(pos=_positions(case, seed)[0])
        w = [None, None]
        if case["norm"]:
            w = [(1 + 0.2 * _normal(seed, k, (D,)).float()).to(torch.bfloat16) for k in ("wq", "wk")]
        if case["kind"] == "rope":
            return {"Q": _spun(case, s, _normal(seed, "Q", (B, n, H_q, D)), w[0]),
                    "K": _spun(case, s, _normal(seed, "K", (B, n, H, D)), w[1])}
        if not case["queries"]:
            return None  # bytes: codes and metadata are bit-exact functions of the input
        return {"image": None, "Q": _spun(case, s, _normal(seed, "Q", (B, n, H_q, D)), w[0])}
    f, B, C, n, G, first = _format(case), case["B"], case["C"], case["suffix"], H_q // H, _first(case)
    kp, vp = _wide(f, _tokens(case, f, seed, "prefix", case["P"], case["prefix"]))
    ks, vs = _wide(f, _tokens(case, f, seed, "suffix", B, n))
    sees = torch.from_numpy(_tree(case, seed)[0]).cuda()
    Q = _normal(seed, "Q", (B, C, H_q, D)).double()
    out = torch.empty_like(Q)
    for g in range(case["P"]):
        for b in range(first[g], first[g + 1]):
            k, v = torch.cat([kp[g], ks[b]], 1), torch.cat([vp[g], vs[b]], 1)
            q = _turn(Q[b]) if f["rotate"] else Q[b]
            hidden = torch.zeros((C, k.shape[1]), dtype=torch.bool, device="cuda")
            hidden[:, k.shape[1] - C:] = ~sees[b]
            x = torch.einsum("chgd,htd->hgct", q.reshape(C, H, G, D), k) / math.sqrt(D)
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
            out[b] = torch.einsum("hgct,htd->chgd", p, v).reshape(C, H_q, D)
    return _turn(out) if f["rotate"] else out
