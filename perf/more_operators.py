"""Operators around a paged key-value cache held in 8 or 4 bits, and rotary positions with several axes, as cases that can be timed
and checked.

Kinds of case
  store  rows of new tokens into the pages, quantised on the way (prompts of unequal lengths, or one token per sequence), and those
         rows read back as the cache now has them
  read   the first rows of every sequence read back, as a prompt that goes on needs them
  attn   attention of one new token per sequence over the quantised rows; `step`: the token's own row is quantised and written in the
         same call (and read back after it); `weights`: every token's accumulated attention weight is brought up to date
  rope   query and key heads of tokens turned by positions with one to four axes; `inverse`: turned back, which is the gradient

The format: 32 consecutive elements of a row share a power of two (one byte, exponent + 127; 255: the block is NaN).  Elements are
E4M3 ("mxfp8", one byte) or E2M1 ("mxfp4", two to a byte, the even one in the low bits), rounded to the nearest, ties to the even
code.  The shared exponent is the smallest with which no element is off by more than half a step.

Head shapes are those of the benchmark configurations (16 and 32 heads of 128, one query per key head) and generic ones whose query
heads share keys.  Lengths lie evenly on a logarithmic scale between `lo` and `hi`, dealt to the sequences by the seed, so that every
seed has the same work.  Pages are handed out in random order, as in a pool that has been in use.

A pass leaves its inputs as they were: accumulated weights and turned rows go to arrays of their own, and a new row is written where
the pass before wrote it.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BITS = {"mxfp8": 8, "mxfp4": 4}
LOWEST = {"mxfp8": -117, "mxfp4": -125}          # of the shared exponent: every element but 0 is a normal number of fp32 and bf16
LEVELS = {"mxfp4": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0],
          "mxfp8": [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1]}
TOP = {"mxfp8": (0.90625, 9), "mxfp4": (0.875, 3)}        # 464 and 7: half a step above the largest level, as frexp gives them


def _store(name, B, Hkv, d, dtype, fmt, page, lo, hi, held=0, layout="heads"):
    """lo, hi: new tokens of a sequence; held: tokens it holds before."""
    return {"name": name, "kind": "store", "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "fmt": fmt, "page": page, "lo": lo, "hi": hi,
            "held": held, "layout": layout}


def _read(name, B, Hkv, d, dtype, fmt, page, lo, hi, layout="heads"):
    return {"name": name, "kind": "read", "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "fmt": fmt, "page": page, "lo": lo, "hi": hi,
            "layout": layout}


def _attn(name, B, H, Hkv, d, dtype, fmt, page, lo, hi, weights=False, step=False, layout="heads"):
    return {"name": name, "kind": "attn", "B": B, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "fmt": fmt, "page": page, "lo": lo, "hi": hi,
            "weights": weights, "step": step, "layout": layout}


def _rope(name, tokens, H, d, dtype, pairs, axes, layout, far, gap=0, inverse=False):
    """pairs: elements 2 * pairs and beyond of a head stay; far: positions reach that far; gap: elements between two tokens' heads."""
    return {"name": name, "kind": "rope", "tokens": tokens, "H": H, "d": d, "dtype": dtype, "pairs": pairs, "axes": axes, "layout": layout,
            "far": far, "gap": gap, "inverse": inverse}


def listed():
    return [
        # one token for each of a few sequences, fp32 and head_dim 64: what the calls cost
        _store("store_8_tokens_f32", B=8, Hkv=16, d=64, dtype="f32", fmt="mxfp8", page=16, lo=1, hi=1, held=96),
        # prompts of 64 requests admitted together, 7B heads
        _store("store_64_prompts", B=64, Hkv=32, d=128, dtype="bf16", fmt="mxfp4", page=16, lo=20, hi=1500),
        # a few short conversations go on, pages that are no power of two in rows of all heads
        _read("read_6_short_f32", B=6, Hkv=5, d=64, dtype="f32", fmt="mxfp4", page=24, lo=1, hi=300, layout="rows"),
        # prefixes of 32 conversations for their next prompts
        _read("read_32_prefixes", B=32, Hkv=8, d=128, dtype="bf16", fmt="mxfp8", page=16, lo=500, hi=8192),
        # a lone user's pair of guided sequences at the beginning of an image, 1B heads: latency
        _attn("attn_1_prompt", B=2, H=16, Hkv=16, d=128, dtype="bf16", fmt="mxfp4", page=16, lo=64, hi=97),
        # 7B heads, 64 prompts at different places of their images (up to 640 tokens), weights kept for an eviction
        _attn("attn_7b_images", B=128, H=32, Hkv=32, d=128, dtype="bf16", fmt="mxfp4", page=16, lo=64, hi=640, weights=True),
        # few long documents, four query heads per key head: the length has to be split
        _attn("attn_4_long", B=4, H=32, Hkv=8, d=128, dtype="bf16", fmt="mxfp4", page=64, lo=30000, hi=131072),
        # fp32 steps, five query heads per key head, pages that are no power of two in rows of all heads, sequences that hold nothing
        _attn("step_f32_ragged", B=48, H=40, Hkv=8, d=64, dtype="f32", fmt="mxfp8", page=24, lo=0, hi=5000, weights=True, step=True,
              layout="rows"),
        # a busy server's step: 128 conversations, eight query heads per key head, new rows written in the call
        _attn("step_128_chats", B=128, H=32, Hkv=4, d=128, dtype="bf16", fmt="mxfp8", page=32, lo=10, hi=8000, weights=True, step=True),
        # one decode step's heads of 16 sequences, fp32, pairs next to each other, one axis, far positions: latency
        _rope("rope_16_far_f32", tokens=16, H=40, d=64, dtype="f32", pairs=32, axes=1, layout="interleaved", far=1000000),
        # prompts with images: time, height and width; query and key heads of a projection turned where they lie between its values
        _rope("rope_64_prompts", tokens=22500, H=40, d=128, dtype="bf16", pairs=64, axes=3, layout="half", far=20000, gap=1024),
        # the gradient of such rows, an odd number of tokens, a quarter of every head left as it is
        _rope("rope_back_images", tokens=4611, H=32, d=128, dtype="bf16", pairs=48, axes=2, layout="half", far=640, inverse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["store", "read", "attn", "rope"], [3, 2, 6, 3])[0]
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    if kind == "rope":
        d = rng.choice([64, 128, 128, 80, 256])
        H = rng.choice([1, 8, 12, 20, 40, 48])
        tokens = _log(rng, 1, 30000)
        while tokens > 1 and tokens * H * d * size > 200 << 20:
            tokens //= 2
        return {"kind": kind, "tokens": tokens, "H": H, "d": d, "dtype": dtype, "pairs": rng.choice([d // 2, d // 2, d // 8 * 2]),
                "axes": rng.choice([1, 2, 3, 3, 4]), "layout": rng.choice(["half", "half", "interleaved"]), "far": _log(rng, 100, 2000000),
                "gap": rng.choice([0, 0, 2 * d]), "inverse": rng.random() < 0.3}
    d = rng.choice([64, 128, 128])
    fmt = rng.choice(["mxfp4", "mxfp4", "mxfp8"])
    page = rng.choice([16, 16, 32, 64, 128, 8, 24, 1])
    layout = rng.choice(["heads", "heads", "rows"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    B = _log(rng, 1, 128)
    if kind != "attn":
        row = 2 * Hkv * d * size
        hi = rng.choice([1, _log(rng, 2, 2000)]) if kind == "store" else rng.choice([_log(rng, 1, 700), _log(rng, 100, 9000)])
        lo = rng.choice([1, hi, (hi + 1) // 2])
        while B > 1 and B * hi * row > 400 << 20:
            B //= 2
        while hi > 1 and B * hi * row > 400 << 20:
            hi //= 2
        case = {"kind": kind, "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "fmt": fmt, "page": page, "lo": min(lo, hi), "hi": hi, "layout": layout}
        if kind == "store":
            case["held"] = rng.choice([0, _log(rng, 1, 500)])
        return case
    row = 2 * Hkv * d * BITS[fmt] // 8
    G = rng.choice([1, 1, 2, 4, 5, 7, 8, 16])
    hi = rng.choice([_log(rng, 1, 700), _log(rng, 100, 9000), _log(rng, 1000, 100000)])
    lo = rng.choice([0, 1, hi // 3, hi])
    while B > 1 and B * hi * row > 300 << 20:
        B //= 2
    while hi > 1 and B * hi * row > 300 << 20:
        hi //= 2
    return {"kind": kind, "B": B, "H": Hkv * G, "Hkv": Hkv, "d": d, "dtype": dtype, "fmt": fmt, "page": page, "lo": min(lo, hi), "hi": hi,
            "weights": rng.random() < 0.5, "step": rng.random() < 0.4, "layout": layout}


# ---- the format in elementary operations ------------------------------------------------------------------------------

def _tables(fmt, dev):
    """Levels of an element, values of all codes of an element, powers of two by exponent + 127, values of all shared exponents."""
    up = LEVELS[fmt]
    codes = up + ([math.nan] if fmt == "mxfp8" else [])
    power = [2.0 ** (i - 127) for i in range(255)]
    return {"levels": torch.tensor(up, device=dev), "value": torch.tensor(codes + [-x for x in codes], device=dev),
            "power": torch.tensor(power, device=dev), "scale": torch.tensor(power + [math.nan], device=dev)}


def _encode(x, fmt, t):
    """Rows x [..., d] in 32 bits as codes [..., d * bits / 8] and shared exponents [..., d / 32]."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    part, up = torch.frexp(most)
    share, exponent = TOP[fmt]
    E = torch.where(part <= share, up - exponent, up - exponent + 1)
    E = torch.where(most > 0, E, LOWEST[fmt]).clamp(LOWEST[fmt], 127)
    fine = torch.isfinite(most)
    E = torch.where(fine, E, 0)
    y = torch.where(fine, x.abs() * t["power"][127 - E], 0.0)
    low, digits = (0, 1) if fmt == "mxfp4" else (-6, 3)
    step = t["power"][(torch.frexp(y)[1] - 1).clamp(min=low) - digits + 127]
    y = (torch.round(y / step) * step).clamp(max=LEVELS[fmt][-1])
    code = torch.searchsorted(t["levels"], y).to(torch.uint8) | (torch.signbit(x) & fine).to(torch.uint8) << BITS[fmt] - 1
    code = code.flatten(-2)
    if fmt == "mxfp4":
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code, torch.where(fine, E + 127, 255).to(torch.uint8).squeeze(-1)


def _decode(code, scale, fmt, t):
    """Codes and shared exponents as the values they stand for, in 32 bits."""
    if fmt == "mxfp4":
        code = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    x = t["value"][code.int()].unflatten(-1, (-1, 32))
    return (x * t["scale"][scale.int()].unsqueeze(-1)).flatten(-2)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _lengths(n, lo, hi):
    """n whole numbers from lo to hi, evenly on a logarithmic scale, the longest first."""
    a = math.log(lo + 1.0)
    b = math.log(hi + 1.0)
    return [min(hi, max(lo, int(round(math.exp(b - (b - a) * (i / (n - 1) if n > 1 else 0.0)) - 1)))) for i in range(n)]


def _shuffled(v, seed):
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(len(v))
    return [v[i] for i in order]


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _pool(case, n_pages, g, dev, t, fill):
    """One pool: codes [pages, kv heads, page, bytes] (a view of [pages, page, kv heads, bytes] in layout "rows") and shared exponents."""
    Hkv, page, d, fmt = case["Hkv"], case["page"], case["d"], case["fmt"]
    row = d * BITS[fmt] // 8
    per = (n_pages, page, Hkv, row) if case["layout"] == "rows" else (n_pages, Hkv, page, row)
    codes = torch.zeros(per, dtype=torch.uint8, device=dev)
    scales = torch.full((n_pages, Hkv, page, d // 32), 127, dtype=torch.uint8, device=dev)
    codes = codes.transpose(1, 2) if case["layout"] == "rows" else codes
    if fill:
        some = max(1, (64 << 20) // (Hkv * page * d))              # pages at a time
        for p in range(0, n_pages, some):
            x = torch.randn((min(some, n_pages - p), Hkv, page, d), device=dev, generator=g)
            codes[p:p + some], scales[p:p + some] = _encode(x, fmt, t)
    return codes, scales


def _weights(shape, g, dev):
    """Accumulated attention weights: a few tokens have most of them, one in sixteen has none yet."""
    w = torch.rand(shape, device=dev, generator=g).clamp_(min=1e-6).pow_(-0.7).sub_(1.0)
    return w.masked_fill_(torch.rand(shape, device=dev, generator=g) < 1 / 16, 0.0)


def _rows(n, case, g, dev):
    """Rows of n tokens' keys or values: a few channels of every head are ten times larger than the others."""
    x = torch.randn((n, case["Hkv"], case["d"]), device=dev, generator=g)
    x[..., 5::37] *= 10.0
    return x.to(DTYPES[case["dtype"]])


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    if case["kind"] == "rope":
        return _prepare_rope(case, g, dev)
    kind, page, fmt, B = case["kind"], case["page"], case["fmt"], case["B"]
    lens = _shuffled(_lengths(B, case["lo"], case["hi"]), seed)
    held = [x + case["held"] for x in lens] if kind == "store" else lens
    t = _tables(fmt, dev)
    s = {"case": case, "tables": t, "lens": lens}
    blocks = [-(-n // page) for n in held]
    n_pages = sum(blocks) + 3
    order = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32).cpu().numpy()
    table = np.full((B, max(max(blocks), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = torch.from_numpy(table).to(dev)
    s["k"], s["k_scales"] = _pool(case, n_pages, g, dev, t, kind != "store")
    s["v"], s["v_scales"] = _pool(case, n_pages, g, dev, t, kind != "store")
    s["seq_len"] = _ints(held, dev)
    places = (n_pages, case["Hkv"], page)
    # rows that are read back: which sequence each belongs to, and its slot
    back = [1 if n else 0 for n in lens] if kind == "attn" else lens
    first = [n - m for n, m in zip(held, back)]
    n = sum(back)
    s["first"], s["start"] = _ints(first, dev), _ints(np.concatenate([[0], np.cumsum(back)]).tolist(), dev)
    if kind == "attn":
        s["q"] = torch.randn((B, case["H"], case["d"]), device=dev, generator=g).mul_(1.5).to(DTYPES[case["dtype"]])
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, case["H"]), device=dev)
        if case["weights"]:
            s["weight"] = _weights(places, g, dev)
            s["weight_out"] = torch.zeros_like(s["weight"])
    if kind == "store" or (kind == "attn" and case["step"]):
        s["k_new"], s["v_new"] = (_rows(n if kind == "store" else B, case, g, dev) for _ in range(2))
        s["pos"] = torch.full(places, -1, dtype=torch.int32, device=dev)
        s["seq_pos"] = s["seq_len"] + 5              # a few tokens were evicted before
    if kind != "attn" or case["step"]:
        s["k_back"], s["v_back"] = (torch.zeros((n, case["Hkv"], case["d"]), dtype=DTYPES[case["dtype"]], device=dev) for _ in range(2))
        s["owner"] = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(back, device=dev))
        s["slot"] = torch.arange(n, device=dev) - s["start"].long()[s["owner"]] + s["first"].long()[s["owner"]]
    if own:
        import paper_2510_18716_amd as ssd
        per = 8 // BITS[fmt]                         # elements of a byte
        k = s["k"]
        s["cfg"] = ssd.make_paged_config(B, case.get("H", case["Hkv"]), case["Hkv"], case["d"], case["dtype"], page, n_pages, s["table"].shape[1],
                                         page_stride=k.stride(0) * per, head_stride=k.stride(1) * per, row_stride=k.stride(2) * per)
        need = ssd.ssd_paged_mx_workspace_bytes(s["cfg"], fmt, max(1, case["hi"]), case["weights"]) if kind == "attn" else 0
        s["work"] = torch.zeros(max(256, need), dtype=torch.uint8, device=dev)
    return s


def _prepare_rope(case, g, dev):
    n, H, d, pairs, axes = case["tokens"], case["H"], case["d"], case["pairs"], case["axes"]
    wide = H * d + case["gap"]                       # the projection's row
    s = {"case": case}
    s["rows"] = torch.randn((n, wide), device=dev, generator=g).to(DTYPES[case["dtype"]])
    s["x"] = s["rows"][:, :H * d].unflatten(1, (H, d))
    s["out"] = torch.zeros((n, H, d), dtype=s["x"].dtype, device=dev)
    s["pos"] = torch.randint(0, case["far"], (axes, n), device=dev, generator=g).to(torch.int32)
    # the axes take the pairs in runs, each of them from fast to slow ones
    s["axis"] = torch.tensor([i * axes // pairs for i in range(pairs)], dtype=torch.uint8, device=dev)
    s["inv_freq"] = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], device=dev)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    return {"store": _run_store, "read": _run_read, "attn": _run_attn, "rope": _run_rope}[s["case"]["kind"]](s)


def _place(s, owner, slot):
    """Page and place in the page of slots of sequences."""
    page = s["case"]["page"]
    return s["table"][owner, slot // page].long().clamp(min=0), slot % page


def _read_back(s):
    if own:
        import paper_2510_18716_amd as ssd
        ssd.ssd_paged_mx_read(s["cfg"], s["case"]["fmt"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"], s["seq_len"],
                              s["k_back"], s["v_back"], row_start=s["start"], first_slot=s["first"])
    else:
        page, place = _place(s, s["owner"], s["slot"])
        s["k_back"].copy_(_decode(s["k"][page, :, place], s["k_scales"][page, :, place], s["case"]["fmt"], s["tables"]))
        s["v_back"].copy_(_decode(s["v"][page, :, place], s["v_scales"][page, :, place], s["case"]["fmt"], s["tables"]))
    return {"k": s["k_back"], "v": s["v_back"]}


def _write(s, owner, slot, k_new, v_new):
    """New rows into their places, in the plain form."""
    page, place = _place(s, owner, slot)
    fmt, t = s["case"]["fmt"], s["tables"]
    s["k"][page, :, place], s["k_scales"][page, :, place] = _encode(k_new.float(), fmt, t)
    s["v"][page, :, place], s["v_scales"][page, :, place] = _encode(v_new.float(), fmt, t)
    s["pos"][page, :, place] = (s["seq_pos"][owner] - s["seq_len"][owner] + slot).to(torch.int32)[:, None].expand(-1, s["case"]["Hkv"])


def _run_store(s):
    if own:
        import paper_2510_18716_amd as ssd
        ssd.ssd_paged_mx_append(s["cfg"], s["case"]["fmt"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"], s["seq_len"],
                                s["k_new"], s["v_new"], pos=s["pos"], seq_pos=s["seq_pos"], new_start=s["start"])
    else:
        _write(s, s["owner"], s["slot"], s["k_new"], s["v_new"])
    return {**_read_back(s), "pos": s["pos"]}


def _run_read(s):
    return _read_back(s)


def _run_attn(s):
    case = s["case"]
    if own:
        import paper_2510_18716_amd as ssd
        more = {"lse": s["lse"], "max_len": max(1, case["hi"]), "workspace": s["work"]}
        if case["weights"]:
            more.update(weight_in=s["weight"], weight_out=s["weight_out"])
        if case["step"]:
            ssd.ssd_paged_mx_decode_step(s["cfg"], case["fmt"], s["q"], s["k_new"], s["v_new"], s["k"], s["v"], s["k_scales"], s["v_scales"],
                                         s["table"], s["seq_len"], s["out"], pos=s["pos"], seq_pos=s["seq_pos"], **more)
        else:
            ssd.ssd_paged_mx_decode_attn(s["cfg"], case["fmt"], s["q"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"],
                                         s["seq_len"], s["out"], **more)
    else:
        B, Hkv, d, most = case["B"], case["Hkv"], case["d"], max(1, case["hi"])
        G = case["H"] // Hkv
        if case["step"]:
            _write(s, s["owner"], s["slot"], s["k_new"][s["owner"]], s["v_new"][s["owner"]])
        slot = torch.arange(most, device=s["q"].device)
        there = slot[None] < s["seq_len"][:, None]                                             # [B, most]
        page, place = _place(s, torch.arange(B, device=slot.device)[:, None], torch.where(there, slot[None], 0))
        k = _decode(s["k"][page, :, place], s["k_scales"][page, :, place], case["fmt"], s["tables"]).transpose(1, 2).contiguous()
        q = s["q"].float().reshape(B, Hkv, G, d).transpose(2, 3).contiguous()
        x = torch.matmul(k, q) * d ** -0.5                                                     # [B, kv heads, most, G]
        del k
        x = torch.where(there[:, None, :, None], x, -math.inf)
        top = x.amax(2, keepdim=True)
        e = torch.where(there[:, None, :, None], torch.exp(x - top), 0.0)
        total = e.sum(2, keepdim=True)
        p = torch.where(total > 0, e / total, 0.0)
        v = _decode(s["v"][page, :, place], s["v_scales"][page, :, place], case["fmt"], s["tables"]).transpose(1, 2).contiguous()
        s["out"].copy_(torch.matmul(p.transpose(2, 3).contiguous(), v).reshape(B, case["H"], d))
        s["lse"].copy_(torch.where(total > 0, top + torch.log(total), -math.inf).reshape(B, case["H"]))
        if case["weights"]:
            before = s["weight"][page, :, place]                                               # [B, most, kv heads]
            if case["step"]:                                                                   # the new token has none yet
                before = torch.where((slot[None] == s["seq_len"][:, None] - 1)[..., None], 0.0, before)
            s["weight_out"][page[there], :, place[there]] = (before + p.sum(3).transpose(1, 2))[there]
    got = {"out": s["out"], "lse": s["lse"]}
    if case["weights"]:
        got["weight"] = s["weight_out"]
    if case["step"]:
        got.update(_read_back(s), pos=s["pos"])
    return got


def _run_rope(s):
    case = s["case"]
    if own:
        import paper_2510_18716_amd as ssd
        layout = ssd.SSD_ROPE_HALF if case["layout"] == "half" else ssd.SSD_ROPE_INTERLEAVED
        ssd.ssd_rope_axes(s["x"], s["out"], case["tokens"], case["H"], case["d"], case["dtype"], s["pos"], s["inv_freq"], axis=s["axis"],
                          n_axes=case["axes"], layout=layout, inverse=case["inverse"])
    else:
        pairs = case["pairs"]
        angle = s["pos"].double()[s["axis"].int()].t() * s["inv_freq"].double()                # [tokens, pairs], in 64 bits: far positions
        c, w = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        w = -w if case["inverse"] else w
        x = s["x"].float()
        if case["layout"] == "half":
            a, b = x[..., :pairs], x[..., pairs:2 * pairs]
            turned = torch.cat([a * c - b * w, b * c + a * w], -1)
        else:
            a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
            turned = torch.stack([a * c - b * w, b * c + a * w], -1).flatten(-2)
        s["out"].copy_(torch.cat([turned, x[..., 2 * pairs:]], -1))
    return {"out": s["out"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rope":
        n = case["tokens"] * case["H"]
        return {"bytes": 2 * n * case["d"] * size + 4 * case["tokens"] * case["axes"], "flops": 6 * n * case["pairs"]}
    lens = _lengths(case["B"], case["lo"], case["hi"])
    n, plain = sum(lens), case["d"] * size
    row = case["d"] * BITS[case["fmt"]] // 8 + case["d"] // 32      # codes and shared exponents
    blocks = 4 * sum(-(-x // case["page"]) for x in lens)
    if case["kind"] == "store":                                     # new rows in, pages out; the same back
        return {"bytes": n * case["Hkv"] * (4 * plain + 4 * row + 4) + blocks, "flops": 0}
    if case["kind"] == "read":
        return {"bytes": n * case["Hkv"] * 2 * (plain + row) + blocks, "flops": 0}
    got = n * case["Hkv"] * (2 * row + (8 if case["weights"] else 0)) + 2 * case["B"] * case["H"] * plain + blocks
    if case["step"]:
        got += case["B"] * case["Hkv"] * (4 * plain + 4 * row)
    return {"bytes": got, "flops": 4 * n * case["H"] * case["d"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"store": _exact_store, "read": _exact_back, "attn": _exact_attn, "rope": _exact_rope}[case["kind"]](s, case)


def _two_to(e):
    """2^e in 64 bits, exactly (torch.ldexp takes a power function's result)."""
    return torch.tensor([2.0 ** i for i in range(-400, 401)], dtype=torch.float64, device=e.device)[e.long() + 400]


def _held(x, fmt):
    """The values that rows x stand for once they are held, in 64 bits: the nearest of all levels, by distance."""
    x = x.double()
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    most = blocks.abs().amax(-1)
    half = 464.0 if fmt == "mxfp8" else 7.0
    E = torch.full(most.shape, LOWEST[fmt], dtype=torch.float64, device=x.device)
    for _ in range(400):                                            # the smallest exponent that reaches
        low = half * _two_to(E) < most
        if not bool(low.any()):
            break
        E += low
    unit = _two_to(E)[..., None]
    y = (blocks / unit).abs()
    levels = torch.tensor(LEVELS[fmt], dtype=torch.float64, device=x.device)
    up = torch.bucketize(y, levels).clamp(max=len(levels) - 1)      # levels[up - 1] < y <= levels[up]
    down = (up - 1).clamp(min=0)
    to_up, to_down = (levels[up] - y).abs(), (y - levels[down]).abs()
    pick = torch.where((to_up < to_down) | ((to_up == to_down) & (up % 2 == 0)), up, down)
    return (torch.copysign(levels[pick], blocks) * unit).reshape(x.shape)


def _values(codes, scales, fmt):
    """What stored rows stand for, in 64 bits, from the fields of their codes."""
    c = codes.long()
    if fmt == "mxfp4":
        c = torch.stack((c % 16, c // 16), -1).reshape(c.shape[:-1] + (-1,))
        sign, e, m, bias, digits = c // 8, c // 2 % 4, c % 2, 1, 1
    else:
        sign, e, m, bias, digits = c // 128, c // 8 % 16, c % 8, 7, 3
    sub = (e == 0).double()
    x = ((1 - sub) + m.double() / 2 ** digits) * _two_to(torch.where(e == 0, 1, e) - bias) * (1 - 2 * sign.double())
    return x * _two_to(scales.long().repeat_interleave(32, -1) - 127)


def _exact_new(s, case, rows):
    lens = s["seq_len"].tolist()
    pos = s["pos"].clone()
    for b, n in enumerate(lens):
        for at in (torch.arange(n - rows[b], n, device=pos.device),):
            pos[s["table"][b].long()[at // case["page"]], :, at % case["page"]] = (at + 5).to(torch.int32)[:, None]
    return pos


def _exact_store(s, case):
    return {"k": _held(s["k_new"], case["fmt"]), "v": _held(s["v_new"], case["fmt"]), "pos": _exact_new(s, case, s["lens"])}


def _sequence(s, case, name, b, n):
    """The n first rows of a sequence [n, kv heads, d]."""
    i = torch.arange(n, device=s["table"].device)
    page, place = s["table"][b].long()[i // case["page"]], i % case["page"]
    return _values(s[name][page, :, place], s[name + "_scales"][page, :, place], case["fmt"])


def _exact_back(s, case):
    return {name: torch.cat([_sequence(s, case, name, b, n) for b, n in enumerate(s["lens"])]) for name in ("k", "v")}


def _exact_attn(s, case):
    G, Hkv = case["H"] // case["Hkv"], case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=out.device)
    got = {"out": out, "lse": lse}
    after = torch.zeros(s["weight"].shape, dtype=torch.float64, device=out.device) if case["weights"] else None
    new = {x: _held(s[x + "_new"], case["fmt"]) for x in "kv"} if case["step"] else None
    for b, n in enumerate(s["lens"]):
        if n == 0:
            continue
        k, v = _sequence(s, case, "k", b, n), _sequence(s, case, "v", b, n)
        if new:
            k[n - 1], v[n - 1] = new["k"][b], new["v"][b]
        i = torch.arange(n, device=out.device)
        page, place = s["table"][b].long()[i // case["page"]], i % case["page"]
        for h in range(Hkv):
            z = k[:, h] @ s["q"][b, h * G:(h + 1) * G].double().t() / math.sqrt(case["d"])
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, 0)
            p = torch.softmax(z, 0)
            out[b, h * G:(h + 1) * G] = p.t() @ v[:, h]
            if case["weights"]:
                w = s["weight"][page, h, place].double()
                if new:
                    w[n - 1] = 0
                after[page, h, place] = w + p.sum(1)
    if case["weights"]:
        got["weight"] = after
    if case["step"]:
        some = torch.tensor([n > 0 for n in s["lens"]], device=out.device)
        got.update(k=new["k"][some], v=new["v"][some], pos=_exact_new(s, case, [min(n, 1) for n in s["lens"]]))
    return got


def _exact_rope(s, case):
    pairs, x = case["pairs"], s["x"].double().clone()
    for i in range(pairs):
        i0, i1 = (i, i + pairs) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        angle = s["pos"][int(s["axis"][i])].double() * float(s["inv_freq"][i]) * (-1 if case["inverse"] else 1)
        z = torch.complex(x[:, :, i0], x[:, :, i1]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        x[:, :, i0], x[:, :, i1] = z.real, z.imag
    return {"out": x}
