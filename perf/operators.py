"""Operators of a serving step over a batch of unequal lengths, as cases that can be timed and checked.

Kinds of case
  append   rows of new tokens into a paged key-value cache: prompts of unequal lengths, or one token per sequence
  attn     attention of one new token per sequence over the paged cache; `step`: the token's own row is written in the same
           call; `weights`: every token's accumulated attention weight is brought up to date
  evict    each sequence is cut to its budget: the tokens of the largest accumulated weight stay
  logits   penalties for repeated tokens, bias, temperature and grammar mask; `guided`: on the guided mix of two rows

Head shapes are those of the benchmark configurations (16 and 32 heads of 128, one query per key head) and generic ones whose
query heads share keys.  Lengths lie evenly on a logarithmic scale between `lo` and `hi`, dealt to the sequences by the seed, so
that every seed has the same work.  Pages are handed out in random order, as in a pool that has been in use.

A pass leaves its inputs as they were: accumulated weights and tables go to arrays of their own, and a moved or new row is
written where the pass before wrote it.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _append(name, B, Hkv, d, dtype, page, lo, hi, held=0, layout="heads", weights=True):
    """lo, hi: new tokens of a sequence; held: tokens it holds before."""
    return {"name": name, "kind": "append", "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": lo, "hi": hi, "held": held,
            "layout": layout, "weights": weights}


def _attn(name, B, H, Hkv, d, dtype, page, lo, hi, weights=False, step=False, layout="heads"):
    return {"name": name, "kind": "attn", "B": B, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": lo, "hi": hi,
            "weights": weights, "step": step, "layout": layout}


def _evict(name, B, Hkv, d, dtype, page, lo, hi, budget, sink, recent, layout="heads"):
    return {"name": name, "kind": "evict", "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": lo, "hi": hi, "budget": budget,
            "sink": sink, "recent": recent, "layout": layout}


def _logits(name, rows, V, dtype, history, prompt, guided=False, bias="none", mask=False):
    """rows: output rows; history: most tokens of a row, prompt: how many of them are its prompt's; bias: none, shared or row."""
    return {"name": name, "kind": "logits", "rows": rows, "V": V, "dtype": dtype, "history": history, "prompt": prompt, "guided": guided,
            "bias": bias, "mask": mask}


def listed():
    return [
        # one token for each of a few sequences, fp32 and head_dim 64: what one call costs
        _append("append_8_tokens_f32", B=8, Hkv=16, d=64, dtype="f32", page=16, lo=1, hi=1, held=96),
        # prompts of 64 requests admitted together, 7B heads, with the weights their prompt scores gave
        _append("append_64_prompts", B=64, Hkv=32, d=128, dtype="bf16", page=16, lo=20, hi=1500),
        # a lone user's pair of guided sequences at the beginning of an image, 1B heads: latency
        _attn("attn_1_prompt", B=2, H=16, Hkv=16, d=128, dtype="bf16", page=16, lo=64, hi=97),
        # 7B heads, 64 prompts at different places of their images (up to 640 tokens), weights kept for an eviction
        _attn("attn_7b_images", B=128, H=32, Hkv=32, d=128, dtype="bf16", page=16, lo=64, hi=640, weights=True),
        # few long documents, four query heads per key head: the length has to be split
        _attn("attn_4_long", B=4, H=32, Hkv=8, d=128, dtype="bf16", page=64, lo=30000, hi=131072),
        # fp32, five query heads per key head, pages that are no power of two in rows of all heads, sequences that hold nothing
        _attn("attn_f32_ragged", B=48, H=40, Hkv=8, d=64, dtype="f32", page=24, lo=0, hi=5000, weights=True, layout="rows"),
        # a busy server's step: 128 conversations, eight query heads per key head, new rows written in the call
        _attn("step_128_chats", B=128, H=32, Hkv=4, d=128, dtype="bf16", page=32, lo=10, hi=8000, weights=True, step=True),
        # one token goes for every one that came, 1B heads, 16 prompts
        _evict("evict_one", B=32, Hkv=16, d=128, dtype="bf16", page=16, lo=129, hi=129, budget=128, sink=1, recent=8),
        # prompts cut to a budget after they were read; the short ones keep everything
        _evict("evict_32_prompts", B=32, Hkv=8, d=128, dtype="bf16", page=16, lo=500, hi=8192, budget=1024, sink=4, recent=64),
        # two long documents down to a sixth
        _evict("evict_2_long", B=2, Hkv=8, d=128, dtype="bf16", page=64, lo=70001, hi=100000, budget=16000, sink=4, recent=512),
        # guided image tokens of 64 prompts, an image so far as history
        _logits("logits_64_guided", rows=64, V=16384, dtype="bf16", history=576, prompt=0, guided=True),
        # text of 256 requests under grammars, an odd vocabulary, long histories, a bias shared by all
        _logits("logits_256_grammar", rows=256, V=128257, dtype="f32", history=8000, prompt=2000, bias="shared", mask=True),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n


def draw(rng):
    return {k: 3071 if v == 3072 else v for k, v in _draw(rng).items()}


def _draw(rng):
    kind = rng.choices(["append", "attn", "evict", "logits"], [2, 5, 3, 2])[0]
    if kind == "logits":
        V = rng.choice([16384, _log(rng, 1000, 200000), _log(rng, 1000, 200000)])
        rows = _log(rng, 1, 256)
        while rows > 1 and rows * V > 30 << 20:
            rows //= 2
        history = _log(rng, 1, 16000)
        return {"kind": kind, "rows": rows, "V": V, "dtype": rng.choice(["bf16", "f32"]), "history": history,
                "prompt": rng.choice([0, history // 3]), "guided": rng.random() < 0.4, "bias": rng.choice(["none", "shared", "row"]),
                "mask": rng.random() < 0.5}
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 16, 32, 64, 128, 8, 24, 1])
    layout = rng.choice(["heads", "heads", "rows"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    row = 2 * Hkv * d * (2 if dtype == "bf16" else 4)
    B = _log(rng, 1, 128)
    if kind == "append":
        hi = rng.choice([1, _log(rng, 2, 2000)])
        lo = rng.choice([1, hi, (hi + 1) // 2])
        while B > 1 and B * hi * row > 1 << 30:
            B //= 2
        return {"kind": kind, "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": min(lo, hi), "hi": hi,
                "held": rng.choice([0, _log(rng, 1, 500)]), "layout": layout, "weights": rng.random() < 0.7}
    if kind == "attn":
        G = rng.choice([1, 1, 2, 4, 5, 7, 8, 16])
        hi = rng.choice([_log(rng, 1, 700), _log(rng, 100, 9000), _log(rng, 1000, 100000)])
        lo = rng.choice([0, 1, hi // 3, hi])
        step = rng.random() < 0.4
        while B > 1 and B * hi * row > 1 << 30:
            B //= 2
        while hi > 1 and B * hi * row > 1 << 30:
            hi //= 2
        return {"kind": kind, "B": B, "H": Hkv * G, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": min(lo, hi), "hi": hi,
                "weights": rng.random() < 0.5, "step": step, "layout": layout}
    hi = rng.choice([_log(rng, 2, 700), _log(rng, 100, 9000), _log(rng, 1000, 100000)])
    budget = rng.choice([hi - 1, max(1, hi // 2), max(1, hi // 6), _log(rng, 1, hi)])
    lo = rng.choice([1, budget, min(hi, budget + 1), hi])
    while B > 1 and B * hi * row > 1 << 30:
        B //= 2
    while hi > 2 and B * hi * row > 1 << 30:
        hi //= 2
    return {"kind": kind, "B": B, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "lo": max(1, min(lo, hi)), "hi": hi,
            "budget": min(budget, hi), "sink": rng.choice([0, 1, 4]), "recent": min(rng.choice([0, 1, 8, 64]), hi), "layout": layout}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _lengths(n, lo, hi):
    """n whole numbers from lo to hi, evenly on a logarithmic scale, the longest first."""
    a = math.log(lo + 1.0)
    b = math.log(hi + 1.0)
    v = [min(hi, max(lo, int(round(math.exp(b - (b - a) * (i / (n - 1) if n > 1 else 0.0)) - 1)))) for i in range(n)]
    return [x - 1 if x == 3072 else x for x in v]


def _generator(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def _shuffled(v, seed):
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(len(v))
    return [v[i] for i in order]


def _pages(case, lens, g, dev, fill=True):
    """The pool's keys and values [pages, kv heads, page, d] (a view of [pages, page, kv heads, d] in layout "rows") and a block
    table with pages in random order, -1 where a sequence has none."""
    dtype, page = DTYPES[case["dtype"]], case["page"]
    blocks = [-(-n // page) for n in lens]
    n_pages = sum(blocks) + 3
    per = [n_pages, case["Hkv"], page, case["d"]]
    if case["layout"] == "rows":
        per = [n_pages, page, case["Hkv"], case["d"]]
    pools = [torch.randn(per, device=dev, dtype=dtype, generator=g) if fill else torch.zeros(per, device=dev, dtype=dtype) for _ in range(2)]
    order = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32).cpu().numpy()
    table = np.full((len(lens), max(max(blocks), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = [p.transpose(1, 2) if case["layout"] == "rows" else p for p in pools]
    return k, v, torch.from_numpy(table).to(dev)


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _weights(shape, g, dev):
    """Accumulated attention weights: a few tokens have most of them, one in sixteen has none yet."""
    w = torch.rand(shape, device=dev, generator=g).clamp_(min=1e-6).pow_(-0.7).sub_(1.0)
    return w.masked_fill_(torch.rand(shape, device=dev, generator=g) < 1 / 16, 0.0)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = _generator(seed, dev)
    kind = case["kind"]
    if kind == "logits":
        return _prepare_logits(case, seed, g, dev)
    lens = _shuffled(_lengths(case["B"], case["lo"], case["hi"]), seed)
    s = {"case": case}
    if kind == "append":
        s["new"], n = lens, sum(lens)
        s["len"] = [x + case["held"] for x in lens]
        s["k_new"], s["v_new"] = (torch.randn((n, case["Hkv"], case["d"]), device=dev, generator=g).to(DTYPES[case["dtype"]]) for _ in range(2))
        s["start"] = _ints(np.concatenate([[0], np.cumsum(lens)]).tolist(), dev)
        s["weight_new"] = _weights((n, case["Hkv"]), g, dev) if case["weights"] else None
        s["max_new"] = case["hi"]
    else:
        s["len"] = lens
    s["k"], s["v"], s["table"] = _pages(case, s["len"], g, dev, fill=kind != "append")
    tables = (s["k"].shape[0], case["Hkv"], case["page"])
    s["seq_len"] = _ints(s["len"], dev)
    if kind == "append":
        s["seq_pos"] = s["seq_len"]
        s["pos"] = torch.full(tables, -1, dtype=torch.int32, device=dev)
        s["weight"] = torch.zeros(tables, device=dev)
    if kind == "attn":
        s["q"] = torch.randn((case["B"], case["H"], case["d"]), device=dev, generator=g).mul_(1.5).to(DTYPES[case["dtype"]])
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((case["B"], case["H"]), device=dev)
        if case["weights"]:
            s["weight"] = _weights(tables, g, dev)
            s["weight_out"] = torch.zeros_like(s["weight"])
        if case["step"]:
            s["k_new"], s["v_new"] = (torch.randn((case["B"], case["Hkv"], case["d"]), device=dev, generator=g).to(DTYPES[case["dtype"]])
                                      for _ in range(2))
            s["pos"] = torch.zeros(tables, dtype=torch.int32, device=dev)
            s["seq_pos"] = s["seq_len"] + 5          # a few tokens were evicted before
    if kind == "evict":
        # slots are in the order of arrival, a few positions having left before; the oldest are still there
        s["weight"] = _weights(tables, g, dev)
        s["pos"] = torch.zeros(tables, dtype=torch.int32, device=dev)
        gone = 7
        for b, n in enumerate(lens):
            i = torch.arange(n, device=dev)
            at = torch.where(i < n // 2, i, i + gone).to(torch.int32)
            s["pos"][s["table"][b].long()[i // case["page"]], :, i % case["page"]] = at[:, None]
        s["seq_pos"] = s["seq_len"] + gone
        s["budget"] = torch.full((case["B"],), case["budget"], dtype=torch.int32, device=dev)
        s["pos_out"], s["weight_out"] = torch.zeros_like(s["pos"]), torch.zeros_like(s["weight"])
        s["len_out"] = torch.zeros_like(s["seq_len"])
    if own:
        import paper_2510_18716_amd as ssd
        k = s["k"]
        s["cfg"] = ssd.make_paged_config(case["B"], case.get("H", case["Hkv"]), case["Hkv"], case["d"], case["dtype"], case["page"], k.shape[0],
                                         s["table"].shape[1], page_stride=k.stride(0), head_stride=k.stride(1), row_stride=k.stride(2))
        size = 0
        if kind == "attn":
            size = ssd.ssd_paged_workspace_bytes(s["cfg"], max(1, case["hi"]), case["weights"])
        if kind == "evict":
            size = ssd.ssd_paged_evict_workspace_bytes(s["cfg"], case["hi"])
        s["work"] = torch.zeros(max(256, size), dtype=torch.uint8, device=dev)
    return s


def _prepare_logits(case, seed, g, dev):
    rows, V, most = case["rows"], case["V"], case["history"]
    n_in = rows * (2 if case["guided"] else 1)
    s = {"case": case, "logits": torch.randn((n_in, V), device=dev, generator=g).mul_(3.0).to(DTYPES[case["dtype"]])}
    # histories: frequent tokens come often, the rest of a row's places are padding
    s["n_tokens"] = _ints(_shuffled(_lengths(rows, max(1, most // 8), most), seed), dev)
    s["tokens"] = (torch.rand((rows, most), device=dev, generator=g).pow_(3.0) * V).to(torch.int32).clamp_(max=V - 1)
    s["tokens"].masked_fill_(torch.arange(most, device=dev)[None] >= s["n_tokens"][:, None], -1)
    s["n_prompt"] = torch.clamp(s["n_tokens"], max=case["prompt"])
    s["repetition"] = torch.rand(rows, device=dev, generator=g) * 0.5 + 1.0
    s["presence"] = torch.rand(rows, device=dev, generator=g) * 0.6
    s["frequency"] = torch.rand(rows, device=dev, generator=g) * 0.2
    s["temperature"] = torch.rand(rows, device=dev, generator=g) * 0.9 + 0.6
    s["bias"] = None if case["bias"] == "none" else torch.randn((1 if case["bias"] == "shared" else rows, V), device=dev, generator=g)
    if case["mask"]:
        words = -(-V // 32)
        few = torch.rand((rows, words), device=dev, generator=g) < 0.9       # most of the vocabulary is forbidden
        s["mask"] = torch.randint(-(1 << 31), 1 << 31, (rows, words), device=dev, generator=g).to(torch.int32).masked_fill_(few, 0)
    else:
        s["mask"] = None
    s["gamma"] = 4.0 if case["guided"] else None
    s["out"] = torch.zeros((rows, V), device=dev)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    return {"append": _run_append, "attn": _run_attn, "evict": _run_evict, "logits": _run_logits}[s["case"]["kind"]](s)


def _places(s, b, first, last):
    """Page and place in the page of the slots first .. last - 1 of sequence b."""
    i = torch.arange(first, last, device=s["table"].device)
    return s["table"][b].long()[i // s["case"]["page"]], i % s["case"]["page"]


def _run_append(s):
    if own:
        import paper_2510_18716_amd as ssd
        ssd.ssd_paged_append(s["cfg"], s["k"], s["v"], s["table"], s["seq_len"], s["k_new"], s["v_new"], pos=s["pos"], weight=s["weight"],
                             seq_pos=s["seq_pos"], new_start=s["start"], weight_new=s["weight_new"])
    else:
        at = 0
        for b, n in enumerate(s["new"]):
            page, place = _places(s, b, s["len"][b] - n, s["len"][b])
            s["k"][page, :, place] = s["k_new"][at:at + n]
            s["v"][page, :, place] = s["v_new"][at:at + n]
            first = s["seq_pos"][b] - n
            s["pos"][page, :, place] = (first + torch.arange(n, device=page.device, dtype=torch.int32))[:, None].expand(n, s["case"]["Hkv"])
            s["weight"][page, :, place] = s["weight_new"][at:at + n] if s["weight_new"] is not None else 0.0
            at += n
    return {"k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}


def _run_attn(s):
    case = s["case"]
    if own:
        import paper_2510_18716_amd as ssd
        more = {"lse": s["lse"], "max_len": max(1, case["hi"]), "workspace": s["work"]}
        if case["weights"]:
            more.update(weight_in=s["weight"], weight_out=s["weight_out"])
        if case["step"]:
            ssd.ssd_paged_decode_step(s["cfg"], s["q"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["seq_len"], s["out"],
                                      pos=s["pos"], seq_pos=s["seq_pos"], **more)
        else:
            ssd.ssd_paged_decode_attn(s["cfg"], s["q"], s["k"], s["v"], s["table"], s["seq_len"], s["out"], **more)
    else:
        G, scale = case["H"] // case["Hkv"], case["d"] ** -0.5
        for b, n in enumerate(s["len"]):
            if n == 0:
                s["out"][b] = 0
                s["lse"][b] = -math.inf
                continue
            page, place = _places(s, b, 0, n)
            if case["step"]:
                s["k"][page[-1], :, place[-1]] = s["k_new"][b]
                s["v"][page[-1], :, place[-1]] = s["v_new"][b]
                s["pos"][page[-1], :, place[-1]] = s["seq_pos"][b] - 1
            k = s["k"][page, :, place].float().transpose(0, 1).contiguous()            # [kv heads, n, d]
            v = s["v"][page, :, place].float().transpose(0, 1).contiguous()
            q = s["q"][b].float().reshape(case["Hkv"], G, case["d"])
            x = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale                  # [kv heads, G, n]
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - top)
            total = e.sum(-1, keepdim=True)
            p = e / total
            s["out"][b] = torch.matmul(p, v).reshape(case["H"], case["d"]).to(s["out"].dtype)
            s["lse"][b] = (top + torch.log(total)).reshape(case["H"])
            if case["weights"]:
                before = s["weight"][page, :, place].clone()
                if case["step"]:
                    before[-1] = 0                                                                # the new token has none yet
                s["weight_out"][page, :, place] = before + p.sum(1).t()
    got = {"out": s["out"], "lse": s["lse"]}
    if case["weights"]:
        got["weight"] = s["weight_out"]
    if case["step"]:
        got.update(k=s["k"], v=s["v"], pos=s["pos"])
    return got


def _run_evict(s):
    case = s["case"]
    if own:
        import paper_2510_18716_amd as ssd
        ssd.ssd_paged_evict(s["cfg"], s["k"], s["v"], s["table"], s["seq_len"], s["budget"], s["pos"], s["pos_out"], s["weight"],
                            s["weight_out"], s["len_out"], n_sink=case["sink"], recent=case["recent"], seq_pos=s["seq_pos"],
                            max_len=case["hi"], workspace=s["work"])
    else:
        torch.minimum(s["seq_len"], s["budget"], out=s["len_out"])
        for b, n in enumerate(s["len"]):
            page, place = _places(s, b, 0, n)
            pos, weight = s["pos"][page, :, place].t(), s["weight"][page, :, place].t()      # [kv heads, n]
            stay = min(n, case["budget"])
            kept = torch.ones_like(pos, dtype=torch.bool)
            if stay < n:
                safe = (pos < case["sink"]) | (pos >= s["seq_pos"][b] - case["recent"])
                order = torch.argsort(pos, dim=1, stable=True)                                     # lower positions first
                order = order.gather(1, torch.argsort(weight.gather(1, order), dim=1, descending=True, stable=True))
                order = order.gather(1, torch.argsort(safe.gather(1, order).to(torch.int32), dim=1, descending=True, stable=True))
                kept = torch.zeros_like(kept).scatter_(1, order[:, :stay], True)
            free, source = torch.nonzero(~kept[:, :stay]), torch.nonzero(kept[:, stay:])
            head, to, at = free[:, 0], free[:, 1], source[:, 1] + stay                      # pairs: both in order of head and slot
            pos, weight = pos.clone(), weight.clone()
            pos[head, to], weight[head, to] = pos[head, at], weight[head, at]
            s["k"][page[to], head, place[to]] = s["k"][page[at], head, place[at]]
            s["v"][page[to], head, place[to]] = s["v"][page[at], head, place[at]]
            s["pos_out"][page[:stay], :, place[:stay]] = pos[:, :stay].t()
            s["weight_out"][page[:stay], :, place[:stay]] = weight[:, :stay].t()
    return {"k": s["k"], "v": s["v"], "pos": s["pos_out"], "weight": s["weight_out"], "len": s["len_out"]}


def _run_logits(s):
    if own:
        import paper_2510_18716_amd as ssd
        ssd.ssd_logits_process(s["logits"], s["case"]["rows"], s["case"]["V"], s["case"]["dtype"], s["out"], gamma=s["gamma"],
                               tokens=s["tokens"], n_tokens=s["n_tokens"], n_prompt=s["n_prompt"],
                               repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], temperature=s["temperature"],
                               bias=s["bias"], bias_shared=s["case"]["bias"] == "shared", mask=s["mask"])
    else:
        x = s["logits"].float()
        if s["gamma"] is not None:
            x = x[0::2] + s["gamma"] * (x[0::2] - x[1::2])
        if s["bias"] is not None:
            x = x + s["bias"]
        at = torch.arange(s["tokens"].shape[1], device=x.device)[None]
        there = (at < s["n_tokens"][:, None]) & (s["tokens"] >= 0) & (s["tokens"] < x.shape[1])
        token = s["tokens"].clamp(0, x.shape[1] - 1).long()
        seen = torch.zeros(x.shape, dtype=torch.int32, device=x.device).scatter_add_(1, token, there.to(torch.int32)) > 0
        count = torch.zeros(x.shape, dtype=torch.int32, device=x.device)
        count.scatter_add_(1, token, (there & (at >= s["n_prompt"][:, None])).to(torch.int32))
        rep = s["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - (s["frequency"][:, None] * count + s["presence"][:, None] * (count > 0))
        x = x / s["temperature"][:, None]
        if s["mask"] is not None:
            bit = torch.arange(x.shape[1], device=x.device)
            allowed = (s["mask"][:, bit // 32] >> (bit % 32).to(torch.int32)) & 1
            x = torch.where(allowed != 0, x, -math.inf)
        s["out"].copy_(x)
    return {"logits": s["out"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "logits":
        rows, V = case["rows"], case["V"]
        size = rows * V * ((2 if case["guided"] else 1) * (2 if case["dtype"] == "bf16" else 4) + 4)
        size += {"none": 0, "shared": 4 * V, "row": 4 * V * rows}[case["bias"]] + (rows * (-(-V // 32)) * 4 if case["mask"] else 0)
        return {"bytes": size + 4 * sum(_lengths(rows, max(1, case["history"] // 8), case["history"])), "flops": 6 * rows * V}
    lens = _lengths(case["B"], case["lo"], case["hi"])
    n, row = sum(lens), case["d"] * (2 if case["dtype"] == "bf16" else 4)
    blocks = 4 * sum(-(-x // case["page"]) for x in lens)
    if kind == "append":
        return {"bytes": n * case["Hkv"] * (4 * row + 8 + (4 if case["weights"] else 0)), "flops": 0}
    if kind == "attn":
        size = n * case["Hkv"] * (2 * row + (8 if case["weights"] else 0)) + 2 * case["B"] * case["H"] * row + blocks
        if case["step"]:
            size += case["B"] * case["Hkv"] * 2 * row
        return {"bytes": size, "flops": 4 * n * case["H"] * case["d"]}
    size = blocks
    for x in lens:
        stay = min(x, case["budget"])
        moved = (x - stay) * stay / x                  # weights have no order: a kept row lies anywhere
        size += case["Hkv"] * (8 * x + 8 * stay + moved * 4 * row)
    return {"bytes": int(size), "flops": 0}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "evict": _exact_evict, "logits": _exact_logits}[case["kind"]](s, case)


def _flat(s, x):
    """x [pages, kv heads, page, ...] by kv head and by place in the pool: [kv heads, pages * page, ...], a copy."""
    y = x.transpose(0, 1)
    return y.reshape((y.shape[0], -1) + tuple(y.shape[3:])).clone()


def _unflat(s, y):
    pages = s["k"].shape[0]
    return y.reshape((y.shape[0], pages, -1) + tuple(y.shape[2:])).transpose(0, 1)


def _pool_slots(s, b, n):
    page = s["case"]["page"]
    return (s["table"][b].long()[:, None] * page + torch.arange(page, device=s["table"].device)[None]).reshape(-1)[:n]


def _exact_append(s, case):
    k, v, pos, weight = (_flat(s, s[x]) for x in ("k", "v", "pos", "weight"))
    start = s["start"].tolist()
    for b in range(case["B"]):
        n = start[b + 1] - start[b]
        to = _pool_slots(s, b, s["len"][b])[s["len"][b] - n:]
        k.index_copy_(1, to, s["k_new"][start[b]:start[b + 1]].transpose(0, 1).contiguous())
        v.index_copy_(1, to, s["v_new"][start[b]:start[b + 1]].transpose(0, 1).contiguous())
        pos[:, to] = torch.arange(case["held"], case["held"] + n, device=to.device, dtype=torch.int32)
        weight[:, to] = 0.0 if s["weight_new"] is None else s["weight_new"][start[b]:start[b + 1]].t()
    return {"k": _unflat(s, k), "v": _unflat(s, v), "pos": _unflat(s, pos), "weight": _unflat(s, weight)}


def _exact_attn(s, case):
    G = case["H"] // case["Hkv"]
    out = torch.zeros((case["B"], case["H"], case["d"]), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((case["B"], case["H"]), -math.inf, dtype=torch.float64, device=out.device)
    got = {"out": out, "lse": lse}
    k, v = _flat(s, s["k"]), _flat(s, s["v"])
    weight = _flat(s, s["weight"]).double() if case["weights"] else None
    after = torch.zeros_like(weight) if case["weights"] else None
    pos = _flat(s, s["pos"]) if case["step"] else None
    for b, n in enumerate(s["len"]):
        if n == 0:
            continue
        at = _pool_slots(s, b, n)
        if case["step"]:
            k[:, at[n - 1]], v[:, at[n - 1]] = s["k_new"][b], s["v_new"][b]
            pos[:, at[n - 1]] = int(s["seq_pos"][b]) - 1
            if case["weights"]:
                weight[:, at[n - 1]] = 0
        for h in range(case["Hkv"]):
            heads = slice(h * G, (h + 1) * G)
            z = (k[h].index_select(0, at).double() @ s["q"][b, heads].double().t()) / math.sqrt(case["d"])      # [n, G]
            lse[b, heads] = torch.logsumexp(z, 0)
            p = torch.softmax(z, 0)
            out[b, heads] = p.t() @ v[h].index_select(0, at).double()
            if case["weights"]:
                after[h, at] = weight[h, at] + p.sum(1)
    if case["weights"]:
        got["weight"] = _unflat(s, after)
    if case["step"]:
        got.update(k=_unflat(s, k), v=_unflat(s, v), pos=_unflat(s, pos))
    return got


def _exact_evict(s, case):
    k, v, pos, weight = (_flat(s, s[x]) for x in ("k", "v", "pos", "weight"))
    pos_out, weight_out = _flat(s, s["pos_out"]), _flat(s, s["weight_out"])
    for b, n in enumerate(s["len"]):
        at = _pool_slots(s, b, n)
        total, stay = int(s["seq_pos"][b]), min(n, case["budget"])
        p_all, w_all = pos[:, at].cpu().numpy(), weight[:, at].cpu().numpy()
        for h in range(case["Hkv"]):
            p, w = p_all[h], w_all[h]
            safe = (p < case["sink"]) | (p >= total - case["recent"])
            best = np.lexsort((np.arange(n), p, -w.astype(np.float64), ~safe))[:stay]
            slot = np.arange(stay)
            inside = np.zeros(stay, dtype=bool)
            inside[best[best < stay]] = True
            slot[~inside] = np.sort(best[best >= stay])                                     # what each slot below `stay` now holds
            source, to = at[torch.from_numpy(slot).to(at.device)], at[:stay]
            k[h, to], v[h, to] = k[h, source], v[h, source]
            pos_out[h, to], weight_out[h, to] = pos[h, source], weight[h, source]
    return {"k": _unflat(s, k), "v": _unflat(s, v), "pos": _unflat(s, pos_out), "weight": _unflat(s, weight_out),
            "len": torch.tensor([min(n, case["budget"]) for n in s["len"]], dtype=torch.int32)}


def _exact_logits(s, case):
    x = s["logits"].double()
    if case["guided"]:
        c, u = x.view(case["rows"], 2, case["V"]).unbind(1)
        x = (1.0 + s["gamma"]) * c - s["gamma"] * u
    rows = []
    for r in range(case["rows"]):
        y = x[r].clone()
        if s["bias"] is not None:
            y += s["bias"][r if case["bias"] == "row" else 0].double()
        told = s["tokens"][r, :int(s["n_tokens"][r])].long()
        seen = torch.bincount(told, minlength=case["V"]) > 0
        count = torch.bincount(told[int(s["n_prompt"][r]):], minlength=case["V"])
        rep = float(s["repetition"][r])
        y[seen] *= torch.where(y[seen] > 0, 1.0 / rep, rep)
        y -= float(s["frequency"][r]) * count + torch.where(count > 0, float(s["presence"][r]), 0.0)
        y /= float(s["temperature"][r])
        if s["mask"] is not None:
            words = s["mask"][r].long()
            bits = ((words[:, None] >> torch.arange(32, device=y.device)[None]) & 1).reshape(-1)[:case["V"]]
            y[bits == 0] = -math.inf
        rows.append(y)
    return {"logits": torch.stack(rows)}
