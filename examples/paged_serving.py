"""Image tokens for requests of unequal lengths, over a cache in pages.

A small random model stands in for the network; what it shows is the order of the library's calls in a server's loop:

    prompts    ssd_prefill_scores  accumulated attention of each prompt's tokens
               ssd_paged_append    their rows, of all prompts at once, with those scores
               ssd_paged_evict     every sequence down to its budget; the pages behind it go back to the pool
    per token  ssd_paged_decode_step (each layer)  the token's row, its attention, everybody's weights
               ssd_paged_evict     when the rows added since the last one fill the slack
               ssd_logits_process  guidance of each request's two sequences, penalties, the tokens that are images'

Every request is two sequences, one with its prompt and one without most of it (classifier-free guidance), so that their lengths differ.  With `pool` "mxfp8" or "mxfp4"
the rows are held in 8 or 4 bits and the calls are the ssd_paged_mx_ ones; with `columns` queries and keys turn by positions in time, height and width (ssd_rope_axes).

    python examples/paged_serving.py [mxfp8 | mxfp4]
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass, field

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_18716_amd as ssd  # noqa: E402


@dataclass
class Settings:
    prompts: tuple = (37, 150, 8, 411)      # tokens of each request's prompt
    bare: int = 3                           # tokens of the sequence without it
    layers: int = 2
    heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    dtype: str = "bf16"
    vocab: int = 1000
    image_tokens: tuple = (200, 1000)       # the part of the vocabulary that may be generated
    page: int = 16
    budget: int = 64                        # rows a sequence keeps
    slack: int = 16                         # tokens between evictions
    sinks: int = 1
    recent: int = 8
    gamma: float = 3.0
    temperature: float = 0.9
    repetition: float = 1.1
    pool: str = "plain"                     # or "mxfp8", "mxfp4"
    columns: int = 0                        # of the image, if queries and keys turn by their positions
    steps: int = 40
    seed: int = 0


@dataclass
class PagePool:
    """Pages by number; a sequence's row of the block table names those it has."""
    free: list
    table: torch.Tensor                     # host int32 [n_seqs, max_blocks]
    held: list = field(default_factory=list)

    def fit(self, seq: int, blocks: int):
        """Give sequence `seq` that many pages, or take those beyond back."""
        while len(self.held[seq]) < blocks:
            self.table[seq, len(self.held[seq])] = self.free[-1]
            self.held[seq].append(self.free.pop())
        while len(self.held[seq]) > blocks:
            self.free.append(self.held[seq].pop())
            self.table[seq, len(self.held[seq])] = -1


def positions(time, i, columns):
    """Positions [3, tokens] of tokens at these times: for the i-th token of an image its time, its row and its column, counted from the image's beginning; i None: the time thrice."""
    return torch.stack([time, time if i is None else time - i + i // columns, time if i is None else time - i + i % columns]).to(torch.int32)


def serve(s: Settings, watch=None):
    """Returns (tokens [requests, steps], rows held, positions held per layer).  watch(layer, state): called after each layer's attention."""
    dev, dt = "cuda", torch.bfloat16 if s.dtype == "bf16" else torch.float32
    g = torch.Generator(device=dev).manual_seed(s.seed)
    n_req, B, H, Hk, d, D = len(s.prompts), 2 * len(s.prompts), s.heads, s.kv_heads, s.head_dim, s.heads * s.head_dim

    def weight(*shape):
        return torch.randn(shape, device=dev, generator=g) * shape[-2] ** -0.5

    embed, head = torch.randn((s.vocab, D), device=dev, generator=g), weight(D, s.vocab) * 2
    qkv = [weight(D, (H + 2 * Hk) * d) for _ in range(s.layers)]
    back = [weight(D, D) for _ in range(s.layers)]

    lens = [n for p in s.prompts for n in (p, s.bare)]                       # sequence 2i with request i's prompt, 2i + 1 without
    prompt = torch.randint(0, s.vocab, (sum(lens),), device=dev, generator=g)
    start = torch.tensor([sum(lens[:i]) for i in range(B + 1)], dtype=torch.int32)
    most = max(max(lens), s.budget + s.slack)
    blocks = -(-most // s.page)
    pool = PagePool(list(range(B * blocks)), torch.full((B, blocks), -1, dtype=torch.int32), [[] for _ in range(B)])
    for b, n in enumerate(lens):
        pool.fit(b, -(-n // s.page))
    table = pool.table.to(dev)
    seq_len = torch.tensor(lens, dtype=torch.int32, device=dev)
    seq_pos = seq_len.clone()
    budget = torch.full((B,), s.budget, dtype=torch.int32, device=dev)
    shape = (B * blocks, Hk, s.page)
    bits = {"plain": 0, "mxfp8": 8, "mxfp4": 4}[s.pool]
    row = (d * bits // 8,) if bits else (d,)
    k = [torch.zeros(shape + row, device=dev, dtype=torch.uint8 if bits else dt) for _ in range(s.layers)]
    v = [torch.zeros_like(x) for x in k]
    scales = [[torch.zeros(shape + (d // 32,), device=dev, dtype=torch.uint8) for _ in "kv"] for _ in range(s.layers if bits else 0)]
    pos = [torch.zeros(shape, dtype=torch.int32, device=dev) for _ in range(s.layers)]
    mass = [torch.zeros(shape, device=dev) for _ in range(s.layers)]
    # rows of the projections are (H + 2 Hk) * d long: q, k and v are read where they lie
    cfg = ssd.make_paged_config(B, H, Hk, d, s.dtype, s.page, B * blocks, blocks, q_stride=(H + 2 * Hk) * d, new_stride=(H + 2 * Hk) * d)
    if bits:
        sizes = ssd.ssd_paged_mx_workspace_bytes(cfg, s.pool, most, True), ssd.ssd_paged_mx_evict_workspace_bytes(cfg, s.pool, most)
    else:
        sizes = ssd.ssd_paged_workspace_bytes(cfg, most, True), ssd.ssd_paged_evict_workspace_bytes(cfg, most)
    work = torch.empty(max(sizes), dtype=torch.uint8, device=dev)
    after = torch.zeros_like(seq_len)

    def parts(x):
        """Views of a projection's q, k and v."""
        return x[:, :H * d], x[:, H * d:(H + Hk) * d], x[:, (H + Hk) * d:]

    def on_pool(name, l, *args, first=(), **more):
        """A paged call on layer l's pool: (config, first.., pool, args..), of the kind that the pool is."""
        if bits:
            getattr(ssd, "ssd_paged_mx_" + name)(cfg, s.pool, *first, k[l], v[l], *scales[l], *args, **more)
        else:
            getattr(ssd, "ssd_paged_" + name)(cfg, *first, k[l], v[l], *args, **more)

    pairs = d // 2
    axis = torch.tensor([i * 3 // pairs for i in range(pairs)], dtype=torch.uint8, device=dev)
    inv_freq = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], device=dev)

    def turned(rows, time, i):
        """Rows of projections whose queries and keys turn by their tokens' positions."""
        if s.columns:
            ssd.ssd_rope_axes(rows, rows, len(rows), H + Hk, d, s.dtype, positions(time, i, s.columns), inv_freq, axis=axis, n_axes=3)
        return rows

    def cut(host_lens):
        nonlocal table
        for l in range(s.layers):
            on_pool("evict", l, table, seq_len, budget, pos[l], pos[l], mass[l], mass[l], after, n_sink=s.sinks, recent=s.recent, seq_pos=seq_pos, max_len=most,
                    workspace=work)
        seq_len.copy_(after)
        host_lens = [min(n, s.budget) for n in host_lens]
        for b, n in enumerate(host_lens):
            pool.fit(b, -(-(n + s.slack) // s.page))                         # room for the tokens until the next eviction
        table = pool.table.to(dev)
        return host_lens

    # the prompts
    for l in range(s.layers):
        rows = turned((embed[prompt] @ qkv[l]).to(dt), torch.cat([torch.arange(n, device=dev) for n in lens]), None)
        qp, kp, vp = parts(rows)
        scores = torch.zeros((len(prompt), Hk), device=dev)
        for b, n in enumerate(lens):                                         # one sequence's heads are the units of one call
            part = slice(int(start[b]), int(start[b]) + n)
            Q = qp[part].reshape(n, H, d).transpose(0, 1).contiguous()
            K = kp[part].reshape(n, Hk, d).transpose(0, 1).repeat_interleave(H // Hk, 0).contiguous()
            one = torch.empty((H, n), device=dev)
            ssd.ssd_prefill_scores(Q, K, H, n, d, s.dtype, one)
            scores[part] = one.reshape(Hk, H // Hk, n).sum(1).t()
        on_pool("append", l, table, seq_len, kp, vp, pos=pos[l], weight=mass[l], seq_pos=seq_pos, new_start=start.to(dev), weight_new=scores)
    lens = cut(lens)

    # the tokens
    allowed = torch.zeros(s.vocab, dtype=torch.bool)
    allowed[s.image_tokens[0]:s.image_tokens[1]] = True
    words = torch.zeros(-(-s.vocab // 32), dtype=torch.int64)
    for i in torch.nonzero(allowed).flatten().tolist():
        words[i // 32] |= 1 << (i % 32)
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).to(dev)
    told = torch.full((n_req, s.steps), -1, dtype=torch.int32, device=dev)
    n_told = torch.zeros(n_req, dtype=torch.int32, device=dev)
    per_row = {name: torch.full((n_req,), x, device=dev) for name, x in (("repetition", s.repetition), ("temperature", s.temperature))}
    token = torch.zeros(n_req, dtype=torch.int64, device=dev)
    logits = torch.empty((n_req, s.vocab), device=dev)
    since = 0
    for step in range(s.steps):
        if since == s.slack:
            lens, since = cut(lens), 0
        seq_len += 1
        seq_pos += 1
        lens = [n + 1 for n in lens]
        since += 1
        x = embed[token].repeat_interleave(2, 0)
        for l in range(s.layers):
            rows = turned((x @ qkv[l]).to(dt), seq_pos - 1, step)
            q, k_new, v_new = parts(rows)
            out = torch.empty((B, H, d), device=dev, dtype=dt)
            on_pool("decode_step", l, table, seq_len, out, first=(q, k_new, v_new), pos=pos[l], seq_pos=seq_pos, weight_in=mass[l], weight_out=mass[l],
                    max_len=most, workspace=work)
            if watch is not None:
                watch(l, {"q": q, "k": k[l], "v": v[l], "scales": scales[l] if bits else None, "table": table, "lens": lens, "out": out})
            x = x + out.reshape(B, D).float() @ back[l]
        x = x / x.norm(dim=-1, keepdim=True) * D ** 0.5
        ssd.ssd_logits_process(x @ head, n_req, s.vocab, "f32", logits, gamma=s.gamma, tokens=told, n_tokens=n_told, mask=mask, mask_shared=True, **per_row)
        token = torch.multinomial(torch.softmax(logits, -1), 1, generator=g).flatten()
        told[:, step] = token.to(torch.int32)
        n_told += 1
    held = [[pos[l][table[b, torch.arange(n) // s.page].long(), :, torch.arange(n) % s.page].t().cpu() for b, n in enumerate(lens)] for l in range(s.layers)]
    return told.cpu(), lens, held


def main():
    s = Settings(pool=sys.argv[1], columns=24) if len(sys.argv) > 1 else Settings()
    tokens, lens, held = serve(s)
    for i, p in enumerate(s.prompts):
        print("request %d: prompt of %d tokens, %d rows held, tokens %s ..." % (i, p, lens[2 * i], tokens[i, :8].tolist()))
    print("the oldest positions the first head of request 3 still holds:", sorted(held[0][6][0].tolist())[:12])


if __name__ == "__main__":
    main()
