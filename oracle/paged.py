"""Plain 64-bit implementations of the calls on a paged cache and of the logits' processing, written from their definitions one
sequence and one head at a time.  Pools are numpy arrays [pages, kv heads, page size, d], whatever their strides on the device."""
import numpy as np


def slot_place(table_row, slot, page_size):
    return int(table_row[slot // page_size]), slot % page_size


def rows_of(pool, table_row, n, page_size, kv):
    """(rows [n, ...] in 64 bits, which of them exist): a table entry outside the pool names no page."""
    out = np.zeros((n,) + pool.shape[3:], dtype=np.float64)
    there = np.zeros(n, dtype=bool)
    for j in range(n):
        page, place = slot_place(table_row, j, page_size)
        if 0 <= page < pool.shape[0]:
            out[j] = pool[page, kv, place]
            there[j] = True
    return out, there


def paged_attend(q, k_pool, v_pool, table_row, n, scale):
    """q [H, d] of one sequence.  Returns out [H, d], lse [H], p [H, n], and sum p |v| [H, d], the size its terms have."""
    H, d = q.shape
    n_kv, page_size = k_pool.shape[1], k_pool.shape[2]
    out, lse, size = np.zeros((H, d)), np.full(H, -np.inf), np.zeros((H, d))
    p = np.zeros((H, n))
    for kv in range(n_kv):
        K, there = rows_of(k_pool, table_row, n, page_size, kv)
        V, _ = rows_of(v_pool, table_row, n, page_size, kv)
        for h in range(kv * (H // n_kv), (kv + 1) * (H // n_kv)):
            z = np.array([float(np.dot(q[h].astype(np.float64), K[j])) * scale for j in range(n)])[there]
            if z.size == 0:
                continue
            top = z.max()
            e = np.exp(z - top)
            lse[h] = top + np.log(e.sum())
            p[h, there] = e / e.sum()
            out[h] = p[h, there] @ V[there]
            size[h] = p[h, there] @ np.abs(V[there])
    return out, lse, p, size


def paged_append(k_pool, v_pool, pos, weight, table, seq_len, seq_pos, k_new, v_new, new_start, weight_new):
    """In place, token by token."""
    page_size = k_pool.shape[2]
    for b in range(len(seq_len)):
        first, end = (b, b + 1) if new_start is None else (new_start[b], new_start[b + 1])
        for row in range(first, end):
            slot = seq_len[b] - (end - row)
            if slot < 0 or slot >= min(seq_len[b], table.shape[1] * page_size):
                continue
            page, place = slot_place(table[b], slot, page_size)
            if not 0 <= page < k_pool.shape[0]:
                continue
            k_pool[page, :, place], v_pool[page, :, place] = k_new[row], v_new[row]
            if pos is not None:
                pos[page, :, place] = seq_pos[b] - (end - row)
            if weight is not None:
                weight[page, :, place] = 0.0 if weight_new is None else weight_new[row]


def evict_order(pos, weight, total, n_sink, recent):
    """The rows of one unit, the best first."""
    def key(j):
        safe = pos[j] < n_sink or pos[j] >= total - recent
        w = -np.inf if np.isnan(weight[j]) else float(weight[j])
        return (0 if safe else 1, 1 if np.isnan(weight[j]) else 0, -w, int(pos[j]), j)
    return sorted(range(len(pos)), key=key)


def evict_moves(pos, weight, total, budget, n_sink, recent, there=None):
    """n' of one unit and the moves (slot that became free, slot its new row comes from).  there: which slots have a page, None: all; the others hold no
    row and take none."""
    n = len(pos)
    stay = min(n, max(0, budget))
    held = [j for j in range(n) if there is None or there[j]]
    places = [j for j in held if j < stay]
    order = evict_order([pos[j] for j in held], [weight[j] for j in held], total, n_sink, recent)
    kept = set(held[i] for i in order[:len(places)])
    free = [j for j in places if j not in kept]
    source = sorted(j for j in kept if j >= stay)
    assert len(free) == len(source)
    return stay, list(zip(free, source))


def process_logits(x, u, gamma, bias, tokens, n_prompt, repetition, presence, frequency, temperature, allowed):
    """One row.  u, bias, allowed: None where there is none."""
    y = np.asarray(x, dtype=np.float64).copy()
    with np.errstate(invalid="ignore"):
        if u is not None:
            y = y + gamma * (y - np.asarray(u, dtype=np.float64))
        if bias is not None:
            y = y + bias
        times = np.zeros(len(y), dtype=np.int64)
        seen = np.zeros(len(y), dtype=bool)
        for j, t in enumerate(tokens):
            if 0 <= t < len(y):
                seen[t] = True
                times[t] += j >= n_prompt
        for v in np.nonzero(seen)[0]:
            y[v] = y[v] / repetition if y[v] > 0 else y[v] * repetition
            y[v] -= frequency * times[v] + (presence if times[v] else 0.0)
        y = y / temperature
    if allowed is not None:
        y[~allowed] = -np.inf
    return y
