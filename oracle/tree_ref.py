"""Plain reference of the operators over trees of tokens (test infrastructure: it imports nothing from the GPU package).

Numpy in fp64 and Python integers, step by step as the definitions read; results are not rounded.  A mask is a list of Python
integers here, bit j for node j of the tail."""
import numpy as np

D = 128


def words_of(masks, words):
    """Masks as int64 [rows, words]; bits behind the words are lost."""
    out = np.zeros((len(masks), words), dtype=np.uint64)
    for i, m in enumerate(masks):
        for w in range(words):
            out[i, w] = (m >> (64 * w)) & (2 ** 64 - 1)
    return out.view(np.int64)


def tree_masks(parents):
    """(masks, depths) of the nodes of one tree; a parent that is not an earlier node makes a root."""
    masks, depths = [], []
    for i, p in enumerate(parents):
        root = not 0 <= p < i
        masks.append(1 << i if root else masks[p] | 1 << i)
        depths.append(0 if root else depths[p] + 1)
    return masks, depths


def attention(q, keys, values, seen, scale):
    """One sequence: q [n, 128 heads], keys and values [kv_heads, S, 128], seen [n, S].  (out, lse [n, heads], sum of p |V| as out, largest
    scale * sum |q| |K| of a pair that is seen)."""
    keys, values = keys.astype(np.float64), values.astype(np.float64)
    n, S = seen.shape
    heads, kv = q.shape[1] // D, keys.shape[0]
    q = q.astype(np.float64).reshape(n, heads, D)
    out, mass, lse, size = np.zeros_like(q), np.zeros_like(q), np.full((n, heads), -np.inf), 0.0
    for i in range(n):
        t = np.flatnonzero(seen[i])
        if not len(t):
            continue
        for h in range(heads):
            g = h // (heads // kv)
            s = scale * (keys[g, t] @ q[i, h])
            top = s.max()
            e = np.exp(s - top)
            lse[i, h] = top + np.log(e.sum())
            out[i, h], mass[i, h] = e @ values[g, t] / e.sum(), e @ np.abs(values[g, t]) / e.sum()
            size = max(size, scale * (np.abs(keys[g, t]) @ np.abs(q[i, h])).max())
    return out.reshape(n, heads * D), lse, mass.reshape(n, heads * D), size


def plan(new, cached, position, parents, held, table, stack, page, tokens, max_q, max_len):
    """What fq_paged_plan writes, as a dict; `stack` is the list of free pages (its last is taken first), tables are changed."""
    table, stack = table.copy(), list(stack)
    for b, n in enumerate(new):
        if n < 0:
            stack += table[b, :held[b]].tolist()
    given = list(stack)
    q_start, seq_len, held_out, positions, slots, masks, lacking = [0], [], [], [], [], [], 0
    for b, n in enumerate(new):
        if n < 0:
            q_start.append(q_start[-1]), seq_len.append(0), held_out.append(0)
            continue
        before = min(max(cached[b], 0), max_len)
        n = min(n, max_q, max_len - before, tokens - q_start[-1])
        have = held[b]
        for c in range(held[b], -(-(before + n) // page)):
            if stack:
                table[b, c], have = stack.pop(), have + 1
            else:
                table[b, c], lacking = -1, lacking + 1
        first = position[b] if position is not None else before
        m, depth = tree_masks(parents[q_start[-1]:q_start[-1] + n]) if parents is not None else ([], range(n))
        masks += m
        positions += [first + d for d in depth]
        for t in range(before, before + n):
            pg = table[b, t // page]
            slots.append(-1 if pg < 0 else pg * page + t % page)
        q_start.append(q_start[-1] + n), seq_len.append(before + n), held_out.append(have)
    rest = tokens - q_start[-1]
    return {"q_start": q_start, "seq_len": seq_len, "held": held_out, "table": table, "given": given, "free": len(stack), "lacking": lacking,
            "positions": positions + [0] * rest, "slots": slots + [-1] * rest, "masks": masks + [0] * rest}


def accept(parents, drafted, following, most):
    """(path, bonus) through one drafted tree."""
    if not len(parents):
        return [], -1
    path = [0]
    while len(path) < most:
        at = path[-1]
        more = [i for i in range(at + 1, len(parents)) if parents[i] == at and drafted[i] == following[at]]
        if not more:
            break
        path.append(more[0])
    return path, following[path[-1]]


def given(path, accepted, tail):
    """The nodes that a given path means: cut to the path's room and to the tail, a node below its place taken for that place, one behind the tail for its last."""
    return [min(max(int(node), k), tail - 1) for k, node in enumerate(path[:max(min(accepted, len(path), tail), 0)])]


def keep(pool, table, base, path, page):
    """Rows of a path moved together in one pool [pages, heads, page, 128]; positions without a page stay out."""
    rows = {}
    for k, node in enumerate(path):
        (p, r), (x, y) = divmod(base + node, page), divmod(base + k, page)
        if table[p] >= 0 and table[x] >= 0:
            rows[table[x], y] = pool[table[p], :, r].copy()
    for (x, y), row in rows.items():
        pool[x, :, y] = row


def beam(logits, scores, done, eos, width):
    """One request: logits [beams, vocab], scores [beams].  (parent, token, score, done) of the best, best first."""
    beams, vocab = logits.shape
    totals = np.full((beams, vocab), -np.inf)
    for b in range(beams):
        if done is not None and done[b]:
            totals[b, eos] = scores[b]
            continue
        x = logits[b].astype(np.float64)
        with np.errstate(all="ignore"):
            top = x.max()
            totals[b] = float(scores[b]) + (x - (top + np.log(np.exp(x - top).sum())))
    flat = totals.reshape(-1)
    live = np.flatnonzero(flat > -np.inf)
    best = live[np.lexsort((live, -flat[live]))][:width]
    pad = width - len(best)
    ended = [bool(done is not None and done[i // vocab]) or i % vocab == eos for i in best]
    return ([int(i // vocab) for i in best] + [-1] * pad, [int(i % vocab) for i in best] + [-1] * pad,
            np.concatenate((flat[best], np.full(pad, -np.inf))), [int(e) for e in ended] + [1] * pad)
