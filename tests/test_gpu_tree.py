"""Operators over trees of tokens against oracle/tree_ref.py (fp64 and Python integers, step by step).

Bounds of the attention, each from the roundings that the kernels make (u = 2^-11, half a step of fp16): scores are fp32 sums of 128
products, so off by at most e = 130 * 2^-24 * (scale sum |q||k|) + 2^-20 absolute, which changes every weight by a factor within 1 +- 2 e; weights
rounded to fp16: u each (or 2^-25 of the largest one, which is at least 2^-25 sum over positions of |v|); output rounded: u |out| + 2^-25; lse
e + 2^-20 |lse|.  Beam scores are held in 64 bits and rounded to fp32 once: 2^-24 of the value, and 2^-40 for the 64-bit part.  All else is whole
numbers, and equal.
"""
import numpy as np
import pytest

from oracle import paged_ref, tree_ref as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -11


@pytest.fixture(scope="module")
def torch():
    import torch

    return torch


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_amd as fq

    fq.fq_init()
    return fq


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def deal(rng, lengths, page, spare=2):
    need = [-(-s // page) for s in lengths]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table, at = np.full((len(lengths), max(max(need), 1)), -1), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def random_tree(rng, n, roots=1):
    return [-1 if i < roots else int(rng.integers(max(0, i - 9), i)) for i in range(n)]


# ------------------------------------------------------------------ attention
def pools(rng, pages, kv, page, table, lengths, std=1.2):
    """Pools that hold NaN wherever no sequence has a position."""
    k, v = (np.full((pages, kv, page, 128), np.nan, dtype=np.float16) for _ in range(2))
    for b, S in enumerate(lengths):
        for t in range(S):
            for pool in (k, v):
                pool[table[b, t // page], :, t % page] = (rng.normal(size=(kv, 128)) * std).astype(np.float16)
    return k, v


def seen_of(masks, tail, S, words):
    """[rows, S]: positions that rows with these masks see."""
    t = range(S)  # Python integers, as the masks are
    out = np.zeros((len(masks), S), dtype=bool)
    for i, m in enumerate(masks):
        out[i] = [x < S - tail or (x - (S - tail) < 64 * words and bool(m >> (x - (S - tail)) & 1)) for x in t]
    return out


def check(got, lse, seqs, masks, words, table, k, v, q, heads, kv, scale):
    at = 0
    for b, (n, tail, S) in enumerate(seqs):
        K, V = paged_ref.rows_of(k, table[b], S), paged_ref.rows_of(v, table[b], S)
        out, L, mass, size = ref.attention(q[at:at + n], K, V, seen_of(masks[at:at + n], min(max(tail, 0), S), S, words), scale)
        e = 130 * 2.0 ** -24 * size + 2.0 ** -20
        floor = 2.0 ** -25 * (1 + (np.abs(V.astype(np.float64)).sum(1).max() if S else 0.0))
        bound = U * (np.abs(out) + mass) * 1.01 + 2 * e * mass + floor
        err = np.abs(got[at:at + n].astype(np.float64) - out)
        assert (err <= bound).all(), (b, n, tail, S, float((err / bound).max()))
        fine = np.isfinite(L)
        assert np.array_equal(fine, np.isfinite(lse[at:at + n])) and np.isneginf(lse[at:at + n][~fine]).all()
        assert (np.abs(lse[at:at + n][fine] - L[fine]) <= e + 2.0 ** -20 * np.abs(L[fine])).all()
        at += n


def masks_for(rng, kind, n, tail):
    if kind == "tree":
        return ref.tree_masks(random_tree(rng, n))[0]
    if kind == "beams":  # random earlier nodes of the tail, and their own
        return [int(sum(1 << int(j) for j in np.flatnonzero(rng.random(tail) < 0.3)) | 1 << (tail - n + i)) for i in range(n)]
    if kind == "none":
        return [0] * n
    return [2 ** (tail + 70) - 1] * n  # all, and bits behind the tail that mean nothing


def attend(fq, torch, rng, seqs, heads, kv, page, words, kinds, given_tail=True, std=1.2):
    """seqs: (tokens, tail, positions)."""
    table, pages = deal(rng, [S for _, _, S in seqs], page)
    k, v = pools(rng, pages, kv, page, table, [S for _, _, S in seqs], std)
    q = (rng.normal(size=(sum(n for n, _, _ in seqs), heads * 128)) * std).astype(np.float16)
    masks = [m for (n, tail, _), kind in zip(seqs, kinds) for m in masks_for(rng, kind, n, tail)]
    b = fq.PagedBatch([n for n, _, _ in seqs], [S for _, _, S in seqs], table, page, pages)
    lse = torch.full((b.tokens, heads), 7.0, device="cuda")
    args = (dev(torch, q), b, dev(torch, ref.words_of(masks, words)), dev(torch, k), dev(torch, v))
    tail = dev(torch, np.array([t for _, t, _ in seqs], dtype=np.int32)) if given_tail else None
    out = fq.fq_attn_tree(*args, tail=tail, lse=lse)
    check(out.cpu().numpy(), lse.cpu().numpy(), seqs, masks, words, table, k, v, q, heads, kv, 128 ** -0.5)
    again = fq.fq_attn_tree(*args, tail=tail)  # the same bits every time, with and without lse
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("heads, kv", [(4, 4), (8, 2), (5, 1), (16, 1)])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("seqs", [
    [(1, 1, 1)], [(1, 1, 40)], [(3, 3, 3)], [(3, 3, 67)], [(2, 2, 64), (0, 0, 9), (4, 4, 131), (1, 1, 2)], [(16, 16, 16)], [(25, 25, 300)],
    [(63, 63, 64), (64, 64, 200), (65, 65, 129)], [(130, 130, 145)], [(0, 0, 0), (7, 7, 1030)]], ids=str)
def test_drafted_trees(fq, torch, heads, kv, page, seqs):
    rng = np.random.default_rng(len(seqs) * 7 + heads + page)
    attend(fq, torch, rng, seqs, heads, kv, page, 3, ["tree"] * len(seqs), given_tail=False)


@pytest.mark.parametrize("heads, kv, page", [(8, 2, 16), (4, 4, 64), (8, 8, 128), (28, 4, 32)])
@pytest.mark.parametrize("seqs, words", [
    ([(4, 40, 300), (4, 4, 90), (4, 64, 64)], 1), ([(5, 300, 1200), (5, 5, 5), (5, 125, 190)], 5), ([(2, 0, 50), (3, 3, 20)], 1),
    ([(6, 700, 720)], 4), ([(1, 500, 501), (1, 1, 130)], 8), ([(4, 10, 0), (3, 90, 40)], 2)], ids=str)
def test_tails_longer_than_the_call(fq, torch, heads, kv, page, seqs, words):
    # bits behind the mask's words are 0, a tail is cut to the positions, and a tail of none leaves everything seen
    rng = np.random.default_rng(heads + page + words)
    for kind in ("beams", "all", "none"):
        attend(fq, torch, rng, [(n, max(t, n) if t else 0, S) for n, t, S in seqs] if kind != "beams" else [(n, max(t, n), S) for n, t, S in seqs],
               heads, kv, page, words, [kind] * len(seqs))


@pytest.mark.parametrize("heads, kv, page, n, S", [(32, 8, 64, 7, 5003), (8, 1, 16, 40, 9001), (4, 4, 128, 16, 20000), (8, 2, 256, 90, 4100)])
def test_long_sequences_are_split(fq, torch, heads, kv, page, n, S):
    rng = np.random.default_rng(S)
    seqs = [(n, n, S), (n, n, 130)]
    b = fq.PagedBatch([n, n], [S, 130], deal(rng, [S, 130], page)[0], page, 1 + -(-S // page) + -(-130 // page) + 1)
    assert fq.fq_attn_tree_workspace_bytes(b, heads, kv) > 0  # parts of rows, to be joined
    attend(fq, torch, rng, seqs, heads, kv, page, 2, ["tree", "tree"])


@pytest.mark.parametrize("heads, kv, page, seqs, parts", [
    (9, 1, 64, [(550, 1500), (3, 700), (40, 90)], 4), (28, 4, 16, [(300, 3000)], 3), (13, 13, 16, [(16, 1100)] * 40, 3),
    (5, 1, 64, [(210, 9000)], 18), (9, 1, 16, [(2, 40), (130, 9000)], 18)], ids=["one_head_left", "four_heads_left", "many_sequences", "spread", "spread_nine_heads"])
def test_more_rows_to_join_than_workgroups(fq, torch, heads, kv, page, seqs, parts):
    """The join has 1024 workgroups, which take eight heads of a token or one in turn: here some have two, the last heads fewer than eight.  Compared are the
    tokens of the second turn and some of the first."""
    rng = np.random.default_rng(heads + page)
    lengths = [S for _, S in seqs]
    table, pages = deal(rng, lengths, page)
    k, v = pools(rng, pages, kv, page, table, lengths)
    b = fq.PagedBatch([n for n, _ in seqs], lengths, table, page, pages)
    items, bytes_ = b.tokens * heads, fq.fq_attn_tree_workspace_bytes(b, heads, kv)
    assert abs(bytes_ - parts * items * 130 * 4) <= 256  # splits of 130 floats a row
    jobs = [n * (heads if parts > 8 * -(-items // 1024) else -(-heads // 8)) for n, S in seqs if S > -(-max(lengths) // parts)]
    assert 1024 < sum(jobs) <= 2048
    q = rng.normal(size=(b.tokens, heads * 128)).astype(np.float16)
    masks = [m for n, _ in seqs for m in ref.tree_masks(random_tree(rng, n))[0]]
    words = -(-b.max_q // 64)
    lse = torch.full((b.tokens, heads), 7.0, device="cuda")
    out = torch.full((b.tokens, heads * 128), 9.0, dtype=torch.float16, device="cuda")
    args = (dev(torch, q), b, dev(torch, ref.words_of(masks, words)), dev(torch, k), dev(torch, v))
    fq.fq_attn_tree(*args, out=out, lse=lse)
    second = b.tokens - -(-(sum(jobs) - 1024) * b.tokens // sum(jobs))  # the first token of the second turn, or one near
    at = 0
    for i, (n, S) in enumerate(seqs):
        late = [at + j for j in range(n) if at + j >= second]
        late = late[::max(len(late) // 12, 1)]
        pick = sorted(set(late) | {at + int(j) for j in rng.choice(n, size=min(n, 6 if len(seqs) < 10 else 1), replace=False)})
        check(out.cpu().numpy()[pick], lse.cpu().numpy()[pick], [(len(pick), n, S)], [masks[j] for j in pick], words, table[i:i + 1], k, v, q[pick], heads, kv,
              128 ** -0.5)
        at += n
    assert torch.isfinite(out).all() and not (out == 9.0).all(1).any()
    assert torch.equal(fq.fq_attn_tree(*args).view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("heads, kv, page, most", [(8, 2, 16, 900), (4, 4, 64, 300), (8, 1, 32, 2500)])
def test_many_sequences(fq, torch, heads, kv, page, most):
    # more sequences than a wavefront has lanes, some without tokens, their lengths from none to many splits
    rng = np.random.default_rng(most)
    seqs = []
    for i in range(83):
        n = int(rng.integers(0, 22)) if i % 7 else 0
        tail = n + (int(rng.integers(0, 60)) if i % 3 else 0)
        seqs.append((n, tail, max(tail, int(rng.integers(0, most if i % 9 == 0 else 60)))))
    attend(fq, torch, rng, seqs, heads, kv, page, 2, ["tree" if n == t else "beams" for n, t, _ in seqs])


def test_rows_that_see_nothing_are_zero(fq, torch):
    rng = np.random.default_rng(4)
    attend(fq, torch, rng, [(5, 70, 70), (3, 3, 3), (2, 0, 0)], 8, 2, 16, 2, ["none", "none", "all"])
    attend(fq, torch, rng, [(40, 70, 70), (30, 200, 200)], 8, 2, 64, 2, ["none", "none"])


@pytest.mark.parametrize("n, S, page", [(3, 50, 16), (40, 200, 64), (70, 300, 16), (24, 64, 32)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(fq, torch, n, S, page, bad):
    rng = np.random.default_rng(n)
    heads, kv = 8, 2
    table, pages = deal(rng, [S], page)
    k, v = pools(rng, pages, kv, page, table, [S])
    node = n - 2
    t = S - n + node
    v[table[0, t // page], :, t % page, 5] = bad
    masks = [m & ~(1 << node) if i != node else m for i, m in enumerate(ref.tree_masks([-1] + list(range(n - 1)))[0])]  # a chain; only its own row sees the node
    b = fq.PagedBatch([n], [S], table, page, pages)
    q = (rng.normal(size=(n, heads * 128))).astype(np.float16)
    out = fq.fq_attn_tree(dev(torch, q), b, dev(torch, ref.words_of(masks, 2)), dev(torch, k), dev(torch, v)).cpu().numpy().reshape(n, heads, 128)
    others = np.arange(n) != node
    assert np.isfinite(out[others]).all()
    assert np.isfinite(np.delete(out[node], 5, axis=1)).all() and not np.isfinite(out[node][:, 5]).any()


def test_keys_that_are_not_finite_and_not_seen(fq, torch):
    rng = np.random.default_rng(9)
    n, S, page, heads, kv = 20, 90, 16, 8, 2
    table, pages = deal(rng, [S], page)
    k, v = pools(rng, pages, kv, page, table, [S])
    t = S - n + 4
    k[table[0, t // page], :, t % page] = np.nan
    masks = [m & ~(1 << 4) for m in ref.tree_masks([-1] + list(range(n - 1)))[0]]
    b = fq.PagedBatch([n], [S], table, page, pages)
    q = (rng.normal(size=(n, heads * 128))).astype(np.float16)
    got, lse = fq.fq_attn_tree(dev(torch, q), b, dev(torch, ref.words_of(masks, 1)), dev(torch, k), dev(torch, v)), None
    assert torch.isfinite(got).all()


def test_a_chain_is_causal_attention(fq, torch):
    rng = np.random.default_rng(11)
    heads, kv, page, seqs = 8, 2, 64, [(30, 30, 400), (60, 60, 61)]
    table, pages = deal(rng, [S for _, _, S in seqs], page)
    k, v = (dev(torch, x) for x in pools(rng, pages, kv, page, table, [S for _, _, S in seqs]))
    q = dev(torch, rng.normal(size=(90, heads * 128)).astype(np.float16))
    b = fq.PagedBatch([30, 60], [400, 61], table, page, pages)
    masks = [m for n, _, _ in seqs for m in ref.tree_masks([-1] + list(range(n - 1)))[0]]
    got, want = fq.fq_attn_tree(q, b, dev(torch, ref.words_of(masks, 1)), k, v), fq.fq_attn_paged(q, b, k, v)
    # both are within the bound of the same formula; here two roundings of the output apart, and of the weights
    assert (got.float() - want.float()).abs().max().item() <= 4 * U * want.float().abs().max().item()


def test_columns_of_a_product_rows_behind_the_last_and_another_stream(fq, torch):
    rng = np.random.default_rng(12)
    heads, kv, page = 8, 2, 32
    table, pages = deal(rng, [100, 50], page)
    k, v = (dev(torch, x) for x in pools(rng, pages, kv, page, table, [100, 50]))
    b = fq.PagedBatch([6, 5], [100, 50], table, page, pages)
    wide = dev(torch, rng.normal(size=(11, heads * 128 + 64)).astype(np.float16))
    mask = dev(torch, ref.words_of([m for n in (6, 5) for m in ref.tree_masks(random_tree(rng, n))[0]], 1))
    want = fq.fq_attn_tree(wide[:, :heads * 128].contiguous(), b, mask, k, v)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = fq.fq_attn_tree(wide[:, :heads * 128], b, mask, k, v, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)
    b.q_start.copy_(dev(torch, np.array([0, 6, 9], dtype=np.int32)))  # two tokens less than rows
    out = torch.full_like(want, 9.0)
    fq.fq_attn_tree(wide[:, :heads * 128], b, mask, k, v, out=out)
    assert (out[9:] == 9.0).all() and torch.equal(out[:6], want[:6])


# ------------------------------------------------------------------ plan
def reserve(fq, torch, seqs, tokens, max_q, max_len, page, pages, words, held, table, stack):
    b = fq.PagedBatch.reserve(seqs, tokens, max_q, max_len, page, pages, mask_words=words)
    b.table.copy_(dev(torch, table.astype(np.int32)))
    b.held.copy_(dev(torch, np.array(held, dtype=np.int32)))
    b.free_pages.fill_(-7)
    b.free_pages[:len(stack)] = dev(torch, np.array(stack, dtype=np.int32))
    b.free_count.fill_(len(stack))
    return b


def check_plan(torch, b, want, held, free):
    ints = lambda t: t.cpu().numpy().tolist()
    for name in ("q_start", "seq_len", "positions", "slots"):
        assert ints(getattr(b, name)) == list(want[name]), name
    assert np.array_equal(b.table.cpu().numpy(), want["table"])
    assert ints(held) == want["held"] and ints(free) == [want["free"]] and ints(b.lacking) == [want["lacking"]]
    assert ints(b.free_pages)[:len(want["given"])] == want["given"]


def plan_case(rng, seqs, page, new_max, cached_max, closed, lack=0, tree=False):
    new = np.where(rng.random(seqs) < closed, -1, rng.integers(0, new_max + 1, seqs))
    cached = rng.integers(0, cached_max + 1, seqs)
    held = -(-cached // page) + (rng.random(seqs) < 0.2)  # some have a page more than they need
    max_len = int(cached.max() + new_max + 1)
    stride = max(-(-max_len // page), int(held.max()))
    need = int(np.maximum(-(-(cached + np.maximum(new, 0)) // page) - held, 0)[new >= 0].sum())
    spare = max(need - lack, 0)
    pages = int(held.sum()) + spare + 1
    order = rng.permutation(pages)
    table = np.full((seqs, stride), -1)
    at = 0
    for i in range(seqs):
        table[i, :held[i]] = order[at:at + held[i]]
        at += held[i]
    tokens = int(np.maximum(new, 0).sum())
    parents = np.concatenate([random_tree(rng, max(int(n), 0), 1 + int(rng.integers(0, 2))) for n in new] + [[]]).astype(int) if tree else None
    return new, cached, held, table, order[at:at + spare].tolist(), pages, stride * page, tokens, parents


@pytest.mark.parametrize("seqs, page, new_max, cached_max, closed, lack, tree", [
    (1, 16, 1, 40, 0, 0, False), (1, 64, 0, 40, 0, 0, False), (5, 16, 40, 100, 0.3, 0, False), (33, 64, 3, 1000, 0.5, 0, False),
    (7, 16, 90, 50, 0, 9, False), (64, 16, 30, 200, 0.2, 40, False), (1500, 16, 3, 60, 0.2, 0, False), (2100, 32, 2, 500, 0.1, 100, False),
    (20, 256, 2000, 3000, 0.1, 0, False), (1100, 16, 40, 300, 0.2, 50, False), (1, 16, 9, 20, 0, 0, True), (6, 16, 64, 90, 0.2, 0, True),
    (50, 64, 33, 300, 0.2, 5, True), (9, 16, 200, 40, 0, 0, True), (300, 16, 50, 40, 0.1, 0, True), (1030, 32, 12, 40, 0.1, 0, True),
    (3, 16, 1500, 100, 0, 0, True), (2, 64, 30000, 100, 0, 0, False), (3000, 16, 10, 60, 0.3, 50, False), (300, 16, 200, 300, 0.3, 0, False),
    (5000, 256, 9, 700, 0.2, 700, False)], ids=str)
def test_plan(fq, torch, seqs, page, new_max, cached_max, closed, lack, tree):
    rng = np.random.default_rng(seqs + page + new_max)
    for given_position in (False, True):
        new, cached, held, table, stack, pages, max_len, tokens, parents = plan_case(rng, seqs, page, new_max, cached_max, closed, lack, tree)
        max_q = max(int(new.max()), 1 if tokens else 0, -(-tokens // seqs))
        words = max(-(-max_q // 64), 1) if tree else 0
        max_q = min(max_q, tokens)
        position = (cached + rng.integers(0, 30, seqs)) if given_position else None
        want = ref.plan(new.tolist(), cached.tolist(), position, parents, held.tolist(), table, stack, page, tokens, max_q, max_len)
        b = reserve(fq, torch, seqs, tokens, max_q, max_len, page, pages, words, held, table, stack)
        ints = lambda a: None if a is None else dev(torch, np.array(a, dtype=np.int32))
        held_out, free_out = torch.full((seqs,), 77, dtype=torch.int32, device="cuda"), torch.full((1,), 77, dtype=torch.int32, device="cuda")
        fq.fq_paged_plan(b, ints(new), ints(cached), next_position=ints(position), parents=ints(parents), held_out=held_out, free_out=free_out)
        check_plan(torch, b, want, held_out, free_out)
        assert b.held.cpu().numpy().tolist() == held.tolist() and b.free_count.item() == len(stack)
        if tree:
            assert np.array_equal(b.mask.cpu().numpy(), ref.words_of(want["masks"], words))
        # in place, with the cached positions where the lengths go
        b2 = reserve(fq, torch, seqs, tokens, max_q, max_len, page, pages, words, held, table, stack)
        b2.seq_len.copy_(ints(cached))
        fq.fq_paged_plan(b2, ints(new), b2.seq_len, next_position=ints(position), parents=ints(parents))
        check_plan(torch, b2, want, b2.held, b2.free_count)


@pytest.mark.parametrize("tokens, max_q, max_len", [(50, 30, 400), (40, 8, 400), (200, 30, 100), (7, 7, 96)])
def test_plan_cuts_to_the_bounds(fq, torch, tokens, max_q, max_len):
    rng = np.random.default_rng(tokens)
    seqs, page = 30, 16
    new, cached = rng.integers(0, 31, seqs), rng.integers(0, 120, seqs)
    cached[3] = -4
    cached = np.minimum(cached, max_len)
    held = -(-np.maximum(cached, 0) // page)
    stride = -(-max_len // page)
    pages = 900
    order = rng.permutation(pages)
    table, at = np.full((seqs, stride), -1), 0
    for i in range(seqs):
        table[i, :held[i]] = order[at:at + held[i]]
        at += held[i]
    stack = order[at:at + 400].tolist()
    want = ref.plan(new.tolist(), cached.tolist(), None, None, held.tolist(), table, stack, page, tokens, max_q, max_len)
    b = reserve(fq, torch, seqs, tokens, max_q, max_len, page, pages, 0, held, table, stack)
    ints = lambda a: dev(torch, np.array(a, dtype=np.int32))
    fq.fq_paged_plan(b, ints(new), ints(cached))
    check_plan(torch, b, want, b.held, b.free_count)
    # numbers that 32 bits hold and sums that they do not
    fq.fq_paged_plan(b, ints(np.full(seqs, 2 ** 31 - 1)), ints(cached))
    assert b.q_start.cpu().numpy()[-1] <= tokens and (b.seq_len.cpu().numpy() <= max_len).all() and b.lacking.item() >= 0


def test_plan_parents_that_are_no_earlier_tokens_make_roots(fq, torch):
    parents = [5, -9, 1, 3, 2 ** 31 - 1, -2 ** 31, 4, 5]
    masks, depths = ref.tree_masks(parents)
    b = fq.PagedBatch.reserve(1, 8, 8, 64, 16, 9, mask_words=1)
    ints = lambda a: dev(torch, np.array(a, dtype=np.int32))
    fq.fq_paged_plan(b, ints([8]), ints([5]), parents=ints(parents))
    assert np.array_equal(b.mask.cpu().numpy(), ref.words_of(masks, 1)) and b.positions.cpu().numpy().tolist() == [5 + d for d in depths]
    b.mask = None  # positions alone
    b.positions.zero_()
    fq.fq_paged_plan(b, ints([8]), ints([5]), parents=ints(parents))
    assert b.positions.cpu().numpy().tolist() == [5 + d for d in depths]


# ------------------------------------------------------------------ commit
def commit_inputs(rng, trees, heads, page, layers):
    """trees: (nodes, positions ahead of them)."""
    lengths = [n + c for n, c in trees]
    table, pages = deal(rng, lengths, page)
    k, v = (rng.normal(size=(layers, pages, heads, page, 128)).astype(np.float16) for _ in range(2))
    parents = [random_tree(rng, n) for n, _ in trees]
    # a small vocabulary: several siblings are drafted alike, and paths are long
    following = [rng.integers(0, 3, n) for n, _ in trees]
    drafted = [np.array([f[p] if p >= 0 and rng.random() < 0.8 else rng.integers(0, 3) for p in ps], dtype=np.int64) for ps, f in zip(parents, following)]
    return table, pages, k, v, parents, drafted, following


def join(parts):
    return np.concatenate([np.asarray(p, dtype=np.int32) for p in parts] + [np.zeros(0, dtype=np.int32)])


@pytest.mark.parametrize("trees, heads, page, layers, stride", [
    ([(1, 0)], 1, 16, 1, 1), ([(1, 5), (0, 30), (2, 15)], 2, 16, 3, 2), ([(25, 611)], 8, 64, 2, 25), ([(64, 3), (65, 40), (63, 16)], 4, 16, 2, 70),
    ([(200, 17), (9, 0), (130, 250)], 2, 32, 2, 200), ([(40, 100), (40, 7)], 3, 256, 1, 4), ([(300, 5)], 1, 16, 2, 300)], ids=str)
def test_commit_of_drafted_trees(fq, torch, trees, heads, page, layers, stride):
    rng = np.random.default_rng(len(trees) + heads + page)
    table, pages, k, v, parents, drafted, following = commit_inputs(rng, trees, heads, page, layers)
    if trees == [(300, 5)]:  # one long chain that is accepted whole but for its end
        parents = [[-1] + list(range(299))]
        drafted = [np.concatenate(([0], following[0][:-1]))]
        drafted[0][280:] += 7
    b = fq.PagedBatch([n for n, _ in trees], [n + c for n, c in trees], table, page, pages)
    dk, dv = dev(torch, k), dev(torch, v)
    path = torch.full((len(trees), stride), 55, dtype=torch.int32, device="cuda")
    got = fq.fq_tree_commit(b, dk, dv, *(dev(torch, join(x)) for x in (parents, drafted, following)), path=path)
    for i, (n, c) in enumerate(trees):
        want, bonus = ref.accept(parents[i], drafted[i], following[i], stride)
        assert path[i].tolist() == want + [-1] * (stride - len(want))
        assert (got[1][i].item(), got[2][i].item(), got[3][i].item()) == (len(want), bonus, c + len(want))
        for l in range(layers):
            ref.keep(k[l], table[i], c, want, page)
            ref.keep(v[l], table[i], c, want, page)
    assert np.array_equal(dk.cpu().numpy(), k) and np.array_equal(dv.cpu().numpy(), v)  # and nothing else has moved


@pytest.mark.parametrize("page, layers", [(16, 2), (128, 1)])
def test_commit_of_given_paths(fq, torch, page, layers):
    rng = np.random.default_rng(page)
    lengths, tails = [300, 90, 40, 200, 33], [250, 5, 0, 200, 33]
    table, pages = deal(rng, lengths, page)
    k, v = (rng.normal(size=(layers, pages, 2, page, 128)).astype(np.float16) for _ in range(2))
    paths = [sorted(rng.choice(250, 130, replace=False).tolist()), [0, 1, 2, 3, 4], [], sorted(rng.choice(200, 64, replace=False).tolist()), [32]]
    stride = 140
    given = np.full((5, stride), -1, dtype=np.int32)
    for i, p in enumerate(paths):
        given[i, :len(p)] = p
    b = fq.PagedBatch([2, 2, 0, 4, 1], lengths, table, page, pages)
    dk, dv = dev(torch, k), dev(torch, v)
    counts = np.array([len(p) for p in paths], dtype=np.int32)
    counts[2] = 9  # cut to the tail, which is empty
    path, accepted, bonus, new_len = fq.fq_tree_commit(b, dk, dv, tail=dev(torch, np.array(tails, dtype=np.int32)), path=dev(torch, given),
                                                       accepted=dev(torch, counts))
    assert bonus is None and new_len.tolist() == [S - t + len(p) for S, t, p in zip(lengths, tails, paths)]
    assert np.array_equal(path.cpu().numpy(), given) and np.array_equal(accepted.cpu().numpy(), counts)
    for i, p in enumerate(paths):
        for l in range(layers):
            ref.keep(k[l], table[i], lengths[i] - tails[i], p, page)
            ref.keep(v[l], table[i], lengths[i] - tails[i], p, page)
    assert np.array_equal(dk.cpu().numpy(), k) and np.array_equal(dv.cpu().numpy(), v)


@pytest.mark.parametrize("page, layers", [(16, 2), (64, 1)])
@pytest.mark.parametrize("path, tail, accepted", [
    ([1, 2, -1], 5, 3), ([7, 9], 2, 2), ([4, 0, 2], 6, 3), ([-3, 2 ** 31 - 1, 1], 40, 99), ([0, 1, 9, -2 ** 31], 4, 4), ([0, 1, 2], 3, 3), ([2, 2, 2, 2], 4, 4),
    ([5, 6, 7], 2, 3), ([6], 30, -1), (list(range(1, 64)) + [-1], 90, 64), (list(range(1, 130)) + [-1], 129, 130), (list(range(64)) + [70, 3, 3, 3], 80, 68)], ids=str)
def test_commit_of_given_paths_that_do_not_rise(fq, torch, page, layers, path, tail, accepted):
    """The nodes of such a path are taken as the header says, and their rows are moved: the last of 64 nodes may be at its place with others that are not."""
    rng = np.random.default_rng(len(path) + tail)
    ahead = [7, 30]  # positions ahead of the tails; the second sequence has the same path
    lengths = [a + tail for a in ahead]
    table, pages = deal(rng, lengths, page)
    k, v = (rng.normal(size=(layers, pages, 3, page, 128)).astype(np.float16) for _ in range(2))
    b = fq.PagedBatch([1, 1], lengths, table, page, pages)
    dk, dv = dev(torch, k), dev(torch, v)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = fq.fq_tree_commit(b, dk, dv, tail=ints(tail, tail), path=dev(torch, np.array([path, path], dtype=np.int32)), accepted=ints(accepted, accepted))
    nodes = ref.given(path, accepted, tail)
    assert got[3].tolist() == [a + len(nodes) for a in ahead]
    for i in range(2):
        for l in range(layers):
            ref.keep(k[l], table[i], ahead[i], nodes, page)
            ref.keep(v[l], table[i], ahead[i], nodes, page)
    assert np.array_equal(dk.cpu().numpy(), k) and np.array_equal(dv.cpu().numpy(), v)


def test_commit_of_a_path_through_a_long_tail(fq, torch):
    """More pages than a wavefront has lanes behind the tail's first, and a path of more than two of its turns."""
    rng = np.random.default_rng(77)
    S, tail, page = 2101, 2050, 16
    table, pages = deal(rng, [S, 33], page)
    k, v = (rng.normal(size=(1, pages, 3, page, 128)).astype(np.float16) for _ in range(2))
    given = sorted(rng.choice(tail, 150, replace=False).tolist())
    paths = np.full((2, 150), -1, dtype=np.int32)
    paths[0], paths[1, :2] = given, [1, 3]
    b = fq.PagedBatch([3, 1], [S, 33], table, page, pages)
    dk, dv = dev(torch, k), dev(torch, v)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = fq.fq_tree_commit(b, dk, dv, tail=ints(tail, 5), path=dev(torch, paths), accepted=ints(150, 2))
    assert got[3].tolist() == [S - tail + 150, 30]
    for pool in (k, v):
        ref.keep(pool[0], table[0], S - tail, given, page)
        ref.keep(pool[0], table[1], 28, [1, 3], page)
    assert np.array_equal(dk.cpu().numpy(), k) and np.array_equal(dv.cpu().numpy(), v)


def test_commit_in_pools_beyond_32_bits(fq, torch):
    """Two layers of 1.15e9 elements each: the second begins behind 2^30 of them, its last pages behind 2^31."""
    rng = np.random.default_rng(5)
    pages, page, kv = 70000, 16, 8
    k, v = (torch.zeros((2, pages, kv, page, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    table = np.array([[pages - 1, 3, pages - 2]])
    rows = rng.normal(size=(2, 2, kv, 40, 128)).astype(np.float16)  # layer, keys or values, head, position
    for which, pool in enumerate((k, v)):
        for t in range(40):
            pool[:, table[0, t // page], :, t % page] = dev(torch, rows[:, which, :, t])
    b = fq.PagedBatch([30], [40], table, page, pages)
    path = [2, 3, 9, 28, 29]
    fq.fq_tree_commit(b, k, v, path=dev(torch, np.array([path], dtype=np.int32)), accepted=dev(torch, np.array([5], dtype=np.int32)))
    want = rows.copy()
    want[:, :, :, 10:15] = rows[:, :, :, [10 + p for p in path]]
    for which, pool in enumerate((k, v)):
        for t in range(40):
            assert np.array_equal(pool[:, table[0, t // page], :, t % page].cpu().numpy(), want[:, which, :, t])
        assert pool[0].count_nonzero().item() <= 40 * kv * 128 and pool[1].count_nonzero().item() <= 40 * kv * 128


def test_commit_without_pages_and_with_bad_paths_stays_inside(fq, torch):
    rng = np.random.default_rng(3)
    b = fq.PagedBatch([20], [50], [[3, 1, 0, 2]], 16, 5)
    b.table[0, 2:] = torch.tensor([-1, 99], device="cuda")
    k = dev(torch, rng.normal(size=(5, 2, 16, 128)).astype(np.float16))  # a pool without layers
    v = k.clone() + 1
    before = k.clone()
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = fq.fq_tree_commit(b, k, v, path=one(4, 9, 19)[None], accepted=one(3))
    # positions 34, 39 and 49 are on pages that the table does not have: nothing to move from
    assert got[3].tolist() == [33] and torch.equal(k, before)
    got = fq.fq_tree_commit(b, k, v, path=one(-3, 2 ** 31 - 1, 7)[None], accepted=one(99))
    assert got[3].tolist() == [33]
    assert torch.equal(k[[0, 2, 4]], before[[0, 2, 4]])


def test_calls_without_tokens(fq, torch):
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    b = fq.PagedBatch.reserve(2, 0, 0, 64, 16, 9, mask_words=1)
    fq.fq_paged_plan(b, ints(0, 3), ints(20, 5), parents=none)
    assert b.q_start.tolist() == [0, 0, 0] and b.seq_len.tolist() == [20, 5] and b.held.tolist() == [2, 1] and b.free_count.item() == 6
    pool = torch.zeros((1, 9, 2, 16, 128), dtype=torch.float16, device="cuda")
    assert fq.fq_attn_tree(torch.zeros((0, 256), dtype=torch.float16, device="cuda"), b, b.mask, pool[0], pool[0].clone()).shape == (0, 256)
    path, accepted, bonus, new_len = fq.fq_tree_commit(b, pool, pool.clone(), none, none, none)
    assert path.tolist() == [[-1], [-1]] and accepted.tolist() == [0, 0] and bonus.tolist() == [-1, -1] and new_len.tolist() == [20, 5]


# ------------------------------------------------------------------ beams
def beam_check(fq, torch, rng, logits, scores, width, done=None, eos=-1, words=0, tail=None, rows=None):
    requests, beams = scores.shape
    vocab = logits.shape[1]
    x = dev(torch, logits) if rows is None else rows
    mask = rng.integers(-2 ** 63, 2 ** 63, size=(requests, beams, words)) if words else None
    got = fq.fq_beam_step(x, dev(torch, scores), width, done=None if done is None else dev(torch, done), eos=eos,
                          mask=None if mask is None else dev(torch, mask), tail=None if tail is None else dev(torch, tail))
    parent, token, out, ended, bits = (None if t is None else t.cpu().numpy() for t in got)
    for r in range(requests):
        p, t, s, d = ref.beam(logits[r * beams:(r + 1) * beams], scores[r], None if done is None else done[r], eos, width)
        assert parent[r].tolist() == p and token[r].tolist() == t, (r, parent[r], p, token[r], t)
        fine = np.isfinite(s)
        assert np.array_equal(fine, np.isfinite(out[r]))
        assert (np.abs(out[r][fine] - s[fine]) <= 2.0 ** -24 * np.abs(s[fine]) + 2.0 ** -40).all()
        if ended is not None:
            assert ended[r].tolist() == d
        if words:
            own = 0 if tail is None else int(tail[r])
            for j in range(width):
                want = [0] * words
                if p[j] >= 0:
                    want = [int(w) % 2 ** 64 for w in mask[r, p[j]]]
                    if 0 <= own + j < 64 * words:
                        want[(own + j) // 64] |= 1 << (own + j) % 64
                assert [int(w) % 2 ** 64 for w in bits[r, j]] == want
    return got


@pytest.mark.parametrize("requests, beams, vocab, width", [
    (1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 8), (1, 4, 32000, 4), (3, 5, 777, 10), (40, 6, 2049, 6), (5, 64, 1000, 64), (2, 64, 40, 64), (9, 16, 32001, 32),
    (1, 2, 262144, 64), (3, 64, 131071, 40), (70, 8, 8191, 8), (33, 1, 50000, 16)])
def test_beam_step(fq, torch, requests, beams, vocab, width):
    rng = np.random.default_rng(vocab + beams)
    logits = (rng.normal(size=(requests * beams, vocab)) * 1.28).astype(np.float16)
    scores = (-rng.random((requests, beams)) * 5).astype(np.float32)
    got = beam_check(fq, torch, rng, logits, scores, min(width, beams * vocab), words=2, tail=rng.integers(0, 140, requests).astype(np.int32))
    again = fq.fq_beam_step(dev(torch, logits), dev(torch, scores), min(width, beams * vocab))
    assert all(torch.equal(a, b) for a, b in zip(got[:3], again[:3])) and again[3] is None and again[4] is None


@pytest.mark.parametrize("vocab, width", [(300, 8), (32000, 20), (9001, 64)])
def test_equal_totals_go_by_index(fq, torch, vocab, width):
    rng = np.random.default_rng(vocab)
    beams = 4
    same = np.zeros((beams, vocab), dtype=np.float16)
    same[:, 1::2] = -0.0  # equal to the others
    zero = np.zeros((1, beams), dtype=np.float32)
    beam_check(fq, torch, rng, same, zero, width)
    steps = np.round(rng.normal(size=(1, vocab)) * 2).astype(np.float16).repeat(beams, 0)  # few different values, all beams alike
    beam_check(fq, torch, rng, steps, zero, width)
    wide = torch.zeros((beams, vocab + 3), dtype=torch.float16, device="cuda")  # rows that begin at other places within 16 bytes
    wide[:, :vocab] = dev(torch, steps)
    beam_check(fq, torch, rng, steps, zero, width, rows=wide[:, :vocab])
    wider = torch.zeros((beams, vocab + 8), dtype=torch.float16, device="cuda")
    wider[:, 5:5 + vocab] = dev(torch, steps)
    beam_check(fq, torch, rng, steps, zero, width, rows=wider[:, 5:5 + vocab])


@pytest.mark.parametrize("requests, beams, vocab, width", [(40, 5, 1, 5), (9, 16, 777, 20), (3, 64, 9000, 64), (1, 4, 32000, 4), (150, 8, 20000, 8), (2, 2, 262144, 3)])
def test_beams_whose_tokens_are_forced_keep_their_scores(fq, torch, requests, beams, vocab, width):
    """A row of one token has a log probability of 0, so its beam's total is its score to the last bit, whatever the logit: equal scores tie, and go by index, also with
    those of beams that have ended."""
    rng = np.random.default_rng(vocab + beams)
    logits = np.full((requests * beams, vocab), -np.inf, dtype=np.float16)
    value = rng.normal(size=requests * beams) * rng.choice([1e-4, 1.0, 30.0, 20000.0], size=requests * beams)
    logits[np.arange(requests * beams), rng.integers(0, vocab, requests * beams)] = np.clip(value, -65504, 65504)
    scores = rng.choice(np.array([0.0, -0.0, -1e-12, -0.1, -0.1, -3.7, -250.3], dtype=np.float32), size=(requests, beams))
    got = beam_check(fq, torch, rng, logits, scores, width)
    done = (rng.random((requests, beams)) < 0.4).astype(np.int32)
    ended = beam_check(fq, torch, rng, logits, scores, width, done=done, eos=vocab // 2, words=1)
    for parent, out in ((g[0].cpu().numpy(), g[2].cpu().numpy()) for g in (got, ended)):
        kept = np.take_along_axis(scores, np.maximum(parent, 0).astype(np.int64), 1)
        assert np.array_equal(out[parent >= 0], kept[parent >= 0]) and np.isneginf(out[parent < 0]).all()


def test_beams_that_are_not_there_and_logits_that_are_not_finite(fq, torch):
    rng = np.random.default_rng(2)
    requests, beams, vocab = 6, 5, 3000
    logits = rng.normal(size=(requests, beams, vocab)).astype(np.float16)
    scores = (-rng.random((requests, beams))).astype(np.float32)
    scores[0, 1:] = -np.inf                 # a first step
    scores[1, 2] = np.nan
    logits[2, 0, 17] = np.nan               # poisons its beam
    logits[2, 1, 2999] = np.inf
    logits[3, :, 5:] = -np.inf              # a vocabulary masked but for five tokens
    logits[4, 1:] = -np.inf                 # beams without any token
    logits[4, 0, 3:] = -np.inf
    scores[5] = -np.inf
    logits[3, 2] = -65504
    with np.errstate(all="ignore"):
        beam_check(fq, torch, rng, logits.reshape(-1, vocab), scores, 9, words=1)
        beam_check(fq, torch, rng, logits.reshape(-1, vocab), scores, 30, eos=2)


@pytest.mark.parametrize("eos", [0, 2, 999])
def test_beams_that_have_ended(fq, torch, eos):
    rng = np.random.default_rng(eos)
    requests, beams, vocab = 9, 6, 1000
    logits = (rng.normal(size=(requests * beams, vocab)) * 1.28).astype(np.float16)
    scores = (-rng.random((requests, beams)) * 20).astype(np.float32)
    done = (rng.random((requests, beams)) < 0.5).astype(np.int32)
    done[0], done[1] = 1, 0
    scores[0, 1] = scores[0, 3]
    scores[2, 0], done[2, 0] = -np.inf, 1
    logits[3 * beams] = np.nan  # not looked at where the beam has ended
    done[3, 0] = 5
    with np.errstate(all="ignore"):
        beam_check(fq, torch, rng, logits, scores, 8, done=done, eos=eos, words=1, tail=np.arange(requests, dtype=np.int32) * 9)
        beam_check(fq, torch, rng, logits, scores, 8, eos=eos)


def test_rows_of_logits_beyond_32_bits(fq, torch):
    rng = np.random.default_rng(6)
    beams, vocab, ld = 10, 3001, (1 << 28) + 1  # rows at odd places, the last one behind 2^31 elements
    wide = torch.empty(9 * ld + vocab, dtype=torch.float16, device="cuda")
    rows = torch.as_strided(wide, (beams, vocab), (ld, 1))
    logits = rng.normal(size=(beams, vocab)).astype(np.float16)
    rows.copy_(dev(torch, logits))
    beam_check(fq, torch, rng, logits, (-rng.random((2, 5))).astype(np.float32), 7, rows=rows)


def test_mask_bits_outside_the_words_are_left_out(fq, torch):
    rng = np.random.default_rng(1)
    logits = rng.normal(size=(4, 50)).astype(np.float16)
    beam_check(fq, torch, rng, logits, np.zeros((2, 2), dtype=np.float32), 5, words=1, tail=np.array([61, -2], dtype=np.int32))


# ------------------------------------------------------------------ graphs
def test_a_captured_step_of_drafted_trees_follows_lengths_on_the_device(fq, torch):
    """Plan, write, attention and commit in one graph; lengths, trees and what the model says change between replays, and pages run from
    closed sequences to growing ones.  Every replay is compared with the same calls made eagerly on a state of their own."""
    rng = np.random.default_rng(8)
    seqs, heads, kv, page, pages, max_q, max_len, layers = 3, 8, 2, 16, 40, 12, 160, 2
    tokens = seqs * max_q
    rope = fq.rope_table(max_len)

    class State:
        def __init__(s):
            s.b = fq.PagedBatch.reserve(seqs, tokens, max_q, max_len, page, pages, mask_words=1)
            s.k, s.v = (torch.zeros((layers, pages, kv, page, 128), dtype=torch.float16, device="cuda") for _ in range(2))
            s.cached, s.new, s.path = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in (seqs, seqs, (seqs, max_q)))
            s.parents, s.drafted, s.following = (torch.zeros(tokens, dtype=torch.int32, device="cuda") for _ in range(3))
            s.accepted, s.bonus, s.new_len = (torch.zeros(seqs, dtype=torch.int32, device="cuda") for _ in range(3))
            s.q, s.kn, s.vn = (torch.zeros((tokens, 128 * h), dtype=torch.float16, device="cuda") for h in (heads, kv, kv))
            s.turned, s.out = torch.zeros_like(s.q), torch.zeros_like(s.q)
            s.ws = torch.zeros(fq.fq_attn_tree_workspace_bytes(s.b, heads, kv) or 16, dtype=torch.uint8, device="cuda")

        def step(s):
            fq.fq_paged_plan(s.b, s.new, s.cached, parents=s.parents)
            for l in range(layers):
                fq.fq_qk_norm_rope(s.q, s.kn, s.vn, s.b, rope, s.k[l], s.v[l], out=s.turned)
                fq.fq_attn_tree(s.turned, s.b, s.b.mask, s.k[l], s.v[l], out=s.out, workspace=s.ws)
            fq.fq_tree_commit(s.b, s.k, s.v, s.parents, s.drafted, s.following, path=s.path, accepted=s.accepted, bonus=s.bonus, new_len=s.new_len)
            s.cached.copy_(s.new_len)

        def all(s):
            return [s.b.q_start, s.b.seq_len, s.b.table, s.b.positions, s.b.slots, s.b.held, s.b.free_count, s.b.lacking, s.b.mask, s.k, s.v, s.path,
                    s.accepted, s.bonus, s.cached, s.out]

    graphed, eager = State(), State()
    warm = State()
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for turn in range(9):
        new = rng.integers(1, max_q + 1, seqs)
        if turn in (4, 7):
            new[turn % seqs] = -1
        parents = join([random_tree(rng, max(n, 0)) for n in new])
        fill = lambda a: np.concatenate((a, np.zeros(tokens - len(a), dtype=a.dtype)))
        following = rng.integers(0, 3, tokens).astype(np.int32)
        drafted = rng.integers(0, 3, tokens).astype(np.int32)
        rows = [rng.normal(size=(tokens, 128 * h)).astype(np.float16) for h in (heads, kv, kv)]
        for s in (graphed, eager):
            s.new.copy_(dev(torch, new.astype(np.int32)))
            s.parents.copy_(dev(torch, fill(parents).astype(np.int32)))
            s.following.copy_(dev(torch, following))
            s.drafted.copy_(dev(torch, drafted))
            for t, a in zip((s.q, s.kn, s.vn), rows):
                t.copy_(dev(torch, a))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(graphed.all(), eager.all())):
            assert torch.equal(a, b), (turn, i)
    assert graphed.cached.min().item() > 0 and graphed.b.lacking.item() == 0


def test_a_captured_beam_step_is_replayed(fq, torch):
    rng = np.random.default_rng(21)
    requests, beams, vocab = 4, 5, 2500
    x = torch.zeros((requests * beams, vocab), dtype=torch.float16, device="cuda")
    scores = torch.zeros((requests, beams), device="cuda")
    ws = torch.zeros(fq.fq_beam_step_workspace_bytes(requests, beams, vocab, beams), dtype=torch.uint8, device="cuda")
    outs = dict(parent=torch.zeros((requests, beams), dtype=torch.int32, device="cuda"), token=torch.zeros((requests, beams), dtype=torch.int32, device="cuda"),
                scores_out=torch.zeros((requests, beams), device="cuda"))
    fq.fq_beam_step(x, scores, beams, workspace=ws, **outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.fq_beam_step(x, scores, beams, workspace=ws, **outs)
    for _ in range(5):
        x.copy_(dev(torch, rng.normal(size=(requests * beams, vocab)).astype(np.float16)))
        scores.copy_(dev(torch, -rng.random((requests, beams)).astype(np.float32)))
        graph.replay()
        got = [t.clone() for t in outs.values()]
        ws.fill_(0xff)  # its contents do not matter
        want = fq.fq_beam_step(x, scores, beams)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[:3]))


# ------------------------------------------------------------------ refusals of the binding
def test_what_the_binding_refuses(fq, torch):
    """Wrong types, shapes, places and batches: nothing of it reaches a launch, with outputs given and without."""
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")
    ints = lambda *s: z(*s, t=torch.int32)
    b, host = (fq.PagedBatch([1, 2], [20, 9], [[0, 1], [2, -1]], 16, 4, device=d) for d in ("cuda", "cpu"))
    q, pool, mask = z(3, 512), z(4, 2, 16, 128), z(3, 1, t=torch.int64)
    out = z(3, 512)
    for more in ({}, {"out": out, "workspace": z(1 << 16, t=torch.uint8)}):
        for args, kw in (((q, host, mask, pool, pool), {}), ((q[:2], b, mask, pool, pool), {}), ((z(3, 300), b, mask, pool, pool), {}),
                         ((q, b, mask.int(), pool, pool), {}), ((q, b, z(2, 1, t=torch.int64), pool, pool), {}), ((q, b, z(3, 65, t=torch.int64), pool, pool), {}),
                         ((q, b, mask, pool[:3], pool[:3]), {}), ((q, b, mask, pool.float(), pool), {}), ((q, b, mask, pool, pool), {"tail": ints(3)}),
                         ((q, b, mask, pool, pool), {"tail": z(2, t=torch.int64)}), ((q, b, mask, pool, pool), {"lse": z(3, 3, t=torch.float32)}),
                         ((q, b, mask.cpu(), pool, pool), {})):
            with pytest.raises((TypeError, ValueError)):
                fq.fq_attn_tree(*args, **kw, **more)
    with pytest.raises(fq.FqError):
        fq.fq_attn_tree(q, b, mask, pool, pool, out=q)
    pools = z(2, 4, 2, 16, 128), z(2, 4, 2, 16, 128)
    three = ints(3)
    for more in ({}, {"path": ints(2, 3), "accepted": ints(2), "bonus": ints(2), "new_len": ints(2)}):
        for kw in ({"parents": three, "drafted": three}, {"parents": ints(2), "drafted": three, "following": three},
                   {"parents": three.long(), "drafted": three, "following": three}, {"parents": three, "drafted": three.cpu(), "following": three}):
            with pytest.raises((TypeError, ValueError)):
                fq.fq_tree_commit(b, *pools, **kw, **more)
        with pytest.raises((TypeError, ValueError)):
            fq.fq_tree_commit(host, *pools, three, three.clone(), three.clone(), **more)
        with pytest.raises((TypeError, ValueError)):
            fq.fq_tree_commit(b, pools[0][:, :3], pools[1][:, :3], three, three.clone(), three.clone(), **more)
    with pytest.raises(ValueError):
        fq.fq_tree_commit(b, *pools)  # neither a tree nor a path
    with pytest.raises(fq.FqError):
        fq.fq_tree_commit(b, *pools, three, three.clone(), three.clone(), new_len=b.seq_len)
    with pytest.raises(fq.FqError):
        fq.fq_tree_commit(b, pools[0], pools[0], three, three.clone(), three.clone())
    r = fq.PagedBatch.reserve(2, 6, 4, 64, 16, 9, mask_words=1)
    for args, kw in (((ints(3), ints(2)), {}), ((ints(2), ints(2).long()), {}), ((ints(2), ints(2)), {"parents": ints(5)}), ((ints(2), ints(2)), {"held_out": ints(1)}),
                     ((ints(2), ints(2)), {"free_out": ints(2)}), ((ints(2), ints(2)), {"next_position": ints(6)}), ((ints(2).cpu(), ints(2)), {}), ((ints(2), None), {})):
        with pytest.raises((TypeError, ValueError)):
            fq.fq_paged_plan(r, *args, **kw)
    with pytest.raises(ValueError):
        fq.fq_paged_plan(b, ints(2), ints(2))  # not a reserved one
    with pytest.raises(fq.FqError):
        fq.fq_paged_plan(r, r.seq_len, ints(2))
    x, scores = z(6, 50), z(2, 3, t=torch.float32)
    outs = {"parent": ints(2, 4), "token": ints(2, 4), "scores_out": z(2, 4, t=torch.float32), "workspace": z(1 << 16, t=torch.uint8)}
    for more in ({}, outs):
        for args, kw in (((x[:5], scores, 4), {}), ((x.float(), scores, 4), {}), ((x, scores.half(), 4), {}), ((x, scores, 4), {"done": ints(2, 4), "eos": 1}),
                         ((x, scores, 4), {"mask": z(2, 4, 1, t=torch.int64)}), ((x, scores, 4), {"tail": ints(3)}), ((x.t(), scores, 4), {}),
                         ((x, scores, 4), {"mask_out": z(2, 3, 1, t=torch.int64)}), ((x, scores.cpu(), 4), {})):
            with pytest.raises((TypeError, ValueError)):
                fq.fq_beam_step(*args, **kw, **more)
        for kw in ({"eos": 50}, {"done": ints(2, 3)}):
            with pytest.raises(fq.FqError):
                fq.fq_beam_step(x, scores, 4, **kw, **more)
    with pytest.raises(fq.FqError):
        fq.fq_beam_step(x, scores, 65)
    torch.cuda.synchronize()
    assert (out == 0).all()
