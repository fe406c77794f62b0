"""Operators over a paged key/value cache against oracle/paged_ref.py (fp64, position by position).

Bounds, each from the roundings that the kernels make (u = 2^-11, half a step of fp16):
  rotation   fp32 in between (norm: a sum of 128, a division, a root) and one rounding: u |y| + 2^-18 (|a| + |b|) of the pair, and 2^-24 for
             results below the fp16 normal range
  attention  scores are fp32 sums of 128 products, so off by at most e = 130 * 2^-24 * (scale sum |q||k|) + 2^-20 absolute, which changes
             every weight by a factor within 1 +- 2 e; weights rounded to fp16: u each (or 2^-25 of the largest one, which is at least
             2^-25 sum over positions of |v|); output rounded: u |out| + 2^-25
  lse        e + 2^-20 |lse|        column sums   factor within 1 +- 2 (e + 2^-20 |lse|), and 2^-20 of what is added up; a weight below the
             fp32 normal range may be zero (its relative error has no bound in fp32): 2^-126 for every row that sees the position
"""
import numpy as np
import pytest

from oracle import paged_ref as ref

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
    """A table of shuffled pages for sequences of these lengths; (table, pages)."""
    need = [-(-s // page) for s in lengths]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table, at = np.full((len(lengths), max(max(need), 1)), -1), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def pools(rng, pages, kv, page, table, lengths, std=1.2):
    """Pools that hold NaN wherever no sequence has a position."""
    k, v = (np.full((pages, kv, page, 128), np.nan, dtype=np.float16) for _ in range(2))
    for b, S in enumerate(lengths):
        for i in range(-(-S // page)):
            rows = min(page, S - i * page)
            for pool in (k, v):
                pool[table[b, i], :, :rows] = (rng.normal(size=(kv, rows, 128)) * std).astype(np.float16)
    return k, v


def case(rng, seqs, heads, kv, page, std=1.2):
    """seqs: (tokens, positions) of every sequence."""
    lengths = [S for _, S in seqs]
    table, pages = deal(rng, lengths, page)
    k, v = pools(rng, pages, kv, page, table, lengths, std)
    q = (rng.normal(size=(sum(n for n, _ in seqs), heads * 128)) * std).astype(np.float16)
    return table, pages, k, v, q


def check(got, lse, w, w_in, seqs, table, k, v, q, heads, kv, scale):
    """Output, lse and column sums (None: not looked at) of every sequence against the reference, within the bounds above."""
    at = 0
    for b, (n, S) in enumerate(seqs):
        K, V = ref.rows_of(k, table[b], S), ref.rows_of(v, table[b], S)
        out, L, sums, mass, size = ref.attention(q[at:at + n], K, V, n, scale)
        e = 130 * 2.0 ** -24 * size + 2.0 ** -20
        floor = 2.0 ** -25 * (1 + (np.abs(V.astype(np.float64)).sum(1).max() if S else 0.0))
        bound = U * (np.abs(out) + mass) * 1.01 + 2 * e * mass + floor
        err = np.abs(got[at:at + n].astype(np.float64) - out)
        assert (err <= bound).all(), (b, n, S, float((err / bound).max()))
        if lse is not None:
            fine = np.isfinite(L)
            assert np.array_equal(fine, np.isfinite(lse[at:at + n])) and np.isneginf(lse[at:at + n][~fine]).all()
            assert (np.abs(lse[at:at + n][fine] - L[fine]) <= e + 2.0 ** -20 * np.abs(L[fine])).all()
        if w is not None:
            rel = 2 * (e + 2.0 ** -20 * (np.abs(L[np.isfinite(L)]).max() if np.isfinite(L).any() else 0.0))
            before = np.where(np.arange(S) < S - n, w_in[b, :, :S].astype(np.float64), 0.0) if w_in is not None else 0.0
            want = before + sums
            err = np.abs(w[b, :, :S] - want)
            assert (err <= rel * sums + 2.0 ** -20 * want + n * (heads // kv) * 2.0 ** -126).all(), (b, n, S, float(err.max()))
        at += n


def run(fq, torch, rng, seqs, heads, kv, page, weights=True, scale=None, std=1.2):
    table, pages, k, v, q = case(rng, seqs, heads, kv, page, std)
    b = fq.PagedBatch([n for n, _ in seqs], [S for _, S in seqs], table, page, pages)
    lse = torch.full((b.tokens, heads), 7.0, device="cuda")
    w_in = rng.exponential(size=(len(seqs), kv, b.max_len + 3)).astype(np.float32) if weights else None
    w_out = torch.full((len(seqs), kv, b.max_len + 3), -5.0, device="cuda") if weights else None
    args = (dev(torch, q), b, dev(torch, k), dev(torch, v))
    more = dict(lse=lse, weights=dev(torch, w_in) if weights else None, weights_out=w_out)
    out = fq.fq_attn_paged(*args, scale=scale, **more)
    w = w_out.cpu().numpy() if weights else None
    check(out.cpu().numpy(), lse.cpu().numpy(), w, w_in, seqs, table, k, v, q, heads, kv, scale or 128 ** -0.5)
    if weights:
        for i, (_, S) in enumerate(seqs):
            assert (w[i, :, S:] == -5.0).all()  # nothing behind a sequence's positions
    # the same bits every time, with and without what is optional
    again = fq.fq_attn_paged(*args, scale=scale)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    if weights:
        w2 = more["weights"].clone()
        fq.fq_attn_paged(*args, scale=scale, weights=w2, weights_out=w2)  # in place
        for i, (_, S) in enumerate(seqs):
            assert torch.equal(w2[i, :, :S], w_out[i, :, :S])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads, kv", [(2, 2), (4, 1), (10, 2), (7, 1), (16, 1), (3, 3)])
def test_single_tokens(fq, torch, heads, kv, page):
    rng = np.random.default_rng(heads * 1000 + page)
    run(fq, torch, rng, [(1, S) for S in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300)], heads, kv, page)


@pytest.mark.parametrize("S", [511, 512, 513, 1000, 1024, 1025, 2049, 4100])
@pytest.mark.parametrize("heads, kv", [(1, 1), (8, 2), (20, 1)])
def test_single_token_of_a_long_sequence(fq, torch, heads, kv, S):
    run(fq, torch, np.random.default_rng(S), [(1, S)], heads, kv, 64)


@pytest.mark.parametrize("heads, kv", [(2, 2), (8, 2), (5, 1), (28, 4), (40, 1)])
@pytest.mark.parametrize("n, cached", [(2, 0), (3, 500), (5, 11), (15, 1), (16, 16), (17, 0), (31, 33), (32, 100), (33, 64), (63, 65), (64, 0),
                                       (65, 127), (100, 300), (129, 1), (150, 700)])
def test_chunks(fq, torch, heads, kv, n, cached):
    run(fq, torch, np.random.default_rng(n + cached), [(n, n + cached)], heads, kv, 32)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("heads, kv", [(2, 2), (8, 2), (7, 1)])
def test_ragged_batches(fq, torch, heads, kv, page):
    """Single tokens, chunks, sequences without tokens, without positions, and with more tokens than positions in one call."""
    rng = np.random.default_rng(page + heads)
    run(fq, torch, rng, [(1, 40), (0, 77), (70, 70), (1, 300), (0, 0), (5, 3), (19, 140), (3, 0), (1, 1), (40, 290), (130, 131)], heads, kv, page)


@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("seqs, heads, kv, route", [
    ([(2048, 2048)], 32, 16, (128, 1)), ([(1700, 1701), (3, 900)], 32, 32, (64, 1)), ([(256, 4000)], 32, 8, (128, 4)),
    ([(100, 2000)], 32, 16, (64, 4)), ([(300, 1000)], 40, 8, (64, 1))], ids=str)
def test_every_division(fq, torch, seqs, heads, kv, route, page):
    """Both heights of the tiles, with and without splits, tiles in one page and of several."""
    table, pages = deal(np.random.default_rng(0), [S for _, S in seqs], page)
    b = fq.PagedBatch([n for n, _ in seqs], [S for _, S in seqs], table, page, pages)
    assert fq.fq_attn_paged_route(b, heads, kv)[:2] == route
    run(fq, torch, np.random.default_rng(47), seqs, heads, kv, page)


@pytest.mark.parametrize("heads, kv, n, cached", [(24, 1, 129, 700), (64, 1, 70, 3), (20, 2, 90, 300)])
def test_column_sums_of_many_rows(fq, torch, heads, kv, n, cached):
    """Rows that are dealt to several parts, some of which see none of the later positions."""
    run(fq, torch, np.random.default_rng(59), [(n, n + cached), (2, 40), (0, 300), (n // 2, n)], heads, kv, 64)


def test_many_sequences(fq, torch):
    """More sequences than a wavefront has lanes; some without tokens."""
    rng = np.random.default_rng(3)
    run(fq, torch, rng, [(int(rng.integers(0, 4)), int(rng.integers(1, 90))) for _ in range(150)], 4, 2, 16)


def test_rows_that_see_nothing_and_calls_without_tokens(fq, torch):
    rng = np.random.default_rng(5)
    run(fq, torch, rng, [(4, 0), (20, 3), (2, 1)], 8, 2, 16)
    run(fq, torch, rng, [(0, 33), (0, 0), (0, 200)], 8, 2, 16)
    run(fq, torch, rng, [(3, 0), (1, 0)], 8, 2, 16)
    run(fq, torch, rng, [(30, 0)], 8, 2, 16)
    run(fq, torch, rng, [(0, 0)], 8, 2, 16)


@pytest.mark.parametrize("scale, std", [(1.0, 1.0), (0.01, 3.0), (128 ** -0.5, 6.0)])
def test_scales(fq, torch, scale, std):
    """Weights from nearly equal to all on one position."""
    run(fq, torch, np.random.default_rng(9), [(1, 700), (40, 333)], 8, 2, 64, scale=scale, std=std)


def test_rows_of_a_wider_product(fq, torch):
    rng = np.random.default_rng(11)
    seqs = [(3, 50), (1, 9)]
    table, pages, k, v, q = case(rng, seqs, 4, 2, 16)
    wide = torch.full((4, 4 * 128 + 64), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 64:] = dev(torch, q)
    b = fq.PagedBatch([3, 1], [50, 9], table, 16, pages)
    got = fq.fq_attn_paged(wide[:, 64:], b, dev(torch, k), dev(torch, v))
    want = fq.fq_attn_paged(dev(torch, q), b, dev(torch, k), dev(torch, v))
    assert torch.equal(got, want)
    with pytest.raises(fq.FqError) as e:
        fq.fq_attn_paged(wide[:, 4:4 + 512], b, dev(torch, k), dev(torch, v))  # rows that start between 16-byte boundaries
    assert e.value.code == -5


def test_pages_shared_by_sequences(fq, torch):
    """Two sequences with one prefix: the same pages in both rows of the table."""
    rng = np.random.default_rng(13)
    table, pages, k, v, q = case(rng, [(1, 48)], 4, 2, 16)
    one = fq.PagedBatch([1], [48], table, 16, pages)
    two = fq.PagedBatch([1, 1], [48, 48], np.concatenate((table, table)), 16, pages)
    a = fq.fq_attn_paged(dev(torch, q), one, dev(torch, k), dev(torch, v))
    b = fq.fq_attn_paged(dev(torch, np.concatenate((q, q))), two, dev(torch, k), dev(torch, v))
    assert torch.equal(a, b[:1]) and torch.equal(a, b[1:])


def test_pools_beyond_four_gib(fq, torch):
    """A page whose byte offset needs more than 32 bits, and whose row times 128 does."""
    heads = kv = 8
    page, pages = 256, 10500  # 5.5 GB each
    rng = np.random.default_rng(17)
    k, v = (torch.empty(pages, kv, page, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    lengths, table = [300, 40], np.array([[pages - 1, 9000], [8300, -1]])
    small = {}
    for name, pool in (("k", k), ("v", v)):
        small[name] = np.zeros((3, kv, page, 128), dtype=np.float16)
        for i, p in enumerate((pages - 1, 9000, 8300)):
            small[name][i] = rng.normal(size=(kv, page, 128)).astype(np.float16)
            pool[p] = dev(torch, small[name][i])
    q = rng.normal(size=(21, heads * 128)).astype(np.float16)
    b = fq.PagedBatch([1, 20], lengths, table, page, pages)
    w = torch.zeros(2, kv, 300, device="cuda")
    out = fq.fq_attn_paged(dev(torch, q), b, k, v, weights_out=w)
    check(out.cpu().numpy(), None, w.cpu().numpy(), None, [(1, 300), (20, 40)], np.array([[0, 1], [2, 2]]), small["k"], small["v"], q, heads, kv,
          128 ** -0.5)
    # and the write into such a page, then a copy from there
    rope = fq.rope_table(300)
    x = dev(torch, rng.normal(size=(21, heads * 128)).astype(np.float16))
    fq.fq_qk_norm_rope(x, x, x, b, rope, k, v)
    assert torch.equal(v[9000, :, 43], x[0].view(kv, 128)) and torch.equal(v[8300, :, 20:40], x[1:].view(20, kv, 128).transpose(0, 1))
    dst = torch.tensor([[10400], [10401]], dtype=torch.int32, device="cuda")
    kept, new_len = fq.fq_cache_evict(b, w, k, v, dst, 200, 50)
    assert new_len.tolist() == [200, 40]
    for h in range(kv):
        t = kept[0, h].long()
        p = torch.where(t < 256, pages - 1, 9000)
        assert torch.equal(k[10400, h, :200], k[p, h, t % 256]) and torch.equal(v[10400, h, :200], v[p, h, t % 256])
    assert torch.equal(k[10401, :, :40], k[8300, :, :40])


def test_other_stream_and_workspace(fq, torch):
    rng = np.random.default_rng(19)
    seqs = [(1, 900), (2, 800)]
    table, pages, k, v, q = case(rng, seqs, 4, 1, 32)
    b = fq.PagedBatch([1, 2], [900, 800], table, 32, pages)
    args = (dev(torch, q), b, dev(torch, k), dev(torch, v))
    w0, w1 = (torch.zeros(2, 1, 900, device="cuda") for _ in range(2))
    want = fq.fq_attn_paged(*args, weights_out=w0)
    need = fq.fq_attn_paged_workspace_bytes(b, 4, 1, True)
    assert need > 0
    guarded = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    out = torch.full((3 * 512 + 256,), 3.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = fq.fq_attn_paged(*args, out=out[128:-128].view(3, 512), weights_out=w1, workspace=guarded[256:-256], stream=s)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(w0, w1)
    assert (guarded[:256] == 0x5A).all() and (guarded[-256:] == 0x5A).all() and (out[:128] == 3).all() and (out[-128:] == 3).all()
    got = fq.fq_attn_paged(*args, stream=s.cuda_stream)  # scratch and output made by the call
    s.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(fq.FqError) as e:
        fq.fq_attn_paged(*args, weights_out=w1, workspace=guarded[:need - 300])
    assert e.value.code == -6


def test_graph_replays_with_other_lengths(fq, torch):
    """A captured step, replayed while the sequences grow inside the bounds it was captured with."""
    rng = np.random.default_rng(23)
    heads, kv, page, most = 8, 2, 16, 700
    table, pages = deal(rng, [most, most, most], page)
    k, v = pools(rng, pages, kv, page, table, [most] * 3)
    dk, dv = dev(torch, k), dev(torch, v)
    q = (rng.normal(size=(3, heads * 128)) * 1.2).astype(np.float16)
    x = dev(torch, q)
    b = fq.PagedBatch([1, 1, 1], [most] * 3, table, page, pages)
    out, lse, w = torch.empty_like(x), torch.empty(3, heads, device="cuda"), torch.zeros(3, kv, most, device="cuda")
    ws = torch.empty(fq.fq_attn_paged_workspace_bytes(b, heads, kv, True), dtype=torch.uint8, device="cuda")
    call = lambda: fq.fq_attn_paged(x, b, dk, dv, out=out, lse=lse, weights_out=w, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([1, 30, 600], [699, 700, 17], [128, 129, 257], [256, 255, 1]):
        b.seq_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check(out.cpu().numpy(), lse.cpu().numpy(), w.cpu().numpy(), None, [(1, S) for S in lengths], table, k, v, q, heads, kv, 128 ** -0.5)


def test_what_is_not_finite_stays_where_it_is_seen(fq, torch):
    """NaN in a key or value reaches the rows that see its position, and no others; so does an infinite value."""
    rng = np.random.default_rng(29)
    heads, kv, page = 4, 2, 16
    for n, S, t in ((1, 60, 20), (20, 60, 20), (150, 400, 300)):
        table, pages, k, v, q = case(rng, [(n, S), (n, S)], heads, kv, page)
        k[table[0, t // page], 1, t % page, 5] = np.nan
        b = fq.PagedBatch([n, n], [S, S], table, page, pages)
        out = fq.fq_attn_paged(dev(torch, q), b, dev(torch, k), dev(torch, v)).cpu().numpy().reshape(2, n, heads, 128)
        sees = np.arange(n) + S - n >= t
        assert np.isnan(out[0][sees][:, 2:]).all() and np.isfinite(out[0][sees][:, :2]).all()
        assert np.isfinite(out[0][~sees]).all() and np.isfinite(out[1]).all()


@pytest.mark.parametrize("heads, kv, n, S", [(4, 2, 1, 60), (4, 2, 5, 60), (2, 2, 16, 16), (4, 2, 20, 60), (8, 2, 150, 400), (4, 4, 200, 201), (2, 1, 70, 5000), (32, 16, 2048, 2048)])
def test_values_that_are_not_finite(fq, torch, heads, kv, n, S):
    """An infinite or NaN value reaches its dimension of the rows that see its position; rows ahead of it, whose weight is none, stay
    as they are, and so do the other dimensions."""
    rng = np.random.default_rng(61)
    table, pages, k, v, q = case(rng, [(n, S)], heads, kv, 16)
    b = fq.PagedBatch([n], [S], table, 16, pages)
    clean = fq.fq_attn_paged(dev(torch, q), b, dev(torch, k), dev(torch, v)).cpu().numpy().reshape(n, heads, 128)
    old = S - n
    marks = [(t, h, d, x) for t, h, d, x in ((S - 1, 0, 3, np.inf), (old, 0, 4, -np.inf), (old + n // 2, kv - 1, 127, np.nan), (old // 2, 0, 64, np.inf),
                                             (old + n // 3, kv - 1, 126, np.inf), (old + n // 2, kv - 1, 126, -np.inf))]
    want = clean.copy()
    for (t, h, d), x in {m[:3]: m[3] for m in marks}.items():  # of two at one place, as for one token, the last
        v[table[0, t // 16], h, t % 16, d] = x
        rows, group = np.arange(n) + old >= t, heads // kv
        for g in range(h * group, (h + 1) * group):
            with np.errstate(invalid="ignore"):
                want[rows, g, d] += np.float16(x)
    got = fq.fq_attn_paged(dev(torch, q), b, dev(torch, k), dev(torch, v)).cpu().numpy().reshape(n, heads, 128)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    assert np.array_equal(got[fine], clean[fine]) and np.array_equal(np.sign(got[np.isinf(want)]), np.sign(want[np.isinf(want)]))


# ----------------------------------------------------------- norm, rotation, write
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("heads, kv, page", [(1, 1, 16), (32, 32, 64), (40, 8, 32), (7, 1, 256)])
def test_norm_rope(fq, torch, heads, kv, page, norm):
    rng = np.random.default_rng(heads)
    q_lens, lens = [1, 37, 0, 5, 1], [300, 50, 20, 3, 1]
    table, pages = deal(rng, lens, page)
    b = fq.PagedBatch(q_lens, lens, table, page, pages)
    tokens = sum(q_lens)
    qkv = (rng.normal(size=(tokens, (heads + 2 * kv) * 128)) * 1.3).astype(np.float16)
    qkv[0, :128] = 0  # a head of zeros
    qkv[1, 128 * heads:128 * heads + 128] *= np.float16(1e-4)
    gains = (1 + 0.3 * rng.normal(size=(2, 128))).astype(np.float16) if norm else (None, None)
    rope = fq.rope_table(300)
    cut = np.split(qkv, [heads * 128, (heads + kv) * 128], axis=1)
    all_ = dev(torch, qkv)
    q, k, v = torch.split(all_, (heads * 128, kv * 128, kv * 128), 1)
    kp, vp = (torch.full((pages, kv, page, 128), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    out = fq.fq_qk_norm_rope(q, k, v, b, rope, kp, vp, *(None if g is None else dev(torch, g) for g in gains), eps=1e-5)
    positions, table64 = b.positions.cpu().numpy(), rope.cpu().numpy()
    slots = b.slots.cpu().numpy()
    assert (slots < 0).sum() == 2  # five tokens in three positions
    want_k = np.full((pages, kv, page, 128), 9.0)
    written = np.zeros((pages, page), dtype=bool)
    for name, x, gain in (("q", cut[0], gains[0]), ("k", cut[1], gains[1])):
        y = ref.norm_rope(x, positions, table64, gain)
        size = ref.norm_rope(np.abs(x), positions, np.abs(table64) * [1, -1], None if gain is None else np.abs(gain))  # |a||c| + |b||s| of even ones
        pair = np.maximum(size.reshape(tokens, -1, 2).max(-1), np.abs(y).reshape(tokens, -1, 2).max(-1))
        bound = U * np.abs(y) + 2.0 ** -18 * 2 * np.repeat(pair, 2, axis=1) + 2.0 ** -24
        if name == "q":
            assert (np.abs(out.cpu().numpy() - y) <= bound).all()
            continue
        got = kp.cpu().numpy()
        for m, s in enumerate(slots):
            if s >= 0:
                written[s // page, s % page] = True
                assert (np.abs(got[s // page, :, s % page].reshape(-1) - y[m]) <= bound[m]).all(), m
                assert np.array_equal(vp.cpu().numpy()[s // page, :, s % page].reshape(-1), cut[2][m])
        assert (np.moveaxis(got, 1, 2)[~written] == 9).all() and (np.moveaxis(vp.cpu().numpy(), 1, 2)[~written] == 9).all()
    if all_.shape[1] == heads * 128 * 3:
        flat = [t.contiguous() for t in (q, k, v)]
        again = fq.fq_qk_norm_rope(*flat, b, rope, kp, vp, *(None if g is None else dev(torch, g) for g in gains), eps=1e-5, out=flat[0])  # in place
        assert torch.equal(again, out)


def test_rotation_agrees_with_the_contiguous_path(fq, torch):
    """Without gains, keys as fq_attn_prefill writes them into its cache, bit for bit."""
    rng = np.random.default_rng(31)
    H, T = 4, 70
    q, k, v = (dev(torch, rng.normal(size=(T, H * 128)).astype(np.float16)) for _ in range(3))
    rope = fq.rope_table(T)
    kc, vc = (torch.zeros(H, T, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    fq.fq_attn_prefill(q, k, v, kc, vc, rope)
    b = fq.PagedBatch([T], [T], [[4, 1, 0, 2, 3]], 16, 5)
    kp, vp = (torch.zeros(5, H, 16, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    fq.fq_qk_norm_rope(q, k, v, b, rope, kp, vp)
    for pool, cache in ((kp, kc), (vp, vc)):
        rows = pool[[4, 1, 0, 2, 3]].transpose(0, 1).reshape(H, 80, 128)[:, :T]
        assert torch.equal(rows, cache)


def test_positions_beyond_the_table_and_slots_outside(fq, torch):
    """What is out of range is cut to the table, or not written."""
    rng = np.random.default_rng(37)
    x = dev(torch, rng.normal(size=(3, 128)).astype(np.float16))
    b = fq.PagedBatch([3], [3], [[0]], 16, 2, positions=[5, 1000, -3])
    b.slots.copy_(torch.tensor([3, 32, -1], dtype=torch.int32))
    rope = fq.rope_table(8)
    kp, vp = (torch.zeros(2, 1, 16, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    out = fq.fq_qk_norm_rope(x, x, x, b, rope, kp, vp).cpu().numpy()
    want = ref.norm_rope(x.cpu().numpy(), [5, 7, 0], rope.cpu().numpy())
    assert np.abs(out - want).max() <= 2.0 ** -10 * np.abs(want).max()
    assert (vp[0, 0, 3] == x[0]).all() and int((vp != 0).any(-1).sum()) == 1


# ----------------------------------------------------------------------- eviction
def weights_like(rng, shape, kind):
    if kind == "spread":
        return rng.exponential(size=shape).astype(np.float32) ** 3
    if kind == "ties":
        return rng.integers(0, 4, size=shape).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, dtype=np.float32)
    w = rng.normal(size=shape).astype(np.float32)  # signs, zeros of both, infinities, NaN
    flat = w.reshape(-1)
    for i, x in enumerate((0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45)):
        flat[i::23] = x
    return w


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("keep, recent", [(1, 0), (1, 1), (16, 5), (100, 0), (100, 100), (333, 64), (1500, 7)])
@pytest.mark.parametrize("lengths", [[1, 0, 40, 100, 101, 1023, 1025, 2200], [1, 0, 63, 64, 65, 101, 334, 1000, 1024]], ids=["long", "short"])
def test_evict(fq, torch, lengths, keep, recent, page, kind):
    rng = np.random.default_rng(keep + page)
    kv = 3
    table, pages = deal(rng, lengths, page)
    k, v = pools(rng, pages, kv, page, table, lengths)
    k, v = np.nan_to_num(k), np.nan_to_num(v)
    w = weights_like(rng, (len(lengths), kv, 2203), kind)
    dst, dst_pages = deal(rng, [min(S, keep) for S in lengths], page)
    b = fq.PagedBatch([0] * len(lengths), lengths, table, page, pages)
    ko, vo = (torch.full((dst_pages, kv, page, 128), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    wo = torch.full((len(lengths), kv, keep + 2), -5.0, device="cuda")
    kept, new_len = fq.fq_cache_evict(b, dev(torch, w), dev(torch, k), dev(torch, v), dev(torch, dst.astype(np.int32)), keep, recent, ko, vo,
                                      weights_out=wo)
    kept, wo, ko, vo = (t.cpu().numpy() for t in (kept, wo, ko, vo))
    assert new_len.tolist() == [min(S, keep) for S in lengths]
    left = np.ones(ko.shape[:3], dtype=bool)
    for i, S in enumerate(lengths):
        m, K, V = min(S, keep), ref.rows_of(k, table[i], S), ref.rows_of(v, table[i], S)
        at = np.arange(m)
        for h in range(kv):
            want = ref.evict(w[i, h, :S], keep, recent)
            assert np.array_equal(kept[i, h, :m], want) and (kept[i, h, m:] == -1).all(), (S, h)
            assert np.array_equal(wo[i, h, :m].view(np.int32), w[i, h, want].view(np.int32)) and (wo[i, h, m:] == -5).all()
            assert np.array_equal(ko[dst[i, at // page], h, at % page], K[h, want]) and np.array_equal(vo[dst[i, at // page], h, at % page], V[h, want])
            left[dst[i, at // page], h, at % page] = False
    assert (ko[left] == 9).all() and (vo[left] == 9).all()


def test_evict_of_a_very_long_sequence(fq, torch):
    """Many trips of the selection, weights that differ in their last bits only."""
    rng = np.random.default_rng(41)
    S, keep, recent, page = 70001, 30000, 1000, 256
    base = np.float32(0.7).view(np.int32)
    w = (base + rng.integers(0, 5000, size=(1, 1, S))).astype(np.int32).view(np.float32)
    table, pages = deal(rng, [S], page)
    dst, dst_pages = deal(rng, [keep], page)
    b = fq.PagedBatch([0], [S], table, page, pages)
    k = torch.randn(pages, 1, page, 128, device="cuda").half()
    ko, vo = (torch.zeros(dst_pages, 1, page, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    kept, _ = fq.fq_cache_evict(b, dev(torch, w), k, k, dev(torch, dst.astype(np.int32)), keep, recent, ko, vo)
    want = ref.evict(w[0, 0], keep, recent)
    assert np.array_equal(kept.cpu().numpy()[0, 0], want)
    t, d = torch.from_numpy(want).cuda(), torch.from_numpy(dst[0]).cuda()
    rows = k[torch.from_numpy(table[0]).cuda()].view(-1, 128)[t]
    assert torch.equal(ko[d].view(-1, 128)[:keep], rows) and torch.equal(vo[d].view(-1, 128)[:keep], rows)


def test_evict_in_one_pool(fq, torch):
    """Destination pages of the same pools; a graph of the call."""
    rng = np.random.default_rng(43)
    lengths, keep, recent, kv, page = [100, 61], 48, 10, 2, 16
    table, pages = deal(rng, lengths, page, spare=8)
    k, v = pools(rng, pages, kv, page, table, lengths)
    free = np.setdiff1d(np.arange(pages), table)[:6].reshape(2, 3)
    dk, dv, dst = dev(torch, k), dev(torch, v), dev(torch, free.astype(np.int32))
    w = rng.exponential(size=(2, kv, 100)).astype(np.float32)
    b = fq.PagedBatch([0, 0], lengths, table, page, pages)
    kept, new_len = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, kv, keep), (2,)))
    call = lambda: fq.fq_cache_evict(b, x, dk, dv, dst, keep, recent, kept=kept, new_len=new_len)
    x = dev(torch, w)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        w = rng.exponential(size=w.shape).astype(np.float32)
        x.copy_(dev(torch, w))
        graph.replay()
        torch.cuda.synchronize()
        for i, S in enumerate(lengths):
            for h in range(kv):
                want = ref.evict(w[i, h, :S], keep, recent)
                assert np.array_equal(kept[i, h].cpu().numpy(), want)
                assert np.array_equal(dk[dst[i].long(), h].view(-1, 128)[:keep].cpu().numpy(), ref.rows_of(k, table[i], S)[h, want])


# ------------------------------------------------------------------------ refusals
def test_refusals(fq, torch):
    f16 = dict(dtype=torch.float16, device="cuda")
    b = fq.PagedBatch([1, 1], [20, 3], [[0, 1], [2, -1]], 16, 3)
    x, pool = torch.zeros(2, 512, **f16), torch.zeros(3, 2, 16, 128, **f16)
    rope = fq.rope_table(32)
    dst = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    w = torch.zeros(2, 2, 20, device="cuda")
    for bad in (lambda: fq.fq_attn_paged(x.float(), b, pool, pool), lambda: fq.fq_attn_paged(x, b, pool.float(), pool),
                lambda: fq.fq_attn_paged(x, b, pool, pool, lse=torch.zeros(2, 4, **f16)), lambda: fq.fq_cache_evict(b, w.double(), pool, pool, dst, 8, 2),
                lambda: fq.fq_cache_evict(b, w, pool, pool, dst.long(), 8, 2), lambda: fq.fq_qk_norm_rope(x, x[:, :256], x[:, :256], b, rope.half(), pool, pool)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: fq.fq_attn_paged(x[:1], b, pool, pool), lambda: fq.fq_attn_paged(x[:, :384].contiguous(), b, pool, pool),
                lambda: fq.fq_attn_paged(x, b, pool[:2], pool[:2]), lambda: fq.fq_attn_paged(x, b, pool, pool[:, :1].contiguous()),
                lambda: fq.fq_attn_paged(x, b, pool, pool, weights=w), lambda: fq.fq_attn_paged(x, b, pool, pool, weights_out=w[:, :, :19].contiguous()),
                lambda: fq.fq_attn_paged(x, b, pool.view(3, 4, 8, 128), pool.view(3, 4, 8, 128)), lambda: fq.fq_attn_paged(x, b, pool, pool, out=x[:1]),
                lambda: fq.fq_attn_paged(x.t().contiguous().t(), b, pool, pool), lambda: fq.fq_qk_norm_rope(x, x, x, b, rope, pool, pool),
                lambda: fq.fq_qk_norm_rope(x, x[:, :256], x[:, :256], b, rope[:, :32].contiguous(), pool, pool),
                lambda: fq.fq_qk_norm_rope(x, x[:, :256], x[:, :256], b, rope, pool, pool, q_gain=torch.ones(64, **f16)),
                lambda: fq.fq_cache_evict(b, w, pool, pool, dst[:1], 8, 2), lambda: fq.fq_cache_evict(b, w[:, :1].contiguous(), pool, pool, dst, 8, 2),
                lambda: fq.fq_cache_evict(b, w, pool, pool, dst, 8, 2, k_out=pool)):
        with pytest.raises(ValueError):
            bad()
    for code, bad in ((-2, lambda: fq.fq_cache_evict(b, w, pool, pool, dst, 0, 0)), (-2, lambda: fq.fq_cache_evict(b, w, pool, pool, dst, 8, 9)),
                      (-2, lambda: fq.fq_cache_evict(b, w, pool, pool, dst, 18, 2)), (-2, lambda: fq.fq_attn_paged(x, b, pool, pool, out=x)), (-2, lambda: fq.fq_attn_paged(x, b, pool, pool, scale=0.0)),
                      (-2, lambda: fq.fq_cache_evict(b, w, pool, pool, dst, 8, 2, weights_out=w))):
        with pytest.raises(fq.FqError) as e:
            bad()
        assert e.value.code == code


def test_both_ways_of_a_call(fq, torch, monkeypatch):
    """Through the extension module and through ctypes: the same bits; the module takes the calls that allocate nothing."""
    rng = np.random.default_rng(53)
    seqs, heads, kv, page = [(1, 700), (1, 33)], 8, 2, 16
    table, pages, k, v, q = case(rng, seqs, heads, kv, page)
    b = fq.PagedBatch([1, 1], [700, 33], table, page, pages)
    rope, dst = fq.rope_table(700), torch.arange(14, dtype=torch.int32, device="cuda").view(2, 7)
    taken = []
    for name in ("qk_norm_rope", "attn_paged", "cache_evict"):
        def watch(*a, real=getattr(fq._bind, name), name=name):
            rc = real(*a)
            taken.append((name, rc))
            return rc
        monkeypatch.setattr(fq._bind, name, watch)
    results = []
    for module in (fq._bind, None):
        monkeypatch.setattr(fq, "_bind", module)
        x, y, z, dk, dv = (dev(torch, a) for a in (q, q[:, :256].copy(), q[:, 256:512].copy(), np.nan_to_num(k), np.nan_to_num(v)))
        gain = dev(torch, rng.normal(size=128).astype(np.float16) if not results else results[0][0].cpu().numpy())
        fq.fq_qk_norm_rope(x, y, z, b, rope, dk, dv, q_gain=gain, out=x)
        out, lse, w = torch.empty_like(x), torch.empty(2, heads, device="cuda"), torch.zeros(2, kv, 700, device="cuda")
        ws = torch.empty(fq.fq_attn_paged_workspace_bytes(b, heads, kv, True), dtype=torch.uint8, device="cuda")
        fq.fq_attn_paged(x, b, dk, dv, out=out, lse=lse, weights=w, weights_out=w, workspace=ws)
        ko, vo = (torch.zeros(14, kv, page, 128, dtype=torch.float16, device="cuda") for _ in range(2))
        kept, new_len, wo = torch.zeros(2, kv, 100, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, kv, 100, device="cuda")
        fq.fq_cache_evict(b, w, dk, dv, dst, 100, 10, ko, vo, kept, new_len, wo)
        results.append([gain, x, dk, dv, out, lse, w, ko, vo, kept, new_len, wo])
    assert taken == [("qk_norm_rope", 0), ("attn_paged", 0), ("cache_evict", 0)]
    for g, h in zip(*results):
        assert torch.equal(g, h)


@pytest.mark.parametrize("seqs", [15, 16, 30], ids=lambda n: f"{n * 32}heads")
def test_evict_of_many_heads(fq, torch, seqs):
    """On both sides of the number of heads from which the copy is a launch of its own, at short lengths."""
    rng = np.random.default_rng(seqs)
    kv, page, keep, recent = 32, 16, 130, 17
    lengths = [int(n) for n in rng.integers(0, 300, size=seqs)]
    table, pages = deal(rng, lengths, page)
    k, v = (rng.normal(size=(pages, kv, page, 128)).astype(np.float16) for _ in range(2))
    w = weights_like(rng, (seqs, kv, 300), "ties")
    dst, dst_pages = deal(rng, [min(S, keep) for S in lengths], page)
    b = fq.PagedBatch([0] * seqs, lengths, table, page, pages)
    dk, dv = dev(torch, k), dev(torch, v)
    ko, vo = (torch.full((dst_pages, kv, page, 128), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    wo = torch.full((seqs, kv, keep), -5.0, device="cuda")
    kept, new_len = fq.fq_cache_evict(b, dev(torch, w), dk, dv, dev(torch, dst.astype(np.int32)), keep, recent, ko, vo, weights_out=wo)
    kept, wo, ko, vo = (t.cpu().numpy() for t in (kept, wo, ko, vo))
    assert new_len.tolist() == [min(S, keep) for S in lengths]
    for i, S in enumerate(lengths):
        m, K, V = min(S, keep), ref.rows_of(k, table[i], S), ref.rows_of(v, table[i], S)
        at = np.arange(m)
        for h in range(kv):
            want = ref.evict(w[i, h, :S], keep, recent)
            assert np.array_equal(kept[i, h, :m], want) and (kept[i, h, m:] == -1).all(), (S, h)
            assert np.array_equal(wo[i, h, :m].view(np.int32), w[i, h, want].view(np.int32)) and (wo[i, h, m:] == -5).all()
            assert np.array_equal(ko[dst[i, at // page], h, at % page], K[h, want]) and np.array_equal(vo[dst[i, at // page], h, at % page], V[h, want])


@pytest.mark.parametrize("seqs, heads, kv", [([(223, 250), (0, 40), (53, 90)], 8, 1), ([(700, 700)], 4, 1), ([(260, 1300), (17, 2000)], 32, 16),
                                             ([(1, 300), (90, 20), (300, 301)], 14, 2)], ids=["parts", "prompt", "few-parts", "beyond"])
def test_column_sums_in_parts(fq, torch, seqs, heads, kv):
    """Parts of few rows, of sequences of other lengths than the longest; tokens ahead of the first position."""
    run(fq, torch, np.random.default_rng(len(seqs) + heads), seqs, heads, kv, 32)


@pytest.mark.parametrize("lengths, kv, keep, recent", [
    ([1025, 4096, 0, 17], 1, 2000, 100), ([4096, 3000, 1], 40, 700, 0), ([4097, 16384, 5, 9001], 2, 4100, 1000), ([9001, 5], 32, 2500, 64),
    ([16385, 33000, 100], 2, 20000, 8)], ids=["up-to-4096", "up-to-4096-many", "up-to-16384", "up-to-16384-many", "beyond"])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict_of_long_sequences(fq, torch, lengths, kv, keep, recent, kind):
    """Every way that long sequences are selected in, few heads and many."""
    rng = np.random.default_rng(keep)
    page = 64
    table, pages = deal(rng, lengths, page)
    w = weights_like(rng, (len(lengths), kv, max(lengths) + 1), kind)
    dst, dst_pages = deal(rng, [min(S, keep) for S in lengths], page)
    b = fq.PagedBatch([0] * len(lengths), lengths, table, page, pages)
    k, v = (torch.randn(pages, kv, page, 128, device="cuda").half() for _ in range(2))
    ko, vo = (torch.full((dst_pages, kv, page, 128), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    wo = torch.full((len(lengths), kv, keep), -5.0, device="cuda")
    kept, new_len = fq.fq_cache_evict(b, dev(torch, w), k, v, dev(torch, dst.astype(np.int32)), keep, recent, ko, vo, weights_out=wo)
    kept, wo = kept.cpu().numpy(), wo.cpu().numpy()
    assert new_len.tolist() == [min(S, keep) for S in lengths]
    for i, S in enumerate(lengths):
        m = min(S, keep)
        pg, d = (torch.from_numpy(t[i].astype(np.int64)).cuda() for t in (table, dst))
        for h in range(kv):
            want = ref.evict(w[i, h, :S], keep, recent)
            assert np.array_equal(kept[i, h, :m], want) and (kept[i, h, m:] == -1).all(), (S, h)
            assert np.array_equal(wo[i, h, :m].view(np.int32), w[i, h, want].view(np.int32)) and (wo[i, h, m:] == -5).all()
            t, at = torch.from_numpy(want.astype(np.int64)).cuda(), torch.arange(m, device="cuda")
            for src, out in ((k, ko), (v, vo)):
                assert torch.equal(out[d[at // page], h, at % page], src[pg[t // page], h, t % page]), (S, h)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("heads, kv", [(8, 2), (4, 4)])
def test_chunk_beside_a_long_sequence(fq, torch, heads, kv, page):
    """Splits that most sequences have nothing in."""
    seqs = [(60, 60), (1, 5000), (1, 33), (0, 400), (2, 1), (9, 700)]
    table, pages = deal(np.random.default_rng(0), [S for _, S in seqs], page)
    b = fq.PagedBatch([n for n, _ in seqs], [S for _, S in seqs], table, page, pages)
    assert fq.fq_attn_paged_route(b, heads, kv)[1] > 4
    run(fq, torch, np.random.default_rng(heads), seqs, heads, kv, page)


def test_batches_on_the_host_are_refused_with_and_without_outputs(fq, torch, monkeypatch):
    """A batch whose arrays are host memory reaches no entry point, by either way; the entry points are replaced, so that nothing is launched."""
    import ctypes

    names = ("fq_qlinear_tile", "fq_qlinear_mixed", "fq_dense_f16", "fq_head_nll", "fq_token_nll", "fq_logit_l2", "fq_qk_norm_rope",
             "fq_attn_paged", "fq_cache_evict")
    reached = []
    stubs = {n: ctypes.CFUNCTYPE(ctypes.c_int, *getattr(fq._lib, n).argtypes)(lambda *a, n=n: reached.append(n) or -2) for n in names[6:]}
    real = [ctypes.cast(getattr(fq._lib, n), ctypes.c_void_p).value for n in names]
    x, pool = (torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((2, 256), (3, 2, 16, 128)))
    rope, w = torch.zeros(32, 64, 2, device="cuda"), torch.zeros(2, 2, 20, device="cuda")
    ws, out = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros_like(x)
    dst, kept, new_len = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 1), (2, 2, 8), (2,)))
    calls = (lambda b: fq.fq_qk_norm_rope(x, x, x, b, rope, pool, pool, out=out), lambda b: fq.fq_attn_paged(x, b, pool, pool, out=out, workspace=ws),
             lambda b: fq.fq_attn_paged(x, b, pool, pool, out=out, weights_out=w, workspace=ws), lambda b: fq.fq_attn_paged(x, b, pool, pool),
             lambda b: fq.fq_cache_evict(b, w, pool, pool, dst, 8, 2, kept=kept, new_len=new_len), lambda b: fq.fq_cache_evict(b, w, pool, pool, dst, 8, 2))
    host, there = (fq.PagedBatch([1, 1], [20, 3], [[0, 1], [2, -1]], 16, 3, device=d) for d in ("cpu", "cuda"))
    for n, stub in stubs.items():
        monkeypatch.setattr(fq._lib, n, stub)
    try:
        fq._bind.bind(*real[:6], *(ctypes.cast(stubs[n], ctypes.c_void_p).value for n in names[6:]))
        for call in calls:
            with pytest.raises((TypeError, ValueError)):
                call(host)
        assert reached == []
        for call in calls:
            with pytest.raises(fq.FqError):
                call(there)
        assert reached == [names[6], names[7], names[7], names[7], names[8], names[8]]
    finally:
        fq._bind.bind(*real)


@pytest.mark.parametrize("lag", [0.0, 7.9])
@pytest.mark.parametrize("n, S, heads, kv, route", [(1, 380, 8, 8, (16, 1)), (3, 380, 8, 2, (16, 1)), (1, 3000, 8, 2, (16, 24)), (300, 3000, 8, 8, (64, 4)),
                                                    (1500, 3000, 16, 8, (64, 1)), (1024, 4000, 32, 8, (128, 1))], ids=str)
def test_weights_far_below_the_largest(fq, torch, n, S, heads, kv, route, lag):
    """One position takes nearly all of the softmax and has a value of zero: the outputs are the many others, each 2.5 * 2^-24 of it.
    As fp16 numbers of that size they would be off by a fifth.  Terms are held to u of each, or 2^-32 of the largest.  `lag`: the first positions lie that
    many powers of two below the largest."""
    rng = np.random.default_rng(67)
    page = 64
    table, pages = deal(rng, [S], page)
    b = fq.PagedBatch([n], [S], table, page, pages)
    assert fq.fq_attn_paged_route(b, heads, kv)[:2] == route
    top = np.zeros(S)
    top[[100, 132, 164, 196]] = 1.0  # a wavefront of single tokens has 32 positions of every 128
    V = np.where(top[:, None] > 0, 0.0, rng.uniform(50.0, 150.0, size=(kv, S, 128))).astype(np.float16)
    height = (24 - np.log2(2.5)) * np.log(2.0)
    K = np.zeros((S, 128), dtype=np.float16)
    K[:, 0] = np.where(top > 0, height / 2, 0.0)
    K[[1, 33, 65, 97], 0] = (height - lag * np.log(2.0)) / 2
    V[:, [1, 33, 65, 97]] = 0.0
    k, v = (np.zeros((pages, kv, page, 128), dtype=np.float16) for _ in range(2))
    for t in range(S):
        k[table[0, t // page], :, t % page], v[table[0, t // page], :, t % page] = K[t], V[:, t]
    q = np.zeros((n, heads * 128), dtype=np.float16)
    q[:, ::128] = 2.0
    lse = torch.empty(n, heads, device="cuda")
    got = fq.fq_attn_paged(dev(torch, q), b, dev(torch, k), dev(torch, v), scale=1.0, lse=lse).cpu().numpy().astype(np.float64).reshape(n, kv, heads // kv, 128)
    w = np.exp(2.0 * K[:, 0].astype(np.float64))  # of every row that sees the position
    norm, rows = np.cumsum(w), np.arange(S - n, S)
    assert np.abs(lse.cpu().numpy() - np.log(norm[rows])[:, None]).max() <= 130 * 2.0 ** -24 * height + 2.0 ** -20 * (1 + np.log(norm[-1]))
    e = 130 * 2.0 ** -24 * height + 2.0 ** -20
    for g in range(kv):
        mass = np.cumsum(w[:, None] * V[g].astype(np.float64), 0)[rows] / norm[rows, None]
        count = np.cumsum(V[g].astype(np.float64), 0)[rows] * 2.0 ** -32
        bound = (2 * U * 1.01 + 2 * e) * mass + count + 2.0 ** -25
        err = np.abs(got[:, g] - mass[:, None])
        assert (err <= bound[:, None]).all(), float((err / bound[:, None]).max())


def test_rotation_between_the_rows_it_reads(fq, torch):
    """q_out right behind a row of keys and ahead of the next is no overlap; a place further on it is."""
    rng = np.random.default_rng(71)
    x = [dev(torch, rng.normal(size=(2, 256)).astype(np.float16)) for _ in range(3)]
    b = fq.PagedBatch([2], [20], [[0, 1]], 16, 2)
    rope = fq.rope_table(20)
    kp, vp, kp1, vp1 = (torch.zeros(2, 2, 16, 128, dtype=torch.float16, device="cuda") for _ in range(4))
    want = fq.fq_qk_norm_rope(*x, b, rope, kp, vp)
    room = torch.zeros(1024, dtype=torch.float16, device="cuda")
    k = room.as_strided((2, 256), (768, 1))
    k.copy_(x[1])
    got = fq.fq_qk_norm_rope(x[0], k, x[2], b, rope, kp1, vp1, out=room[256:768].view(2, 256))
    assert torch.equal(got, want) and torch.equal(kp1, kp) and torch.equal(vp1, vp) and torch.equal(k, x[1])
    for at in (248, 264):
        with pytest.raises(fq.FqError) as e:
            fq.fq_qk_norm_rope(x[0], k, x[2], b, rope, kp1, vp1, out=room[at:at + 512].view(2, 256))
        assert e.value.code == -2


def test_rows_too_far_apart_are_refused(fq, torch):
    """A distance of rows whose lower 32 bits look like a small one."""
    b = fq.PagedBatch([2], [2], [[0]], 16, 1)
    far = torch.zeros((1 << 32) + 512, dtype=torch.float16, device="cuda").as_strided((2, 256), ((1 << 32) + 256, 1))
    near, pool, rope = torch.zeros(2, 256, dtype=torch.float16, device="cuda"), torch.zeros(1, 2, 16, 128, dtype=torch.float16, device="cuda"), fq.rope_table(2)
    for out in (None, torch.zeros_like(near)):
        for call in (lambda: fq.fq_attn_paged(far, b, pool, pool, out=out), lambda: fq.fq_qk_norm_rope(far, near, near, b, rope, pool, pool, out=out),
                     lambda: fq.fq_qk_norm_rope(near, far, near, b, rope, pool, pool, out=out), lambda: fq.fq_qk_norm_rope(near, near, far, b, rope, pool, pool, out=out)):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("most, heads, kv, splits", [(1400, 8, 4, 3), (2500, 16, 4, 5), (9000, 4, 2, 18)])
def test_single_tokens_of_many_long_sequences(fq, torch, most, heads, kv, splits):
    """More sequences than a wavefront has lanes, more workgroups than are resident, several splits: workgroups find their sequence and split by
    the lengths.  Some sequences have no tokens, no positions, or two tokens."""
    rng = np.random.default_rng(most)
    lengths = np.exp(rng.uniform(0, np.log(most), 150)).astype(int)
    lengths[[3, 64, 127, 149]] = 0, most, most - 1, 1
    seqs = [(int(rng.choice((0, 1, 1, 1, 2))), int(S)) for S in lengths]
    seqs[64], seqs[3] = (1, most), (1, 0)
    table, pages = deal(np.random.default_rng(0), [S for _, S in seqs], 64)
    b = fq.PagedBatch([n for n, _ in seqs], [S for _, S in seqs], table, 64, pages)
    assert fq.fq_attn_paged_route(b, heads, kv)[:2] == (16, splits) and len(seqs) * kv * splits > 768
    run(fq, torch, rng, seqs, heads, kv, 64)


@pytest.mark.parametrize("n, S, heads, kv, splits", [(1, 9000, 4, 1, 71), (2, 40000, 8, 1, 313), (1, 70000, 2, 2, 137)])
def test_tokens_with_more_splits_than_lanes(fq, torch, n, S, heads, kv, splits):
    """Sixteen wavefronts join the splits of a row."""
    table, pages = deal(np.random.default_rng(0), [S], 256)
    assert fq.fq_attn_paged_route(fq.PagedBatch([n], [S], table, 256, pages), heads, kv)[:2] == (16, splits)
    run(fq, torch, np.random.default_rng(S), [(n, S)], heads, kv, 256)


def test_rotation_of_more_tokens_than_a_grid_has_rows(fq, torch):
    """Two launches: tokens from the 65536th on have their own positions and slots."""
    T, page = 65535 + 300, 256
    rng = np.random.default_rng(79)
    pages = -(-T // page)
    table = rng.permutation(pages)[None]
    b = fq.PagedBatch([T], [T], table, page, pages, positions=np.arange(T)[::-1] % 1000)
    x = rng.normal(size=(3, T, 128)).astype(np.float16)
    rope, gain = fq.rope_table(1000), (1 + 0.3 * rng.normal(size=(2, 128))).astype(np.float16)
    kp, vp = (torch.zeros(pages, 1, page, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    out = fq.fq_qk_norm_rope(*(dev(torch, t) for t in x), b, rope, kp, vp, *(dev(torch, g) for g in gain))
    at = torch.from_numpy(table[0]).cuda()
    rows_k, rows_v = (p[at].reshape(-1, 128)[:T].cpu().numpy() for p in (kp, vp))
    assert np.array_equal(rows_v, x[2])
    for got, t, g in ((out.cpu().numpy(), x[0], gain[0]), (rows_k, x[1], gain[1])):
        y = ref.norm_rope(t, b.positions.cpu().numpy(), rope.cpu().numpy(), g)
        size = ref.norm_rope(np.abs(t), b.positions.cpu().numpy(), np.abs(rope.cpu().numpy()) * [1, -1], np.abs(g))
        pair = np.maximum(size.reshape(T, -1, 2).max(-1), np.abs(y).reshape(T, -1, 2).max(-1))
        assert (np.abs(got - y) <= U * np.abs(y) + 2.0 ** -18 * 2 * np.repeat(pair, 2, axis=1) + 2.0 ** -24).all()


def test_handles_of_streams(fq, torch, monkeypatch):
    """What a call makes for a stream that is not the current one waits for the current one and is told to the allocator for that very stream, the
    default one (handle 0) among them."""
    side, device, waits, records = torch.cuda.Stream(), torch.device("cuda", torch.cuda.current_device()), [], []
    wait, record = torch.cuda.Stream.wait_stream, torch.Tensor.record_stream
    monkeypatch.setattr(torch.cuda.Stream, "wait_stream", lambda self, other: (waits.append((self.cuda_stream, other.cuda_stream)), wait(self, other))[1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: (records.append(s.cuda_stream), record(self, s))[1])
    with torch.cuda.stream(side):
        for handle in (0, torch.cuda.default_stream()):
            fq._fresh((8,), torch.float32, device, handle)
        for handle in (None, side, side.cuda_stream):
            fq._fresh((8,), torch.float32, device, handle)
    fq._fresh((8,), torch.float32, device, side.cuda_stream)
    fq._fresh((8,), torch.float32, device, 0)
    assert waits == [(0, side.cuda_stream)] * 2 + [(side.cuda_stream, 0)] and records == [0, 0, side.cuda_stream]
    rng = np.random.default_rng(83)
    table, pages, k, v, q = case(rng, [(1, 900)], 4, 1, 32)
    args = (dev(torch, q), fq.PagedBatch([1], [900], table, 32, pages), dev(torch, k), dev(torch, v))
    want = fq.fq_attn_paged(*args)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = fq.fq_attn_paged(*args, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
