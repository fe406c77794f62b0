"""Serving over a paged cache: the account of pages (CPU), and the blocks against the contiguous path and plain attention (GPU)."""
import numpy as np
import pytest

import fq_synth
import oracle


def test_page_pool():
    from paper_2501_07139_amd.serve import PagePool

    p = PagePool(5, 16)
    assert (p.free, p.need(0), p.need(1), p.need(16), p.need(17)) == (5, 0, 1, 1, 2)
    a, b = p.take(2), p.take(3)
    assert a == [0, 1] and b == [2, 3, 4] and p.free == 0
    with pytest.raises(MemoryError):
        p.take(1)
    p.give(a)
    assert p.free == 2 and p.take(2) == [0, 1] and p.take(0) == []


@pytest.fixture(scope="module")
def gpu():
    import torch

    import paper_2501_07139_amd as fq

    fq.fq_init()
    return fq, torch


def build(fq, kv_heads, L=2, heads=4, ffn=640, seed=3):
    """Blocks with 128 rows a head, every matrix at 4 bits and at 8."""
    H = 128 * heads
    shapes = [(H, H), (128 * kv_heads, H), (128 * kv_heads, H), (H, H), (ffn, H), (ffn, H), (H, ffn)]
    layers = []
    for l in range(L):
        mats = []
        for j, (N, K) in enumerate(shapes):
            W = fq_synth.weights(seed + 16 * l + j, N, K)
            by = {}
            for bits in (4, 8):
                codes, s, z = oracle.quantize_rtn(W, bits)
                by[bits] = fq.PackedMatrix.from_host(codes, s, z, bits)
            mats.append(by)
        layers.append(mats)
    return fq.Stack(layers), np.array([4, 8, 4, 8, 4, 4, 8] * L, dtype=np.uint8)


def close(torch, got, want, bound):
    got, want = got.double(), want.double()
    rms = want.pow(2).mean(-1, keepdim=True).sqrt()
    assert float(((got - want).abs() / torch.maximum(want.abs(), rms)).max()) <= bound


@pytest.mark.gpu
def test_steps_agree_with_the_contiguous_path(gpu):
    """Prompts in chunks and token by token, two sequences at once, against one prefill of each sequence."""
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    stack, bitvec = build(fq, kv_heads=4)
    server = PagedServer(stack, slots=3, pages=40, page=16, max_positions=256)
    a, b = server.open(), server.open()
    xs = {a: torch.randn(90, 512, device="cuda").half(), b: torch.randn(61, 512, device="cuda").half()}
    got = {a: [], b: []}
    at = {a: 0, b: 0}
    for na, nb in ((50, 0), (1, 33), (20, 1), (1, 1), (17, 25), (1, 0), (0, 1)):
        tokens = {i: xs[i][at[i]:at[i] + n] for i, n in ((a, na), (b, nb)) if n}
        out = server.step(stack, bitvec, tokens)
        for i in tokens:
            got[i].append(out[i])
            at[i] += len(tokens[i])
    assert at == {a: 90, b: 61} and server.length(a) == 90 and server.pool.free == 40 - 6 - 4
    rope = fq.rope_table(256)
    for i in (a, b):
        T = len(xs[i])
        kc, vc = (torch.zeros(2, 4, 256, 128, dtype=torch.float16, device="cuda") for _ in range(2))
        want = fq.fq_prefill_forward(stack, bitvec, xs[i], kc, vc, rope)
        # both ways round every named tensor to fp16; two blocks of the same weights differ by what the linears' and the attention's
        # bounds (2e-3 of a row each) add up to
        close(torch, torch.cat(got[i]), want, 8e-3)
        pages = torch.tensor(server.seqs[i].pages, device="cuda")
        rows = server.v[0][pages].transpose(0, 1).reshape(4, -1, 128)[:, :T]
        close(torch, rows, vc[0][:, :T], 4e-3)
    server.close(a)
    assert server.pool.free == 36 and server.open() == a


@pytest.mark.gpu
def test_a_cut_sequence_goes_on(gpu):
    """After a cut, a token attends to what was kept, with its true position; norms of the heads, shared key/value heads."""
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    stack, bitvec = build(fq, kv_heads=2, L=1)
    gains = [tuple((1 + 0.2 * torch.randn(128, device="cuda")).half() for _ in range(2))]
    server = PagedServer(stack, slots=2, pages=24, page=16, max_positions=128, gains=gains, keep=40, recent=12, limit=64)
    s, other = server.open(), server.open()
    free = server.pool.free
    xs = torch.randn(70, 512, device="cuda").half()
    server.step(stack, bitvec, {s: xs[:60], other: xs[:5]})
    assert server.length(s) == 60
    server.step(stack, bitvec, {s: xs[60:69]})  # 69 positions: cut to 40
    assert server.length(s) == 40 and server.seqs[s].position == 69 and server.pool.free == free - 3 - 1
    assert server.cache_bytes() == 4 * 16 * 2 * 128 * 2 * 2
    pages = torch.tensor(server.seqs[s].pages, device="cuda")
    K, V = (t[0][pages].transpose(0, 1).reshape(2, -1, 128)[:, :40].double() for t in (server.k, server.v))
    got = server.step(stack, bitvec, {s: xs[69:]})[s]
    # the same block in plain attention over the kept rows
    w = [stack.layers[0][j][int(bitvec[j])] for j in range(7)]
    u = fq.fq_glue(0, xs[69:])
    q, k, v = (fq.fq_qlinear(u, w[j]).double().view(-1, 128) for j in range(3))
    rope = server.rope[69].double()

    def turn(x, gain):
        x = x / (x.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * gain.double()
        y = torch.empty_like(x)
        y[:, 0::2] = x[:, 0::2] * rope[:, 0] - x[:, 1::2] * rope[:, 1]
        y[:, 1::2] = x[:, 0::2] * rope[:, 1] + x[:, 1::2] * rope[:, 0]
        return y.half().double()

    q, k = turn(q, gains[0][0]), turn(k, gains[0][1])
    K, V = torch.cat((K, k[:, None]), 1), torch.cat((V, v[:, None]), 1)
    a = torch.cat([torch.softmax(K[h // 2] @ q[h] / 128 ** 0.5, 0) @ V[h // 2] for h in range(4)])[None].half()
    x1 = fq.fq_glue(2, xs[69:], fq.fq_qlinear(a, w[3]))
    u = fq.fq_glue(0, x1)
    m = fq.fq_glue(5, fq.fq_qlinear(u, w[4]), fq.fq_qlinear(u, w[5]))
    close(torch, got, fq.fq_glue(2, x1, fq.fq_qlinear(m, w[6])), 4e-3)
    # weights of what was kept moved with it, and the last positions are the ones before the cut
    assert bool((server.weights[0, s, :, 41:] == 0).all()) and bool((server.weights[0, s, :, :41] > 0).all())


@pytest.mark.gpu
def test_what_does_not_fit_is_refused_and_changes_nothing(gpu):
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    stack, bitvec = build(fq, kv_heads=4, L=1)
    server = PagedServer(stack, slots=1, pages=2, page=16, max_positions=64)
    s = server.open()
    with pytest.raises(MemoryError):
        server.open()
    x = torch.randn(33, 512, device="cuda").half()
    with pytest.raises(MemoryError):
        server.step(stack, bitvec, {s: x})
    assert server.length(s) == 0 and server.pool.free == 2
    server.step(stack, bitvec, {s: x[:32]})
    assert server.step(stack, bitvec, {}) == {}
    with pytest.raises(ValueError):
        server.step(stack, bitvec, {s: x[:0]})
    server.seqs[s].position = 40
    with pytest.raises(fq.FqError):
        server.step(stack, bitvec, {s: x[:30]})  # past the last position of the table
    with pytest.raises(ValueError):
        PagedServer(stack, 1, 8, keep=4, recent=5)



@pytest.mark.gpu
def test_cuts_wait_for_room(gpu):
    """Pages for the rows that stay are taken before the old ones are free: one sequence after the other, or at a later step."""
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    stack, bitvec = build(fq, kv_heads=4, L=1)
    server = PagedServer(stack, slots=3, pages=9, page=16, max_positions=128, keep=30, recent=30, limit=32)
    a, b, c = server.open(), server.open(), server.open()
    x = torch.randn(64, 512, device="cuda").half()
    server.step(stack, bitvec, {a: x[:40], b: x[:40]})  # three pages each, two for what stays: not both at once
    assert [server.length(i) for i in (a, b)] == [30, 30] and server.pool.free == 9 - 4
    rows = [server.v[0][torch.tensor(server.seqs[i].pages, device="cuda")].transpose(0, 1).reshape(4, -1, 128)[:, :30] for i in (a, b)]
    assert torch.equal(*rows)
    server.step(stack, bitvec, {c: x[:64]})  # four pages, one left: stays as it is
    assert server.length(c) == 64 and server.pool.free == 1
    server.close(a)
    server.step(stack, bitvec, {b: x[:1]})
    assert server.length(c) == 30 and server.length(b) == 31 and server.pool.free == 9 - 4
