"""Serving of trees: the account of nodes and pages (CPU), drafted trees and beams against the same tokens one after the other (GPU)."""
import numpy as np
import pytest

from oracle import tree_ref as ref
from test_serve import build, close, gpu  # noqa: F401


def test_masks_as_words():
    from paper_2501_07139_amd.serve import _mask_words

    masks = [1, 1 << 63 | 1 << 64, (1 << 128) - 1]
    assert np.array_equal(_mask_words(masks, 2), ref.words_of(masks, 2))


def model(torch, rng, vocab, hidden):
    """Rows that tokens start from, and a head."""
    return (torch.from_numpy((rng.normal(size=(vocab, hidden))).astype(np.float16)).cuda() for _ in range(2))


@pytest.mark.gpu
@pytest.mark.parametrize("page", [16, 64])
def test_drafted_trees_are_checked_in_one_pass(gpu, page):  # noqa: F811
    """Tokens drafted right and wrong, several a step, two sequences, one of them with a chunk of its prompt beside the other's tree: the nodes on the
    right path give what the same tokens give one by one, and after they are kept the sequence goes on as that one does."""
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    rng = np.random.default_rng(page)
    stack, bitvec = build(fq, kv_heads=2)
    server, plain = (PagedServer(stack, slots=3, pages=40, page=page, max_positions=256) for _ in range(2))
    embed, head = model(torch, rng, 64, 512)
    truth = torch.from_numpy(rng.integers(0, 64, 120)).cuda()  # the sequence that will turn out to be right, and another
    prompt = 37
    s, p, other = server.open(), plain.open(), server.open()
    first = {s: embed[truth[:prompt]], other: embed[truth[50:80]]}
    close(torch, server.step(stack, bitvec, first)[s], plain.step(stack, bitvec, {p: embed[truth[:prompt]]})[p], 8e-3)
    at, held = prompt, server.pool.free
    for turn in range(5):
        # the right tokens in a chain of its own, wrong ones around it
        right = int(rng.integers(1, 7))
        parents, tokens, chain = [-1], [int(truth[at])], [0]
        for k in range(1, right):
            for _ in range(int(rng.integers(0, 3))):
                parents.append(int(rng.integers(0, len(parents))))
                tokens.append((int(truth[at + k]) + 1) % 64)
            parents.append(chain[-1])
            tokens.append(int(truth[at + k]))
            chain.append(len(parents) - 1)
        step = {s: embed[torch.tensor(tokens, device="cuda")]}
        if turn == 2:
            step[other] = embed[truth[80:100]]
        out = server.step(stack, bitvec, step, parents={s: parents})
        want = torch.cat([plain.step(stack, bitvec, {p: embed[truth[at + k]][None]})[p] for k in range(right)])
        close(torch, out[s][chain], want, 8e-3)
        # what the model says, made so that it agrees with the right tokens and with none of the wrong ones
        following = torch.full((len(parents),), 63, dtype=torch.int32, device="cuda")
        drafted = torch.tensor(tokens, dtype=torch.int32, device="cuda") + 64
        for a, b in zip(chain, chain[1:] + [None]):
            following[a] = 500 if b is None else drafted[b]
        wrong = [i for i in range(len(parents)) if i not in chain]
        drafted[wrong] += 1000
        assert server.length(s) == at
        assert server.accept({s: drafted}, {s: following}) == {s: (chain, 500)}
        at += right
        assert server.length(s) == at == plain.length(p)
        assert len(server.seqs[s].pages) == server.pool.need(at)
    kept, one = (x.k[0][torch.tensor(x.seqs[i].pages, device="cuda")].transpose(0, 1).reshape(2, -1, 128)[:, :at] for x, i in ((server, s), (plain, p)))
    close(torch, kept, one, 4e-3)
    assert server.length(other) == 50 and server.pool.free == 40 - server.pool.need(at) - server.pool.need(50)
    out = server.step(stack, bitvec, {s: embed[truth[at:at + 9]]})[s]  # a chunk again
    close(torch, out, plain.step(stack, bitvec, {p: embed[truth[at:at + 9]]})[p], 8e-3)


@pytest.mark.gpu
def test_beams_are_nodes_of_one_sequence(gpu):  # noqa: F811
    """Beam search over a prompt that is in the cache once: each beam's hidden states are those of its tokens as a sequence of their own, the search is that
    of the reference on the same logits, and the winner goes on as an ordinary sequence."""
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    rng = np.random.default_rng(5)
    stack, bitvec = build(fq, kv_heads=2, L=1)
    server, plain = (PagedServer(stack, slots=2, pages=30, page=16, max_positions=128) for _ in range(2))
    embed, head = model(torch, rng, 96, 512)
    beams, steps = 3, 7
    prompt = torch.from_numpy(rng.integers(0, 96, 21)).cuda()
    s = server.open()
    hidden = server.step(stack, bitvec, {s: embed[prompt]})[s][-1:]
    scores = torch.full((1, beams), -float("inf"), device="cuda")
    scores[0, 0] = 0.0
    hidden = hidden.expand(beams, -1).contiguous()
    mask = torch.zeros((1, beams, 1), dtype=torch.int64, device="cuda")
    nodes, texts = [-1] * beams, [[] for _ in range(beams)]
    for k in range(steps):
        logits = fq.fq_dense_f16(fq.fq_glue(0, hidden), (head * 0.05).contiguous())
        tail = torch.full((1,), beams * k, dtype=torch.int32, device="cuda")
        parent, token, new_scores, _, mask = fq.fq_beam_step(logits, scores, beams, mask=mask, tail=tail)
        want = ref.beam(logits.cpu().numpy(), scores[0].cpu().numpy(), None, -1, beams)
        assert parent[0].tolist() == want[0] and token[0].tolist() == want[1]
        scores = new_scores
        texts = [texts[q] + [t] for q, t in zip(want[0], want[1])]
        nodes, before = [beams * k + j for j in range(beams)], nodes
        hidden = server.step(stack, bitvec, {s: embed[token[0].long()]}, parents={s: [before[q] for q in want[0]]})[s]
        words = [m % 2 ** 64 for m in mask[0, :, 0].tolist()]
        assert server.seqs[s].masks[-beams:] == words  # the search's masks are the tree's
        for j in range(beams):
            p = plain.open()
            alone = plain.step(stack, bitvec, {p: embed[torch.cat((prompt, torch.tensor(texts[j], device="cuda")))]})[p]
            close(torch, hidden[j:j + 1], alone[-1:], 8e-3)
            plain.close(p)
    path = [n for n in range(beams * steps) if server.seqs[s].masks[nodes[0]] >> n & 1]
    server.keep_path({s: path})
    assert server.length(s) == 21 + steps and len(server.seqs[s].pages) == 2 and server.pool.free == 28
    p = plain.open()
    plain.step(stack, bitvec, {p: embed[torch.cat((prompt, torch.tensor(texts[0], device="cuda")))]})
    more = embed[torch.from_numpy(rng.integers(0, 96, 4)).cuda()]
    close(torch, server.step(stack, bitvec, {s: more})[s], plain.step(stack, bitvec, {p: more})[p], 8e-3)


@pytest.mark.gpu
def test_what_a_server_refuses_of_trees(gpu):  # noqa: F811
    fq, torch = gpu
    from paper_2501_07139_amd.serve import PagedServer

    stack, bitvec = build(fq, kv_heads=2, L=1)
    server = PagedServer(stack, slots=2, pages=6, page=16, max_positions=40)
    s = server.open()
    x = torch.randn(9, 512, device="cuda").half()
    for parents in ({s: [0]}, {s: [-1, 1]}, {s: [-1, -2]}, {1 - s: [-1, 0]}, {s: [-1, 0, 1]}):
        with pytest.raises(ValueError):
            server.step(stack, bitvec, {s: x[:2]}, parents=parents)
    assert server.pool.free == 6 and server.length(s) == 0
    server.step(stack, bitvec, {s: x[:5]}, parents={s: [-1, 0, 0, 1, 2]})
    with pytest.raises(ValueError):  # nodes first
        server.step(stack, bitvec, {s: x[:1]})
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        server.accept({s: ints(1, 2)}, {s: ints(1, 2)})
    with pytest.raises(ValueError):
        server.accept({s: ints(1, 2, 3, 4, 5)}, {})
    for path in ([1], [0, 3], [0, 1, 4], [0, 9], [-1]):
        with pytest.raises(ValueError):
            server.keep_path({s: path})
    with pytest.raises(fq.FqError):  # deeper than there are positions
        server.step(stack, bitvec, {s: torch.randn(40, 512, device="cuda").half()}, parents={s: [4] + list(range(5, 44))})
    with pytest.raises(MemoryError):
        server.step(stack, bitvec, {s: torch.randn(95, 512, device="cuda").half()}, parents={s: [0] * 95})
    assert server.seqs[s].tail == 5 and server.length(s) == 0
    server.keep_path({s: [0, 2, 4]})
    assert server.length(s) == 3 and server.accept({}, {}) == {} and server.keep_path({}) is None
    assert server.accept({s: ints()}, {s: ints()}) == {s: ([], -1)} and server.length(s) == 3  # no nodes, nothing to keep
    server.step(stack, bitvec, {s: x[:3]}, parents={s: [-1, 0, -1]})
    server.keep_path({s: []})
    assert server.length(s) == 3 and server.seqs[s].tail == 0
    cutting = PagedServer(stack, slots=1, pages=6, page=16, max_positions=40, keep=8, limit=20)
    with pytest.raises(ValueError):
        cutting.step(stack, bitvec, {cutting.open(): x[:1]}, parents={0: [-1]})
