"""Trees of tokens, host side: what the entry points refuse, reserved batches, and the reference itself (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2501_07139_amd as fq
from oracle import tree_ref as ref


def batch(**changes):
    b = fq.fq_paged_batch(q_start=0x100000, seq_len=0x110000, table=0x120000, seqs=2, tokens=5, max_q=3, max_len=100, table_stride=8, page=16, pages=40)
    for k, v in changes.items():
        setattr(b, k, v)
    return b


def plan(b, **c):
    a = dict(new=0x10000, cached=0x11000, next=None, parents=None, held=0x12000, held_out=0x12000, pages=0x13000, count=0x14000, count_out=0x14000,
             lacking=0x15000, positions=0x16000, slots=0x17000, mask=None, words=0)
    a.update(c)
    return fq._lib.fq_paged_plan(None if b is None else ctypes.byref(b), a["new"], a["cached"], a["next"], a["parents"], a["held"], a["held_out"],
                                 a["pages"], a["count"], a["count_out"], a["lacking"], a["positions"], a["slots"], a["mask"], a["words"], None)


@pytest.mark.parametrize("code, call, changes", [
    (-1, {}, None), (-1, {}, {"q_start": None}), (-1, {"new": None}, {}), (-1, {"cached": None}, {}), (-1, {"held": None}, {}), (-1, {"held_out": None}, {}),
    (-1, {"pages": None}, {}), (-1, {"count": None}, {}), (-1, {"count_out": None}, {}), (-1, {"lacking": None}, {}), (-1, {"positions": None}, {}),
    (-1, {"slots": None}, {}), (-1, {"mask": 0x20000, "words": 1}, {}), (-2, {"words": 1}, {}), (-2, {"parents": 0x18000, "mask": 0x20000}, {}),
    (-2, {"parents": 0x18000, "mask": 0x20000, "words": 65}, {}), (-2, {"parents": 0x18000, "mask": 0x20000, "words": 1}, {"tokens": 70, "max_q": 65}),
    (-2, {"parents": 0x18000}, {"tokens": 5000, "max_q": 4097}), (-2, {}, {"tokens": 1 << 28, "max_q": 1 << 27}), (-2, {}, {"max_q": 2}),
    (-2, {}, {"max_len": 129}), (-2, {}, {"page": 24}), (-2, {}, {"seqs": 0}), (-5, {"parents": 0x18000, "mask": 0x20004, "words": 1}, {}),
    (-2, {"next": 0x110000}, {}), (-2, {"new": 0x110004}, {}), (-2, {"cached": 0x110004}, {}), (-2, {"held_out": 0x12004}, {}), (-2, {"positions": 0x17000}, {}),
    (-2, {"lacking": 0x14000}, {}), (-2, {"positions": 0x100004}, {}), (-2, {"parents": 0x16000}, {}), (-2, {"slots": 0x120000 + 60}, {})], ids=str)
def test_plan_refuses(code, call, changes):
    assert plan(None if changes is None else batch(**changes), **call) == code
    assert "fq_paged_plan" in fq.fq_last_error()


def attn(b, **c):
    a = dict(mask=1 << 16, words=1, tail=None, q=16, ldq=256, heads=2, kv=2, k=16, v=16, scale=1.0, out=1 << 20, lse=None, ws=16, ws_bytes=1 << 30)
    a.update(c)
    return fq._lib.fq_attn_tree(None if b is None else ctypes.byref(b), a["mask"], a["words"], a["tail"], a["q"], a["ldq"], a["heads"], a["kv"], a["k"],
                                a["v"], a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("code, call, changes", [
    (-1, {}, None), (-1, {}, {"table": None}), (-1, {"mask": None}, {}), (-1, {"q": None}, {}), (-1, {"k": None}, {}), (-1, {"v": None}, {}), (-1, {"out": None}, {}),
    (-2, {"words": 0}, {}), (-2, {"words": 65}, {}), (-2, {"words": -1}, {}), (-2, {"heads": 3}, {}), (-2, {"kv": 0}, {}), (-2, {"ldq": 255}, {}),
    (-2, {"ldq": 260}, {}), (-2, {"scale": 0.0}, {}), (-2, {"scale": float("nan")}, {}), (-2, {}, {"max_q": 6}), (-2, {}, {"page": 8}),
    (-2, {"q": 4096, "out": 4096}, {}), (-2, {"q": 4096, "out": 4096 + 5 * 512 - 16}, {}), (-5, {"q": 8}, {}), (-5, {"k": 24}, {}), (-5, {"v": 24}, {}),
    (-5, {"out": 8}, {}), (-5, {"mask": 4}, {}), (-6, {"ws": None}, {"max_len": 4000, "table_stride": 250}),
    (-6, {"ws_bytes": 8}, {"max_len": 4000, "table_stride": 250})], ids=str)
def test_attention_refuses(code, call, changes):
    assert attn(None if changes is None else batch(**changes), **call) == code
    assert "fq_attn_tree" in fq.fq_last_error()


def test_no_tokens_are_nothing_to_do():
    assert attn(batch(tokens=0, max_q=0), q=None, out=None, mask=None) == 0


def commit(b, **c):
    a = dict(tail=None, parents=0x1000, drafted=0x2000, following=0x3000, k=1 << 24, v=1 << 28, layers=2, kv=2, path=0x10000, stride=5, accepted=0x11000,
             bonus=0x12000, new_len=0x13000)
    a.update(c)
    return fq._lib.fq_tree_commit(None if b is None else ctypes.byref(b), a["tail"], a["parents"], a["drafted"], a["following"], a["k"], a["v"],
                                  a["layers"], a["kv"], a["path"], a["stride"], a["accepted"], a["bonus"], a["new_len"], None)


PATH = {"parents": None, "drafted": None, "following": None, "bonus": None}


@pytest.mark.parametrize("code, call, changes", [
    (-1, {}, None), (-1, {}, {"seq_len": None}), (-1, {"k": None}, {}), (-1, {"v": None}, {}), (-1, {"path": None}, {}), (-1, {"accepted": None}, {}),
    (-1, {"new_len": None}, {}), (-1, {"parents": None}, {}), (-1, {"drafted": None}, {}), (-1, {"following": None}, {}), (-2, {"tail": 0x4000}, {}),
    (-2, dict(PATH, bonus=0x12000), {}), (-2, {"layers": 0}, {}), (-2, {"layers": 65536}, {}), (-2, {"layers": 60000, "kv": 1000}, {}), (-2, {"layers": 1 << 15, "kv": 256}, {}), (-2, {"kv": 0}, {}),
    (-2, {"stride": 0}, {}), (-2, {}, {"page": 24}), (-5, {"k": (1 << 24) + 8}, {}), (-5, {"v": (1 << 28) + 8}, {}), (-2, {"v": (1 << 24) + 4096}, {}),
    (-2, {"new_len": 0x110000}, {}), (-2, {"new_len": 0x11004}, {}), (-2, {"path": 0x1000 - 8}, {}), (-2, {"bonus": 0x3000}, {}),
    (-2, dict(PATH, tail=0x13004), {}), (-2, {"accepted": 0x120010}, {})], ids=str)
def test_commit_refuses(code, call, changes):
    assert commit(None if changes is None else batch(**changes), **call) == code
    assert "fq_tree_commit" in fq.fq_last_error()


def beam(**c):
    a = dict(logits=1 << 24, ld=1000, scores=0x1000, done=None, eos=-1, requests=3, beams=4, vocab=1000, width=5, parent=0x2000, token=0x3000, out=0x4000,
             done_out=None, mask=None, mask_out=None, words=0, tail=None, ws=1 << 30, bytes=1 << 28)
    a.update(c)
    return fq._lib.fq_beam_step(a["logits"], a["ld"], a["scores"], a["done"], a["eos"], a["requests"], a["beams"], a["vocab"], a["width"], a["parent"],
                                a["token"], a["out"], a["done_out"], a["mask"], a["mask_out"], a["words"], a["tail"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("code, call", [
    (-1, {"logits": None}), (-1, {"scores": None}), (-1, {"parent": None}), (-1, {"token": None}), (-1, {"out": None}), (-2, {"requests": 0}), (-2, {"beams": 0}),
    (-2, {"beams": 65}), (-2, {"width": 0}), (-2, {"width": 65}), (-2, {"vocab": 0}), (-2, {"vocab": (1 << 18) + 1, "ld": 1 << 19}),
    (-2, {"requests": 1 << 23}), (-2, {"requests": 1 << 19, "beams": 1, "vocab": 1 << 18, "ld": 1 << 18}), (-2, {"ld": 999}), (-2, {"ld": (1 << 32) + 1}), (-2, {"eos": 1000}), (-2, {"done": 0x5000}), (-2, {"mask": 0x6000}),
    (-2, {"words": 1}), (-2, {"mask_out": 0x7000}), (-2, {"mask_out": 0x7000, "words": 65}), (-6, {"ws": None}), (-6, {"bytes": 100}),
    (-5, {"ws": (1 << 30) + 8}), (-5, {"logits": (1 << 24) + 1}), (-5, {"mask_out": 0x7004, "words": 1}), (-2, {"parent": 0x3000}), (-2, {"out": 0x1000}),
    (-2, {"done": 0x2000, "eos": 3}), (-2, {"mask": 0x6000, "mask_out": 0x6010, "words": 1}), (-2, {"ws": (1 << 24) + 4096}), (-2, {"tail": 0x4000})], ids=str)
def test_beam_step_refuses(code, call):
    assert beam(**call) == code
    assert "fq_beam_step" in fq.fq_last_error()


def test_workspaces():
    assert fq.fq_beam_step_workspace_bytes(0, 1, 1, 1) == 0 and fq.fq_beam_step_workspace_bytes(1, 1, 1, 1) > 0
    most = fq.fq_beam_step_workspace_bytes(4, 64, 1 << 18, 64)
    assert 4 * 64 * 32 * (16 + 4 * 64) <= most < 1 << 28
    assert fq._lib.fq_attn_tree_workspace_bytes(None, 2, 2) == 0
    b = batch(max_len=4000, table_stride=250)
    assert fq._lib.fq_attn_tree_workspace_bytes(ctypes.byref(b), 2, 2) > 0
    # whatever the sizes: no more than 2^20 rows' parts, a split covers 128 positions at least
    for tokens, max_q, max_len, seqs in ((60000, 60000, 1 << 24, 1), (65535, 1, 1 << 24, 65535), (3, 3, 1 << 24, 1), (40, 20, 1, 2), (5000, 1000, 0, 300)):
        b = batch(tokens=tokens, max_q=max_q, seqs=seqs, max_len=max_len, table_stride=1 << 20)
        assert fq._lib.fq_attn_tree_workspace_bytes(ctypes.byref(b), 16, 2) <= (1 << 20) * 520 + 256 or max_q == 1


def test_reserved_batch():
    b = fq.PagedBatch.reserve(3, 9, 4, 100, 16, 20, mask_words=2, device="cpu")
    assert b.q_start.shape == (4,) and b.table.shape == (3, 7) and (b.table == -1).all() and b.mask.shape == (9, 2) and b.mask.dtype.is_signed
    assert b.free_pages.tolist() == list(range(19, -1, -1)) and b.free_count.tolist() == [20] and b.held.tolist() == [0, 0, 0]
    s = b.struct
    assert (s.seqs, s.tokens, s.max_q, s.max_len, s.table_stride, s.page, s.pages) == (3, 9, 4, 100, 7, 16, 20)
    assert fq.PagedBatch.reserve(1, 0, 0, 1, 16, 1, device="cpu").mask is None


@pytest.mark.parametrize("args, words", [((0, 1, 1, 10, 16, 4), 0), ((65536, 1, 1, 10, 16, 4), 0), ((2, 9, 4, 10, 16, 4), 0), ((2, 3, 4, 10, 16, 4), 0),
                                         ((2, 3, 2, 0, 16, 4), 0), ((2, 3, 2, (1 << 24) + 1, 16, 4), 0), ((2, 3, 2, 10, 24, 4), 0), ((2, 3, 2, 10, 16, 0), 0),
                                         ((2, 70, 65, 100, 16, 9), 1), ((2, 3, 2, 10, 16, 4), 65), ((2, 3, 2, 10, 16, 4), -1)], ids=str)
def test_reserve_refuses(args, words):
    with pytest.raises(fq.FqError) as e:
        fq.PagedBatch.reserve(*args, mask_words=words, device="cpu")
    assert e.value.code == -2


def test_python_wants_device_tensors():
    import torch

    b = fq.PagedBatch.reserve(2, 4, 2, 64, 16, 9, mask_words=1, device="cpu")
    two, pool = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 9, 2, 16, 128, dtype=torch.float16)
    with pytest.raises(TypeError):
        fq.fq_paged_plan(b, two, two)
    with pytest.raises(ValueError):
        fq.fq_paged_plan(fq.PagedBatch([1], [4], [[0]], 16, 4, device="cpu"), two, two)
    with pytest.raises(TypeError):
        fq.fq_attn_tree(torch.zeros(4, 256, dtype=torch.float16), b, b.mask, pool[0], pool[0])
    with pytest.raises(TypeError):
        fq.fq_tree_commit(b, pool, pool, two, two, two)
    with pytest.raises(TypeError):
        fq.fq_beam_step(torch.zeros(4, 10, dtype=torch.float16), torch.zeros(2, 2), 2)


# ------------------------------------------------------------------ the reference, on cases worked by hand
def test_reference_tree():
    #      0
    #    1   2
    #   3   4 5        6: a root of its own
    masks, depths = ref.tree_masks([-1, 0, 0, 1, 2, 2, 9])
    assert masks == [0b1, 0b11, 0b101, 0b1011, 0b10101, 0b100101, 0b1000000] and depths == [0, 1, 1, 2, 2, 2, 0]
    assert ref.words_of([1 << 63 | 1 << 64], 2).tolist() == [[-2 ** 63, 1]]
    # node 0 is followed by 7: drafted at 1 and 2, the first counts; node 1 by 8, drafted at 3 only under it
    assert ref.accept([-1, 0, 0, 1, 2, 2], [9, 7, 7, 8, 8, 8], [7, 8, 8, 5, 6, 6], 9) == ([0, 1, 3], 5)
    assert ref.accept([-1, 0], [9, 1], [2, 3], 9) == ([0], 2) and ref.accept([], [], [], 9) == ([], -1)
    assert ref.accept([-1, 0, 0, 1, 2, 2], [9, 7, 7, 8, 8, 8], [7, 8, 8, 5, 6, 6], 2) == ([0, 1], 8)


def test_reference_given_path():
    assert ref.given([1, 2, -1], 3, 5) == [1, 2, 2] and ref.given([7, 9], 2, 2) == [1, 1] and ref.given([3, 4], 9, 6) == [3, 4]
    assert ref.given([3, 4], -1, 6) == [] and ref.given([3, 4], 2, 1) == [0] and ref.given([], 2, 5) == [] and ref.given([4, 0, 2], 3, 6) == [4, 1, 2]


def test_reference_plan():
    table = np.array([[4, -1, -1], [0, 1, -1], [3, -1, -1]])
    # sequence 1 is closed and gives 0 and 1; sequence 0 grows by two pages, sequence 2 by none
    got = ref.plan([30, -1, 5], [10, 20, 3], None, None, [1, 2, 1], table, [6, 5], 16, 40, 40, 48)
    assert got["q_start"] == [0, 30, 30, 35] and got["seq_len"] == [40, 0, 8] and got["held"] == [3, 0, 1] and got["free"] == 2 and got["lacking"] == 0
    assert got["given"] == [6, 5, 0, 1] and got["table"].tolist() == [[4, 1, 0], [0, 1, -1], [3, -1, -1]]
    assert got["slots"][:7] == [74, 75, 76, 77, 78, 79, 16] and got["slots"][30:] == [51, 52, 53, 54, 55] + [-1] * 5
    short = ref.plan([40], [0], None, None, [0], np.full((1, 3), -1), [9], 16, 40, 40, 48)
    assert short["lacking"] == 2 and short["held"] == [1] and short["table"].tolist() == [[9, -1, -1]] and short["slots"][15:17] == [159, -1]


def test_reference_beam():
    logits = np.log(np.array([[1, 2, 1], [4, 4, 8]]) / 4.0)
    parent, token, score, done = ref.beam(logits, [0.0, np.log(0.25)], None, 2, 4)
    # totals: 1/4 1/2 1/4 of the first, 1/16 1/16 1/8 of the second: 1/2, then 1/4 twice by index, then 1/8
    assert (parent, token, done) == ([0, 0, 0, 1], [1, 0, 2, 2], [0, 0, 1, 1])
    assert np.allclose(score, np.log([0.5, 0.25, 0.25, 0.125]))
    assert ref.beam(logits, [-1.0, -2.0], [1, 1], 0, 3)[0] == [0, 1, -1]
