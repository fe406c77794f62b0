"""Paged cache, host side: the batch that Python lays out, and what the entry points refuse (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2501_07139_amd as fq
from oracle import paged_ref


def batch(**changes):
    b = fq.fq_paged_batch(q_start=16, seq_len=16, table=16, seqs=2, tokens=5, max_q=3, max_len=100, table_stride=8, page=16, pages=40)
    for k, v in changes.items():
        setattr(b, k, v)
    return b


def test_batch_lays_out_lengths_positions_and_slots():
    table = [[5, 2, -1], [1, 7, 3], [0, 0, 0], [4, -7, 99]]
    b = fq.PagedBatch([1, 4, 0, 3], [17, 35, 0, 2], table, 16, 8, device="cpu")
    assert (b.seqs, b.tokens, b.max_q, b.max_len) == (4, 8, 4, 35)
    assert b.q_start.tolist() == [0, 1, 5, 5, 8] and b.seq_len.tolist() == [17, 35, 0, 2]
    assert b.table.tolist() == [[5, 2, -1], [1, 7, 3], [-1, -1, -1], [4, -1, -1]]
    assert b.positions.tolist() == [16, 31, 32, 33, 34, 0, 0, 1]
    # the last sequence has three tokens and two positions: its first token is in no slot
    assert b.slots.tolist() == [32, 7 * 16 + 15, 48, 49, 50, -1, 64, 65]
    assert all(t.data_ptr() % 16 == 0 for t in (b.q_start, b.seq_len, b.table, b.positions, b.slots))
    s = b.struct
    assert (s.seqs, s.tokens, s.max_q, s.max_len, s.table_stride, s.page, s.pages) == (4, 8, 4, 35, 3, 16, 8)
    assert s.table == b.table.data_ptr() and s.q_start == b.q_start.data_ptr() and s.seq_len == b.seq_len.data_ptr()
    given = fq.PagedBatch([2], [2], [[0]], 16, 1, positions=[70, 71], device="cpu")
    assert given.positions.tolist() == [70, 71] and given.slots.tolist() == [0, 1]
    none = fq.PagedBatch([0], [20], [[1, 0]], 16, 2, device="cpu")
    assert none.tokens == 0 and none.max_q == 0 and none.slots.numel() == 0


@pytest.mark.parametrize("args", [([1], [17], [[0]], 16, 4), ([1], [4], [[4]], 16, 4), ([1], [4], [[-1]], 16, 4), ([-1], [4], [[0]], 16, 4),
                                  ([1], [-4], [[0]], 16, 4), ([1], [4], [[0]], 24, 4), ([1], [4], [[0]], 16, 0), ([1, 1], [4], [[0]], 16, 4),
                                  ([1], [4], [[0], [1]], 16, 4), ([], [], [[0]], 16, 4), ([1], [4], [[0]], 256, 1 << 23)], ids=str)
def test_batch_refuses(args):
    with pytest.raises(fq.FqError) as e:
        fq.PagedBatch(*args, device="cpu")
    assert e.value.code == -2


def test_batch_refuses_positions_of_another_length():
    with pytest.raises(fq.FqError):
        fq.PagedBatch([2], [4], [[0]], 16, 4, positions=[1], device="cpu")


def attn(lib, b, **c):
    a = dict(q=16, ldq=256, heads=2, kv=2, k=16, v=16, scale=1.0, out=1 << 20, lse=None, weights=None, weights_out=None, stride=0,
             ws=16, ws_bytes=1 << 30)
    a.update(c)
    return lib.fq_attn_paged(None if b is None else ctypes.byref(b), a["q"], a["ldq"], a["heads"], a["kv"], a["k"], a["v"], a["scale"], a["out"],
                             a["lse"], a["weights"], a["weights_out"], a["stride"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("code, call, changes", [
    (-1, {}, None), (-1, {}, {"q_start": None}), (-1, {}, {"seq_len": None}), (-1, {}, {"table": None}), (-1, {"q": None}, {}), (-1, {"k": None}, {}),
    (-1, {"v": None}, {}), (-1, {"out": None}, {}), (-1, {"weights": 16}, {}), (-2, {"heads": 3}, {}), (-2, {"heads": 0}, {}), (-2, {"kv": 0}, {}),
    (-2, {"ldq": 255}, {}), (-2, {"ldq": 260}, {}), (-2, {"scale": 0.0}, {}), (-2, {"scale": -1.0}, {}), (-2, {"scale": float("nan")}, {}),
    (-2, {"scale": float("inf")}, {}), (-2, {"weights_out": 16, "stride": 99}, {}), (-2, {}, {"seqs": 0}), (-2, {}, {"seqs": 65536}),
    (-2, {}, {"tokens": -1}), (-2, {}, {"max_q": 6}), (-2, {}, {"max_q": 2}), (-2, {}, {"max_len": 129}), (-2, {}, {"max_len": -1}), (-2, {}, {"max_len": (1 << 24) + 1, "table_stride": 1 << 21}),
    (-2, {}, {"table_stride": 0}), (-2, {}, {"page": 8}), (-2, {}, {"page": 48}), (-2, {}, {"page": 512}), (-2, {}, {"pages": 0}),
    (-2, {}, {"pages": 1 << 27, "page": 16}), (-2, {"heads": 1 << 25, "kv": 1}, {"tokens": 3}), (-2, {"kv": 1024, "heads": 1024}, {"seqs": 8192}),
    (-2, {"kv": 64, "heads": 64, "ldq": 8192, "out": 1 << 30, "weights_out": 16, "stride": 1 << 22}, {"max_len": 1 << 22, "table_stride": 1 << 18}),
    (-2, {"q": 4096, "out": 4096}, {}), (-2, {"q": 4096, "out": 4096 + 5 * 512 - 16}, {}), (-2, {"q": 4096, "out": 4096 - 5 * 512 + 16}, {}),
    (-2, {"q": 4096, "ldq": 1024, "out": 4096 + 8192}, {}), (-5, {"q": 8}, {}), (-5, {"k": 24}, {}),
    (-5, {"v": 24}, {}), (-5, {"out": 8}, {}), (-6, {"ws": None, "weights_out": 16, "stride": 100}, {}),
    (-6, {"ws_bytes": 8, "weights_out": 16, "stride": 100}, {})], ids=str)
def test_attention_refuses(code, call, changes):
    b = None if changes is None else batch(**changes)
    assert attn(fq._lib, b, **call) == code
    assert "fq_attn_paged" in fq.fq_last_error()


def test_workspace_of_bad_arguments_is_none():
    lib = fq._lib
    assert lib.fq_attn_paged_workspace_bytes(None, 2, 2, 0) == 0
    assert lib.fq_attn_paged_workspace_bytes(ctypes.byref(batch(page=5)), 2, 2, 0) == 0
    assert lib.fq_attn_paged_workspace_bytes(ctypes.byref(batch()), 3, 2, 0) == 0
    assert lib.fq_attn_paged_workspace_bytes(ctypes.byref(batch()), 2, 2, 1) >= 5 * 2 * 4


def test_division_of_calls():
    """One split where that is no longer, splits that cover the positions, 128-row tiles for the largest calls only."""
    one = lambda q, S, seqs=1: fq.PagedBatch([q] * seqs, [S] * seqs, np.zeros((seqs, S // 16 + 1), dtype=np.int64), 16, 4, device="cpu")
    assert fq.fq_attn_paged_route(one(1, 300), 32, 32) == (16, 1, 384)
    assert fq.fq_attn_paged_route(one(1, 1000, 64), 32, 8)[:2] == (16, 1)
    assert fq.fq_attn_paged_route(one(1, 1000), 32, 8) == (16, 8, 128)
    assert fq.fq_attn_paged_route(one(1, 100000), 32, 8) == (16, 196, 512)
    assert fq.fq_attn_paged_route(one(16, 16000), 32, 8)[0] == 64 and fq.fq_attn_paged_route(one(2048, 2048), 32, 32)[:2] == (128, 1)
    rng = np.random.default_rng(0)
    for _ in range(3000):
        kv, group, n, S = (int(2 ** rng.uniform(0, t)) for t in (5, 5, 12, 17))
        rows, splits, chunk = fq.fq_attn_paged_route(one(n, S), kv * group, kv)
        assert (rows == 16) == (n * group <= 16) and chunk % 128 == 0 and (splits - 1) * chunk < S <= splits * chunk, (kv, group, n, S)
    lib, out = fq._lib, np.zeros(3, dtype=np.int32)
    assert lib.fq_attn_paged_route(ctypes.byref(batch()), 2, 2, None) == -1
    assert lib.fq_attn_paged_route(ctypes.byref(batch(page=5)), 2, 2, out.ctypes.data_as(ctypes.c_void_p)) == -2


def rope(lib, **c):
    a = dict(q=16, ldq=256, k=16, ldk=256, v=16, ldv=256, tokens=3, heads=2, kv=2, positions=16, slots=16, rope=16, rows=9, qg=None, kg=None,
             eps=1e-5, out=1 << 20, kp=16, vp=16, page=16, pages=4)
    a.update(c)
    return lib.fq_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("code, call", [(-1, {n: None}) for n in ("q", "k", "v", "positions", "slots", "rope", "out", "kp", "vp")] + [
    (-2, {"tokens": -1}), (-2, {"heads": 3}), (-2, {"heads": 0}), (-2, {"kv": 0}), (-2, {"rows": 0}), (-2, {"eps": -1.0}),
    (-2, {"eps": float("nan")}), (-2, {"ldq": 255}), (-2, {"ldk": 252}), (-2, {"ldv": 260}), (-2, {"page": 20}), (-2, {"pages": 0}),
    (-2, {"out": 16, "ldq": 512}), (-2, {"out": 32}), (-2, {"q": 4096, "out": 4096 + 512}), (-2, {"q": 4096, "out": 4096 - 512}), (-5, {"q": 8}), (-5, {"k": 8}), (-5, {"v": 8}), (-5, {"rope": 8}), (-5, {"qg": 8}), (-5, {"kg": 8}),
    (-5, {"out": 40}), (-5, {"kp": 8}), (-5, {"vp": 8})], ids=str)
def test_norm_rope_refuses(code, call):
    assert rope(fq._lib, **call) == code
    assert "fq_qk_norm_rope" in fq.fq_last_error()


def test_norm_rope_of_no_tokens_does_nothing():
    assert rope(fq._lib, tokens=0) == 0


def evict(lib, b, **c):
    a = dict(k=16, v=16, kv=2, w=16, ws=100, keep=40, recent=8, dst=16, ds=3, dp=9, ko=16, vo=16, kept=16, new=16, wo=None, wos=0)
    a.update(c)
    return lib.fq_cache_evict(None if b is None else ctypes.byref(b), *a.values(), None)


@pytest.mark.parametrize("code, call, changes", [(-1, {n: None}, {}) for n in ("k", "v", "w", "dst", "ko", "vo", "kept", "new")] + [
    (-1, {}, None), (-2, {"kv": 0}, {}), (-2, {"ws": 99}, {}), (-2, {"keep": 0}, {}), (-2, {"recent": -1}, {}), (-2, {"recent": 41}, {}),
    (-2, {"ds": 2}, {}), (-2, {"ds": 0}, {}), (-2, {"dp": 0}, {}), (-2, {"wo": 32, "wos": 39}, {}), (-2, {"wo": 16, "wos": 100}, {}),
    (-2, {}, {"page": 17}), (-2, {}, {"max_len": 500}), (-5, {"k": 8}, {}), (-5, {"v": 8}, {}), (-5, {"ko": 8}, {}), (-5, {"vo": 8}, {})], ids=str)
def test_evict_refuses(code, call, changes):
    assert evict(fq._lib, None if changes is None else batch(**changes), **call) == code
    assert "fq_cache_evict" in fq.fq_last_error()


def test_device_calls_refuse_host_tensors():
    import torch

    b = fq.PagedBatch([1], [4], [[0]], 16, 1, device="cpu")
    x, pool = torch.zeros(1, 256, dtype=torch.float16), torch.zeros(1, 2, 16, 128, dtype=torch.float16)
    for call in (lambda: fq.fq_attn_paged(x, b, pool, pool), lambda: fq.fq_qk_norm_rope(x, x, x, b, x, pool, pool),
                 lambda: fq.fq_cache_evict(b, x, pool, pool, x, 4, 2)):
        with pytest.raises(TypeError):
            call()


def test_reference_attention_of_equal_keys_is_the_mean():
    V = np.arange(2 * 5 * 128, dtype=np.float64).reshape(2, 5, 128)
    out, lse, sums, mass, _ = paged_ref.attention(np.ones((3, 4 * 128)), np.zeros((2, 5, 128)), V, 3, 0.5)
    for i, seen in enumerate((3, 4, 5)):
        assert np.allclose(out[i].reshape(4, 128), np.repeat(V[:, :seen].mean(1), 2, axis=0)) and np.allclose(lse[i], np.log(seen))
    assert np.allclose(sums.sum(1), 6) and np.allclose(sums[:, 4], 2 / 5) and np.allclose(mass, out)
    # more tokens than positions: the first ones see nothing
    out, lse, sums, _, _ = paged_ref.attention(np.ones((3, 256)), np.zeros((2, 1, 128)), V[:, :1], 3, 1.0)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(lse[2], 0) and np.allclose(sums, 1)


def test_reference_eviction():
    w = np.array([3.0, 1.0, 3.0, np.nan, 0.0, 2.0, 9.0])
    assert paged_ref.evict(w, 4, 2).tolist() == [0, 3, 5, 6]
    assert paged_ref.evict(w, 5, 2).tolist() == [0, 2, 3, 5, 6]
    assert paged_ref.evict(w, 9, 2).tolist() == list(range(7))
    assert paged_ref.evict(w, 3, 3).tolist() == [4, 5, 6]
    assert paged_ref.evict(w, 2, 0).tolist() == [3, 6]
    assert paged_ref.evict(w[:0], 2, 0).tolist() == []


@pytest.mark.parametrize("call, changes", [({"new": 4096 + 4}, {"seq_len": 4096}), ({"new": 4096 - 4}, {"seq_len": 4096}),
                                           ({"w": 4096, "wo": 4096 + 400 * 4 - 4, "wos": 40}, {}), ({"w": 4096, "wo": 4096 - 160 * 4 + 4, "wos": 40}, {})], ids=str)
def test_evict_refuses_outputs_over_what_it_reads(call, changes):
    """Two sequences of two heads: lengths of 8 bytes, weights of 3 * 100 + 100 floats, written ones of 3 * 40 + 40."""
    assert evict(fq._lib, batch(**changes), **{"new": 1 << 20, "kept": 1 << 21, **call}) == -2
    assert "must not be" in fq.fq_last_error()


def test_division_of_sequences_of_other_lengths():
    """Positions and pairs are those of the sequences with tokens; a chunk beside one long sequence is split, and known lengths do not change one sequence's call."""
    b = fq.PagedBatch([1, 4, 0, 3], [17, 35, 400, 2], np.zeros((4, 25), dtype=np.int64), 16, 8, device="cpu")
    assert b.struct.positions == 17 + 35 + 2 and b.struct.pairs == 16 + 31 * 4 + 8 + 2
    lone = fq.PagedBatch([300] + [1] * 20, [300] + [200] * 19 + [30000], np.zeros((21, 1876), dtype=np.int64), 16, 8, device="cpu")
    rows, splits, chunk = fq.fq_attn_paged_route(lone, 32, 8)
    assert splits > 4 and (splits - 1) * chunk < 30000 <= splits * chunk
    most = fq.fq_attn_paged_workspace_bytes(lone, 32, 8)
    assert 0 < most < 1 << 30
    lone.struct.positions = lone.struct.pairs = 0
    assert fq.fq_attn_paged_route(lone, 32, 8)[0] == rows
    one = fq.PagedBatch([300], [5000], np.zeros((1, 313), dtype=np.int64), 16, 8, device="cpu")
    with_lengths = fq.fq_attn_paged_route(one, 32, 8)
    one.struct.positions = one.struct.pairs = 0
    assert fq.fq_attn_paged_route(one, 32, 8) == with_lengths


@pytest.mark.parametrize("weights, out, stride", [(4096, 4096 + 4, 100), (4096, 4096 + 400 * 4 - 4, 100), (4096 + 400 * 4 - 4, 4096, 100), (4096, 4096 - 120 * 4, 100),
                                                  (4096, 4096 + 404, 200), (4096, 4096 + 396, 200), (4096 + 2 * 800 + 404, 4096, 200)])
def test_attention_refuses_weights_over_part_of_what_it_adds_to(weights, out, stride):
    """Two sequences of two heads: 3 * 100 + 100 floats each; sums that one workgroup writes are read by another."""
    assert attn(fq._lib, batch(), weights=weights, weights_out=out, stride=stride) == -2
    assert "weights_out overlaps weights" in fq.fq_last_error()
    for apart, stride in ((4096 + 400 * 4, 100), (4096, 100), (4096 + 400, 200), (4096 - 400 - 800, 200), (4096 - 400 * 4, 100)):
        # side by side, the same, or row between row: the next check's refusal
        assert attn(fq._lib, batch(), weights=4096, weights_out=apart, stride=stride, ws=None) == -6
    assert attn(fq._lib, batch(max_len=0), weights=4096, weights_out=4100, stride=0, ws=None) == -6  # rows of nothing


@pytest.mark.parametrize("call", [{"k": 1 << 20}, {"v": 1 << 20}, {"k": (1 << 20) + 1536 - 16}, {"v": (1 << 20) - 1536 + 16}, {"k": (1 << 20) - 8192, "ldk": 4096 + 128},
                                  {"v": (1 << 20) - 8192 - 512, "ldv": 4096 + 256}], ids=str)
def test_norm_rope_refuses_q_out_over_keys_or_values(call):
    """Three tokens of two heads, rows of 512 bytes: one workgroup would write what another reads."""
    assert rope(fq._lib, **call) == -2
    assert "q_out overlaps k or v" in fq.fq_last_error()


def test_batch_keeps_positions_on_their_side():
    """Positions that int32 does not hold stay beyond the table's end, or ahead of its start."""
    b = fq.PagedBatch([4], [4], [[0]], 16, 4, positions=[2 ** 31 + 5, -2 ** 31 - 5, 2 ** 32, 7], device="cpu")
    assert b.positions.tolist() == [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 7]


def test_splits_of_single_tokens_are_within_a_wavefront_of_pages():
    """At most 1024 positions, 64 blocks of sixteen: a lane holds the page of one, and nothing asks for more on the way."""
    rng = np.random.default_rng(1)
    for _ in range(3000):
        kv, group, seqs, S = (int(2 ** rng.uniform(0, t)) for t in (6, 4, 8, 20))
        n = int(rng.integers(1, max(16 // group, 1) + 1))
        b = batch(seqs=seqs, tokens=seqs * n, max_q=n, max_len=S, table_stride=(S + 15) // 16)
        if n * seqs * kv * group >= 1 << 26:
            continue
        out = np.zeros(3, dtype=np.int32)
        assert fq._lib.fq_attn_paged_route(ctypes.byref(b), kv * group, kv, out.ctypes.data_as(ctypes.c_void_p)) == 0
        assert out[0] == 16 and 128 <= out[2] <= 1024 and (out[1] - 1) * out[2] < S <= out[1] * out[2], (kv, group, seqs, n, S)


@pytest.mark.parametrize("q_lens, seq_lens, heads, kv", [
    ([202, 52], [472, 988], 28, 4), ([14, 2, 6], [2765, 148, 7], 40, 8),
    ([34, 167, 212, 48, 91, 100, 49, 127], [53, 203, 214, 49, 114, 101, 104, 1707], 28, 4), ([40] * 4, [16000, 15963, 15926, 15889], 32, 8),
    ([40] * 4, [16000, 15963, 15926, 15889], 32, 32), ([67] * 3, [2000, 1963, 1926], 32, 8)], ids=str)
def test_known_lengths_change_the_division_for_a_real_gain_only(q_lens, seq_lens, heads, kv):
    """Calls that took 1 to 24 % longer in the splits that known lengths gave them for a gain within the estimate's error."""
    b = fq.PagedBatch(q_lens, seq_lens, np.zeros((len(q_lens), max(seq_lens) // 64 + 1), dtype=np.int64), 64, 4, device="cpu")
    known = fq.fq_attn_paged_route(b, heads, kv)
    b.struct.positions = b.struct.pairs = 0
    assert fq.fq_attn_paged_route(b, heads, kv) == known


def test_known_lengths_change_the_division_where_it_pays():
    """One long sequence among short ones: 528 us in one split, 111 in several; no more parts than the workspace is meant for."""
    b = fq.PagedBatch([1] * 63 + [300], [655] * 62 + [32768, 400], np.zeros((64, 512), dtype=np.int64), 64, 4, device="cpu")
    assert fq.fq_attn_paged_route(b, 32, 8)[1] >= 8
    b = fq.PagedBatch([25, 19, 27, 7, 31], [2339, 639, 58, 22, 32], np.zeros((5, 37), dtype=np.int64), 64, 4, device="cpu")
    assert fq.fq_attn_paged_route(b, 32, 8)[1] <= 8  # ten, which a workgroup a row joins, took 20.6 us; four 17.7, seven 18.4
    b = fq.PagedBatch([500] * 8, [6000] * 7 + [60000], np.zeros((8, 1000), dtype=np.int64), 64, 4, device="cpu")
    rows, splits, _ = fq.fq_attn_paged_route(b, 40, 8)
    assert splits == 1 or 4000 * 40 * splits <= 1 << 20
