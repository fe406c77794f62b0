"""Serving several sequences at once out of one pool of cache pages (FlexQuant, arXiv 2501.07139, Sections "Introduction" and
"Elastic Serving": a hosted model answers requests while the memory that it may take varies).

The weights' part of that memory is what ``elastic.ElasticModel`` moves along the ensemble; the cache's part is what is kept
here.  Every block has its keys and values in pages of a pool, a sequence holds as many pages as it has positions, a step takes
any mixture of prompts, chunks of prompts and single tokens, and a sequence that has outgrown its share is cut back to the
positions that its tokens have looked at most, and its last ones.  The bit vector may change from step to step.

All arithmetic is the library's; this module keeps account of pages and lengths.
"""
from __future__ import annotations

from typing import Dict, List, Optional

import numpy as np
import torch

from . import (FqError, PagedBatch, Stack, fq_attn_paged, fq_cache_evict, fq_glue, fq_qk_norm_rope, fq_qlinear, rope_table)


class PagePool:
    """Numbers of the pages that no sequence holds; the same page of every block's pools belongs together."""

    def __init__(self, pages: int, page: int):
        self.page, self.pages = page, pages
        self._free = list(range(pages - 1, -1, -1))

    @property
    def free(self) -> int:
        return len(self._free)

    def need(self, positions: int) -> int:
        return -(-positions // self.page)

    def take(self, count: int) -> List[int]:
        if count > len(self._free):
            raise MemoryError(f"{count} pages needed, {len(self._free)} free of {self.pages}")
        taken = [self._free.pop() for _ in range(count)]
        return taken

    def give(self, pages: List[int]) -> None:
        self._free.extend(reversed(pages))


class _Sequence:
    def __init__(self):
        self.pages: List[int] = []
        self.length = 0    # positions in the cache
        self.position = 0  # of the next token: runs ahead of the length once positions have been dropped


class PagedServer:
    """Blocks of a hosted model over a paged cache.

    stack: its shapes decide heads and key/value heads (rows of q and k over 128).  slots: sequences at once.  gains: per block
    (q_gain, k_gain), fp16 [128] on the device, for models that normalise their heads.  With `keep`, a sequence that is longer than
    `limit` after a step is cut to `keep` positions a head, the last `recent` among them.
    """

    def __init__(self, stack: Stack, slots: int, pages: int, page: int = 64, max_positions: int = 4096, gains=None,
                 keep: Optional[int] = None, recent: int = 0, limit: Optional[int] = None, device="cuda"):
        q, k = (next(iter(stack.layers[0][j].values())) for j in (0, 1))
        if q.N % 128 or k.N % 128 or (q.N // 128) % (k.N // 128):
            raise ValueError("q and k must have 128 rows a head, the query heads a multiple of the key/value heads")
        if gains is not None and len(gains) != stack.L:
            raise ValueError("a pair of gains for every block")
        if keep is not None and not (0 <= recent <= keep <= (limit if limit is not None else keep) and keep > 0):
            raise ValueError("need 0 <= recent <= keep <= limit, 0 < keep")
        self.heads, self.kv_heads, self.L, self.hidden = q.N // 128, k.N // 128, stack.L, q.K
        self.pool = PagePool(pages, page)
        self.max_positions, self.device = max_positions, torch.device(device)
        self.keep, self.recent, self.limit = keep, recent, keep if limit is None else limit
        self.gains = gains
        shape = (self.L, pages, self.kv_heads, page, 128)
        self.k, self.v = (torch.zeros(shape, dtype=torch.float16, device=self.device) for _ in range(2))
        self.rope = rope_table(max_positions, device=self.device)
        self.slots = slots
        self.seqs: Dict[int, _Sequence] = {}
        self.weights = None
        if keep is not None:  # what every position has received of the softmax, per block
            self.weights = torch.zeros((self.L, slots, self.kv_heads, max_positions), dtype=torch.float32, device=self.device)

    # ------------------------------------------------------------------ sequences
    def open(self) -> int:
        """A slot for a new sequence."""
        for i in range(self.slots):
            if i not in self.seqs:
                self.seqs[i] = _Sequence()
                return i
        raise MemoryError(f"all {self.slots} slots are taken")

    def close(self, slot: int) -> None:
        self.pool.give(self.seqs.pop(slot).pages)

    def length(self, slot: int) -> int:
        return self.seqs[slot].length

    def cache_bytes(self) -> int:
        """Bytes of the pages that sequences hold, all blocks together."""
        return (self.pool.pages - self.pool.free) * self.pool.page * self.kv_heads * 128 * 2 * 2 * self.L

    def _table(self, rows: Dict[int, List[int]]) -> np.ndarray:
        table = np.full((self.slots, max([1] + [len(p) for p in rows.values()])), -1, dtype=np.int64)
        for i, pages in rows.items():
            table[i, :len(pages)] = pages
        return table

    # ----------------------------------------------------------------------- steps
    def step(self, stack: Stack, bitvec, tokens: Dict[int, torch.Tensor]) -> Dict[int, torch.Tensor]:
        """tokens: for some slots the hidden states of their next tokens, fp16 [n, hidden] (one token, or a chunk of a prompt).
        Returns the last block's output for each.  Pages, lengths and positions change only with a step that has gone through: after an error
        they are as before, and the same tokens may be given again (of an error behind the first block, memory that cannot be
        had, the weights that cuts go by may have that attempt's share)."""
        order = sorted(tokens)
        if not order:
            return {}
        rows = {}
        for i in order:
            s, t = self.seqs[i], tokens[i]
            if t.dim() != 2 or t.shape[1] != self.hidden or t.dtype != torch.float16 or t.device != self.k.device:
                raise ValueError(f"slot {i}: tokens must be fp16 [n, {self.hidden}] on {self.k.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
            rows[i] = t.shape[0]
            if rows[i] == 0:
                raise ValueError(f"slot {i}: no tokens")
            if s.position + rows[i] > self.max_positions:
                raise FqError(-2, f"slot {i}: position {s.position + rows[i]} of {self.max_positions}")
        matrices = self._matrices(stack, bitvec)
        more = {i: self.pool.need(self.seqs[i].length + rows[i]) - len(self.seqs[i].pages) for i in order}
        if sum(more.values()) > self.pool.free:
            raise MemoryError(f"{sum(more.values())} pages needed, {self.pool.free} free of {self.pool.pages}")
        taken = {i: self.pool.take(more[i]) for i in order}
        try:
            x = self._blocks(matrices, order, tokens, rows, taken)
        except BaseException:
            for i in reversed(order):
                self.pool.give(taken[i])
            raise
        for i in order:
            s = self.seqs[i]
            s.pages += taken[i]
            s.length += rows[i]
            s.position += rows[i]
        if self.keep is not None:
            self.cut([i for i in self.seqs if self.seqs[i].length > self.limit])
        return dict(zip(order, torch.split(x, [rows[i] for i in order])))

    def _matrices(self, stack: Stack, bitvec) -> List[list]:
        """The matrices that the bit vector picks, seven a block: all there, and of shapes that go together."""
        bitvec = np.asarray(bitvec, dtype=np.uint8).reshape(-1)
        if stack.L != self.L or bitvec.size != 7 * self.L:
            raise ValueError(f"{stack.L} blocks, {bitvec.size} bit widths; the server has {self.L} blocks of seven matrices")
        picked = []
        for l, bits in enumerate(bitvec.reshape(self.L, 7).tolist()):
            for j, n in enumerate(bits):
                if n not in stack.layers[l][j]:
                    raise ValueError(f"block {l}, matrix {j}: no packing of {n} bits")
            w = [stack.layers[l][j][n] for j, n in enumerate(bits)]
            H, Q, KV, F = self.hidden, 128 * self.heads, 128 * self.kv_heads, w[4].N
            if [(m.N, m.K) for m in w] != [(Q, H), (KV, H), (KV, H), (H, Q), (F, H), (F, H), (H, F)]:
                raise ValueError(f"block {l}: matrices of shapes {[(m.N, m.K) for m in w]}")
            picked.append(w)
        return picked

    def _blocks(self, matrices: List[list], order: List[int], tokens: Dict[int, torch.Tensor], rows: Dict[int, int],
                taken: Dict[int, List[int]]) -> torch.Tensor:
        """All blocks over the tokens, their sequences as long as they are with them; the account stays as it is."""
        positions = [np.arange(self.seqs[i].position, self.seqs[i].position + rows[i]) for i in order]
        # sequences without tokens count as empty: nothing of theirs is read or changed, and the longest decides how a call is divided
        batch = PagedBatch([rows.get(i, 0) for i in range(self.slots)], [self.seqs[i].length + rows[i] if i in rows else 0 for i in range(self.slots)],
                           self._table({i: self.seqs[i].pages + taken[i] for i in order}), self.pool.page, self.pool.pages,
                           positions=np.concatenate(positions), device=self.device)
        x = torch.cat([tokens[i] for i in order])
        for l, w in enumerate(matrices):
            q_gain, k_gain = self.gains[l] if self.gains is not None else (None, None)
            acc = None if self.weights is None else self.weights[l]
            u = fq_glue(0, x)
            q, k, v = (fq_qlinear(u, w[j]) for j in range(3))
            q = fq_qk_norm_rope(q, k, v, batch, self.rope, self.k[l], self.v[l], q_gain, k_gain, out=q)
            a = fq_attn_paged(q, batch, self.k[l], self.v[l], weights=acc, weights_out=acc)
            x1 = fq_glue(2, x, fq_qlinear(a, w[3]))
            u = fq_glue(0, x1)
            m = fq_glue(5, fq_qlinear(u, w[4]), fq_qlinear(u, w[5]))
            x = fq_glue(2, x1, fq_qlinear(m, w[6]))
        return x

    def cut(self, slots: List[int]) -> List[int]:
        """Cut these sequences to `keep` positions a head, into pages of their own; their old pages are free afterwards.  All at once
        if the free pages hold the new rows of all, else one after the other.  Returns the slots for which there was no room, of
        pages or of device memory: they stay as they are, and the next step tries again."""
        slots = list(dict.fromkeys(slots))
        need = {i: self.pool.need(min(self.keep, self.seqs[i].length)) for i in slots}
        if sum(need.values()) <= self.pool.free and self._cut(slots):
            return []
        return [i for i in slots if need[i] > self.pool.free or not self._cut([i])]

    def _cut(self, slots: List[int]) -> bool:
        """False, and nothing changed, if the device's memory does not suffice."""
        if not slots:
            return True
        lengths = [self.seqs[i].length for i in slots]
        new = [self.pool.take(self.pool.need(min(self.keep, n))) for n in lengths]
        try:
            batch = PagedBatch([0] * len(slots), lengths, self._table({n: self.seqs[i].pages for n, i in enumerate(slots)})[:len(slots)],
                               self.pool.page, self.pool.pages, device=self.device)
            dst = torch.from_numpy(self._table(dict(enumerate(new)))[:len(slots)].astype(np.int32)).to(self.device)
            index = torch.tensor(slots, device=self.device)
            most = max(1, *lengths)  # the library wants weights for sequences without positions, too
            kept = torch.zeros((self.L, len(slots), self.kv_heads, most), dtype=torch.float32, device=self.device)
            for l in range(self.L):  # the running weights stay until every block's rows are copied
                fq_cache_evict(batch, self.weights[l, :, :, :most].index_select(0, index), self.k[l], self.v[l], dst, self.keep, self.recent,
                               weights_out=kept[l])
            self.weights[:, :, :, :most].index_copy_(1, index, kept)  # zeros behind what stays
        except BaseException as e:
            for pages in reversed(new):
                self.pool.give(pages)
            if isinstance(e, torch.OutOfMemoryError):
                return False
            raise
        for i, pages in zip(slots, new):
            s = self.seqs[i]
            self.pool.give(s.pages)
            s.pages, s.length = pages, min(self.keep, s.length)
        return True
