"""Serving several sequences at once out of one pool of cache pages (FlexQuant, arXiv 2501.07139, Sections "Introduction" and
"Elastic Serving": a hosted model answers requests while the memory that it may take varies).

The weights' part of that memory is what ``elastic.ElasticModel`` moves along the ensemble; the cache's part is what is kept
here.  Every block has its keys and values in pages of a pool, a sequence holds as many pages as it has positions, a step takes
any mixture of prompts, chunks of prompts and single tokens, and a sequence that has outgrown its share is cut back to the
positions that its tokens have looked at most, and its last ones.  The bit vector may change from step to step.

A sequence may also go on in several ways at once: the tokens of a step are then nodes of a tree behind its positions (a drafted tree that one pass
checks, or the beams of a search, a node each step), until one path through them is kept.

All arithmetic is the library's; this module keeps account of pages and lengths.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

from . import (TREE_WORDS, FqError, PagedBatch, Stack, fq_attn_paged, fq_attn_tree, fq_cache_evict, fq_glue, fq_qk_norm_rope, fq_qlinear,
               fq_tree_commit, rope_table)


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
        # nodes behind them that are not kept yet, in the order of the cache: what each goes on from (-1: the sequence), how deep, whom it sees
        self.parents: List[int] = []
        self.depths: List[int] = []
        self.masks: List[int] = []

    @property
    def tail(self) -> int:
        return len(self.parents)


def _mask_words(masks: List[int], words: int) -> np.ndarray:
    """Masks as rows of 64-bit words."""
    return np.frombuffer(b"".join(m.to_bytes(8 * words, "little") for m in masks), dtype=np.int64).reshape(len(masks), words)


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
    def step(self, stack: Stack, bitvec, tokens: Dict[int, torch.Tensor],
             parents: Optional[Dict[int, Sequence[int]]] = None) -> Dict[int, torch.Tensor]:
        """tokens: for some slots the hidden states of their next tokens, fp16 [n, hidden] (one token, or a chunk of a prompt).
        parents: for some of these slots, of each token the node that it goes on from, -1 for the sequence itself: they become nodes, counted from 0 with
        those of the steps before, and stay so until ``accept`` or ``keep_path`` keeps some of them; meanwhile the slot takes nodes only.  Not with `keep`.
        Returns the last block's output for each.  Pages, lengths and positions change only with a step that has gone through: after an error
        they are as before, and the same tokens may be given again (of an error behind the first block, memory that cannot be
        had, the weights that cuts go by may have that attempt's share)."""
        order = sorted(tokens)
        if not order:
            return {}
        parents = {} if parents is None else {i: [int(p) for p in parents[i]] for i in parents}
        if parents and self.keep is not None:
            raise ValueError("a server that cuts its sequences takes no trees: what nodes have looked at is not added up")
        if not parents.keys() <= tokens.keys():
            raise ValueError(f"parents for slots {sorted(parents.keys() - tokens.keys())}, which get no tokens")
        rows = {}
        for i in order:
            s, t = self.seqs[i], tokens[i]
            if t.dim() != 2 or t.shape[1] != self.hidden or t.dtype != torch.float16 or t.device != self.k.device:
                raise ValueError(f"slot {i}: tokens must be fp16 [n, {self.hidden}] on {self.k.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
            rows[i] = t.shape[0]
            if rows[i] == 0:
                raise ValueError(f"slot {i}: no tokens")
            if i not in parents:
                if s.tail:
                    raise ValueError(f"slot {i}: {s.tail} nodes are not kept yet")
                if s.position + rows[i] > self.max_positions:
                    raise FqError(-2, f"slot {i}: position {s.position + rows[i]} of {self.max_positions}")
        nodes = {i: self._nodes(i, parents[i] if i in parents else None, rows[i], bool(parents)) for i in order}
        matrices = self._matrices(stack, bitvec)
        more = {i: self.pool.need(self.seqs[i].length + self.seqs[i].tail + rows[i]) - len(self.seqs[i].pages) for i in order}
        if sum(more.values()) > self.pool.free:
            raise MemoryError(f"{sum(more.values())} pages needed, {self.pool.free} free of {self.pool.pages}")
        taken = {i: self.pool.take(more[i]) for i in order}
        try:
            x = self._blocks(matrices, order, tokens, rows, taken, nodes if parents else None)
        except BaseException:
            for i in reversed(order):
                self.pool.give(taken[i])
            raise
        for i in order:
            s = self.seqs[i]
            s.pages += taken[i]
            if i in parents:
                s.parents += parents[i]
                s.depths += nodes[i][0]
                s.masks += nodes[i][1]
            else:
                s.length += rows[i]
                s.position += rows[i]
        if self.keep is not None:
            self.cut([i for i in self.seqs if self.seqs[i].length > self.limit])
        return dict(zip(order, torch.split(x, [rows[i] for i in order])))

    def _nodes(self, i: int, parents: Optional[List[int]], n: int, tree: bool) -> Tuple[List[int], List[int]]:
        """(depths, masks) of a slot's tokens: as nodes, or as the chain that they are beside other slots' trees."""
        s = self.seqs[i]
        if parents is None:
            if tree and n > 64 * TREE_WORDS:
                raise ValueError(f"slot {i}: {n} tokens beside trees (at most {64 * TREE_WORDS})")
            return list(range(n)), [(2 << k) - 1 for k in range(n)] if tree else []
        if len(parents) != n:
            raise ValueError(f"slot {i}: {len(parents)} parents for {n} tokens")
        if s.tail + n > 64 * TREE_WORDS:
            raise ValueError(f"slot {i}: {s.tail + n} nodes (at most {64 * TREE_WORDS})")
        depths, masks = list(s.depths), list(s.masks)
        for k, p in enumerate(parents):
            node = s.tail + k
            if not -1 <= p < node:
                raise ValueError(f"slot {i}: node {node} goes on from {p}")
            depths.append(0 if p < 0 else depths[p] + 1)
            masks.append((0 if p < 0 else masks[p]) | 1 << node)
            if s.position + depths[-1] >= self.max_positions:
                raise FqError(-2, f"slot {i}: position {s.position + depths[-1] + 1} of {self.max_positions}")
        return depths[s.tail:], masks[s.tail:]

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
                taken: Dict[int, List[int]], nodes: Optional[Dict[int, Tuple[List[int], List[int]]]]) -> torch.Tensor:
        """All blocks over the tokens, their sequences as long as they are with them; the account stays as it is.  nodes: of a step with trees."""
        if nodes is None:
            positions = [np.arange(self.seqs[i].position, self.seqs[i].position + rows[i]) for i in order]
        else:
            positions = [self.seqs[i].position + np.array(nodes[i][0]) for i in order]
            tails = [self.seqs[i].tail + rows[i] if i in rows else 0 for i in range(self.slots)]
            mask = np.concatenate([_mask_words(nodes[i][1], -(-max(tails) // 64)) for i in order])
            mask, tail = torch.from_numpy(mask).to(self.device), torch.tensor(tails, dtype=torch.int32, device=self.device)
        # sequences without tokens count as empty: nothing of theirs is read or changed, and the longest decides how a call is divided
        batch = PagedBatch([rows.get(i, 0) for i in range(self.slots)], [self.seqs[i].length + self.seqs[i].tail + rows[i] if i in rows else 0 for i in range(self.slots)],
                           self._table({i: self.seqs[i].pages + taken[i] for i in order}), self.pool.page, self.pool.pages,
                           positions=np.concatenate(positions), device=self.device)
        x = torch.cat([tokens[i] for i in order])
        for l, w in enumerate(matrices):
            q_gain, k_gain = self.gains[l] if self.gains is not None else (None, None)
            acc = None if self.weights is None else self.weights[l]
            u = fq_glue(0, x)
            q, k, v = (fq_qlinear(u, w[j]) for j in range(3))
            q = fq_qk_norm_rope(q, k, v, batch, self.rope, self.k[l], self.v[l], q_gain, k_gain, out=q)
            if nodes is None:
                a = fq_attn_paged(q, batch, self.k[l], self.v[l], weights=acc, weights_out=acc)
            else:
                a = fq_attn_tree(q, batch, mask, self.k[l], self.v[l], tail=tail)
            x1 = fq_glue(2, x, fq_qlinear(a, w[3]))
            u = fq_glue(0, x1)
            m = fq_glue(5, fq_qlinear(u, w[4]), fq_qlinear(u, w[5]))
            x = fq_glue(2, x1, fq_qlinear(m, w[6]))
        return x

    # ----------------------------------------------------------------------- trees
    def accept(self, drafted: Dict[int, torch.Tensor], following: Dict[int, torch.Tensor]) -> Dict[int, Tuple[List[int], int]]:
        """Keeps of these slots' nodes the path that the model itself takes: from the first node on to the first node that goes on from it and is
        drafted as the token that the model has following it.  drafted, following: int32 [nodes] on the device, the tokens that the nodes are, and those that
        the model says come after them.  Returns (nodes kept, the token after the last of them) of every slot."""
        order = sorted(drafted)
        if order != sorted(following):
            raise ValueError("drafted and following must have the same slots")
        for i in order:
            for t in (drafted[i], following[i]):
                if t.dtype != torch.int32 or tuple(t.shape) != (self.seqs[i].tail,) or t.device != self.k.device:
                    raise ValueError(f"slot {i}: drafted and following must be int32 [{self.seqs[i].tail}] on {self.k.device}")
        if not order:
            return {}
        parents = torch.tensor(sum((self.seqs[i].parents for i in order), []), dtype=torch.int32, device=self.device)
        path, accepted, bonus, _ = self._commit(order, parents=parents, drafted=torch.cat([drafted[i] for i in order]),
                                                following=torch.cat([following[i] for i in order]))
        path, accepted, bonus = path.cpu().tolist(), accepted.cpu().tolist(), bonus.cpu().tolist()
        self._kept({i: accepted[n] for n, i in enumerate(order)})
        return {i: (path[n][:accepted[n]], bonus[n]) for n, i in enumerate(order)}

    def keep_path(self, paths: Dict[int, Sequence[int]]) -> None:
        """Keeps of these slots' nodes those of a path, in rising order (the beam that has won, say; none: all are dropped)."""
        order = sorted(paths)
        for i in order:
            s, p = self.seqs[i], list(paths[i])
            if any(s.parents[node] != (p[k - 1] if k else -1) for k, node in enumerate(p) if 0 <= node < s.tail) or not all(0 <= node < s.tail for node in p):
                raise ValueError(f"slot {i}: {p} is no path through the {s.tail} nodes")
        if not order:
            return
        most = max(1, *(len(paths[i]) for i in order))
        path = np.full((len(order), most), -1, dtype=np.int32)
        for n, i in enumerate(order):
            path[n, :len(paths[i])] = list(paths[i])
        counts = torch.tensor([len(paths[i]) for i in order], dtype=torch.int32, device=self.device)
        self._commit(order, path=torch.from_numpy(path).to(self.device), accepted=counts)
        self._kept({i: len(paths[i]) for i in order})

    def _commit(self, order: List[int], **what):
        seqs = [self.seqs[i] for i in order]
        batch = PagedBatch([s.tail for s in seqs], [s.length + s.tail for s in seqs],
                           self._table({n: s.pages for n, s in enumerate(seqs)})[:len(seqs)], self.pool.page, self.pool.pages, device=self.device)
        return fq_tree_commit(batch, self.k, self.v, **what)

    def _kept(self, counts: Dict[int, int]) -> None:
        """The account after a commit: kept nodes are positions, pages behind them are free."""
        for i, m in counts.items():
            s = self.seqs[i]
            s.length += m
            s.position += m
            s.parents, s.depths, s.masks = [], [], []
            need = self.pool.need(s.length)
            self.pool.give(s.pages[need:])
            s.pages = s.pages[:need]

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
