// Trees of tokens over the paged cache, what is integers: page tables, slots and masks of a batch from request lengths (fq_paged_plan), and
// the accepting of a drafted tree with the move of its rows in the cache (fq_tree_commit).
#include "fq_paged.h"

namespace {

// ------------------------------------------------------------------ plan
// From lengths to the arrays of a batch.  With f pages on the stack of free ones, R given back by closed sequences and t_b taken by sequence b:
//   stack' = stack ++ pages of closed sequences, in order;    page j that sequence b takes = stack'[f + R - 1 - (t_0 + .. + t_(b-1) + j)],
// so that everything is prefix sums over the sequences and then work on items (pages, tokens) that find their sequence by the sums.  One workgroup does
// the sums, and the items too where they are few: such a call is a launch, the loads that wait for each other (what the sequences have, then free pages
// and tables) and the code on its way to the one CU that runs it.  So all inputs are asked for at once, nothing that is written is read again, loops are
// not unrolled (eight pages at a time in flight took 14.0 instead of 7.9 for the trees of 48 sequences), and few sequences take a quarter of the
// threads, whose barriers cost less: 7 sequences of a token 5.9 -> 4.3 us, kernel 3.1.  The tokens of many are left to a second launch with a workgroup for 1024
// of a sequence, and the nodes of trees to one with a workgroup a tree (301 sequences, 70000 tokens and 5000 pages 12.8: 9.3 and 3.6).
constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_TOKENS = 8192;   // that the first launch does itself
constexpr int TREE_NODES = 64 * 64; // of a sequence: FQ_TREE_WORDS words of 64
constexpr int SUM_CAP = 1 << 29;    // sums stay there: min(a + b, cap) is as good as + for sums of what is not negative

struct PlanArgs {
    int *q_start, *seq_len, *table;
    fq_plan_arrays a;
    int seqs, tokens, max_q, max_len, table_stride, page_log2, pages;
};

__device__ __forceinline__ int capped(int a, int b) { return min(a + b, SUM_CAP); }

// Inclusive sums of N numbers a thread over the workgroup.
template <int N, int THREADS>
__device__ __forceinline__ void block_sums(int (&x)[N], int (&scratch)[N][THREADS / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int v = __shfl_up(x[n], o, 64);
            x[n] = lane >= o ? capped(x[n], v) : x[n];
        }
    if (lane == 63)
#pragma unroll
        for (int n = 0; n < N; ++n)
            scratch[n][wave] = x[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int before = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w)
            before = w < wave ? capped(before, scratch[n][w]) : before;
        x[n] = capped(x[n], before);
    }
}

// The first of `count` entries of rising sums that is above k, which is below the last one.
__device__ __forceinline__ int find_above(const int *upto, int count, int k)
{
    int at = 0;
#pragma unroll 1
    for (int step = 1 << (31 - __builtin_clz(max(count, 1))); step > 0; step >>= 1) // entries ahead of `at` are not above
        at += at + step <= count && upto[at + step - 1] <= k ? step : 0;
    return min(at, count - 1);
}

// Page and place of position t of sequence b, as a slot; -1 where it has no page.
__device__ __forceinline__ int slot_of(const PlanArgs &p, int b, int t)
{
    const int pg = p.table[(size_t)b * p.table_stride + min(t >> p.page_log2, p.table_stride - 1)];
    return pg < 0 || pg >= p.pages ? -1 : (pg << p.page_log2) | (t & ((1 << p.page_log2) - 1));
}

// Word `word` of the mask of node i, and its depth: up the parents, which lie ahead of their children, so that the walk ends.
__device__ __forceinline__ uint64_t ancestors(const int *parents, int i, int word, int *depth)
{
    uint64_t bits = 0;
    int up = 0;
    for (int at = i;;) {
        bits |= at >> 6 == word ? 1ull << (at & 63) : 0ull;
        const int q = parents[at];
        if (q < 0 || q >= at)
            break;
        at = q;
        ++up;
    }
    *depth = up;
    return bits;
}

// Rows behind the last sequence's.
__device__ __forceinline__ void clear_rows(const PlanArgs &p, int from, int first, int step)
{
    for (int m = from + first; m < p.tokens; m += step) {
        p.a.positions[m] = 0;
        p.a.slots[m] = -1;
        for (int w = 0; w < p.a.mask_words; ++w)
            p.a.mask[(size_t)m * p.a.mask_words + w] = 0;
    }
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_kernel(PlanArgs p, int with_tokens)
{
    constexpr int TOKENS = THREADS == PLAN_THREADS ? PLAN_TOKENS : 1024, AHEAD = TOKENS / THREADS;
    __shared__ int scratch[2][THREADS / 64], scratch1[1][THREADS / 64];
    __shared__ int upto[THREADS], taken_upto[THREADS], back_upto[THREADS], held_of[THREADS], ahead[THREADS], next[THREADS];
    __shared__ int parents[TOKENS];
    const int tid = threadIdx.x;
    const int capacity = min((long long)p.max_len, (long long)p.table_stride << p.page_log2);
    const int free0 = min(max(p.a.free_count[0], 0), p.pages);
    const bool with_parents = with_tokens && p.a.parents, one_turn = p.seqs <= THREADS;
    int parent[AHEAD];
    if (with_parents && one_turn) // of the first tokens, whichever sequences they are of
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            parent[i] = tid + THREADS * i < p.tokens ? p.a.parents[tid + THREADS * i] : 0;

    // Pages that closed sequences give back go on the stack, from place `from` on.
    const auto give_back = [&](int c0, int from, int total) {
#pragma unroll 1
        for (int k = tid; k < total; k += THREADS) {
            const int s = find_above(back_upto, min(p.seqs - c0, THREADS), k), j = k - (s > 0 ? back_upto[s - 1] : 0);
            if (from + k < p.pages)
                p.a.free_pages[from + k] = p.table[(size_t)(c0 + s) * p.table_stride + j];
        }
    };
    int back = 0; // of all sequences; more than one turn of them: all are looked at ahead of the rest
    if (!one_turn)
        for (int c0 = 0; c0 < p.seqs; c0 += THREADS) {
            const int b = c0 + tid;
            int sum[1] = {b < p.seqs && p.a.new_tokens[b] < 0 ? min(max(p.a.held[b], 0), p.table_stride) : 0};
            block_sums<1, THREADS>(sum, scratch1);
            back_upto[tid] = sum[0];
            __syncthreads();
            const int total = back_upto[THREADS - 1];
            give_back(c0, min(capped(free0, back), p.pages), total);
            back = capped(back, total);
            __syncthreads();
        }

    int tokens = 0, taken = 0;
    for (int c0 = 0; c0 < p.seqs; c0 += THREADS) {
        const int b = c0 + tid, seqs = min(p.seqs - c0, THREADS);
        int n = 0, before = 0, held = 0, position = 0;
        bool open = false;
        if (b < p.seqs) {
            const int want = p.a.new_tokens[b];
            before = p.a.cached[b];
            held = p.a.held[b];
            position = p.a.next_position ? p.a.next_position[b] : 0;
            open = want >= 0;
            before = min(max(before, 0), capacity);
            held = min(max(held, 0), p.table_stride);
            position = p.a.next_position ? position : before;
            n = min(min(max(want, 0), p.max_q), capacity - before);
        }
        int sum[2] = {n, open || b >= p.seqs ? 0 : held};
        block_sums<2, THREADS>(sum, scratch);
        const int end = min(capped(tokens, sum[0]), p.tokens), first = min(capped(tokens, sum[0] - n), p.tokens);
        n = end - first;
        const int len = open ? before + n : 0;
        const int need = open ? max(((len + (1 << p.page_log2) - 1) >> p.page_log2) - held, 0) : 0;
        int need_upto[1] = {need};
        block_sums<1, THREADS>(need_upto, scratch1);
        upto[tid] = end;
        taken_upto[tid] = need_upto[0];
        back_upto[tid] = sum[1];
        held_of[tid] = held;
        ahead[tid] = before;
        next[tid] = position;
        if (with_parents && one_turn)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                parents[tid + THREADS * i] = parent[i];
        __syncthreads();
        const int all_tokens = upto[THREADS - 1], pages = taken_upto[THREADS - 1];
        if (one_turn && back_upto[THREADS - 1] > 0) {
            back = back_upto[THREADS - 1];
            give_back(0, free0, back);
            __syncthreads();
        }
        const int have = min(free0 + min(back, p.pages), p.pages);
        if (b < p.seqs) {
            p.q_start[b] = first;
            p.seq_len[b] = len;
            p.a.held_out[b] = open ? held + min(max(have - capped(taken, need_upto[0] - need), 0), need) : 0;
        }
#pragma unroll 1
        for (int k = tid; k < pages; k += THREADS) {
            const int s = find_above(taken_upto, seqs, k), at = have - 1 - capped(taken, k), column = held_of[s] + k - (s > 0 ? taken_upto[s - 1] : 0);
            if (column < p.table_stride)
                p.table[(size_t)(c0 + s) * p.table_stride + column] = at >= 0 ? p.a.free_pages[at] : -1;
        }
        if (with_tokens) {
            const int count = all_tokens - tokens;
            if (with_parents && !one_turn) {
                for (int k = tid; k < count; k += THREADS)
                    parents[k] = p.a.parents[tokens + k];
                __syncthreads();
            }
            const int words = p.a.mask_words > 1 ? p.a.mask_words : 1;
#pragma unroll 1
            for (int k = tid; k < count * words; k += THREADS) {
                const int m = words > 1 ? k / words : k, word = k - m * words;
                const int s = find_above(upto, seqs, tokens + m), first_of = s > 0 ? upto[s - 1] : tokens, i = tokens + m - first_of;
                int page = -1, t = 0;
                if (word == 0) { // its page: one that the sequence had, or the one that it gets above, from where that comes
                    t = ahead[s] + i;
                    const int column = t >> p.page_log2, mine = capped(taken, s > 0 ? taken_upto[s - 1] : 0), top = have - 1 - (mine + column - held_of[s]);
                    const int *from = column < held_of[s] ? p.table + (size_t)(c0 + s) * p.table_stride + column : top >= 0 ? p.a.free_pages + top : nullptr;
                    page = from ? *from : -1;
                }
                int depth = i;
                if (p.a.parents) {
                    const uint64_t bits = ancestors(parents + (first_of - tokens), i, word, &depth);
                    if (p.a.mask_words)
                        p.a.mask[(size_t)(tokens + m) * p.a.mask_words + word] = bits;
                }
                if (word == 0) {
                    p.a.positions[tokens + m] = next[s] + depth;
                    p.a.slots[tokens + m] = page < 0 || page >= p.pages ? -1 : (page << p.page_log2) | (t & ((1 << p.page_log2) - 1));
                }
            }
        }
        tokens = all_tokens;
        taken = capped(taken, pages);
        if (c0 + THREADS >= p.seqs && tid == 0) {
            p.q_start[p.seqs] = tokens;
            p.a.free_out[0] = max(have - taken, 0);
            p.a.lacking[0] = max(taken - have, 0);
        }
        if (!one_turn)
            __syncthreads();
    }
    if (with_tokens)
        clear_rows(p, tokens, tid, THREADS);
}

// The tokens of many: a workgroup for 1024 tokens of a sequence, or for all nodes of a tree; the last one for what is behind the tokens.
__global__ __launch_bounds__(256) void plan_tokens_kernel(PlanArgs p)
{
    __shared__ int parents[TREE_NODES];
    const int b = blockIdx.x, tid = threadIdx.x;
    if (b == p.seqs) {
        clear_rows(p, p.q_start[p.seqs], blockIdx.y * 256 + tid, gridDim.y * 256);
        return;
    }
    const int first = p.q_start[b], n = p.q_start[b + 1] - first, older = p.seq_len[b] - n;
    const int position = p.a.next_position ? p.a.next_position[b] : older;
    if (!p.a.parents) {
        for (int i0 = blockIdx.y * 1024; i0 < n; i0 += gridDim.y * 1024)
            for (int i = i0 + tid; i < min(n, i0 + 1024); i += 256) {
                p.a.positions[first + i] = position + i;
                p.a.slots[first + i] = slot_of(p, b, older + i);
            }
        return;
    }
    for (int i = tid; i < n; i += 256)
        parents[i] = p.a.parents[first + i];
    __syncthreads();
    const int words = p.a.mask_words > 1 ? p.a.mask_words : 1;
    for (int k = tid; k < n * words; k += 256) {
        const int i = words > 1 ? k / words : k, word = k - i * words;
        int depth;
        const uint64_t bits = ancestors(parents, i, word, &depth);
        if (p.a.mask_words)
            p.a.mask[(size_t)(first + i) * p.a.mask_words + word] = bits;
        if (word == 0) {
            p.a.positions[first + i] = position + depth;
            p.a.slots[first + i] = slot_of(p, b, older + i);
        }
    }
}

// ------------------------------------------------------------------ commit
// A workgroup for one sequence, layer and two or eight heads.  Every wavefront finds the path itself (64 nodes a step, a ballot for the children: a barrier
// would cost as much) and takes every fourth of the items, an item being a row of the path for one head of keys or values, sixteen lanes wide.  Thirty-two items
// a turn, loads ahead of stores, rows in rising order for each head.  Node path[k] is at least k (a path that is found rises, of a given one each node is taken so):
// what a turn reads lies at or behind what it writes, and no later turn reads what an earlier one wrote.  No other wavefront has its heads.  Bound by the chain of loads for one sequence
// (lengths, nodes and pages, rows), by starting workgroups and the rows' way for many (29 sequences, 32 layers of 8 heads, 26 MB: a wavefront for each head of
// keys and of values 15.6 us, so 10.8: 3.1 TB/s read and written).
constexpr int COMMIT_ITEMS = 32; // of a turn

struct CommitArgs {
    PagedSeqs s;
    const int *tail, *parents, *drafted, *following;
    _Float16 *k, *v;
    int *path, *accepted, *bonus, *new_len;
    int layers, kv_heads, path_stride, group_heads, head_groups;
};

__global__ __launch_bounds__(256) void commit_kernel(CommitArgs p)
{
    const int b = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int layer = blockIdx.x / p.head_groups, head0 = (blockIdx.x - layer * p.head_groups) * p.group_heads, heads = min(p.kv_heads - head0, p.group_heads);
    const SeqRange s = seq_range(p.s, b);
    const bool walk = p.parents != nullptr, writes = blockIdx.x == 0 && wave == 0;
    const int tail = min(max(p.tail ? p.tail[b] : s.n, 0), s.len), base = s.len - tail, nodes = min(s.n, tail);
    int *const path_out = p.path + (size_t)b * p.path_stride;
    const int most = walk ? min(nodes, p.path_stride) : min(min(max(p.accepted[b], 0), p.path_stride), tail);
    const size_t layer_at = (((size_t)layer * p.s.pages * p.kv_heads) << p.s.page_log2) * PD;

    // asked for together: the pages from the tail's first on, a lane each, and the first 64 nodes
    const int page0 = base >> p.s.page_log2;
    const int *const table = p.s.table + (size_t)b * p.s.table_stride;
    const int pages = table[min(page0 + lane, p.s.table_stride - 1)];
    const int node = min(lane, max(nodes, 1) - 1);
    int parent0 = -2, drafted0 = 0, next0 = 0;
    if (walk && nodes > 0) {
        parent0 = p.parents[s.first + node];
        drafted0 = p.drafted[s.first + node];
        next0 = p.following[s.first + node];
    }
    // Row of a position in the pools of one layer, or -1 where its page is none.
    const auto row_of = [&](int kvh, int t) -> long long {
        const int at = (t >> p.s.page_log2) - page0, held = __shfl(pages, at & 63, 64); // every lane takes part
        const int pg = at < 64 ? held : table[min(page0 + at, p.s.table_stride - 1)];
        return pg < 0 || pg >= p.s.pages ? -1 : (((long long)pg * p.kv_heads + kvh) << p.s.page_log2) | (t & ((1 << p.s.page_log2) - 1));
    };
    int cur = 0, next_token = -1, k0 = 0;
    bool more = most > 0;
    while (k0 < most && more) {
        // up to 64 of the path, lane k has path[k0 + k]
        int mine = -1, count = 0;
        if (walk) {
            while (count < 64 && k0 + count < most && more) {
                mine = lane == count ? cur : mine;
                ++count;
                next_token = cur < 64 ? __builtin_amdgcn_readlane(next0, cur) : p.following[s.first + cur];
                int child = -1;
                for (int c0 = cur & ~63; c0 < nodes && child < 0; c0 += 64) {
                    bool is;
                    if (c0 == 0)
                        is = lane < nodes && lane > cur && parent0 == cur && drafted0 == next_token;
                    else
                        is = c0 + lane < nodes && c0 + lane > cur && p.parents[s.first + c0 + lane] == cur && p.drafted[s.first + c0 + lane] == next_token;
                    const unsigned long long found = __builtin_amdgcn_ballot_w64(is);
                    child = found ? c0 + __builtin_ctzll(found) : -1;
                }
                more = child >= 0;
                cur = more ? child : cur;
            }
        } else {
            count = min(64, most - k0);
            mine = lane < count ? min(max(path_out[k0 + lane], k0 + lane), tail - 1) : -1;
        }
        if (walk && writes && lane < count)
            path_out[k0 + lane] = mine;
        // Rows ahead of the first one that moves need nothing.  Others behind it may be at their places too, the last one among them: a given path need not rise.
        const unsigned long long moves = __builtin_amdgcn_ballot_w64(lane < count && mine != k0 + lane);
        const int still = moves ? __builtin_ctzll(moves) : count;
        // Items: rows of the path in order, for each of the wavefront's pools (keys and values of a head are two) in turn.
        const int rows = count - still, items = rows * ((2 * heads - wave + 3) / 4);
        const uint32_t inverse = rows > 1 ? 0xffffffffu / (uint32_t)rows + 1 : 0; // 2^32 / rows rounded up: item / rows, both small
        for (int i0 = 0; i0 < items; i0 += COMMIT_ITEMS) {
            h8 moved[COMMIT_ITEMS / 4];
            _Float16 *to[COMMIT_ITEMS / 4];
#pragma unroll
            for (int i = 0; i < COMMIT_ITEMS / 4; ++i) {
                to[i] = nullptr;
                if (i0 + 4 * i >= items) // uniform
                    continue;
                const int item = min(i0 + 4 * i + (lane >> 4), items - 1), set = inverse ? (int)__umulhi((uint32_t)item, inverse) : item;
                const int k = still + item - set * rows, which = wave + 4 * set, kvh = head0 + (which >> 1);
                const long long from = row_of(kvh, base + __shfl(mine, k, 64)), at = row_of(kvh, base + k0 + k);
                _Float16 *const pool = (which & 1 ? p.v : p.k) + layer_at + 8 * (lane & 15);
                to[i] = i0 + 4 * i + (lane >> 4) < items && from >= 0 && at >= 0 ? pool + at * PD : nullptr;
                moved[i] = h8{};
                if (to[i])
                    moved[i] = *reinterpret_cast<const h8 *>(pool + from * PD);
            }
            __builtin_amdgcn_s_waitcnt(FQ_WAIT_VMCNT0); // every load of the turn is back before its first store
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < COMMIT_ITEMS / 4; ++i)
                if (to[i])
                    *reinterpret_cast<h8 *>(to[i]) = moved[i];
        }
        k0 += count;
    }
    if (!writes)
        return;
    if (walk) {
        for (int k = k0 + lane; k < p.path_stride; k += 64)
            path_out[k] = -1;
        if (lane == 0) {
            p.accepted[b] = k0;
            if (p.bonus)
                p.bonus[b] = next_token;
        }
    }
    if (lane == 0)
        p.new_len[b] = base + k0;
}

} // namespace

int fq_launch_paged_plan(const fq_paged_batch &b, const fq_plan_arrays &a, fq_stream st)
{
    const PagedSeqs s = paged_seqs(b);
    PlanArgs p{const_cast<int *>(b.q_start), const_cast<int *>(b.seq_len), const_cast<int *>(b.table), a, b.seqs, b.tokens, b.max_q, b.max_len,
               b.table_stride, s.page_log2, b.pages};
    const long long rows = (long long)b.tokens * (a.mask_words > 1 ? a.mask_words : 1);
    const int with_tokens = rows <= (a.parents ? 1024 : PLAN_TOKENS);
    if (b.seqs <= 256 && (rows <= 1024 || !with_tokens))
        hipLaunchKernelGGL(plan_kernel<256>, dim3(1), dim3(256), 0, st, p, with_tokens);
    else
        hipLaunchKernelGGL(plan_kernel<PLAN_THREADS>, dim3(1), dim3(PLAN_THREADS), 0, st, p, with_tokens);
    const int parts = (b.max_q + 1023) / 1024, most = (1 << 22) / (b.seqs + 1); // of a sequence's tokens; workgroups that a grid has room for
    int rc = (int)hipGetLastError();
    if (rc != 0 || with_tokens)
        return rc;
    hipLaunchKernelGGL(plan_tokens_kernel, dim3(b.seqs + 1, a.parents ? 1 : parts < most ? parts : most), dim3(256), 0, st, p);
    return (int)hipGetLastError();
}

int fq_launch_tree_commit(const fq_paged_batch &b, const int32_t *tail, const int32_t *parents, const int32_t *drafted, const int32_t *following,
                          void *k_pages, void *v_pages, int layers, int kv_heads, int32_t *path, int path_stride, int32_t *accepted, int32_t *bonus,
                          int32_t *new_len, fq_stream st)
{
    // few workgroups: two heads each, so that a wavefront has one pool (one sequence, four layers of eight heads: 4.9 -> 4.0 us)
    const int group_heads = (long long)layers * ((kv_heads + 7) / 8) * b.seqs >= 256 ? 8 : 2;
    CommitArgs p{paged_seqs(b), tail, parents, drafted, following, static_cast<_Float16 *>(k_pages), static_cast<_Float16 *>(v_pages), path, accepted,
                 bonus, new_len, layers, kv_heads, path_stride, group_heads, (kv_heads + group_heads - 1) / group_heads};
    hipLaunchKernelGGL(commit_kernel, dim3(layers * p.head_groups, b.seqs), dim3(256), 0, st, p);
    return (int)hipGetLastError();
}
