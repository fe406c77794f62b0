// Attention of new tokens over a paged key/value cache (serving several sequences out of one pool of pages).
//
// Token i of the n new ones of a sequence of S positions sees the positions t <= S - n + i (its own key is in the cache already).
// Query head h reads key/value head h / G, G = heads / kv_heads:
//   out = sum_t p[t] V[t],  p = softmax_t(scale * q . K[t]),  lse = log sum_t exp(scale * q . K[t]),
// and for the eviction of positions the column sums w[t] = w_in[t] + sum over tokens and the G heads of p[t].
//
// The (token, head of the group) pairs of one key/value head are the rows of the matrix products, token after token, so heads that
// share keys share their loads.  With keys as the first operand of 16x16x32 MFMAs a lane holds scores of ONE row (column l % 16 of
// S^T = K . Q^T): maximum and sum need in-lane work and two cross-lane steps, and exp(S - max), rounded to fp16, is the second
// operand of O^T = V^T . P^T as it stands.  The weights are fp16 (their sum and lse are of the unrounded fp32 ones) and taken 2^15 or 2^7 times too large, so
// that fp16's least normal number, 2^-14, is 2^-29 or 2^-21 of the largest: above that an error of at most 2^-11 of each term, as the output's own
// rounding, and below it at most 2^-40 or 2^-32 of the largest, however many positions one row's reference spans (as they stood, terms below 2^-25 were lost
// from the product and kept in the sum: a row whose many positions have 2^-23 of the largest each was off by a fifth).
// V^T comes from row-major values through the transposing LDS read.
//
// With TREE the kernels are those of fq_attn_tree: the last `tail` positions of a sequence are nodes of a tree (drafted tokens, or the steps of
// several beams), and token i sees all positions ahead of them and of the nodes those whose bits its mask has.  Nothing else differs: what
// is shared by all rows is read once for all of them, and the masks are looked at in the tiles that the tail reaches into only.
#include "fq_paged.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct PagedAttnArgs {
    PagedSeqs s;
    const _Float16 *q, *k, *v;
    _Float16 *out;            // [tokens][heads][128]
    float *lse;               // [tokens][heads] or NULL
    float *part_o, *part_ml;  // [splits][tokens][heads][128], [..][2]: unnormalised output; maximum (in powers of 2) and sum
    const float *weights;     // [seqs][kv_heads][weights_stride], or NULL: zeros
    float *weights_out;
    float *scores;            // [tokens][heads][scores_stride]: scaled scores of sequences of few rows; [parts][seqs][kv_heads][..]: parts of column sums
    float scale;              // times log2(e): scores are powers of 2
    int scores_stride, parts, part_rows, ldq, heads, kv_heads, group, splits, chunk, tiles, weights_stride, packed;
    const uint64_t *mask; // TREE: [tokens][mask_words], bit j of word w: node 64 w + j of the tail
    const int *tail;      // TREE: [seqs], or NULL: the tokens of the call
    int mask_words;
};

// Positions ahead of the tail of a sequence.
__device__ __forceinline__ int ahead_of_tail(const PagedAttnArgs &p, const SeqRange &s, int b)
{
    return s.len - min(max(p.tail ? p.tail[b] : s.n, 0), s.len);
}

// 64 bits of a mask from bit `at` on, which may be negative: ahead of the mask everything is seen, behind its words nothing.
__device__ __forceinline__ uint64_t mask_window(const uint64_t *row, int words, int at)
{
    const int w = at >> 6, shift = at & 63;
    const uint64_t lo = w < 0 ? ~0ull : w < words ? row[w] : 0, hi = w < -1 ? ~0ull : w + 1 < words ? row[w + 1] : 0;
    return shift ? lo >> shift | hi << (64 - shift) : lo;
}

// A tile of rows of one sequence and key/value head.
struct RowTile {
    SeqRange s;
    int b, row0, rows, seen; // first row, rows of the sequence and head, positions that the tile's last row sees
    int older;               // positions ahead of the tokens (may be negative), with TREE ahead of the tail
};

// Tile `tile` of TR rows, counted over the sequences; rows < 0 where there is none.  Every wavefront scans the sequences' tile counts.
// TREE with p.packed: item `tile` of the splits of all tiles, a sequence's splits in turn and in each the tiles, which read the same positions; *split takes
// its number.
template <int TR, bool TREE>
__device__ __forceinline__ RowTile find_tile(const PagedAttnArgs &p, int tile, int *split)
{
    const bool packed = TREE && p.packed;
    const int lane = threadIdx.x & 63;
    RowTile r;
    r.rows = -1;
    int base = 0;
    for (int i = 0; i < p.s.seqs; i += 64) {
        int count = 0, older = 0;
        SeqRange s = {0, 0, 0};
        if (i + lane < p.s.seqs) {
            s = seq_range(p.s, i + lane);
            older = TREE ? ahead_of_tail(p, s, i + lane) : s.len - s.n;
            count = (s.n * p.group + TR - 1) / TR;
            if (packed)
                count *= max((s.len + p.chunk - 1) / p.chunk, 1);
        }
        int upto = count; // inclusive sums over the lanes
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            upto += lane >= o ? v : 0;
        }
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(base + upto > tile);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            r.b = i + at;
            int mine = tile - base - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(count, at));
            r.s.first = __builtin_amdgcn_readlane(s.first, at); // not loaded again: a tile waits for fewer loads in turn
            r.s.n = __builtin_amdgcn_readlane(s.n, at);
            r.s.len = __builtin_amdgcn_readlane(s.len, at);
            r.older = __builtin_amdgcn_readlane(older, at);
            r.rows = r.s.n * p.group;
            if (packed) {
                const int tiles = (r.rows + TR - 1) / TR;
                *split = mine / tiles;
                mine -= *split * tiles;
            }
            r.row0 = mine * TR;
            const int last = min(r.row0 + TR, r.rows) - 1;
            r.seen = TREE ? r.s.len : max(min(r.s.len - r.s.n + last / p.group + 1, r.s.len), 0);
            return r;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return r;
}

typedef float f2 __attribute__((ext_vector_type(2)));
typedef short s4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bool is_finite(_Float16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7c00) != 0x7c00; }

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// The largest magnitudes of both halves of the dwords, as bits: 0x7c00 and above are not finite.
__device__ __forceinline__ us2 largest_bits(h8 x, us2 so_far)
{
    const u4v u = __builtin_bit_cast(u4v, x) & 0x7fff7fffu;
    const uint32_t d[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        so_far = __builtin_elementwise_max(so_far, __builtin_bit_cast(us2, d[i]));
    return so_far;
}

__device__ __forceinline__ bool finite_bits(us2 m) { return m.x < 0x7c00 && m.y < 0x7c00; }

__device__ __forceinline__ bool all_finite(h8 x) { return finite_bits(largest_bits(x, us2{0, 0})); }

__device__ __forceinline__ h8 finite_only(h8 x)
{
    h8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        y[e] = is_finite(x[e]) ? x[e] : (_Float16)0.f;
    return y;
}

// Four halves of one column from four consecutive rows: lane j of sixteen names the 8 bytes of row j / 4, columns 4 (j % 4)... of a
// 4 x 16 block and gets column j of it.
__device__ __forceinline__ h4 lds_column(const _Float16 *at)
{
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v *)(at)));
}

// ------------------------------------------------- up to sixteen rows a sequence
// Single tokens: one tile a sequence and head.  Four wavefronts, 32 positions of every 128 each: keys straight into registers as MFMA
// operands, values through a part of LDS of the wavefront's own (no barrier in the loop), and one merge of the four at the end.  Bound by the read
// of the cache (one token of 32 heads over 100003 positions of 8 key/value heads: 410 MB in 69 us, 5.9 TB/s, and 6 for the join), short calls by the chain of
// loads: length and table, keys and values, output (330 positions of 32 heads 7.5 us).  With SCORES the scaled scores of every row are left for the column sums, which need the sum over all splits first.
constexpr int FEW = 16, FEW_CHUNK = 16 * 64; // rows; the most positions of a split: a lane of a wavefront has the page of sixteen
constexpr float RAISE_FEW = 15.f, DOWN_FEW = 0x1p-15f; // powers of two; a weight is at most 1 here, and 65504 the largest in fp16

typedef const __attribute__((address_space(4))) int *const_ints; // read through the scalar cache; nothing writes them in these kernels

// Sequence and split of workgroup `job` of a large grid whose sequences have several splits: those that there are come first, so that the
// workgroups with nothing to do (sequences shorter than the longest) follow them (64 sequences of 17 to 4096 positions, caches cold: 48.0 -> 44.8 us).
__device__ __forceinline__ bool find_split(const PagedAttnArgs &p, int job, int *b, int *split)
{
    const int lane = threadIdx.x & 63;
    for (int i = 0, base = 0; i < p.s.seqs; i += 64) {
        int count = 0;
        if (i + lane < p.s.seqs) {
            const SeqRange s = seq_range(p.s, i + lane);
            count = s.n > 0 ? max((s.len + p.chunk - 1) / p.chunk, 1) : 0;
        }
        int upto = count;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            upto += lane >= o ? v : 0;
        }
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(base + upto > job);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            *b = i + at;
            *split = job - base - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(count, at));
            return true;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

template <bool SCORES, bool TREE = false>
__global__ __launch_bounds__(256, 2) void attn_paged_few_kernel(PagedAttnArgs p)
{
    // values of a step: 32 rows of 16 chunks of eight, chunk ch of row r at ch ^ 2 (r % 8), so that the transposing read of sixteen rows by
    // two chunks meets every bank twice; afterwards the wavefronts' outputs
    __shared__ h8 Vs[4][32 * 16];
    __shared__ float ms[4][FEW], ls[4][FEW];
    const int kvh = blockIdx.x % p.kv_heads;
    int b = blockIdx.x / p.kv_heads, split = blockIdx.y;
    if (p.packed && !find_split(p, b, &b, &split))
        return;
    const int begin = split * p.chunk;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The pages of all blocks of sixteen positions of the split, a lane each, asked for together with the lengths: one wait less ahead of the cache.
    const int pages = p.s.table[(size_t)b * p.s.table_stride + min(((begin >> 4) + lane) >> (p.s.page_log2 - 4), p.s.table_stride - 1)];
    const int q0 = ((const_ints)p.s.q_start)[b], q1 = ((const_ints)p.s.q_start)[b + 1], len = min(max(((const_ints)p.s.seq_len)[b], 0), p.s.max_len);
    const int first = min(max(q0, 0), p.s.tokens), n = min(max(q1, first), p.s.tokens) - first, rows = min(n * p.group, FEW);
    const int end = min(len, begin + p.chunk);
    if (rows == 0 || (begin >= end && split > 0))
        return;
    const int col = lane & 15, g = lane >> 4;
    const int token = min(col, rows - 1) / p.group, head = kvh * p.group + min(col, rows - 1) - token * p.group;
    // positions this lane's row sees; ... that every row sees; may be negative.  TREE: both are the positions ahead of the tail
    const int base = TREE ? ahead_of_tail(p, SeqRange{first, n, len}, b) : 0;
    const int seen = TREE ? base : len - n + token + 1, all_seen = TREE ? base : len - n + 1;
    const uint64_t *const mask = TREE ? p.mask + (size_t)(first + token) * p.mask_words : nullptr;

    h8 qb[4];
    {
        const _Float16 *src = p.q + (size_t)(first + token) * p.ldq + head * PD + 8 * g;
#pragma unroll
        for (int s = 0; s < 4; ++s)
            qb[s] = *reinterpret_cast<const h8 *>(src + 32 * s);
    }
    f4 acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        acc[i] = f4{0.f, 0.f, 0.f, 0.f};
    float mx = -INFINITY, l = 0.f;

    h8 *const V = Vs[wave];
    // the lane's part of the transposing reads: rows 4g + col / 4 of a block of sixteen, columns 4 (col % 4)
    const int vrow = 4 * g + (col >> 2);
    const int vbase = vrow * 256 + ((vrow & 7) << 5) + ((col & 3) << 3);
    float *scores = nullptr;
    if constexpr (SCORES)
        scores = p.scores + ((size_t)(first + token) * p.heads + head) * p.scores_stride + 4 * g;
    // Read once, and past the caches' usual order of eviction: a token over 100003 positions 83.8 -> 75.6 us, with column sums of 24 sequences 70 -> 63.
    for (int t0 = begin + 32 * wave; t0 < end; t0 += 128) {
        const int block = (t0 - begin) >> 4; // of the split
        h8 kk[2][4], vv[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int page = min(max(__builtin_amdgcn_readlane(pages, block + i), 0), p.s.pages - 1);
            const size_t at = ((((size_t)page * p.kv_heads + kvh) << p.s.page_log2) | (size_t)((t0 + 16 * i) & ((1 << p.s.page_log2) - 1))) * PD;
            const _Float16 *k = p.k + at, *v = p.v + at;
#pragma unroll
            for (int s = 0; s < 4; ++s)
                kk[i][s] = __builtin_nontemporal_load(reinterpret_cast<const h8 *>(k + (col * PD + 32 * s + 8 * g)));
#pragma unroll
            for (int s = 0; s < 4; ++s)
                vv[i][s] = __builtin_nontemporal_load(reinterpret_cast<const h8 *>(v + ((4 * s + g) * PD + 8 * col)));
        }
        f4 st[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            st[i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s)
                st[i] = mfma16x16x32(kk[i][s], qb[s], st[i]);
            st[i] *= p.scale;
        }
        uint32_t not_finite = 0; // rows of the step, bit 16 i + 4 s + g, with values that not every row sees and that are not finite
        if (t0 + 32 > min(all_seen, end)) { // uniform; rows that nobody sees may hold anything, and 0 * NaN is NaN
            const uint32_t bits = TREE ? (uint32_t)(mask_window(mask, p.mask_words, t0 - base) >> (4 * g)) : 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if constexpr (TREE)
                        st[i][v] = t0 + 16 * i + 4 * g + v < end && (bits >> (16 * i + v) & 1) ? st[i][v] : -INFINITY;
                    else
                        st[i][v] = t0 + 16 * i + 4 * g + v < min(seen, end) ? st[i][v] : -INFINITY;
                    if (t0 + 16 * i + 4 * v + g >= end)
                        vv[i][v] = h8{};
                    if (all_seen < end) { // a chunk's own positions: out of the product, and added for the rows that see them (below)
                        const unsigned long long bad = __builtin_amdgcn_ballot_w64(!all_finite(vv[i][v]));
                        if (bad) {
                            vv[i][v] = finite_only(vv[i][v]);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                not_finite |= (bad >> (16 * r) & 0xffffu) ? 1u << (16 * i + 4 * v + r) : 0u;
                        }
                    }
                }
        }
        if constexpr (SCORES) {
            if (col < rows) {
                *reinterpret_cast<f4 *>(scores + t0) = st[0];
                *reinterpret_cast<f4 *>(scores + t0 + 16) = st[1];
            }
        }
        float top = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mnew = fmaxf(mx, top), mref = mnew == -INFINITY ? 0.f : mnew;
        if (__builtin_amdgcn_ballot_w64(mnew != mx) != 0) { // some row's maximum moved
            const float alpha = __builtin_amdgcn_exp2f(mx - mref);
            mx = mnew;
            l *= alpha;
#pragma unroll
            for (int db = 0; db < 8; ++db)
                acc[db] *= alpha;
        }
        h8 pb;
        float sum = 0.f;
        const float low = mref - RAISE_FEW;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = __builtin_amdgcn_exp2f(st[i][v] - low);
                sum += e;
                pb[4 * i + v] = (_Float16)e;
            }
        l += sum;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int r = 16 * i + 4 * s + g;
                V[r * 16 + (col ^ (2 * (r & 7)))] = vv[i][s];
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const char *at = reinterpret_cast<const char *>(V) + (vbase ^ (db << 5));
            const h4 lo = lds_column(reinterpret_cast<const _Float16 *>(at)), hi = lds_column(reinterpret_cast<const _Float16 *>(at + 4096));
            acc[db] = mfma16x16x32(h8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, pb, acc[db]);
        }
        __builtin_amdgcn_wave_barrier();
        for (; not_finite; not_finite &= not_finite - 1) {
            const int t = t0 + __builtin_ctz(not_finite);
            if (TREE ? !(mask_window(mask, p.mask_words, t - base) & 1) : t >= seen)
                continue;
            const _Float16 *v = p.v + pool_row(p.s.table, p.s.table_stride, p.s.page_log2, p.s.pages, p.kv_heads, kvh, b, t) * PD + 4 * g;
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                const h4 x = *reinterpret_cast<const h4 *>(v + 16 * db);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[db][e] += is_finite(x[e]) ? 0.f : (float)x[e];
            }
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();
    f4 *const O = reinterpret_cast<f4 *>(&Vs[wave][0]);
#pragma unroll
    for (int db = 0; db < 8; ++db)
        O[64 * db + lane] = acc[db];
    if (g == 0) {
        ms[wave][col] = mx;
        ls[wave][col] = l;
    }
    __syncthreads();
    if (col >= rows)
        return;
    // thread: row col, dimensions 16 db + 4 g of two db's
    const float m = fmaxf(fmaxf(ms[0][col], ms[1][col]), fmaxf(ms[2][col], ms[3][col])), mref = m == -INFINITY ? 0.f : m;
    float w[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_exp2f(ms[i][col] - mref) * DOWN_FEW;
        sum += w[i] * ls[i][col];
    }
    const bool only = len <= p.chunk; // no other split has any of it
    const size_t at = (size_t)(first + token) * p.heads + head, part = (size_t)split * p.s.tokens * p.heads + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int db = 2 * wave + i;
        f4 o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            o += reinterpret_cast<const f4 *>(&Vs[k][0])[64 * db + lane] * w[k];
        if (only) {
            const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum); // a row that sees nothing: zeros; NaN stays
            *reinterpret_cast<h4 *>(p.out + at * PD + 16 * db + 4 * g) =
                h4{(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
        } else
            *reinterpret_cast<f4 *>(p.part_o + part * PD + 16 * db + 4 * g) = o;
    }
    if (wave == 0 && g == 0) {
        if (only) {
            if (p.lse)
                p.lse[at] = (m + log2f(sum)) * LN2; // log2(0) is -inf
        } else {
            p.part_ml[2 * part] = m;
            p.part_ml[2 * part + 1] = sum;
        }
    }
}

// ------------------------------------------------- tiles of 64 and 128 rows
// Chunks.  Four wavefronts, 32 rows each (KS = 1), or two by two with every key tile of 64 positions halved between them (KS = 2: 64 rows).
// Keys and values go through double-buffered LDS tiles, keys straight from memory, values through registers (the compiler keeps
// track of only a few copies into LDS, and waits for all of them at once beyond those).  32x32x16 MFMAs: a lane has 32 scores of one row, so
// half as many reads of LDS per product as with sixteen rows, and one step across lanes for a row's maximum.  Where a tile lies in one page (WHOLE:
// pages of 64 positions and more) its address is formed once, not for each block of sixteen: a quarter of a step's instructions.
// Bound by the issue of vector and matrix instructions together at the clock that this load allows (2048 tokens of 32 heads behind 30720 positions:
// 1.06 ms, 1.01 PFLOP/s; an exponential takes sixteen clocks, a step of 128 rows 32 of them and 32 products a wavefront), short chunks by the latency of
// their steps.
constexpr int KT = 64; // positions of a tile
constexpr float LAG = 8.f, RAISE = 7.f, DOWN = 0x1p-7f; // powers of two: the largest weight is at most LAG + RAISE = 15, fp16 ends at 16

constexpr int tile_rows_of(int KS) { return 128 / KS; }

typedef float f16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f16v mfma32x32x16(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float other_half(float x, float (*f)(float, float))
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1]; // values of their own: a bit cast of a vector's element reads its first one
    return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

template <int KS, bool WHOLE, bool TREE = false>
__global__ __launch_bounds__(256, 2) void attn_paged_tile_kernel(PagedAttnArgs p)
{
    constexpr int TR = tile_rows_of(KS), KB = 2 / KS; // KB: blocks of 32 positions that a wavefront has of a tile
    constexpr int PARTS = WHOLE ? 1 : 4;              // runs of rows in a page that a key tile is made of: itself, or blocks of sixteen
    // Key tiles: chunk ch (eight dimensions) of row r at ch ^ (r % 16); value tiles: at ch ^ 4 (r % 4), for the transposing reads of eight rows by
    // four chunks.  Separate arrays, named statically in a loop unrolled by two: the tile being read is then known not to be the one
    // that copies in flight write.
    __shared__ h8 Ks0[KT * 16], Ks1[KT * 16];
    __shared__ h8 Vs0[KT * 16], Vs1[KT * 16];
    __shared__ __align__(8) unsigned short not_finite[2][4]; // of a value tile that not every row sees all of: rows with such a value, per wavefront that copied them

    // Longest tiles first; where all workgroups are resident together, two a CU, dealt from both ends: b and b + half share a CU.
    const int jobs = (int)gridDim.x, half = (jobs + 1) >> 1, bidx = (int)blockIdx.x;
    const int job = bidx < half || jobs * (int)gridDim.y > 512 || (TREE && p.packed) ? bidx : jobs - 1 - (bidx - half);
    const int kvh = job % p.kv_heads;
    int split = blockIdx.y;
    const RowTile tile = find_tile<TR, TREE>(p, TREE && p.packed ? job / p.kv_heads : p.tiles - 1 - job / p.kv_heads, &split);
    if (tile.rows < 0)
        return;
    const int begin = split * p.chunk, end = min(tile.seen, begin + p.chunk);
    if (begin >= end && split > 0)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int kpart = wave % KS, qpart = wave / KS;
    const int row0 = tile.row0 + 32 * qpart; // first row of the wavefront
    const int row = row0 + col, rowc = min(row, tile.rows - 1), token = rowc / p.group, head = kvh * p.group + rowc - token * p.group;
    const int older = tile.older;
    const int seen = min(older + token + 1, tile.s.len);                               // positions this lane's row sees (not with TREE)
    const int all_seen = TREE ? older : older + min(row0, tile.rows - 1) / p.group + 1; // ... that every row of the wavefront sees
    const int any_seen = TREE ? tile.s.len : older + min(row0 + 31, tile.rows - 1) / p.group + 1;
    const uint64_t *const mask = TREE ? p.mask + (size_t)(tile.s.first + token) * p.mask_words : nullptr;
    // A wavefront without rows copies its share of the tiles and leaves the rest of the CU to others: trees have few rows, and the last tile of most is not full.
    const bool idle = TREE && row0 >= tile.rows;

    h8 qb[8];
    {
        const _Float16 *src = p.q + (size_t)(tile.s.first + token) * p.ldq + head * PD + 8 * h;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            qb[s] = *reinterpret_cast<const h8 *>(src + 16 * s);
    }

    const const_ints table = (const_ints)(p.s.table + (size_t)tile.b * p.s.table_stride);
    const int tiles = (end - begin + KT - 1) / KT, last_run = max(end - 1, 0) & ~(KT / PARTS - 1);
    const int krow = 4 * wave + (lane >> 4); // the lane's row of every block of sixteen that it copies
    const uint32_t koff = (uint32_t)(krow * 256 + (((lane & 15) ^ krow) << 4)), voff = (uint32_t)(krow * 256 + ((lane & 15) << 4));
    int pg[PARTS];
    auto load_pages = [&](int jt) { // runs behind the last one repeat it
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
            pg[i] = table[min(begin + KT * jt + 16 * i, last_run) >> p.s.page_log2];
    };
    h8 vreg[4];
    fq_rsrc kr, vr;
    auto load_block = [&](h8 *Kdst, int jt, int i) { // block i of both tiles; behind the last tile that one again
        if (i < PARTS) {
            const int t = min(begin + KT * jt + 16 * i, last_run), page = min(max(pg[i], 0), p.s.pages - 1);
            const size_t at = (((((size_t)page * p.kv_heads + kvh) << p.s.page_log2) | (size_t)(t & ((1 << p.s.page_log2) - 1)))) * 256;
            kr = make_rsrc(reinterpret_cast<const char *>(p.k) + at, KT / PARTS * 256);
            // values of positions that nobody sees may be anything, and 0 * NaN is NaN: the descriptor ends ahead of them, what is behind reads 0
            vr = make_rsrc(reinterpret_cast<const char *>(p.v) + at, (uint32_t)min(end - t, KT / PARTS) * 256u);
        }
        const uint32_t block = WHOLE ? 4096 * i : 0;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, &Kdst[64 * (wave + 4 * i)], 16, koff, block, 0, 0);
        vreg[i] = __builtin_bit_cast(h8, buf_load_b128(vr, voff, block));
    };
    const int vdst = krow * 16 + ((lane & 15) ^ (4 * (lane >> 4)));
    auto store_block = [&](h8 *Vdst, int i) { Vdst[256 * i + vdst] = vreg[i]; };
    // A weight of zero takes nothing from a position, but the matrix product has 0 * inf = NaN.  In tiles that reach behind the first row's last
    // position, values that are not finite are therefore zeros in LDS, and rows that see them get them added (below).
    const int every = TREE ? older : older + tile.row0 / p.group + 1; // positions that every row of the tile sees
    auto clear_not_finite = [&](h8 *Vdst, int jt, unsigned short *flags) {
        if (begin + KT * jt + KT <= every)
            return;
        uint32_t found = 0; // bit 4 i + r: row 16 i + 4 wave + r
        us2 most = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            most = largest_bits(vreg[i], most);
        if (__builtin_amdgcn_ballot_w64(!finite_bits(most))) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned long long bad = __builtin_amdgcn_ballot_w64(!all_finite(vreg[i]));
                Vdst[256 * i + vdst] = finite_only(vreg[i]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    found |= (bad >> (16 * r) & 0xffffu) ? 1u << (4 * i + r) : 0u;
            }
        }
        if (lane == 0)
            flags[wave] = (unsigned short)found;
    };

    f16v acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        acc[i] = f16v{};
    float mx = -INFINITY, l = 0.f;
    // byte offsets of the lane's operands in a tile: its key row, and its part of the transposing reads
    const int kat = (32 * KB * kpart + col) * 256 + ((h ^ (lane & 15)) << 4);
    const int vat = (32 * KB * kpart + 4 * h + ((lane & 15) >> 2)) * 256 + (((lane & 15) >> 2) << 6) + ((lane & 16) << 1) + ((lane & 3) << 3);

    if (tiles > 0) {
        load_pages(0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            load_block(Ks0, 0, i);
        load_pages(1);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_block(Vs0, i);
        clear_not_finite(Vs0, 0, not_finite[0]);
    }
    __builtin_amdgcn_s_waitcnt(FQ_WAIT_VMCNT0);
    __syncthreads();

    // PLAIN: this tile and the next are seen by all rows.
    auto tile_step = [&](int jt, auto parity, auto plain) {
        constexpr int PAR = decltype(parity)::value;
        constexpr bool PLAIN = decltype(plain)::value;
        const char *const Kcur = reinterpret_cast<const char *>(PAR ? Ks1 : Ks0), *const Vcur = reinterpret_cast<const char *>(PAR ? Vs1 : Vs0);
        h8 *const Knext = PAR ? Ks0 : Ks1, *const Vnext = PAR ? Vs0 : Vs1;
        const int first = begin + KT * jt + 32 * KB * kpart; // first position of the wavefront's part
        if (!idle && (PLAIN || first < min(any_seen, end))) {
            // the next tile's copies go out between the products: issued in a row they wait for each other
            f16v st[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                st[kb] = f16v{};
#pragma unroll
            for (int s = 0; s < 8; ++s) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    st[kb] = mfma32x32x16(*reinterpret_cast<const h8 *>(Kcur + ((kat ^ (s << 5)) + 8192 * kb)), qb[s], st[kb]);
                if (s & 1) {
                    load_block(Knext, jt + 1, s >> 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (!PLAIN && (first + 32 * KB > all_seen || first + 32 * KB > end)) { // uniform per wavefront
                if constexpr (TREE) {
                    uint64_t bits = mask_window(mask, p.mask_words, first - older);
                    bits &= end - first < 64 ? (1ull << (end - first)) - 1 : ~0ull; // first < end
                    bits >>= 4 * h;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            st[kb][v] = (uint32_t)(bits >> (32 * kb)) >> (8 * (v >> 2) + (v & 3)) & 1 ? st[kb][v] : -INFINITY;
                } else {
                    const int limit = min(seen, end) - first - 4 * h;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            st[kb][v] = 32 * kb + 8 * (v >> 2) + (v & 3) < limit ? st[kb][v] : -INFINITY;
                }
            }
            float top = st[0][0];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    top = fmaxf(top, st[kb][v]);
            top = other_half(top, larger) * p.scale;
            // The reference that exponentials are taken from follows the maximum once that is 2^LAG above it: the outputs are rescaled that
            // much less often, and weights up to 2^15 are as good in fp16 as those up to 1.
            if (__builtin_amdgcn_ballot_w64(top > mx + LAG) != 0) {
                const float mnew = fmaxf(mx, top);
                const float alpha = __builtin_amdgcn_exp2f(mx - (mnew == -INFINITY ? 0.f : mnew));
                mx = mnew;
                l *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[i] *= alpha;
            }
            const float raise = RAISE - (mx == -INFINITY ? 0.f : mx);
            float sum = 0.f;
            h8 pb[KB][2];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(st[kb][v], p.scale, raise));
                    sum += e;
                    pb[kb][v >> 3][v & 7] = (_Float16)e;
                }
            l += sum;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int db = 0; db < 4; ++db) {
                        const char *at = Vcur + ((vat ^ (db << 6)) + 8192 * kb + 4096 * j);
                        const h4 lo = lds_column(reinterpret_cast<const _Float16 *>(at)), hi = lds_column(reinterpret_cast<const _Float16 *>(at + 2048));
                        acc[db] = mfma32x32x16(h8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, pb[kb][j], acc[db]);
                    }
#pragma unroll
                    for (int i = (2 * kb + j) * 2 / KB; i < (2 * kb + j + 1) * 2 / KB; ++i)
                        store_block(Vnext, i); // last read in the previous step, before its barrier
                }
            if (!PLAIN && begin + KT * jt + KT > every) {
                const u2v flags = *reinterpret_cast<const u2v *>(not_finite[PAR]); // bit 16 wave + 4 i + r
                unsigned long long bits = (unsigned long long)__builtin_amdgcn_readfirstlane(flags.y) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane(flags.x);
#pragma unroll 1
                for (; bits; bits &= bits - 1) {
                    const int b = __builtin_ctzll(bits);
                    const int r = 16 * ((b & 15) >> 2) + 4 * (b >> 4) + (b & 3), t = begin + KT * jt + r;
                    if (r / (32 * KB) != kpart || (TREE ? t >= end || !(mask_window(mask, p.mask_words, t - older) & 1) : t >= seen))
                        continue;
                    const _Float16 *v = p.v + pool_row(p.s.table, p.s.table_stride, p.s.page_log2, p.s.pages, p.kv_heads, kvh, tile.b, t) * PD + 4 * h;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const h4 x = *reinterpret_cast<const h4 *>(v + 8 * i);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i >> 2][4 * (i & 3) + e] += is_finite(x[e]) ? 0.f : (float)x[e];
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_block(Knext, jt + 1, i);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_block(Vnext, i);
        }
        if constexpr (!PLAIN)
            clear_not_finite(Vnext, jt + 1, not_finite[PAR ^ 1]);
        load_pages(jt + 2);
        __builtin_amdgcn_s_waitcnt(FQ_WAIT_VMCNT0);
        __syncthreads();
    };
    const int seen_by_all = min((min(every, end) - begin) / KT, tiles); // tiles
    int jt = 0;
    for (; jt + 2 < seen_by_all; jt += 2) {
        tile_step(jt, std::integral_constant<int, 0>{}, std::true_type{});
        tile_step(jt + 1, std::integral_constant<int, 1>{}, std::true_type{});
    }
    for (; jt < tiles; jt += 2) {
        tile_step(jt, std::integral_constant<int, 0>{}, std::false_type{});
        if (jt + 1 < tiles)
            tile_step(jt + 1, std::integral_constant<int, 1>{}, std::false_type{});
    }
    l = other_half(l, add);

    if constexpr (KS == 2) { // both halves meet in LDS, in the wavefront of the first
        f4 *const acc_at = reinterpret_cast<f4 *>(qpart == 0 ? Ks0 : Ks1);
        float *const row_at = reinterpret_cast<float *>(Vs0) + 128 * qpart;
        if (kpart == 1) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc_at[64 * i + lane] = f4{acc[i >> 2][4 * (i & 3)], acc[i >> 2][4 * (i & 3) + 1], acc[i >> 2][4 * (i & 3) + 2], acc[i >> 2][4 * (i & 3) + 3]};
            row_at[lane] = mx;
            row_at[64 + lane] = l;
        }
        __syncthreads();
        if (kpart == 1)
            return;
        const float m2 = row_at[lane], l2 = row_at[64 + lane];
        const float mnew = fmaxf(mx, m2), mref = mnew == -INFINITY ? 0.f : mnew;
        const float s1 = __builtin_amdgcn_exp2f(mx - mref), s2 = __builtin_amdgcn_exp2f(m2 - mref);
        mx = mnew;
        l = l * s1 + l2 * s2;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const f4 o = acc_at[64 * i + lane];
#pragma unroll
            for (int v = 0; v < 4; ++v)
                acc[i >> 2][4 * (i & 3) + v] = acc[i >> 2][4 * (i & 3) + v] * s1 + o[v] * s2;
        }
    }
    if (row >= tile.rows)
        return;
    const bool only = p.splits == 1 || tile.seen <= p.chunk;
    const size_t at = (size_t)(tile.s.first + token) * p.heads + head;
    if (only) {
        const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l); // a row that sees nothing: zeros; NaN stays
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const h4 o = {(_Float16)(acc[i >> 2][4 * (i & 3)] * inv), (_Float16)(acc[i >> 2][4 * (i & 3) + 1] * inv),
                          (_Float16)(acc[i >> 2][4 * (i & 3) + 2] * inv), (_Float16)(acc[i >> 2][4 * (i & 3) + 3] * inv)};
            *reinterpret_cast<h4 *>(p.out + at * PD + 8 * i + 4 * h) = o;
        }
        if (h == 0 && p.lse)
            p.lse[at] = (mx + log2f(l * DOWN)) * LN2; // log2(0) is -inf
    } else {
        const size_t part = ((size_t)split * p.s.tokens + tile.s.first + token) * p.heads + head;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            *reinterpret_cast<f4 *>(p.part_o + part * PD + 8 * i + 4 * h) =
                f4{acc[i >> 2][4 * (i & 3)], acc[i >> 2][4 * (i & 3) + 1], acc[i >> 2][4 * (i & 3) + 2], acc[i >> 2][4 * (i & 3) + 3]} * DOWN;
        if (h == 0) {
            p.part_ml[2 * part] = mx;
            p.part_ml[2 * part + 1] = l * DOWN;
        }
    }
}

// Joins the splits of a row.  WAVES wavefronts each, which deal the splits among them; a wavefront takes 64 of its own at a time: a lane has one's
// maximum and sum, then two dimensions of the outputs, eight loads at a time (those are what a row waits for: a token over 100003 positions, 196
// splits of 32 rows, 9.5 us with four wavefronts, 6.2 with sixteen; 4.6 for up to eight splits, which is the launch and two loads in turn).  Rows of tiles that one split has served are done already.
template <int WAVES>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void attn_paged_merge_kernel(PagedAttnArgs p, int tile_rows)
{
    __shared__ float sums[WAVES][PD + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = WAVES > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave, part = WAVES > 1 ? wave : 0; // token * heads + head
    if (item >= p.s.tokens * p.heads)
        return;
    const int m = item / p.heads, head = item - m * p.heads;
    const SeqRange s = seq_range(p.s, seq_of_token(p.s, m));
    const int token = m - s.first;
    if (token < 0 || token >= s.n)
        return;
    const int row = token * p.group + head % p.group;
    const int last = min((row / tile_rows + 1) * tile_rows, s.n * p.group) - 1;
    if (s.len - s.n + last / p.group + 1 <= p.chunk)
        return;
    const int live = (max(s.len - s.n + token + 1, 0) + p.chunk - 1) / p.chunk;
    const size_t stride = (size_t)p.s.tokens * p.heads;
    const f2 *ml = reinterpret_cast<const f2 *>(p.part_ml) + item, *o = reinterpret_cast<const f2 *>(p.part_o) + (size_t)item * (PD / 2) + lane;
    float mx = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
    const int mine_all = (live - part + WAVES - 1) / WAVES; // splits part, part + WAVES, ...
    const auto at = [&](int i) { return (size_t)(part + WAVES * min(i, mine_all - 1)) * stride; };
    for (int i0 = 0; i0 < mine_all; i0 += 64) {
        const f2 mine = ml[at(i0 + lane)];
        float top = i0 + lane < mine_all ? mine[0] : -INFINITY;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1)
            top = fmaxf(top, __shfl_xor(top, d, 64));
        const float mnew = fmaxf(mx, top), mref = mnew == -INFINITY ? 0.f : mnew;
        const float w = i0 + lane < mine_all ? __builtin_amdgcn_exp2f(mine[0] - mref) : 0.f, alpha = __builtin_amdgcn_exp2f(mx - mref);
        float sum = i0 + lane < mine_all ? w * mine[1] : 0.f;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1)
            sum += __shfl_xor(sum, d, 64);
        mx = mnew;
        l = l * alpha + sum;
        a0 *= alpha;
        a1 *= alpha;
        const int count = min(64, mine_all - i0);
        for (int i = 0; i < count; i += 8) {
            f2 v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) // those past the last one repeat it, with a weight of zero
                v[e] = o[at(i0 + i + e) * (PD / 2)];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float we = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i + e));
                if (i + e < count) {
                    a0 = fmaf(we, v[e][0], a0);
                    a1 = fmaf(we, v[e][1], a1);
                }
            }
        }
    }
    if constexpr (WAVES > 1) {
        sums[wave][2 * lane] = a0;
        sums[wave][2 * lane + 1] = a1;
        if (lane == 0) {
            sums[wave][PD] = mx;
            sums[wave][PD + 1] = l;
        }
        __syncthreads();
        if (wave != 0)
            return;
        mx = sums[0][PD];
#pragma unroll
        for (int i = 1; i < WAVES; ++i)
            mx = fmaxf(mx, sums[i][PD]);
        l = a0 = a1 = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float w = __builtin_amdgcn_exp2f(sums[i][PD] - (mx == -INFINITY ? 0.f : mx));
            l = fmaf(w, sums[i][PD + 1], l);
            a0 = fmaf(w, sums[i][2 * lane], a0);
            a1 = fmaf(w, sums[i][2 * lane + 1], a1);
        }
    }
    const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
    *reinterpret_cast<h2 *>(p.out + (size_t)item * PD + 2 * lane) = h2{(_Float16)(a0 * inv), (_Float16)(a1 * inv)};
    if (lane == 0 && p.lse)
        p.lse[item] = (mx + log2f(l)) * LN2;
}

// The same for trees, whose rows have all splits of their sequence.  Half a wavefront has four dimensions a lane and asks for all it needs of eight splits at
// once.  A workgroup has eight heads of a token, one each half wavefront; or with SPREAD, where there are many splits for the jobs, one head, and they deal the
// splits.  Jobs are counted over the sequences that have several splits, and a grid of 1024 workgroups takes them in turn: to start a workgroup takes an XCD about
// 20 clocks (704 tokens of 40 heads, 178 of them with up to 4 splits: 10.6 us with a wavefront for each head of each token, 8.7 with a workgroup for each eight, so 6.0).
template <bool SPREAD>
__global__ __launch_bounds__(256) void attn_tree_merge_kernel(PagedAttnArgs p)
{
    __shared__ f4 sums[8][PD / 4];
    __shared__ float tops[8], norms[8];
    const int half = threadIdx.x >> 5, d = threadIdx.x & 31, groups = SPREAD ? p.heads : (p.heads + 7) / 8;
    const size_t stride = (size_t)p.s.tokens * p.heads;
    const int lane = threadIdx.x & 63;
    for (int job = blockIdx.x;; job += gridDim.x) {
        SeqRange s;
        int at = -1, base = 0; // of the job in its sequence
        for (int i = 0; i < p.s.seqs && at < 0; i += 64) {
            SeqRange mine = {0, 0, 0};
            if (i + lane < p.s.seqs)
                mine = seq_range(p.s, i + lane);
            const int count = mine.len > p.chunk ? mine.n * groups : 0;
            int upto = count; // inclusive sums over the lanes
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(upto, o, 64);
                upto += lane >= o ? v : 0;
            }
            const unsigned long long behind = __builtin_amdgcn_ballot_w64(base + upto > job);
            if (behind) {
                const int l = __builtin_ctzll(behind);
                at = job - base - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(count, l));
                s.first = __builtin_amdgcn_readlane(mine.first, l);
                s.n = __builtin_amdgcn_readlane(mine.n, l);
                s.len = __builtin_amdgcn_readlane(mine.len, l);
            }
            base += __builtin_amdgcn_readlane(upto, 63);
        }
        if (at < 0) // no more of them
            return;
        const int token = at / groups, part = at - token * groups, m = s.first + token, own = SPREAD ? part : 8 * part + half;
        const int head = min(own, p.heads - 1); // behind the last one that one again, not written: every lane comes to the next turn's sums
        const int live = (s.len + p.chunk - 1) / p.chunk, mine = SPREAD ? max((live - half + 7) / 8, 0) : live; // splits of half a wavefront, every eighth
        const size_t item = (size_t)m * p.heads + head;
        const f2 *ml = reinterpret_cast<const f2 *>(p.part_ml) + item;
        const f4 *o = reinterpret_cast<const f4 *>(p.part_o) + item * (PD / 4) + d;
        float mx = -INFINITY, l = 0.f;
        f4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < mine; i0 += 8) {
            f2 a[8];
            f4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { // those past the last one repeat it, with a weight of zero
                const int split = min(i0 + i, mine - 1) * (SPREAD ? 8 : 1) + (SPREAD ? half : 0);
                a[i] = ml[split * stride];
                v[i] = o[split * stride * (PD / 4)];
            }
            float top = mx;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                top = fmaxf(top, a[i][0]);
            const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(mx - ref);
            mx = top;
            l *= alpha;
            acc *= alpha;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i0 + i < mine) {
                    const float w = __builtin_amdgcn_exp2f(a[i][0] - ref);
                    l = fmaf(w, a[i][1], l);
                    acc += v[i] * w;
                }
        }
        if constexpr (SPREAD) {
            sums[half][d] = acc;
            if (d == 0) {
                tops[half] = mx;
                norms[half] = l;
            }
            __syncthreads();
#pragma unroll
            for (int i = 1; i < 8; ++i)
                mx = fmaxf(mx, tops[i]);
            const float ref = mx == -INFINITY ? 0.f : mx;
            l = 0.f;
            acc = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = __builtin_amdgcn_exp2f(tops[i] - ref);
                l = fmaf(w, norms[i], l);
                acc += sums[i][d] * w;
            }
            __syncthreads(); // read ahead of the next turn's
        }
        if (SPREAD ? half == 0 : own < p.heads) {
            const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
            *reinterpret_cast<h4 *>(p.out + item * PD + 4 * d) = h4{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv), (_Float16)(acc[3] * inv)};
            if (d == 0 && p.lse)
                p.lse[item] = (mx + log2f(l)) * LN2;
        }
    }
}

// --------------------------------------------------------------- column sums
// w[t] of 256 positions from a part of the rows that see them, 64 positions a wavefront, whose keys stay in registers.  The rows come by 64 a
// step through double-buffered LDS, straight from memory; with lse known a weight is one exponential.  Rows are the first operand here, so that a
// lane has sixteen weights of ONE position and adds them up in place; what differs by row (lse, positions seen) is laid beside the rows.  One
// workgroup owns its sums and the parts are added in order: no atomics, the same sums every time.  Bound by the exponentials and the unequal work of the
// workgroups (three prompts, 2628 tokens of 32 heads and 8 key/value heads: 33 us beside the attention's 41, and 4.6 for the join).
constexpr int WK = 256, WR = 64; // positions of a workgroup, rows of a step

// Rows of part `part` that see positions from t0 on: [lo, hi).
__device__ __forceinline__ void part_rows(const PagedAttnArgs &p, const SeqRange &s, int t0, int part, int *lo, int *hi)
{
    *lo = max(max(t0 - (s.len - s.n), 0) * p.group, part * p.part_rows);
    *hi = min(s.n * p.group, part * p.part_rows + p.part_rows);
}

__global__ __launch_bounds__(256, 2) void attn_paged_weights_kernel(PagedAttnArgs p)
{
    __shared__ h8 Q0[WR * 16], Q1[WR * 16]; // chunk ch of row r at ch ^ (r % 16)
    __shared__ __align__(16) float row_lse[2][WR];
    __shared__ __align__(16) int row_seen[2][WR];
    const int kvh = blockIdx.x % p.kv_heads, job = blockIdx.x / p.kv_heads, part = job % p.parts, t0 = job / p.parts * WK, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5, mine = t0 + 64 * wave; // first position of the wavefront
    int page[2]; // of the lane's positions; asked for together with the lengths
#pragma unroll
    for (int i = 0; i < 2; ++i)
        page[i] = p.s.table[(size_t)b * p.s.table_stride + min((mine + 32 * i + col) >> p.s.page_log2, p.s.table_stride - 1)];
    SeqRange s;
    s.first = min(max(((const_ints)p.s.q_start)[b], 0), p.s.tokens);
    s.n = min(max(((const_ints)p.s.q_start)[b + 1], s.first), p.s.tokens) - s.first;
    s.len = min(max(((const_ints)p.s.seq_len)[b], 0), p.s.max_len);
    if (t0 >= s.len)
        return;
    int lo, hi;
    part_rows(p, s, t0, part, &lo, &hi);
    if (lo >= hi && p.parts > 1)
        return;
    const int older = s.len - s.n;
    h8 kk[2][8]; // positions behind the last one count for nothing: what their page holds is read where it has one, page 0 or the last where not
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = mine + 32 * i + col, pg = min(max(page[i], 0), p.s.pages - 1);
        const size_t at = ((((size_t)pg * p.kv_heads + kvh) << p.s.page_log2) | (size_t)(t & ((1 << p.s.page_log2) - 1))) * PD;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            kk[i][k] = *reinterpret_cast<const h8 *>(p.k + at + 16 * k + 8 * h);
    }
    // A wavefront copies rows 16 wave + 4 i + lane / 16, i < 4, of a step; token and head of the group of each, kept up from step to step.  Rows
    // behind the last one repeat it and count for nothing.
    constexpr int NC = WR / 16;      // copies
    int token[NC + 1], head[NC + 1]; // of each, and of the row whose lse the thread looks up
#pragma unroll
    for (int i = 0; i <= NC; ++i) {
        const int ahead = i < NC ? 4 * (NC * wave + i) + (lane >> 4) : tid & (WR - 1);
        token[i] = (lo + ahead) / p.group;
        head[i] = lo + ahead - token[i] * p.group;
    }
    const int step_tokens = WR / p.group, step_heads = WR % p.group;
    float lse_n; // used where the step ends, so that nothing waits for it
    int seen_n;
    bool real_n;
    auto load = [&](h8 *dst) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const bool real = token[i] < s.n;
            const int row = 4 * ((NC * wave + i) & 3) + (lane >> 4); // modulo sixteen
            const _Float16 *src = p.q + (size_t)(s.first + (real ? token[i] : s.n - 1)) * p.ldq + (kvh * p.group + (real ? head[i] : 0)) * PD;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + 8 * ((lane & 15) ^ row)),
                                             (__attribute__((address_space(3))) void *)(dst + 64 * (NC * wave + i)), 16, 0, 0);
        }
        real_n = token[NC] < s.n && token[NC] * p.group + head[NC] < hi;
        lse_n = p.lse[(size_t)(s.first + (real_n ? token[NC] : 0)) * p.heads + kvh * p.group + (real_n ? head[NC] : 0)];
        seen_n = older + token[NC] + 1;
#pragma unroll
        for (int i = 0; i <= NC; ++i) {
            token[i] += step_tokens;
            head[i] += step_heads;
            if (head[i] >= p.group) {
                head[i] -= p.group;
                ++token[i];
            }
        }
    };
    auto store_rows = [&](int to) {
        if (tid < WR) {
            row_lse[to][tid] = real_n && lse_n != -INFINITY ? lse_n * LOG2E : INFINITY;
            row_seen[to][tid] = seen_n;
        }
    };
    float sum[2] = {0.f, 0.f};
    if (lo < hi) {
        load(Q0);
        store_rows(0);
    }
    __builtin_amdgcn_s_waitcnt(FQ_WAIT_VMCNT0);
    __syncthreads();
    const int qat = col * 256 + ((h ^ (col & 15)) << 4);
    auto step = [&](int r0, auto parity) {
        constexpr int PAR = decltype(parity)::value;
        const char *const Q = reinterpret_cast<const char *>(PAR ? Q1 : Q0);
        const bool more = r0 + WR < hi;
        if (more)
            load(PAR ? Q0 : Q1);
        if (older + (min(r0 + WR, hi) - 1) / p.group >= mine) { // some row sees some of the wavefront's positions (uniform)
            const bool whole = older + r0 / p.group + 1 >= mine + 64;
#pragma unroll
            for (int rb = 0; rb < WR / 32; ++rb) {
                f16v st[2] = {f16v{}, f16v{}};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const h8 qa = *reinterpret_cast<const h8 *>(Q + ((qat ^ (k << 5)) + 8192 * rb));
                    st[0] = mfma32x32x16(qa, kk[0][k], st[0]);
                    st[1] = mfma32x32x16(qa, kk[1][k], st[1]);
                }
                if (!whole) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int4 seen = *reinterpret_cast<const int4 *>(&row_seen[PAR][32 * rb + 8 * u + 4 * h]);
                        const int limit[4] = {seen.x, seen.y, seen.z, seen.w};
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int v = 0; v < 4; ++v)
                                st[i][4 * u + v] = mine + 32 * i + col < limit[v] ? st[i][4 * u + v] : -INFINITY;
                    }
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const f4 lse = *reinterpret_cast<const f4 *>(&row_lse[PAR][32 * rb + 8 * u + 4 * h]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            sum[i] += __builtin_amdgcn_exp2f(fmaf(st[i][4 * u + v], p.scale, -lse[v]));
                }
            }
        }
        if (more)
            store_rows(PAR ^ 1);
        __builtin_amdgcn_s_waitcnt(FQ_WAIT_VMCNT0);
        __syncthreads();
    };
    for (int r0 = lo; r0 < hi; r0 += 2 * WR) {
        step(r0, std::integral_constant<int, 0>{});
        if (r0 + WR < hi)
            step(r0 + WR, std::integral_constant<int, 1>{});
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float both = other_half(sum[i], add);
        const int t = mine + 32 * i + col;
        if (h != 0 || t >= s.len)
            continue;
        if (p.parts > 1) {
            p.scores[(((size_t)part * p.s.seqs + b) * p.kv_heads + kvh) * p.scores_stride + t] = both;
        } else {
            const size_t at = ((size_t)b * p.kv_heads + kvh) * p.weights_stride + t;
            p.weights_out[at] = (p.weights && t < older ? p.weights[at] : 0.f) + both;
        }
    }
}

// Adds the parts up, in order.
__global__ __launch_bounds__(256) void attn_paged_weights_join_kernel(PagedAttnArgs p)
{
    const int kvh = blockIdx.x % p.kv_heads, t = blockIdx.x / p.kv_heads * 256 + threadIdx.x, b = blockIdx.y;
    const SeqRange s = seq_range(p.s, b);
    if (t >= s.len)
        return;
    const size_t at = ((size_t)b * p.kv_heads + kvh) * p.weights_stride + t;
    float sum = p.weights && t < s.len - s.n ? p.weights[at] : 0.f;
    // parts that have rows which see the 256 positions, eight loads at a time
    const int part0 = max(t / WK * WK - (s.len - s.n), 0) * p.group / p.part_rows, part1 = min((s.n * p.group + p.part_rows - 1) / p.part_rows, p.parts);
    const size_t stride = (size_t)p.s.seqs * p.kv_heads * p.scores_stride;
    const float *from = p.scores + ((size_t)b * p.kv_heads + kvh) * p.scores_stride + t;
    for (int part = part0; part < part1; part += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = from[min(part + e, part1 - 1) * stride];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum += part + e < part1 ? v[e] : 0.f;
    }
    p.weights_out[at] = sum;
}

// The same where every sequence has at most sixteen rows: their scores are there already, and nothing is read twice but those.  With JOIN the
// call has 2 to 8 splits, and their parts are joined here as well (in the order of the kernel above), a launch less: every workgroup forms the rows' lse from the splits' maxima
// and sums, and the first of a sequence and head joins the outputs (24 sequences of 100 to 2048 positions, 40 heads: 11.6 -> 9.0 us).
template <bool JOIN>
__global__ __launch_bounds__(256) void attn_paged_few_weights_kernel(PagedAttnArgs p)
{
    constexpr int PER = 4; // positions a thread
    __shared__ float row_lse[FEW];
    const int kvh = blockIdx.x % p.kv_heads, block = blockIdx.x / p.kv_heads, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SeqRange s = seq_range(p.s, b);
    const int rows = min(s.n * p.group, FEW), t0 = block * (256 * PER) + tid;
    if (block * 256 * PER >= s.len && block > 0)
        return;
    const auto item_of = [&](int r) { return (size_t)(s.first + r / p.group) * p.heads + kvh * p.group + r % p.group; };
    if (JOIN && s.len > p.chunk) {
        const size_t stride = (size_t)p.s.tokens * p.heads;
        for (int r = wave; r < rows; r += 4) {
            const size_t item = item_of(r);
            const int live = (max(s.len - s.n + r / p.group + 1, 0) + p.chunk - 1) / p.chunk;
            const f2 ml = reinterpret_cast<const f2 *>(p.part_ml)[item + min(lane, max(live - 1, 0)) * stride];
            float mx = lane < live ? ml[0] : -INFINITY;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1)
                mx = fmaxf(mx, __shfl_xor(mx, d, 64));
            const float w = lane < live ? __builtin_amdgcn_exp2f(ml[0] - (mx == -INFINITY ? 0.f : mx)) : 0.f;
            float l = lane < live ? w * ml[1] : 0.f;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1)
                l += __shfl_xor(l, d, 64);
            const float lse = mx + log2f(l);
            if (lane == 0)
                row_lse[r] = lse;
            if (block > 0)
                continue;
            const f2 *o = reinterpret_cast<const f2 *>(p.part_o) + item * (PD / 2) + lane;
            float a0 = 0.f, a1 = 0.f;
            for (int i = 0; i < live; i += 8) {
                f2 v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) // those past the last one repeat it
                    v[e] = o[min(i + e, live - 1) * stride * (PD / 2)];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (i + e < live) { // uniform
                        const float we = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i + e));
                        a0 = fmaf(we, v[e][0], a0);
                        a1 = fmaf(we, v[e][1], a1);
                    }
            }
            const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
            *reinterpret_cast<h2 *>(p.out + item * PD + 2 * lane) = h2{(_Float16)(a0 * inv), (_Float16)(a1 * inv)};
            if (lane == 0)
                p.lse[item] = lse * LN2;
        }
    } else if (tid < rows) {
        row_lse[tid] = p.lse[item_of(tid)] * LOG2E;
    }
    __syncthreads();
    float sum[PER] = {};
    for (int r = 0; r < rows; ++r) {
        const size_t item = item_of(r);
        const float lse = row_lse[r];
        if (lse == -INFINITY) // a row that sees nothing
            continue;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (t0 + 256 * i < s.len)
                sum[i] += __builtin_amdgcn_exp2f(p.scores[item * p.scores_stride + t0 + 256 * i] - lse);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = t0 + 256 * i;
        if (t < s.len) {
            const size_t at = ((size_t)b * p.kv_heads + kvh) * p.weights_stride + t;
            p.weights_out[at] = (p.weights && t < s.len - s.n ? p.weights[at] : 0.f) + sum[i];
        }
    }
}

// How a call is divided: one tile of up to sixteen rows a sequence, or tiles of 64 or 128, and the positions into splits.
//
// Single tokens: a step of 128 positions takes a workgroup 1.8 us, nearly all of it the wait for memory, until about 150 workgroups together reach the
// rate of HBM; joining splits takes 3 us more, the launch.  So one split where that is no longer than short ones and the join (384 positions, and
// more where sequences and heads fill the chip), else splits as short as keep the workgroups at about 384, but no longer than 512 positions, as
// sequences differ in length.  Measured with caches cold (us at splits of 128 / 256 / 512 / 1024 positions / one split): 32 heads, 1000 positions
// 10.3 / 12.0 / 15.2 / 19.3, 4000 19.2 / 17.7 / 17.1 / 24 / 65; 8 heads, 8000 positions 13.4 / 12.4 / 15.9 / 22.9 / 121; 16 sequences of 8 heads, 500
// positions 13.0 / 13.0 / 12.4 (one), 1000 21.5 / 17.5 / 17.7 / 21.0 (one); 20 of 700 20.6 / 17.3 / 18.9 / 16.4 (one); 64 of 600 38 / 36 / 42 / 28 (one).
//
// Chunks: what an estimate (us) of these finds shortest, for tiles of 64 and 128 rows: 6 for the launch, the first loads and the end; a step of 64
// positions takes a workgroup 0.69 (128 rows: 1.0) by itself, and 256 CUs together do one in 0.9 (1.36) each, as the card lowers its clock
// under that load; joining splits takes 4 and two passes over the parts at 4 TB/s.  Where the caller says how many positions and (token, position) pairs
// several sequences have together, those are the steps and the parts, workgroups without work are 0.001 each, and the longest tile's steps count by 0.3 in
// any case, as such tiles come late and alone, and more than 8 splits cost 4 more (a workgroup a row joins them); without, all are taken to be half as
// long as the longest.  That choice stays unless the other is to save 2.5 us, which is how far the estimate is off on calls of 15 to 30 us: 300 tokens and 63 single
// ones, one of them at the end of 32768 positions, 528 -> 110 us, and 500 with 15 at up to 16384 185 -> 65; of 720 ragged batches of 2 to 8 chunks
// 158 are divided otherwise and take 20 % less on average, three of them over 5 % longer, at most 11 % (without the two, 18 of 300, at most 24 %).  Over 37 sizes of 5 to 3000 tokens and 256
// to 16000 positions its choice takes 1.8 % longer than the best of both heights and six lengths, at most 8 % (17 % where several sequences are all as
// long as the longest).  Some, as measured: 16 tokens, 8 key/value
// heads of 4 queries, 16000 positions 171 in one split, 23.5 / 21.2 / 24.8 in splits of 1024 / 512 / 256; 2048 tokens of 32 heads 50 in tiles of 128 rows, 66
// in tiles of 64; 1000 tokens 24.5 and 21.2.
//
// Column sums of chunks: into how many rows a workgroup's part goes, by an estimate too: 3.3 us and 1.8 a step of 64 rows for the longest one by itself, or
// 4 and 2.5 for all of them on 512 places (two a CU); joining the parts 4.5, 0.05 a part, and a write and a read of them at 2 TB/s.  Over 25 sizes of
// 60 to 2048 tokens and 200 to 30000 positions its choice takes 6 % longer than the best of twelve heights; parts of 512 rows (or what makes eight)
// took 38 % longer: 223 and 53 tokens of one key/value head of 8 queries 31.9 -> 19.8 us with the attention, 500 tokens of 8 heads of 4 21.7 -> 11.2 without.
struct AttnPlan {
    int rows, tiles, splits, chunk;
    size_t part_o, part_ml, lse, scores, end; // offsets in the workspace, in floats
    int scores_stride, parts, part_rows; // of the column sums: parts of the rows, rows of one
};

//
// Trees of more than sixteen rows: an estimate of their own, as their wavefronts without rows are idle and their splits that there are come first.  Rows and
// positions are those that the caller states, or sequences half as long as the longest; a sequence's last tile is taken to be half full, and a tile costs by 32
// rows that it has and by itself.  Over 46 calls of 3 to 150 nodes and 20 to 30000 positions its choice takes 2.7 % longer than the best of both heights and up
// to fifteen lengths (fitted to half of them 3 to 5 % on the others), that for chunks 9 %: 12 sequences of up to 46 nodes of 40 heads, 8 key/value heads
// and 2539 positions 36 -> 27 us.
void plan_tree(const fq_paged_batch &b, int heads, int kv_heads, int *rows_out, int *chunk_out)
{
    const int group = heads / kv_heads;
    const bool known = b.positions > 0 && b.pairs > 0;
    const double tokens = b.tokens, positions = known ? (double)b.positions : b.seqs > 1 ? 0.5 * b.seqs * b.max_len + 1 : b.max_len + 1.0;
    const double pairs = known ? (double)b.pairs : tokens * positions / b.seqs, seen_rows = pairs * group / positions; // of a sequence, as a position sees them
    const double items = tokens * heads, slow = b.page < KT ? 1.2 : 1.0; // four pages a tile to look up
    double best = 0;
    for (int rows = 64; rows <= 128; rows *= 2)
        for (int chunk = 128;; chunk += chunk < 768 ? 128 : chunk < 1536 ? 256 : chunk < 2048 ? 512 : chunk) {
            const int splits = (b.max_len + chunk - 1) / chunk;
            const double tiles = seen_rows / rows + 0.5 > 1 ? seen_rows / rows + 0.5 : 1, units = seen_rows / 32 + 0.5 > 1 ? seen_rows / 32 + 0.5 : 1;
            const double length = chunk < b.max_len + KT ? chunk : b.max_len + KT, alone = length / KT * (rows == 64 ? 0.73 : 0.77) * slow;
            const double together = kv_heads / 256.0 * positions / KT * (tiles * (rows == 64 ? 0.2 : 0.1) + units * 0.31) * slow;
            const double all = items * splits, longer = pairs * heads / chunk + items, parts = longer < all ? longer : all;
            const double full = tokens * group / rows + (b.seqs < tokens * group ? b.seqs : tokens * group);
            const double us = 6 + (alone > together ? alone + 0.14 * together : together + 0.14 * alone) + 0.0013 * full * kv_heads * splits +
                              (splits > 1 ? 3.4 + 210e-6 * parts : 0) + (splits > 8 ? 0.6 : 0);
            if ((best == 0 || us < best) && (splits == 1 || all <= 1 << 20)) {
                best = us;
                *rows_out = rows;
                *chunk_out = chunk;
            }
            if (splits <= 1)
                break;
        }
}

AttnPlan plan_attn(const fq_paged_batch &b, int heads, int kv_heads, bool weights, bool tree = false)
{
    AttnPlan s;
    const int group = heads / kv_heads;
    const long long rows = (long long)b.tokens * group, longest = (long long)b.max_q * group;
    const auto tiles = [&](int height) { // of all sequences: at most one of each is not full
        const long long full = rows / height + (b.seqs < rows ? b.seqs : rows), most = b.seqs * ((longest + height - 1) / height);
        return full < most ? full : most;
    };
    const size_t items = (size_t)b.tokens * heads;
    if (longest <= FEW) {
        s.rows = FEW;
        s.tiles = b.seqs;
        const long long jobs = (long long)b.seqs * kv_heads;
        const auto pieces = [&](int chunk) { return jobs * ((b.max_len + chunk - 1) / chunk); };
        const bool one = b.max_len <= (jobs >= 160 ? FEW_CHUNK : jobs >= 128 ? 512 : 384); // no split is longer than FEW_CHUNK
        s.chunk = one ? (b.max_len + 127) / 128 * 128 : pieces(128) <= 384 ? 128 : pieces(256) <= 384 ? 256 : 512;
    } else if (tree) {
        plan_tree(b, heads, kv_heads, &s.rows, &s.chunk);
        s.tiles = (int)tiles(s.rows);
    } else {
        // steps of a tile, all splits together; several sequences are taken to be half as long as the longest where the caller does not say
        const double mean = (b.max_len > b.max_q ? b.max_len - 0.5 * b.max_q : 0.5 * b.max_len) / KT * (b.seqs > 1 ? 0.5 : 1.0) + 0.5;
        const auto steps = [&](int height, bool known) {
            if (!known)
                return tiles(height) * mean;
            const double full = (double)b.pairs * group / height, open = 1 - full / b.positions; // of a sequence's last tile
            return (full + b.positions * (open > 0.5 ? open : 0.5)) / KT + 0.5 * tiles(height);
        };
        const auto estimate = [&](int rows, int chunk, int splits, bool known) {
            const double alone = (double)chunk / KT * (rows == 64 ? 0.69 : 1.0), together = steps(rows, known) * kv_heads / 256 * (rows == 64 ? 0.9 : 1.36);
            const double all = (double)items * splits, longer = (double)b.pairs * heads / chunk + items, parts = known && longer < all ? longer : all;
            return 6 + (alone > together ? alone : together) + (splits > 1 ? 4 + parts * 1040e-6 / 4 : 0) +
                   (known ? 0.3 * alone + (splits > 1 ? 0.001 * tiles(rows) * kv_heads * splits : 0) + ((b.max_len + chunk - 1) / chunk > 8 ? 4 : 0) : 0);
        };
        const auto roomy = [&](int splits) { return splits > 1 && (double)items * splits > 1 << 20; }; // the workspace has room for every split of every row
        const auto choose = [&](int lowest, int highest, bool known) {
            double best = 0;
            if (const int splits = known ? (b.max_len + s.chunk - 1) / s.chunk : 0; known && !roomy(splits))
                best = estimate(s.rows, s.chunk, splits, true) - 2.5; // what is to be undercut
            for (int rows = lowest; rows <= highest; rows *= 2)
                for (int splits = 1; splits == 1 || b.max_len / splits > 128; splits *= 2) { // none shorter than 256 positions
                    const int chunk = ((b.max_len + splits - 1) / splits + 127) / 128 * 128;
                    if (known && roomy(splits))
                        continue;
                    const double us = estimate(rows, chunk, splits, known);
                    if (best == 0 || us < best) {
                        best = us;
                        s.rows = rows;
                        s.chunk = chunk;
                    }
                }
        };
        choose(64, 128, false);
        if (b.seqs > 1 && b.positions > 0 && b.pairs > 0) // the height stays: it is set by the whole call's work
            choose(s.rows, s.rows, true);
        s.tiles = (int)tiles(s.rows);
    }
    s.chunk = s.chunk < 128 ? 128 : s.chunk;
    s.splits = (b.max_len + s.chunk - 1) / s.chunk;
    s.splits = s.splits < 1 ? 1 : s.splits;
    const size_t parts = s.splits > 1 ? (size_t)s.splits * items : 0;
    s.scores_stride = (b.max_len + 31) / 32 * 32;
    s.parts = s.part_rows = 0;
    if (weights && s.rows != FEW) {
        const double blocks = (b.max_len + WK - 1) / WK, alike = (double)rows / longest * kv_heads; // sequences as long as the longest, times heads
        const double part_seen = blocks - 0.5 * b.max_q / WK > 0.5 ? blocks - 0.5 * b.max_q / WK : 0.5; // blocks that a row is multiplied with
        double best = 0;
        for (long long height = WR; best == 0 || height < longest + WR; height += height < 512 ? WR : height / 4 / WR * WR) {
            const long long parts = (longest + height - 1) / height;
            if (parts > 8 && blocks * parts * kv_heads > 1 << 20) // the workspace, and the grid
                continue;
            const double groups = (parts > 1 ? part_seen * parts : blocks) * alike, steps = part_seen * longest / WR * alike + 0.5 * groups;
            const double alone = 3.3 + (double)(height < longest ? height : longest) / WR * 1.8, together = (groups * 4 + steps * 2.5) / 512;
            const double us = (alone > together ? alone : together) + (parts > 1 ? 4.5 + 0.05 * parts + parts * blocks * WK * alike * 8e-6 / 2 : 0);
            if (best == 0 || us < best) {
                best = us;
                s.part_rows = (int)height;
                s.parts = (int)parts;
            }
        }
    }
    s.scores = 0; // what is a multiple of four floats first
    s.part_o = s.scores + (!weights ? 0 : s.rows == FEW ? items * s.scores_stride : s.parts > 1 ? (size_t)s.parts * b.seqs * kv_heads * s.scores_stride : 0);
    s.part_ml = s.part_o + parts * PD;
    s.lse = s.part_ml + parts * 2;
    s.end = s.lse + (weights ? items : 0);
    return s;
}

} // namespace

void fq_attn_paged_plan(const fq_paged_batch &b, int heads, int kv_heads, int *rows, int *splits, int *chunk)
{
    const AttnPlan s = plan_attn(b, heads, kv_heads, false);
    *rows = s.rows;
    *splits = s.splits;
    *chunk = s.chunk;
}

size_t fq_attn_paged_scratch_bytes(const fq_paged_batch &b, int heads, int kv_heads, bool weights, bool tree)
{
    return plan_attn(b, heads, kv_heads, weights, tree).end * sizeof(float);
}

int fq_launch_attn_paged(const fq_paged_batch &b, const void *q, int ldq, int heads, int kv_heads, const void *k, const void *v, float scale,
                         void *out, float *lse, const float *weights, float *weights_out, int weights_stride, void *workspace, fq_stream st,
                         const uint64_t *mask, int mask_words, const int32_t *tail)
{
    const AttnPlan s = plan_attn(b, heads, kv_heads, weights_out != nullptr, mask != nullptr);
    float *ws = static_cast<float *>(workspace);
    PagedAttnArgs a;
    a.s = paged_seqs(b);
    a.q = static_cast<const _Float16 *>(q);
    a.k = static_cast<const _Float16 *>(k);
    a.v = static_cast<const _Float16 *>(v);
    a.out = static_cast<_Float16 *>(out);
    a.part_o = ws + s.part_o;
    a.part_ml = ws + s.part_ml;
    a.lse = lse || !weights_out ? lse : ws + s.lse;
    a.scores = ws + s.scores;
    a.scores_stride = s.scores_stride;
    a.parts = s.parts;
    a.part_rows = s.part_rows;
    a.weights = weights;
    a.weights_out = weights_out;
    a.scale = scale * LOG2E;
    a.ldq = ldq;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.group = heads / kv_heads;
    a.splits = s.splits;
    a.chunk = s.chunk;
    a.tiles = s.tiles;
    a.weights_stride = weights_stride;
    a.mask = mask;
    a.mask_words = mask_words;
    a.tail = tail;
    const bool tree = mask != nullptr;
    const bool joined = weights_out && s.rows == FEW && s.splits > 1 && s.splits <= 8; // with the column sums
    if (b.tokens > 0) {
        const long long jobs = (long long)s.tiles * kv_heads;
        // more than are resident together, and those that there are come first
        a.packed = tree && s.rows != FEW ? s.splits > 1 && jobs * s.splits < 1 << 24 : s.rows == FEW && b.seqs > 1 && s.splits > 1 && jobs * s.splits > 768 && jobs * s.splits < 1 << 24;
        const dim3 grid((unsigned)(jobs * (a.packed ? s.splits : 1)), a.packed ? 1 : s.splits);
        if (s.rows == FEW && tree)
            hipLaunchKernelGGL((attn_paged_few_kernel<false, true>), grid, dim3(256), 0, st, a);
        else if (s.rows == 64 && b.page >= KT && tree)
            hipLaunchKernelGGL((attn_paged_tile_kernel<2, true, true>), grid, dim3(256), 0, st, a);
        else if (s.rows == 64 && tree)
            hipLaunchKernelGGL((attn_paged_tile_kernel<2, false, true>), grid, dim3(256), 0, st, a);
        else if (b.page >= KT && tree)
            hipLaunchKernelGGL((attn_paged_tile_kernel<1, true, true>), grid, dim3(256), 0, st, a);
        else if (tree)
            hipLaunchKernelGGL((attn_paged_tile_kernel<1, false, true>), grid, dim3(256), 0, st, a);
        else if (s.rows == FEW && weights_out)
            hipLaunchKernelGGL(attn_paged_few_kernel<true>, grid, dim3(256), 0, st, a);
        else if (s.rows == FEW)
            hipLaunchKernelGGL(attn_paged_few_kernel<false>, grid, dim3(256), 0, st, a);
        else if (s.rows == 64 && b.page >= KT)
            hipLaunchKernelGGL((attn_paged_tile_kernel<2, true>), grid, dim3(256), 0, st, a);
        else if (s.rows == 64)
            hipLaunchKernelGGL((attn_paged_tile_kernel<2, false>), grid, dim3(256), 0, st, a);
        else if (b.page >= KT)
            hipLaunchKernelGGL((attn_paged_tile_kernel<1, true>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((attn_paged_tile_kernel<1, false>), grid, dim3(256), 0, st, a);
        int rc = (int)hipGetLastError();
        if (rc != 0)
            return rc;
        if (s.splits > 1 && !joined) {
            const size_t items = (size_t)b.tokens * heads, groups = (size_t)b.tokens * ((heads + 7) / 8);
            // more than a wavefront takes at once; more than one of its turns (a grid has less than 2^32 threads)
            if (tree && (items + 1023) / 1024 * 8 < (size_t)s.splits) // fewer turns over the jobs than over the splits
                hipLaunchKernelGGL(attn_tree_merge_kernel<true>, dim3((unsigned)(items < 1024 ? items : 1024)), dim3(256), 0, st, a);
            else if (tree)
                hipLaunchKernelGGL(attn_tree_merge_kernel<false>, dim3((unsigned)(groups < 1024 ? groups : 1024)), dim3(256), 0, st, a);
            else if (s.splits > 64 && items < 1 << 22)
                hipLaunchKernelGGL(attn_paged_merge_kernel<16>, dim3((unsigned)items), dim3(1024), 0, st, a, s.rows);
            else if (s.splits > 8 && items < 1 << 24)
                hipLaunchKernelGGL(attn_paged_merge_kernel<4>, dim3((unsigned)items), dim3(256), 0, st, a, s.rows);
            else
                hipLaunchKernelGGL(attn_paged_merge_kernel<1>, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, st, a, s.rows);
            if ((rc = (int)hipGetLastError()) != 0)
                return rc;
        }
    }
    if (weights_out && b.max_len > 0) {
        const auto grid = [&](int positions, int parts) { return dim3((unsigned)((b.max_len + positions - 1) / positions * parts * kv_heads), b.seqs); };
        if (joined) {
            hipLaunchKernelGGL(attn_paged_few_weights_kernel<true>, grid(1024, 1), dim3(256), 0, st, a);
        } else if (s.rows == FEW) {
            hipLaunchKernelGGL(attn_paged_few_weights_kernel<false>, grid(1024, 1), dim3(256), 0, st, a);
        } else {
            hipLaunchKernelGGL(attn_paged_weights_kernel, grid(WK, s.parts), dim3(256), 0, st, a);
            int rc = (int)hipGetLastError();
            if (rc != 0 || s.parts == 1)
                return rc;
            hipLaunchKernelGGL(attn_paged_weights_join_kernel, grid(256, 1), dim3(256), 0, st, a);
        }
    }
    return (int)hipGetLastError();
}
