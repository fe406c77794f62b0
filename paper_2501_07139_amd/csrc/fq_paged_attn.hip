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
// operand of O^T = V^T . P^T as it stands.  The weights are fp16 (their sum and lse are of the unrounded fp32 ones): an error of at most
// 2^-11 of each term, as the output's own rounding.  V^T comes from row-major values through the transposing LDS read.
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
    float scale;              // times log2(e): scores are powers of 2
    int ldq, heads, kv_heads, group, splits, chunk, tiles, weights_stride;
};

// A tile of rows of one sequence and key/value head.
struct RowTile {
    SeqRange s;
    int b, row0, rows, seen; // first row, rows of the sequence and head, positions that the tile's last row sees
};

// Tile `tile` of TR rows, counted over the sequences; rows < 0 where there is none.  Every wavefront scans the sequences' tile counts.
template <int TR>
__device__ __forceinline__ RowTile find_tile(const PagedAttnArgs &p, int tile)
{
    const int lane = threadIdx.x & 63;
    RowTile r;
    r.rows = -1;
    int base = 0;
    for (int i = 0; i < p.s.seqs; i += 64) {
        int count = 0;
        if (i + lane < p.s.seqs)
            count = (seq_range(p.s, i + lane).n * p.group + TR - 1) / TR;
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
            r.row0 = (tile - base - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(count, at))) * TR;
            r.s = seq_range(p.s, r.b);
            r.rows = r.s.n * p.group;
            const int last = min(r.row0 + TR, r.rows) - 1;
            r.seen = max(min(r.s.len - r.s.n + last / p.group + 1, r.s.len), 0);
            return r;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return r;
}

typedef short s4v __attribute__((ext_vector_type(4)));

// Four halves of one column from four consecutive rows: lane j of sixteen names the 8 bytes of row j / 4, columns 4 (j % 4)... of a
// 4 x 16 block and gets column j of it.
__device__ __forceinline__ h4 lds_column(const _Float16 *at)
{
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v *)(at)));
}

// ------------------------------------------------- up to sixteen rows a tile
// Four wavefronts, 32 positions of every 128 each: keys straight into registers as MFMA operands, values through a part of LDS of the
// wavefront's own (no barrier in the loop), and one merge of the four at the end.  Bound by the read of the cache.
constexpr int FEW = 16;

__global__ __launch_bounds__(256, 2) void attn_paged_few_kernel(PagedAttnArgs p)
{
    // values of a step: 32 rows of 16 chunks of eight, chunk ch of row r at ch ^ 2 (r % 8), so that the transposing read of sixteen rows by
    // two chunks meets every bank twice; afterwards the wavefronts' outputs
    __shared__ h8 Vs[4][32 * 16];
    __shared__ float ms[4][FEW], ls[4][FEW];
    const int kvh = blockIdx.x % p.kv_heads, split = blockIdx.y;
    const RowTile tile = find_tile<FEW>(p, blockIdx.x / p.kv_heads);
    if (tile.rows < 0)
        return;
    const int begin = split * p.chunk, end = min(tile.seen, begin + p.chunk);
    if (begin >= end && split > 0)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int row = tile.row0 + col, token = min(row, tile.rows - 1) / p.group;
    const int head = kvh * p.group + min(row, tile.rows - 1) - token * p.group;
    const int seen = min(tile.s.len - tile.s.n + token + 1, tile.s.len); // positions this lane's row sees; may be negative
    const int all_seen = max(tile.s.len - tile.s.n + tile.row0 / p.group + 1, 0); // ... that every row of the tile sees

    h8 qb[4];
    {
        const _Float16 *src = p.q + (size_t)(tile.s.first + token) * p.ldq + head * PD + 8 * g;
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
    for (int t0 = begin + 32 * wave; t0 < end; t0 += 128) {
        h8 kk[2][4], vv[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const size_t at = pool_row(p.s.table, p.s.table_stride, p.s.page_log2, p.s.pages, p.kv_heads, kvh, tile.b, t0 + 16 * b) * PD;
#pragma unroll
            for (int s = 0; s < 4; ++s)
                kk[b][s] = *reinterpret_cast<const h8 *>(p.k + at + col * PD + 32 * s + 8 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vv[b][i] = *reinterpret_cast<const h8 *>(p.v + at + (4 * i + g) * PD + 8 * col);
                if (t0 + 16 * b + 4 * i + g >= end) // rows that nobody sees may hold anything, and 0 * NaN is NaN
                    vv[b][i] = h8{};
            }
        }
        f4 st[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            st[b] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s)
                st[b] = mfma16x16x32(kk[b][s], qb[s], st[b]);
        }
        const bool whole = t0 + 32 <= all_seen; // uniform
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float x = st[b][v] * p.scale;
                st[b][v] = whole || t0 + 16 * b + 4 * g + v < seen ? x : -INFINITY;
                top = fmaxf(top, st[b][v]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mnew = fmaxf(mx, top), mref = mnew == -INFINITY ? 0.f : mnew;
        const float alpha = __builtin_amdgcn_exp2f(mx - mref);
        mx = mnew;
        h8 pb;
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = __builtin_amdgcn_exp2f(st[b][v] - mref);
                sum += e;
                pb[4 * b + v] = (_Float16)e;
            }
        l = l * alpha + sum;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * b + 4 * i + g;
                V[r * 16 + (col ^ (2 * (r & 7)))] = vv[b][i];
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const char *at = reinterpret_cast<const char *>(V) + (vbase ^ (db << 5));
            const h4 lo = lds_column(reinterpret_cast<const _Float16 *>(at)), hi = lds_column(reinterpret_cast<const _Float16 *>(at + 4096));
            acc[db] = mfma16x16x32(h8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, pb, acc[db] * alpha);
        }
        __builtin_amdgcn_wave_barrier();
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
    // thread: row col, dimensions 16 db + 4 g of two db's
    const float m = fmaxf(fmaxf(ms[0][col], ms[1][col]), fmaxf(ms[2][col], ms[3][col])), mref = m == -INFINITY ? 0.f : m;
    float w[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_exp2f(ms[i][col] - mref);
        sum += w[i] * ls[i][col];
    }
    if (row >= tile.rows)
        return;
    const bool only = p.splits == 1 || tile.seen <= p.chunk;
    const size_t at = (size_t)(tile.s.first + token) * p.heads + head;
    const size_t part = ((size_t)split * p.s.tokens + tile.s.first + token) * p.heads + head;
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

// Joins the splits of a row: one wavefront each, two dimensions a lane.  Rows of tiles that one split has served are done already.
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(PagedAttnArgs p, int tile_rows)
{
    const int lane = threadIdx.x & 63;
    const int item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); // token * heads + head
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
    const float *ml = p.part_ml + 2 * (size_t)item, *o = p.part_o + (size_t)item * PD + 2 * lane;
    float mx = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
    for (int i = 0; i < live; ++i) {
        const float m2 = ml[2 * i * stride], l2 = ml[2 * i * stride + 1];
        const float mnew = fmaxf(mx, m2), mref = mnew == -INFINITY ? 0.f : mnew;
        const float s1 = __builtin_amdgcn_exp2f(mx - mref), s2 = __builtin_amdgcn_exp2f(m2 - mref);
        l = l * s1 + l2 * s2;
        a0 = a0 * s1 + o[i * stride * PD] * s2;
        a1 = a1 * s1 + o[i * stride * PD + 1] * s2;
        mx = mnew;
    }
    const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
    *reinterpret_cast<h2 *>(p.out + (size_t)item * PD + 2 * lane) = h2{(_Float16)(a0 * inv), (_Float16)(a1 * inv)};
    if (lane == 0 && p.lse)
        p.lse[item] = (mx + log2f(l)) * LN2;
}

// --------------------------------------------------------------- column sums
// w[t] of 64 positions: their keys stay in registers, the rows that see them stream by, sixteen a step and wavefront, and with lse known
// a weight is one exponential.  One workgroup owns its positions: no atomics, the same sums every time.
__global__ __launch_bounds__(256, 2) void attn_paged_weights_kernel(PagedAttnArgs p)
{
    __shared__ float part[4][64];
    const int kvh = blockIdx.x, t0 = blockIdx.y * 64, b = blockIdx.z;
    const SeqRange s = seq_range(p.s, b);
    if (t0 >= s.len)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    h8 kk[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const size_t at = pool_row(p.s.table, p.s.table_stride, p.s.page_log2, p.s.pages, p.kv_heads, kvh, b, t0 + 16 * i) * PD;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            kk[i][k] = *reinterpret_cast<const h8 *>(p.k + at + col * PD + 32 * k + 8 * g);
    }
    float sum[4][4] = {};
    const int rows = s.n * p.group, first = max(t0 - (s.len - s.n), 0) * p.group; // rows ahead see none of the positions
    for (int r0 = first + 16 * wave; r0 < rows; r0 += 64) {
        const int row = r0 + col, token = min(row, rows - 1) / p.group, head = kvh * p.group + min(row, rows - 1) - token * p.group;
        const _Float16 *src = p.q + (size_t)(s.first + token) * p.ldq + head * PD + 8 * g;
        h8 qb[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            qb[k] = *reinterpret_cast<const h8 *>(src + 32 * k);
        const float lse = p.lse[(size_t)(s.first + token) * p.heads + head] * LOG2E;
        const int seen = row < rows ? min(s.len - s.n + token + 1, s.len) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f4 st = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                st = mfma16x16x32(kk[i][k], qb[k], st);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = __builtin_amdgcn_exp2f(st[v] * p.scale - lse);
                sum[i][v] += t0 + 16 * i + 4 * g + v < seen ? e : 0.f;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
#pragma unroll
            for (int o = 1; o < 16; o <<= 1)
                sum[i][v] += __shfl_xor(sum[i][v], o, 64);
            if (col == 0)
                part[wave][16 * i + 4 * g + v] = sum[i][v];
        }
    __syncthreads();
    const int t = t0 + tid;
    if (tid < 64 && t < s.len) {
        const size_t at = ((size_t)b * p.kv_heads + kvh) * p.weights_stride + t;
        const float before = p.weights && t < s.len - s.n ? p.weights[at] : 0.f;
        p.weights_out[at] = before + ((part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]));
    }
}

// Splits of the positions: as many as bring a few workgroups to every CU, none shorter than 256 positions.
struct SplitPlan {
    int tiles, splits, chunk;
};

SplitPlan plan_splits(const fq_paged_batch &b, int heads, int kv_heads)
{
    SplitPlan s;
    const int group = heads / kv_heads;
    // tiles of all sequences: at most one of each sequence is not full
    const long long rows = (long long)b.tokens * group, full = rows / FEW + (b.seqs < rows ? b.seqs : rows);
    const long long most = (long long)b.seqs * (((long long)b.max_q * group + FEW - 1) / FEW);
    s.tiles = (int)(full < most ? full : most);
    const long long jobs = (long long)s.tiles * kv_heads;
    long long splits = jobs > 0 ? 1024 / jobs : 1;
    const long long longest = (b.max_len + 255) / 256;
    splits = splits < 1 ? 1 : (splits > longest ? longest : splits);
    if (splits < 1)
        splits = 1;
    s.chunk = (int)((b.max_len + splits - 1) / splits + 127) / 128 * 128;
    if (s.chunk < 128)
        s.chunk = 128;
    s.splits = (b.max_len + s.chunk - 1) / s.chunk;
    if (s.splits < 1)
        s.splits = 1;
    return s;
}

} // namespace

size_t fq_attn_paged_scratch_bytes(const fq_paged_batch &b, int heads, int kv_heads, bool weights)
{
    const SplitPlan s = plan_splits(b, heads, kv_heads);
    const size_t items = (size_t)b.tokens * heads;
    return (s.splits > 1 ? (size_t)s.splits * items * (PD + 2) * sizeof(float) : 0) + (weights ? items * sizeof(float) : 0);
}

int fq_launch_attn_paged(const fq_paged_batch &b, const void *q, int ldq, int heads, int kv_heads, const void *k, const void *v, float scale,
                         void *out, float *lse, const float *weights, float *weights_out, int weights_stride, void *workspace, fq_stream st)
{
    const SplitPlan s = plan_splits(b, heads, kv_heads);
    const size_t items = (size_t)b.tokens * heads;
    PagedAttnArgs a;
    a.s = paged_seqs(b);
    a.q = static_cast<const _Float16 *>(q);
    a.k = static_cast<const _Float16 *>(k);
    a.v = static_cast<const _Float16 *>(v);
    a.out = static_cast<_Float16 *>(out);
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = a.part_o + (s.splits > 1 ? (size_t)s.splits * items * PD : 0);
    a.lse = lse || !weights_out ? lse : a.part_ml + (s.splits > 1 ? (size_t)s.splits * items * 2 : 0);
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
    if (b.tokens > 0) {
        hipLaunchKernelGGL(attn_paged_few_kernel, dim3(s.tiles * kv_heads, s.splits), dim3(256), 0, st, a);
        int rc = (int)hipGetLastError();
        if (rc != 0)
            return rc;
        if (s.splits > 1) {
            hipLaunchKernelGGL(attn_paged_merge_kernel, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, st, a, FEW);
            if ((rc = (int)hipGetLastError()) != 0)
                return rc;
        }
    }
    if (weights_out && b.max_len > 0)
        hipLaunchKernelGGL(attn_paged_weights_kernel, dim3(kv_heads, (b.max_len + 63) / 64, b.seqs), dim3(256), 0, st, a);
    return (int)hipGetLastError();
}
