// Around the attention over a paged cache: what writes its rows and what thins them out.  Bound by the bytes they move, or by the launch.
#include "fq_paged.h"

namespace {

// ------------------------------------------------------- norm, rotation, write
// Per token and head of 128 (q and k): x / sqrt(mean x^2 + eps) * gain where there is a gain, then the adjacent pairs turned by the
// position's angles; fp32 throughout, one rounding.  v is copied.  Sixteen lanes hold a row, eight values each, so a sum of squares is four steps
// across lanes and every load and store 16 bytes a lane.  Bound by HBM (10400 tokens of 32 and 8 heads: 261 MB in 48 us, 5.4 TB/s), a token by the launch.
struct RopeArgs {
    const _Float16 *q, *k, *v;
    const int *positions, *slots;
    const float *rope;
    const _Float16 *q_gain, *k_gain;
    _Float16 *q_out, *k_pages, *v_pages;
    int ldq, ldk, ldv, tokens, heads, kv_heads, rope_rows, page_log2, slots_end;
    float eps;
};

constexpr int ROPE_ROWS = 16; // rows a workgroup of 256 threads

__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeArgs p)
{
    const int m = blockIdx.y, r = threadIdx.x & 15;
    const int row = blockIdx.x * ROPE_ROWS + (threadIdx.x >> 4); // head of q, then of k, then of v
    if (row >= p.heads + 2 * p.kv_heads)
        return;
    const bool is_q = row < p.heads, is_v = row >= p.heads + p.kv_heads;
    const int head = is_q ? row : (is_v ? row - p.heads - p.kv_heads : row - p.heads);
    const _Float16 *src = (is_q ? p.q + (size_t)m * p.ldq : is_v ? p.v + (size_t)m * p.ldv : p.k + (size_t)m * p.ldk) + head * PD + 8 * r;
    h8 x = *reinterpret_cast<const h8 *>(src);
    if (!is_v) {
        const int pos = min(max(p.positions[m], 0), p.rope_rows - 1);
        const f4 lo = *reinterpret_cast<const f4 *>(p.rope + (size_t)pos * PD + 8 * r);
        const f4 hi = *reinterpret_cast<const f4 *>(p.rope + (size_t)pos * PD + 8 * r + 4);
        const _Float16 *gain = is_q ? p.q_gain : p.k_gain;
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            t[e] = (float)x[e];
        if (gain) {
            const h8 g = *reinterpret_cast<const h8 *>(gain + 8 * r);
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                ss = fmaf(t[e], t[e], ss);
#pragma unroll
            for (int o = 1; o < 16; o <<= 1)
                ss += __shfl_xor(ss, o, 64);
            const float inv = 1.0f / sqrtf(ss * (1.0f / PD) + p.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                t[e] = t[e] * inv * (float)g[e];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = i < 2 ? lo[2 * i] : hi[2 * i - 4], s = i < 2 ? lo[2 * i + 1] : hi[2 * i - 3];
            x[2 * i] = (_Float16)(t[2 * i] * c - t[2 * i + 1] * s);
            x[2 * i + 1] = (_Float16)(t[2 * i] * s + t[2 * i + 1] * c);
        }
    }
    if (is_q) {
        *reinterpret_cast<h8 *>(p.q_out + ((size_t)m * p.heads + head) * PD + 8 * r) = x;
        return;
    }
    const int slot = p.slots[m];
    if (slot < 0 || slot >= p.slots_end)
        return; // a token that is not cached
    const size_t at = (((size_t)(slot >> p.page_log2) * p.kv_heads + head) << p.page_log2) | (size_t)(slot & ((1 << p.page_log2) - 1));
    *reinterpret_cast<h8 *>((is_v ? p.v_pages : p.k_pages) + at * PD + 8 * r) = x;
}

// ------------------------------------------------------------------- eviction
// Of a head's len positions the last `recent` stay, and of the others the keep - recent that weigh most (equal weights: the lower
// position).  The weight that the last one kept has is found eight bits at a time (radix selection over keys that order like the weights), then
// one pass in order numbers what stays.  Selecting is bound by latency: the length, the weights, a barrier and a scan of 256 counts a digit.  Each
// wavefront has consecutive positions, few enough to stay in registers, and scans the counts for itself.  Beyond 16384 positions they are read again for every digit
// by the one workgroup of a head (100003 positions of 8 heads, 4096 stay: 117 us, and 8 for the copy).
//
// Where a call has few heads, a head's rows that stay are dealt to several workgroups, each of which selects for itself and then copies its share:
// one launch, the whole chip copying (caches cold, one launch against two: one sequence of 611 positions, 32 heads, 512 stay 11.4 against 14.0 us in the first
// form of both and 8.8 now; 2000, 8 heads, half stay 8.7 / 10.0; 9000, 8 heads, 4096 stay 20.5 / 22.6).  Of many heads the copy is a launch of its own (64
// sequences of 1000, 32 heads 235 / 222; 15 of 9000, 8 heads 129 / 114); level at 64 heads of 9000 positions and at 512 of up to 1024.
struct EvictArgs {
    PagedSeqs s;
    const _Float16 *k, *v;
    const float *weights;
    _Float16 *k_out, *v_out;
    const int *dst_table;
    int *kept, *new_len;
    float *weights_out;
    int kv_heads, weights_stride, weights_out_stride, keep, recent, dst_stride, dst_pages, share;
};

// Larger weight, larger key; -0 and 0 alike; NaN above everything, as it says nothing against its position.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w)
        return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the lanes up to this one: inside rows of sixteen lanes, then row ends handed on.
__device__ __forceinline__ int lanes_upto(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false); // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false); // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false); // row_bcast:31 into rows 2 and 3
    return v;
}

// Copies the rows that stay, in order, sixteen lanes a row of keys and its row of values.  Bound by HBM (15 sequences, 8 heads, about 4096 rows each: 510 MB
// in 101 us, 5.0 TB/s).
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs p)
{
    const int head = blockIdx.y, b = blockIdx.z, r = threadIdx.x & 15;
    const int j = blockIdx.x * 16 + (threadIdx.x >> 4);
    const int m = min(min(max(p.s.seq_len[b], 0), p.s.max_len), p.keep);
    if (j >= m)
        return;
    const int t = max(p.kept[((size_t)b * p.kv_heads + head) * p.keep + j], 0);
    const size_t from = pool_row(p.s.table, p.s.table_stride, p.s.page_log2, p.s.pages, p.kv_heads, head, b, t) * PD + 8 * r;
    const size_t to = pool_row(p.dst_table, p.dst_stride, p.s.page_log2, p.dst_pages, p.kv_heads, head, b, j) * PD + 8 * r;
    const h8 k = *reinterpret_cast<const h8 *>(p.k + from), v = *reinterpret_cast<const h8 *>(p.v + from);
    *reinterpret_cast<h8 *>(p.k_out + to) = k;
    *reinterpret_cast<h8 *>(p.v_out + to) = v;
}

constexpr int share_rows(int waves) { return waves == 4 ? 64 : 128; } // the least rows of a share: what the workgroup's threads have in flight

// One workgroup selects among all positions of a head; WAVES wavefronts have up to K blocks of 64 consecutive positions each, whose weights stay in
// registers (LONG: several rounds of them, read again for every digit).
template <int WAVES, int K, bool COPY, bool LONG>
__global__ __launch_bounds__(64 * WAVES) void evict_kernel(EvictArgs p)
{
    // The first digit (sign and seven bits of the exponent) has few values, and additions to one place follow one another: where a workgroup has
    // thousands of keys it is counted in eight places, by lane (16000 positions of a head 24.3 -> 19.2 us, 2000 of 8 heads 10.3 -> 10.0).
    constexpr int THREADS = 64 * WAVES, ROUND = THREADS * K, PLACES = WAVES > 4 ? 8 : 1;
    static_assert(ROUND <= 16384, "counts in halves of 32 bits, positions in 16");
    __shared__ __align__(16) int hist[4][256], first_digit[PLACES > 1 ? 256 : 1][8];
    __shared__ int of_wave[2][WAVES]; // what stays of a wavefront's positions: keys above the last one kept, equal ones in the upper half
    __shared__ short stays[COPY ? ROUND : 1];
    __shared__ int page_of[2][COPY ? ROUND / 16 : 1]; // pages read and written; asked for beside the selection
    const int head = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool writes = blockIdx.x == 0; // what is written once a head
    const int most = min(max(p.s.seq_len[b], 0), p.s.max_len), len = LONG ? most : min(most, ROUND);
    const int m = min(len, p.keep), old = len - min(p.recent, m), need = m - (len - old);
    const int j0 = COPY ? blockIdx.x * p.share : 0, j1 = COPY ? min(j0 + p.share, m) : 0;
    if (!writes && j0 >= m)
        return;
    const int blocks = LONG || K <= 4 ? K : min((len + THREADS - 1) / THREADS, K); // of 64 positions a wavefront
    const int first = 64 * blocks * wave + lane;
    const float *w = p.weights + ((size_t)b * p.kv_heads + head) * p.weights_stride;
    float held[K];
    uint32_t key[K];
    auto load = [&](int r0) {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i < blocks) {
                const int t = r0 + first + 64 * i;
                held[i] = t < len ? w[t] : 0.f;
            }
    };
    auto keys = [&] {
#pragma unroll
        for (int i = 0; i < K; ++i)
            key[i] = weight_key(held[i]);
    };
    if constexpr (!LONG)
        load(0);
    if (tid < 256)
        *reinterpret_cast<int4 *>(&hist[tid >> 6][4 * lane]) = int4{0, 0, 0, 0};
    if constexpr (PLACES > 1)
        for (int i = tid; i < 512; i += THREADS)
            *reinterpret_cast<int4 *>(&first_digit[i >> 1][4 * (i & 1)]) = int4{0, 0, 0, 0};
    if constexpr (COPY)
        for (int i = tid; i < ROUND / 8; i += THREADS) {
            const int dst = i >= ROUND / 16, at = i & (ROUND / 16 - 1);
            if (at << p.s.page_log2 >= ROUND)
                continue;
            const int page = dst ? p.dst_table[(size_t)b * p.dst_stride + min(at, p.dst_stride - 1)] : p.s.table[(size_t)b * p.s.table_stride + min(at, p.s.table_stride - 1)];
            page_of[dst][at] = min(max(page, 0), (dst ? p.dst_pages : p.s.pages) - 1);
        }
    if constexpr (!LONG)
        keys();
    const bool all = need >= old, none = need <= 0;
    uint32_t prefix = 0;
    int left = need; // how many of the keys that match the prefix so far are kept
    __syncthreads();
    if (!all && !none) { // the same in every thread, and so is the loop
        for (int d = 0; d < 4; ++d) {
            const int shift = 24 - 8 * d;
            const uint32_t mask = d == 0 ? 0u : 0xffffffffu << (shift + 8);
            for (int r0 = 0; r0 < (LONG ? old : 1); r0 += ROUND) {
                if constexpr (LONG) {
                    load(r0);
                    keys();
                }
#pragma unroll
                for (int i = 0; i < K; ++i)
                    if (i < blocks) {
                        if (r0 + first + 64 * i < old && (key[i] & mask) == prefix)
                            atomicAdd(PLACES > 1 && d == 0 ? &first_digit[key[i] >> 24][lane & 7] : &hist[d][(key[i] >> shift) & 255], 1);
                    }
            }
            __syncthreads();
            if (PLACES > 1 && d == 0) {
                if (tid < 256) {
                    const int4 x = *reinterpret_cast<const int4 *>(&first_digit[tid][0]), y = *reinterpret_cast<const int4 *>(&first_digit[tid][4]);
                    hist[0][tid] = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w;
                }
                __syncthreads();
            }
            const int4 h = *reinterpret_cast<const int4 *>(&hist[d][252 - 4 * lane]); // four digits a lane, from the highest down
            const int count[4] = {h.w, h.z, h.y, h.x};
            int above = lanes_upto(h.x + h.y + h.z + h.w) - (h.x + h.y + h.z + h.w), digit = -1, rest = 0, size = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (above < left && left <= above + count[i]) { // one lane and digit
                    digit = 255 - 4 * lane - i;
                    rest = left - above;
                    size = count[i];
                }
                above += count[i];
            }
            const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(digit >= 0));
            prefix |= (uint32_t)__builtin_amdgcn_readlane(digit, at) << shift;
            left = __builtin_amdgcn_readlane(rest, at);
            if (left == __builtin_amdgcn_readlane(size, at)) { // all of them: what is at least this prefix stays (and not everything does, so it is not 0)
                prefix -= 1;
                left = 0;
                break;
            }
        }
    }
    // in order: a key above the last one kept stays, equal ones while they last
    int *kept = p.kept + ((size_t)b * p.kv_heads + head) * p.keep;
    float *wo = p.weights_out && writes ? p.weights_out + ((size_t)b * p.kv_heads + head) * p.weights_out_stride : nullptr;
    const unsigned long long lower = (1ull << lane) - 1;
    int gt_rounds = 0, eq_rounds = 0, parity = 0; // of the rounds before
    for (int r0 = 0; r0 < (LONG ? len : 1); r0 += ROUND, parity ^= 1) {
        if constexpr (LONG) {
            load(r0);
            keys();
        }
        unsigned long long gts[K], eqs[K];
        int found = 0;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int t = r0 + first + 64 * i;
            gts[i] = eqs[i] = 0;
            if (i < blocks) {
                gts[i] = __builtin_amdgcn_ballot_w64(t < len && (t >= old || all || (!none && key[i] > prefix)));
                eqs[i] = __builtin_amdgcn_ballot_w64(t < old && !all && !none && key[i] == prefix);
                found += (int)__popcll(gts[i]) | (int)__popcll(eqs[i]) << 16;
            }
        }
        if (lane == 0)
            of_wave[parity][wave] = found;
        __syncthreads();
        int before = 0, whole = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            before += i < wave ? of_wave[parity][i] : 0;
            whole += of_wave[parity][i];
        }
        int gt_before = gt_rounds + (before & 0xffff), eq_before = eq_rounds + (before >> 16);
        gt_rounds += whole & 0xffff;
        eq_rounds += whole >> 16;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i < blocks) {
                const int t = r0 + first + 64 * i, e = eq_before + (int)__popcll(eqs[i] & lower);
                const int at = gt_before + (int)__popcll(gts[i] & lower) + min(e, left);
                if (((gts[i] >> lane & 1) || ((eqs[i] >> lane & 1) && e < left)) && at < m) {
                    if constexpr (COPY)
                        stays[at] = (short)t;
                    if (writes)
                        kept[at] = t;
                    if (wo)
                        wo[at] = held[i];
                }
                gt_before += (int)__popcll(gts[i]);
                eq_before += (int)__popcll(eqs[i]);
            }
    }
    if (writes) {
        if (head == 0 && tid == 0)
            p.new_len[b] = m;
        for (int t = m + tid; t < p.keep; t += THREADS)
            kept[t] = -1;
    }
    if constexpr (COPY) {
        constexpr int U = share_rows(WAVES) / (THREADS / 16); // rows that sixteen lanes have in flight
        __syncthreads();
        const auto row_at = [&](int dst, int t) {
            return (((((size_t)page_of[dst][t >> p.s.page_log2] * p.kv_heads + head) << p.s.page_log2) | (size_t)(t & ((1 << p.s.page_log2) - 1)))) * PD + 8 * (tid & 15);
        };
        for (int j = j0 + (tid >> 4); j < j1; j += U * (THREADS / 16)) {
            h8 k[U], v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) { // behind the last one that one again
                const size_t from = row_at(0, stays[min(j + THREADS / 16 * i, j1 - 1)]);
                k[i] = *reinterpret_cast<const h8 *>(p.k + from);
                v[i] = *reinterpret_cast<const h8 *>(p.v + from);
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (j + THREADS / 16 * i < j1) {
                    const size_t to = row_at(1, j + THREADS / 16 * i);
                    *reinterpret_cast<h8 *>(p.k_out + to) = k[i];
                    *reinterpret_cast<h8 *>(p.v_out + to) = v[i];
                }
        }
    }
}

// Whether the copy went with it.
template <int WAVES, int K>
bool launch_evict(EvictArgs &a, int most, int kv_heads, int seqs, fq_stream st)
{
    constexpr int MANY = WAVES == 4 ? 512 : 64, GROUPS = WAVES == 4 ? 1024 : 256; // heads; workgroups of the one launch, about
    const long long heads = (long long)kv_heads * seqs;
    if (heads >= MANY) {
        hipLaunchKernelGGL((evict_kernel<WAVES, K, false, false>), dim3(1, kv_heads, seqs), dim3(64 * WAVES), 0, st, a);
        return false;
    }
    const int shares = (int)(GROUPS / heads), even = (most + shares - 1) / shares, step = share_rows(WAVES);
    a.share = even < step ? step : (even + step - 1) / step * step;
    hipLaunchKernelGGL((evict_kernel<WAVES, K, true, false>), dim3(most > a.share ? (most + a.share - 1) / a.share : 1, kv_heads, seqs), dim3(64 * WAVES), 0, st, a);
    return true;
}

} // namespace

int fq_launch_qk_norm_rope(const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, int tokens, int heads, int kv_heads,
                           const int32_t *positions, const int32_t *slots, const float *rope, int rope_rows, const void *q_gain,
                           const void *k_gain, float eps, void *q_out, void *k_pages, void *v_pages, int page_log2, int pages, fq_stream st)
{
    RopeArgs a;
    a.q = static_cast<const _Float16 *>(q);
    a.k = static_cast<const _Float16 *>(k);
    a.v = static_cast<const _Float16 *>(v);
    a.positions = positions;
    a.slots = slots;
    a.rope = rope;
    a.q_gain = static_cast<const _Float16 *>(q_gain);
    a.k_gain = static_cast<const _Float16 *>(k_gain);
    a.q_out = static_cast<_Float16 *>(q_out);
    a.k_pages = static_cast<_Float16 *>(k_pages);
    a.v_pages = static_cast<_Float16 *>(v_pages);
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.tokens = tokens;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.rope_rows = rope_rows;
    a.page_log2 = page_log2;
    a.slots_end = pages << page_log2;
    a.eps = eps;
    for (int m0 = 0; m0 < tokens; m0 += 65535) { // the second extent of a grid ends there
        RopeArgs part = a;
        part.tokens = tokens - m0 < 65535 ? tokens - m0 : 65535;
        part.q += (size_t)m0 * ldq;
        part.k += (size_t)m0 * ldk;
        part.v += (size_t)m0 * ldv;
        part.positions += m0;
        part.slots += m0;
        part.q_out += (size_t)m0 * heads * PD;
        hipLaunchKernelGGL(qk_norm_rope_kernel, dim3((heads + 2 * kv_heads + ROPE_ROWS - 1) / ROPE_ROWS, part.tokens), dim3(256), 0, st, part);
        if (int rc = (int)hipGetLastError())
            return rc;
    }
    return 0;
}

int fq_launch_cache_evict(const fq_paged_batch &batch, const void *k, const void *v, int kv_heads, const float *weights, int weights_stride, int keep,
                          int recent, const int32_t *dst_table, int dst_stride, int dst_pages, void *k_out, void *v_out, int32_t *kept,
                          int32_t *new_len, float *weights_out, int weights_out_stride, fq_stream st)
{
    EvictArgs a;
    a.s = paged_seqs(batch);
    a.k = static_cast<const _Float16 *>(k);
    a.v = static_cast<const _Float16 *>(v);
    a.weights = weights;
    a.k_out = static_cast<_Float16 *>(k_out);
    a.v_out = static_cast<_Float16 *>(v_out);
    a.dst_table = dst_table;
    a.kept = kept;
    a.new_len = new_len;
    a.weights_out = weights_out;
    a.kv_heads = kv_heads;
    a.weights_stride = weights_stride;
    a.weights_out_stride = weights_out_stride;
    a.keep = keep;
    a.recent = recent;
    a.dst_stride = dst_stride;
    a.dst_pages = dst_pages;
    const int most = batch.max_len < keep ? batch.max_len : keep;
    bool copied = false;
    if (batch.max_len <= 1024)
        copied = launch_evict<4, 4>(a, most, kv_heads, batch.seqs, st);
    else if (batch.max_len <= 4096)
        copied = launch_evict<16, 4>(a, most, kv_heads, batch.seqs, st);
    else if (batch.max_len <= 16384)
        copied = launch_evict<16, 16>(a, most, kv_heads, batch.seqs, st);
    else
        hipLaunchKernelGGL((evict_kernel<16, 16, false, true>), dim3(1, kv_heads, batch.seqs), dim3(1024), 0, st, a);
    if (int rc = (int)hipGetLastError())
        return rc;
    if (copied || most == 0)
        return 0;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((most + 15) / 16, kv_heads, batch.seqs), dim3(256), 0, st, a);
    return (int)hipGetLastError();
}
