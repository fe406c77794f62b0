// Around the attention over a paged cache: what writes its rows and what thins them out.  Bound by the bytes they move, or by the launch.
#include "fq_paged.h"

namespace {

// ------------------------------------------------------- norm, rotation, write
// Per token and head of 128 (q and k): x / sqrt(mean x^2 + eps) * gain where there is a gain, then the adjacent pairs turned by the
// position's angles; fp32 throughout, one rounding.  v is copied.  Sixteen lanes hold a row, eight values each.
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
// position).  Selecting kernel, one workgroup per (sequence, head): the weight that the last one kept has is found eleven bits at a
// time (radix selection over keys that order like the weights), then one pass in order numbers what stays.
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

constexpr int SEL = 1024, HELD = 16;             // threads; weights a thread keeps in registers: 16384 positions are read once
constexpr int DIGIT = 11, DIGITS = 1 << DIGIT; // three digits of a key, the last of ten bits

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

__global__ __launch_bounds__(SEL) void evict_select_kernel(EvictArgs p)
{
    constexpr int WAVES = SEL / 64;
    __shared__ int hist[DIGITS];
    __shared__ __align__(16) int wave_sum[WAVES];
    __shared__ int found[3];
    __shared__ uint32_t counts[HELD * WAVES]; // of a trip and wavefront: keys above the last one kept, equal ones in the upper half
    const int head = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = min(max(p.s.seq_len[b], 0), p.s.max_len);
    const int m = min(len, p.keep), old = len - min(p.recent, m), need = m - (len - old);
    const float *w = p.weights + ((size_t)b * p.kv_heads + head) * p.weights_stride;
    int *kept = p.kept + ((size_t)b * p.kv_heads + head) * p.keep;
    float *wo = p.weights_out ? p.weights_out + ((size_t)b * p.kv_heads + head) * p.weights_out_stride : nullptr;
    if (head == 0 && tid == 0)
        p.new_len[b] = m;
    float held[HELD];
    uint32_t key[HELD];
    auto load = [&](int t0) { // trips behind the last position are left out here and below (uniform)
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (t0 + SEL * i < len)
                held[i] = w[min(t0 + SEL * i + tid, len - 1)];
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (t0 + SEL * i < len)
                key[i] = weight_key(held[i]);
    };
    const bool once = len <= HELD * SEL; // uniform: the weights are read once
    if (once)
        load(0);
    const bool all = need >= old, none = need <= 0;
    uint32_t prefix = 0;
    int left = need; // how many of the keys that match the prefix so far are kept
    if (!all && !none) {
        for (int shift = 32 - DIGIT; shift > -DIGIT; shift -= DIGIT) { // 21, 10, and the last ten bits
            const int low = max(shift, 0), bits = DIGIT + min(shift, 0);
            for (int d = tid; d < DIGITS; d += SEL)
                hist[d] = 0;
            __syncthreads();
            const uint32_t mask = low + bits == 32 ? 0u : 0xffffffffu << (low + bits);
            for (int t0 = 0; t0 < old; t0 += HELD * SEL) {
                if (!once)
                    load(t0);
#pragma unroll
                for (int i = 0; i < HELD; ++i)
                    if (t0 + SEL * i < old) {
                        if (t0 + SEL * i + tid < old && (key[i] & mask) == prefix)
                            atomicAdd(&hist[(key[i] >> low) & ((1u << bits) - 1)], 1);
                    }
            }
            __syncthreads();
            // thread: two digits, from the highest down; keys of higher digits than these by a scan of the workgroup
            const int d0 = DIGITS - 1 - 2 * tid, h0 = hist[d0], h1 = hist[d0 - 1];
            const int upto = lanes_upto(h0 + h1);
            if (lane == 63)
                wave_sum[wave] = upto;
            __syncthreads();
            int above = upto - h0 - h1;
#pragma unroll
            for (int i = 0; i < WAVES; ++i)
                above += i < wave ? wave_sum[i] : 0;
            if (above < left && left <= above + h0) { // one thread and digit
                found[0] = d0;
                found[1] = left - above;
                found[2] = h0;
            } else if (above + h0 < left && left <= above + h0 + h1) {
                found[0] = d0 - 1;
                found[1] = left - above - h0;
                found[2] = h1;
            }
            __syncthreads();
            prefix |= (uint32_t)found[0] << low;
            left = found[1];
            if (left == found[2]) { // all of them: what is at least this prefix stays (and not everything does, so the prefix is not 0)
                prefix -= 1;
                left = 0;
                break;
            }
        }
    }
    // in order: a key above the last one kept stays, equal ones while they last
    int gt_before = 0, eq_before = 0;
    for (int t0 = 0; t0 < len; t0 += HELD * SEL) {
        if (!once)
            load(t0);
        unsigned long long gts[HELD], eqs[HELD];
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int t = t0 + SEL * i + tid;
            gts[i] = eqs[i] = 0;
            if (t0 + SEL * i < len) {
                gts[i] = __builtin_amdgcn_ballot_w64(t < len && (t >= old || all || (!none && key[i] > prefix)));
                eqs[i] = __builtin_amdgcn_ballot_w64(t < old && !all && !none && key[i] == prefix);
            }
            if (lane == 0)
                counts[WAVES * i + wave] = (uint32_t)__popcll(gts[i]) | (uint32_t)__popcll(eqs[i]) << 16;
        }
        __syncthreads();
        if (tid < 64) { // sums ahead of every entry: four a lane, over the trips' wavefronts in order
            static_assert(HELD * WAVES == 256 && HELD * SEL < 65536, "four entries a lane, sixteen bits a sum");
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = counts[4 * lane + i];
                sum += c[i];
            }
            uint32_t ahead = (uint32_t)lanes_upto((int)sum) - sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                counts[4 * lane + i] = ahead;
                ahead += c[i];
            }
            if (lane == 63)
                found[0] = (int)ahead;
        }
        __syncthreads();
        const unsigned long long lower = (1ull << lane) - 1;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (t0 + SEL * i >= len)
                continue;
            const uint32_t ahead = counts[WAVES * i + wave];
            const int gt = gt_before + (int)(ahead & 0xffffu) + (int)__popcll(gts[i] & lower);
            const int eq = eq_before + (int)(ahead >> 16) + (int)__popcll(eqs[i] & lower);
            const bool is_gt = gts[i] >> lane & 1, is_eq = eqs[i] >> lane & 1;
            const int at = gt + min(eq, left);
            if ((is_gt || (is_eq && eq < left)) && at < m) {
                kept[at] = t0 + SEL * i + tid;
                if (wo)
                    wo[at] = held[i];
            }
        }
        gt_before += found[0] & 0xffff;
        eq_before += (int)((uint32_t)found[0] >> 16);
        __syncthreads();
    }
    for (int t = m + tid; t < p.keep; t += SEL)
        kept[t] = -1;
}

// Copies the rows that stay, in order, sixteen lanes a row of keys and its row of values.
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

// Selection for up to 1024 positions by four wavefronts, 256 positions each: digits of eight bits, counted in a part of LDS of their own so that a
// digit takes one barrier, and every wavefront scans the counts for itself.  Bound by latency.  With COPY, both steps in one launch: a
// workgroup selects for itself, though it copies only `share` of the head's rows that stay.  That pays while heads are few (one sequence of 611
// positions, 32 heads, 512 stay, caches cold: 14.0 -> 11.4 us; 4 sequences of 800, 8 heads: 13.8 -> 11.8); at 512 heads and more the copy in a launch
// of its own does (64 sequences of 1000, 32 heads: 235 -> 222).
constexpr int SMALL = 4, SHARES = 512; // keys a thread; heads from which on the copy is a launch of its own

template <bool COPY>
__global__ __launch_bounds__(256) void evict_small_kernel(EvictArgs p)
{
    __shared__ __align__(16) int hist[4][256];
    __shared__ int of_wave[4]; // what stays of a wavefront's positions: keys above the last one kept, equal ones in the upper half
    __shared__ short stays[COPY ? 256 * SMALL : 1];
    __shared__ int page_of[2][COPY ? 64 : 1]; // pages read and written, of up to 1024 positions; asked for beside the selection
    const int head = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool writes = blockIdx.x == 0; // what is written once a head
    const int len = min(min(max(p.s.seq_len[b], 0), p.s.max_len), 256 * SMALL);
    const int m = min(len, p.keep), old = len - min(p.recent, m), need = m - (len - old);
    const int j0 = COPY ? blockIdx.x * p.share : 0, j1 = COPY ? min(j0 + p.share, m) : 0;
    if (!writes && j0 >= m)
        return;
    const int t0 = 64 * SMALL * wave + lane; // the thread's first position
    const float *w = p.weights + ((size_t)b * p.kv_heads + head) * p.weights_stride;
    float held[SMALL];
#pragma unroll
    for (int i = 0; i < SMALL; ++i)
        held[i] = t0 + 64 * i < len ? w[t0 + 64 * i] : 0.f;
    *reinterpret_cast<int4 *>(&hist[wave][4 * lane]) = int4{0, 0, 0, 0};
    if (COPY && tid < 128) {
        const int page = wave ? p.dst_table[(size_t)b * p.dst_stride + min(lane, p.dst_stride - 1)] : p.s.table[(size_t)b * p.s.table_stride + min(lane, p.s.table_stride - 1)];
        page_of[wave][lane] = min(max(page, 0), (wave ? p.dst_pages : p.s.pages) - 1);
    }
    uint32_t key[SMALL];
#pragma unroll
    for (int i = 0; i < SMALL; ++i)
        key[i] = weight_key(held[i]);
    const bool all = need >= old, none = need <= 0;
    uint32_t prefix = 0;
    int left = need; // how many of the keys that match the prefix so far are kept
    __syncthreads();
    if (!all && !none) { // the same in every thread, and so is the loop
        for (int d = 0; d < 4; ++d) {
            const int shift = 24 - 8 * d;
            const uint32_t mask = d == 0 ? 0u : 0xffffffffu << (shift + 8);
#pragma unroll
            for (int i = 0; i < SMALL; ++i)
                if (t0 + 64 * i < old && (key[i] & mask) == prefix)
                    atomicAdd(&hist[d][(key[i] >> shift) & 255], 1);
            __syncthreads();
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
    unsigned long long gts[SMALL], eqs[SMALL];
    int found = 0;
#pragma unroll
    for (int i = 0; i < SMALL; ++i) {
        const int t = t0 + 64 * i;
        gts[i] = __builtin_amdgcn_ballot_w64(t < len && (t >= old || all || (!none && key[i] > prefix)));
        eqs[i] = __builtin_amdgcn_ballot_w64(t < old && !all && !none && key[i] == prefix);
        found += (int)__popcll(gts[i]) | (int)__popcll(eqs[i]) << 16;
    }
    if (lane == 0)
        of_wave[wave] = found;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        before += i < wave ? of_wave[i] : 0;
    int gt_before = before & 0xffff, eq_before = before >> 16;
    int *kept = p.kept + ((size_t)b * p.kv_heads + head) * p.keep;
    float *wo = p.weights_out && writes ? p.weights_out + ((size_t)b * p.kv_heads + head) * p.weights_out_stride : nullptr;
    const unsigned long long lower = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < SMALL; ++i) {
        const int e = eq_before + (int)__popcll(eqs[i] & lower), at = gt_before + (int)__popcll(gts[i] & lower) + min(e, left);
        if (((gts[i] >> lane & 1) || ((eqs[i] >> lane & 1) && e < left)) && at < m) {
            if constexpr (COPY)
                stays[at] = (short)(t0 + 64 * i);
            if (writes)
                kept[at] = t0 + 64 * i;
            if (wo)
                wo[at] = held[i];
        }
        gt_before += (int)__popcll(gts[i]);
        eq_before += (int)__popcll(eqs[i]);
    }
    if (writes) {
        if (head == 0 && tid == 0)
            p.new_len[b] = m;
        for (int t = m + tid; t < p.keep; t += 256)
            kept[t] = -1;
    }
    if constexpr (COPY) {
        __syncthreads();
        const auto row_at = [&](int dst, int t) {
            return (((((size_t)page_of[dst][t >> p.s.page_log2] * p.kv_heads + head) << p.s.page_log2) | (size_t)(t & ((1 << p.s.page_log2) - 1)))) * PD + 8 * (tid & 15);
        };
        for (int j = j0 + (tid >> 4); j < j1; j += 64) { // four rows a lane's sixteen at a time
            h8 k[4], v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { // behind the last one that one again
                const size_t from = row_at(0, stays[min(j + 16 * i, j1 - 1)]);
                k[i] = *reinterpret_cast<const h8 *>(p.k + from);
                v[i] = *reinterpret_cast<const h8 *>(p.v + from);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j + 16 * i < j1) {
                    const size_t to = row_at(1, j + 16 * i);
                    *reinterpret_cast<h8 *>(p.k_out + to) = k[i];
                    *reinterpret_cast<h8 *>(p.v_out + to) = v[i];
                }
        }
    }
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
    const long long heads = (long long)kv_heads * batch.seqs;
    if (batch.max_len <= 256 * SMALL && heads < SHARES) {
        const int shares = (int)(2 * SHARES / heads), even = (most + shares - 1) / shares;
        a.share = even < 64 ? 64 : (even + 63) / 64 * 64; // four rows in flight for sixteen lanes
        hipLaunchKernelGGL(evict_small_kernel<true>, dim3(most > a.share ? (most + a.share - 1) / a.share : 1, kv_heads, batch.seqs), dim3(256), 0, st, a);
        return (int)hipGetLastError();
    }
    if (batch.max_len <= 256 * SMALL)
        hipLaunchKernelGGL(evict_small_kernel<false>, dim3(1, kv_heads, batch.seqs), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL(evict_select_kernel, dim3(kv_heads, batch.seqs), dim3(SEL), 0, st, a);
    if (int rc = (int)hipGetLastError())
        return rc;
    if (most == 0)
        return 0;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((most + 15) / 16, kv_heads, batch.seqs), dim3(256), 0, st, a);
    return (int)hipGetLastError();
}
