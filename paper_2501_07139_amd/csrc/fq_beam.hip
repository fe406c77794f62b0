// Beam search: the best continuations of the beams of a request over the vocabulary, and the masks of the beams that go on.
//
//   total[b][v] = score[b] + logit[b][v] - lse[b],  lse[b] = log sum_v exp(logit[b][v]),
// the `width` largest of beams * vocab, of equal ones the lower b * vocab + v.  Which one comes ahead of another is decided by differences of
// totals of several beams, so lse and totals are held in 64 bits: with 32, one step in about ten over 64 requests of 16 beams would have two
// of them the wrong way round.  That costs little here: a multiply-add of 64 bits issues as fast as one of 32.
//
// Two launches.  A workgroup of the first has a part of a row in registers, read once: its maximum, its sum of exponentials, and its `width` best logits
// in order.  They are found without sorting: every thread has the largest of its own values; the width-th of these is a bound that at least
// `width` values reach and that at most `width` threads have values above, so few are left, and each of them counts those ahead of it.  A
// workgroup of the second has a request: lse of its beams from the parts, and the best of the parts' lists by the same count over their heads.
#include "fq_device.h"
#include "fq_internal.h"

namespace {

constexpr int BEAM_THREADS = 256, BEAM_MOST = 64; // most beams, and most of them that go on
constexpr int BEAM_LISTS = BEAM_MOST * 32;        // of a request: parts of 8192 values of up to 2^18

struct BeamPart {
    double sum; // of exp(logit - max); NaN where a logit is NaN or +inf
    float max;  // -inf where there is none above
    int count;  // of its list
};

struct BeamArgs {
    const _Float16 *logits;
    long long ld;
    fq_beam_arrays a;
    BeamPart *parts_out;  // [rows][parts]
    uint32_t *candidates; // [rows][parts][width]: order of the value, 65535 - place in the part
    int requests, beams, vocab, width, parts;
};

// Whether anything goes on from a beam: not from one that isn't there (-inf) or is not a number.
__device__ __forceinline__ bool alive(float score) { return score > -INFINITY; }

// exp of x <= 0 in 64 bits: 2^k exp(r), |r| <= ln 2 / 2, by the series up to r^11 (the rest is below 1e-14).
__device__ __forceinline__ double exp_down(double x)
{
    x = fmax(x, -700.0); // 1e-304 for what is below; 2^k stays a normal number
    const double k = __builtin_rint(x * 1.4426950408889634074);
    const double r = fma(k, -1.9082149292705877e-10, fma(k, -0.69314718036912381649, x)); // ln 2 in two parts, the first of 32 bits: exact
    double e = 1.0 / 39916800;
    e = fma(e, r, 1.0 / 3628800);
    e = fma(e, r, 1.0 / 362880);
    e = fma(e, r, 1.0 / 40320);
    e = fma(e, r, 1.0 / 5040);
    e = fma(e, r, 1.0 / 720);
    e = fma(e, r, 1.0 / 120);
    e = fma(e, r, 1.0 / 24);
    e = fma(e, r, 1.0 / 6);
    e = fma(e, r, 0.5);
    e = fma(e, r, 1.0);
    e = fma(e, r, 1.0);
    return e * __builtin_bit_cast(double, (uint64_t)(1023 + (int)k) << 52);
}

// fp16 as whole numbers in the same order: NaN above all, both zeros alike, 0 for what is no candidate (-inf).
__device__ __forceinline__ uint32_t order_of(uint32_t bits)
{
    const uint32_t size = bits & 0x7fff;
    if (size > 0x7c00)
        return 0xffff;
    if (bits == 0xfc00)
        return 0;
    return bits & 0x8000 ? (size == 0 ? 0x8000 : 0xffff - bits) : bits | 0x8000;
}
__device__ __forceinline__ float value_of(uint32_t order) // of a candidate
{
    const uint32_t bits = order & 0x8000 ? order & 0x7fff : 0xffff - order;
    return (float)__builtin_bit_cast(_Float16, (unsigned short)bits);
}

// 16 bytes at any even address: rows of an odd vocabulary begin anywhere, and a row is divided alike wherever it begins, so that beams of the same
// logits have the same lse to the last bit, and tie.
struct __attribute__((packed, aligned(2))) LooseChunk {
    u4v bits;
};

// CHUNKS: 16-byte pieces of a row that a thread has.
template <int CHUNKS>
__global__ __launch_bounds__(BEAM_THREADS) void beam_rows_kernel(BeamArgs p)
{
    __shared__ __align__(16) uint32_t tops[BEAM_THREADS];
    __shared__ uint32_t list[BEAM_MOST * CHUNKS * 8];
    __shared__ uint32_t wave_top[4], bound;
    __shared__ double wave_sum[4];
    __shared__ int listed;
    const int row = blockIdx.x / p.parts, part = blockIdx.x - row * p.parts, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (!alive(p.a.scores[row]) || (p.a.done && p.a.done[row] != 0))
        return;
    const _Float16 *const x = p.logits + (size_t)row * p.ld;
    uint32_t mine[CHUNKS * 8], top = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * ((part * CHUNKS + c) * BEAM_THREADS + tid); // of its first value in the row
        u4v bits = {0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u};
        if (at + 8 <= p.vocab) {
            bits = reinterpret_cast<const LooseChunk *>(x + at)->bits;
        } else if (at < p.vocab) { // the end of a row, value by value: nothing is read behind it
            uint32_t d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = at + 2 * e;
                const uint32_t lo = i < p.vocab ? __builtin_bit_cast(unsigned short, x[i]) : 0xfc00u;
                const uint32_t hi = i + 1 < p.vocab ? __builtin_bit_cast(unsigned short, x[i + 1]) : 0xfc00u;
                d[e] = hi << 16 | lo;
            }
            bits = u4v{d[0], d[1], d[2], d[3]};
        }
        const uint32_t d[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t order = order_of(d[e >> 1] >> (16 * (e & 1)) & 0xffff);
            mine[8 * c + e] = order ? order << 16 | (0xffff - (8 * (c * BEAM_THREADS + tid) + e)) : 0;
            top = max(top, mine[8 * c + e]);
        }
    }
    tops[tid] = top;
    uint32_t all = top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        all = max(all, (uint32_t)__shfl_xor((int)all, o, 64));
    if (lane == 0)
        wave_top[wave] = all;
    if (tid == 0)
        listed = 0;
    __syncthreads();
    all = max(max(wave_top[0], wave_top[1]), max(wave_top[2], wave_top[3]));
    BeamPart *const out = p.parts_out + (size_t)row * p.parts + part;
    if (all == 0 || all >> 16 >= 0xfc00) { // nothing but -inf, or a NaN or +inf (uniform)
        if (tid == 0)
            *out = BeamPart{all == 0 ? 0.0 : (double)NAN, all == 0 ? -INFINITY : 0.f, 0};
        return;
    }
    const float high = value_of(all >> 16);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < CHUNKS * 8; ++e)
        sum += mine[e] ? exp_down((double)value_of(mine[e] >> 16) - (double)high) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        sum += __shfl_xor(sum, o, 64);
    if (lane == 0)
        wave_sum[wave] = sum;
    // how many threads' largest are ahead of this one's
    int ahead = 0;
#pragma unroll 8
    for (int i = 0; i < BEAM_THREADS; i += 4) {
        const u4v t = *reinterpret_cast<const u4v *>(&tops[i]);
        ahead += (t.x > top || (t.x == top && i < tid)) + (t.y > top || (t.y == top && i + 1 < tid)) + (t.z > top || (t.z == top && i + 2 < tid)) +
                 (t.w > top || (t.w == top && i + 3 < tid));
    }
    if (ahead == p.width - 1)
        bound = max(top, 1u);
    __syncthreads();
    const uint32_t least = bound;
    if (top >= least) {
#pragma unroll
        for (int e = 0; e < CHUNKS * 8; ++e)
            if (mine[e] >= least)
                list[atomicAdd(&listed, 1)] = mine[e];
    }
    __syncthreads();
    const int count = listed;
    uint32_t *const to = p.candidates + ((size_t)row * p.parts + part) * p.width;
    for (int i = tid; i < count; i += BEAM_THREADS) { // all different: a place is part of each
        int before = 0;
        for (int j = 0; j < count; ++j)
            before += list[j] > list[i];
        if (before < p.width)
            to[before] = list[i];
    }
    if (tid == 0)
        *out = BeamPart{wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3], high, min(count, p.width)};
}

// 64 bits in the order of their values; 0 is below all numbers.
__device__ __forceinline__ uint64_t order_of(double x)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    return bits >> 63 ? ~bits : bits | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t order)
{
    return __builtin_bit_cast(double, order >> 63 ? order & ~(1ull << 63) : ~order);
}

__global__ __launch_bounds__(BEAM_THREADS) void beam_merge_kernel(BeamArgs p, int part_values)
{
    __shared__ uint64_t heads[BEAM_LISTS], keys[BEAM_MOST * BEAM_MOST];
    __shared__ uint32_t index[BEAM_MOST * BEAM_MOST];
    __shared__ double offset[BEAM_MOST]; // score - lse
    __shared__ int parent[BEAM_MOST], ended[BEAM_MOST], chosen[BEAM_MOST];
    __shared__ uint64_t bound;
    __shared__ int listed, found;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = r * p.beams, lists = p.beams * p.parts;
    for (int b = wave; b < p.beams; b += BEAM_THREADS / 64) {
        const float score = p.a.scores[row0 + b];
        const bool over = p.a.done && p.a.done[row0 + b] != 0;
        double at = NAN;
        if (over) {
            at = score;
        } else if (alive(score)) {
            const BeamPart *const parts = p.parts_out + (size_t)(row0 + b) * p.parts;
            float high = -INFINITY;
            for (int i = lane; i < p.parts; i += 64)
                high = fmaxf(high, parts[i].max);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1)
                high = fmaxf(high, __shfl_xor(high, o, 64));
            double sum = 0.0;
            for (int i = lane; i < p.parts; i += 64)
                sum += parts[i].max == -INFINITY ? 0.0 : parts[i].sum * exp_down((double)parts[i].max - (double)high);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1)
                sum += __shfl_xor(sum, o, 64);
            at = sum > 0.0 ? (double)score - ((double)high + log(sum)) : (double)NAN;
        }
        if (lane == 0) {
            offset[b] = at;
            ended[b] = over;
        }
    }
    if (tid == 0) {
        bound = 1;
        listed = found = 0;
    }
    __syncthreads();
    // the order of entry j of a list, 0 where it has none that counts
    const auto entry = [&](int b, int part, int j, int *token) -> uint64_t {
        const double at = offset[b];
        if (ended[b]) {
            *token = p.a.eos;
            return part == 0 && j == 0 && at > -INFINITY ? order_of(at) : 0;
        }
        if (!(at > -INFINITY) || j >= p.parts_out[(size_t)(row0 + b) * p.parts + part].count)
            return 0;
        const uint32_t c = p.candidates[((size_t)(row0 + b) * p.parts + part) * p.width + j];
        *token = part * part_values + (int)(0xffff - (c & 0xffff));
        return order_of(at + (double)value_of(c >> 16));
    };
    int token;
    for (int i = tid; i < lists; i += BEAM_THREADS)
        heads[i] = entry(i / p.parts, i % p.parts, 0, &token);
    __syncthreads();
    // Lists whose heads are among the `width` first: no other list has any of the best, and of these what the last of the heads is not ahead of.
    for (int i = tid; i < lists; i += BEAM_THREADS) {
        const uint64_t head = heads[i];
        if (head == 0)
            continue;
        int ahead = 0;
        for (int j = 0; j < lists; ++j)
            ahead += heads[j] > head || (heads[j] == head && j < i);
        if (ahead < p.width)
            chosen[ahead] = i;
        if (ahead == p.width - 1)
            bound = head;
        atomicMax(&found, min(ahead + 1, p.width));
    }
    __syncthreads();
    for (int i = tid; i < found * p.width; i += BEAM_THREADS) { // at most 64 lists of 64 entries
        const int l = chosen[i / p.width], b = l / p.parts;
        const uint64_t key = entry(b, l - b * p.parts, i % p.width, &token);
        if (key >= bound) {
            const int to = atomicAdd(&listed, 1);
            keys[to] = key;
            index[to] = (uint32_t)b * p.vocab + token;
        }
    }
    __syncthreads();
    const int count = listed;
    const size_t out = (size_t)r * p.width;
    for (int i = tid; i < max(count, p.width); i += BEAM_THREADS) {
        int at = i; // places behind those that are found are empty
        if (i < count) {
            at = 0;
            for (int j = 0; j < count; ++j)
                at += keys[j] > keys[i] || (keys[j] == keys[i] && index[j] < index[i]);
        }
        if (at >= p.width)
            continue;
        const int b = i < count ? (int)(index[i] / (uint32_t)p.vocab) : -1, v = i < count ? (int)(index[i] - (uint32_t)b * p.vocab) : -1;
        parent[at] = b;
        p.a.parent[out + at] = b;
        p.a.token[out + at] = v;
        p.a.scores_out[out + at] = i < count ? (float)value_of(keys[i]) : -INFINITY;
        if (p.a.done_out)
            p.a.done_out[out + at] = i < count ? (ended[b] || v == p.a.eos) : 1;
    }
    if (!p.a.mask_out)
        return;
    __syncthreads();
    const int tail = p.a.tail ? p.a.tail[r] : 0;
    for (int i = tid; i < p.width * p.a.mask_words; i += BEAM_THREADS) {
        const int j = i / p.a.mask_words, w = i - j * p.a.mask_words, b = parent[j];
        const long long own = (long long)tail + j;
        uint64_t bits = 0;
        if (b >= 0)
            bits = (p.a.mask ? p.a.mask[((size_t)row0 + b) * p.a.mask_words + w] : 0) | (own >= 0 && own >> 6 == w ? 1ull << (own & 63) : 0ull);
        p.a.mask_out[out * p.a.mask_words + i] = bits;
    }
}

// Small parts where there are few rows: a part is read by one workgroup, and 512 of them fill the chip.
struct BeamPlan {
    int chunks, parts;
    size_t end;
};

BeamPlan plan_beam(int requests, int beams, int vocab, int width)
{
    const long long rows = (long long)requests * beams;
    const auto parts = [&](int chunks) { return (vocab + 8 * BEAM_THREADS * chunks - 1) / (8 * BEAM_THREADS * chunks); };
    BeamPlan s;
    s.chunks = rows * parts(1) <= 512 ? 1 : 4;
    s.parts = parts(s.chunks);
    s.end = (size_t)rows * s.parts * (sizeof(BeamPart) + sizeof(uint32_t) * width);
    return s;
}

} // namespace

size_t fq_beam_scratch_bytes(int requests, int beams, int vocab, int width) { return plan_beam(requests, beams, vocab, width).end; }

int fq_launch_beam_step(const void *logits, long long ld, int requests, int beams, int vocab, int width, const fq_beam_arrays &a, void *workspace, fq_stream st)
{
    const BeamPlan s = plan_beam(requests, beams, vocab, width);
    const size_t rows = (size_t)requests * beams;
    BeamArgs p{static_cast<const _Float16 *>(logits), ld, a, static_cast<BeamPart *>(workspace),
               reinterpret_cast<uint32_t *>(static_cast<BeamPart *>(workspace) + rows * s.parts), requests, beams, vocab, width, s.parts};
    const dim3 grid((unsigned)(rows * s.parts));
    if (s.chunks == 1)
        hipLaunchKernelGGL(beam_rows_kernel<1>, grid, dim3(BEAM_THREADS), 0, st, p);
    else
        hipLaunchKernelGGL(beam_rows_kernel<4>, grid, dim3(BEAM_THREADS), 0, st, p);
    const int rc = (int)hipGetLastError();
    if (rc != 0)
        return rc;
    hipLaunchKernelGGL(beam_merge_kernel, dim3(requests), dim3(BEAM_THREADS), 0, st, p, 8 * BEAM_THREADS * s.chunks);
    return (int)hipGetLastError();
}
