// Beam search: the best continuations of the beams of a request over the vocabulary, and the masks of the beams that go on.
//
//   total[b][v] = score[b] + (logit[b][v] - lse[b]),  lse[b] = m[b] + log sum_v exp(logit[b][v] - m[b]) with the largest logit m[b],
// the `width` largest of beams * vocab, of equal ones the lower b * vocab + v.  Which one comes ahead of another is decided by differences of
// totals of several beams, so lse and totals are held in 64 bits: with 32, one step in about ten over 64 requests of 16 beams would have two
// of them the wrong way round.  That costs little here: a multiply-add of 64 bits issues as fast as one of 32.
//
// Two launches.  A workgroup of the first has a part of a row in registers, read once: its maximum, its sum of exponentials, and its `width` best logits
// in order.  They are found without sorting: the width-th of the threads' largest is a bound that at least `width` values reach, in at most
// `width` threads if no two of those are equal and in at most BEAM_MOST if some are (the list is sized for that), so few are left, and each of them
// counts those ahead of it.  A workgroup of the second has a request: lse of its beams from the
// parts, and the best of the parts' lists by the same count over their heads.  Many rows are bound by the exponentials, 25 vector
// instructions a value with all that goes with them, behind a first wait of all workgroups for memory (732 rows of 32000, a twelfth of them ended: 24 us, 13.9 of them the issue of 8.52
// million vector instructions, and 7 for the second launch); few by two launches and their barriers (4 rows 5.7 and 5.6).  Workgroups that take several parts, the loads of the next ahead of the work on one,
// were slower (33): fewer of them fit a CU, and each waits for its own barriers.
#include "fq_device.h"
#include "fq_internal.h"

namespace {

constexpr int BEAM_THREADS = 256, BEAM_MOST = 64; // most beams, and most of them that go on
constexpr int BEAM_LISTS = BEAM_MOST * 32;        // of a request: parts of 8192 values of up to 2^18

constexpr int BEAM_NONE = -(1 << 20); // below the power of two of any logit

struct BeamPart {
    double sum, unit; // of exp(logit) 2^-scale, NaN where a logit is NaN or +inf; the same of the largest logit alone
    int scale;        // BEAM_NONE where there is none above -inf
    unsigned short largest, count; // order of the largest logit; entries of its list
};

struct BeamArgs {
    const _Float16 *logits;
    long long ld;
    fq_beam_arrays a;
    BeamPart *parts_out;  // [rows][parts]
    uint32_t *candidates; // [rows][parts][width]: order of the value, 65535 - place in the part
    int requests, beams, vocab, width, parts, part_chunks;
};

// Whether anything goes on from a beam: not from one that isn't there (-inf) or is not a number.
__device__ __forceinline__ bool alive(float score) { return score > -INFINITY; }

// exp(x) 2^-scale in 64 bits, as 2^(i / 256) exp(r) with |r| <= ln 2 / 512, by the series up to r^3 (the rest is below 2e-13 of it).  i - 256 scale comes from the sum
// with `shift`, 1.5 * 2^52 - 256 scale, whose lowest bits it is then.  table: entry k has 2^(k / 256), less k << 12 in its upper word, so that adding i << 12 there
// leaves the power of two alone.  |x| < 2^17, and x / ln 2 - scale at least -1020.
constexpr int EXP_TABLE = 256;

struct ExpTable {
    double entry[EXP_TABLE];
};
constexpr ExpTable exp_entries()
{
    ExpTable t{};
    for (int k = 0; k < EXP_TABLE; ++k) {
        const double x = k * 0.0027076061740622863;
        double sum = 1.0;
        for (int n = 22; n > 0; --n) // the series of exp from its end
            sum = 1.0 + sum * x / n;
        t.entry[k] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, sum) - ((uint64_t)k << 44));
    }
    return t;
}
__device__ constexpr ExpTable exp_table = exp_entries();

struct ExpTerms {
    double shift, steps, step, sixth; // 1.5 * 2^52 - 256 scale; 256 / ln 2; -ln 2 / 256, whose error is below 3e-19, times i
    __device__ explicit ExpTerms(int scale) : shift(6755399441055744.0 - 256.0 * scale), steps(369.32993046757464), step(-0.0027076061740622863), sixth(1.0 / 6)
    {
        asm("" : "+v"(shift), "+v"(steps), "+v"(step), "+v"(sixth)); // in registers: moved there for every use otherwise
    }
};
__device__ __forceinline__ double add_exp(double sum, double x, const ExpTerms &c, const u2v *table)
{
    const double shifted = fma(x, c.steps, c.shift);
    const double r = fma(shifted - c.shift, c.step, x);
    const uint32_t i = (uint32_t)__builtin_bit_cast(uint64_t, shifted);
    double e = fma(r, c.sixth, 0.5);
    e = fma(e, r, 1.0);
    e = fma(e, r, 1.0);
    const u2v t = table[i & (EXP_TABLE - 1)];
    return fma(e, __builtin_bit_cast(double, u2v{t.x, t.y + (i << 12)}), sum);
}

// fp16 as whole numbers in the same order, both zeros alike; ORDER_LEAST and above are candidates, -inf is below, +inf and what of NaN is positive from
// ORDER_INF on.
constexpr uint32_t ORDER_LEAST = 0x400, ORDER_INF = 0xfc00;

__device__ __forceinline__ uint32_t order_of(_Float16 x)
{
    const uint32_t bits = __builtin_bit_cast(unsigned short, x), order = bits ^ (bits & 0x8000 ? 0xffff : 0x8000);
    return order == 0x7fff ? 0x8000 : order;
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

// CHUNKS: 16-byte pieces of a row that a thread has.  Chunks are numbered along the row, so a chunk whose largest value is smaller, or as large and
// the chunk further on, has nothing ahead of the other's: the order of chunks by (largest value, number) bounds that of their values.
template <int CHUNKS>
__global__ __launch_bounds__(BEAM_THREADS, 8) void beam_rows_kernel(BeamArgs p)
{
    __shared__ __align__(16) uint32_t tops[BEAM_THREADS];
    __shared__ uint32_t list[BEAM_MOST * CHUNKS * 8];
    __shared__ u2v table[EXP_TABLE];
    __shared__ double wave_sum[4], unit;
    __shared__ uint32_t bound;
    __shared__ int listed;
    const int row = blockIdx.x / p.parts, part = blockIdx.x - row * p.parts, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool goes_on = alive(p.a.scores[row]) && !(p.a.done && p.a.done[row] != 0); // uniform
    if (CHUNKS > 1 && !goes_on) // where there are few rows, what is read for nothing costs less than to wait for the score first
        return;
    const _Float16 *const x = p.logits + (size_t)row * p.ld;
    h8 mine[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int chunk = c * BEAM_THREADS + tid, at = 8 * (part * p.part_chunks + chunk); // its first value's place in the row
        u4v bits = {0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u};
        if (chunk >= p.part_chunks) {
        } else if (at + 8 <= p.vocab) {
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
        mine[c] = __builtin_bit_cast(h8, bits);
    }
    if (CHUNKS == 1 && !goes_on)
        return;
    table[tid] = __builtin_bit_cast(u2v, exp_table.entry[tid]);
    if (tid == 0)
        listed = 0;
    uint32_t order[CHUNKS], top = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        h2 high = {mine[c][0], mine[c][1]};
#pragma unroll
        for (int e = 1; e < 4; ++e)
            high = __builtin_elementwise_maximum(high, h2{mine[c][2 * e], mine[c][2 * e + 1]}); // NaN where there is one
        const _Float16 h = __builtin_elementwise_maximum(high[0], high[1]);
        order[c] = (h != h ? 0xffff : order_of(h)) << 16 | (0xffff - (c * BEAM_THREADS + tid));
        top = max(top, order[c]);
    }
    tops[tid] = top;
    __syncthreads();
    const u4v four = *reinterpret_cast<const u4v *>(&tops[4 * lane]); // every wavefront has them all
    uint32_t all = max(max(four.x, four.y), max(four.z, four.w));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        all = max(all, (uint32_t)__shfl_xor((int)all, o, 64));
    BeamPart *const out = p.parts_out + (size_t)row * p.parts + part;
    const bool none = all >> 16 < ORDER_LEAST;
    if (none || all >> 16 >= ORDER_INF) { // nothing but -inf, or a NaN or +inf (uniform)
        if (tid == 0)
            *out = BeamPart{none ? 0.0 : (double)NAN, 1.0, none ? BEAM_NONE : 0, 0, 0};
        return;
    }
    if (wave == 0) {
        // The width-th largest, bit by bit: the largest bound that `width` of them reach.  Their lower half is 0xfc00 at least; it matters only where
        // ties would be more than the list holds.
        uint32_t least = 0;
        const auto reach = [&](uint32_t b) {
            return (int)(__popcll(__builtin_amdgcn_ballot_w64(four.x >= b)) + __popcll(__builtin_amdgcn_ballot_w64(four.y >= b)) +
                         __popcll(__builtin_amdgcn_ballot_w64(four.z >= b)) + __popcll(__builtin_amdgcn_ballot_w64(four.w >= b)));
        };
#pragma unroll 1
        for (uint32_t bit = 1u << 31; bit > 0x8000; bit >>= 1)
            least = reach(least | bit) >= p.width ? least | bit : least;
        if (least >= ORDER_LEAST << 16 && reach(least) > BEAM_MOST) {
            least |= 0xfc00;
#pragma unroll 1
            for (uint32_t bit = 0x200; bit; bit >>= 1)
                least = reach(least | bit) >= p.width ? least | bit : least;
        }
        if (lane == 0)
            bound = max(least, ORDER_LEAST << 16);
    }
    const float high = value_of(all >> 16);
    const int scale = (int)rintf(high * 1.44269504f); // sums as of 2^scale, near exp(high)
    const ExpTerms terms(scale);
    const float low = high - 700.f; // -inf and what else is below counts as exp(-700) of the largest
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum = add_exp(sum, (double)fmaxf((float)mine[c][e], low), terms, table);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        sum += __shfl_xor(sum, o, 64);
    if (lane == 0)
        wave_sum[wave] = sum;
    if (tid == BEAM_THREADS - 64)
        unit = add_exp(0.0, (double)high, terms, table);
    __syncthreads();
    const uint32_t least = bound;
    if (top >= least) { // at most BEAM_MOST threads: all of theirs fit the list
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (order[c] >= least) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t o = order_of(mine[c][e]);
                    if (o >= least >> 16)
                        list[atomicAdd(&listed, 1)] = o << 16 | (0xffff - (8 * (c * BEAM_THREADS + tid) + e));
                }
            }
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
        *out = BeamPart{wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3], unit, scale, (unsigned short)(all >> 16), (unsigned short)min(count, p.width)};
}

// 64 bits in the order of their values, both zeros alike; 0 is below all numbers.
__device__ __forceinline__ uint64_t order_of(double x)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x + 0.0);
    return bits >> 63 ? ~bits : bits | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t order)
{
    return __builtin_bit_cast(double, order >> 63 ? order & ~(1ull << 63) : ~order);
}

// i / d for i * d < 2^32, with 2^32 / d rounded up.
__device__ __forceinline__ int quotient(int i, uint32_t inverse) { return inverse ? (int)__umulhi((uint32_t)i, inverse) : i; }

// How many of up to 64 Q keys in LDS are ahead of each, added to ahead[]: a lane has Q of them, a wavefront compares a quarter of all with those.  Of equal
// ones the lower index[] is ahead, or the lower place without one.
template <int Q>
__device__ __forceinline__ void count_ahead(const uint64_t *keys, const uint32_t *index, int count, int *ahead)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint64_t key[Q];
    uint32_t place[Q];
    int found[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int i = lane + 64 * q, at = min(i, max(count - 1, 0));
        key[q] = keys[at];
        place[q] = index ? index[at] : (uint32_t)i;
        found[q] = 0;
    }
#pragma unroll 2
    for (int j = wave; j < count; j += BEAM_THREADS / 64) {
        const uint64_t other = keys[j];
        const uint32_t other_place = index ? index[j] : (uint32_t)j;
#pragma unroll
        for (int q = 0; q < Q; ++q)
            found[q] += other > key[q] || (other == key[q] && other_place < place[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (lane + 64 * q < count)
            atomicAdd(&ahead[lane + 64 * q], found[q]);
}

// Everything that the call has left in memory is asked for at once, as far as registers hold it: the parts, PER entries of lists and a word
// of masks a thread.  Entries beyond those are read once the lists that matter are known.
template <int PER>
__global__ __launch_bounds__(BEAM_THREADS) void beam_merge_kernel(BeamArgs p, uint32_t per_width, uint32_t per_parts)
{
    __shared__ uint64_t heads[BEAM_LISTS], keys[BEAM_MOST * BEAM_MOST], masks[BEAM_THREADS];
    __shared__ uint32_t index[BEAM_MOST * BEAM_MOST];
    __shared__ double lse[BEAM_MOST]; // NaN of beams that do not go on
    __shared__ float scores[BEAM_MOST];
    __shared__ int parent[BEAM_MOST], ended[BEAM_MOST], chosen[BEAM_MOST], ahead_of[2][BEAM_THREADS]; // heads; what is left of the entries
    __shared__ unsigned char counts[BEAM_LISTS];
    __shared__ uint64_t bound;
    __shared__ int listed, found;
    double *const sums = reinterpret_cast<double *>(heads), *const units = reinterpret_cast<double *>(keys); // of the parts, until the heads are known
    int *const scales = reinterpret_cast<int *>(index);
    uint32_t *const largest = index + BEAM_LISTS;
    const int r = blockIdx.x, tid = threadIdx.x;
    const int row0 = r * p.beams, lists = p.beams * p.parts, entries = lists * p.width, mask_entries = p.beams * p.a.mask_words;
    const BeamPart *const parts = p.parts_out + (size_t)row0 * p.parts;
    const uint32_t *const candidates = p.candidates + (size_t)row0 * p.parts * p.width;
    uint32_t held[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k)
        held[k] = candidates[min(tid + BEAM_THREADS * k, entries - 1)];
    const bool masks_here = p.a.mask && mask_entries <= BEAM_THREADS;
    if (masks_here && tid < mask_entries)
        masks[tid] = p.a.mask[(size_t)row0 * p.a.mask_words + tid];
    const int tail = p.a.mask_out && p.a.tail ? p.a.tail[r] : 0;
    for (int i = tid; i < lists; i += BEAM_THREADS) { // of beams that nobody has looked at, anything
        const BeamPart part = parts[i];
        sums[i] = part.sum;
        units[i] = part.unit;
        scales[i] = part.scale;
        largest[i] = (uint32_t)part.largest << 16 | i;
        counts[i] = (unsigned char)part.count;
    }
    if (tid < p.beams) {
        scores[tid] = p.a.scores[row0 + tid];
        ended[tid] = p.a.done && p.a.done[row0 + tid] != 0;
    }
    ahead_of[0][tid] = ahead_of[1][tid] = 0;
    if (tid == 0) {
        bound = 1;
        listed = found = 0;
    }
    __syncthreads();
    if (tid < p.beams) {
        // In units of the largest logit's term, which is one of the sum's, a row of one token has a sum of 1 and goes on with its beam's score to the last
        // bit: beams of equal scores whose tokens are forced tie, whatever the logits.  The largest logit has the largest scale, too.
        double at = NAN;
        if (!ended[tid] && alive(scores[tid])) {
            double sum = 0.0;
            const int part0 = tid * p.parts;
            uint32_t high = 0; // and the list that it is of
#pragma unroll 4
            for (int j = 0; j < p.parts; ++j)
                high = max(high, largest[part0 + j]);
            const int scale = scales[high & 0xffff];
            const double unit = units[high & 0xffff];
#pragma unroll 4
            for (int j = 0; j < p.parts; ++j)
                sum += ldexp(sums[part0 + j], scales[part0 + j] - scale);
            at = sum > 0.0 ? (double)value_of(high >> 16) + log(sum / unit) : (double)NAN;
        }
        lse[tid] = at;
    }
    __syncthreads();
    // The order of entry j of list l, 0 where it has none that counts, and its index; c: what the list has there.
    const auto entry = [&](int l, int j, uint32_t c, uint32_t *at) -> uint64_t {
        const int b = quotient(l, per_parts), part = l - b * p.parts;
        const double score = scores[b], total = score + ((double)value_of(c >> 16) - lse[b]);
        if (ended[b]) {
            *at = (uint32_t)b * p.vocab + p.a.eos;
            return part == 0 && j == 0 && score > -INFINITY ? order_of(score) : 0;
        }
        *at = (uint32_t)b * p.vocab + part * p.part_chunks * 8 + (0xffff - (c & 0xffff));
        return j < counts[l] && total > -INFINITY ? order_of(total) : 0;
    };
    const bool all_held = entries <= PER * BEAM_THREADS;
    const int firsts = all_held ? max(min(64 / lists, p.width), 1) : 1, firsts_all = lists * firsts; // entries of a list that the bound is taken from
    uint64_t held_key[PER];
    uint32_t held_at[PER];
    if (all_held) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = tid + BEAM_THREADS * k, l = quotient(i, per_width), j = i - l * p.width;
            held_key[k] = 0;
            if (i < entries) {
                held_key[k] = entry(l, j, held[k], &held_at[k]);
                if (j < firsts)
                    heads[l * firsts + j] = held_key[k];
            }
        }
    } else {
        uint32_t at;
        for (int l = tid; l < lists; l += BEAM_THREADS)
            heads[l] = entry(l, 0, candidates[(size_t)l * p.width], &at);
    }
    __syncthreads();
    // The width-th of the heads bounds what is among the best; and no list whose head is not among the `width` first has any of them.
    const auto head_is = [&](int i, int ahead) {
        const uint64_t head = heads[i];
        if (ahead < p.width && head != 0) {
            if (!all_held) {
                chosen[ahead] = i;
                atomicMax(&found, ahead + 1);
            }
            if (ahead == p.width - 1)
                bound = head;
        }
    };
    if (firsts_all <= BEAM_THREADS) {
        if (firsts_all <= 64)
            count_ahead<1>(heads, nullptr, firsts_all, ahead_of[0]);
        else
            count_ahead<4>(heads, nullptr, firsts_all, ahead_of[0]);
        __syncthreads();
        if (tid < firsts_all)
            head_is(tid, ahead_of[0][tid]);
    } else {
        for (int i = tid; i < firsts_all; i += BEAM_THREADS) {
            const uint64_t head = heads[i];
            int ahead = 0;
#pragma unroll 4
            for (int j = 0; j < firsts_all; ++j)
                ahead += heads[j] > head || (heads[j] == head && j < i);
            head_is(i, ahead);
        }
    }
    __syncthreads();
    const auto take = [&](uint64_t key, uint32_t at) {
        if (key >= bound) {
            const int to = atomicAdd(&listed, 1);
            keys[to] = key;
            index[to] = at;
        }
    };
    if (all_held) { // at most PER * 256 of them
#pragma unroll
        for (int k = 0; k < PER; ++k)
            take(held_key[k], held_at[k]);
    } else { // at most 64 lists of 64 entries
        for (int i = tid; i < found * p.width; i += BEAM_THREADS) {
            const int n = quotient(i, per_width), l = chosen[n], j = i - n * p.width;
            uint32_t at;
            const uint64_t key = entry(l, j, candidates[(size_t)l * p.width + j], &at);
            take(key, at);
        }
    }
    __syncthreads();
    const int count = listed;
    const size_t out = (size_t)r * p.width;
    if (count <= BEAM_THREADS) {
        if (count <= 64)
            count_ahead<1>(keys, index, count, ahead_of[1]);
        else
            count_ahead<4>(keys, index, count, ahead_of[1]);
        __syncthreads();
    }
    for (int i = tid; i < max(count, p.width); i += BEAM_THREADS) {
        int at = i; // places behind those that are found are empty
        if (i < count) {
            at = 0;
            if (count <= BEAM_THREADS)
                at = ahead_of[1][i];
            else
#pragma unroll 4
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
    for (int i = tid; i < p.width * p.a.mask_words; i += BEAM_THREADS) {
        const int j = i / p.a.mask_words, w = i - j * p.a.mask_words, b = parent[j];
        const long long own = (long long)tail + j;
        uint64_t bits = 0;
        if (b >= 0) {
            bits = own >= 0 && own >> 6 == w ? 1ull << (own & 63) : 0ull;
            if (masks_here)
                bits |= masks[b * p.a.mask_words + w];
            else if (p.a.mask)
                bits |= p.a.mask[((size_t)row0 + b) * p.a.mask_words + w];
        }
        p.a.mask_out[out * p.a.mask_words + i] = bits;
    }
}

uint32_t inverse(int d) { return d > 1 ? (uint32_t)(((1ull << 32) + d - 1) / d) : 0; } // for quotient()

// The largest parts of which there are enough to fill the chip, and no more of them than a request's lists may be: what a workgroup does once costs as
// much as 16 values a thread (37 requests of 5 beams, one of them live, 32000 tokens: parts of 2048 values 7.7 us, 4096 7.2; 61 of 12: 8192 values
// 24.0, 16384 25.7, as their workgroups wait for memory all at once).
struct BeamPlan {
    int chunks, parts, part_chunks;
    size_t end;
};

BeamPlan plan_beam(int requests, int beams, int vocab, int width)
{
    const long long rows = (long long)requests * beams;
    const int all = (vocab + 7) / 8;
    const auto parts = [&](int chunks) { return (all + BEAM_THREADS * chunks - 1) / (BEAM_THREADS * chunks); };
    BeamPlan s;
    s.chunks = 4;
    while (s.chunks > 1 && rows * parts(s.chunks) < 1200 && beams * parts(s.chunks / 2) <= BEAM_LISTS)
        s.chunks /= 2;
    s.parts = parts(s.chunks);
    s.part_chunks = (all + s.parts - 1) / s.parts;
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
               reinterpret_cast<uint32_t *>(static_cast<BeamPart *>(workspace) + rows * s.parts), requests, beams, vocab, width, s.parts, s.part_chunks};
    const dim3 grid((unsigned)(rows * s.parts));
    const auto kernel = s.chunks == 1 ? beam_rows_kernel<1> : s.chunks == 2 ? beam_rows_kernel<2> : beam_rows_kernel<4>;
    hipLaunchKernelGGL(kernel, grid, dim3(BEAM_THREADS), 0, st, p);
    const int rc = (int)hipGetLastError();
    if (rc != 0)
        return rc;
    hipLaunchKernelGGL(beam_merge_kernel<4>, dim3(requests), dim3(BEAM_THREADS), 0, st, p, inverse(width), inverse(s.parts));
    return (int)hipGetLastError();
}
