// dps_beam.hip -- the next beams from logits over the vocabulary (gfx950).
//
// Beam w of a batch item, token t:  score = cum_w + (x_wt - log sum_t exp x_wt).
// The `keep` best over all beams and tokens, of equal ones those with the lowest
// (w, t).  Within a beam the order is that of the logits alone, so a piece of a
// row can give up all but its `keep` best before the row's sum is known.  (Where different
// logits end in the same 64-bit score, which of them were given up depends on their
// pieces: the lowest tokens among those that were not are taken.)
//
// Two launches.  The first reads every logit once: a block of threads holds a piece
// of a row in registers, sums its exponentials (a wave each) and lists its best.  The second, a
// block a batch item, joins the sums and picks from the lists.
//
// Bound: HBM for the first where rows are many (2 or 4 bytes a logit), else latency: of 512
// rows of 100003 FP32 logits the 459 that live (184 MB) take 31.4 us, 5.9 TB/s, and the
// second launch 10.4; 128 rows of 131072 BF16 logits 13.3 + 10.4, 4 of 32000 6.0 + 7.5.
//
// The best of a piece: the keep-th largest of the threads' maxima is a bound that
// `keep` values reach at least; what reaches it (hardly more than that, of values
// in no order) is listed in LDS and ranked.  Where ties or an order in the data bring
// more than the list holds, the keep-th best value, and the last index among its
// equals, are found by bisection over the register values: exact whatever the data.
//
// Precision: exponentials in fp32 of differences from the wave's largest (of which
// none is above 0), the values of a 16-byte vector added in fp32, in pairs; their
// sums, log and scores in 64 bits, since candidates of different beams may lie closer
// than fp32 tells apart.  A sum is good to 2^-19.8 of itself (fp32 logits 2^-20), in units of
// 2^-24: 3 (2) for the pairs' roundings, 2 for the exponential, and 2.23 |d| for its
// argument (the difference d and the product are rounded, log2 e is 0.23 off), where the mean
// of |d| under the weights e^d is at most 5.6 of a wave's 4096 values (5.0 of 2048): (n - 1) t /
// (e^t + n - 1), which is what one value and n - 1 others t below it have.  Such rows came
// out up to 8.2 units off (16 bits: 6.5).
#include <type_traits>

#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kBeamWaves;
static_assert(kThreads == 64 * kWaves, "a sum a wave");
constexpr int kList = 1024;
constexpr int kFew = 64;  // threads whose values are looked through one by one
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

// Whole numbers in the order of the values; NaN is not looked for.
__device__ __forceinline__ int32_t ordered(float x)
{
    const int32_t i = __builtin_bit_cast(int32_t, x + 0.0f);  // -0 as 0
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int32_t k)
{
    return __builtin_bit_cast(float, k ^ ((k >> 31) & 0x7fffffff));
}
__device__ __forceinline__ int64_t ordered(double x)
{
    const int64_t i = __builtin_bit_cast(int64_t, x + 0.0);
    return i ^ ((i >> 63) & 0x7fffffffffffffffll);
}

// Over all threads, for every thread; `s` holds a value a wave.
template <typename T, typename F>
__device__ __forceinline__ T over_block(T x, T *s, const F &f)
{
    for (int d = 32; d > 0; d >>= 1)
        x = f(x, __shfl_xor(x, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i)
        x = f(x, s[i]);
    return x;
}

__device__ __forceinline__ float lane_of(float x, int i)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
}
__device__ __forceinline__ double lane_of(double x, int i)
{
    const u32x2 u = __builtin_bit_cast(u32x2, x);
    return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_readlane((int)u.x, i),
                                            (uint32_t)__builtin_amdgcn_readlane((int)u.y, i)});
}

// A value that at least `keep` of the block's values reach, from each thread's largest,
// for every thread: the keep-th largest of 64 groups of kWaves threads where keep is
// at most kGrouped, else of the threads themselves (the least of them where keep is the
// larger).  One wave counts, for each group, the groups that are no smaller; the
// others wait, and leave the SIMDs to other blocks.  Counted by every thread over all
// of them it was most of the kernel's time (512 rows of 100003 fp32 logits 102 us,
// 41 so).
constexpr int kGrouped = 32;
template <typename T>
__device__ __forceinline__ T bound_of(T mine, int keep, T *s_all, T *s_one)
{
    const int tid = threadIdx.x;
    s_all[tid] = mine;
    __syncthreads();
    if (tid < 64) {
        T x[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i)
            x[i] = s_all[tid + 64 * i];
        T best = -(T)kInf;
        if (keep <= kGrouped) {
            T m = x[0];
#pragma unroll
            for (int i = 1; i < kWaves; ++i)
                m = m > x[i] ? m : x[i];
            int reach = 0;
#pragma unroll 16
            for (int i = 0; i < 64; ++i)
                reach += lane_of(m, i) >= m;
            best = reach >= keep ? m : best;
        } else {
            int reach[kWaves] = {};
#pragma unroll 4
            for (int i = 0; i < 64; ++i) {
#pragma unroll
                for (int j = 0; j < kWaves; ++j) {
                    const T other = lane_of(x[j], i);
#pragma unroll
                    for (int k = 0; k < kWaves; ++k)
                        reach[k] += other >= x[k];
                }
            }
#pragma unroll
            for (int k = 0; k < kWaves; ++k)
                best = reach[k] >= keep && x[k] > best ? x[k] : best;
        }
        for (int d = 32; d > 0; d >>= 1) {
            const T other = __shfl_xor(best, d);
            best = best > other ? best : other;
        }
        if (tid == 0)
            *s_one = best;
    }
    __syncthreads();
    return *s_one;
}

// Exclusive sum of n over the threads, and the sum of all.
__device__ __forceinline__ int place_of(int n, int32_t *s, int &all)
{
    const int incl = wave_scan(n);
    __syncthreads();
    if ((threadIdx.x & 63) == 63)
        s[threadIdx.x >> 6] = incl;
    __syncthreads();
    int at = incl - n;
    all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        at += i < (int)(threadIdx.x >> 6) ? s[i] : 0;
        all += s[i];
    }
    return at;
}

template <int TYPE>
__device__ __forceinline__ float wide(const u32x4 &v, int i)
{
    if (TYPE == BEAM_F32)
        return __builtin_bit_cast(float, (uint32_t)v[i & 3]);
    const uint32_t w = v[(i >> 1) & 3];
    if (TYPE == BEAM_BF16)
        return __builtin_bit_cast(float, i & 1 ? w & 0xffff0000u : w << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w));
}

template <int TYPE>
__device__ __forceinline__ float read(const uint8_t *row, int32_t at)
{
    if (TYPE == BEAM_F32)
        return reinterpret_cast<const float *>(row)[at];
    const uint16_t x = reinterpret_cast<const uint16_t *>(row)[at];
    if (TYPE == BEAM_BF16)
        return __builtin_bit_cast(float, (uint32_t)x << 16);
    return (float)__builtin_bit_cast(_Float16, x);
}

// VECS 16-byte vectors a thread.  Rows may begin anywhere an element may: vectors lie
// on the 16-byte grid of memory, the one before a row's first element included.
template <int TYPE, int VECS>
__global__ __launch_bounds__(kThreads) void beam_rows_kernel(const BeamProblem p)
{
    constexpr int kElt = TYPE == BEAM_F32 ? 4 : 2;
    constexpr int kPer = 16 / kElt;  // values a vector
    constexpr int kPiece = kThreads * VECS * kPer;
    __shared__ float s_all[kThreads];
    __shared__ float s_value[kList];
    __shared__ int32_t s_index[kList];
    __shared__ float s_f[kWaves];
    __shared__ double s_d[kWaves];
    __shared__ int32_t s_n[kWaves];
    __shared__ float s_one;
    __shared__ int32_t s_thread[kFew], s_threads, s_found;
    __shared__ u32x4 s_raw[kFew * VECS];

    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / p.pieces;
    const int piece = blockIdx.x % p.pieces;
    const float cum = p.score[row];
    // an ended beam stands for itself, and one whose score is no number for nothing
    if ((p.done && p.done[row]) || !(__builtin_fabsf(cum) < kInf))
        return;
    const uint8_t *first = p.logits + row * p.row_bytes;
    // elements before the row in its first vector
    const int skew = (int)((uintptr_t)first & 15) / kElt;
    const uint8_t *base = first - skew * kElt;
    const int32_t vocab = p.vocab;
    const int32_t at0 = piece * kPiece - skew;  // index of the piece's first element

    // ---- the piece, -inf where the row has nothing ------------------------------
    u32x4 v[VECS];
    constexpr uint32_t kNone = TYPE == BEAM_F32 ? 0xff800000u
                                                : (TYPE == BEAM_BF16 ? 0xff80ff80u : 0xfc00fc00u);
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int32_t at = at0 + (j * kThreads + tid) * kPer;
        v[j] = u32x4{kNone, kNone, kNone, kNone};
        if (at >= 0 && at + kPer <= vocab) {
            v[j] = *reinterpret_cast<const u32x4 *>(base + (int64_t)(at + skew) * kElt);
        } else if (at + kPer > 0 && at < vocab) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (at + i < 0 || at + i >= vocab)
                    continue;
                const uint8_t *e = first + (int64_t)(at + i) * kElt;
                if (kElt == 4) {
                    v[j][i & 3] = *reinterpret_cast<const uint32_t *>(e);
                } else {
                    const uint32_t x = *reinterpret_cast<const uint16_t *>(e);
                    const uint32_t w = v[j][(i >> 1) & 3];
                    v[j][(i >> 1) & 3] = i & 1 ? (w & 0xffffu) | x << 16 : (w & 0xffff0000u) | x;
                }
            }
        }
    }
    const auto each = [&](const auto &f) {
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                f(wide<TYPE>(v[j], i), at0 + (j * kThreads + tid) * kPer + i);
    };

    // ---- the sum of exponentials, a wave's beside its largest value ---------------
    float mine = -kInf;
    each([&](float x, int) { mine = fmaxf(mine, x); });
    float top = mine;
    for (int d = 32; d > 0; d >>= 1)
        top = fmaxf(top, __shfl_xor(top, d));
    const float ref = top == -kInf ? 0.0f : top;
    // a NaN, or an infinity less itself, makes the sum no number, and the row count for nothing
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        float e[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            e[i] = __builtin_amdgcn_exp2f((wide<TYPE>(v[j], i) - ref) * kLog2e);
#pragma unroll
        for (int d = kPer / 2; d > 0; d /= 2)
#pragma unroll
            for (int i = 0; i < d; ++i)
                e[i] += e[i + d];
        sum += e[0];
    }
    for (int d = 32; d > 0; d >>= 1)
        sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) {
        s_f[tid >> 6] = ref;
        s_d[tid >> 6] = sum;
    }

    // ---- the keep best --------------------------------------------------------------
    const int keep = p.keep;
    float least = bound_of(mine, keep, s_all, &s_one);  // of the values taken
    const float wave_ref = s_f[tid & (kWaves - 1)];
    const double wave_sum = s_d[tid & (kWaves - 1)];
    // the threads whose largest reaches it: seldom more than keep
    if (tid == 0)
        s_threads = s_found = 0;
    __syncthreads();
    if (mine >= least && mine > -kInf) {
        const int i = atomicAdd(&s_threads, 1);
        if (i < kFew) {
            s_thread[i] = tid;
#pragma unroll
            for (int j = 0; j < VECS; ++j)
                s_raw[i * VECS + j] = v[j];
        }
    }
    __syncthreads();
    int n = 0, all = s_threads;
    bool listed = all <= kFew;
    if (listed) {
        // a wave a thread's values, a lane a value
        constexpr int kEach = VECS * kPer;
        const uint8_t *raw = reinterpret_cast<const uint8_t *>(s_raw);
        for (int c = tid >> 6; c < all; c += kWaves) {
            const int i = tid & 63;
            const float x = i < kEach ? read<TYPE>(raw, c * kEach + i) : -kInf;
            if (x >= least && x > -kInf) {
                const int o = atomicAdd(&s_found, 1);  // they are ranked below
                if (o < kList) {
                    s_value[o] = x;
                    s_index[o] = at0 + ((i / kPer) * kThreads + s_thread[c]) * kPer + i % kPer;
                }
            }
        }
        __syncthreads();
        all = s_found;
        listed = all <= kList;
        __syncthreads();
    }
    if (!listed) {
        // the keep-th largest value is the least that fewer than `keep` are above
        const auto above = [&](float m) {
            n = 0;
            each([&](float x, int) { n += x > m; });
        };
        above(least);
        int at = place_of(n, s_n, all);
        if (all >= keep) {
            top = over_block(top, s_f, [](float a, float b) { return fmaxf(a, b); });
            int32_t lo = ordered(least), hi = ordered(top);
            while (lo < hi) {
                const int32_t mid = (int32_t)(((int64_t)lo + hi) >> 1);
                above(value_of(mid));
                if (over_block(n, s_n, [](int a, int b) { return a + b; }) < keep)
                    hi = mid;
                else
                    lo = mid + 1;
            }
            least = value_of(lo);
            above(least);
            at = place_of(n, s_n, all);
        }
        const int more = all;
        if (n > 0) {
            each([&](float x, int i) {
                if (x > least) {
                    s_value[at] = x;
                    s_index[at++] = i;
                }
            });
        }
        // of its equals the first: a vector of all threads at a time, which lie in order
        int taken = more;
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            if (taken < keep && least > -kInf) {
                n = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    n += wide<TYPE>(v[j], i) == least;
                at = taken + place_of(n, s_n, all);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (wide<TYPE>(v[j], i) == least) {
                        if (at < keep) {
                            s_value[at] = least;
                            s_index[at] = at0 + (j * kThreads + tid) * kPer + i;
                        }
                        ++at;
                    }
                }
                taken += all;
            }
        }
        all = min(taken, keep);
    }
    __syncthreads();
    const int64_t list = row * p.pieces + piece;
    for (int c = tid; c < all; c += kThreads) {
        const float x = s_value[c];
        const int32_t i = s_index[c];
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < all; ++o)
            rank += s_value[o] > x || (s_value[o] == x && s_index[o] < i);
        if (rank < keep) {
            p.values[list * keep + rank] = x;
            p.indexes[list * keep + rank] = i;
        }
    }
    for (int r = all + tid; r < keep; r += kThreads)
        p.values[list * keep + r] = -kInf;  // its index is not read
    if (tid < kWaves) {  // a pair a wave; the second kernel joins them
        p.sums[(list * kWaves + tid) * 2] = (double)wave_ref;
        p.sums[(list * kWaves + tid) * 2 + 1] = wave_sum;
    }
}

// Candidates of a batch item are numbered by rank in their lists, then by list (beam,
// piece), so that the best of all lists are dealt to different threads: numbered as they
// lie they fell to one thread in `keep`, whose largest made a low bound (16 items of 8
// beams, 16 kept: 14.4 us, 10.0 so).  Each rank begins `pieces` threads of 64 after the one
// before, so that a good beam's lists fall to one of bound_of's groups after the other:
// with the same list first in every rank, 64 lists had all of theirs in one group each (the
// same with 8 pieces a beam: 18.2 us, 10.5 so).  Their place among equals is the beam, then
// the token.
constexpr int kHeld = 8;  // scores of candidates that a thread keeps in registers

// What LDS holds of a beam.
struct Beam {
    double lse;   // log of its sum of exponentials; NaN: it has no candidates
    float score;  // of a beam that has ended: the score of its one candidate, and lse 0
    int32_t ended;
};

// HELD: the item has at most kHeld candidates a thread, else their scores are made anew
// for each of the few passes over them.
template <bool HELD>
__global__ __launch_bounds__(kThreads) void beam_pick_kernel(const BeamProblem p)
{
    extern __shared__ Beam s_beam[];
    __shared__ double s_all[kThreads], s_one;
    __shared__ double s_score[kList];
    __shared__ int64_t s_place[kList];
    __shared__ int32_t s_n[kWaves];
    __shared__ int64_t s_top[kWaves];

    const int tid = threadIdx.x;
    const int64_t item = blockIdx.x, row0 = item * p.beams;
    const double none = -(double)kInf;
    const uint32_t keep = p.keep, lists = (uint32_t)p.pieces * p.beams, slots = lists * keep;
    const float *values = p.values + item * slots;
    const uint32_t turn = (lists - p.pieces) & 63;
    const auto list_of = [&](uint32_t i) { return (i % lists + i / lists * turn) % lists; };
    const auto where = [&](uint32_t i) { return list_of(i) * keep + i / lists; };
    float value[kHeld];
    if (HELD) {  // on their way while the sums are joined
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            value[j] = values[where(min(tid + j * kThreads, (int)slots - 1))];
    }
    // `per` lanes a beam (a power of two, at most a wave), a lane the sum of a wave's values
    int per = 64;
    while (per > 1 && per * p.beams > kThreads)
        per >>= 1;
    for (int w = tid / per; w < p.beams; w += kThreads / per) {
        const int64_t row = row0 + w;
        const int pairs = p.pieces * kWaves;
        const double *sums = p.sums + row * pairs * 2;
        const float cum = p.score[row];
        const bool ended = p.done && p.done[row], finite = __builtin_fabsf(cum) < kInf;
        const bool counts = !ended && finite;
        double top = none, sum = 0.0;
        for (int c = tid % per; c < pairs; c += per)
            if (counts && sums[c * 2 + 1] != 0.0)
                top = fmax(top, sums[c * 2]);
        for (int d = per / 2; d > 0; d >>= 1)
            top = fmax(top, __shfl_xor(top, d));
        for (int c = tid % per; c < pairs; c += per) {
            const double s = sums[c * 2 + 1];
            if (counts && s != 0.0)  // an infinite top leaves no number
                sum += s * exp(sums[c * 2] - top);
        }
        for (int d = per / 2; d > 0; d >>= 1)
            sum += __shfl_xor(sum, d);
        if (tid % per == 0)
            s_beam[w] = Beam{counts ? top + log(sum) : finite ? 0.0 : __builtin_nan(""), cum,
                             ended};
    }
    __syncthreads();

    const auto score_of = [&](uint32_t i, float x) {
        const uint32_t list = list_of(i), w = list / p.pieces;
        const Beam b = s_beam[w];
        double s = (double)b.score + ((double)x - b.lse);
        if (b.ended)  // the first of its first list
            s = i < lists && list == w * p.pieces ? (double)b.score - b.lse : none;
        return s == s ? s : none;
    };
    const auto place_at = [&](uint32_t i) {
        const uint32_t w = list_of(i) / p.pieces;
        const int32_t token = s_beam[w].ended ? p.end : p.indexes[item * slots + where(i)];
        return (int64_t)w << 32 | (uint32_t)token;
    };
    double held[kHeld];
    if (HELD) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            held[j] = none;
            if (tid + j * kThreads < slots)
                held[j] = score_of(tid + j * kThreads, value[j]);
        }
    }
    // f(score, number) for the thread's candidates
    const auto each = [&](const auto &f) {
        if (HELD) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (held[j] > none)
                    f(held[j], (uint32_t)(tid + j * kThreads));
        } else {
            for (uint32_t i = tid; i < slots; i += kThreads) {
                const double s = score_of(i, values[where(i)]);
                if (s > none)
                    f(s, i);
            }
        }
    };
    const auto count = [&](const auto &f) {
        int n = 0;
        each([&](double s, uint32_t i) { n += f(s, i); });
        return n;
    };
    double mine = none;
    each([&](double s, uint32_t) { mine = fmax(mine, s); });
    double least = bound_of(mine, (int)keep, s_all, &s_one);
    int64_t last = 0x7fffffffffffffffll;  // the last place taken of those with that score
    const auto plus = [](int a, int b) { return a + b; };
    int all;
    int at = place_of(count([&](double s, uint32_t) { return s >= least; }), s_n, all);
    if (all > kList) {
        const auto above = [&](double m) {
            return over_block(count([&](double s, uint32_t) { return s > m; }), s_n, plus);
        };
        int more = above(least);
        if (more >= (int)keep) {  // as in the pieces
            int64_t lo = ordered(least);
            int64_t hi = over_block(ordered(mine), s_top,
                                    [](int64_t a, int64_t b) { return a > b ? a : b; });
            while (lo < hi) {
                const int64_t mid = lo + (int64_t)(((uint64_t)hi - (uint64_t)lo) >> 1);
                if (above(__builtin_bit_cast(double, mid ^ ((mid >> 63) & 0x7fffffffffffffffll))) <
                    (int)keep)
                    hi = mid;
                else
                    lo = mid + 1;
            }
            least = __builtin_bit_cast(double, lo ^ ((lo >> 63) & 0x7fffffffffffffffll));
            more = above(least);
        }
        int64_t l = 0, h = ((int64_t)p.beams << 32) - 1;
        while (l < h) {
            const int64_t mid = (l + h) >> 1;
            const int c = over_block(
                count([&](double s, uint32_t i) { return s == least && place_at(i) <= mid; }), s_n,
                plus);
            if (c >= (int)keep - more)
                h = mid;
            else
                l = mid + 1;
        }
        last = l;
        at = place_of(count([&](double s, uint32_t i) {
                          return s > least || (s == least && place_at(i) <= last);
                      }),
                      s_n, all);
    }
    const bool ties = last != 0x7fffffffffffffffll;  // beyond the list
    each([&](double s, uint32_t i) {
        if (s > least || (s == least && (!ties || place_at(i) <= last))) {
            if (at < kList) {
                s_score[at] = s;
                s_place[at] = i;
            }
            ++at;
        }
    });
    __syncthreads();
    all = min(all, kList);
    for (int c = tid; c < all; c += kThreads)  // one latency for all of them
        s_place[c] = place_at((uint32_t)s_place[c]);
    __syncthreads();
    const auto put = [&](int rank, float score, int32_t parent, int32_t token, bool ended) {
        const int64_t o = item * keep + rank;
        p.new_score[o] = score;
        p.parent[o] = parent;
        p.token[o] = token;
        p.new_done[o] = ended;
    };
    for (int c = tid; c < all; c += kThreads) {
        const double s = s_score[c];
        const int64_t place = s_place[c];
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < all; ++o)
            rank += s_score[o] > s || (s_score[o] == s && s_place[o] < place);
        if (rank < (int)keep) {
            const int32_t w = (int32_t)(place >> 32), token = (int32_t)place;
            put(rank, (float)s, (int32_t)row0 + w, token, token == p.end);
        }
    }
    for (int r = all + tid; r < (int)keep; r += kThreads)
        put(r, -kInf, -1, -1, false);
}

template <int TYPE>
hipError_t launch_rows(const BeamProblem &p, int vecs, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.batch * p.beams * p.pieces));
    if (vecs == kBeamVecs)
        hipLaunchKernelGGL((beam_rows_kernel<TYPE, kBeamVecs>), grid, dim3(kThreads), 0, stream, p);
    else
        hipLaunchKernelGGL((beam_rows_kernel<TYPE, kBeamFewVecs>), grid, dim3(kThreads), 0, stream,
                           p);
    return hipGetLastError();
}

}  // namespace

// Elements a piece covers; one vector less, for a row that begins inside one.
int64_t beam_piece(int type, int vecs)
{
    return (int64_t)kThreads * vecs * (type == BEAM_F32 ? 4 : 8);
}

hipError_t launch_beam(const BeamProblem &p, int type, int vecs, hipStream_t stream)
{
    const hipError_t e = type == BEAM_F32    ? launch_rows<BEAM_F32>(p, vecs, stream)
                         : type == BEAM_BF16 ? launch_rows<BEAM_BF16>(p, vecs, stream)
                                             : launch_rows<BEAM_F16>(p, vecs, stream);
    if (e != hipSuccess)
        return e;
    const bool held = (int64_t)p.beams * p.pieces * p.keep <= kThreads * kHeld;
    const dim3 grid((unsigned)p.batch);
    const size_t lds = (size_t)p.beams * sizeof(Beam);
    if (held)
        hipLaunchKernelGGL(beam_pick_kernel<true>, grid, dim3(kThreads), lds, stream, p);
    else
        hipLaunchKernelGGL(beam_pick_kernel<false>, grid, dim3(kThreads), lds, stream, p);
    return hipGetLastError();
}

}  // namespace dps
