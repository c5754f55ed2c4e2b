// dps_beam.hip -- the next beams from logits over the vocabulary (gfx950).
//
// Beam w of a batch item, token t:  score = cum_w + (x_wt - log sum_t exp x_wt).
// The `keep` best over all beams and tokens, of equal ones those with the lowest
// (w, t).  Within a beam the order is that of the logits alone, so a piece of a
// row can give up all but its `keep` best before the row's sum is known.
//
// Two launches.  The first reads every logit once: a block of threads holds a piece
// of a row in registers, sums its exponentials and lists its best.  The second, a
// block a batch item, joins the sums and picks from the lists.
//
// Bound: HBM for the first where rows are many (2 or 4 bytes a logit), else latency.
//
// The best of a piece: the keep-th largest of the threads' maxima is a bound that
// `keep` values reach at least; what reaches it (hardly more than that, of values
// in no order) is listed in LDS and ranked.  Where ties or an order in the data bring
// more than the list holds, the keep-th best value, and the last index among its
// equals, are found by bisection over the register values: exact whatever the data.
//
// Precision: exponentials in fp32 of differences from the piece's largest (of which
// none is above 0), the values of a 16-byte vector added in fp32, in pairs; their
// sums, log and scores in 64 bits, since candidates of different beams may lie closer
// than fp32 tells apart.  A sum is good to 2^-21 of itself: 3 roundings of 2^-24 in
// the pairs, 2^-23 of the exponential, and 3 of 2^-24 |d| e^d (at most 0.37 of that) in
// its argument d.
#include <type_traits>

#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kList = 1024;
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

// The keep-th largest of the threads' values (the smallest where there are fewer
// threads), for every thread.  Equal ones rank by thread.
template <typename T>
__device__ __forceinline__ T nth_of_threads(T mine, int keep, T *s_all, T *s_one)
{
    const int tid = threadIdx.x;
    s_all[tid] = mine;
    __syncthreads();
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < kThreads; ++i) {
        const T other = s_all[i];
        rank += other > mine || (other == mine && i < tid);
    }
    if (rank == min(keep, kThreads) - 1)
        *s_one = mine;
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

    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / p.pieces;
    const int piece = blockIdx.x % p.pieces;
    const float cum = p.score[row];
    // an ended beam stands for itself, and one whose score is no number for nothing
    if ((p.done && p.done[row]) || !(__builtin_fabsf(cum) < kInf))
        return;
    const uint8_t *first = p.logits + row * p.row_bytes;
    const int skew = (int)((uintptr_t)first & 15) / kElt;  // elements before the row in its first vector
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
            v[j] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4 *>(base + (int64_t)(at + skew) * kElt));
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

    // ---- the sum of exponentials -------------------------------------------------
    float mine = -kInf;
    each([&](float x, int) { mine = fmaxf(mine, x); });
    const float top = over_block(mine, s_f, [](float a, float b) { return fmaxf(a, b); });
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
    const double total = over_block(sum, s_d, [](double a, double b) { return a + b; });

    // ---- the keep best --------------------------------------------------------------
    const int keep = p.keep;
    const float bound = nth_of_threads(mine, keep, s_all, &s_one);
    int n = 0;
    each([&](float x, int) { n += x >= bound && x > -kInf; });
    int all;
    int at = place_of(n, s_n, all);
    int32_t least = ordered(bound), last = 0x7fffffff;  // of the values taken: the least, its last index
    if (all > kList) {
        // the keep-th largest value: the largest that `keep` values reach
        int32_t lo = least, hi = ordered(top);
        while (lo < hi) {
            const int32_t mid = (int32_t)(((int64_t)lo + hi + 1) >> 1);
            const float m = value_of(mid);
            int c = 0;
            each([&](float x, int) { c += x >= m; });
            c = over_block(c, s_n, [](int a, int b) { return a + b; });
            if (c >= keep)
                lo = mid;
            else
                hi = mid - 1;
        }
        least = lo;
        const float m = value_of(least);
        int more = 0;
        each([&](float x, int) { more += x > m; });
        more = over_block(more, s_n, [](int a, int b) { return a + b; });
        // of its equals the first keep - more: the lowest index that as many do not pass
        int32_t l = 0, h = vocab - 1;
        while (l < h) {
            const int32_t mid = (l + h) >> 1;
            int c = 0;
            each([&](float x, int i) { c += x == m && i <= mid; });
            c = over_block(c, s_n, [](int a, int b) { return a + b; });
            if (c >= keep - more)
                h = mid;
            else
                l = mid + 1;
        }
        last = l;
        n = 0;
        each([&](float x, int i) { n += x > m || (x == m && i <= last); });
        at = place_of(n, s_n, all);
    }
    const float m = value_of(least);
    each([&](float x, int i) {
        if ((x > m || (x == m && i <= last)) && x > -kInf) {
            if (at < kList) {
                s_value[at] = x;
                s_index[at] = i;
            }
            ++at;
        }
    });
    __syncthreads();
    all = min(all, kList);
    const int64_t list = row * p.pieces + piece;
    for (int c = tid; c < all; c += kThreads) {
        const float x = s_value[c];
        const int32_t i = s_index[c];
        int rank = 0;
        for (int o = 0; o < all; ++o)
            rank += s_value[o] > x || (s_value[o] == x && s_index[o] < i);
        if (rank < keep) {
            p.values[list * keep + rank] = x;
            p.indexes[list * keep + rank] = i;
        }
    }
    if (tid == 0) {
        p.sums[list * 2] = (double)ref;
        p.sums[list * 2 + 1] = total;
        p.listed[list] = min(all, keep);
    }
}

// A candidate: its place among all of its batch item is beam * vocab + token.
struct Candidate {
    double score;
    int64_t place;
};
__device__ __forceinline__ bool before(double a, int64_t pa, double b, int64_t pb)
{
    return a > b || (a == b && pa < pb);
}

__global__ __launch_bounds__(kThreads) void beam_pick_kernel(const BeamProblem p)
{
    extern __shared__ double s_lse[];  // a beam's log of the sum; NaN: it counts for nothing
    __shared__ double s_all[kThreads], s_one;
    __shared__ double s_score[kList];
    __shared__ int64_t s_place[kList];
    __shared__ int32_t s_n[kWaves];
    __shared__ int64_t s_top[kWaves];

    const int tid = threadIdx.x;
    const int64_t item = blockIdx.x, row0 = item * p.beams;
    const double none = -(double)kInf;
    for (int w = tid; w < p.beams; w += kThreads) {
        const int64_t row = row0 + w;
        const float cum = p.score[row];
        double lse = __builtin_nan("");
        if (!(p.done && p.done[row]) && __builtin_fabsf(cum) < kInf) {
            double top = none;
            for (int c = 0; c < p.pieces; ++c) {
                const int64_t list = row * p.pieces + c;
                if (p.sums[list * 2 + 1] != 0.0)
                    top = fmax(top, p.sums[list * 2]);
            }
            double sum = 0.0;
            for (int c = 0; c < p.pieces; ++c) {
                const int64_t list = row * p.pieces + c;
                const double s = p.sums[list * 2 + 1];
                if (s != 0.0)
                    sum += s * exp(p.sums[list * 2] - top);
            }
            lse = top + log(sum);
        }
        s_lse[w] = lse;
    }
    __syncthreads();

    const int keep = p.keep;
    const int64_t slots = (int64_t)p.beams * p.pieces * keep;
    const auto candidate = [&](int64_t i) {
        Candidate c = {none, 0};
        const int64_t list = i / keep;
        const int k = (int)(i % keep), w = (int)(list / p.pieces);
        const int64_t row = row0 + w;
        if (p.done && p.done[row]) {
            const float cum = p.score[row];
            if (i % ((int64_t)p.pieces * keep) == 0 && __builtin_fabsf(cum) < kInf)
                c = Candidate{(double)cum, (int64_t)w * p.vocab + p.end};
            return c;
        }
        const double lse = s_lse[w];
        if (lse != lse)
            return c;
        const int64_t at = row0 * p.pieces + list;
        if (k >= p.listed[at])
            return c;
        const double s = (double)p.score[row] + ((double)p.values[at * keep + k] - lse);
        if (s == s)
            c = Candidate{s, (int64_t)w * p.vocab + p.indexes[at * keep + k]};
        return c;
    };
    double mine = none;
    for (int64_t i = tid; i < slots; i += kThreads)
        mine = fmax(mine, candidate(i).score);
    const double bound = nth_of_threads(mine, keep, s_all, &s_one);
    const auto count = [&](const auto &f) {
        int n = 0;
        for (int64_t i = tid; i < slots; i += kThreads) {
            const Candidate c = candidate(i);
            n += c.score > none && f(c);
        }
        return n;
    };
    const auto plus = [](int a, int b) { return a + b; };
    int all;
    int at = place_of(count([&](const Candidate &c) { return c.score >= bound; }), s_n, all);
    double least = bound;
    int64_t last = 0x7fffffffffffffffll;
    if (all > kList) {
        // as in the pieces: the keep-th best score, then the last place among its equals
        int64_t lo = ordered(bound);
        int64_t hi = over_block(ordered(mine), s_top,
                                [](int64_t a, int64_t b) { return a > b ? a : b; });
        while (lo < hi) {
            const int64_t mid = lo + (int64_t)(((uint64_t)hi - (uint64_t)lo + 1) >> 1);
            const int c = over_block(
                count([&](const Candidate &x) { return ordered(x.score) >= mid; }), s_n, plus);
            if (c >= keep)
                lo = mid;
            else
                hi = mid - 1;
        }
        least = __builtin_bit_cast(double, lo ^ ((lo >> 63) & 0x7fffffffffffffffll));
        const int more =
            over_block(count([&](const Candidate &x) { return x.score > least; }), s_n, plus);
        int64_t l = 0, h = (int64_t)p.beams * p.vocab - 1;
        while (l < h) {
            const int64_t mid = (l + h) >> 1;
            const int c = over_block(count([&](const Candidate &x) {
                                         return x.score == least && x.place <= mid;
                                     }),
                                     s_n, plus);
            if (c >= keep - more)
                h = mid;
            else
                l = mid + 1;
        }
        last = l;
        at = place_of(count([&](const Candidate &c) {
                          return c.score > least || (c.score == least && c.place <= last);
                      }),
                      s_n, all);
    }
    for (int64_t i = tid; i < slots; i += kThreads) {
        const Candidate c = candidate(i);
        if (c.score > none && (c.score > least || (c.score == least && c.place <= last))) {
            if (at < kList) {
                s_score[at] = c.score;
                s_place[at] = c.place;
            }
            ++at;
        }
    }
    __syncthreads();
    all = min(all, kList);
    const auto put = [&](int rank, float score, int32_t parent, int32_t token, bool ended) {
        const int64_t o = item * keep + rank;
        p.new_score[o] = score;
        p.parent[o] = parent;
        p.token[o] = token;
        p.new_done[o] = ended;
    };
    for (int c = tid; c < all; c += kThreads) {
        const double s = s_score[c];
        const int64_t at_ = s_place[c];
        int rank = 0;
        for (int o = 0; o < all; ++o)
            rank += before(s_score[o], s_place[o], s, at_);
        if (rank < keep) {
            const int32_t w = (int32_t)(at_ / p.vocab), token = (int32_t)(at_ % p.vocab);
            put(rank, (float)s, (int32_t)row0 + w, token, token == p.end);
        }
    }
    for (int r = all + tid; r < keep; r += kThreads)
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
    hipLaunchKernelGGL(beam_pick_kernel, dim3((unsigned)p.batch), dim3(kThreads),
                       (size_t)p.beams * 8, stream, p);
    return hipGetLastError();
}

}  // namespace dps
