// dps_attn.hip -- attention of one new token a row over the paged KV cache
// (gfx950).
//
// For row j, query head h and its key/value head: s_t = scale * q . K_t over
// the row's live tokens t, o = sum_t exp(s_t) V_t / sum_t exp(s_t), in one
// pass over K and V with a running maximum and sum per head.
//
// Bound: HBM.  A token of a key/value head is read once (2 * head_dim
// elements) for 4 * group * head_dim flops, a few flops a byte, so the kernel
// is built to keep loads in flight and never to move a byte twice:
//   - A wave takes 32 tokens of one key/value head at a time.  S^T = K Q^T and
//     O^T = V^T P^T run on 16 x 16 x 32 matrix instructions, up to 16 query
//     heads as the columns.  The lane that holds S^T of (token, head) is the
//     lane whose P^T operand needs it, so P never crosses lanes; V is turned
//     in registers (one byte permute per two values); the main loop has no LDS
//     and no barrier.
//   - Token 4 r + c of 16 sits in operand row 4 c + r.  With the cache's
//     64-byte key segments every load of a wave is then contiguous (1 KiB at
//     16 bytes a lane) for K and for V.
//   - The tokens of all rows, in units of 128 (32 a wave), form one line per
//     key/value head, cut into as many equal ranges as there are blocks:
//     ragged lengths load every CU alike, and a block writes at most two
//     partial rows however long a row is.  attn_join_kernel combines a row's
//     partials in their order, so results do not depend on timing.
//
// Precision: products and softmax in fp32.  The weights P enter the matrix
// cores as two 16-bit terms (value and remainder), which keeps them to about
// 2^-16 or better; one 16-bit term would add an error as large as the
// rounding of the output.
#include <type_traits>

#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kTile = 32;               // tokens a wave takes at a time
constexpr int kUnit = kTile * kWaves;   // tokens of a work unit
constexpr int64_t kLongest = 0x7fffff00;  // tokens of a row (a tile past it still fits 31 bits)
constexpr float kNone = -1e30f;         // reference score before any token
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Weights are 2^(score - ref).  ref is set kLift below the largest score so far,
// and follows a larger one only once that is kRoom above ref: weights stay
// below 2^14, inside the FP16 range, the largest is at least 2^6, so that the
// FP16 terms resolve weights down to 2^-30 of it, and most tiles rescale
// nothing.
constexpr float kLift = 6.0f, kRoom = 14.0f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int TYPE>
__device__ __forceinline__ f32x4 mfma32(u32x4 a, u32x4 b, f32x4 c)
{
    if (TYPE == KV_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(a), as_half8(b), c, 0, 0, 0);
}

// Two E4M3 values (half `HI` of the dword) as two 16-bit values, exactly.
template <int TYPE, bool HI>
__device__ __forceinline__ uint32_t wide2(uint32_t codes)
{
    if (TYPE == KV_BF16)
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, HI));
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, HI));
}

// Two fp32 weights as two 16-bit terms each: hi (truncated) and the rest.
template <int TYPE>
__device__ __forceinline__ void split2(float p0, float p1, uint32_t &hi, uint32_t &lo)
{
    if (TYPE == KV_BF16) {
        const uint32_t b0 = __builtin_bit_cast(uint32_t, p0);
        const uint32_t b1 = __builtin_bit_cast(uint32_t, p1);
        hi = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
        const float r0 = p0 - __builtin_bit_cast(float, b0 & 0xffff0000u);
        const float r1 = p1 - __builtin_bit_cast(float, b1 & 0xffff0000u);
        lo = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, r1),
                                   __builtin_bit_cast(uint32_t, r0), 0x07060302u);
    } else {
        const auto h = __builtin_amdgcn_cvt_pkrtz(p0, p1);
        hi = __builtin_bit_cast(uint32_t, h);
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(p0 - (float)h[0],
                                                                     p1 - (float)h[1]));
    }
}

// Largest value over the four 16-lane quarters that share a head.
__device__ __forceinline__ float quarters_ref(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarters_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

template <int BYTES>
struct Piece;
template <>
struct Piece<16> { typedef u32x4 T; };
template <>
struct Piece<8> { typedef u32x2 T; };
template <>
struct Piece<4> { typedef uint32_t T; };

// Bytes streamed once: loaded past the caches' retention.
template <typename T>
__device__ __forceinline__ T stream(const uint8_t *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const T *>(p));
}

// The live tokens [lo, hi) of row r and its table row; hi = 0: none.
struct RowSpan {
    int32_t lo, hi;
    int32_t req;
};

__device__ __forceinline__ RowSpan row_span(const AttnProblem &p, int64_t r)
{
    RowSpan s;
    s.req = p.req ? p.req[r] : (int32_t)r;
    const int64_t room = min(p.table_cols << p.log2_tokens, kLongest);
    int64_t n = p.kv_len[r];
    if (s.req < 0 || s.req >= p.requests)
        n = 0;
    n = n < 0 ? 0 : (n > room ? room : n);
    s.hi = (int32_t)n;
    s.lo = p.window > 0 && n > p.window ? (int32_t)(n - p.window) : 0;
    return s;
}

// Work units of a row (its live tokens on the grid of kUnit tokens).
__device__ __forceinline__ int32_t row_units(const RowSpan &s)
{
    return s.hi == 0 ? 0 : (int32_t)(((uint32_t)s.hi + kUnit - 1) / kUnit) - s.lo / kUnit;
}

// Range of block w of `parts` over `units` work units.
__device__ __forceinline__ int32_t range_begin(int32_t w, int32_t units, int32_t parts)
{
    return (int32_t)((int64_t)w * units / parts);
}
// The block whose range holds unit u: the last w with w * units / parts <= u.
__device__ __forceinline__ int32_t range_of(int32_t u, int32_t units, int32_t parts)
{
    return (int32_t)((((int64_t)u + 1) * parts - 1) / units);
}

// Four values of a finished row's head: o / sum, rounded once, and its lse.
template <int TYPE>
__device__ __forceinline__ void attn_store(const AttnProblem &p, int64_t row, int head, int dim,
                                           int d, f32x4 o, float ref, float sum)
{
    const float scale = sum == 0.0f ? 0.0f : p.value_scale / sum;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = o[i] * scale;
        h[i] = TYPE == KV_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v)
                               : __builtin_bit_cast(uint16_t, (_Float16)v);
    }
    uint16_t *at = static_cast<uint16_t *>(p.out) + row * p.out_stride + (int64_t)head * dim + d;
    *reinterpret_cast<u32x2 *>(at) =
        u32x2{(uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16};
    if (d == 0 && p.lse)
        p.lse[row * (p.kv_heads * p.group) + head] =
            sum == 0.0f ? -__builtin_inff() : (ref + log2f(sum)) * kLn2;
}

template <int TYPE, bool FP8, int D>
struct Shape {
    static constexpr int kElt = FP8 ? 1 : 2;
    static constexpr int kSteps = D / 32;              // matrix steps over head_dim
    static constexpr int kKeyLoads = D * kElt / 64;    // 16-byte loads a lane per 16 tokens
    static constexpr int kAcc = D / 16;                // output tiles
    // head_dim of V in pieces of 16 lanes x W values: whole 128s, then 64, 32
    static constexpr int kP8 = D / 128;
    static constexpr int kP4 = (D % 128) / 64;
    static constexpr int kP2 = (D % 64) / 32;
    // 16-bit keys of 256: two tiles' keys and a tile's values do not fit the
    // registers beside the output, so loads wait for the piece they replace and
    // the query stays in LDS (where the waves' outputs are joined later).
    static constexpr bool kTight = D * kElt >= 512;
};

// One piece of V (16 lanes x W values of head_dim from d0 on) of a tile's 32
// tokens, turned into W matrix operands.
template <int TYPE, bool FP8, int W>
struct VPiece {
    typedef typename Piece<W * (FP8 ? 1 : 2)>::T Raw;
    Raw raw[8];

    __device__ __forceinline__ uint32_t dword(int j, int i) const
    {
        // values 2i and 2i + 1 of token j as two 16-bit values
        const uint32_t *d = reinterpret_cast<const uint32_t *>(&raw[j]);
        if (!FP8)
            return d[i];
        return i & 1 ? wide2<TYPE, true>(d[i >> 1]) : wide2<TYPE, false>(d[i >> 1]);
    }
};

template <int TYPE, bool FP8, int D>
__global__ __launch_bounds__(kThreads, 2) void attn_kernel(const AttnProblem p)
{
    typedef Shape<TYPE, FP8, D> S;
    constexpr int kRow = D + 4;  // LDS floats of a head's output (padded off the banks)
    __shared__ __align__(16) float s_out[kWaves * 16 * kRow];
    __shared__ float s_ref[kWaves][16], s_sum[kWaves][16];
    __shared__ int32_t s_wave_units[kWaves];
    __shared__ int32_t s_row, s_row_first;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;   // query head of the pass (matrix column)
    const int quarter = lane >> 4;
    const int32_t w = blockIdx.x;
    const int hv = blockIdx.y;   // (key/value head, group of at most 16 query heads)
    const int kvh = hv / p.head_groups;
    const int sub = hv % p.head_groups;
    const int first_head = kvh * p.group + sub * p.group_step;
    const int n_heads = min(p.group_step, p.group - sub * p.group_step);

    // ---- this block's range of the work line --------------------------------
    // thread i sums rows [i * per, (i + 1) * per)
    const int32_t per = (int32_t)((p.rows + kThreads - 1) / kThreads);
    const int32_t r0 = min(tid * per, (int32_t)p.rows), r1 = min(r0 + per, (int32_t)p.rows);
    int32_t mine = 0;
    for (int32_t r = r0; r < r1; ++r)
        mine += row_units(row_span(p, r));
    int32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t up = __shfl_up(incl, d);
        incl += lane >= d ? up : 0;
    }
    if (lane == 63)
        s_wave_units[wave] = incl;
    __syncthreads();
    int32_t units = 0, before = incl - mine;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        before += i < wave ? s_wave_units[i] : 0;
        units += s_wave_units[i];
    }
    const int32_t parts = min((int32_t)gridDim.x, units);
    if (w == 0 && hv == 0) {  // the work line for the join
        int32_t at = before;
        for (int32_t r = r0; r < r1; ++r) {
            p.first_unit[r] = at;
            at += row_units(row_span(p, r));
        }
        if (tid == 0)
            p.first_unit[p.rows] = units;
    }
    if (w >= parts)
        return;
    const int32_t begin = range_begin(w, units, parts), end = range_begin(w + 1, units, parts);
    if (begin >= before && begin < before + mine) {
        int32_t at = before, r = r0;
        for (;; ++r) {
            const int32_t n = row_units(row_span(p, r));
            if (begin < at + n)
                break;
            at += n;
        }
        s_row = r;
        s_row_first = at;
    }
    __syncthreads();
    // wave-uniform values, kept in scalar registers
    int row = __builtin_amdgcn_readfirstlane(s_row);
    int skip = __builtin_amdgcn_readfirstlane(begin - s_row_first);  // units of the row
    int left = __builtin_amdgcn_readfirstlane(end - begin);

    const uint32_t tokens = 1u << p.log2_tokens;
    const uint32_t key_lane = (4 * (col & 3) + (col >> 2)) * 64 + quarter * 16;
    const uint32_t key_head = (uint32_t)kvh * S::kKeyLoads * tokens * 64;
    const uint32_t val_head = (uint32_t)(p.kv_heads + kvh) * tokens * (D * S::kElt);
    const float to_log2 = p.score_scale * kLog2e;

    while (left > 0 && row < p.rows) {
        const RowSpan span = row_span(p, row);
        const int lo = __builtin_amdgcn_readfirstlane(span.lo);
        const int hi = __builtin_amdgcn_readfirstlane(span.hi);
        const int req = __builtin_amdgcn_readfirstlane(span.req);
        const int row_n = hi == 0 ? 0 : (int)(((uint32_t)hi + kUnit - 1) / kUnit) - lo / kUnit;
        const int n_units = min(row_n - skip, left);
        if (n_units <= 0) {  // an empty row
            ++row;
            continue;
        }
        const int32_t *__restrict__ table = p.table + (int64_t)req * p.table_cols;
        const int unit0 = lo / kUnit + skip;

        // ---- query fragments ------------------------------------------------
        u32x4 q[S::kTight ? 1 : S::kSteps];
        u32x4 *q_lds = reinterpret_cast<u32x4 *>(&s_out[wave * 16 * kRow]) + lane;
        {
            const uint8_t *qp = static_cast<const uint8_t *>(p.q) +
                                ((int64_t)row * p.q_stride + (int64_t)(first_head + col) * D) * 2;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                // 8-bit keys hold 16 values a lane: two steps' operands side by side
                const int d = FP8 ? 64 * (s >> 1) + 16 * quarter + 8 * (s & 1)
                                  : 32 * s + 8 * quarter;
                u32x4 v = {0u, 0u, 0u, 0u};
                if (col < n_heads)
                    v = load16(qp + d * 2);
                if (S::kTight)
                    q_lds[64 * s] = v;
                else
                    q[s] = v;
            }
        }

        float ref = kNone, sum = 0.0f;
        f32x4 acc[S::kAcc];
#pragma unroll
        for (int i = 0; i < S::kAcc; ++i)
            acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

        // Base of the block that holds token t0 (a multiple of 16), at the
        // token's place in it; a block outside the pool is never read.
        const auto block_of = [&](int t0, bool &ok) -> const uint8_t * {
            int64_t c = (int64_t)((uint32_t)t0 >> p.log2_tokens);
            c = min(c, p.table_cols - 1);
            const int32_t b = table[c];
            ok = b >= 0 && b < p.n_blocks;
            return p.pool + (int64_t)(ok ? b : 0) * p.block_stride;
        };

        u32x4 key[2][S::kKeyLoads];
        VPiece<TYPE, FP8, 8> v8[S::kP8 ? S::kP8 : 1];
        VPiece<TYPE, FP8, 4> v4[1];
        VPiece<TYPE, FP8, (FP8 ? 4 : 2)> v2[1];
        const uint8_t *base[2];
        bool ok[2];

        const auto load_keys = [&](int t0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                base[h] = block_of(t0 + 16 * h, ok[h]);
                const uint32_t at = key_head + (((uint32_t)t0 + 16 * h) & (tokens - 1)) * 64;
#pragma unroll
                for (int s = 0; s < S::kKeyLoads; ++s)
                    key[h][s] = stream<u32x4>(base[h] + (at + s * tokens * 64) + key_lane);
            }
        };
        // values of piece i: [i * 128, ...) of head_dim, the last ones narrower
        const auto load_piece = [&](auto &v, int t0, int d0, int width) {
            typedef typename std::remove_reference<decltype(v)>::type::Raw Raw;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int h = j >> 2;
                const uint32_t t = (((uint32_t)t0 + 16 * h) & (tokens - 1)) + 4 * (j & 3);
                v.raw[j] = stream<Raw>(base[h] + (val_head + (t * D + d0) * S::kElt) +
                                       (quarter * D + col * width) * S::kElt);
            }
        };
        const auto load_values = [&](int t0, int first, int last) {
#pragma unroll
            for (int i = 0; i < S::kP8; ++i)
                if (i >= first && i < last)
                    load_piece(v8[i], t0, 128 * i, 8);
            if (S::kP4 && last > S::kP8)
                load_piece(v4[0], t0, 128 * S::kP8, 4);
            if (S::kP2 && last > S::kP8)
                load_piece(v2[0], t0, 128 * S::kP8 + 64 * S::kP4, 2);
        };

        const int tile0 = unit0 * kUnit + wave * kTile;
        load_keys(tile0);
        if (S::kTight)
            load_values(tile0, 0, 1);
        for (int u = 0; u < n_units; ++u) {
            const int t0 = tile0 + u * kUnit;
            const bool ok0 = ok[0], ok1 = ok[1];
            if (!S::kTight)
                load_values(t0, 0, 9);

            // ---- S^T = K Q^T -------------------------------------------------
            f32x4 s2[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s2[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) {
                    u32x4 a;
                    if (FP8) {
                        const u32x4 k16 = key[h][s >> 1];
                        const uint32_t c0 = s & 1 ? k16.z : k16.x, c1 = s & 1 ? k16.w : k16.y;
                        a = u32x4{wide2<TYPE, false>(c0), wide2<TYPE, true>(c0),
                                  wide2<TYPE, false>(c1), wide2<TYPE, true>(c1)};
                    } else {
                        a = key[h][s];
                    }
                    s2[h] = mfma32<TYPE>(a, S::kTight ? q_lds[64 * s] : q[S::kTight ? 0 : s], s2[h]);
                }
            }
            if (S::kTight) {
                __builtin_amdgcn_sched_barrier(0);
                load_values(t0, 1, 9);
            } else if (u + 1 < n_units) {
                load_keys(t0 + kUnit);
            }

            // ---- softmax over this lane's 8 tokens ----------------------------
            float x[8];
            bool live[8];
            const bool edge = t0 < lo || t0 + kTile > hi || !ok0 || !ok1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = s2[j >> 2][j & 3] * to_log2;
                live[j] = true;
            }
            if (edge) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = t0 + 16 * (j >> 2) + 4 * (j & 3) + quarter;
                    live[j] = t >= lo && t < hi && (j < 4 ? ok0 : ok1);
                    x[j] = live[j] ? x[j] : -__builtin_inff();
                }
            }
            float m = x[0];
#pragma unroll
            for (int j = 1; j < 8; ++j)
                m = fmaxf(m, x[j]);
            if (__any(m > ref + kRoom)) {
                m = fmaxf(quarters_ref(m) - kLift, ref);
                const float shrink = __builtin_amdgcn_exp2f(ref - m);
                ref = m;
                sum *= shrink;
#pragma unroll
                for (int i = 0; i < S::kAcc; ++i)
                    acc[i] *= shrink;
            }
            u32x4 p_hi, p_lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = __builtin_amdgcn_exp2f(x[j] - ref);
                sum += x[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t hi2, lo2;
                split2<TYPE>(x[2 * j], x[2 * j + 1], hi2, lo2);
                p_hi[j] = hi2;
                p_lo[j] = lo2;
            }

            // ---- O^T += V^T P^T -----------------------------------------------
            int tile = 0;
            const auto turn = [&](auto &v, int width) {
                if (edge) {
                    // whatever a place past the row holds must not meet a zero weight
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!live[j])
                            v.raw[j] = 0;
                }
#pragma unroll
                for (int i = 0; i < width / 2; ++i) {
                    uint32_t d[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        d[j] = v.dword(j, i);
                    u32x4 even, odd;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        even[j] = __builtin_amdgcn_perm(d[2 * j + 1], d[2 * j], 0x05040100u);
                        odd[j] = __builtin_amdgcn_perm(d[2 * j + 1], d[2 * j], 0x07060302u);
                    }
                    acc[tile] = mfma32<TYPE>(even, p_hi, acc[tile]);
                    acc[tile] = mfma32<TYPE>(even, p_lo, acc[tile]);
                    acc[tile + 1] = mfma32<TYPE>(odd, p_hi, acc[tile + 1]);
                    acc[tile + 1] = mfma32<TYPE>(odd, p_lo, acc[tile + 1]);
                    tile += 2;
                }
            };
#pragma unroll
            for (int i = 0; i < S::kP8; ++i) {
                turn(v8[i], 8);
                if (S::kTight && i == 0) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (u + 1 < n_units)
                        load_keys(t0 + kUnit);
                }
            }
            if (S::kP4)
                turn(v4[0], 4);
            if (S::kP2)
                turn(v2[0], 2);
            if (S::kTight) {
                __builtin_amdgcn_sched_barrier(0);
                if (u + 1 < n_units)
                    load_values(t0 + kUnit, 0, 1);
            }
        }

        // ---- join the four waves -------------------------------------------
        sum = quarters_sum(sum);
        if (quarter == 0) {
            s_ref[wave][col] = ref;
            s_sum[wave][col] = sum;
        }
        __syncthreads();
        float all = fmaxf(fmaxf(s_ref[0][col], s_ref[1][col]), fmaxf(s_ref[2][col], s_ref[3][col]));
        const float shrink = __builtin_amdgcn_exp2f(ref - all);
        {
            float *o = &s_out[(wave * 16 + col) * kRow];
            int tile = 0;
            const auto put = [&](int d0, int width) {
                // lane's rows 4 quarter + r hold values d0 + width * row + i
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < width; ++i)
                        o[d0 + width * (4 * quarter + r) + i] = acc[tile + i][r] * shrink;
                tile += width;
            };
#pragma unroll
            for (int i = 0; i < S::kP8; ++i)
                put(128 * i, 8);
            if (S::kP4)
                put(128 * S::kP8, 4);
            if (S::kP2)
                put(128 * S::kP8 + 64 * S::kP4, 2);
        }
        __syncthreads();
        const bool whole = skip == 0 && n_units == row_n;
        // at most one partial begins inside its row and one at its start
        const int64_t slot = ((int64_t)(w * 2 + (skip > 0 ? 0 : 1)) * gridDim.y + hv) * p.group_step;
        for (int i = tid; i < n_heads * (D / 4); i += kThreads) {
            const int head = i / (D / 4), d = (i % (D / 4)) * 4;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
            float m = s_ref[0][head], l = 0.0f;
#pragma unroll
            for (int k = 1; k < kWaves; ++k)
                m = fmaxf(m, s_ref[k][head]);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                o += *reinterpret_cast<const f32x4 *>(&s_out[(k * 16 + head) * kRow + d]);
                l += s_sum[k][head] * __builtin_amdgcn_exp2f(s_ref[k][head] - m);
            }
            if (whole) {
                attn_store<TYPE>(p, row, first_head + head, D, d, o, m, l);
            } else {
                *reinterpret_cast<f32x4 *>(p.part_out + (slot + head) * D + d) = o;
                if (d == 0) {
                    p.part_stat[(slot + head) * 2] = m;
                    p.part_stat[(slot + head) * 2 + 1] = l;
                }
            }
        }
        __syncthreads();
        left -= n_units;
        ++row;
        skip = 0;
    }
}

// Combines a row's partials, one block per (row, head group), in the order of
// the blocks that made them; rows without tokens get zeros.  A row that one
// block finished is left as it is.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(const AttnProblem p, int blocks,
                                                             int dim)
{
    const int64_t row = blockIdx.x;
    const int hv = blockIdx.y;
    const int kvh = hv / p.head_groups;
    const int sub = hv % p.head_groups;
    const int first_head = kvh * p.group + sub * p.group_step;
    const int n_heads = min(p.group_step, p.group - sub * p.group_step);
    const int32_t units = p.first_unit[p.rows];
    const int32_t parts = min(blocks, units);
    const int32_t u0 = p.first_unit[row], u1 = p.first_unit[row + 1];
    int32_t w0 = 0, count = 0;
    if (u1 > u0) {
        w0 = range_of(u0, units, parts);
        count = range_of(u1 - 1, units, parts) - w0 + 1;
        if (count == 1)
            return;
    }
    for (int i = threadIdx.x; i < n_heads * (dim / 4); i += kThreads) {
        const int head = i / (dim / 4), d = (i % (dim / 4)) * 4;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        float ref = kNone, sum = 0.0f;
        for (int k = 0; k < count; ++k) {
            // the row's first partial begins at its start, the others inside it
            const int64_t slot =
                ((int64_t)((w0 + k) * 2 + (k == 0 ? 1 : 0)) * gridDim.y + hv) * p.group_step + head;
            const f32x4 part = *reinterpret_cast<const f32x4 *>(p.part_out + slot * dim + d);
            const float r = p.part_stat[slot * 2], l = p.part_stat[slot * 2 + 1];
            const float to = fmaxf(ref, r);
            const float a = __builtin_amdgcn_exp2f(ref - to), b = __builtin_amdgcn_exp2f(r - to);
            o = o * a + part * b;
            sum = sum * a + l * b;
            ref = to;
        }
        attn_store<TYPE>(p, row, first_head + head, dim, d, o, ref, sum);
    }
}

template <int TYPE, bool FP8, int D>
hipError_t launch(const AttnProblem &p, int blocks, hipStream_t stream)
{
    const int heads = p.kv_heads * p.head_groups;
    hipLaunchKernelGGL((attn_kernel<TYPE, FP8, D>), dim3((unsigned)blocks, (unsigned)heads),
                       dim3(kThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((attn_join_kernel<TYPE>), dim3((unsigned)p.rows, (unsigned)heads),
                       dim3(kThreads), 0, stream, p, blocks, D);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_type(const AttnProblem &p, bool fp8, int dim, int blocks, hipStream_t stream)
{
    switch (dim) {
    case 64: return fp8 ? launch<TYPE, true, 64>(p, blocks, stream)
                        : launch<TYPE, false, 64>(p, blocks, stream);
    case 96: return fp8 ? hipErrorInvalidValue : launch<TYPE, false, 96>(p, blocks, stream);
    case 128: return fp8 ? launch<TYPE, true, 128>(p, blocks, stream)
                         : launch<TYPE, false, 128>(p, blocks, stream);
    case 192: return fp8 ? launch<TYPE, true, 192>(p, blocks, stream)
                         : launch<TYPE, false, 192>(p, blocks, stream);
    case 256: return fp8 ? launch<TYPE, true, 256>(p, blocks, stream)
                         : launch<TYPE, false, 256>(p, blocks, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_attn(const AttnProblem &p, int type, bool fp8, int dim, int blocks,
                       hipStream_t stream)
{
    return type == KV_BF16 ? launch_type<KV_BF16>(p, fp8, dim, blocks, stream)
                           : launch_type<KV_F16>(p, fp8, dim, blocks, stream);
}

}  // namespace dps
