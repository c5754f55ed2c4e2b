// dps_attn.h -- what the attention kernels share (gfx950): matrix products and
// conversions by type, the two-term split of softmax weights, and the turn of values
// that lie token by token into matrix operands.
#pragma once

#include "dps_device.h"

namespace dps {

namespace {

constexpr int kTile = 32;               // tokens a wave takes at a time
constexpr int64_t kLongest = 0x7fffff00;  // tokens of a row (a tile past it still fits 31 bits)
constexpr float kNone = -__FLT_MAX__;   // reference score before any token: no finite one is below
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Weights are 2^(score - ref).  ref is set kLift below the largest score so far,
// and follows a larger one only once that is kRoom above ref: weights stay
// below 2^14, inside the FP16 range, the largest is at least 2^6, so that the
// FP16 terms resolve weights down to 2^-30 of it, and most tiles rescale
// nothing.
constexpr float kLift = 6.0f, kRoom = 14.0f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

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

// Two fp32 weights as two 16-bit terms each: hi and what it leaves.  BF16: both to
// nearest, within 2^-17 of the weight to either side (truncated they lost 2^-17 on
// average, and outputs came out that much nearer to zero).  FP16: both truncated,
// within 2^-21 of the weight or 2^-24.
template <int TYPE>
__device__ __forceinline__ void split2(float p0, float p1, uint32_t &hi, uint32_t &lo)
{
    if (TYPE == KV_BF16) {
        hi = narrow2<TYPE>(p0, p1);
        lo = narrow2<TYPE>(p0 - __builtin_bit_cast(float, hi << 16),
                           p1 - __builtin_bit_cast(float, hi & 0xffff0000u));
    } else {
        const auto h = __builtin_amdgcn_cvt_pkrtz(p0, p1);
        hi = __builtin_bit_cast(uint32_t, h);
        // (a multiply-add takes the 16-bit value as it is)
        lo = __builtin_bit_cast(uint32_t,
                                __builtin_amdgcn_cvt_pkrtz(__builtin_fmaf((float)h[0], -1.0f, p0),
                                                           __builtin_fmaf((float)h[1], -1.0f, p1)));
    }
}

// Over the four 16-lane quarters that share a head: each swap leaves a lane and
// its partner's value in the two results.
template <typename F>
__device__ __forceinline__ float over_quarters(float x, const F &f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    const uint32_t v = __builtin_bit_cast(
        uint32_t, f(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return f(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ __forceinline__ float quarters_max(float x)
{
    return over_quarters(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quarters_sum(float x)
{
    return over_quarters(x, [](float a, float b) { return a + b; });
}

template <int BYTES>
struct Piece;
template <>
struct Piece<16> { typedef u32x4 T; };
template <>
struct Piece<8> { typedef u32x2 T; };
template <>
struct Piece<4> { typedef uint32_t T; };
template <>
struct Piece<2> { typedef uint16_t T; };

// Bytes streamed once: loaded past the caches' retention.
template <typename T>
__device__ __forceinline__ T stream(const uint8_t *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const T *>(p));
}

template <int TYPE, bool FP8, int D, int HT>
struct Shape {
    static constexpr int kElt = FP8 ? 1 : 2;
    static constexpr int kSteps = D / 32;              // matrix steps over head_dim
    static constexpr int kKeyLoads = D * kElt / 64;    // 16-byte loads a lane per 16 tokens
    static constexpr int kAcc = D / 16;                // output tiles
    // head_dim of V in pieces of 16 lanes x W values: whole 128s, then 64, 32
    static constexpr int kP8 = D / 128;
    static constexpr int kP4 = (D % 128) / 64;
    static constexpr int kP2 = (D % 64) / 32;
    // Waves a SIMD is compiled for: 256 registers a lane, all 512 where two tiles'
    // keys and a tile's values beside the output need them.
    static constexpr int kWavesPerSimd = D * kElt >= (HT == 1 ? 512 : 192) ? 1 : 2;
};

// One piece of V (16 lanes x W values of head_dim from d0 on) of a tile's 32
// tokens, turned into W matrix operands.
template <int TYPE, bool FP8, int W>
struct VPiece {
    typedef typename Piece<W * (FP8 ? 1 : 2)>::T Raw;
    Raw raw[8];

    // values 2i (even) and 2i + 1 (odd) of tokens 2j and 2j + 1, side by side
    __device__ __forceinline__ void turn(int i, int j, uint32_t &even, uint32_t &odd) const
    {
        const uint32_t *a = reinterpret_cast<const uint32_t *>(&raw[2 * j]);
        const uint32_t *b = reinterpret_cast<const uint32_t *>(&raw[2 * j + 1]);
        if (FP8) {
            const uint32_t t = __builtin_amdgcn_perm(b[i >> 1], a[i >> 1],
                                                     i & 1 ? 0x07030602u : 0x05010400u);
            even = wide2<TYPE, false>(t);
            odd = wide2<TYPE, true>(t);
        } else {
            even = __builtin_amdgcn_perm(b[i], a[i], 0x05040100u);
            odd = __builtin_amdgcn_perm(b[i], a[i], 0x07060302u);
        }
    }
};

}  // namespace

}  // namespace dps
