// dps_kv.hip -- what fills the paged KV cache (gfx950): a step's block tables
// and slot maps from request lengths, and the store of keys and values with
// the per-head norms and the rotation of queries and keys in the same pass.
#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMapRows = 1024;  // rows of a block of kv_map_kernel

// ---- step maps ------------------------------------------------------------------
// With c = ctx_len, n = new_len of a request and B(x) = ceil(x / T): it takes
// B(c + n) - B(c) blocks off the list, and its i-th new token sits at position
// c + i.  Two prefix sums over the requests (new tokens, new blocks) say where
// each request's rows and blocks begin; a row then finds its request by
// bisection.
//
// Bound: latency (20 bytes a row; a step of 256 rows moves 12 KB).  One launch:
// every block sums the requests anew into its LDS, which costs it two reads of
// the length arrays from L2, instead of a second launch that would wait for
// the first.

struct Lengths {
    int32_t have;  // blocks held before the step
    int32_t need;  // blocks to take
    int32_t ctx, fresh;  // tokens before the step, new tokens
};

__device__ __forceinline__ Lengths lengths(const KvMapProblem &p, int r)
{
    const int64_t round = (int64_t(1) << p.log2_tokens) - 1;
    const int64_t c = max(p.ctx_len[r], 0);
    const int64_t n = min((int64_t)max(p.new_len[r], 0), (int64_t)0x7fffffff - c);
    Lengths l;
    l.ctx = (int32_t)c;
    l.fresh = (int32_t)n;
    // a table row holds table_cols blocks: none are taken past them
    l.have = (int32_t)min((c + round) >> p.log2_tokens, p.table_cols);
    l.need = (int32_t)min((c + n + round) >> p.log2_tokens, p.table_cols) - l.have;
    return l;
}

// The last i in [0, n) with first[i] <= x; first[0] <= x.
__device__ __forceinline__ int last_from(const int32_t *first, int n, int32_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void kv_map_kernel(const KvMapProblem p)
{
    extern __shared__ int32_t s_first[];
    int32_t *s_row = s_first;                  // [requests + 1] first row
    int32_t *s_block = s_first + p.requests + 1;  // [requests + 1] first new block
    __shared__ int64_t s_rows[kWaves];
    __shared__ int32_t s_blocks[kWaves];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int r0 = min(tid * per, p.requests), r1 = min(r0 + per, p.requests);
    int64_t rows = 0;
    int32_t blocks = 0;
    for (int r = r0; r < r1; ++r) {
        const Lengths l = lengths(p, r);
        rows += l.fresh;
        blocks += l.need;
    }
    int64_t row_incl = rows;
    int32_t block_incl = blocks;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t a = __shfl_up(row_incl, d);
        const int32_t b = __shfl_up(block_incl, d);
        if (lane >= d) {
            row_incl += a;
            block_incl += b;
        }
    }
    if (lane == 63) {
        s_rows[wave] = row_incl;
        s_blocks[wave] = block_incl;
    }
    __syncthreads();
    int64_t row_at = row_incl - rows, all_rows = 0;
    int32_t block_at = block_incl - blocks, all_blocks = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        row_at += i < wave ? s_rows[i] : 0;
        block_at += i < wave ? s_blocks[i] : 0;
        all_rows += s_rows[i];
        all_blocks += s_blocks[i];
    }
    for (int r = r0; r < r1; ++r) {
        const Lengths l = lengths(p, r);
        s_row[r] = (int32_t)min(row_at, (int64_t)p.rows);
        s_block[r] = block_at;
        if (blockIdx.x == 0) {
            p.q_start[r] = s_row[r];
            p.seq_len[r] = l.ctx + l.fresh;
        }
        row_at += l.fresh;
        block_at += l.need;
    }
    if (blockIdx.x == 0 && tid == 0) {
        p.q_start[p.requests] = (int32_t)min(all_rows, (int64_t)p.rows);
        p.counts[0] = (int32_t)min(all_rows, (int64_t)0x7fffffff);
        p.counts[1] = all_blocks;
    }
    __syncthreads();

    // new blocks into the tables
    for (int64_t i = (int64_t)blockIdx.x * kThreads + tid; i < all_blocks;
         i += (int64_t)gridDim.x * kThreads) {
        const int r = last_from(s_block, p.requests, (int32_t)i);
        const int64_t col = lengths(p, r).have + (i - s_block[r]);
        p.table[(int64_t)r * p.table_cols + col] = i < p.n_fresh ? p.fresh[i] : -1;
    }

    // rows
    const int64_t first = (int64_t)blockIdx.x * kMapRows;
    for (int64_t j = first + tid; j < min(first + kMapRows, (int64_t)p.rows); j += kThreads) {
        int32_t pos = 0, req = -1;
        int64_t slot = -1;
        if (j < all_rows) {
            req = last_from(s_row, p.requests, (int32_t)j);
            const Lengths l = lengths(p, req);
            pos = l.ctx + ((int32_t)j - s_row[req]);
            const int32_t col = pos >> p.log2_tokens;
            int32_t block = -1;
            if (col < l.have) {  // a block the request held before
                block = p.table[(int64_t)req * p.table_cols + col];
            } else if (col < p.table_cols) {
                const int64_t i = (int64_t)s_block[req] + (col - l.have);
                block = i < p.n_fresh ? p.fresh[i] : -1;
            }
            if (block >= 0)
                slot = ((int64_t)block << p.log2_tokens) + (pos & ((1 << p.log2_tokens) - 1));
        }
        p.pos[j] = pos;
        p.slot[j] = slot;
        p.req[j] = req;
        p.kv_len[j] = req < 0 ? 0 : pos + 1;
    }
}

// ---- store ------------------------------------------------------------------------
// Per query and key head: y = x * rsqrt(mean(x^2) + eps) * w, then over the
// first rot values the pairs (a, b) turn to (a cos - b sin, b cos + a sin).
// fp32 throughout, rounded once at the end.
//
// Bound: HBM for prompts (each value read and written once), latency for a
// decode step.  A head is the work of a group of head_dim / 16 lanes (rounded
// up to a power of two), 16 values a lane in two 16-byte chunks.  With pairs
// (i, i + rot / 2) a lane takes chunks j and j + rot / 16, so both values of
// every pair are its own and the only exchange is the sum of squares.

template <int TYPE>
__device__ __forceinline__ float wide(uint16_t v)
{
    if (TYPE == KV_BF16)
        return __builtin_bit_cast(float, (uint32_t)v << 16);
    return (float)__builtin_bit_cast(_Float16, v);
}

template <int TYPE>
__device__ __forceinline__ uint16_t narrow(float v)
{
    return TYPE == KV_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v)
                           : __builtin_bit_cast(uint16_t, (_Float16)v);
}

template <int TYPE>
__device__ __forceinline__ void widen8(u32x4 raw, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = wide<TYPE>((uint16_t)raw[i]);
        x[2 * i + 1] = wide<TYPE>((uint16_t)(raw[i] >> 16));
    }
}

template <int TYPE>
__device__ __forceinline__ u32x4 narrow8(const float *x)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = (uint32_t)narrow<TYPE>(x[2 * i]) | (uint32_t)narrow<TYPE>(x[2 * i + 1]) << 16;
    return r;
}

// Eight values / scale as E4M3 codes, nearest even, clamped to +-448 (NaN stays).
__device__ __forceinline__ u32x2 codes8(const float *x, float inv_scale)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = x[i] * inv_scale;
        y[i] = v > 448.0f ? 448.0f : (v < -448.0f ? -448.0f : v);
    }
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int c = 0;
        c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], c, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], c, true);
        r[i] = (uint32_t)c;
    }
    return r;
}

template <int TYPE, bool FP8, int D>
__global__ __launch_bounds__(kThreads) void kv_store_kernel(const KvStoreProblem p)
{
    constexpr int kLanes = D / 16;  // lanes with work in a group
    constexpr int kGroup = kLanes <= 4 ? 4 : (kLanes <= 8 ? 8 : 16);
    constexpr int kElt = FP8 ? 1 : 2;
    const int j = threadIdx.x % kGroup;
    const int kv_heads = p.cache.kv_heads;
    const int64_t per_row = p.heads + 2 * (int64_t)kv_heads;
    const int64_t items = p.rows * per_row;
    const int64_t step = (int64_t)gridDim.x * (kThreads / kGroup);
    for (int64_t it = (int64_t)blockIdx.x * (kThreads / kGroup) + threadIdx.x / kGroup; it < items;
         it += step) {
        const int64_t row = it / per_row;
        const int head = (int)(it - row * per_row);
        const bool is_q = head < p.heads, is_v = head >= p.heads + kv_heads;
        const bool works = j < kLanes;
        const bool turns = !is_v && p.rope && 16 * j < p.rot;
        // the lane's two chunks of eight values
        const bool split = turns && !p.adjacent;
        const int c0 = split ? j : 2 * j, c1 = split ? j + p.rot / 16 : 2 * j + 1;
        float x[16];
        if (works) {
            const uint16_t *src = p.qkv + row * p.qkv_stride + (int64_t)head * D;
            widen8<TYPE>(load16(src + 8 * c0), x);
            widen8<TYPE>(load16(src + 8 * c1), x + 8);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = 0.0f;
        }
        const uint16_t *weight = is_q ? p.q_weight : p.k_weight;
        if (!is_v && weight) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                ss += x[i] * x[i];
#pragma unroll
            for (int d = 1; d < kGroup; d <<= 1)
                ss += __shfl_xor(ss, d, kGroup);
            const float inv = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
            if (works) {
                float w[16];
                widen8<TYPE>(load16(weight + 8 * c0), w);
                widen8<TYPE>(load16(weight + 8 * c1), w + 8);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = x[i] * inv * w[i];
            }
        }
        if (turns) {
            const int64_t pos = p.pos[row];
            float cs[8], sn[8];
            if (pos >= 0 && pos < p.max_pos) {
                const float *at = p.rope + pos * p.rot + 8 * j;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    cs[i] = at[i];
                    sn[i] = at[i + p.rot / 2];
                }
            } else {  // no such angle: the row is not a number rather than wrong
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    cs[i] = sn[i] = __builtin_nanf("");
            }
            if (p.adjacent) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = x[2 * i], b = x[2 * i + 1];
                    x[2 * i] = a * cs[i] - b * sn[i];
                    x[2 * i + 1] = b * cs[i] + a * sn[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = x[i], b = x[i + 8];
                    x[i] = a * cs[i] - b * sn[i];
                    x[i + 8] = b * cs[i] + a * sn[i];
                }
            }
        }
        if (!works)
            continue;
        if (is_q) {
            uint16_t *dst = p.q_out + row * p.q_out_stride + (int64_t)head * D;
            *reinterpret_cast<u32x4 *>(dst + 8 * c0) = narrow8<TYPE>(x);
            *reinterpret_cast<u32x4 *>(dst + 8 * c1) = narrow8<TYPE>(x + 8);
            continue;
        }
        const int kvh = head - p.heads - (is_v ? kv_heads : 0);
        if (!is_v && p.k_out) {
            uint16_t *dst = p.k_out + row * p.k_out_stride + (int64_t)kvh * D;
            *reinterpret_cast<u32x4 *>(dst + 8 * c0) = narrow8<TYPE>(x);
            *reinterpret_cast<u32x4 *>(dst + 8 * c1) = narrow8<TYPE>(x + 8);
        }
        const int64_t slot = p.slot[row];
        const int64_t tokens = int64_t(1) << p.cache.log2_tokens;
        const int64_t block = slot >> p.cache.log2_tokens;
        if (slot < 0 || block >= p.cache.n_blocks)
            continue;
        const int64_t t = slot & (tokens - 1);
        uint8_t *base = p.cache.pool + block * p.cache.block_stride;
        const float inv_scale = FP8 ? 1.0f / (is_v ? p.cache.v_scale : p.cache.k_scale) : 1.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = 8 * kElt * (h ? c1 : c0);  // byte in the row
            uint8_t *dst =
                is_v ? base + ((kv_heads + kvh) * tokens + t) * (D * kElt) + at
                     : base + ((int64_t)kvh * (D * kElt / 64) + at / 64) * tokens * 64 + t * 64 +
                           at % 64;
            if (FP8)
                *reinterpret_cast<u32x2 *>(dst) = codes8(x + 8 * h, inv_scale);
            else
                *reinterpret_cast<u32x4 *>(dst) = narrow8<TYPE>(x + 8 * h);
        }
    }
}

template <int TYPE, bool FP8, int D>
hipError_t store(const KvStoreProblem &p, hipStream_t stream)
{
    constexpr int lanes = D / 16, group = lanes <= 4 ? 4 : (lanes <= 8 ? 8 : 16);
    const int64_t items = p.rows * (p.heads + 2 * (int64_t)p.cache.kv_heads);
    int64_t blocks = (items * group + kThreads - 1) / kThreads;
    if (blocks > (1 << 20))
        blocks = 1 << 20;
    hipLaunchKernelGGL((kv_store_kernel<TYPE, FP8, D>), dim3((unsigned)blocks), dim3(kThreads), 0,
                       stream, p);
    return hipGetLastError();
}

template <int TYPE>
hipError_t store_type(const KvStoreProblem &p, bool fp8, hipStream_t stream)
{
    switch (p.cache.dim) {
    case 64: return fp8 ? store<TYPE, true, 64>(p, stream) : store<TYPE, false, 64>(p, stream);
    case 96: return fp8 ? hipErrorInvalidValue : store<TYPE, false, 96>(p, stream);
    case 128: return fp8 ? store<TYPE, true, 128>(p, stream) : store<TYPE, false, 128>(p, stream);
    case 192: return fp8 ? store<TYPE, true, 192>(p, stream) : store<TYPE, false, 192>(p, stream);
    case 256: return fp8 ? store<TYPE, true, 256>(p, stream) : store<TYPE, false, 256>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv_map(const KvMapProblem &p, hipStream_t stream)
{
    const int64_t blocks = p.rows > kMapRows ? ((int64_t)p.rows + kMapRows - 1) / kMapRows : 1;
    hipLaunchKernelGGL(kv_map_kernel, dim3((unsigned)blocks), dim3(kThreads),
                       2 * (p.requests + 1) * sizeof(int32_t), stream, p);
    return hipGetLastError();
}

hipError_t launch_kv_store(const KvStoreProblem &p, int type, bool fp8, hipStream_t stream)
{
    return type == KV_BF16 ? store_type<KV_BF16>(p, fp8, stream)
                           : store_type<KV_F16>(p, fp8, stream);
}

}  // namespace dps
