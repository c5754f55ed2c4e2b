// dps_kv.hip -- what fills the paged KV cache (gfx950): a step's block tables
// and slot maps from request lengths, and the store of keys and values with
// the per-head norms and the rotation of queries and keys in the same pass.
#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;

// ---- step maps ------------------------------------------------------------------
// With c = ctx_len, n = new_len of a request and B(x) = ceil(x / T): it takes
// B(c + n) - B(c) blocks off the list, and its i-th new token sits at position
// c + i.  Two prefix sums over the requests (new tokens, new blocks) say where
// each request's rows and blocks begin; a row then finds its request by
// bisection.
//
// Bound: latency (20 bytes a row; a step of 256 rows moves 12 KB).  One launch:
// every block sums the requests anew into its LDS, which costs it a read of the
// length arrays from L2, instead of a second launch that would wait for the
// first; a thread then has one row.  Past 256 requests the blocks are of 1024
// threads, so that a thread sums 4 requests at most.  MI355X, kernel time: 8
// requests that decode 2.5 us, 256 3.3, 201 prompts of 92000 tokens (2.6 MB) 4.5,
// where an empty launch takes 1.5.

struct Lengths {
    int32_t have;        // blocks held before the step
    int32_t need;        // blocks to take
    int32_t ctx, fresh;  // tokens before the step, new tokens
};

// Blocks of n tokens, as far as a table row holds them.
__device__ __forceinline__ int32_t held(const KvMapProblem &p, int64_t n)
{
    const int64_t round = (int64_t(1) << p.log2_tokens) - 1;
    return (int32_t)min((n + round) >> p.log2_tokens, p.table_cols);
}

__device__ __forceinline__ Lengths lengths(const KvMapProblem &p, int r)
{
    const int64_t c = max(p.ctx_len[r], 0);
    const int64_t n = min((int64_t)max(p.new_len[r], 0), (int64_t)0x7fffffff - c);
    Lengths l;
    l.ctx = (int32_t)c;
    l.fresh = (int32_t)n;
    l.have = held(p, c);
    l.need = held(p, c + n) - l.have;
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

template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_map_kernel(const KvMapProblem p)
{
    constexpr int kWaves = THREADS / 64;
    constexpr int kMost = THREADS == 256 ? 1 : 4;  // requests a thread
    __shared__ int32_t s_row[THREADS * kMost];    // first row of a request
    __shared__ int32_t s_block[THREADS * kMost];  // its first new block
    __shared__ int32_t s_ctx[THREADS * kMost];
    __shared__ int32_t s_low[kWaves], s_high[kWaves], s_blocks[kWaves];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // thread i has requests [i * per, (i + 1) * per)
    const int per = (p.requests + THREADS - 1) / THREADS;
    const int r0 = tid * per;
    Lengths l[kMost];
    int32_t low = 0, high = 0, blocks = 0;  // new tokens in two halves: their sum passes 32 bits
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        l[i] = Lengths{0, 0, 0, 0};
        if (i < per && r0 + i < p.requests)
            l[i] = lengths(p, r0 + i);
        low += l[i].fresh & 0xffff;
        high += l[i].fresh >> 16;
        blocks += l[i].need;
    }
    const int32_t low_incl = wave_scan(low), high_incl = wave_scan(high);
    const int32_t block_incl = wave_scan(blocks);
    if (lane == 63) {
        s_low[wave] = low_incl;
        s_high[wave] = high_incl;
        s_blocks[wave] = block_incl;
    }
    __syncthreads();
    int32_t low_at = low_incl - low, high_at = high_incl - high;
    int32_t block_at = block_incl - blocks, all_low = 0, all_high = 0, all_blocks = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        low_at += i < wave ? s_low[i] : 0;
        high_at += i < wave ? s_high[i] : 0;
        block_at += i < wave ? s_blocks[i] : 0;
        all_low += s_low[i];
        all_high += s_high[i];
        all_blocks += s_blocks[i];
    }
    int64_t row_at = ((int64_t)high_at << 16) + low_at;
    const int64_t all_rows = ((int64_t)all_high << 16) + all_low;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int r = r0 + i;
        if (i < per && r < p.requests) {
            const int32_t first = (int32_t)min(row_at, (int64_t)p.rows);
            s_row[r] = first;
            s_block[r] = block_at;
            s_ctx[r] = l[i].ctx;
            if (blockIdx.x == 0) {
                p.q_start[r] = first;
                p.seq_len[r] = l[i].ctx + l[i].fresh;
            }
            row_at += l[i].fresh;
            block_at += l[i].need;
        }
    }
    if (blockIdx.x == 0 && tid == 0) {
        p.q_start[p.requests] = (int32_t)min(all_rows, (int64_t)p.rows);
        p.counts[0] = (int32_t)min(all_rows, (int64_t)0x7fffffff);
        p.counts[1] = all_blocks;
    }
    __syncthreads();

    // new blocks into the tables
    for (int64_t i = (int64_t)blockIdx.x * THREADS + tid; i < all_blocks;
         i += (int64_t)gridDim.x * THREADS) {
        const int r = last_from(s_block, p.requests, (int32_t)i);
        const int64_t col = held(p, s_ctx[r]) + (i - s_block[r]);
        p.table[(int64_t)r * p.table_cols + col] = i < p.n_fresh ? p.fresh[i] : -1;
    }

    // rows
    const int64_t j = (int64_t)blockIdx.x * THREADS + tid;
    if (j < p.rows) {
        int32_t pos = 0, req = -1;
        int64_t slot = -1;
        if (j < all_rows) {
            req = last_from(s_row, p.requests, (int32_t)j);
            const int32_t ctx = s_ctx[req], have = held(p, ctx);
            pos = ctx + ((int32_t)j - s_row[req]);
            const int32_t col = pos >> p.log2_tokens;
            int32_t block = -1;
            if (col < have) {  // a block the request held before
                block = p.table[(int64_t)req * p.table_cols + col];
            } else if (col < p.table_cols) {
                const int64_t i = (int64_t)s_block[req] + (col - have);
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
// Results are stored past the caches' retention, and the QKV rows, which the
// product before has just written, loaded through them.  MI355X, from a graph:
// 8192 rows of 32 + 16 heads of 128 39.4 us (206 MB, 5.2 TB/s; a plain copy of 1 GiB
// 5.15, but part of these rows is still in the Infinity Cache), 1531 rows into an
// E4M3 cache 10.7, one row 6.3.  With plain stores 8192 rows took 43.3 us against
// 40.5, with nontemporal loads too 41.0 (4038 rows of 32 + 32 heads, partly in the
// Infinity Cache: 31.6 and 32.3 against 26.0).

template <int TYPE>
__device__ __forceinline__ float wide(uint16_t v)
{
    if (TYPE == KV_BF16)
        return __builtin_bit_cast(float, (uint32_t)v << 16);
    return (float)__builtin_bit_cast(_Float16, v);
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
        r[i] = narrow2<TYPE>(x[2 * i], x[2 * i + 1]);
    return r;
}

// Eight values / scale as E4M3 codes, nearest even, clamped to +-448 (NaN stays).  The
// conversion has to see which side of a code's middle the quotient is on: fp32
// quotients that are not exact go to their odd neighbour, which is no middle and lies
// on the same side of all of them.  Quotients by a power of two are exact as they are
// (1531 rows 10.7 us, with the other scales' steps 10.9).
__device__ __forceinline__ u32x2 codes8(const float *x, const CodeScale &s)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v = __builtin_amdgcn_ldexpf(x[i], s.shift);
        v = v != v ? v : __builtin_amdgcn_fmed3f(v, -s.most, s.most);
        y[i] = v;
    }
    if (s.unit != 1.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = y[i];
            float q = v * s.inv;
            q = __builtin_fmaf(__builtin_fmaf(-q, s.unit, v), s.inv, q);  // less than a unit off
            const float rest = __builtin_fmaf(-q, s.unit, v);             // exact
            const uint32_t bits = __builtin_bit_cast(uint32_t, q);
            const int32_t down = (int32_t)(__builtin_bit_cast(uint32_t, rest) ^ bits) >> 31;
            if (__builtin_islessgreater(rest, 0.0f))
                q = __builtin_bit_cast(float, (bits + down) | 1);
            y[i] = q;
        }
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

template <int CONTROL>
__device__ __forceinline__ float moved(float x)
{
    return __builtin_bit_cast(
        float,
        __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, false));
}

// Sum over each group of 4, 8 or 16 lanes, in every lane of it.  Quads swap
// lanes; then a half row, then a row of 16 is mirrored, which meets the other
// quad's, the other half's sum.
template <int GROUP>
__device__ __forceinline__ float group_sum(float x)
{
    x += moved<0xB1>(x);  // quad_perm 1 0 3 2
    x += moved<0x4E>(x);  // quad_perm 2 3 0 1
    if (GROUP >= 8)
        x += moved<0x141>(x);  // row_half_mirror
    if (GROUP >= 16)
        x += moved<0x140>(x);  // row_mirror
    return x;
}

// Stored past the caches' retention.
template <typename V>
__device__ __forceinline__ void put(void *p, V v)
{
    __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
}

template <int TYPE, bool FP8, int D, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void kv_store_kernel(const KvStoreProblem p)
{
    constexpr int kLanes = D / 16;  // lanes with work in a group
    constexpr int kGroup = kLanes <= 4 ? 4 : (kLanes <= 8 ? 8 : 16);
    constexpr int kElt = FP8 ? 1 : 2;
    const int j = threadIdx.x % kGroup;
    const uint32_t q_heads = (uint32_t)p.heads, kv_heads = (uint32_t)p.cache.kv_heads;
    const uint32_t heads = q_heads + 2 * kv_heads;
    const uint32_t item = blockIdx.x * (kThreads / kGroup) + threadIdx.x / kGroup;
    const uint32_t row = item / heads, head = item - row * heads;
    if (row >= (uint32_t)p.rows)
        return;
    const bool is_q = head < q_heads, is_v = head >= q_heads + kv_heads;
    const bool works = j < kLanes;
    const bool turns = !is_v && 16 * j < p.rot;
    // the lane's two chunks of eight values
    const bool split = turns && !ADJACENT;
    const int c0 = split ? j : 2 * j, c1 = split ? j + p.rot / 16 : 2 * j + 1;
    u32x4 a = {0u, 0u, 0u, 0u}, b = a;
    if (works) {
        const uint16_t *src = p.qkv + row * p.qkv_stride + head * D;
        a = load16(src + 8 * c0);
        b = load16(src + 8 * c1);
    }
    const int64_t slot = is_q ? 0 : p.slot[row];
    const int64_t pos = turns ? p.pos[row] : 0;
    float x[16];
    if (!is_v) {
        const uint16_t *weight = is_q ? p.q_weight : p.k_weight;
        u32x4 wa, wb;
        if (weight && works) {
            wa = load16(weight + 8 * c0);
            wb = load16(weight + 8 * c1);
        }
        f32x4 cs[2], sn[2];
        if (turns) {
            const bool known = pos >= 0 && pos < p.max_pos;
            const float *at = p.rope + (known ? pos : 0) * p.rot + 8 * j;
            cs[0] = *reinterpret_cast<const f32x4 *>(at);
            cs[1] = *reinterpret_cast<const f32x4 *>(at + 4);
            sn[0] = *reinterpret_cast<const f32x4 *>(at + p.rot / 2);
            sn[1] = *reinterpret_cast<const f32x4 *>(at + p.rot / 2 + 4);
            if (!known)  // no such angle: the row is not a number rather than wrong
                cs[0] = cs[1] = sn[0] = sn[1] = __builtin_nanf("");
        }
        widen8<TYPE>(a, x);
        widen8<TYPE>(b, x + 8);
        if (weight) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                ss += x[i] * x[i];
            const float inv = __builtin_amdgcn_rsqf(group_sum<kGroup>(ss) * (1.0f / D) + p.eps);
            if (works) {
                float w[16];
                widen8<TYPE>(wa, w);
                widen8<TYPE>(wb, w + 8);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = x[i] * inv * w[i];
            }
        }
        if (turns) {
            if (ADJACENT) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = cs[i / 4][i % 4], s = sn[i / 4][i % 4];
                    const float u = x[2 * i], v = x[2 * i + 1];
                    x[2 * i] = u * c - v * s;
                    x[2 * i + 1] = v * c + u * s;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = cs[i / 4][i % 4], s = sn[i / 4][i % 4];
                    const float u = x[i], v = x[i + 8];
                    x[i] = u * c - v * s;
                    x[i + 8] = v * c + u * s;
                }
            }
        }
        a = narrow8<TYPE>(x);
        b = narrow8<TYPE>(x + 8);
    } else if (FP8) {
        widen8<TYPE>(a, x);
        widen8<TYPE>(b, x + 8);
    }
    if (!works)
        return;
    const uint32_t kvh = head - q_heads - (is_v ? kv_heads : 0);
    if (is_q || (!is_v && p.k_out)) {
        uint16_t *dst = is_q ? p.q_out + row * p.q_out_stride + head * D
                             : p.k_out + row * p.k_out_stride + kvh * D;
        put(dst + 8 * c0, a);
        put(dst + 8 * c1, b);
        if (is_q)
            return;
    }
    const int64_t block = slot >> p.cache.log2_tokens;
    if (slot < 0 || block >= p.cache.n_blocks)
        return;
    // places inside a block fit 32 bits
    const uint32_t tokens = 1u << p.cache.log2_tokens, t = (uint32_t)slot & (tokens - 1);
    uint8_t *base = p.cache.pool + block * p.cache.block_stride;
    const uint32_t at0 = 8 * kElt * c0, at1 = 8 * kElt * c1;  // bytes in the row
    uint32_t to0, to1;
    if (is_v) {
        const uint32_t first = ((kv_heads + kvh) * tokens + t) * (D * kElt);
        to0 = first + at0;
        to1 = first + at1;
    } else {
        const uint32_t first = kvh * (D * kElt / 64);
        to0 = ((first + at0 / 64) * tokens + t) * 64 + at0 % 64;
        to1 = ((first + at1 / 64) * tokens + t) * 64 + at1 % 64;
    }
    if (FP8) {
        // values, not places: a choice of places is a vector load from the arguments
        const CodeScale k = p.k_code, v = p.v_code;
        const CodeScale scale = {is_v ? +v.unit : +k.unit, is_v ? +v.inv : +k.inv,
                                 is_v ? +v.most : +k.most, is_v ? +v.shift : +k.shift};
        put(base + to0, codes8(x, scale));
        put(base + to1, codes8(x + 8, scale));
    } else {
        put(base + to0, a);
        put(base + to1, b);
    }
}

template <int TYPE, bool FP8, int D>
hipError_t store(const KvStoreProblem &p, hipStream_t stream)
{
    constexpr int lanes = D / 16, group = lanes <= 4 ? 4 : (lanes <= 8 ? 8 : 16);
    const int64_t items = p.rows * (p.heads + 2 * (int64_t)p.cache.kv_heads);
    const int64_t blocks = (items * group + kThreads - 1) / kThreads;
    if (p.adjacent)
        hipLaunchKernelGGL((kv_store_kernel<TYPE, FP8, D, true>), dim3((unsigned)blocks),
                           dim3(kThreads), 0, stream, p);
    else
        hipLaunchKernelGGL((kv_store_kernel<TYPE, FP8, D, false>), dim3((unsigned)blocks),
                           dim3(kThreads), 0, stream, p);
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
    const int threads = p.requests <= 256 ? 256 : 1024;
    const int64_t blocks = p.rows > 0 ? ((int64_t)p.rows + threads - 1) / threads : 1;
    const dim3 grid((unsigned)blocks), block((unsigned)threads);
    if (threads == 256)
        hipLaunchKernelGGL(kv_map_kernel<256>, grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL(kv_map_kernel<1024>, grid, block, 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_kv_store(const KvStoreProblem &p, int type, bool fp8, hipStream_t stream)
{
    return type == KV_BF16 ? store_type<KV_BF16>(p, fp8, stream)
                           : store_type<KV_F16>(p, fp8, stream);
}

}  // namespace dps
