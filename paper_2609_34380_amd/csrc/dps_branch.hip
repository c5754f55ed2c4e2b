// dps_branch.hip -- blocks of the paged KV cache when sequences branch (gfx950):
// the block tables of a step whose rows go on from other rows (beams, several
// answers to one prompt), copies of blocks, and tables after blocks have moved.
#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kMostRows = 4096;  // rows of a table

// ---- copies -----------------------------------------------------------------------
// Pair i: the first n tokens of every head's keys and values of block src[i] into
// block dst[i].  In a block the 16-byte units of a key segment lie token by token
// (4 a token), those of a value row too (dim * element bytes / 16 a token), so a
// unit's token follows from its index alone and a thread moves unit u to unit u.
//
// Bound: HBM, 2 bytes moved a byte of live tokens.  A block of threads takes kUnits
// units a thread of one pair, all loads ahead of the first store (3000 blocks of 64 KiB:
// 393 MB moved in 61 us, 6.5 TB/s, some of it in the Infinity Cache; 40 blocks 3.5 us).
constexpr int kUnits = 4;

template <bool PART>
__global__ __launch_bounds__(kThreads) void kv_copy_kernel(
    const KvCopyProblem p, const int32_t *__restrict__ srcs, const int32_t *__restrict__ dsts,
    const int32_t *__restrict__ parts, const int32_t *__restrict__ count)
{
    const uint32_t pair = blockIdx.x / p.pieces, piece = blockIdx.x % p.pieces;
    if (count && (int32_t)pair >= *count)
        return;
    const int32_t src = srcs[pair], dst = dsts[pair];
    const int32_t most = 1 << p.log2_tokens;
    const int32_t part = PART ? min(parts[pair], most) : most;
    if (src < 0 || src >= p.n_blocks || dst < 0 || dst >= p.n_blocks || src == dst || part <= 0)
        return;
    const u32x4 *from = reinterpret_cast<const u32x4 *>(p.pool + src * p.block_stride);
    u32x4 *to = reinterpret_cast<u32x4 *>(p.pool + dst * p.block_stride);
    u32x4 x[kUnits];
    bool live[kUnits];
    const uint32_t u0 = piece * (kThreads * kUnits) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * kThreads;
        live[i] = u < p.units;
        if (PART && part < most) {
            // units a token: 4 of keys; of values 2^row_shift, or three times that
            uint32_t token = u >> 2;
            if (u >= p.key_units) {
                token = (u - p.key_units) >> p.row_shift;
                if (p.thirds)
                    token /= 3;
            }
            live[i] = live[i] && (int32_t)(token & (most - 1)) < part;
        }
        if (live[i])
            x[i] = __builtin_nontemporal_load(from + u);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
        if (live[i])
            to[u0 + i * kThreads] = x[i];
}

// ---- tables after blocks have moved --------------------------------------------------
// An entry that names src[i] becomes dst[i]; src ascends, so a thread finds its
// entry by bisection in a copy of the list in LDS (log2 n steps of LDS latency each).
// Lists too long for that are searched where they lie.
//
// Bound: latency.  kEntries entries a thread share the steps (131072 entries and a list of
// 3000: 6.6 us, 2048 and 40: 3.0).
constexpr int kEntries = 4;
constexpr int kListed = 12288;  // 48 KiB

template <bool LDS>
__global__ __launch_bounds__(kThreads) void kv_remap_kernel(int32_t *__restrict__ table,
                                                            int64_t entries,
                                                            const int32_t *__restrict__ src,
                                                            const int32_t *__restrict__ dst,
                                                            int32_t n)
{
    extern __shared__ int32_t s_src[];
    const int64_t e0 = (int64_t)blockIdx.x * (kThreads * kEntries) + threadIdx.x;
    int32_t id[kEntries];
#pragma unroll
    for (int i = 0; i < kEntries; ++i)
        id[i] = e0 + i * kThreads < entries ? table[e0 + i * kThreads] : -1;
    if (LDS) {
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += kThreads)
            s_src[i] = src[i];
        __syncthreads();
    }
    const int32_t *list = LDS ? s_src : src;
    // the last entry <= id, if any is: lo, by halving steps that all four share
    int32_t lo[kEntries] = {0, 0, 0, 0};
    for (int32_t step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step > 0; step >>= 1) {
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            const int32_t at = lo[i] + step;
            if (at < n && list[at] <= id[i])
                lo[i] = at;
        }
    }
#pragma unroll
    for (int i = 0; i < kEntries; ++i)
        if (id[i] >= 0 && list[lo[i]] == id[i])
            table[e0 + i * kThreads] = dst[lo[i]];
}

// ---- forked tables -------------------------------------------------------------------
// New row r goes on from old row p = parent[r].  Rows share whole blocks.  A last
// block that is only partly filled stays with the first child (the lowest r) of its
// row; the others get a block off `fresh` each, in row order, and an entry in the
// list of copies.  Freed are the blocks of the old tables that no new one holds: a
// byte a block for either side, set by the kernel that writes the tables (all writers
// of a byte store the same, so plain stores do; bits set by atomics took 700 us of a
// call with 2000 rows of 1300 columns).
//
// Bound: latency, and 4 bytes in and out a table entry.  Three launches (one for small
// tables), each of which needs all of the one before: who copies (and cleared bytes),
// tables and bytes, the list of freed blocks (256 rows of 512 columns 3.6 + 5.9 + 3.6 us,
// 1000 of 1300 4.4 + 8.4 + 5.5).

__device__ __forceinline__ bool in_range(int32_t x, int32_t n) { return x >= 0 && x < n; }

// Tokens of an old row, and the columns that hold them.
__device__ __forceinline__ int32_t length_of(const KvForkProblem &p, int32_t row)
{
    return max(p.seq_len[row], 0);
}
__device__ __forceinline__ int32_t columns(const KvForkProblem &p, int32_t len)
{
    const uint32_t t = 1u << p.log2_tokens;
    return min((int32_t)(((uint32_t)len + t - 1) >> p.log2_tokens), p.cols);
}
// Whether the row's last token lies in the table, in a block with room after it.
__device__ __forceinline__ bool open_ended(const KvForkProblem &p, int32_t len)
{
    return (len & ((1 << p.log2_tokens) - 1)) != 0 && (len >> p.log2_tokens) < p.cols;
}

// Who copies: lengths, the list of copies, and what replaces each new row's last block.
// By kPlanThreads threads; s_eldest holds old_rows entries.
__device__ __forceinline__ void plan_copies(const KvForkProblem &p, int32_t *s_eldest,
                                            int32_t *s_sums)
{
    constexpr int kPer = kMostRows / kPlanThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < p.old_rows; i += kPlanThreads)
        s_eldest[i] = 0x7fffffff;  // its first child
    __syncthreads();
    const int r0 = tid * kPer;
    int32_t from[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        from[i] = r0 + i < p.rows ? p.parent[r0 + i] : -1;
        if (in_range(from[i], p.old_rows))
            atomicMin(&s_eldest[from[i]], r0 + i);
        else
            from[i] = -1;
    }
    int32_t len[kPer], n = 0;
    bool copies[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        len[i] = from[i] >= 0 ? length_of(p, from[i]) : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        copies[i] = from[i] >= 0 && open_ended(p, len[i]) && s_eldest[from[i]] != r0 + i;
        n += copies[i];
    }
    const int32_t incl = wave_scan(n);
    if (lane == 63)
        s_sums[wave] = incl;
    __syncthreads();
    int32_t at = incl - n, all = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        at += i < wave ? s_sums[i] : 0;
        all += s_sums[i];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i;
        if (r >= p.rows)
            break;
        p.new_len[r] = len[i];
        int32_t block = kKeep;
        if (copies[i]) {
            block = at < p.n_fresh ? p.fresh[at] : -1;
            const int32_t col = len[i] >> p.log2_tokens;
            p.src[at] = p.table[(int64_t)from[i] * p.cols + col];
            p.dst[at] = block;
            p.tokens[at] = len[i] & ((1 << p.log2_tokens) - 1);
            ++at;
        }
        p.last[r] = block;
    }
    for (int i = all + tid; i < p.rows; i += kPlanThreads)
        p.src[i] = p.dst[i] = p.tokens[i] = -1;
    if (tid == 0)
        p.counts[0] = all;
}

// The block of a new row's column.
__device__ __forceinline__ int32_t block_of(const KvForkProblem &p, int32_t row, int32_t col)
{
    const int32_t from = p.parent[row];
    if (!in_range(from, p.old_rows))
        return -1;
    const int32_t last = p.last[row], have = columns(p, length_of(p, from));
    if (col >= have)
        return -1;
    return col == have - 1 && last != kKeep ? last : p.table[(int64_t)from * p.cols + col];
}

__global__ __launch_bounds__(kPlanThreads) void kv_fork_plan_kernel(const KvForkProblem p)
{
    __shared__ int32_t s_eldest[kMostRows];
    __shared__ int32_t s_sums[kPlanThreads / 64];
    // bytes of both sides, by every block
    for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < 2 * p.words;
         i += (int64_t)gridDim.x * kPlanThreads)
        p.held[i] = u32x4{0u, 0u, 0u, 0u};
    if (blockIdx.x == 0)
        plan_copies(p, s_eldest, s_sums);
}

// All of it in one block of threads, a bit a block in LDS: for tables so small that the
// time is that of the launches (8 rows of 256 columns: one of 6 us for three of 3-5 each).
constexpr int64_t kSmallEntries = 16384;  // of both tables, 16 a thread
constexpr int64_t kSmallBlocks = 131072;
constexpr int kSmallWords = kSmallBlocks / 32;
constexpr int kSmallRows = 1024;

__global__ __launch_bounds__(kPlanThreads) void kv_fork_small_kernel(const KvForkProblem p)
{
    __shared__ int32_t s_eldest[kSmallRows];
    __shared__ int32_t s_sums[kPlanThreads / 64];
    __shared__ uint32_t s_old[kSmallWords], s_new[kSmallWords];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t words = (int32_t)((p.n_blocks + 31) / 32);
    for (int i = tid; i < words; i += kPlanThreads)
        s_old[i] = s_new[i] = 0;
    plan_copies(p, s_eldest, s_sums);  // meets at its barriers
    __threadfence_block();
    __syncthreads();
    const auto mark = [&](uint32_t *bits, int32_t block) {
        if (block >= 0 && block < p.n_blocks)
            atomicOr(&bits[block >> 5], 1u << (block & 31));
    };
    const int32_t olds = p.old_rows * p.cols, news = p.rows * p.cols;
#pragma unroll 4
    for (int i = tid; i < olds; i += kPlanThreads)
        mark(s_old, p.table[i]);
#pragma unroll 4
    for (int i = tid; i < news; i += kPlanThreads) {
        const int32_t row = i / p.cols, block = block_of(p, row, i - row * p.cols);
        p.new_table[i] = block;
        mark(s_new, block);
    }
    __syncthreads();
    constexpr int kPer = kSmallWords / kPlanThreads;
    uint32_t freed[kPer];
    int32_t n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int w = tid * kPer + i;
        freed[i] = w < words ? s_old[w] & ~s_new[w] : 0;
        n += __popc(freed[i]);
    }
    const int32_t incl = wave_scan(n);
    if (lane == 63)
        s_sums[wave] = incl;
    __syncthreads();
    int32_t at = incl - n, all = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        at += i < wave ? s_sums[i] : 0;
        all += s_sums[i];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        for (uint32_t left = freed[i]; left; left &= left - 1, ++at)
            if (at < p.n_freed)
                p.freed[at] = (tid * kPer + i) * 32 + __builtin_ctz(left);
    for (int64_t i = all + tid; i < p.n_freed; i += kPlanThreads)
        p.freed[i] = -1;
    if (tid == 0)
        p.counts[1] = all;
}

// A thread has one column of kRows rows.  Rows that share a prefix lie side by side:
// an entry that repeats the one above it is marked already.
constexpr int kRows = 8;

__global__ __launch_bounds__(kThreads) void kv_fork_tables_kernel(const KvForkProblem p)
{
    const int32_t col = blockIdx.x * kThreads + threadIdx.x;
    if (col >= p.cols)
        return;
    const int32_t groups = (p.rows + kRows - 1) / kRows;
    const bool old = (int32_t)blockIdx.y >= groups;
    const int32_t r0 = ((int32_t)blockIdx.y - (old ? groups : 0)) * kRows;
    const int32_t rows = old ? p.old_rows : p.rows;
    int32_t block[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int32_t row = r0 + i;
        block[i] = -1;
        if (row >= rows)
            continue;
        if (old) {
            block[i] = p.table[(int64_t)row * p.cols + col];
        } else {
            block[i] = block_of(p, row, col);
            p.new_table[(int64_t)row * p.cols + col] = block[i];
        }
    }
    uint8_t *held = reinterpret_cast<uint8_t *>(p.held + (old ? 0 : p.words));
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (block[i] >= 0 && block[i] < p.n_blocks && (i == 0 || block[i] != block[i - 1]))
            held[block[i]] = 1;
}

// A block of threads lists the freed blocks of its share of the 16-byte words, kPlanThreads
// at a time, after those of all words before, which it counts itself: 16 bytes a block of
// either side, read by at most kListers blocks.
constexpr int64_t kListers = 256;

__device__ __forceinline__ u32x4 freed_of(const KvForkProblem &p, int64_t w)
{
    return p.held[w] & ~p.held[p.words + w];
}
__device__ __forceinline__ int count(u32x4 x)
{
    return __popc(x.x) + __popc(x.y) + __popc(x.z) + __popc(x.w);
}

__global__ __launch_bounds__(kPlanThreads) void kv_fork_freed_kernel(const KvForkProblem p,
                                                                     int64_t share)
{
    __shared__ int32_t s_before[kPlanThreads / 64], s_after[kPlanThreads / 64],
        s_sums[kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t w0 = (int64_t)blockIdx.x * share, w1 = min(w0 + share, p.words);
    int32_t before = 0, after = 0;  // of the words before its share, and of the others
#pragma unroll 4
    for (int64_t w = tid; w < w0; w += kPlanThreads)
        before += count(freed_of(p, w));
    u32x4 freed = {0u, 0u, 0u, 0u};
    if (w0 + tid < w1)
        freed = freed_of(p, w0 + tid);
#pragma unroll 4
    for (int64_t w = w0 + tid + kPlanThreads; w < p.words; w += kPlanThreads)
        after += count(freed_of(p, w));
    const int32_t incl_before = wave_scan(before), incl_after = wave_scan(after + count(freed));
    if (lane == 63) {
        s_before[wave] = incl_before;
        s_after[wave] = incl_after;
    }
    __syncthreads();
    int32_t base = 0, all = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        base += s_before[i];
        all += s_before[i] + s_after[i];
    }
    for (int64_t w = w0; w < w1; w += kPlanThreads) {
        const int64_t mine = w + tid;
        if (w > w0)
            freed = mine < w1 ? freed_of(p, mine) : u32x4{0u, 0u, 0u, 0u};
        const int32_t n = count(freed), incl = wave_scan(n);
        __syncthreads();  // the sums before have been read
        if (lane == 63)
            s_sums[wave] = incl;
        __syncthreads();
        int32_t at = base + incl - n;
        for (int i = 0; i < kPlanThreads / 64; ++i) {
            at += i < wave ? s_sums[i] : 0;
            base += s_sums[i];
        }
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if ((freed[i >> 2] >> (i & 3) * 8) & 1) {
                    if (at < p.n_freed)
                        p.freed[at] = (int32_t)(mine * 16) + i;
                    ++at;
                }
            }
        }
    }
    for (int64_t i = all + (int64_t)blockIdx.x * kPlanThreads + tid; i < p.n_freed;
         i += (int64_t)gridDim.x * kPlanThreads)
        p.freed[i] = -1;
    if (blockIdx.x == 0 && tid == 0)
        p.counts[1] = all;
}

}  // namespace

hipError_t launch_kv_copy(const KvCopyProblem &p, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.n * p.pieces));
    if (p.tokens)
        hipLaunchKernelGGL(kv_copy_kernel<true>, grid, dim3(kThreads), 0, stream, p, p.src, p.dst,
                           p.tokens, p.count);
    else
        hipLaunchKernelGGL(kv_copy_kernel<false>, grid, dim3(kThreads), 0, stream, p, p.src, p.dst,
                           p.tokens, p.count);
    return hipGetLastError();
}

int kv_copy_piece_units() { return kThreads * kUnits; }

hipError_t launch_kv_remap(int32_t *table, int64_t entries, const int32_t *src, const int32_t *dst,
                           int64_t n, hipStream_t stream)
{
    const int64_t each = kThreads * kEntries;
    const dim3 grid((unsigned)((entries + each - 1) / each));
    if (n <= kListed)
        hipLaunchKernelGGL(kv_remap_kernel<true>, grid, dim3(kThreads), (size_t)n * 4, stream,
                           table, entries, src, dst, (int32_t)n);
    else
        hipLaunchKernelGGL(kv_remap_kernel<false>, grid, dim3(kThreads), 0, stream, table, entries,
                           src, dst, (int32_t)n);
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvForkProblem &p, hipStream_t stream)
{
    if (p.rows <= kSmallRows && p.old_rows <= kSmallRows && p.n_blocks <= kSmallBlocks &&
        ((int64_t)p.rows + p.old_rows) * p.cols <= kSmallEntries) {
        hipLaunchKernelGGL(kv_fork_small_kernel, dim3(1), dim3(kPlanThreads), 0, stream, p);
        return hipGetLastError();
    }
    const int64_t clears = (2 * p.words + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
    hipLaunchKernelGGL(kv_fork_plan_kernel, dim3((unsigned)(clears < 1 ? 1 : clears)),
                       dim3(kPlanThreads), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    if (p.cols > 0 && p.rows + p.old_rows > 0) {
        hipLaunchKernelGGL(kv_fork_tables_kernel,
                           dim3((unsigned)((p.cols + kThreads - 1) / kThreads),
                                (unsigned)((p.rows + kRows - 1) / kRows +
                                           (p.old_rows + kRows - 1) / kRows)),
                           dim3(kThreads), 0, stream, p);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    int64_t share = (p.words + kListers - 1) / kListers;
    share = (share + kPlanThreads - 1) / kPlanThreads * kPlanThreads;
    const int64_t lists = share > 0 ? (p.words + share - 1) / share : 1;
    hipLaunchKernelGGL(kv_fork_freed_kernel, dim3((unsigned)lists), dim3(kPlanThreads), 0, stream,
                       p, share);
    return hipGetLastError();
}

}  // namespace dps
