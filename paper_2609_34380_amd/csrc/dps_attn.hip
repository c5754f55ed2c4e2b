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
//     heads as the columns, or 17 to 32 in two column tiles (HT) that share
//     every load and permute.  The lane that holds S^T of (token, head) is the
//     lane whose P^T operand needs it, so P never crosses lanes; V is turned
//     in registers (one byte permute per two values); the main loop has no LDS
//     and no barrier.
//   - Token 4 r + c of 16 sits in operand row 4 c + r.  With the cache's
//     64-byte key segments every key load of a wave is then 1 KiB of contiguous
//     memory.  A value load takes 16 lanes' worth (up to 8 values each) of four
//     neighbouring tokens: contiguous where that is the whole row (1 KiB for 16-bit
//     heads of 128, 512 bytes for 16-bit heads of 64 and E4M3 heads of 128), else
//     four runs of 64 to 256 bytes.
//   - The tokens of all rows, in tiles of 32, form one line per key/value head,
//     cut into equal ranges, one per wave: ragged lengths load every CU alike.
//     A wave steps through the rows of its range one by one (an idle one costs a
//     scalar load's latency, 0.2 us) and finishes those inside by itself; what the
//     four waves of a block share is joined in LDS, what blocks share (at most
//     two partial rows a block, however long a row is) in attn_join_kernel.
//     Partials are joined in their order, so results do not depend on timing.
//   - Block ids come through scalar loads one tile ahead: a vector load of them
//     would wait for every value load issued before it.
//
// Precision: products and softmax in fp32.  The weights P enter the matrix cores
// as two 16-bit terms (value and remainder).  BF16 terms keep a weight to 2^-17 of
// itself.  FP16 terms keep it to 2^-21 of itself or 2^-30 of the row's largest
// weight, whichever is more: beside a token that outweighs it 2^24 times a token
// loses up to 1.6% of its own share, under 2^-30 all of it (the sum counts it
// whole).  One term would add an error of the size of the output's own rounding
// (relative error 2.1e-4 -> 2.9e-4 in FP16 over an E4M3 cache, 1.7e-3 -> 2.1e-3 in
// BF16) and save 0-1% of the time.
//
// Measured on MI355X, both launches replayed from a graph, 32 query and 8
// key/value heads of 128: one row of 131000 tokens beside 16 short ones (598 MB)
// 97.6 us, 6.1 TB/s; 34 FP16 rows of up to 4096 (272 MB) 46.8; 256 BF16 rows of
// up to 600, 64 query heads (305 MB) 56.4; 16 rows of 30000 in E4M3 (930 MB) 142
// (one call at a time 146), 6.5 TB/s, where a nontemporal read of memory reaches
// 6.6-6.9.  A pass over a key/value head fetches every byte once (FETCH_SIZE).
// With loads that caches retain the first three take 112, 52 and 65 us (kernel
// alone) against 99, 46 and 57.  The second launch and its join cost about 4 us, a
// block's start and end about 5.
#include <type_traits>

#include "dps_attn.h"
#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kJoinThreads = 512;

// The live tokens [lo, hi) of a row and its table row; hi = 0: none.
struct RowSpan {
    int32_t lo, hi;
    int32_t req;
};

// UNIFORM: r is the wave's, and the result lies in scalar registers.  SHARED: the row
// shares its first tokens with others, and this kernel has those after them.
template <bool UNIFORM, bool SHARED>
__device__ __forceinline__ RowSpan row_span(const AttnProblem &p, const int32_t *__restrict__ req,
                                            const int32_t *__restrict__ kv_len,
                                            const SharedRow *__restrict__ shared, int32_t r)
{
    RowSpan s;
    s.req = req ? req[r] : r;
    int32_t len = kv_len[r];
    const int32_t own = SHARED ? shared[r].start : 0;
    // both loads under way before either is looked at: one latency, not two (0.1-0.5 us)
    if (UNIFORM)
        asm("" : "+s"(s.req), "+s"(len));
    else
        asm("" : "+v"(s.req), "+v"(len));
    const int64_t room = min(p.table_cols << p.log2_tokens, kLongest);
    int64_t n = len;
    if (s.req < 0 || s.req >= p.requests)
        n = 0;
    n = n < 0 ? 0 : (n > room ? room : n);
    s.hi = (int32_t)n;
    if (SHARED)  // at most n: only a row that has all of them shares tokens
        s.lo = own;
    else
        s.lo = p.window > 0 && n > p.window ? (int32_t)(n - p.window) : 0;
    return s;
}

// Tiles of a row (its live tokens on the grid of kTile tokens; none where lo = hi on it).
__device__ __forceinline__ int32_t row_tiles(const RowSpan &s)
{
    return s.hi == 0 ? 0 : (int32_t)(((uint32_t)s.hi + kTile - 1) / kTile) - s.lo / kTile;
}

// The work line of a key/value head cut into `waves` ranges of `each` tiles, the
// first `more` of them one longer.
struct WorkLine {
    uint32_t waves, each, more;

    __device__ __forceinline__ WorkLine(uint32_t tiles, uint32_t most)
        : waves(min(tiles, most)), each(tiles / max(waves, 1u)), more(tiles - each * waves)
    {
    }
    __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * each + min(w, more); }
    __device__ __forceinline__ uint32_t count(uint32_t w) const
    {
        return w < waves ? each + (w < more ? 1 : 0) : 0;
    }
    // the wave that has tile t
    __device__ __forceinline__ uint32_t of(uint32_t t) const
    {
        const uint32_t cut = more * (each + 1);
        return t < cut ? t / (each + 1) : more + (t - cut) / each;
    }
};

// Place of this block on its work line.  The chip deals blocks to its eight XCDs
// in turn: neighbours on the line, which share rows, go to one XCD, here and in
// the join (0.5-1.5% on calls of 50 to 100 us).
__device__ __forceinline__ int line_block()
{
    constexpr uint32_t kXcds = 8;
    const uint32_t x = blockIdx.x, n = gridDim.x;
    return (int)(n % kXcds == 0 ? x % kXcds * (n / kXcds) + x / kXcds : x);
}

// Four values of a finished row's head: o / sum, rounded once, and its lse.
template <int TYPE>
__device__ __forceinline__ void attn_store(const AttnProblem &p, int64_t row, int head, int dim,
                                           int d, f32x4 o, float ref, float sum)
{
    const float scale = sum == 0.0f ? 0.0f : p.value_scale / sum;
    uint16_t *at = static_cast<uint16_t *>(p.out) + row * p.out_stride + (int64_t)head * dim + d;
    *reinterpret_cast<u32x2 *>(at) =
        u32x2{narrow2<TYPE>(o[0] * scale, o[1] * scale), narrow2<TYPE>(o[2] * scale, o[3] * scale)};
    if (d == 0 && p.lse)
        p.lse[row * (p.kv_heads * p.group) + head] =
            sum == 0.0f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

// A wave's output of one row: acc (value d of a head in the lane and register
// that the matrix instruction leaves it), reference score and sum per head.
template <int KACC>
struct Partial {
    f32x4 acc[KACC];
    float ref, sum;

    __device__ __forceinline__ void clear()
    {
        ref = kNone;
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < KACC; ++i)
            acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // Joins a partial that lies in LDS, a register of all lanes at a time.
    __device__ __forceinline__ void join(const f32x4 *at, const float *stat, int lane)
    {
        const float r = stat[lane], to = fmaxf(ref, r);
        const float a = __builtin_amdgcn_exp2f(ref - to), b = __builtin_amdgcn_exp2f(r - to);
        sum = sum * a + stat[64 + lane] * b;
        ref = to;
#pragma unroll
        for (int i = 0; i < KACC; ++i)
            acc[i] = acc[i] * a + at[i * 64 + lane] * b;
    }
};

// SHARED: a row's output goes to p.own unfinished, for the join with its shared tokens,
// and what it takes to find a row's partials to p.found.
template <int TYPE, bool FP8, int D, int HT, bool SHARED>
__global__ __launch_bounds__(kThreads, (Shape<TYPE, FP8, D, HT>::kWavesPerSimd)) void attn_kernel(
    const AttnProblem p, const int32_t *__restrict__ tables, const int32_t *__restrict__ reqs,
    const int32_t *__restrict__ kv_len, const SharedRow *__restrict__ shared)
{
    typedef Shape<TYPE, FP8, D, HT> S;
    __shared__ f32x4 s_head[kWaves][HT][S::kAcc * 64];  // rows that began before the wave
    __shared__ float s_stat[kWaves][HT][128];
    __shared__ int32_t s_first[kThreads];
    __shared__ int32_t s_sums[kWaves];
    __shared__ int32_t s_state[kWaves];
    __shared__ int32_t s_join[8];

    const int block = line_block();
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;   // query head of a column tile (matrix column)
    const int quarter = lane >> 4;
    const int hv = blockIdx.y;   // (key/value head, pass over its query heads)
    const int kvh = hv / p.head_groups;
    const int sub = hv % p.head_groups;
    const int first_head = kvh * p.group + sub * p.group_step;
    const int n_heads = min(p.group_step, p.group - sub * p.group_step);
    const int rows = (int)p.rows;

    // ---- this wave's range of the work line ----------------------------------
    // up to 64 rows: a row a lane, in every wave; above, thread i sums rows
    // [i * per, (i + 1) * per)
    int32_t tiles, chunk = 0, chunk_first = 0;
    const int32_t per = rows <= 64 ? 64 : (rows + kThreads - 1) / kThreads;
    RowSpan span;
    int32_t mine = 0, incl = 0;
    if (rows <= 64) {
        span = RowSpan{0, 0, 0};
        if (lane < rows)
            span = row_span<false, SHARED>(p, reqs, kv_len, shared, lane);
        mine = row_tiles(span);
        incl = wave_scan(mine);
        tiles = __builtin_amdgcn_readlane(incl, 63);
    } else {
        const int32_t r1 = min((tid + 1) * per, rows);
        for (int32_t r = tid * per; r < r1; ++r)
            mine += row_tiles(row_span<false, SHARED>(p, reqs, kv_len, shared, r));
        incl = wave_scan(mine);
        if (lane == 63)
            s_sums[wave] = incl;
        __syncthreads();
        tiles = 0;
        int32_t before = incl - mine;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            before += i < wave ? s_sums[i] : 0;
            tiles += s_sums[i];
        }
        tiles = __builtin_amdgcn_readfirstlane(tiles);
        s_first[tid] = before;
        __syncthreads();
    }
    const WorkLine line((uint32_t)tiles, gridDim.x * kWaves);
    const uint32_t me = block * kWaves + wave;
    const int32_t begin = (int32_t)line.begin(me);
    int left = (int)line.count(me);
    if (tid < 8) {
        s_join[tid] = 0;
        if (hv == 0 && line.waves <= block * kWaves)
            p.join[block * 8 + tid] = 0;
    }
    if (line.waves <= block * kWaves)  // no tile for the whole block
        return;
    int row = 0, skip = 0;  // the row of the range's first tile, and that tile's index in it
    if (left > 0) {
        if (rows > 64) {
            int below = 0;
#pragma unroll
            for (int i = 0; i < kWaves; ++i)
                below += __popcll(__ballot(s_first[i * 64 + lane] <= begin));
            chunk = below - 1;
            chunk_first = __builtin_amdgcn_readfirstlane(s_first[chunk]);
        }
        if (per == 1) {
            row = chunk;
            skip = begin - chunk_first;
            span = row_span<false, SHARED>(p, reqs, kv_len, shared, row);
        } else {
            const int32_t r1 = min((chunk + 1) * per, rows);
            for (int32_t r = chunk * per; r < r1; r += 64) {
                if (rows > 64) {
                    span = RowSpan{0, 0, 0};
                    if (r + lane < r1)
                        span = row_span<false, SHARED>(p, reqs, kv_len, shared, r + lane);
                    mine = row_tiles(span);
                    incl = wave_scan(mine);
                }
                const uint64_t past = __ballot(chunk_first + incl > begin);
                if (past) {
                    const int at = __builtin_ctzll(past);
                    row = r + at;
                    skip = begin - (chunk_first + __builtin_amdgcn_readlane(incl - mine, at));
                    span.lo = __builtin_amdgcn_readlane(span.lo, at);
                    span.hi = __builtin_amdgcn_readlane(span.hi, at);
                    span.req = __builtin_amdgcn_readlane(span.req, at);
                    break;
                }
                chunk_first += __builtin_amdgcn_readlane(incl, 63);
            }
        }
    }
    int lo = __builtin_amdgcn_readfirstlane(span.lo);
    int hi = __builtin_amdgcn_readfirstlane(span.hi);
    int req = __builtin_amdgcn_readfirstlane(span.req);

    const uint32_t tokens = 1u << p.log2_tokens;
    const uint32_t key_lane = (4 * (col & 3) + (col >> 2)) * 64 + quarter * 16;
    const uint32_t key_head = (uint32_t)kvh * S::kKeyLoads * tokens * 64;
    const uint32_t val_head = (uint32_t)(p.kv_heads + kvh) * tokens * (D * S::kElt);
    const float to_log2 = p.score_scale * kLog2e;
    const int32_t last_col = (int32_t)p.table_cols - 1;

    // values d .. d + W - 1 of a head, one piece register by register
    const auto each_piece = [&](const auto &put) {
#pragma unroll
        for (int i = 0; i < S::kP8; ++i)
            put(std::integral_constant<int, 8>(), 128 * i, 8 * i);
        if (S::kP4)
            put(std::integral_constant<int, 4>(), 128 * S::kP8, 8 * S::kP8);
        if (S::kP2)
            put(std::integral_constant<int, 2>(), 128 * S::kP8 + 64 * S::kP4,
                8 * S::kP8 + 4 * S::kP4);
    };
    Partial<S::kAcc> o[HT];
    // a partial row of one head, in fp32
    const auto put_wide = [&](const Partial<S::kAcc> &f, float *at) {
        each_piece([&](auto width, int d0, int tile) {
            constexpr int W = width;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[W];
#pragma unroll
                for (int k = 0; k < W; ++k)
                    v[k] = f.acc[tile + k][i];
                __builtin_memcpy(at + d0 + W * (4 * quarter + i), v, sizeof(v));
            }
        });
    };
    const auto finish = [&](int c, int r) {
        const Partial<S::kAcc> &f = o[c];
        const int head = 16 * c + col;
        if (SHARED && hv == 0 && lane == 0)
            p.found[r] = int2{0, 0};
        if (head >= n_heads)
            return;
        if (SHARED) {
            const int64_t at = (int64_t)r * (p.kv_heads * p.group) + first_head + head;
            put_wide(f, p.own + at * D);
            if (quarter == 0)
                *reinterpret_cast<f32x2 *>(p.own_stat + at * 2) = f32x2{f.ref, f.sum};
            return;
        }
        const float scale = f.sum == 0.0f ? 0.0f : p.value_scale / f.sum;
        uint16_t *at = static_cast<uint16_t *>(p.out) + r * p.out_stride +
                       (int64_t)(first_head + head) * D;
        each_piece([&](auto width, int d0, int tile) {
            constexpr int W = width;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t v[W / 2];
#pragma unroll
                for (int k = 0; k < W / 2; ++k)
                    v[k] = narrow2<TYPE>(f.acc[tile + 2 * k][i] * scale,
                                         f.acc[tile + 2 * k + 1][i] * scale);
                typedef typename Piece<2 * W>::T Vec;
                Vec x;
                __builtin_memcpy(&x, v, sizeof(x));
                *reinterpret_cast<Vec *>(at + d0 + W * (4 * quarter + i)) = x;
            }
        });
        if (quarter == 0 && p.lse)
            p.lse[(int64_t)r * (p.kv_heads * p.group) + first_head + head] =
                f.sum == 0.0f ? -__builtin_inff() : (f.ref + __builtin_amdgcn_logf(f.sum)) * kLn2;
    };
    // a partial row for the join: slot 0 of the block began before it, slot 1 in it
    const auto slot_at = [&](int which) {
        return ((int64_t)(block * 2 + which) * gridDim.y + hv) * p.group_step;
    };
    const auto hand_on = [&](int c) {
        const Partial<S::kAcc> &f = o[c];
        const int head = 16 * c + col;
        if (head >= n_heads)
            return;
        const int64_t slot = slot_at(1) + head;
        put_wide(f, p.part_out + slot * D);
        if (quarter == 0) {
            p.part_stat[slot * 2] = f.ref;
            p.part_stat[slot * 2 + 1] = f.sum;
        }
    };

    // kHead: a row that began before the range, in s_head; kEnds: and ended in it;
    // kOpen: a row that began in the range and did not end, in registers
    enum { kHead = 1, kEnds = 2, kOpen = 4 };
    int state = 0;
    int row_n = row_tiles(RowSpan{lo, hi, req}), row_first = begin - skip;  // on the line
    const int head_row = row, head_n = row_n, head_first = row_first;
    const auto next_row = [&] {
        if (++row >= rows)
            return;
        skip = 0;
        row_first += row_n;
        const RowSpan next = row_span<true, SHARED>(p, reqs, kv_len, shared, row);
        lo = next.lo;
        hi = next.hi;
        req = next.req;
        row_n = row_tiles(next);
    };
    for (; left > 0 && row < rows; next_row()) {
        const int n_tiles = min(row_n - skip, left);
        if (n_tiles == 0)
            continue;
        const int32_t *__restrict__ table = tables + (int64_t)req * p.table_cols;

        // ---- query fragments ------------------------------------------------
        u32x4 q[HT][S::kSteps];
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            const int head = 16 * c + col;
            const uint8_t *qp = static_cast<const uint8_t *>(p.q) +
                                ((int64_t)row * p.q_stride + (int64_t)(first_head + head) * D) * 2;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                // 8-bit keys hold 16 values a lane: two steps' operands side by side
                const int d = FP8 ? 64 * (s >> 1) + 16 * quarter + 8 * (s & 1)
                                  : 32 * s + 8 * quarter;
                q[c][s] = u32x4{0u, 0u, 0u, 0u};
                if (head < n_heads)
                    q[c][s] = load16(qp + d * 2);
            }
            o[c].clear();
        }

        // Places in their blocks of a tile's two halves of 16 tokens, and the blocks' ids.
        // A half without live tokens reads the other one's bytes again, from the cache,
        // instead of its own from memory.
        uint32_t place[2];
        int32_t id[2];
        const auto find = [&](int t0) {
            const uint32_t first = (uint32_t)t0 + (t0 + 16 > lo ? 0 : 16);
            const uint32_t second = (uint32_t)t0 + (t0 + 16 < hi ? 16 : 0);
            place[0] = first & (tokens - 1);
            place[1] = second & (tokens - 1);
            id[0] = table[min((int32_t)(first >> p.log2_tokens), last_col)];
            id[1] = table[min((int32_t)(second >> p.log2_tokens), last_col)];
        };

        u32x4 key[2][S::kKeyLoads];
        VPiece<TYPE, FP8, 8> v8[S::kP8 ? S::kP8 : 1];
        VPiece<TYPE, FP8, 4> v4[1];
        VPiece<TYPE, FP8, (FP8 ? 4 : 2)> v2[1];
        const uint8_t *base[2];
        bool ok[2];  // a block outside the cache is never read: the first one stands in
        uint32_t at[2];

        const auto load_keys = [&] {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ok[h] = id[h] >= 0 && id[h] < p.n_blocks;
                base[h] = p.pool + (int64_t)(ok[h] ? id[h] : 0) * p.block_stride;
                at[h] = place[h];
#pragma unroll
                for (int s = 0; s < S::kKeyLoads; ++s)
                    key[h][s] = stream<u32x4>(
                        base[h] + (key_head + at[h] * 64 + s * tokens * 64) + key_lane);
            }
        };
        // values d0 ... of the lane's 8 tokens, `width` of them a lane
        const auto load_piece = [&](auto &v, int d0, int width) {
            typedef typename std::remove_reference<decltype(v)>::type::Raw Raw;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int h = j >> 2;
                const uint32_t t = at[h] + 4 * (j & 3);
                v.raw[j] = stream<Raw>(base[h] + (val_head + (t * D + d0) * S::kElt) +
                                       (quarter * D + col * width) * S::kElt);
            }
        };
        const auto load_values = [&] {
#pragma unroll
            for (int i = 0; i < S::kP8; ++i)
                load_piece(v8[i], 128 * i, 8);
            if (S::kP4)
                load_piece(v4[0], 128 * S::kP8, 4);
            if (S::kP2)
                load_piece(v2[0], 128 * S::kP8 + 64 * S::kP4, 2);
        };
        const int tile0 = (lo / kTile + skip) * kTile;
        find(tile0);
        load_keys();
        find(tile0 + kTile);
        // one tile; with more to come, its softmax runs under the next one's key loads
        const auto take = [&](int t0, auto more) {
            const bool ok0 = ok[0], ok1 = ok[1];
            load_values();

            // ---- S^T = K Q^T -------------------------------------------------
            f32x4 scores[HT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int c = 0; c < HT; ++c)
                    scores[c][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
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
#pragma unroll
                    for (int c = 0; c < HT; ++c)
                        scores[c][h] = mfma32<TYPE>(a, q[c][s], scores[c][h]);
                }
            }
            if (more) {
                load_keys();
                find(t0 + 2 * kTile);
            }

            // ---- softmax over this lane's 8 tokens ----------------------------
            float to_ref = to_log2;
            uint32_t keep[8];  // of V: what lies in a dead token's place may be no number
#pragma unroll
            for (int j = 0; j < 8; ++j)
                keep[j] = ~0u;
            if (t0 < lo || t0 + kTile > hi || !ok0 || !ok1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = t0 + 16 * (j >> 2) + 4 * (j & 3) + quarter;
                    const bool live = t >= lo && t < hi && (j < 4 ? ok0 : ok1);
#pragma unroll
                    for (int c = 0; c < HT; ++c) {
                        const float x = scores[c][j >> 2][j & 3] * to_log2;
                        scores[c][j >> 2][j & 3] = live ? x : -__builtin_inff();
                    }
                    keep[j] = live ? ~0u : 0u;
                }
                to_ref = 1.0f;
            }
            u32x4 p_hi[HT], p_lo[HT];
#pragma unroll
            for (int c = 0; c < HT; ++c) {
                float x[8];  // score - ref, in powers of two
                // the product is rounded before the difference: the largest score, which
                // the reference came from, is then kLift above it whatever its size
                const auto weigh = [&](float ref) {
#pragma clang fp contract(off)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] = scores[c][j >> 2][j & 3] * to_ref - ref;
                    float m = x[0];
#pragma unroll
                    for (int j = 1; j < 8; ++j)
                        m = fmaxf(m, x[j]);
                    return m;
                };
                if (__any(weigh(o[c].ref) > kRoom)) {
                    const float ref = fmaxf(quarters_max(weigh(0.0f)) - kLift, o[c].ref);
                    const float shrink = __builtin_amdgcn_exp2f(o[c].ref - ref);
                    o[c].ref = ref;
                    o[c].sum *= shrink;
#pragma unroll
                    for (int i = 0; i < S::kAcc; ++i)
                        o[c].acc[i] *= shrink;
                    weigh(ref);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = __builtin_amdgcn_exp2f(x[j]);
                // added up first: beside a large sum one small weight would round away
                o[c].sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t hi2, lo2;
                    split2<TYPE>(x[2 * j], x[2 * j + 1], hi2, lo2);
                    p_hi[c][j] = hi2;
                    p_lo[c][j] = lo2;
                }
            }

            // ---- O^T += V^T P^T -----------------------------------------------
            int tile = 0;
            const auto turn = [&](auto &v, int width) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v.raw[j] &= keep[j];
#pragma unroll
                for (int i = 0; i < width / 2; ++i) {
                    u32x4 even, odd;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t e, d;
                        v.turn(i, j, e, d);
                        even[j] = e;
                        odd[j] = d;
                    }
#pragma unroll
                    for (int c = 0; c < HT; ++c) {
                        f32x4 &x = o[c].acc[tile], &y = o[c].acc[tile + 1];
                        x = mfma32<TYPE>(even, p_hi[c], x);
                        x = mfma32<TYPE>(even, p_lo[c], x);
                        y = mfma32<TYPE>(odd, p_hi[c], y);
                        y = mfma32<TYPE>(odd, p_lo[c], y);
                    }
                    tile += 2;
                }
            };
#pragma unroll
            for (int i = 0; i < S::kP8; ++i)
                turn(v8[i], 8);
            if (S::kP4)
                turn(v4[0], 4);
            if (S::kP2)
                turn(v2[0], 2);
        };
        for (int u = 0; u < n_tiles - 1; ++u)
            take(tile0 + u * kTile, std::true_type());
        take(tile0 + (n_tiles - 1) * kTile, std::false_type());
        left -= n_tiles;
        const bool ends = skip + n_tiles == row_n;
        state |= skip > 0 ? kHead | (ends ? kEnds : 0) : ends ? 0 : kOpen;
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            o[c].sum = quarters_sum(o[c].sum);
            if (skip > 0) {
#pragma unroll
                for (int i = 0; i < S::kAcc; ++i)
                    s_head[wave][c][i * 64 + lane] = o[c].acc[i];
                s_stat[wave][c][lane] = o[c].ref;
                s_stat[wave][c][64 + lane] = o[c].sum;
            } else if (ends) {
                finish(c, row);
            }
        }
        if (left == 0)
            break;
    }

    // ---- what the block's waves share ------------------------------------------
    if (lane == 0)
        s_state[wave] = state;
    __syncthreads();
    const int states = s_state[lane & (kWaves - 1)];
    const auto state_of = [&](int i) { return __builtin_amdgcn_readlane(states, i); };
    if (state & kOpen) {
        bool ends = false;
        for (int i = wave + 1; i < kWaves && !ends; ++i) {
#pragma unroll
            for (int c = 0; c < HT; ++c)
                o[c].join(s_head[i][c], s_stat[i][c], lane);
            ends = state_of(i) & kEnds;
        }
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            if (ends)
                finish(c, row);
            else
                hand_on(c);
        }
        if (!ends && hv == 0) {
            const int blocks = (int)line.of(row_first + row_n - 1) / kWaves - block + 1;
            s_join[3] = row;
            s_join[4] = blocks;
            if (SHARED && lane == 0)
                p.found[row] = int2{block, blocks};
        }
    }
    // A row that began in an earlier block: all of its parts lie in LDS, and the waves
    // share their join.  Against wave 0 alone: one row of 777 tokens 11.1 / 11.6 us,
    // 131000 tokens beside 16 short rows 97.3 / 97.9.
    if (state_of(0) & kHead) {
        int n = 1;  // waves that have parts of it
        while (n < kWaves && !(state_of(n - 1) & kEnds) && (state_of(n) & kHead))
            ++n;
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            const int head = 16 * c + col;
            float weight[kWaves], ref = kNone, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                weight[i] = i < n ? s_stat[i][c][lane] : kNone;
                ref = fmaxf(ref, weight[i]);
            }
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                weight[i] = __builtin_amdgcn_exp2f(weight[i] - ref);
                if (i < n)
                    sum += s_stat[i][c][64 + lane] * weight[i];
            }
            const int64_t slot = slot_at(0) + head;
            // a pair of output tiles at a time, dealt to the waves
            for (int t = 2 * wave; t < S::kAcc; t += 2 * kWaves) {
                f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
#pragma unroll
                for (int i = 0; i < kWaves; ++i) {
                    if (i < n) {
                        x += s_head[i][c][t * 64 + lane] * weight[i];
                        y += s_head[i][c][(t + 1) * 64 + lane] * weight[i];
                    }
                }
                const int width = t < 8 * S::kP8 ? 8 : (t < 8 * S::kP8 + 4 * S::kP4 ? 4 : 2);
                float *at = p.part_out + slot * D + (t & -width) * 16 + (t & (width - 1)) +
                            width * 4 * quarter;
                if (head < n_heads) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x2 *>(at + width * i) = f32x2{x[i], y[i]};
                }
            }
            if (wave == 0 && quarter == 0 && head < n_heads) {
                p.part_stat[slot * 2] = ref;
                p.part_stat[slot * 2 + 1] = sum;
            }
        }
        if (wave == 0 && hv == 0) {
            const int first_block = (int)line.of(head_first) / kWaves;
            s_join[0] = head_row;
            s_join[1] = first_block;
            s_join[2] = (int)line.of(head_first + head_n - 1) / kWaves - first_block + 1;
        }
    }
    if (hv == 0) {
        __syncthreads();
        if (tid < 8)
            p.join[block * 8 + tid] = s_join[tid];
    }
}

// (The join of rows that share tokens is dps_shared.hip's.)
// Joins the rows that several blocks share, and gives rows without tokens their
// zeros.  Block w of the attention left in join[w]: the row it continued from an
// earlier block (row, first block of the row, blocks of the row), and the row it
// began and handed on (row, blocks).  A row of up to kFew blocks is joined by its
// first one, which loads the partials at once, before it knows whether there are
// any: one memory latency less than in the general form (0.4-0.9 us of a call at
// 34 to 300 rows, 1.2 at 24 heads of 192).  For a longer row, the (head, 4 values)
// items are dealt to as many of its blocks as gives a thread about four partials;
// threads that share an item combine through LDS, in a fixed order.
template <int TYPE, int D>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(
    const AttnProblem p, const int32_t *__restrict__ reqs, const int32_t *__restrict__ kv_len,
    const int32_t *__restrict__ joins)
{
    constexpr int kFew = 4;
    __shared__ f32x4 s_out[kJoinThreads];
    __shared__ float s_ref[kJoinThreads], s_sum[kJoinThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int w = line_block(), blocks = gridDim.x;
    const int hv = blockIdx.y;
    const int kvh = hv / p.head_groups;
    const int sub = hv % p.head_groups;
    const int first_head = kvh * p.group + sub * p.group_step;
    const int n_heads = min(p.group_step, p.group - sub * p.group_step);
    const int items = n_heads * (D / 4);
    const int32_t *join = joins + w * 8;

    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float ref = kNone, sum = 0.0f;
    const auto add = [&](f32x4 part, float r, float l) {
        const float to = fmaxf(ref, r);
        const float a = __builtin_amdgcn_exp2f(ref - to), b = __builtin_amdgcn_exp2f(r - to);
        o = o * a + part * b;
        sum = sum * a + l * b;
        ref = to;
    };
    // place of partial k of a row whose first block is w0: the first one is what that
    // block began, the others what theirs continued
    const auto slot_of = [&](int w0, int k) {
        return ((int64_t)((w0 + k) * 2 + (k == 0 ? 1 : 0)) * gridDim.y + hv) * p.group_step;
    };

    f32x4 part[kFew];
    float part_ref[kFew], part_sum[kFew];
    const auto load = [&](int item) {
#pragma unroll
        for (int k = 0; k < kFew; ++k) {  // past the last block: its own partial again
            const int64_t slot = slot_of(w, min(k, blocks - 1 - w)) + item / (D / 4);
            part[k] = *reinterpret_cast<const f32x4 *>(p.part_out + slot * D + item % (D / 4) * 4);
            part_ref[k] = p.part_stat[slot * 2];
            part_sum[k] = p.part_stat[slot * 2 + 1];
        }
    };
    load(min(tid, items - 1));
    const int began = join[4];  // blocks of the row that block w began
    if (began > 0 && began <= kFew) {
        for (int item = tid; item < items;) {
            o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            ref = kNone;
            sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kFew; ++k)
                if (k < began)
                    add(part[k], part_ref[k], part_sum[k]);
            attn_store<TYPE>(p, join[3], first_head + item / (D / 4), D, item % (D / 4) * 4, o, ref,
                             sum);
            item += kJoinThreads;
            if (item < items)
                load(item);
        }
    }

    for (int64_t r0 = w + (int64_t)wave * 64 * blocks; r0 < p.rows;
         r0 += (int64_t)kJoinThreads * blocks) {
        const int64_t r = r0 + (int64_t)lane * blocks;
        uint64_t none =
            __ballot(r < p.rows && row_span<false, false>(p, reqs, kv_len, nullptr, (int32_t)r).hi == 0);
        for (; none; none &= none - 1) {
            const int64_t row = r0 + (int64_t)__builtin_ctzll(none) * blocks;
            for (int i = lane; i < items; i += 64)
                attn_store<TYPE>(p, row, first_head + i / (D / 4), D, i % (D / 4) * 4,
                                 f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0.0f, 0.0f);
        }
    }

    for (int mine = 0; mine < 2; ++mine) {
        const int row = join[mine ? 3 : 0], count = join[mine ? 4 : 2];
        if (count <= kFew)
            continue;
        const int w0 = mine ? w : join[1];
        // the w - w0-th of the row's blocks takes that slice of the items
        const int slices = min(count, (count * items + 4 * kJoinThreads - 1) / (4 * kJoinThreads));
        if (w - w0 >= slices)
            continue;
        const int each = (items + slices - 1) / slices;
        const int end = min((w - w0 + 1) * each, items);
        for (int i0 = (w - w0) * each; i0 < end; i0 += kJoinThreads) {
            const int n = min(end - i0, kJoinThreads);
            int groups = 1;  // threads an item
            while (2 * groups * n <= kJoinThreads && groups < count)
                groups *= 2;
            const int g = tid / n, item = i0 + tid % n;
            const int head = item / (D / 4), d = item % (D / 4) * 4;
            o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            ref = kNone;
            sum = 0.0f;
            if (g < groups) {
#pragma unroll 4
                for (int k = g; k < count; k += groups) {
                    const int64_t slot = slot_of(w0, k) + head;
                    add(*reinterpret_cast<const f32x4 *>(p.part_out + slot * D + d),
                        p.part_stat[slot * 2], p.part_stat[slot * 2 + 1]);
                }
            }
            for (int half = groups / 2; half > 0; half /= 2) {
                if (g >= half && g < 2 * half) {
                    s_out[tid] = o;
                    s_ref[tid] = ref;
                    s_sum[tid] = sum;
                }
                __syncthreads();
                if (g < half)
                    add(s_out[tid + half * n], s_ref[tid + half * n], s_sum[tid + half * n]);
                __syncthreads();
            }
            if (g == 0)
                attn_store<TYPE>(p, row, first_head + head, D, d, o, ref, sum);
        }
    }
}

template <int TYPE, bool FP8, int D, bool SHARED>
hipError_t launch(const AttnProblem &p, int blocks, hipStream_t stream)
{
    const int heads = p.kv_heads * p.head_groups;
    const dim3 grid((unsigned)blocks, (unsigned)heads);
    constexpr int most = attn_heads_a_pass(FP8, D) / 16;
    if (p.group_step > 16)
        hipLaunchKernelGGL((attn_kernel<TYPE, FP8, D, most, SHARED>), grid, dim3(kThreads), 0,
                           stream, p, p.table, p.req, p.kv_len, p.shared);
    else
        hipLaunchKernelGGL((attn_kernel<TYPE, FP8, D, 1, SHARED>), grid, dim3(kThreads), 0, stream,
                           p, p.table, p.req, p.kv_len, p.shared);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || SHARED)
        return e;
    hipLaunchKernelGGL((attn_join_kernel<TYPE, D>), dim3((unsigned)blocks, (unsigned)heads),
                       dim3(kJoinThreads), 0, stream, p, p.req, p.kv_len, p.join);
    return hipGetLastError();
}

template <int TYPE, bool SHARED>
hipError_t launch_type(const AttnProblem &p, bool fp8, int dim, int blocks, hipStream_t stream)
{
    switch (dim) {
    case 64: return fp8 ? launch<TYPE, true, 64, SHARED>(p, blocks, stream)
                        : launch<TYPE, false, 64, SHARED>(p, blocks, stream);
    case 96: return fp8 ? hipErrorInvalidValue : launch<TYPE, false, 96, SHARED>(p, blocks, stream);
    case 128: return fp8 ? launch<TYPE, true, 128, SHARED>(p, blocks, stream)
                         : launch<TYPE, false, 128, SHARED>(p, blocks, stream);
    case 192: return fp8 ? launch<TYPE, true, 192, SHARED>(p, blocks, stream)
                         : launch<TYPE, false, 192, SHARED>(p, blocks, stream);
    case 256: return fp8 ? launch<TYPE, true, 256, SHARED>(p, blocks, stream)
                         : launch<TYPE, false, 256, SHARED>(p, blocks, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_attn(const AttnProblem &p, int type, bool fp8, int dim, int blocks,
                       hipStream_t stream)
{
    if (p.shared)
        return type == KV_BF16 ? launch_type<KV_BF16, true>(p, fp8, dim, blocks, stream)
                               : launch_type<KV_F16, true>(p, fp8, dim, blocks, stream);
    return type == KV_BF16 ? launch_type<KV_BF16, false>(p, fp8, dim, blocks, stream)
                           : launch_type<KV_F16, false>(p, fp8, dim, blocks, stream);
}

}  // namespace dps
