// dps_shared.hip -- attention of one new token a row where rows share a prefix
// (gfx950).
//
// Rows of a group attend the group's first L tokens, which lie in the same blocks for
// all of them, and then tokens of their own.  With (o, m, l) the weighted values, the
// reference score and the sum of weights of a part of a row's tokens, two parts join as
//     m = max(m1, m2),  o = o1 2^(m1 - m) + o2 2^(m2 - m),  l alike,
// so the shared part is computed for all rows of a group at once: their query heads
// (of one key/value head) are the columns of the same matrix products, and a key or
// value is read once for all of them.  Three launches: shared_kernel here, attn_kernel
// (dps_attn.hip) over each row's own tokens, and shared_join_kernel.
//
// shared_kernel.  An item is up to `columns` columns of a group.  The tiles of all items
// of a key/value head, each as long as it takes a block, form one line, cut into equal
// ranges, one a block of threads; a block has a contiguous part of an item at a time, and
// leaves one partial for it (slot block + item: of two neighbours on the line that share
// an item, or of two items that share a block, no two slots are the same).  A block's
// waves have different tokens, and join in LDS.  shared_wide_kernel takes more columns at a
// time: as many of its waves as the item needs have columns of their own, and teams of them
// different tokens.  Where groups are few, there every item gets whole blocks of its own
// instead, as many as make the longest range shortest: a block that begins and ends an item
// twice loses 6 to 10 us (240 rows of 64 heads under 16384 tokens: 250 us on the line, 230
// so).  In shared_kernel one or two groups of several items do the same where that makes no
// range more than an eighth longer: the items' blocks then read the same tokens at the same
// time (96 columns of 60000 FP16 tokens, 8 key/value heads: 123 us on the line, 77 so; of
// 16384 50 and 40, and 51 with a bound of a sixteenth).  Longer ranges go either way: 192
// columns of 16384 tokens and 16 key/value heads 81 us on the line, 94 with whole blocks, 84
// columns of each of two prefixes of 9000 and 24 heads 134 and 87.
//
// The tile is attn_kernel's: S^T = K Q^T and O^T = V^T P^T on 16 x 16 x 32 matrix
// instructions, 32 tokens at a time, HT column tiles of 16 a wave; keys and values go
// from memory to registers, values are turned there, and the weights enter the matrix
// cores as two 16-bit terms (dps_attn.hip has the precision).
#include <type_traits>

#include "dps_attn.h"
#include "dps_gemm_common.h"
#include "dps_internal.h"

namespace dps {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kFewGroups = 16;  // whose items get whole blocks where they can, of many columns

// What every lane of the wave holds, in a scalar register.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// How a kernel deals columns to a block's waves, MOST of them with columns of their own,
// and how long a tile takes it, of at most MOST: what is its own of memory and LDS (BASE),
// and team turns for the rest.
template <int WAVES, int COLUMNS, int MOST, int BASE>
struct Deal {
    static constexpr int kWaves = WAVES;
    static constexpr int kMost = MOST;

    static __device__ __forceinline__ int32_t waves(const SharedProblem &p, int32_t rows)
    {
        return (rows * p.attn.group_step + COLUMNS - 1) / COLUMNS;
    }
    static __device__ __forceinline__ int32_t weight(const SharedProblem &p, int32_t rows)
    {
        if (MOST == 1)
            return 1;
        const int32_t turns = MOST / (MOST / waves(p, rows));
        return (BASE * MOST + (MOST - BASE) * turns + MOST / 2) / MOST;
    }
};

// Where the groups lie: the length of the line of a key/value head before each group, the
// items, and the table row of its first row where that has the whole prefix (-1: another
// may).
struct Groups {
    int32_t line[kSharedGroups + 1];
    int32_t items[kSharedGroups + 1];
    int32_t lead[kSharedGroups];
    int32_t first[kSharedGroups], rows[kSharedGroups], length[kSharedGroups];
    int32_t sums[2][8];  // a wave
    int32_t best;        // the least share tried that fits
    int32_t share;       // > 0: items have whole blocks, of at most so much of the line; and
                         // `line` counts blocks
};

// Tokens that a row has, as far as its table row holds them.
__device__ __forceinline__ int32_t tokens_of(const SharedProblem &p, int32_t row, int32_t &req)
{
    const AttnProblem &a = p.attn;
    req = a.req ? a.req[row] : row;
    if (req < 0 || req >= a.requests)
        return 0;
    const int64_t room = min(a.table_cols << a.log2_tokens, kLongest);
    return (int32_t)min((int64_t)max(a.kv_len[row], 0), room);
}

// Rows of group g and its length.  A length past the table's columns is no row's, and
// the group shares nothing.  rows < 0: it does not lie within the rows.
struct Group {
    int32_t first, rows, length;
};
__device__ __forceinline__ Group group_of(const SharedProblem &p, int32_t g)
{
    Group x;
    x.first = p.group_start[g];
    const int32_t next = p.group_start[g + 1];
    x.rows = x.first < 0 || next < x.first || next > p.attn.rows ? -1 : next - x.first;
    const int64_t room = min(p.attn.table_cols << p.attn.log2_tokens, kLongest);
    x.length = max(p.shared_len[g], 0);
    if (x.length > room)
        x.length = 0;
    return x;
}
__device__ __forceinline__ int32_t tiles_of(const Group &x)
{
    return (int32_t)(((uint32_t)x.length + kTile - 1) / kTile);
}
__device__ __forceinline__ int32_t items_of(const SharedProblem &p, const Group &x)
{
    return x.length > 0 ? (x.rows + p.item_rows - 1) / p.item_rows : 0;
}

// The items of a group on the line: full ones, and a last one that may have fewer rows.
template <typename DEAL>
struct Items {
    int32_t tiles, count, full, last;  // tiles and weights

    __device__ __forceinline__ Items(const SharedProblem &p, const Group &x)
        : tiles(tiles_of(x)), count(items_of(p, x)), full(0), last(0)
    {
        if (count > 0) {
            full = DEAL::weight(p, p.item_rows);
            last = DEAL::weight(p, x.rows - (count - 1) * p.item_rows);
        }
    }
    // whole blocks of an item, at `share` each, and of all
    __device__ __forceinline__ int32_t blocks(int32_t weight, int32_t share) const
    {
        const int32_t length = weight * tiles;
        int32_t n = (int32_t)((float)length * __builtin_amdgcn_rcpf((float)share));
        while ((int64_t)n * share < length)  // at most a few: the quotient was rounded
            ++n;
        return n;
    }
    __device__ __forceinline__ int32_t blocks(int32_t share) const
    {
        return count > 0 ? (count - 1) * blocks(full, share) + blocks(last, share) : 0;
    }
    __device__ __forceinline__ int32_t begin(int32_t i) const { return i * full * tiles; }
    __device__ __forceinline__ int32_t weight(int32_t i) const
    {
        return i < count - 1 ? full : last;
    }
    __device__ __forceinline__ int32_t length() const
    {
        return count > 0 ? begin(count - 1) + last * tiles : 0;
    }
};

// Fills s for all groups; false: the groups do not ascend within the rows, and nothing
// is shared.
template <typename DEAL>
__device__ __forceinline__ bool find_groups(const SharedProblem &p, Groups &s, int32_t blocks)
{
    constexpr int WAVES = DEAL::kWaves;
    constexpr int kPer = kSharedGroups / (64 * WAVES);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t lengths[kPer], items[kPer], length = 0, n_items = 0;
    int32_t req[kPer], has[kPer];  // of the groups' first rows; they arrive under the scan
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int32_t g = i * (64 * WAVES) + tid;
        if (g < p.groups) {
            const Group x = group_of(p, g);
            bad = bad || x.rows < 0;
            s.first[g] = x.first;
            s.rows[g] = x.rows;
            s.length[g] = x.length;
            has[i] = -1;
            if (x.rows > 0)
                has[i] = tokens_of(p, x.first, req[i]) - x.length;
        }
    }
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int32_t g = tid * kPer + i;
        lengths[i] = items[i] = 0;
        if (g < p.groups && !bad) {
            const Items<DEAL> x(p, Group{s.first[g], s.rows[g], s.length[g]});
            items[i] = x.count;
            lengths[i] = x.length();
        }
        length += lengths[i];
        n_items += items[i];
    }
    const int32_t incl_length = wave_scan(length), incl_items = wave_scan(n_items);
    if (lane == 63) {
        s.sums[0][wave] = incl_length;
        s.sums[1][wave] = incl_items;
    }
    __syncthreads();
    int32_t at = incl_length - length, at_item = incl_items - n_items;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        at += i < wave ? s.sums[0][i] : 0;
        at_item += i < wave ? s.sums[1][i] : 0;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int32_t g = tid * kPer + i;
        if (g <= p.groups) {
            s.line[g] = at;
            s.items[g] = at_item;
        }
        at += lengths[i];
        at_item += items[i];
    }
    if (tid == 64 * WAVES - 1 && p.groups == kSharedGroups) {
        s.line[p.groups] = at;
        s.items[p.groups] = at_item;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int32_t g = i * (64 * WAVES) + tid;
        if (g < p.groups)
            s.lead[g] = has[i] >= 0 ? req[i] : -1;
    }
    if (tid == 0) {
        s.share = 0;
        s.best = 0x7fffffff;
    }
    __syncthreads();
    const int32_t all = s.line[p.groups], all_items = s.items[p.groups];
    constexpr int kMostGroups = DEAL::kMost > 1 ? kFewGroups : kSharedAligned;
    if (bad || p.groups > kMostGroups || all_items > blocks || all <= DEAL::kMost * blocks ||
        (DEAL::kMost == 1 && all_items <= p.groups))
        return !bad;
    const int32_t mean = (all + blocks - 1) / blocks;
    {
        // thread i tries 1 + i / 128 times the mean
        const int32_t share = mean + (int32_t)((int64_t)mean * tid / 128);
        int32_t n = 0;
        for (int g = 0; g < p.groups; ++g)
            n += Items<DEAL>(p, Group{s.first[g], s.rows[g], s.length[g]}).blocks(share);
        if (n <= blocks)
            atomicMin(&s.best, share);
    }
    __syncthreads();
    const int32_t share = s.best;
    const bool use = share != 0x7fffffff && (DEAL::kMost > 1 || (share - mean) <= mean / 8);
    if (use && tid == 0) {
        s.share = share;
        int32_t at_block = 0;
        for (int g = 0; g <= p.groups; ++g) {
            s.line[g] = at_block;
            if (g < p.groups)
                at_block +=
                    Items<DEAL>(p, Group{s.first[g], s.rows[g], s.length[g]}).blocks(share);
        }
    }
    __syncthreads();
    return !bad;
}

// The last g in [0, n) with first[g] <= x, or 0.
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

// The line cut into `blocks` ranges of `each`, the first `more` one longer.  A range has
// the tiles that begin in it, and is as long as the longest tile: a block between two
// that have tiles of an item has one, too.
struct Line {
    int32_t blocks, each, more;

    __device__ __forceinline__ Line(int32_t length, int32_t most, int32_t tile)
        : blocks(length > 0 ? max(1, min(length / tile, most)) : 0), each(length / max(blocks, 1)),
          more(length - each * blocks)
    {
    }
    __device__ __forceinline__ int32_t begin(int32_t b) const { return b * each + min(b, more); }
    __device__ __forceinline__ int32_t of(int32_t t) const
    {
        const int32_t cut = more * (each + 1);
        return t < cut ? t / (each + 1) : more + (t - cut) / each;
    }
};

// What every row shares, and that no own token of it has been met.
template <typename DEAL>
__device__ __forceinline__ void put_rows(const SharedProblem &p, const Groups &s, bool good,
                                         const Line &line, int32_t block, int32_t blocks)
{
    constexpr int WAVES = DEAL::kWaves;
    for (int64_t r = (int64_t)block * (64 * WAVES) + threadIdx.x; r < p.attn.rows;
         r += (int64_t)blocks * (64 * WAVES)) {
        SharedRow x = {0, 0, 0, 0};
        // the last group that begins at or before r
        const int lo = good && p.groups > 0 ? last_from(s.first, p.groups, (int32_t)r) : 0;
        if (good && p.groups > 0 && r >= s.first[lo] && r < s.first[lo] + s.rows[lo]) {
            const Group g = {s.first[lo], s.rows[lo], s.length[lo]};
            int32_t req;
            if (g.length > 0 && tokens_of(p, (int32_t)r, req) >= g.length) {
                const Items<DEAL> items(p, g);
                const int32_t at = ((int32_t)r - g.first) / p.item_rows;
                x.start = g.length;
                x.column = (((int32_t)r - g.first) % p.item_rows) * p.attn.group_step;
                if (s.share > 0) {
                    x.slot = s.line[lo] + at * items.blocks(items.full, s.share);
                    x.count = items.blocks(items.weight(at), s.share);
                } else {
                    const int32_t begin = s.line[lo] + items.begin(at);
                    const int32_t b0 = line.of(begin);
                    x.slot = b0 + s.items[lo] + at;
                    x.count = line.of(begin + (items.tiles - 1) * items.weight(at)) - b0 + 1;
                }
            }
        }
        p.rows[r] = x;
        p.attn.found[r] = int2{0, -1};
    }
}

// A block's next part of an item: tiles skip ... skip + part - 1 (none: part <= 0) of item
// `at` of its group, and where it goes on.
struct Part {
    int32_t at, skip, part, next;
};
template <typename DEAL>
__device__ __forceinline__ Part next_part(const SharedProblem &p, const Group &grp, int32_t line,
                                          int32_t share, int32_t from, int32_t end)
{
    const Items<DEAL> items(p, grp);
    const int32_t x = from - line;
    Part r;
    if (share > 0) {
        const int32_t each = items.blocks(items.full, share);
        r.at = min(x / each, items.count - 1);
        const int32_t n = items.blocks(items.weight(r.at), share), k = x - r.at * each;
        r.skip = (int32_t)((int64_t)items.tiles * k / n);
        r.part = (int32_t)((int64_t)items.tiles * (k + 1) / n) - r.skip;
        r.next = end;
        return r;
    }
    r.at = min(x / (items.full * items.tiles), items.count - 1);
    const int32_t begin = items.begin(r.at), w = items.weight(r.at);
    const int32_t stop = min(end - line, begin + w * items.tiles);
    r.skip = (x - begin + w - 1) / w;
    r.part = (stop - begin + w - 1) / w - r.skip;
    r.next = line + stop;
    return r;
}

// The table row through which a group's prefix is read: that of the first row that has
// all of it; -1: none has.
__device__ __forceinline__ int32_t lead_of(const SharedProblem &p, const Group &grp, int32_t first,
                                           int lane)
{
    if (first >= 0)
        return first;
    for (int32_t r = grp.first; r < grp.first + grp.rows; r += 64) {
        int32_t req = -1;
        const bool has = r + lane < grp.first + grp.rows &&
                         tokens_of(p, r + lane, req) >= grp.length;
        const uint64_t any = __ballot(has);
        if (any)
            return __builtin_amdgcn_readlane(req, __builtin_ctzll(any));
    }
    return -1;
}

template <int TYPE, bool FP8, int D, int HT>
__global__ __launch_bounds__(kThreads, (Shape<TYPE, FP8, D, HT>::kWavesPerSimd)) void shared_kernel(
    const SharedProblem p, const int32_t *__restrict__ tables)
{
    typedef Shape<TYPE, FP8, D, HT> S;
    __shared__ Groups s_groups;
    __shared__ f32x4 s_part[kWaves][S::kAcc * 64];  // a column tile at a time
    __shared__ float s_stat[kWaves][128];

    const AttnProblem &a = p.attn;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    // the heads of one key/value head on one XCD, which deals blocks in turn: their items
    // read the same tokens
    const int heads = a.kv_heads * a.head_groups;
    const int hv = blockIdx.x % heads, block = blockIdx.x / heads, blocks = gridDim.x / heads;
    const int kvh = hv / a.head_groups, sub = hv % a.head_groups;
    const int first_head = kvh * a.group + sub * a.group_step;
    const int n_heads = min(a.group_step, a.group - sub * a.group_step);

    typedef Deal<kWaves, 16 * HT, 1, 0> DealT;
    const bool good = find_groups<DealT>(p, s_groups, blocks);
    const int32_t share = uniform(s_groups.share);
    const Line line(good ? s_groups.line[p.groups] : 0, blocks, DealT::kMost);
    if (hv == 0)
        put_rows<DealT>(p, s_groups, good, line, block, blocks);
    if (block >= (share > 0 ? uniform(s_groups.line[p.groups]) : line.blocks))
        return;

    const uint32_t tokens = 1u << a.log2_tokens;
    const uint32_t key_lane = (4 * (col & 3) + (col >> 2)) * 64 + quarter * 16;
    const uint32_t key_head = (uint32_t)kvh * S::kKeyLoads * tokens * 64;
    const uint32_t val_head = (uint32_t)(a.kv_heads + kvh) * tokens * (D * S::kElt);
    const float to_log2 = a.score_scale * kLog2e;
    const int32_t last_col = (int32_t)a.table_cols - 1;

    int32_t at = share > 0 ? block : uniform(line.begin(block));
    const int32_t end = share > 0 ? block + 1 : uniform(line.begin(block + 1));
    int g = uniform(last_from(s_groups.line, p.groups, at));
    while (at < end) {
        while (uniform(s_groups.line[g + 1]) <= at)  // past groups without tiles
            ++g;
        const Group grp = {uniform(s_groups.first[g]), uniform(s_groups.rows[g]),
                           uniform(s_groups.length[g])};
        const Part now = next_part<DealT>(p, grp, uniform(s_groups.line[g]), share, at, end);
        at = now.next;
        const int32_t skip = now.skip, part = now.part;
        const int32_t item = share > 0 ? 0 : uniform(s_groups.items[g]) + now.at;
        const int32_t row0 = grp.first + now.at * p.item_rows;
        const int32_t n_rows = min(p.item_rows, grp.first + grp.rows - row0);
        if (part <= 0)
            continue;
        const int32_t lead = lead_of(p, grp, uniform(s_groups.lead[g]), lane);
        if (lead < 0)
            continue;  // no row reads the partials
        const int32_t *__restrict__ table = tables + (int64_t)lead * a.table_cols;

        // ---- query fragments ------------------------------------------------------
        int32_t column[HT];
        bool used[HT];
        u32x4 q[HT][S::kSteps];
        f32x4 acc[HT][S::kAcc];
        float ref[HT], sum[HT];
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            column[c] = c * 16 + col;
            const int32_t r = column[c] / a.group_step, head = column[c] % a.group_step;
            used[c] = r < n_rows && head < n_heads;
            const uint8_t *qp = static_cast<const uint8_t *>(a.q) +
                                ((int64_t)(row0 + r) * a.q_stride +
                                 (int64_t)(first_head + head) * D) * 2;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                const int d = FP8 ? 64 * (s >> 1) + 16 * quarter + 8 * (s & 1)
                                  : 32 * s + 8 * quarter;
                q[c][s] = u32x4{0u, 0u, 0u, 0u};
                if (used[c])
                    q[c][s] = load16(qp + d * 2);
            }
            ref[c] = kNone;
            sum[c] = 0.0f;
#pragma unroll
            for (int i = 0; i < S::kAcc; ++i)
                acc[c][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        // this wave's tiles of the part
        const int32_t u0 = skip + (int32_t)((int64_t)part * wave / kWaves);
        const int32_t u1 = skip + (int32_t)((int64_t)part * (wave + 1) / kWaves);
        const int32_t hi = grp.length;

        uint32_t place[2];
        int32_t id[2];
        const auto find = [&](int t0) {
            const uint32_t second = (uint32_t)t0 + (t0 + 16 < hi ? 16 : 0);
            place[0] = t0 & (tokens - 1);
            place[1] = second & (tokens - 1);
            id[0] = table[min(t0 >> a.log2_tokens, last_col)];
            id[1] = table[min((int32_t)(second >> a.log2_tokens), last_col)];
        };
        u32x4 key[2][S::kKeyLoads];
        VPiece<TYPE, FP8, 8> v8[S::kP8 ? S::kP8 : 1];
        VPiece<TYPE, FP8, 4> v4[1];
        VPiece<TYPE, FP8, (FP8 ? 4 : 2)> v2[1];
        const uint8_t *base[2];
        bool ok[2];  // a block outside the cache is never read: the first one stands in
        uint32_t at_[2];
        // again: other items read the same tokens, so the caches keep them (64 rows in 8
        // groups, up to 4 items each, of 12000 E4M3 tokens: 42.7 us without, 39.2 so)
        constexpr bool kBoth = FP8 || D != 192 || HT > 1;  // else all registers are in use
        const auto load = [&](auto *to, const uint8_t *from, auto again) {
            typedef typename std::remove_reference<decltype(*to)>::type T;
            if (again)
                *to = *reinterpret_cast<const T *>(from);
            else
                *to = stream<T>(from);
        };
        const auto load_keys = [&](auto again) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ok[h] = id[h] >= 0 && id[h] < a.n_blocks;
                base[h] = a.pool + (int64_t)(ok[h] ? id[h] : 0) * a.block_stride;
                at_[h] = place[h];
#pragma unroll
                for (int s = 0; s < S::kKeyLoads; ++s)
                    load(&key[h][s],
                         base[h] + (key_head + at_[h] * 64 + s * tokens * 64) + key_lane, again);
            }
        };
        const auto load_piece = [&](auto &v, int d0, int width, auto again) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int h = j >> 2;
                const uint32_t t = at_[h] + 4 * (j & 3);
                load(&v.raw[j],
                     base[h] + (val_head + (t * D + d0) * S::kElt) +
                         (quarter * D + col * width) * S::kElt,
                     again);
            }
        };
        const auto load_values = [&](auto again) {
#pragma unroll
            for (int i = 0; i < S::kP8; ++i)
                load_piece(v8[i], 128 * i, 8, again);
            if (S::kP4)
                load_piece(v4[0], 128 * S::kP8, 4, again);
            if (S::kP2)
                load_piece(v2[0], 128 * S::kP8 + 64 * S::kP4, 2, again);
        };
        const auto take = [&](int t0, auto more, auto again) {
            const bool ok0 = ok[0], ok1 = ok[1];
            load_values(again);
            f32x4 scores[HT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int c = 0; c < HT; ++c)
                    scores[c][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) {
                    u32x4 k;
                    if (FP8) {
                        const u32x4 k16 = key[h][s >> 1];
                        const uint32_t c0 = s & 1 ? k16.z : k16.x, c1 = s & 1 ? k16.w : k16.y;
                        k = u32x4{wide2<TYPE, false>(c0), wide2<TYPE, true>(c0),
                                  wide2<TYPE, false>(c1), wide2<TYPE, true>(c1)};
                    } else {
                        k = key[h][s];
                    }
#pragma unroll
                    for (int c = 0; c < HT; ++c)
                        scores[c][h] = mfma32<TYPE>(k, q[c][s], scores[c][h]);
                }
            }
            if (more) {
                load_keys(again);
                find(t0 + 2 * kTile);
            }
            float to_ref = to_log2;
            uint32_t keep[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                keep[j] = ~0u;
            if (t0 + kTile > hi || !ok0 || !ok1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = t0 + 16 * (j >> 2) + 4 * (j & 3) + quarter;
                    const bool live = t < hi && (j < 4 ? ok0 : ok1);
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
                float x[8];
                const auto weigh = [&](float r) {
#pragma clang fp contract(off)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] = scores[c][j >> 2][j & 3] * to_ref - r;
                    float m = x[0];
#pragma unroll
                    for (int j = 1; j < 8; ++j)
                        m = fmaxf(m, x[j]);
                    return m;
                };
                if (__any(weigh(ref[c]) > kRoom)) {
                    const float r = fmaxf(quarters_max(weigh(0.0f)) - kLift, ref[c]);
                    const float shrink = __builtin_amdgcn_exp2f(ref[c] - r);
                    ref[c] = r;
                    sum[c] *= shrink;
#pragma unroll
                    for (int i = 0; i < S::kAcc; ++i)
                        acc[c][i] *= shrink;
                    weigh(r);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = __builtin_amdgcn_exp2f(x[j]);
                sum[c] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t hi2, lo2;
                    split2<TYPE>(x[2 * j], x[2 * j + 1], hi2, lo2);
                    p_hi[c][j] = hi2;
                    p_lo[c][j] = lo2;
                }
            }
            int out = 0;
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
                        f32x4 &x = acc[c][out], &y = acc[c][out + 1];
                        x = mfma32<TYPE>(even, p_hi[c], x);
                        x = mfma32<TYPE>(even, p_lo[c], x);
                        y = mfma32<TYPE>(odd, p_hi[c], y);
                        y = mfma32<TYPE>(odd, p_lo[c], y);
                    }
                    out += 2;
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
        const auto take_all = [&](auto again) {
            find(u0 * kTile);
            load_keys(again);
            find(u0 * kTile + kTile);
            for (int u = u0; u < u1 - 1; ++u)
                take(u * kTile, std::true_type(), again);
            take((u1 - 1) * kTile, std::false_type(), again);
        };
        if (u0 < u1) {
            if (kBoth && grp.rows > p.item_rows)
                take_all(std::true_type());
            else
                take_all(std::false_type());
        }

        // ---- the block's partial of the item -----------------------------------------
        const int64_t slot = ((int64_t)hv * p.slots + block + item) * p.columns;
        // the values of output tiles t and t + 1 of a column
        const auto put2 = [&](int32_t column, int t, f32x4 x, f32x4 y) {
            const int width = t < 8 * S::kP8 ? 8 : (t < 8 * S::kP8 + 4 * S::kP4 ? 4 : 2);
            float *to = p.part_out + (slot + column) * D + (t & -width) * 16 +
                        (t & (width - 1)) + width * 4 * quarter;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<f32x2 *>(to + width * k) = f32x2{x[k], y[k]};
        };
        const auto put_stat = [&](int32_t column, float r, float l) {
            *reinterpret_cast<f32x2 *>(p.part_stat + (slot + column) * 2) = f32x2{r, l};
        };
#pragma unroll
        for (int c = 0; c < HT; ++c) {
            sum[c] = quarters_sum(sum[c]);
            // the waves' parts, a pair of output tiles at a time, dealt to them
            __syncthreads();  // the column tile before has been read
#pragma unroll
            for (int i = 0; i < S::kAcc; ++i)
                s_part[wave][i * 64 + lane] = acc[c][i];
            s_stat[wave][lane] = ref[c];
            s_stat[wave][64 + lane] = sum[c];
            __syncthreads();
            float weight[kWaves], top = kNone, total = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                weight[i] = s_stat[i][lane];
                top = fmaxf(top, weight[i]);
            }
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                weight[i] = __builtin_amdgcn_exp2f(weight[i] - top);
                total += s_stat[i][64 + lane] * weight[i];
            }
            if (!used[c])
                continue;
            for (int t = 2 * wave; t < S::kAcc; t += 2 * kWaves) {
                f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
#pragma unroll
                for (int k = 0; k < kWaves; ++k) {
                    x += s_part[k][t * 64 + lane] * weight[k];
                    y += s_part[k][(t + 1) * 64 + lane] * weight[k];
                }
                put2(column[c], t, x, y);
            }
            if (wave == 0 && quarter == 0)
                put_stat(column[c], top, total);
        }
    }
}

// The same for items of many columns.  A block of waves takes ST tiles of 32 tokens at a
// time.  Each wave brings a piece of them, some keys and some values, from memory to
// registers one stage ahead, makes matrix operands of it (E4M3 widened, values turned,
// tokens that are not there cleared) and puts them into LDS, lane by lane as the
// matrix instructions take them, so that all reads and writes of LDS are 1 KiB in the
// order of the lanes.  As many waves as the item has 32 columns have columns of their own;
// as often as they go into the block's, teams of them take a stage's tiles in turn and
// join at the item's end.
//
// Products are 32 x 32 x 16: S^T of 32 tokens and 32 columns, O^T of 32 values and 32
// columns.  They read half the operands of 16 x 16 x 32 for the same work, which leaves
// the vector ALUs more of the register file: 8 waves of 16 x 16 x 32 instructions and 24
// multiply-adds beside each 8 of them take 1.45 times the instructions' own time, here
// 1.34.
//   - Lane (m, hf) = (lane % 32, lane / 32) holds row (or column) m and 8 of a step's 16
//     places in the sum, hf * 8 + j; of a result it holds column m, in register i
//     row 8 (i / 4) + 4 hf + i % 4.
//   - Keys: row m is token m, places are values 16 s + 8 hf + j of step s (E4M3: 16
//     values of a 16-byte load in two steps; the queries lie accordingly).
//   - Weights: registers 8 u + j of S^T are the places of step u of P^T as they are,
//     so token 8 (i / 4) + 4 hf + i % 4, i = 8 u + j, is what the values bring there.
//   - Values: 32 lanes read W = D / 32 neighbouring values each of a token, and value
//     W m + e is row m of output tile e (192: W = 4, then W = 2).
template <bool FP8, int D>
struct Wide {
    static constexpr int kWaves = D > 128 ? 4 : 8;  // 512 registers a lane, or 256
    static constexpr int kStage = D > 128 ? 2 : 4;  // tiles
    static constexpr int kParts = kWaves / kStage;  // pieces of a tile
    static constexpr int kFrags = D / 16;           // 1 KiB operands of a tile's keys, and values
    static constexpr int kKeys = kFrags / kParts;   // of keys in a piece
    static constexpr int kAcc = D / 32;             // output tiles
    static constexpr int kElt = FP8 ? 1 : 2;
};
// Up to here a score's product with its factor is off by less than 2^-8 when rounded, and
// weights may come from the exact one.
constexpr float kFar = 65536.0f;

typedef float f32x16 __attribute__((ext_vector_type(16)));
template <int TYPE>
__device__ __forceinline__ f32x16 mfma16(u32x4 a, u32x4 b, f32x16 c)
{
    if (TYPE == KV_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(as_half8(a), as_half8(b), c, 0, 0, 0);
}

// Over the two lanes that share a column.
template <typename F>
__device__ __forceinline__ float over_halves(float x, const F &f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    return f(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
}

template <int TYPE, bool FP8, int D>
__global__ __launch_bounds__((64 * Wide<FP8, D>::kWaves), (Wide<FP8, D>::kWaves / 4)) void
shared_wide_kernel(const SharedProblem p, const int32_t *__restrict__ tables)
{
    typedef Wide<FP8, D> W;
    constexpr int ST = W::kStage, kFrags = W::kFrags, kAcc = W::kAcc, kWideWaves = W::kWaves;
    constexpr int kFirst = D == 192 ? 4 : kAcc;  // output tiles of the values' first piece
    static_assert(W::kKeys % 2 == 0, "an E4M3 load is two steps");
    // [2 stages][tiles][keys: step; values: output tile, step]
    __shared__ u32x4 s_op[2][ST][2 * kFrags * 64];
    __shared__ uint32_t s_live[2][ST];  // tokens of a tile that are there
    __shared__ float s_stat[kWideWaves][128];
    __shared__ Groups s_groups;

    const AttnProblem &a = p.attn;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hf = lane >> 5;
    const int heads = a.kv_heads * a.head_groups;
    const int hv = blockIdx.x % heads, block = blockIdx.x / heads, blocks = gridDim.x / heads;
    const int kvh = hv / a.head_groups, sub = hv % a.head_groups;
    const int first_head = kvh * a.group + sub * a.group_step;
    const int n_heads = min(a.group_step, a.group - sub * a.group_step);

    // of a tile's time 3 of 8 parts are its own, the rest goes with its columns: 300 rows of 8
    // heads under 20 FP16 prefixes of up to 4000 tokens take 155 us with 0 of 8, 118 with 2, 111
    // with 3, 110 with 4 and 122 with 6, under 30 prefixes 179, 142, 145, 139 and 153, 256 rows
    // under 7 E4M3 prefixes of 12000 238, 188, 199, 196 and 206
    typedef Deal<kWideWaves, 32, kWideWaves, kWideWaves * 3 / 8> DealT;
    const bool good = find_groups<DealT>(p, s_groups, blocks);
    const int32_t share = uniform(s_groups.share);
    const Line line(good ? s_groups.line[p.groups] : 0, blocks, DealT::kMost);
    if (hv == 0)
        put_rows<DealT>(p, s_groups, good, line, block, blocks);
    if (block >= (share > 0 ? uniform(s_groups.line[p.groups]) : line.blocks))
        return;

    const uint32_t tokens = 1u << a.log2_tokens;
    const uint32_t key_head = (uint32_t)kvh * tokens * (D * W::kElt);
    const uint32_t val_head = (uint32_t)(a.kv_heads + kvh) * tokens * (D * W::kElt);
    const float to_log2 = a.score_scale * kLog2e;
    const int32_t last_col = (int32_t)a.table_cols - 1;
    const int my_tile = wave / W::kParts, my_part = wave % W::kParts;
    const int my_step = my_part;  // of the values: 16 of the tile's tokens
    static_assert(W::kParts == 2, "a piece is half of a tile");

    int32_t at = share > 0 ? block : uniform(line.begin(block));
    const int32_t end = share > 0 ? block + 1 : uniform(line.begin(block + 1));
    int g = uniform(last_from(s_groups.line, p.groups, at));
    while (at < end) {
        while (uniform(s_groups.line[g + 1]) <= at)  // past groups without tiles
            ++g;
        const Group grp = {uniform(s_groups.first[g]), uniform(s_groups.rows[g]),
                           uniform(s_groups.length[g])};
        const Part now = next_part<DealT>(p, grp, uniform(s_groups.line[g]), share, at, end);
        at = now.next;
        const int32_t skip = now.skip, part = now.part;
        const int32_t item = share > 0 ? 0 : uniform(s_groups.items[g]) + now.at;
        const int32_t row0 = grp.first + now.at * p.item_rows;
        const int32_t n_rows = min(p.item_rows, grp.first + grp.rows - row0);
        if (part <= 0)
            continue;
        const int32_t lead = lead_of(p, grp, uniform(s_groups.lead[g]), lane);
        if (lead < 0)
            continue;
        const int32_t *__restrict__ table = tables + (int64_t)lead * a.table_cols;
        const int32_t hi = grp.length;

        // ---- a piece of a stage: from memory, and into LDS as operands -----------------
        constexpr int kKeyLoads = FP8 ? W::kKeys / 2 : W::kKeys;
        u32x4 key[FP8 ? kKeyLoads : 1];
        constexpr int kVal = (D / 32 * W::kElt + 3) / 4;
        uint32_t val[8][kVal];    // of eight tokens
        uint32_t live = 0;        // bits of the tile's tokens
        int32_t id[2];
        const auto find = [&](int32_t stage) {  // block ids, one stage ahead of their use
            // past the longest prefix no signed number holds it
            const uint32_t t0 = (uint32_t)(skip + stage * ST + my_tile) * kTile;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                id[h] = table[min((int32_t)(min(t0 + 16 * h, (uint32_t)hi - 1) >> a.log2_tokens),
                                  last_col)];
        };
        // N values a lane of eight tokens, into val from dword to on
        const auto fetch_values = [&](auto width, const uint8_t *from, uint32_t place, int d0,
                                     auto to) {
            constexpr int N = width;
            typedef typename Piece<N * W::kElt>::T T;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t t = place + 8 * (j >> 2) + 4 * hf + (j & 3);
                const T x = *reinterpret_cast<const T *>(
                    from + (val_head + (t * D + d0 + col * N) * W::kElt));
                uint32_t v[4] = {};
                __builtin_memcpy(v, &x, sizeof(x));
#pragma unroll
                for (int k = 0; k < (int)(sizeof(x) + 3) / 4; ++k)
                    val[j][to + k] = v[k];
            }
        };
        const auto fetch = [&](int32_t stage) {
            const int32_t u = stage * ST + my_tile;
            if (u >= part)
                return;
            const int32_t t0 = (skip + u) * kTile;
            const uint8_t *base[2];
            uint32_t place[2];
            live = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool ok = id[h] >= 0 && id[h] < a.n_blocks;
                base[h] = a.pool + (int64_t)(ok ? id[h] : 0) * a.block_stride;
                place[h] = (uint32_t)(t0 + 16 * h) & (tokens - 1);
                const int32_t left = max(0, min(hi - (t0 + 16 * h), 16));
                if (ok)
                    live |= ((1u << left) - 1u) << 16 * h;
            }
            const uint8_t *from = (col < 16 ? base[0] : base[1]) +
                                  (key_head + ((col < 16 ? place[0] : place[1]) + (col & 15)) * 64 +
                                   hf * 16);
#pragma unroll
            for (int i = 0; i < kKeyLoads; ++i) {
                const int s = my_part * kKeyLoads + i;  // 32 bytes of a token
                const uint8_t *at = from + (s >> 1) * tokens * 64 + (s & 1) * 32;
                if (FP8)
                    key[i] = *reinterpret_cast<const u32x4 *>(at);
                else  // operands as they are
                    dma16_at<AUX_CACHED>(at, (lds_u8 *)(s_op[stage & 1][my_tile] + s * 64));
            }
            const uint8_t *vals = my_step ? base[1] : base[0];
            const uint32_t vplace = my_step ? place[1] : place[0];
            fetch_values(std::integral_constant<int, kFirst>(), vals, vplace, 0,
                        std::integral_constant<int, 0>());
            if constexpr (kFirst < kAcc)
                fetch_values(std::integral_constant<int, 2>(), vals, vplace, 128,
                            std::integral_constant<int, W::kElt>());
        };
        // the values from dword d of val on, into output tiles e0 ...
        const auto turn = [&](auto width, u32x4 *to, auto d, int e0) {
            constexpr int N = width;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                u32x4 even, odd;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (FP8) {
                        const uint32_t t = __builtin_amdgcn_perm(val[2 * j + 1][d + (i >> 1)],
                                                                 val[2 * j][d + (i >> 1)],
                                                                 i & 1 ? 0x07030602u : 0x05010400u);
                        even[j] = wide2<TYPE, false>(t);
                        odd[j] = wide2<TYPE, true>(t);
                    } else {
                        const uint32_t x = val[2 * j][d + i], y = val[2 * j + 1][d + i];
                        even[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                        odd[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                    }
                }
                to[(2 * (e0 + 2 * i) + my_step) * 64] = even;
                to[(2 * (e0 + 2 * i + 1) + my_step) * 64] = odd;
            }
        };
        const auto stash = [&](int32_t stage) {
            const int32_t u = stage * ST + my_tile;
            if (u >= part)
                return;
            u32x4 *to = s_op[stage & 1][my_tile] + lane;
            const int first = my_part * W::kKeys;
#pragma unroll
            for (int i = 0; FP8 && i < W::kKeys; ++i) {
                const u32x4 k16 = key[i >> 1];
                const uint32_t c0 = i & 1 ? k16.z : k16.x, c1 = i & 1 ? k16.w : k16.y;
                to[(first + i) * 64] = u32x4{wide2<TYPE, false>(c0), wide2<TYPE, true>(c0),
                                             wide2<TYPE, false>(c1), wide2<TYPE, true>(c1)};
            }
            if (my_part == 0 && lane == 0)
                s_live[stage & 1][my_tile] = live;
            if (live != ~0u) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(live >> (16 * my_step + 8 * (j >> 2) + 4 * hf + (j & 3)) & 1))
#pragma unroll
                        for (int k = 0; k < kVal; ++k)
                            val[j][k] = 0u;
            }
            turn(std::integral_constant<int, kFirst>(), to + kFrags * 64,
                 std::integral_constant<int, 0>(), 0);
            if constexpr (kFirst < kAcc)
                turn(std::integral_constant<int, 2>(), to + kFrags * 64,
                     std::integral_constant<int, W::kElt>(), 4);
        };

        // ---- query fragments ------------------------------------------------------
        find(0);
        __syncthreads();  // the item before has been joined, in the memory of the stages
        fetch(0);
        find(1);
        const int n_waves = DealT::waves(p, n_rows);  // with columns
        const int teams = kWideWaves / n_waves;
        const int team = wave / n_waves, wc = wave - team * n_waves;
        const int32_t column = wc * 32 + col;
        const bool active = team < teams;
        const bool used =
            active && column / a.group_step < n_rows && column % a.group_step < n_heads;
        u32x4 q[kFrags];
        f32x16 acc[kAcc];
        float ref = kNone, sum = 0.0f;
        {
            const uint8_t *qp = static_cast<const uint8_t *>(a.q) +
                                ((int64_t)(row0 + column / a.group_step) * a.q_stride +
                                 (int64_t)(first_head + column % a.group_step) * D) * 2;
#pragma unroll
            for (int s = 0; s < kFrags; ++s) {
                const int d = FP8 ? 32 * (s >> 1) + 16 * hf + 8 * (s & 1) : 16 * s + 8 * hf;
                q[s] = u32x4{0u, 0u, 0u, 0u};
                if (used)
                    q[s] = load16(qp + d * 2);
            }
#pragma unroll
            for (int i = 0; i < kAcc; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    acc[i][j] = 0.0f;
        }

        bool far = false;  // a reference score so large that products are rounded first
        // operands on their way under the softmax: values, and the next tile's keys, as far
        // as registers go; the others wait for LDS where they are due
        constexpr bool kEarly = D <= 128, kEarlyKeys = D * (FP8 ? 2 : 1) <= 128;
        u32x4 k[kFrags];
        const auto read_keys = [&](const u32x4 *op) {
#pragma unroll
            for (int s = 0; s < kFrags; ++s)
                k[s] = op[s * 64];
        };
        // a tile; `next`: the one after it
        const auto take = [&](const u32x4 *op, uint32_t there, const u32x4 *next) {
            f32x16 scores;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                scores[i] = 0.0f;
#pragma unroll
            for (int s = 0; s < kFrags; ++s)
                scores = mfma16<TYPE>(kEarlyKeys ? k[s] : op[s * 64], q[s], scores);
            u32x4 v[kAcc];
            const auto read_values = [&](int u) {
#pragma unroll
                for (int i = 0; i < kAcc; ++i)
                    v[i] = op[(kFrags + 2 * i + u) * 64];
            };
            if (kEarly) {
                read_values(0);
                if (kEarlyKeys)
                    read_keys(next);
                __builtin_amdgcn_sched_barrier(0);
            }
            float x[16];
            const auto weigh = [&](float factor, float r) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = __builtin_fmaf(scores[i], factor, -r);
                float m = x[0];
#pragma unroll
                for (int i = 1; i < 16; ++i)
                    m = fmaxf(m, x[i]);
                return m;
            };
            if (__any(weigh(to_log2, ref) > kRoom) || far || there != ~0u) {
                // the products rounded before the differences: the largest score, which the
                // reference came from, is then kLift above it whatever its size
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool live = there >> (8 * (i >> 2) + 4 * hf + (i & 3)) & 1;
                    const float s = scores[i] * to_log2;
                    scores[i] = live ? s : -__builtin_inff();
                }
                const float most = over_halves(weigh(1.0f, 0.0f),
                                               [](float a, float b) { return fmaxf(a, b); });
                const float r = fmaxf(most - kLift, ref);
                const float shrink = __builtin_amdgcn_exp2f(ref - r);
                ref = r;
                sum *= shrink;
#pragma unroll
                for (int i = 0; i < kAcc; ++i)
                    acc[i] *= shrink;
                weigh(1.0f, r);
                far = __any(__builtin_fabsf(r) > kFar);
            }
            u32x4 p_hi[2], p_lo[2];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = __builtin_amdgcn_exp2f(x[i]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t hi2, lo2;
                split2<TYPE>(x[2 * i], x[2 * i + 1], hi2, lo2);
                p_hi[i >> 2][i & 3] = hi2;
                p_lo[i >> 2][i & 3] = lo2;
            }
#pragma unroll
            for (int d = 8; d > 0; d /= 2)
#pragma unroll
                for (int i = 0; i < d; ++i)
                    x[i] += x[i + d];
            sum += x[0];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (!kEarly || u > 0) {
                    __builtin_amdgcn_sched_barrier(0);
                    read_values(u);
                }
#pragma unroll
                for (int i = 0; i < kAcc; ++i)
                    acc[i] = mfma16<TYPE>(v[i], p_hi[u], acc[i]);
#pragma unroll
                for (int i = 0; i < kAcc; ++i)
                    acc[i] = mfma16<TYPE>(v[i], p_lo[u], acc[i]);
            }
        };
        // what this wave has put into LDS, its direct loads among it, is there
        const auto meet = [&] {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };

        const int32_t stages = (part + ST - 1) / ST;
        stash(0);
        meet();
        for (int32_t stage = 0; stage < stages; ++stage) {
            fetch(stage + 1);  // past the part: nothing
            find(stage + 2);
            const auto op = s_op[stage & 1];
            const int here = active ? min(ST, part - stage * ST) : 0;  // tiles of the stage
            bool stashed = false;
            if (kEarlyKeys && team < here)
                read_keys(op[team] + lane);
#pragma unroll 1
            for (int i = team; i < here; i += teams) {
                if (i >= ST / 2 && !stashed) {  // the loads have had half of the stage
                    stash(stage + 1);
                    stashed = true;
                }
                take(op[i] + lane, uniform((int32_t)s_live[stage & 1][i]),
                     op[i + teams < here ? i + teams : i] + lane);
            }
            if (!stashed)
                stash(stage + 1);
            meet();
        }

        // ---- the block's partial of the item -----------------------------------------
        const int64_t slot = ((int64_t)hv * p.slots + block + item) * p.columns;
        float *out = p.part_out + (slot + column) * D;
        const auto put_stat = [&](float r, float l) {
            *reinterpret_cast<f32x2 *>(p.part_stat + (slot + column) * 2) = f32x2{r, l};
        };
        // register i of output tiles e0 ... e0 + N - 1: neighbouring values
        const auto put = [&](auto width, int d0, int i, const float *x) {
            constexpr int N = width;
            __builtin_memcpy(out + d0 + N * (8 * (i >> 2) + 4 * hf + (i & 3)), x, 4 * N);
        };
        sum = over_halves(sum, [](float a, float b) { return a + b; });
        if (teams == 1) {
            if (used) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x[kAcc];
#pragma unroll
                    for (int e = 0; e < kAcc; ++e)
                        x[e] = acc[e][i];
                    put(std::integral_constant<int, kFirst>(), 0, i, x);
                    if constexpr (kFirst < kAcc)
                        put(std::integral_constant<int, 2>(), 128, i, x + kFirst);
                }
                if (hf == 0)
                    put_stat(ref, sum);
            }
            continue;
        }
        // teams: through LDS, kJoin registers of every output tile at a time, dealt to them
        constexpr int kJoin = sizeof(s_op) >= 4096ull * kWideWaves * kAcc ? 16 : 4;
        float *parts = reinterpret_cast<float *>(&s_op[0][0][0]);  // [waves][kJoin][kAcc][64]
        static_assert(sizeof(s_op) >= 256ull * kWideWaves * kAcc * kJoin, "they fit the stages");
        s_stat[wave][lane] = ref;
        s_stat[wave][64 + lane] = sum;
        float weight[kWideWaves], top = kNone, total = 0.0f;
#pragma unroll
        for (int i0 = 0; i0 < 16; i0 += kJoin) {
            if (i0 > 0)
                __syncthreads();
#pragma unroll
            for (int i = 0; i < kJoin; ++i)
#pragma unroll
                for (int e = 0; e < kAcc; ++e)
                    parts[((wave * kJoin + i) * kAcc + e) * 64 + lane] = acc[e][i0 + i];
            __syncthreads();
            if (i0 == 0) {
#pragma unroll
                for (int k = 0; k < kWideWaves; ++k) {
                    weight[k] = kNone;
                    if (k < teams)
                        weight[k] = s_stat[k * n_waves + wc][lane];
                    top = fmaxf(top, weight[k]);
                }
#pragma unroll
                for (int k = 0; k < kWideWaves; ++k) {
                    weight[k] = __builtin_amdgcn_exp2f(weight[k] - top);
                    if (k < teams)
                        total += s_stat[k * n_waves + wc][64 + lane] * weight[k];
                }
            }
            if (!used)
                continue;
            for (int i = team; i < kJoin; i += teams) {
                float x[kAcc];
#pragma unroll
                for (int e = 0; e < kAcc; ++e)
                    x[e] = 0.0f;
#pragma unroll
                for (int k = 0; k < kWideWaves; ++k) {
                    if (k >= teams)
                        break;
#pragma unroll
                    for (int e = 0; e < kAcc; ++e)
                        x[e] += parts[(((k * n_waves + wc) * kJoin + i) * kAcc + e) * 64 + lane] *
                                weight[k];
                }
                put(std::integral_constant<int, kFirst>(), 0, i0 + i, x);
                if constexpr (kFirst < kAcc)
                    put(std::integral_constant<int, 2>(), 128, i0 + i, x + kFirst);
            }
        }
        if (used && team == 0 && hf == 0)
            put_stat(top, total);
    }
}

// Joins a row's partials: of its shared tokens, and of its own.  A block a row and
// key/value head (and pass); the (head, 4 values) items are dealt to threads, several
// threads an item where there are many partials, which combine through LDS in a fixed
// order.
template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(const SharedProblem p)
{
    __shared__ f32x4 s_out[kThreads];
    __shared__ float s_ref[kThreads], s_sum[kThreads];
    const AttnProblem &a = p.attn;
    const int tid = threadIdx.x;
    const int heads = a.kv_heads * a.head_groups;
    const int hv = blockIdx.x % heads;
    const int64_t row = blockIdx.x / heads;
    const int kvh = hv / a.head_groups, sub = hv % a.head_groups;
    const int first_head = kvh * a.group + sub * a.group_step;
    const int n_heads = min(a.group_step, a.group - sub * a.group_step);
    const int items = n_heads * (D / 4);
    const SharedRow shared = p.rows[row];
    const int2 found = a.found[row];
    const int own = found.y < 0 ? 0 : max(found.y, 1), count = own + shared.count;

    int groups = 1;  // threads an item
    while (2 * groups * items <= kThreads && groups < count)
        groups *= 2;
    const int each = min(items, kThreads / groups);
    for (int i0 = 0; i0 < items; i0 += each) {
        const int g = tid / each, item = i0 + tid % each;
        const bool live = g < groups && item < items;
        const int head = item / (D / 4), d = item % (D / 4) * 4;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        float ref = kNone, sum = 0.0f;
        const auto add = [&](f32x4 part, float r, float l) {
            const float to = fmaxf(ref, r);
            const float x = __builtin_amdgcn_exp2f(ref - to), y = __builtin_amdgcn_exp2f(r - to);
            o = o * x + part * y;
            sum = sum * x + l * y;
            ref = to;
        };
        if (live) {
#pragma unroll 4
            for (int k = g; k < count; k += groups) {
                const float *out, *stat;
                if (k < shared.count) {
                    const int64_t at = ((int64_t)hv * p.slots + shared.slot + k) * p.columns +
                                       shared.column + head;
                    out = p.part_out + at * D;
                    stat = p.part_stat + at * 2;
                } else if (found.y == 0) {
                    const int64_t at = row * (a.kv_heads * a.group) + first_head + head;
                    out = a.own + at * D;
                    stat = a.own_stat + at * 2;
                } else {
                    const int b = k - shared.count;  // of the row's blocks
                    const int64_t at = ((int64_t)((found.x + b) * 2 + (b == 0 ? 1 : 0)) * heads + hv) *
                                           a.group_step + head;
                    out = a.part_out + at * D;
                    stat = a.part_stat + at * 2;
                }
                const f32x2 s = *reinterpret_cast<const f32x2 *>(stat);
                add(*reinterpret_cast<const f32x4 *>(out + d), s[0], s[1]);
            }
        }
        for (int half = groups / 2; half > 0; half /= 2) {
            if (live && g >= half && g < 2 * half) {
                s_out[tid] = o;
                s_ref[tid] = ref;
                s_sum[tid] = sum;
            }
            __syncthreads();
            if (live && g < half)
                add(s_out[tid + half * each], s_ref[tid + half * each], s_sum[tid + half * each]);
            __syncthreads();
        }
        if (live && g == 0) {
            const float scale = sum == 0.0f ? 0.0f : a.value_scale / sum;
            uint16_t *at = static_cast<uint16_t *>(a.out) + row * a.out_stride +
                           (int64_t)(first_head + head) * D + d;
            *reinterpret_cast<u32x2 *>(at) = u32x2{narrow2<TYPE>(o[0] * scale, o[1] * scale),
                                                   narrow2<TYPE>(o[2] * scale, o[3] * scale)};
            if (d == 0 && a.lse)
                a.lse[row * (a.kv_heads * a.group) + first_head + head] =
                    sum == 0.0f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
}

template <int TYPE, bool FP8, int D>
hipError_t launch(const SharedProblem &p, int blocks, int attn_blocks, hipStream_t stream)
{
    const int heads = p.attn.kv_heads * p.attn.head_groups;
    const dim3 grid((unsigned)(blocks * heads));
    switch (p.kind) {
    case SHARED_16:
        hipLaunchKernelGGL((shared_kernel<TYPE, FP8, D, 1>), grid, dim3(kThreads), 0, stream, p,
                           p.attn.table);
        break;
    case SHARED_32:
        if constexpr (attn_heads_a_pass(FP8, D) == 32)
            hipLaunchKernelGGL((shared_kernel<TYPE, FP8, D, 2>), grid, dim3(kThreads), 0, stream,
                               p, p.attn.table);
        else
            return hipErrorInvalidValue;
        break;
    default:
        if constexpr (D % 64 == 0)
            hipLaunchKernelGGL((shared_wide_kernel<TYPE, FP8, D>), grid,
                               dim3(64 * Wide<FP8, D>::kWaves), 0, stream, p, p.attn.table);
        else
            return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    e = launch_attn(p.attn, TYPE, FP8, D, attn_blocks, stream);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((shared_join_kernel<TYPE, D>), dim3((unsigned)(p.attn.rows * heads)),
                       dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_type(const SharedProblem &p, bool fp8, int dim, int blocks, int attn_blocks,
                       hipStream_t stream)
{
    switch (dim) {
    case 64: return fp8 ? launch<TYPE, true, 64>(p, blocks, attn_blocks, stream)
                        : launch<TYPE, false, 64>(p, blocks, attn_blocks, stream);
    case 96: return fp8 ? hipErrorInvalidValue
                        : launch<TYPE, false, 96>(p, blocks, attn_blocks, stream);
    case 128: return fp8 ? launch<TYPE, true, 128>(p, blocks, attn_blocks, stream)
                         : launch<TYPE, false, 128>(p, blocks, attn_blocks, stream);
    case 192: return fp8 ? launch<TYPE, true, 192>(p, blocks, attn_blocks, stream)
                         : launch<TYPE, false, 192>(p, blocks, attn_blocks, stream);
    case 256: return fp8 ? launch<TYPE, true, 256>(p, blocks, attn_blocks, stream)
                         : launch<TYPE, false, 256>(p, blocks, attn_blocks, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_shared(const SharedProblem &p, int type, bool fp8, int dim, int blocks,
                         int attn_blocks, hipStream_t stream)
{
    return type == KV_BF16 ? launch_type<KV_BF16>(p, fp8, dim, blocks, attn_blocks, stream)
                           : launch_type<KV_F16>(p, fp8, dim, blocks, attn_blocks, stream);
}

}  // namespace dps
