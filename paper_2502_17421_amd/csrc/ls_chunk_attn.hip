// Causal attention of a step's new tokens over a paged cache (16-bit inputs, matrix cores).
//
// Request b has n new tokens, the last of its kv rows; token i stands at row p = kv - n + i and sees rows
// max(0, p - window + 1) .. p.  The n * G query rows that share a KV head (G query heads a KV head) are ordered token
// first, row r = token r / G, head r % G, so that what a row sees grows with r.
//
// Two forms of work, in one launch, because a step mixes them.  Keys go in tiles of 32:
//   row blocks    up to 256 query rows (128 at head_dim 64) of a request and KV head; waves of 32 rows share the tiles, which
//                 they copy into rings in LDS.  Bound by the matrix cores: 512 flops per byte of a tile.
//   few rows      requests with at most 32 rows per KV head (single tokens); the four or eight waves of a workgroup hold the
//                 same rows, deal the tiles out, pass them without barriers and are merged at the end.  Bound by HBM.
//
// Which piece a workgroup takes is worked out on the device, from the lengths, by every wave for itself: a program has
// them there, and the host knows upper bounds only.  A block of more tiles than a compute unit's share of all tiles is cut into
// pieces along the keys, whose partial rows (fp32, with the running maximum and sum) a second kernel merges.  Pieces
// go out longest first, since the hardware deals them as compute units become free.  The workgroups of one KV head are 8
// apart at least where there are 8 heads, so an XCD sees one head and its L2 holds the tiles that its workgroups share.
//
// Products (operand layouts: ls_mfma.hpp).  S^T = K Q^T, so a lane holds 16 scores of ONE query row, and the numerators go
// from the accumulators to the operand of O^T = V^T P^T by a pack to 16 bits, which the row sum does not take part in.  Row blocks
// round the numerators once, to nearest: on average as much as the result's own rounding (error 1.3 to 1.4 times that of a result
// rounded once).  What that leaves as a second operand would end this (error 1.00 times), for half again as many matrix instructions and,
// for every two scores, two subtractions and a pack on the vector ALUs, which bind at head_dim 64: there 2048 tokens after 30 thousand
// rows took 427 us in place of 321, a window of 512 49 in place of 40, 19 prompts of 300 to 700 tokens 34 in place of 30.  At
// head_dim 128, where the matrix cores bind, there are no registers for it (248 of 256 are taken; it spills).  The few rows wait for
// memory: they take the second operand, and err no more than the result's rounding.
//
// Softmax state of a row: reference exponent m (raw scores) and l, the sum of exp2((s - m) c), c = scale * log2(e).  Any m
// gives the same result, so the row blocks only raise it when a step's sum leaves the range of the operand type.
//
// Masks.  A tile that every row of a wave sees whole has none; in the others scores are replaced by -inf.  Infinite or NaN
// values of an unseen row would still come through the product as 0 * inf: in the tiles that some row does not see whole
// they are replaced by zeros, and put into the rows that see them at the end.
//
// Measured on MI355X, from cold caches, bf16, 32 query and 8 KV heads of 128 unless said otherwise:
//   2048 tokens after 30 thousand rows          0.86 to 0.91 ms, 1.14 to 1.21 PFLOP/s (a plain matrix product of 16384: 1.35)
//   four first prompts of 611 to 4003 tokens    237 us, 0.95 PFLOP/s
//   24 single tokens, 1 to 30 thousand rows     264 us, 5.8 TB/s
//   18 single tokens and two pieces of prompts, up to 9 thousand rows, 40 query heads   180 us
//   window of 512, 16 and 4 heads of 64, f16    38 us;  four single tokens, up to 1.5 thousand rows    13 us
//   16 and 4 heads of 64: 2048 tokens after 30 thousand rows 328 us, 0.79 PFLOP/s; four first prompts of 611 to 4003 tokens 86 to 90
//   128 single tokens, 500 to 4000 rows         212 us, 5.6 TB/s (of which the list of the pieces 8); 100 to 900 rows, not cut    54
// Long row blocks are held by the power limit (with zeros for inputs the first takes 0.63 ms; 1.5 to 1.95 GHz), head_dim 64 by the vector
// ALUs (16 exponentials a lane and tile at a quarter of their rate), long few rows by HBM, short calls by latency.
#include <type_traits>

#include "ls_mfma.hpp"
#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int TK = 32;            // keys per tile
template <int D> constexpr int kWaves = D == 128 ? 8 : 4;  // per workgroup; at head_dim 64 two workgroups share a compute unit
template <int D> constexpr int kRows = 32 * kWaves<D>;  // query rows per row block
constexpr int FEW = 32;           // rows per KV head up to which the waves split the keys
constexpr int PD = 4;             // requests (a K and a V tile) in flight of a row block
constexpr int RS = 8;             // stages of its K ring, and of its V ring
static_assert(RS >= PD + 4, "V rows are requested PD tiles ahead and read until two steps after");
constexpr float kWhole = 24.f;     // blocks that cost so many tiles or less are not cut, row blocks into pieces of no less
constexpr float kFewSplit = 8.f;   // (few rows)
constexpr float kFewTile = 0.35f;  // what a tile of the few rows counts: 0.32 us next to row blocks that take 0.9 to 1.0 for theirs
constexpr float kLazy = 8.f;      // the reference exponent is raised when a score exceeds it by 2^8
template <bool F16> constexpr float kSumCap = F16 ? 0x1p15f : 0x1p40f;  // largest sum of a step's numerators without raising it

template <int D> constexpr int kTileBytes = TK * D * 2;
// Few rows: two stages per wave, and (m, l) of the rows; at head_dim 64 four workgroups then share a compute unit.
template <int D, int NW> constexpr int kLdsFew = 2 * NW * kTileBytes<D> + NW * FEW * 8;
// Row blocks: the rings, a stage for the query rows that find no free one, page ids, a flag.  At the end of either the times of the shares.
constexpr int kShares = 8;
template <int D, bool BLOCKS, int NW> constexpr int kLds = (BLOCKS ? (2 * RS + 1) * kTileBytes<D> + NW * 512 + 16 : kLdsFew<D, NW>) + kShares * 4;
static_assert(kLdsFew<128, 8> < kLds<128, true, 8> && kLdsFew<64, 4> < kLds<64, true, 4>, "LDS of the few rows");

// Row r of a tile keeps its 16-byte chunk c at place c ^ swizzle(r).  Rows of 256 bytes (head_dim 128) all begin at the same bank,
// rows of 128 at one of two, so that there pairs of rows go together.  (With the swizzles for 256 bytes half of the LDS cycles at
// head_dim 64 were conflicts.)
template <int D> __device__ __forceinline__ int k_swizzle(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? vswz(row) : (row & 2) << 1; }

// ---- which piece --------------------------------------------------------------------------------

// One request, and what its pieces are worked out from.  Work is counted in tiles of a row block.
struct Request {
    int32_t first, n, kv;  // first token, new tokens, rows
    int32_t rows;          // query rows per KV head
    int32_t blocks;        // row blocks (few rows: one)
    float cost, work;      // of the longest block; of all of them, about
    float start, per_step; // block k costs about start + (k + 1) / per_step, and no more than `cost`
};

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }

// First tile and tiles of block k.
template <int ROWS> __device__ __forceinline__ int2 block_tiles(const ChunkArgs &a, const Request &q, int k)
{
    const int top = (k + 1) * ROWS < q.rows ? (k + 1) * ROWS : q.rows;
    const int place0 = q.kv - q.n;
    const int hi = place0 + (int)a.by_group.div((uint32_t)(top - 1)) + 1;
    int lo = a.window > 0 ? place0 + (int)a.by_group.div((uint32_t)(k * ROWS)) - a.window + 1 : 0;
    lo = lo > 0 ? lo : 0;
    return hi > lo ? make_int2(lo / TK, (hi + TK - 1) / TK - lo / TK) : make_int2(0, 0);
}

template <int ROWS> __device__ __forceinline__ Request load_request(const ChunkArgs &a, int b)
{
    Request q{};
    q.per_step = 1.f;
    if (b >= a.batch) return q;
    int first = a.cu_new[b], end = a.cu_new[b + 1], kv = a.kv_lens[b];
    first = first < 0 ? 0 : (first > a.n_tokens ? a.n_tokens : first);
    end = end < first ? first : (end > a.n_tokens ? a.n_tokens : end);
    q.first = first;
    q.n = end - first;
    q.kv = kv < 0 ? 0 : (kv > a.max_kv_len ? a.max_kv_len : kv);
    q.rows = (q.n < a.max_new_len ? q.n : a.max_new_len) * a.group;
    q.blocks = (q.rows + ROWS - 1) / ROWS;
    if (q.blocks == 0) return q;
    const float t0 = (float)block_tiles<ROWS>(a, q, 0).y, t1 = (float)block_tiles<ROWS>(a, q, q.blocks - 1).y;
    if (q.rows <= FEW) {
        q.cost = q.work = kFewTile * t0;
        q.start = q.cost - 1.f;
    } else {
        q.cost = fmaxf(t0, t1);
        q.work = 0.5f * (float)q.blocks * (t0 + t1);
        q.per_step = (float)(TK * a.group) / (float)ROWS;
        q.start = a.window > 0 ? (float)(q.kv - q.n) * (1.f / TK) : t1 - (float)q.blocks / q.per_step;
    }
    return q;
}

// Above which cost a block is cut.
struct Shares {
    float rows, few;
};
// Pieces per block.
__device__ __forceinline__ int cut_of(const Request &q, const Shares &share)
{
    // (no branches here and in what follows: every workgroup goes through this before its first load)
    const float few = __builtin_amdgcn_rcpf(fmaxf(share.few, kFewSplit)), rows = __builtin_amdgcn_rcpf(fmaxf(share.rows, kWhole));
    const int cut = (int)ceilf(q.cost * (q.rows <= FEW ? few : rows));
    return q.cost <= kWhole ? 1 : cut;
}
// Query rows of a block's partial results, if it is cut.
template <int ROWS> __device__ __forceinline__ int block_rows(const Request &q) { return q.rows < ROWS ? q.rows : ROWS; }

// Pieces of a request that cost about x or more: those of its last blocks.  (Any order will do; every wave must find the same.)
__device__ __forceinline__ int pieces_from(const Request &q, int cut, float x)
{
    const float want = x * (float)cut, k = ceilf((want - q.start) * q.per_step) - 1.f;  // first block with that cost
    int below = (int)__builtin_amdgcn_fmed3f(k, 0.f, (float)q.blocks);
    below = want > q.cost ? q.blocks : below;
    below = x > 0.f ? below : 0;
    return (q.blocks - below) * cut;
}

// The largest of values that are not negative (so ordered like their bits), in every lane of a wave.
__device__ __forceinline__ float most_of_lanes(float value)
{
    int x = __builtin_bit_cast(int, value);
    auto take = [&](auto ctrl, auto row_mask) __attribute__((always_inline)) {
        const int y = __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(row_mask)::value, 0xf, false);
        x = x > y ? x : y;
    };
    using all = std::integral_constant<int, 0xf>;
    take(std::integral_constant<int, 0x111>{}, all{});
    take(std::integral_constant<int, 0x112>{}, all{});
    take(std::integral_constant<int, 0x114>{}, all{});
    take(std::integral_constant<int, 0x118>{}, all{});
    take(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    take(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __builtin_bit_cast(float, last_lane(x));
}

// Sums over the lanes of a wave, in every lane.
template <typename T, int N> __device__ __forceinline__ void sum_lanes(T (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = last_lane(scan_lanes(x[i]));
}

struct Piece {
    Request q;
    int32_t b, block, split, cut, slot, entry;  // slot, entry: of this block
    bool valid;
};

// The shares of the work above which blocks are cut.  sums(x, f): x[] as f adds them up for every request; most(f): over all requests; least(time): the candidate with the least time.
// Three blocks for each compute unit and more even out by themselves; only a block beyond a unit's share is cut.  With fewer blocks
// the least of some candidates' expected times is taken, in tiles: one round of pieces lasts as long as the longest; in several
// the units end apart by some part of it, which the few rows' pieces, dealt last and cut small, fill up.  (Against the best of 100
// pairs of shares in a simulation of 300 steps of the ranges that the performance cases draw from: 0.2 % longer, worst 23 %.
// Without the pairs that cut the few rows alone a step of two pieces of prompts and 18 single tokens took 15 % longer there.)
constexpr float kPieceCost = 8.f;  // what a piece costs besides its tiles: its place, the first loads, the rows out
constexpr float kMergeCost = 5.f, kMergeBlock = 18.f;  // the merge: its launch, and a partial block's way to memory and back
constexpr float kUneven = 0.3f;
constexpr float kNever = 1e9f;
__device__ __forceinline__ Shares shares_of(int candidate, float mean)
{
    constexpr float kRows[kShares] = {kNever, 2.f, 1.4f, 1.1f, 0.7f, 0.4f, kNever, 1.2f};
    constexpr float kFew[kShares] = {kNever, 2.f, 1.4f, 1.1f, 0.7f, 0.4f, 0.2f, 0.2f};
    float rows = kRows[0], few = kFew[0];
#pragma unroll
    for (int k = 1; k < kShares; ++k) {
        rows = candidate == k ? kRows[k] : rows;
        few = candidate == k ? kFew[k] : few;
    }
    return {rows == kNever ? rows : rows * mean, few == kNever ? few : few * mean};
}
template <int ROWS, typename Sums, typename Most, typename Least>
__device__ __forceinline__ Shares choose_shares(const ChunkArgs &a, Sums sums, Most most, Least least)
{
    if (a.slots == 0) return {kNever, kNever};
    float of_all[3] = {0.f, 0.f, 0.f};  // blocks, work, work of the few rows
    sums(of_all, [](const Request &q, float (&x)[3]) {
        x[0] += (float)q.blocks;
        x[1] += q.work;
        x[2] += q.rows <= FEW ? q.work : 0.f;
    });
    const float blocks = of_all[0], units = (float)a.units, by_units = __builtin_amdgcn_rcpf(units), mean = of_all[1] * by_units;
    const float few_work = of_all[2];
    auto time_of = [&](const Shares &share) __attribute__((always_inline)) {
        float cuts[2] = {0.f, 0.f};  // pieces, partial rows
        sums(cuts, [&](const Request &q, float (&x)[2]) {
            const float c = (float)cut_of(q, share);
            x[0] += (float)q.blocks * c;
            x[1] += c > 1.f ? (float)q.blocks * c * (float)block_rows<ROWS>(q) : 0.f;
        });
        const float pieces = cuts[0], slots = cuts[1];
        auto longest = [&](bool few) __attribute__((always_inline)) {
            return most([&](const Request &q) { return (q.rows <= FEW) == few ? q.cost * __builtin_amdgcn_rcpf((float)cut_of(q, share)) : 0.f; });
        };
        const float rows = longest(false), few = longest(true), longer = fmaxf(rows, few) + kPieceCost;
        const float merge = slots > 0.f ? kMergeCost + kMergeBlock * slots * (1.f / ROWS) * by_units : 0.f;
        const float several = fmaxf(longer, mean + kPieceCost * pieces * by_units + fmaxf(kUneven * rows - few_work * by_units, kUneven * few));
        const float time = merge + (pieces <= units ? longer : several);
        // (room for the partial rows, and for the pieces that cutting adds)
        return slots > (float)a.slots || pieces - blocks > (float)a.extra ? 2.f * kNever : time;
    };
    if (blocks >= 3.f * units) {
        if (most([](const Request &q) { return q.cost; }) <= 1.25f * mean) return {kNever, kNever};
        const Shares share{1.25f * mean, 1.25f * mean};
        return time_of(share) < kNever ? share : Shares{kNever, kNever};
    }
    return shares_of(least([&](int candidate) { return time_of(shares_of(candidate, mean)); }), mean);
}

// Piece i of those of a KV head, up to 64 requests, a lane each (every wave for itself).
// times: kShares words of LDS.
template <int ROWS, int NW, bool BLOCKS> __device__ __forceinline__ Piece find_piece(const ChunkArgs &a, int i, int lane, float *times)
{
    Piece p{};
    if (!BLOCKS && a.slots == 0) {  // single tokens, nothing to cut: a piece is a request
        p.q = load_request<ROWS>(a, i);
        p.b = i;
        p.cut = 1;
        p.valid = p.q.blocks > 0;
        return p;
    }
    const Request q = load_request<ROWS>(a, lane);
    const Shares share = choose_shares<ROWS>(
        a,
        [&](auto &x, auto f) {
            f(q, x);
            sum_lanes(x);
        },
        [&](auto f) { return most_of_lanes(f(q)); },
        [&](auto time) {  // the waves share the candidates
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            for (int k = wave; k < kShares; k += NW) {
                const float t = time(k);
                if (lane == 0) times[k] = t;
            }
            __syncthreads();
            int best = 0;
            float least = times[0];
#pragma unroll
            for (int k = 1; k < kShares; ++k) {
                const float t = times[k];
                best = t < least ? k : best;
                least = fminf(t, least);
            }
            return __builtin_amdgcn_readfirstlane(best);
        });
    const int cut = cut_of(q, share), pieces = q.blocks * cut;
    const int slots = cut > 1 ? pieces * block_rows<ROWS>(q) : 0, entries = cut > 1 ? q.blocks : 0;
    const int piece_end = scan_lanes(pieces);
    int slot_end = 0, entry_end = 0;
    if (share.rows != kNever || share.few != kNever) {
        slot_end = scan_lanes(slots);
        entry_end = scan_lanes(entries);
    }
    if (blockIdx.x == 0 && threadIdx.x == 63 && a.slots > 0) *a.n_entries = entry_end;  // for the merge
    const int total = last_lane(piece_end);
    if (i >= total) return p;
    int b, at;  // the request; the piece's place among the request's, last block first
    if (total <= a.units) {  // all at once: any order
        b = __builtin_ctzll(__ballot(piece_end > i));
        at = i - __builtin_amdgcn_readlane(piece_end - pieces, b);
    } else {
        // longest first, by sixteenths of the longest: the largest x such that more than i pieces cost x sixteenths or more
        const float unit = most_of_lanes(q.cost * __builtin_amdgcn_rcpf((float)cut)) * (1.f / 16.f) + 0x1p-10f;
        int lo = 0, hi = 17;  // (none costs 17 or more)
        while (hi - lo > 1) {  // by quarters: three sums at a time
            const int step = (hi - lo + 3) >> 2;
            const int x1 = lo + step, x2 = x1 + step < hi ? x1 + step : hi, x3 = x2 + step < hi ? x2 + step : hi;
            int c[3] = {pieces_from(q, cut, (float)x1 * unit), pieces_from(q, cut, (float)x2 * unit), pieces_from(q, cut, (float)x3 * unit)};
            sum_lanes(c);
            lo = c[2] > i ? x3 : c[1] > i ? x2 : c[0] > i ? x1 : lo;
            hi = c[2] > i ? hi : c[1] > i ? x3 : c[0] > i ? x2 : x1;
        }
        const int above = pieces_from(q, cut, (float)hi * unit), same = pieces_from(q, cut, (float)lo * unit) - above, upto = scan_lanes(same);
        int all_above[1] = {above};
        sum_lanes(all_above);
        const int rest = i - all_above[0];
        b = __builtin_ctzll(__ballot(upto > rest) | 1ull << 63);
        at = __builtin_amdgcn_readlane(above + rest - (upto - same), b);
    }
    auto of = [&](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, b); };
    p.b = b;
    p.q = Request{of(q.first), of(q.n), of(q.kv), of(q.rows), of(q.blocks), 0.f, 0.f, 0.f, 0.f};
    p.cut = of(cut);
    const int from_end = p.cut == 1 ? at : at / p.cut;
    p.block = p.q.blocks - 1 - from_end;
    p.split = at - from_end * p.cut;
    p.slot = of(slot_end - slots) + from_end * p.cut * block_rows<ROWS>(p.q);
    p.entry = of(entry_end - entries) + from_end;
    p.valid = p.block >= 0;
    return p;
}

// More requests: a kernel of one workgroup sorts them by their longest piece and writes down where the pieces of each begin.
struct Listed {
    int32_t begin;  // pieces of the requests before it in this order; the last entry: all of them
    int32_t b, cut, slot, entry;
};
constexpr int LIST_THREADS = 1024, LIST_PER = LS_MAX_STEP_BATCH / LIST_THREADS;

template <int ROWS>
__global__ void __launch_bounds__(LIST_THREADS)
chunk_list_kernel(ChunkArgs a)
{
    __shared__ float part_f[LIST_THREADS / kWave];
    __shared__ int32_t part_i[LIST_THREADS / kWave], bucket[64], bucket_at[64];
    __shared__ int32_t order[LS_MAX_STEP_BATCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Request q[LIST_PER];
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) q[j] = load_request<ROWS>(a, tid + j * LIST_THREADS);
    auto sum_threads = [&](auto x) {
        auto *part = [&] { if constexpr (std::is_same_v<decltype(x), float>) return part_f; else return part_i; }();
        x = scan_lanes(x);
        if (lane == 63) part[wave] = x;
        __syncthreads();
        decltype(x) all = 0;
#pragma unroll
        for (int w = 0; w < LIST_THREADS / kWave; ++w) all += part[w];
        __syncthreads();
        return all;
    };
    auto most_threads = [&](float x) {
        x = most_of_lanes(x);
        if (lane == 63) part_f[wave] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < LIST_THREADS / kWave; ++w) x = fmaxf(x, part_f[w]);
        __syncthreads();
        return x;
    };
    const Shares share = choose_shares<ROWS>(
        a,
        [&](auto &x, auto f) {
#pragma unroll
            for (int j = 0; j < LIST_PER; ++j) f(q[j], x);
#pragma unroll
            for (float &part : x) part = sum_threads(part);
        },
        [&](auto f) {
            float x = f(q[0]);
#pragma unroll
            for (int j = 1; j < LIST_PER; ++j) x = fmaxf(x, f(q[j]));
            return most_threads(x);
        },
        [&](auto time) {
            int best = 0;
            float least = time(0);
#pragma unroll 1
            for (int k = 1; k < kShares; ++k) {
                const float t = time(k);
                best = t < least ? k : best;
                least = fminf(t, least);
            }
            return best;
        });
    // sort by the longest piece, by its bits: bucket 63 - 2 * log2 - next bit
    if (tid < 64) bucket[tid] = 0;
    __syncthreads();
    int in[LIST_PER], place[LIST_PER];
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) {
        const uint32_t key = (uint32_t)(q[j].cost / (float)cut_of(q[j], share)) + 1;
        const int top = 31 - __builtin_clz(key);
        in[j] = 63 - (2 * top + (top > 0 ? (key >> (top - 1)) & 1 : 0));
        if (tid + j * LIST_THREADS < a.batch) place[j] = atomicAdd(&bucket[in[j]], 1);
    }
    __syncthreads();
    if (tid < 64) bucket_at[tid] = scan_lanes(bucket[tid]) - bucket[tid];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j)
        if (tid + j * LIST_THREADS < a.batch) order[bucket_at[in[j]] + place[j]] = tid + j * LIST_THREADS;
    __syncthreads();
    // LIST_PER requests in a row per thread, in that order: sums of pieces, partial blocks and cut blocks before each
    Request r[LIST_PER];
    int cut[LIST_PER], pieces = 0, slots = 0, entries = 0;
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) {
        const int at = tid * LIST_PER + j;
        r[j] = load_request<ROWS>(a, at < a.batch ? order[at] : a.batch);
        cut[j] = cut_of(r[j], share);
        pieces += r[j].blocks * cut[j];
        slots += cut[j] > 1 ? r[j].blocks * cut[j] * block_rows<ROWS>(r[j]) : 0;
        entries += cut[j] > 1 ? r[j].blocks : 0;
    }
    auto before = [&](int x) {  // sum over the threads before this one
        const int upto = scan_lanes(x);
        if (lane == 63) part_i[wave] = upto;
        __syncthreads();
        int sum = upto - x;
#pragma unroll
        for (int w = 0; w < LIST_THREADS / kWave; ++w) sum += w < wave ? part_i[w] : 0;
        __syncthreads();
        return sum;
    };
    int piece = before(pieces), slot = before(slots), entry = before(entries);
    Listed *list = (Listed *)a.list;
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) {
        const int at = tid * LIST_PER + j;
        if (at >= a.batch) continue;
        list[at] = Listed{piece, order[at], cut[j], slot, entry};
        piece += r[j].blocks * cut[j];
        slot += cut[j] > 1 ? r[j].blocks * cut[j] * block_rows<ROWS>(r[j]) : 0;
        entry += cut[j] > 1 ? r[j].blocks : 0;
        if (at == a.batch - 1) {
            list[a.batch] = Listed{piece, 0, 1, 0, 0};
            *a.n_entries = entry;
        }
    }
}

// Piece i by the list: the last request that begins at or before it, 64 candidates at a time.
template <int ROWS> __device__ __forceinline__ Piece find_listed(const ChunkArgs &a, int i, int lane)
{
    const Listed *list = (const Listed *)a.list;
    Piece p{};
    int lo = 0, n = a.batch + 1;  // the one looked for is among lo .. lo + n - 1
    while (n > 1) {
        const int step = div_up(n, kWave);
        const int at = lo + lane * step;
        const bool below = lane * step < n && list[at].begin <= i;
        const int last = 63 - __builtin_clzll(__ballot(below) | 1);
        lo += last * step;
        n = n - last * step < step ? n - last * step : step;
    }
    if (lo >= a.batch) return p;
    const Listed e = list[lo];
    p.b = __builtin_amdgcn_readfirstlane(e.b);
    p.q = load_request<ROWS>(a, p.b);
    p.cut = __builtin_amdgcn_readfirstlane(e.cut);
    const int at = i - __builtin_amdgcn_readfirstlane(e.begin);
    const int from_end = at / p.cut;
    p.block = p.q.blocks - 1 - from_end;
    p.split = at - from_end * p.cut;
    p.slot = __builtin_amdgcn_readfirstlane(e.slot) + from_end * p.cut * block_rows<ROWS>(p.q);
    p.entry = __builtin_amdgcn_readfirstlane(e.entry) + from_end;
    p.valid = p.block >= 0;
    return p;
}

// ---- what both forms share ----------------------------------------------------------------------

// Result of 32 query rows in the accumulator layout: lane l has row l % 32.
template <int D> struct RowState {
    floatx16 o[D / 32];
    float m, l;  // l: the numerators of this lane's half of the keys until they are joined
};

// What a lane's query row is, and sees.
struct QueryRow {
    bool ok;
    int32_t token, head;    // token of the packed rows
    int32_t lo, place;      // rows seen: lo .. place
};

__device__ __forceinline__ QueryRow query_row(const ChunkArgs &a, const Request &q, int g, int r)
{
    QueryRow x;
    x.ok = r < q.rows;
    r = x.ok ? r : q.rows - 1;  // rows past the end repeat the last
    const int i = (int)a.by_group.div((uint32_t)r);
    x.token = q.first + i;
    x.head = g * a.group + r - i * a.group;
    x.place = q.kv - q.n + i;
    x.lo = a.window > 0 && x.place - a.window + 1 > 0 ? x.place - a.window + 1 : 0;
    return x;
}

// Byte offsets of query rows r, r + step, r + 2 step ... in q or out, by additions.  Past the last row it stays where it is.
struct RowWalk {
    int64_t at, jump, wrap;  // jump: step rows further; wrap: from a group's end to the next token's first
    int32_t head, heads, r, step, rows, group;
    __device__ __forceinline__ RowWalk(const ChunkArgs &a, const Request &q, int g, int first, int row_step, const int64_t (&stride)[2])
    {
        const QueryRow x = query_row(a, q, g, first);
        at = x.token * stride[0] + x.head * stride[1];
        group = a.group;
        head = x.head - g * group;
        const int tokens = (int)a.by_group.div((uint32_t)row_step);
        heads = row_step - tokens * group;
        jump = tokens * stride[0] + heads * stride[1];
        wrap = stride[0] - group * stride[1];
        r = first;
        step = row_step;
        rows = q.rows;
    }
    __device__ __forceinline__ void next()
    {
        r += step;
        head += heads;
        const bool over = head >= group;
        head -= over ? group : 0;
        const int64_t by = jump + (over ? wrap : 0);
        at += r < rows ? by : 0;
    }
};

// Partial rows of a piece, its first one number `row` of KV head g: [row][D] fp32 sums, and (m, l) of every row.
template <int D> __device__ __forceinline__ float *part_rows(const ChunkArgs &a, int row, int g) { return a.parts + ((int64_t)g * a.slots + row) * D; }
__device__ __forceinline__ float2 *part_state(const ChunkArgs &a, int row, int g) { return a.part_ml + (int64_t)g * a.slots + row; }

// Blocks that are cut, for the merge.
struct Entry {
    int32_t first, row0, rows;  // first token of the request, first row of the block, its rows
    int32_t cut, slot, part;    // pieces, first partial row, partial rows of a piece
};
template <int ROWS> __device__ __forceinline__ void write_entry(const ChunkArgs &a, const Piece &p, int g)
{
    const int row0 = p.block * ROWS;
    ((Entry *)a.entries)[p.entry * a.n_kv_heads + g] = Entry{p.q.first, row0, p.q.rows - row0 < ROWS ? p.q.rows - row0 : ROWS, p.cut, p.slot, block_rows<ROWS>(p.q)};
}

// ---- row blocks -------------------------------------------------------------------------------------

// A copy of 64 lanes whose LDS and global addresses are AT bytes further than lds_base and the lane's own.
template <int AT> __device__ __forceinline__ void copy_tile_rows(const uint8_t *base, uint32_t voff, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" : : "s"(lds_base), "v"(voff), "s"(base), "n"(AT) : "memory");
}

// What bounds it, power apart: two waves share a SIMD, and each issues an instruction in five cycles or more, so 16 matrix
// instructions of 32 cycles leave a wave some 200 slots.  A tile's arithmetic and LDS reads take 110 of them; hence rings of 8
// stages, which a turn of the loop goes once around, so that stages are constants in the instructions (document 905 -> 894 us),
// half of the waves for K and half for V, every other tile a wave, addresses of 64 tiles worked out at a time, a tile per lane, and
// one comparison per mask.  (With 85 scalar instructions per tile and wave instead of 20 the matrix cores were busy half of the time.)
template <int D, bool F16>
__device__ __forceinline__ void row_block(const ChunkArgs &a, const Piece &piece, int g, uint8_t *smem)
{
    constexpr int NW = kWaves<D>, ROWS = kRows<D>;
    constexpr int KSTEPS = D / 16, MT = D / 32, CH = D / 8, ROWB = D * 2, TILEB = kTileBytes<D>;
    constexpr int RPL = 64 / CH;          // rows one copy of 64 lanes covers
    constexpr int TPT = TK / RPL;         // copies per tile and tensor
    // A wave copies 16 rows in a row of a tile, which share a page: of every tile (head_dim 64), or of every other one.
    constexpr int MINE = 16, LOADS = MINE / RPL, STEP = NW / 2 * MINE / TK;
    constexpr uint32_t RING = RS * TILEB; // bytes of a ring: K, then V
    static_assert(STEP <= 2 && PD == 4 && (PD + 1) * LOADS + TPT + 1 <= 63, "copies of a wave");
    const Request &q = piece.q;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int row0 = piece.block * ROWS, wave_row0 = row0 + wave * 32;
    const bool has_rows = wave_row0 < q.rows;

    // tiles of this piece
    const int2 span = block_tiles<ROWS>(a, q, piece.block);
    int per = div_up(span.y, piece.cut);
    per += piece.cut > 1 ? per & 1 : 0;  // tiles go in pairs
    int t_lo = piece.split * per, t_hi = t_lo + per;
    t_hi = span.x + (t_hi < span.y ? t_hi : span.y);
    t_lo = span.x + (t_lo < span.y ? t_lo : span.y);
    const int n_tiles = t_hi - t_lo;
    const int kv = q.kv;

    RowState<D> st;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) st.o[mt][e] = 0.f;
    st.m = -INFINITY;
    st.l = 0.f;

    if (n_tiles > 0) {
        // ---- copies -----------------------------------------------------------------------------
        // The first half of the waves copies K rows, the other half V rows.
        const uint32_t base = lds_offset(smem);
        const bool is_v = wave >= NW / 2;
        const int64_t *stride = is_v ? a.vc_s : a.kc_s;
        const uint8_t *pool = uniform_ptr((is_v ? a.v_pages : a.k_pages) + g * stride[1]);
        const int32_t rb = (int32_t)stride[2];
        const int page_mask = (1 << a.page_shift) - 1;
        const int ld_row = lane / CH, ld_pos = lane % CH;
        const int my_row = wave % (TK / MINE) * MINE;
        // Every other one: of K waves 0 and 1 tiles 0, 2, 4 ..., of V waves 4 and 5 tiles 1, 3, 5 ...
        const int first_tile = STEP == 1 ? 0 : (wave / (TK / MINE) & 1) ^ (int)is_v;
        auto chunk_at = [&](int row) __attribute__((always_inline)) { return (uint32_t)(ld_pos ^ (is_v ? v_swizzle<D>(row) : k_swizzle<D>(row))) * 16; };
        // Lane's offset for copy j from the first of those rows, less what the instruction adds (rows are at least ROWB apart).
        uint32_t voff[LOADS];
#pragma unroll
        for (int j = 0; j < LOADS; ++j) voff[j] = (uint32_t)((j * RPL + ld_row) * rb) + chunk_at(my_row + j * RPL + ld_row) - j * RPL * ROWB;
        // Where this wave's rows of 64 tiles are, a tile per lane, as byte offsets into the pool; rows past the end repeat the last
        // one, tiles past the last repeat it.  The page ids of the 64 tiles after those are on their way to LDS.
        const int32_t *tab = a.block_table + (int64_t)piece.b * a.bt_stride;
        uint32_t *const ids = (uint32_t *)(smem + (2 * RS + 1) * TILEB) + wave * 128;
        uint32_t *const found = (uint32_t *)(smem + (2 * RS + 1) * TILEB) + NW * 128;  // whether values were replaced by zeros
        auto tile_row = [&](int tile) __attribute__((always_inline)) {
            const int row = (t_lo + (tile < n_tiles ? tile : n_tiles - 1)) * TK + my_row;
            return row < kv ? row : kv - 1;
        };
        uint64_t offs = 0;
        auto place = [&](int first, uint32_t page) __attribute__((always_inline)) {
            offs = (uint64_t)page * (uint64_t)stride[0] + (uint64_t)((int64_t)(tile_row(first + lane) & page_mask) * rb);
        };
        auto fetch_ids = [&](int first) __attribute__((always_inline)) {
            const int32_t *src = tab + (tile_row(first + lane) >> a.page_shift);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                         : : "s"(__builtin_amdgcn_readfirstlane(lds_offset(ids + (first & 64)))), "v"(src) : "memory");
        };
        place(0, (uint32_t)tab[tile_row(lane) >> a.page_shift]);
        if (tid == 0) *found = 0;
        if (n_tiles + PD + 2 > 64) fetch_ids(64);

        // One tile after the other: request r (r >= -(PD + 1)) is the K rows of tile r + PD + 1 and the V rows of tile r + PD; every
        // other one: request r (r >= -3) is those of K tiles 2 r + 6 and 2 r + 7, of V tiles 2 r + 5 and 2 r + 6.
        int rq = first_tile;  // tile of this wave's next request
        uint32_t rq_off = (uint32_t)first_tile * TILEB;  // its place in the ring
        const uint32_t rq_base = base + (is_v ? RING : 0) + my_row * ROWB;
        const int tail = kv < t_hi * TK ? n_tiles - 1 : 1 << 30;  // first tile that is not whole
        auto request = [&]() __attribute__((always_inline)) {
            const int i = rq & 63;
            if (i < STEP && rq >= 64) {
                place(rq - i, ids[(rq & 64) + lane]);
                fetch_ids(rq - i + 64);
            }
            const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)offs, i) |
                                 (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(offs >> 32), i) << 32;
            const uint8_t *src = pool + off;
            const uint32_t to = rq_base + rq_off;
            if (rq < tail) {
                copy_tile_rows<0>(src, voff[0], to);
                copy_tile_rows<RPL * ROWB>(src, voff[1], to);
                if constexpr (LOADS == 4) {
                    copy_tile_rows<2 * RPL * ROWB>(src, voff[2], to);
                    copy_tile_rows<3 * RPL * ROWB>(src, voff[3], to);
                }
            } else {
                const int last = kv - 1 - (t_hi - 1) * TK, first = my_row < last ? my_row : last;  // src is that row
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    const int r = my_row + j * RPL + ld_row;
                    copy_to_lds(src, (uint32_t)(((r < last ? r : last) - first) * rb) + chunk_at(r), to + j * RPL * ROWB);
                }
            }
            rq += STEP;
            rq_off = (rq_off + STEP * TILEB) & (RING - 1);
        };
        if (!is_v) request();
        // Query rows: through LDS, in stages that the first requests leave free, in the layout of a K tile.
        const uint32_t q_at = (uint32_t)(wave < RS - PD - 1 ? PD + 1 + wave : wave < RS - PD - 1 + RS - PD ? RS + PD + wave - (RS - PD - 1) : 2 * RS) * TILEB;
        if (has_rows) {
            RowWalk y(a, q, g, wave_row0 + ld_row, RPL, a.q_s);
#pragma unroll
            for (int j = 0; j < TPT; ++j) {
                copy_row_to_lds(a.q + y.at + (ld_pos ^ k_swizzle<D>(j * RPL + ld_row)) * 16,
                                __builtin_amdgcn_readfirstlane(base + q_at + j * RPL * ROWB));
                y.next();
            }
        }
        if constexpr (STEP == 1) {
#pragma unroll
            for (int r = 0; r < PD; ++r) request();
            wait_vmem<PD * LOADS>();
        } else {
            if (is_v && first_tile == 0) request();
            request();
            wait_vmem<LOADS>();  // also K tile 1 and V tile 0
        }
        __syncthreads();  // K tile 0 and the query rows are in LDS

        auto ring_barrier = [&]() __attribute__((always_inline)) { asm volatile("s_barrier" ::: "memory"); };
        // Tiles (of this piece) that all rows between two see whole: the first of them, and how many; and the first one past whose
        // end some row does not see.
        auto seen_whole = [&](int first_row, int last_row) __attribute__((always_inline)) {
            const QueryRow top = query_row(a, q, g, first_row), end = query_row(a, q, g, last_row);
            const int from = div_up(end.lo, TK) - t_lo, to = (top.place + 1 > 0 ? top.place + 1 : 0) / TK - t_lo;
            return int3{__builtin_amdgcn_readfirstlane(from), __builtin_amdgcn_readfirstlane(to > from ? to - from : 0), __builtin_amdgcn_readfirstlane(to)};
        };
        auto inside = [&](int t, int3 range) __attribute__((always_inline)) { return (uint32_t)(t - range.x) < (uint32_t)range.y; };
        const int3 block_whole = seen_whole(row0, row0 + ROWS - 1);
        // V tiles h and h + 1 are there: values that are not finite leave tiles that some row of the block does not see whole.
        // (A tile's first fragments are read a half-step later, at the earliest.)
        auto clean = [&](int from, int to) __attribute__((always_inline)) {
            to = to < n_tiles ? to : n_tiles;
            if (from >= to || (inside(from, block_whole) && inside(to - 1, block_whole))) return;
            for (int t = from; t < to; ++t) {
                if (inside(t, block_whole)) continue;  // (the same in all waves)
                for (int i = tid; i < TILEB / 16; i += NW * 64) {
                    uint4 *at = (uint4 *)(smem + RING + ((t * TILEB) & (RING - 1)) + i * 16);
                    bf16x8 v[1] = {__builtin_bit_cast(bf16x8, *at)};
                    if (drop_not_finite<F16>(v)) {
                        *at = __builtin_bit_cast(uint4, v[0]);
                        *found = 1;
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        // Before half-step 1, which reads K rows of tile 1: request -PD has landed; request 0 (-1) follows, over query rows.
        auto advance0 = [&]() __attribute__((always_inline)) {
            if constexpr (STEP == 1) wait_vmem<(PD - 1) * LOADS>();
            ring_barrier();
            request();
            clean(0, 1);
        };
        // Before half-steps h and h + 1 (h odd), which read K rows up to tile h + 2, V rows up to tile h: requests up to h + 1 - PD
        // ((h - 5) / 2) have landed.  Requests h and h + 1 ((h - 1) / 2) follow in these half-steps, into stages last read in
        // half-step h - 1 or earlier: K tiles up to h + 6, V tiles up to h + 5.
        auto advance_pair = [&](int h) __attribute__((always_inline)) {
            wait_vmem<(STEP == 1 ? PD - 2 : 1) * LOADS>();
            ring_barrier();
            if (!(inside(h, block_whole) && inside(h + 1, block_whole))) clean(h, h + 2);
        };
        // After the pairs: the V rows of the last tile have landed, request n_tiles - 1 - PD of n_tiles - 2 at least ((h - 5) / 2 of
        // (h - 3) / 2).
        auto advance_last = [&](int h) __attribute__((always_inline)) {
            wait_vmem<(STEP == 1 ? PD - 1 : 1) * LOADS>();
            ring_barrier();
            clean(h, n_tiles);
        };

        if (!has_rows) {  // only feeds the rings
            advance0();
            int h = 1;
            for (; h + 1 < n_tiles; h += 2) {
                advance_pair(h);
                request();
                if constexpr (STEP == 1) request();
            }
            advance_last(h);
        } else {
            typedef __attribute__((address_space(3))) const uint4 *lds_u4;
            typedef __attribute__((address_space(3))) shortx4 *lds_s4;
            const float c = a.scale_log2;
            const QueryRow x = query_row(a, q, g, wave_row0 + li);
            const uint32_t k_off0 = base + li * ROWB + ((lh ^ k_swizzle<D>(li)) * 16);
            const int tr_s = lane & 15, tr_row = 4 * lh + (tr_s >> 2);
            const int tr_dchunk = 2 * ((lane >> 4) & 1) + ((tr_s & 3) >> 1);
            const uint32_t v_off0 = base + RING + tr_row * ROWB + ((tr_dchunk ^ v_swizzle<D>(tr_row)) * 16) + (tr_s & 1) * 8;
            // A fragment's place in stage 0, kept: the stages of the main loop are constants and go into the instructions' offsets.
            uint32_t k_at[KSTEPS], v_at[MT];
#pragma unroll
            for (int f = 0; f < KSTEPS; ++f) k_at[f] = k_off0 ^ (uint32_t)(f << 5);
#pragma unroll
            for (int f = 0; f < MT; ++f) v_at[f] = v_off0 ^ (uint32_t)(f << 6);
#pragma unroll
            for (int f = 0; f < KSTEPS; ++f) asm volatile("" : "+v"(k_at[f]));  // (they would be worked out again in the loop)
#pragma unroll
            for (int f = 0; f < MT; ++f) asm volatile("" : "+v"(v_at[f]));
            auto read_k = [&](uint32_t stage, int f) __attribute__((always_inline)) {
                return __builtin_bit_cast(bf16x8, *(lds_u4)(uintptr_t)(k_at[f] + stage));
            };
            auto read_v = [&](uint32_t stage, int f) __attribute__((always_inline)) {  // f = 16-key half * MT + d tile
                const uint32_t at = v_at[f % MT] + (stage + (f / MT) * 16 * ROWB);
                const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)at));
                const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)(at + 8 * ROWB)));
                return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
            };
            const int3 wave_whole = seen_whole(wave_row0, wave_row0 + 31);
            auto mask = [&](floatx16 &s, int t) __attribute__((always_inline)) {
                if (inside(t, wave_whole)) return;
                const int key0 = (t_lo + t) * TK + 4 * lh;  // (one comparison a score at either edge)
                if (t >= wave_whole.z)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) <= x.place - key0 ? s[e] : -INFINITY;
                if (t < wave_whole.x)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) >= x.lo - key0 ? s[e] : -INFINITY;
            };
            auto numerators = [&](const floatx16 &s, uint32_t (&pp)[8]) __attribute__((always_inline)) {  // with the current m
                const float mc = st.m == -INFINITY ? 0.f : st.m * c;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -mc)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], c, -mc));
                    pp[e >> 1] = pack16<F16>(p0, p1);
                    sum += p0 + p1;
                }
                return sum;
            };
            auto raise = [&](const floatx16 &s) __attribute__((always_inline)) {
                float mx = s[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
                mx = half_max(mx);
                if (__any((mx - st.m) * c > kLazy)) {  // also true while m is -inf
                    const float m_new = fmaxf(st.m, mx);
                    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((st.m - m_new) * c);
                    st.m = m_new;
                    st.l *= alpha;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 16; ++e) st.o[mt][e] *= alpha;
                }
            };

            bf16x8 q_reg[KSTEPS];
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk) q_reg[kk] = read_k(q_at, kk);

            // ---- pipeline -----------------------------------------------------------------------
            // A step is one tile: KSTEPS matrix instructions for the scores, the softmax arithmetic of 16 scores a lane, and KSTEPS for
            // the output.  Half-step h issues the score product of step h and the output product of step h - 2, and between them
            // the softmax of step h - 1, in two register slots that alternate, and this wave's copies of a request.  K and V
            // fragments rotate through FS registers each, refilled right after the instructions that read them.  The scheduling
            // barriers pin this order.
            constexpr int FS = KSTEPS / 2, PPG = 8 / KSTEPS;
            bf16x8 k_frag[FS], v_frag[FS];
            floatx16 s_sl[2];
            uint32_t p_sl[2][8];
            float neg_mc = 0.f;
            using yes = std::true_type;
            using no = std::false_type;
            auto half_step = [&](auto x_tag, auto qk_tag, auto sm_tag, auto kn_tag, auto vn_tag, auto rq_tag, auto k_cur, auto k_next, auto v_cur,
                                 auto v_next) __attribute__((always_inline)) {
                constexpr int X = decltype(x_tag)::value, Y = 1 - X;
                constexpr bool QK = decltype(qk_tag)::value, SM = decltype(sm_tag)::value;
                constexpr bool KN = decltype(kn_tag)::value, VN = decltype(vn_tag)::value, RQ = decltype(rq_tag)::value;
                bf16x8 pb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    pb[i] = __builtin_bit_cast(bf16x8, make_uint4(p_sl[X][4 * i], p_sl[X][4 * i + 1], p_sl[X][4 * i + 2], p_sl[X][4 * i + 3]));
                const uint32_t kc = k_cur, kn = k_next, vc = v_cur, vn = v_next;
                float sum = 0.f;
                floatx16 s_new;
#pragma unroll
                for (int e = 0; e < 16; ++e) s_new[e] = 0.f;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    float pe[PPG][2];
                    st.o[i % MT] = mfma32<F16>(v_frag[i % FS], pb[i / MT], st.o[i % MT]);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (SM) {
#pragma unroll
                        for (int u = 0; u < PPG; ++u) {
                            const int e = 2 * (i * PPG + u);
                            pe[u][0] = __builtin_amdgcn_exp2f(__builtin_fmaf(s_sl[Y][e], c, neg_mc));
                            pe[u][1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s_sl[Y][e + 1], c, neg_mc));
                        }
                    }
                    if (i < FS) v_frag[i % FS] = read_v(vc, i + FS);
                    else if constexpr (VN) v_frag[i % FS] = read_v(vn, i - FS);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (QK) s_new = mfma32<F16>(k_frag[i % FS], q_reg[i], s_new);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (SM) {
#pragma unroll
                        for (int u = 0; u < PPG; ++u) {
                            p_sl[Y][i * PPG + u] = pack16<F16>(pe[u][0], pe[u][1]);
                            sum += pe[u][0] + pe[u][1];
                            asm volatile("" : "+v"(p_sl[Y][i * PPG + u]), "+v"(sum));  // (they would be sunk below the loop)
                        }
                    }
                    if (i < FS) {
                        if constexpr (QK) k_frag[i % FS] = read_k(kc, i + FS);
                    } else if constexpr (KN) {
                        k_frag[i % FS] = read_k(kn, i - FS);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (RQ)
                        if (i == 0) request();
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (QK) s_sl[X] = s_new;
                if constexpr (SM) {
                    if (__any(!(sum < kSumCap<F16>))) {  // also infinities and NaN, and rows that have seen nothing yet
                        raise(s_sl[Y]);
                        sum = numerators(s_sl[Y], p_sl[Y]);
                        neg_mc = -(st.m * c);
                    }
                    st.l += sum;
                }
            };
            using X0 = std::integral_constant<int, 0>;
            using X1 = std::integral_constant<int, 1>;

#pragma unroll
            for (int f = 0; f < FS; ++f) v_frag[f] = k_frag[f] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) p_sl[0][e] = p_sl[1][e] = 0;  // an output product of zeros adds nothing
            // scores of step 0; their largest is the reference exponent
#pragma unroll
            for (int e = 0; e < 16; ++e) s_sl[0][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk) s_sl[0] = mfma32<F16>(read_k(0, kk), q_reg[kk], s_sl[0]);
            mask(s_sl[0], 0);
            {
                float mx = s_sl[0][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s_sl[0][e]);
                st.m = half_max(mx);
                neg_mc = -(st.m * c);
            }
            advance0();
#pragma unroll
            for (int f = 0; f < FS; ++f) k_frag[f] = read_k(TILEB, f);
            // Step -1 does not exist: its numerators are zeros, the V stage they are multiplied with is any, and what comes of it is
            // thrown away.
            int h = 1;
            auto first_output = [&]() __attribute__((always_inline)) {
                if (h != 1) return;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) st.o[mt][e] = 0.f;
            };
            auto stage = [&](int tile) __attribute__((always_inline)) { return (uint32_t)(tile * TILEB) & (RING - 1); };
            // Half-steps h and h + 1: K tiles h to h + 2, V tiles h - 2 to h.
            auto pair = [&](auto k0, auto k1, auto k2, auto v0, auto v1) __attribute__((always_inline)) {
                advance_pair(h);
                half_step(X1{}, yes{}, yes{}, yes{}, yes{}, yes{}, k0, k1, v0, v1);
                first_output();
                mask(s_sl[1], h);
                half_step(X0{}, yes{}, yes{}, yes{}, yes{}, std::bool_constant<STEP == 1>{}, k1, k2, v1, k0);
                mask(s_sl[0], h + 1);
                h += 2;
            };
            auto pair_at = [&](auto first) __attribute__((always_inline)) {  // h = first + a multiple of RS
                constexpr uint32_t T = decltype(first)::value;
                pair(std::integral_constant<uint32_t, T % RS * TILEB>{}, std::integral_constant<uint32_t, (T + 1) % RS * TILEB>{},
                     std::integral_constant<uint32_t, (T + 2) % RS * TILEB>{}, std::integral_constant<uint32_t, (T + RS - 2) % RS * TILEB>{},
                     std::integral_constant<uint32_t, (T + RS - 1) % RS * TILEB>{});
            };
            while (h + RS - 1 < n_tiles) {
                pair_at(std::integral_constant<uint32_t, 1>{});
                pair_at(std::integral_constant<uint32_t, 3>{});
                pair_at(std::integral_constant<uint32_t, 5>{});
                pair_at(std::integral_constant<uint32_t, 7>{});
            }
            while (h + 1 < n_tiles) pair(stage(h), stage(h + 1), stage(h + 2), stage(h - 2), stage(h - 1));
            advance_last(h);
            // h = n_tiles - 1 (one step left to score) or h = n_tiles (none: the step scored here is void)
            const bool is_void = h >= n_tiles;
            const uint32_t v1 = stage(h - 1), v2 = stage(h);
            half_step(X1{}, yes{}, yes{}, no{}, yes{}, no{}, stage(h), 0u, stage(h - 2), v1);
            first_output();
            if (is_void) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s_sl[1][e] = -INFINITY;
            } else {
                mask(s_sl[1], h);
            }
            half_step(X0{}, no{}, yes{}, no{}, yes{}, no{}, 0u, 0u, v1, v2);  // output h - 1, softmax h
            if (!is_void) half_step(X1{}, no{}, no{}, no{}, no{}, no{}, 0u, 0u, v2, 0u);  // output h
        }
        wait_vmem<0>();   // requests past the last tile
        __syncthreads();  // every wave is done reading tiles: the rings are free
        if (has_rows && __builtin_amdgcn_readfirstlane(*found)) {
            const QueryRow x = query_row(a, q, g, wave_row0 + li);
            for (int t = t_lo; t < t_hi; ++t) {
                if (inside(t - t_lo, block_whole)) continue;
                for (int key = t * TK; key < t * TK + TK && key < kv; ++key)
                    if (key >= x.lo && key <= x.place)
                        add_not_finite<F16>(st.o, a.v_pages + (int64_t)tab[key >> a.page_shift] * a.vc_s[0] + g * a.vc_s[1] + (key & page_mask) * a.vc_s[2], lh);
            }
        }
    }
    if (!has_rows) return;

    // ---- rows out ------------------------------------------------------------------------------
    int out_row = wave_row0 + li;
    asm volatile("" : "+v"(out_row));  // (worked out again: kept, the row's place would take registers over the loop)
    const QueryRow x = query_row(a, q, g, out_row);
    const float l = half_sum(st.l);
    if (piece.cut > 1) {
        if (piece.split == 0 && tid == 0) write_entry<ROWS>(a, piece, g);
        const int r = wave * 32 + li, part_row = piece.slot + piece.split * block_rows<ROWS>(q);
        if (!x.ok) return;
        float *dst = part_rows<D>(a, part_row, g) + (int64_t)r * D;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int rg = 0; rg < 4; ++rg)
                *(float4 *)(dst + mt * 32 + 8 * rg + 4 * lh) = make_float4(st.o[mt][4 * rg], st.o[mt][4 * rg + 1], st.o[mt][4 * rg + 2], st.o[mt][4 * rg + 3]);
        if (lh == 0) part_state(a, part_row, g)[r] = make_float2(st.m, l);
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing; NaN stays NaN
    // through LDS (each wave its own rows), so that they leave whole, 16 bytes a lane
    uint8_t *mine = smem + wave * TILEB;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg)
            *(uint2 *)(mine + li * ROWB + ((4 * mt + rg) ^ k_swizzle<D>(li)) * 16 + lh * 8) =
                make_uint2(pack16<F16>(st.o[mt][4 * rg] * inv, st.o[mt][4 * rg + 1] * inv),
                           pack16<F16>(st.o[mt][4 * rg + 2] * inv, st.o[mt][4 * rg + 3] * inv));
    RowWalk y(a, q, g, wave_row0 + lane / CH, RPL, a.o_s);
#pragma unroll
    for (int j = 0; j < TPT; ++j) {
        const int r = j * RPL + lane / CH, pos = lane % CH;
        const uint4 v = *(const uint4 *)(mine + r * ROWB + ((pos ^ k_swizzle<D>(r)) * 16));
        if (y.r < q.rows) *(uint4 *)(a.out + y.at + pos * 16) = v;
        y.next();
    }
    if (lh == 0 && x.ok) a.lse[(int64_t)x.token * a.n_q_heads + x.head] = l == 0.f ? -INFINITY : (st.m * a.scale_log2 + log2f(l)) * kLn2;
}

// ---- few rows ---------------------------------------------------------------------------------------

// A word that no kernel of the call writes, at a wave-uniform address: through the scalar cache, so that
// waiting for it does not wait for the copies in flight.
__device__ __forceinline__ int32_t scalar_load(const int32_t *p)
{
    return *(__attribute__((address_space(4))) const int32_t *)(uintptr_t)p;
}

// Shapes of the products: R = 16 or 32 query rows.  A lane holds scores of row lane % R, keys (256 / R) (e / 4) + 4 (lane / R) + e % 4; the
// operands of the output product take the keys in this order.
template <int R> struct FewShape {
    static constexpr int KD = 512 / R;              // depth of a matrix instruction
    static constexpr int SCORES = R / 2;            // per lane and tile
    static constexpr int ACC = R * R / 64;          // per accumulator
    typedef float Acc __attribute__((ext_vector_type(ACC)));
};
template <int R, bool F16>
__device__ __forceinline__ typename FewShape<R>::Acc few_product(bf16x8 x, bf16x8 y, typename FewShape<R>::Acc z)
{
    typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
    if constexpr (R == 32) return mfma32<F16>(x, y, z);
    else if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, x), __builtin_bit_cast(halfx8, y), z, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0);
}
// Largest and sum over the 64 / R lanes that share a row.
template <int R> __device__ __forceinline__ float row_max(float x)
{
    x = half_max(x);
    if constexpr (R == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}
template <int R> __device__ __forceinline__ float row_sum(float x)
{
    x = half_sum(x);
    if constexpr (R == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}
// Where chunks of a V row go (see v_swizzle): with 16 rows a transposing read takes 32 bytes of eight rows, not 64 of four.
template <int D, int R> __device__ __forceinline__ int few_v_swizzle(int row)
{
    if constexpr (R == 32) return v_swizzle<D>(row);
    else return D == 128 ? (row & 7) << 1 : row & 6;
}

template <bool F16, int DT>
__device__ __forceinline__ void few_add_not_finite(typename FewShape<16>::Acc (&o)[DT], const uint8_t *v_row, int lg)
{
    constexpr uint32_t kInf = F16 ? 0x7c00u : 0x7f80u;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        const uint2 x = *(const uint2 *)(v_row + dt * 32 + lg * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = i < 2 ? x.x : x.y;
            const bool bad = ((i & 1 ? pair >> 16 : pair) & 0x7fffu) >= kInf;
            o[dt][i] += bad ? (i & 1 ? high16<F16>(pair) : low16<F16>(pair)) : 0.f;
        }
    }
}

// R: query rows there is room for.  Up to 16 (single tokens of up to 16 heads a KV head) take half the instructions of 32 (four
// single tokens, 32 and 8 heads, f16: 11.8 us from warm caches, by 32 rows 14.3).
template <int D, bool F16, int R, int NW>
__device__ __forceinline__ void few_rows(const ChunkArgs &a, const Piece &piece, int g, uint8_t *smem)
{
    constexpr int ROWS = kRows<D>;
    constexpr int CH = D / 8, ROWB = D * 2, TILEB = kTileBytes<D>;
    constexpr int RPL = 64 / CH, LOADS = TK / RPL;
    typedef FewShape<R> S;
    constexpr int FRAGS = D / 16;                              // of a tile, K or V
    constexpr int KS = D / S::KD, DT = D / R;                  // steps of a score product, accumulators of the output
    typedef std::conditional_t<F16, half_t, uint16_t> T16;
    typedef __attribute__((address_space(3))) const uint4 *lds_u4;
    typedef __attribute__((address_space(3))) shortx4 *lds_s4;
    const Request &q = piece.q;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, li = lane % R, lg = lane / R;
    const QueryRow x = query_row(a, q, g, li);
    const int2 span = block_tiles<ROWS>(a, q, 0);
    const int per = div_up(span.y, piece.cut);
    int t_lo = piece.split * per, t_hi = t_lo + per;
    t_hi = span.x + (t_hi < span.y ? t_hi : span.y);
    t_lo = span.x + (t_lo < span.y ? t_lo : span.y);
    const int n_tiles = t_hi - t_lo, kv = q.kv;
    const bool busy = wave < n_tiles;

    const uint32_t base = lds_offset(smem), stage = base + wave * 2 * TILEB;  // K; the V stage follows
    const uint8_t *kp = uniform_ptr(a.k_pages + g * a.kc_s[1]), *vp = uniform_ptr(a.v_pages + g * a.vc_s[1]);
    const int page_mask = (1 << a.page_shift) - 1;
    const int32_t *tab = a.block_table + (int64_t)piece.b * a.bt_stride;
    const int ld_row = lane / CH, ld_pos = lane % CH;
    const uint32_t k_chunk = (uint32_t)(ld_pos ^ k_swizzle<D>(ld_row)), v_chunk = (uint32_t)(ld_pos ^ few_v_swizzle<D, R>(ld_row));
    // the pages of rows 0..15 and 16..31 of tile t
    auto pages_of = [&](int t) __attribute__((always_inline)) {
        int r0 = (t_lo + t) * TK, r1 = r0 + 16;
        r0 = r0 < kv ? r0 : kv - 1;
        r1 = r1 < kv ? r1 : kv - 1;
        return make_int2(scalar_load(tab + (r0 >> a.page_shift)), scalar_load(tab + (r1 >> a.page_shift)));
    };
    auto request = [&](auto v_tag, int t, int2 pages) __attribute__((always_inline)) {
        constexpr bool V = decltype(v_tag)::value;
        const uint32_t dst = __builtin_amdgcn_readfirstlane(stage + (V ? TILEB : 0));
        const int first = (t_lo + t) * TK, last = kv - 1 - first;
        const int64_t page_bytes = V ? a.vc_s[0] : a.kc_s[0];
        const int32_t rb = (int32_t)(V ? a.vc_s[2] : a.kc_s[2]);
        const uint8_t *p0 = (V ? vp : kp) + (int64_t)pages.x * page_bytes + (int64_t)(first & page_mask) * rb;
        const uint8_t *p1 = (V ? vp : kp) + (int64_t)pages.y * page_bytes + (int64_t)((first + 16) & page_mask) * rb;
        const uint32_t chunk = (V ? v_chunk : k_chunk) * 16;
        // (copy j's rows are RPL further, a power of two above theirs: the swizzle of the sum is that of both)
        auto chunk_of = [&](int j) __attribute__((always_inline)) {
            return chunk ^ (uint32_t)((V ? few_v_swizzle<D, R>(j * RPL) : k_swizzle<D>(j * RPL)) * 16);
        };
        if (last >= TK - 1) {
            const uint32_t off = (uint32_t)(ld_row * rb);
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                copy_to_lds((j * RPL < 16 ? p0 : p1) + (j * RPL % 16) * rb, off + chunk_of(j), dst + j * RPL * ROWB);
        } else {
            // rows past the end repeat the last one, by that row's own group
            const int last_group = last & ~(RPL - 1);
#pragma unroll 1
            for (int j = 0; j < LOADS; ++j) {
                const int src0 = j * RPL < last_group ? j * RPL : last_group;
                int src = src0 + ld_row;
                src = src < last ? src : last;
                copy_to_lds(uniform_ptr((src0 < 16 ? p0 : p1) + (src0 % 16) * rb), (uint32_t)((src - src0) * rb) + chunk_of(j),
                            __builtin_amdgcn_readfirstlane(dst + j * RPL * ROWB));
            }
        }
    };
    struct {
        typename S::Acc o[DT];
        float m, l;  // l: the numerators of this lane's keys until they are joined
    } st;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < S::ACC; ++e) st.o[dt][e] = 0.f;
    st.m = -INFINITY;
    st.l = 0.f;
    if (busy) {
        int2 pages = pages_of(wave);
        // query rows into the V stage, in the layout of a K tile, and on into registers
#pragma unroll
        for (int j = 0; j < R / RPL; ++j) {
            const int r = j * RPL + ld_row;
            const QueryRow y = query_row(a, q, g, r);
            copy_row_to_lds(a.q + y.token * a.q_s[0] + y.head * a.q_s[1] + (ld_pos ^ k_swizzle<D>(r)) * 16,
                            __builtin_amdgcn_readfirstlane(stage + TILEB + j * RPL * ROWB));
        }
        request(std::false_type{}, wave, pages);
        const uint32_t k_off0 = stage + li * ROWB + ((lg ^ k_swizzle<D>(li)) * 16);
        const int tr_s = lane & 15, tr_row = 4 * lg + (tr_s >> 2);
        const int tr_dchunk = (R == 32 ? 2 * ((lane >> 4) & 1) : 0) + ((tr_s & 3) >> 1);
        const uint32_t v_off0 = stage + TILEB + tr_row * ROWB + ((tr_dchunk ^ few_v_swizzle<D, R>(tr_row)) * 16) + (tr_s & 1) * 8;
        // K rows to registers, fragment KS * (16 or 32 rows) + step; query rows the same way
        auto read_rows = [&](uint32_t off, auto &frag) __attribute__((always_inline)) {
            constexpr int N = sizeof(frag) / sizeof(frag[0]);
            asm volatile("" : "+v"(off));  // the fragments' addresses are formed here, not kept over the loop
#pragma unroll
            for (int f = 0; f < N; ++f)
                frag[f] = __builtin_bit_cast(bf16x8, *(lds_u4)(uintptr_t)((off ^ (uint32_t)(f % KS * (S::KD * 2))) + f / KS * R * ROWB));
#pragma unroll
            for (int f = 0; f < N; ++f) asm volatile("" : "+v"(frag[f]));  // in registers: the stage is free
        };
        bf16x8 q_reg[KS];
        wait_vmem<LOADS>();
        read_rows(k_off0 + TILEB, q_reg);
        request(std::true_type{}, wave, pages);
        pages = pages_of(wave + NW);
        const float c = a.scale_log2;
        const int all_hi = __builtin_amdgcn_readfirstlane(x.place) + 1, all_lo = __builtin_amdgcn_readlane(x.lo, R - 1);
        // Copies in flight, oldest first: K of tile t, V of tile t.  A tile's rows go to registers as soon as they are there, and the
        // stage is asked for the next tile's.
        for (int t = wave; t < n_tiles; t += NW) {
            bf16x8 frag[FRAGS];
            uint32_t pp[2][S::SCORES / 2];
            const bool more = t + NW < n_tiles;
            wait_vmem<LOADS>();
            read_rows(k_off0, frag);
            if (more) request(std::false_type{}, t + NW, pages);
            typename S::Acc scores[TK / R];
            float s[S::SCORES];
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) {
                if (f % KS == 0)
#pragma unroll
                    for (int e = 0; e < S::ACC; ++e) scores[f / KS][e] = 0.f;
                scores[f / KS] = few_product<R, F16>(frag[f], q_reg[f % KS], scores[f / KS]);
            }
#pragma unroll
            for (int e = 0; e < S::SCORES; ++e) s[e] = scores[e / S::ACC][e % S::ACC];
            const int key0 = (t_lo + t) * TK;
            const bool part = key0 + TK > all_hi || key0 < all_lo;  // some row does not see all of the tile
            if (part) {
#pragma unroll
                for (int e = 0; e < S::SCORES; ++e) {
                    const int key = key0 + 256 / R * (e >> 2) + 4 * lg + (e & 3);
                    s[e] = key >= x.lo && key <= x.place ? s[e] : -INFINITY;
                }
            }
            float mx = s[0];
#pragma unroll
            for (int e = 1; e < S::SCORES; ++e) mx = fmaxf(mx, s[e]);
            mx = row_max<R>(mx);
            if (__any((mx - st.m) * c > kLazy)) {  // also while m is -inf
                const float m_new = fmaxf(st.m, mx);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((st.m - m_new) * c);
                st.m = m_new;
                st.l *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e = 0; e < S::ACC; ++e) st.o[dt][e] *= alpha;
            }
            const float mc = st.m == -INFINITY ? 0.f : st.m * c;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < S::SCORES; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -mc)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], c, -mc));
                sum += p0 + p1;
                pp[0][e >> 1] = pack16<F16>(p0, p1);
                pp[1][e >> 1] = pack16<F16>(p0 - low16<F16>(pp[0][e >> 1]), p1 - high16<F16>(pp[0][e >> 1]));
            }
            st.l += sum;
            if (more) wait_vmem<LOADS>();
            else wait_vmem<0>();
            {
                uint32_t off = v_off0;
                asm volatile("" : "+v"(off));
#pragma unroll
                for (int f = 0; f < FRAGS; ++f) {
                    const uint32_t at = (off ^ (uint32_t)(f % DT * (R * 2))) + f / DT * 16 * ROWB;
                    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)at));
                    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)(at + 256 / R * ROWB)));
                    frag[f] = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
#pragma unroll
                for (int f = 0; f < FRAGS; ++f) asm volatile("" : "+v"(frag[f]));
            }
            if (more) request(std::true_type{}, t + NW, pages);
            pages = pages_of(t + 2 * NW);
            const bool found = part && drop_not_finite<F16>(frag);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int f = 0; f < FRAGS; ++f) {
                    const uint32_t *u = pp[part] + 4 * (f / DT);
                    st.o[f % DT] = few_product<R, F16>(frag[f], __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3])), st.o[f % DT]);
                }
            if (found)
                for (int key = key0; key < key0 + TK && key < kv; ++key)
                    if (key >= x.lo && key <= x.place) {
                        const uint8_t *v_row = vp + (int64_t)tab[key >> a.page_shift] * a.vc_s[0] + (int64_t)(key & page_mask) * a.vc_s[2];
                        if constexpr (R == 32) add_not_finite<F16>(st.o, v_row, lg);
                        else few_add_not_finite<F16>(st.o, v_row, lg);
                    }
        }
    }

    // ---- merge of the waves, in fp32, through the stages (each wave its own: nothing reads them any more)
    constexpr int CPR = D / 4;                // 16-byte pieces (4 floats) per row
    constexpr int TPR = NW * 64 / R;          // threads per row
    constexpr int PASSES = CPR / TPR;         // pieces per thread
    float2 *ml = (float2 *)(smem + 2 * NW * TILEB);  // (m, l) [row][wave]
    const int row = tid / TPR;                // the row this thread finishes
    const float l_tot = row_sum<R>(st.l);
    if (lg == 0) ml[li * NW + wave] = make_float2(st.m, l_tot);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)  // (waves without a tile: zeros, so that what follows has no branches and its reads go out together)
#pragma unroll
        for (int e = 0; e < S::ACC; e += 4)
            *(float4 *)(smem + wave * 2 * TILEB + li * (D * 4) + ((R / 4 * dt + e / 4 * (64 / R) + lg) ^ (li & (CPR - 1))) * 16) =
                make_float4(st.o[dt][e], st.o[dt][e + 1], st.o[dt][e + 2], st.o[dt][e + 3]);
    __syncthreads();
    if (piece.cut > 1 && piece.split == 0 && tid == 0) write_entry<ROWS>(a, piece, g);
    if (row >= q.rows) return;
    float2 states[NW];
#pragma unroll
    for (int k = 0; k < NW; k += 2) {
        const float4 two = *(const float4 *)(ml + row * NW + k);
        states[k] = make_float2(two.x, two.y);
        states[k + 1] = make_float2(two.z, two.w);
    }
    float4 parts[NW][PASSES];
#pragma unroll
    for (int k = 0; k < NW; ++k)
#pragma unroll
        for (int u = 0; u < PASSES; ++u)
            parts[k][u] = *(const float4 *)(smem + k * 2 * TILEB + row * (D * 4) + (((tid % TPR + u * TPR) ^ (row & (CPR - 1))) * 16));
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < NW; ++k) top = fmaxf(top, states[k].x);
    float o[PASSES][4], l_sum = 0.f;
#pragma unroll
    for (int u = 0; u < PASSES; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[u][i] = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
        const float2 s = states[k];
        const float scale = s.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((s.x - top) * a.scale_log2);  // (NaN stays NaN)
        l_sum += scale * s.y;
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const float4 v = parts[k][u];
            o[u][0] += scale * v.x;
            o[u][1] += scale * v.y;
            o[u][2] += scale * v.z;
            o[u][3] += scale * v.w;
        }
    }
    if (piece.cut > 1) {
        const int part_row = piece.slot + piece.split * q.rows;
        float *dst = part_rows<D>(a, part_row, g) + row * D;
#pragma unroll
        for (int u = 0; u < PASSES; ++u) *(float4 *)(dst + (tid % TPR + u * TPR) * 4) = make_float4(o[u][0], o[u][1], o[u][2], o[u][3]);
        if (tid % TPR == 0) part_state(a, part_row, g)[row] = make_float2(top, l_sum);
        return;
    }
    const QueryRow y = query_row(a, q, g, row);
    const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;  // a row that sees nothing; NaN stays NaN
    T16 *dst = (T16 *)(a.out + y.token * a.o_s[0] + y.head * a.o_s[1]);
#pragma unroll
    for (int u = 0; u < PASSES; ++u)
        *(uint2 *)(dst + (tid % TPR + u * TPR) * 4) = make_uint2(pack16<F16>(o[u][0] * inv, o[u][1] * inv), pack16<F16>(o[u][2] * inv, o[u][3] * inv));
    if (tid % TPR == 0) a.lse[(int64_t)y.token * a.n_q_heads + y.head] = l_sum == 0.f ? -INFINITY : (top * a.scale_log2 + log2f(l_sum)) * kLn2;
}

// BLOCKS: the call may have requests with more than FEW rows
template <int D, bool F16, bool BLOCKS, int NW>
__global__ void __launch_bounds__(NW * 64, 2)
chunk_attn_kernel(ChunkArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int i = (int)a.by_kv_heads.div(blockIdx.x), g = (int)blockIdx.x - i * a.n_kv_heads;
    const int lane = threadIdx.x & 63;
    const Piece piece = a.list ? find_listed<kRows<D>>(a, i, lane) : find_piece<kRows<D>, NW, BLOCKS>(a, i, lane, (float *)(smem + kLds<D, BLOCKS, NW> - kShares * 4));
    if (!piece.valid) return;
    if (!BLOCKS || piece.q.rows <= FEW) {
        if (piece.q.rows <= 16) few_rows<D, F16, 16, NW>(a, piece, g, smem);
        else few_rows<D, F16, 32, NW>(a, piece, g, smem);
    }
    else if constexpr (BLOCKS) row_block<D, F16>(a, piece, g, smem);
}

// Joins the partial rows of the blocks that were cut: sum of O 2^((m - top) c) over that of l.  D / 4 threads pass a row's pieces, with
// the loads of BATCH of them in flight; the many pieces of a few rows are dealt to all groups of the workgroup, which then join theirs
// in LDS.  Bound by round trips to memory: entry, pieces, and out.
constexpr int MERGE_THREADS = 256, MERGE_GROUPS = 1024;
template <int D> __device__ __forceinline__ int merge_turns(int part_rows)  // of a block and KV head
{
    constexpr int GROUPS = MERGE_THREADS / (D / 4);
    const int by_rows = (part_rows + GROUPS - 1) / GROUPS, few = part_rows < FEW ? part_rows : FEW;
    return by_rows > few ? by_rows : few;
}
template <int D, bool F16>
__global__ void __launch_bounds__(MERGE_THREADS)
chunk_merge_kernel(ChunkArgs a)
{
    constexpr int TPR = D / 4, GROUPS = MERGE_THREADS / TPR, BATCH = 8;
    __shared__ float4 sums[MERGE_THREADS];
    __shared__ float2 states[GROUPS];
    const int turns = merge_turns<D>(a.part_rows), all = *a.n_entries * a.n_kv_heads * turns;
    const int group = threadIdx.x / TPR, col = threadIdx.x % TPR * 4;
    for (int i = blockIdx.x; i < all; i += gridDim.x) {
        const int block = i / turns, turn = i - block * turns;  // entry by KV head
        const Entry x = ((const Entry *)a.entries)[block];
        const bool few = x.rows <= FEW;  // a row a turn; else a group takes one
        const int r = few ? turn : turn * GROUPS + group;
        if (few ? turn >= x.rows : turn * GROUPS >= x.rows) continue;
        const int g = block % a.n_kv_heads;
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < x.rows) {
            const float2 *ml = part_state(a, x.slot, g) + r;
            const float *rows = part_rows<D>(a, x.slot, g) + (int64_t)r * D + col;
            for (int k0 = few ? group : 0; k0 < x.cut; k0 += few ? GROUPS * BATCH : BATCH) {
                float2 s[BATCH];
                float4 v[BATCH];
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const int k = k0 + (few ? GROUPS : 1) * j;
                    const int at = k < x.cut ? k : k0;
                    s[j] = ml[at * x.part];
                    v[j] = *(const float4 *)(rows + (int64_t)at * x.part * D);
                    if (k >= x.cut) s[j].y = 0.f;
                }
                float top = m;
#pragma unroll
                for (int j = 0; j < BATCH; ++j) top = fmaxf(top, s[j].x);
                const float old = l == 0.f ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.scale_log2);  // (NaN stays NaN)
                m = top;
                l *= old;
                o.x *= old, o.y *= old, o.z *= old, o.w *= old;
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const float scale = s[j].y == 0.f ? 0.f : __builtin_amdgcn_exp2f((s[j].x - top) * a.scale_log2);
                    const bool none = k0 + (few ? GROUPS : 1) * j >= x.cut;
                    l += scale * s[j].y;
                    o.x += none ? 0.f : scale * v[j].x;
                    o.y += none ? 0.f : scale * v[j].y;
                    o.z += none ? 0.f : scale * v[j].z;
                    o.w += none ? 0.f : scale * v[j].w;
                }
            }
        }
        if (few) {  // (the same for the whole workgroup)
            __syncthreads();  // the turn before is done with the sums
            sums[threadIdx.x] = o;
            if (col == 0) states[group] = make_float2(m, l);
            __syncthreads();
            if (group != 0) continue;
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, states[k].x);
            m = top;
            l = 0.f;
            o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) {
                const float2 s = states[k];
                const float4 v = sums[k * TPR + threadIdx.x];
                const float scale = s.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((s.x - top) * a.scale_log2);
                l += scale * s.y;
                o.x += scale * v.x;
                o.y += scale * v.y;
                o.z += scale * v.z;
                o.w += scale * v.w;
            }
        }
        if (r >= x.rows) continue;
        const int row = x.row0 + r, token = (int)a.by_group.div((uint32_t)row), head = g * a.group + row - token * a.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *(uint2 *)(a.out + (x.first + token) * a.o_s[0] + head * a.o_s[1] + col * 2) =
            make_uint2(pack16<F16>(o.x * inv, o.y * inv), pack16<F16>(o.z * inv, o.w * inv));
        if (col == 0) a.lse[(int64_t)(x.first + token) * a.n_q_heads + head] = l == 0.f ? -INFINITY : (m * a.scale_log2 + log2f(l)) * kLn2;
    }
}

template <int D, bool F16, bool BLOCKS, int NW> hipError_t launch_form(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream)
{
    auto kernel = chunk_attn_kernel<D, F16, BLOCKS, NW>;
    static std::atomic<uint64_t> allowed{0};
    if (const hipError_t e = allow_dynamic_lds((const void *)kernel, kLds<D, BLOCKS, NW>, allowed); e != hipSuccess) return e;
    if (a.list) {
        hipLaunchKernelGGL(chunk_list_kernel<kRows<D>>, dim3(1), dim3(LIST_THREADS), 0, stream, a);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.pieces * a.n_kv_heads), dim3(NW * 64), (kLds<D, BLOCKS, NW>), stream, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || plan.slots == 0) return e;
    hipLaunchKernelGGL((chunk_merge_kernel<D, F16>), dim3(MERGE_GROUPS), dim3(MERGE_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

ChunkPlan plan_chunk(const ls_chunk_desc &d, int compute_units)
{
    ChunkPlan plan{};
    const int64_t group = d.n_q_heads / d.n_kv_heads, most = d.max_new_len * group;
    const int64_t per_block = d.head_dim == 128 ? kRows<128> : kRows<64>;
    plan.blocks_possible = most > FEW;
    // At head_dim 64 two workgroups share a compute unit, of few rows alone four; counted as two they are cut less fine (one token after
    // 30 thousand rows, 4 KV heads: 14.4 us, counted as four 19.3; 24 of 1 to 30 thousand: 77 and 76).
    plan.units = (d.head_dim == 128 ? 1 : 2) * compute_units / d.n_kv_heads;
    if (plan.units < 2) plan.units = 2;
    // blocks at most: those of the rows there are, and one more per request with any
    const int64_t rows = (int64_t)d.n_tokens * group, requests = d.batch < d.n_tokens ? d.batch : d.n_tokens;
    int64_t blocks = (rows + (per_block - 1) * requests) / per_block, by_request = requests * ((most + per_block - 1) / per_block);
    if (blocks > by_request) blocks = by_request;
    if (blocks > rows) blocks = rows;
    // tiles of a block at most: the rows it sees, and a part of one at either end
    int64_t seen = d.max_kv_len;
    if (d.window > 0 && seen > d.window + (per_block + group - 1) / group) seen = d.window + (per_block + group - 1) / group;
    const int64_t tiles = (seen + TK - 1) / TK + 1;
    const bool may_cut = (float)tiles * (plan.blocks_possible ? 1.f : kFewTile) > kWhole;
    // room for the pieces that cutting adds, and for partial rows
    plan.part_rows = (int)(most < per_block ? most : per_block);
    plan.extra = may_cut ? (plan.blocks_possible ? 2 : 4) * plan.units : 0;
    plan.slots = plan.extra * plan.part_rows;
    const bool one_each = !plan.blocks_possible && !may_cut;  // a piece is a request
    plan.pieces = one_each ? d.batch : blocks + plan.extra;
    plan.listed = d.batch > kWave && !one_each;
    // Few requests that are cut: workgroups of four waves, of which two share a compute unit and one loads while the other ends (one token
    // after 30 thousand rows, 8 KV heads: 33.0 -> 26.4 us, eight after 9 thousand 57.5 -> 51.9, twelve after 3 thousand 31.7 -> 30.9; but 24
    // after 1 to 30 thousand 262.5 -> 265, 16 of 32 KV heads 205 -> 214).  Not cut, eight are faster: four after 1500 11.7 us, by four 15.1.
    plan.few_waves = may_cut && requests * d.n_kv_heads <= compute_units / 2 ? 4 : 8;
    return plan;
}

hipError_t launch_chunk_attn(const ChunkArgs &a, const ChunkPlan &plan, int dtype, int head_dim, hipStream_t stream)
{
#define LS_CHUNK_CASE(HH)                                                                    \
    (plan.blocks_possible  ? (head_dim == 128 ? launch_form<128, HH, true, 8>(a, plan, stream) \
                                              : launch_form<64, HH, true, 4>(a, plan, stream)) \
     : head_dim == 64      ? launch_form<64, HH, false, 4>(a, plan, stream)                     \
     : plan.few_waves == 4 ? launch_form<128, HH, false, 4>(a, plan, stream)                    \
                           : launch_form<128, HH, false, 8>(a, plan, stream))
    return dtype == LS_F16 ? LS_CHUNK_CASE(true) : LS_CHUNK_CASE(false);
#undef LS_CHUNK_CASE
}

size_t chunk_list_bytes(int batch) { return ((size_t)batch + 1) * sizeof(Listed); }
size_t chunk_entry_bytes() { return sizeof(Entry); }

}  // namespace ls
