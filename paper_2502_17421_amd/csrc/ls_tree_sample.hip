// Acceptance of a drafted tree at a temperature, by rejection from given random numbers.
//
// At a node with the target's distribution p and the draft's q, children x_1, x_2, ... in turn: x_j is accepted with probability
// min(1, p_j(x_j) / q_j(x_j)), p_1 = p, q_1 = q; after a refusal p_{j+1} is the normalised positive part of p_j - q_j, and q_{j+1} is q_j
// (independent draws) or q_j without x_j, normalised (without replacement).  All the p_j are one family: with
//   a_1 = 0, S_1 = W_1 = 1;   a_{j+1} = a_j + S_j / W_j
//   S_j = sum over v of max(p(v) - a_j q(v), 0),   W_j = the mass of q that is left (1 with replacement)
// p_j = max(p - a_j q, 0) / S_j: the positive part of a positive part is the positive part of the sum of what is taken away, and
// a refused token, p_j(x) < q_j(x), is at zero from then on, so that it can be set to p(x) = q(x) = 0.  x is accepted if
//   (p(x) - a_j q(x)) W_j > u q(x) S_j,
// and the next token is the first v at which the sum of max(p - a q, 0) passes u' S.  A node costs one pass over two rows, and each refusal
// a sum over what is then in registers.
//
// Tokens that were chosen: q(x) = 1, a = 0, and a refused x is set to p(x) = 0.
//
// Everything is in 64 bits: the border between two neighbouring tokens in a cumulated sum over 150 thousand of them is missed by 32 bits about
// once in a hundred draws.
//
// A sequence belongs to a group of workgroups, one per slice of the vocabulary, which walk its tree together: each keeps its slice of p and q
// in registers, tells the others its sums, and decides what all of them decide from all sums in the same order.  See Exchange.
#include <float.h>

#include <type_traits>

#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = kSampleThreads;
constexpr int WAVES = NT / kWave;
constexpr int kNone = INT32_MAX;
template <int N> using Const = std::integral_constant<int, N>;

// 2^y for y <= 0, to 1e-14 of its value: the Taylor series of exp(f ln 2), |f| <= 1/2, whose first term left out is
// (ln 2 / 2)^12 / 12! = 6e-15.
__device__ __forceinline__ double exp2_of(double y)
{
    y = y > -1100.0 ? y : -1100.0;  // 0 after the last step
    const double n = __builtin_rint(y), f = y - n;
    double r = 4.4455382718708116e-10;   // ln2^11 / 11!
    r = __builtin_fma(r, f, 7.0549116208011233e-09);
    r = __builtin_fma(r, f, 1.0178086009239699e-07);
    r = __builtin_fma(r, f, 1.3215486790144309e-06);
    r = __builtin_fma(r, f, 1.5252733804059841e-05);
    r = __builtin_fma(r, f, 1.5403530393381610e-04);
    r = __builtin_fma(r, f, 1.3333558146428443e-03);
    r = __builtin_fma(r, f, 9.6181291076284772e-03);
    r = __builtin_fma(r, f, 5.5504108664821580e-02);
    r = __builtin_fma(r, f, 2.4022650695910072e-01);
    r = __builtin_fma(r, f, 6.9314718055994531e-01);
    r = __builtin_fma(r, f, 1.0);
    return __builtin_ldexp(r, (int)n);
}

// exp(logit - top) at a temperature; heat = log2(e) / temperature
__device__ __forceinline__ double weight(float logit, float top, double heat)
{
    return logit == -INFINITY ? 0.0 : exp2_of(((double)logit - (double)top) * heat);
}

__device__ __forceinline__ float cleaned(float x) { return x != x ? -INFINITY : (x > FLT_MAX ? FLT_MAX : x); }

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T x[8];
};

// Entries at .. at + 7 of a row
template <typename T> __device__ __forceinline__ void load_run(const T *row, int at, int vocab, float (&x)[8])
{
    if (at + 8 <= vocab) {
        const Run<T> r = *(const Run<T> *)(row + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = cleaned(Elem<T>::load(&r.x[e]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < vocab ? cleaned(Elem<T>::load(row + at + e)) : -INFINITY;
    }
}

// x of the lane that a DPP control names; `other` where there is none
template <int CTRL, int ROWS> __device__ __forceinline__ int from_lane(int x, int other)
{
    return __builtin_amdgcn_update_dpp(other, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ double from_lane(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)from_lane<CTRL, ROWS>((int)(u >> 32), 0) << 32 | (uint32_t)from_lane<CTRL, ROWS>((int)u, 0));
}
// Sums over the lanes up to this one: from 1, 2, 4 and 8 lanes below in the row of 16, the last lane of the row before to rows 1 and 3, lane 31 to rows 2 and 3
__device__ __forceinline__ double lanes_scan(double x)
{
    x += from_lane<0x111, 0xf>(x);
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);
    x += from_lane<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ double of_lane(double x, int lane)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)u, lane));
}
// A value that is the same in all lanes, in scalar registers
__device__ __forceinline__ double uniform(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 |
                                          (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
__device__ __forceinline__ double lanes_sum(double x) { return of_lane(lanes_scan(x), 63); }
__device__ __forceinline__ float lanes_max(float x)
{
    auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        x = fmaxf(x, __int_as_float(from_lane<decltype(ctrl)::value, decltype(rows)::value>(__float_as_int(x), __float_as_int(-INFINITY))));
    };
    step(Const<0x111>{}, Const<0xf>{});
    step(Const<0x112>{}, Const<0xf>{});
    step(Const<0x114>{}, Const<0xf>{});
    step(Const<0x118>{}, Const<0xf>{});
    step(Const<0x142>{}, Const<0xa>{});
    step(Const<0x143>{}, Const<0xc>{});
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ int lanes_min(int v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int y = __shfl_xor(v, off, kWave);
        v = y < v ? y : v;
    }
    return v;
}

// What the workgroups of a group tell each other: per exchange a record each, of 32-bit words with the exchange's number in the upper half
// of 64 bits.  A word is written and read at once, so its number says that its value is there, and no fence is needed; two sets of records
// take turns, since nobody is at exchange n + 2 before everybody has read those of n.  The numbers start at 1 in records that
// a kernel before this one has cleared.
//
// The workgroups of a group are next to each other in the launch, so that all of the first group that is not done yet are on the card, or
// will be when what else runs there is done.  No wait is unbounded all the same: who has polled spin_limit times gives up on
// the group, and the first of them (the state word says so) walks the tree alone, slice after slice, with the same sums in the same order.
// What it writes are the bits that the group writes if it gets to the end after all.
constexpr int kRecordWords = 8;  // p: 0 largest entry, 1-2 sum, 3 where the largest is; q: 4 largest entry, 5-6 sum

struct Exchange {
    uint64_t *records;  // [2][slices][kRecordWords]
    uint64_t *state;    // 1: some workgroup walks alone
    int slices, slice, spin_limit;
    uint32_t number;

    __device__ __forceinline__ uint64_t *record(int of) const { return records + ((number & 1) * slices + of) * kRecordWords; }
    // lane i < 4 of wave 0 or 1 writes word 4 * wave + i
    __device__ __forceinline__ void tell(int wave, int lane, uint32_t value) const
    {
        if (lane < 4)
            __hip_atomic_store(record(slice) + 4 * wave + lane, (uint64_t)number << 32 | value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // lane i reads the half record of slice i; false: given up
    __device__ __forceinline__ bool hear(int wave, int lane, uint32_t (&value)[4]) const
    {
        const uint64_t *from = record(lane < slices ? lane : 0) + 4 * wave;
        for (int poll = 0; poll < spin_limit; ++poll) {
            bool there = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t word = __hip_atomic_load(from + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                value[i] = (uint32_t)word;
                there &= (uint32_t)(word >> 32) == number;
            }
            if (__all(there)) return true;
            if ((poll & 15) == 15 && __hip_atomic_load(state, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0) return false;
        }
        return false;
    }
};

__device__ __forceinline__ double from_words(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }

__global__ void __launch_bounds__(256)
sample_clear_kernel(uint64_t *words, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) words[i] = 0;
}

// The walk is a sequence of passes over a slice (over all of them, one after the other, where a workgroup is alone): the weights of a node's
// rows and their sums; the sums of max(p - a q, 0) after a refusal; the search for the next token.
enum Pass { kRows, kResidual, kDraw };

template <typename TT, typename TD, int EPT>
__global__ void __launch_bounds__(NT, EPT == 8 ? 2 : 2)
tree_sample_kernel(SampleArgs a)
{
    constexpr int RUNS = EPT / 8;  // a thread's entries: runs of 8, the lanes' runs side by side; a wave's are contiguous
    constexpr int SLICE = NT * EPT;
    static_assert(LS_MAX_TREE <= NT, "a thread per node");
    __shared__ int32_t tok[LS_MAX_TREE], path[LS_MAX_TREE];
    __shared__ float accept_u[LS_MAX_TREE];
    __shared__ double kid_p[LS_MAX_TREE], kid_q[LS_MAX_TREE], kid_logit[LS_MAX_TREE];
    __shared__ double new_logit[LS_MAX_TREE], new_total[LS_MAX_TREE];  // of the new tokens: logit / temperature below the largest, and the sum of the weights
    __shared__ uint64_t kid_mask[LS_MAX_TREE / kWave];
    __shared__ float wave_top[2][WAVES];
    __shared__ double wave_sum[2][WAVES];
    __shared__ int32_t wave_best[WAVES];
    // of the slices: largest entry, sum of the weights relative to it, and where the largest of p is first; then the sums of max(p - a q, 0) and of q
    __shared__ float part_top[2][kSampleSlices];
    __shared__ double part_sum[2][kSampleSlices];
    __shared__ int32_t part_best[kSampleSlices];
    __shared__ int32_t first_sh, last_sh, heard_sh[2];

    const int b = (int)(blockIdx.x / (uint32_t)a.slices), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Exchange ex;
    ex.slices = a.slices, ex.slice = (int)(blockIdx.x % (uint32_t)a.slices), ex.spin_limit = a.spin_limit, ex.number = 0;
    ex.state = a.records + (int64_t)b * (2 * a.slices + 1) * kRecordWords;
    ex.records = ex.state + kRecordWords;
    bool alone = false;  // this workgroup does all slices
    const bool told = a.slices > 1;
    if (told && __syncthreads_or(tid == 0 && __hip_atomic_load(ex.state, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0)) return;
    const TT *target = (const TT *)a.target + b * a.t_stride[0];
    const TD *draft = (const TD *)a.draft + (a.draft ? b * a.d_stride[0] : 0);

    // thread i has node i
    const bool is_node = tid < a.n_tree;
    int my_parent = -1, my_tok = -1, bad = 0;
    if (is_node) {
        my_parent = a.parents[(int64_t)b * a.n_tree + tid];
        if (my_parent < -1 || my_parent >= tid) bad = 1, my_parent = -1;
        my_tok = tok[tid] = a.draft_tokens[(int64_t)b * a.n_tree + tid];
        accept_u[tid] = a.accept_uniforms[(int64_t)b * a.n_tree + tid];
        path[tid] = tid == 0 ? 0 : -1;
        if ((uint32_t)my_tok >= (uint32_t)a.vocab) my_parent = -1;  // nobody's child
    }
    int err = __syncthreads_or(bad) ? 1 : 0;

    float temp = a.temperature[b], draft_temp = a.draft_temperature ? a.draft_temperature[b] : temp;
    if (!(temp >= 0.f && temp <= FLT_MAX)) err |= 2, temp = 0.f;
    if (!(draft_temp >= 0.f && draft_temp <= FLT_MAX)) err |= 2, draft_temp = 0.f;
    const bool greedy = temp == 0.f;
    const bool drawn = a.draft && !greedy && draft_temp > 0.f;
    const double heat = uniform(1.4426950408889634074 / (greedy ? 1.0 : (double)temp));
    const double draft_heat = uniform(drawn ? 1.4426950408889634074 / (double)draft_temp : 0.0);

    Pass pass = kRows;
    int cur = 0, len = 1, next = -1;
    int writer = 0;                     // the slice whose workgroup draws the token and writes the outputs
    bool inner = false;                 // the node has children, and what they were drawn from counts
    bool scaled = false;                // p and q are probabilities, and not weights relative to the wave's largest entries
    float wt = 0.f, wq = 0.f;           // these entries
    float top = 0.f, draft_top = 0.f;   // the largest of the rows
    double total = 0, draft_total = 0;  // sums of the weights relative to them
    double taken = 0, mass = 1, left = 1;  // a, S, W
    double rest = 0;                    // what the sum has to pass in the writer's slice
    int refused = 0;                    // the children before this node have been
    double p[EPT], q[EPT];

    const int own = wave * (kWave * EPT) + lane * 8;  // this thread's first entry in a slice

    while (true) {
        if (pass == kRows) {
            const uint64_t kids = __ballot(my_parent == cur && tid > cur);
            if (lane == 0) kid_mask[wave] = kids;
            inner = __syncthreads_or(kids != 0) && drawn;
            taken = 0, mass = left = 1;
            refused = 0;
            scaled = false;
        }
        ++ex.number;
        bool heard = true;
        int slice = alone ? 0 : ex.slice, end = alone ? a.slices : ex.slice + 1;
        if (pass == kDraw) slice = writer, end = writer + 1;
        for (; slice < end && heard; ++slice) {
            if (pass == kRows || alone) {
                const TT *row = target + cur * a.t_stride[1];
                const int at = slice * SLICE + own;
                float x[RUNS][8], y[RUNS][8];
#pragma unroll
                for (int r = 0; r < RUNS; ++r) load_run(row, at + r * kWave * 8, a.vocab, x[r]);
                if (inner) {
                    const TD *drow = draft + cur * a.d_stride[1];
#pragma unroll
                    for (int r = 0; r < RUNS; ++r) load_run(drow, at + r * kWave * 8, a.vocab, y[r]);
                }
                float m = -INFINITY, mq = -INFINITY;
#pragma unroll
                for (int r = 0; r < RUNS; ++r)
#pragma unroll
                    for (int e = 0; e < 8; ++e) m = fmaxf(m, x[r][e]);
                wt = lanes_max(m);
                if (greedy) {
                    int best = kNone;
#pragma unroll
                    for (int r = RUNS - 1; r >= 0; --r)
#pragma unroll
                        for (int e = 7; e >= 0; --e)
                            if (x[r][e] == wt) best = at + r * kWave * 8 + e;
                    best = wt > -INFINITY ? lanes_min(best) : kNone;
                    if (lane == 0) wave_best[wave] = best;
                }
#pragma unroll
                for (int r = 0; r < RUNS; ++r)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        p[r * 8 + e] = weight(x[r][e], wt, heat);
                        if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                    }
                if (inner) {
#pragma unroll
                    for (int r = 0; r < RUNS; ++r)
#pragma unroll
                        for (int e = 0; e < 8; ++e) mq = fmaxf(mq, y[r][e]);
                    wq = lanes_max(mq);
#pragma unroll
                    for (int r = 0; r < RUNS; ++r)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            q[r * 8 + e] = weight(y[r][e], wq, draft_heat);
                            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                        }
                } else {
                    wq = -INFINITY;
#pragma unroll
                    for (int e = 0; e < EPT; ++e) q[e] = 0.0;
                }
            }
            if (pass != kRows) {
                // to probabilities, with the refused tokens at zero
                const bool anew = alone || !scaled;
                if (anew) {
                    const double f = wt > -INFINITY ? exp2_of(((double)wt - top) * heat) / total : 0.0;
                    const double fq = wq > -INFINITY ? exp2_of(((double)wq - draft_top) * draft_heat) / draft_total : 0.0;
#pragma unroll
                    for (int e = 0; e < EPT; ++e) {
                        p[e] *= f;
                        q[e] *= fq;
                    }
                    scaled = true;
                }
                for (int w = anew ? 0 : (refused - 1) / kWave; w * kWave < refused; ++w)
                    for (uint64_t m = kid_mask[w]; m; m &= m - 1) {
                        const int k = w * kWave + __builtin_ctzll(m);
                        if (k >= refused) break;
                        const int at = tok[k] - (slice * SLICE + own);
#pragma unroll
                        for (int e = 0; e < EPT; ++e)
                            if (at == (e >> 3) * kWave * 8 + (e & 7)) p[e] = q[e] = 0.0;
                    }
            }
            if (pass == kDraw) break;
            // sums over the thread, the wave, the slice (in waves 0 and 1), relative to the largest of the waves' tops; then to everybody
            double s = 0, sq = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                const double r = p[e] - taken * q[e];
                s += r > 0 ? r : 0.0;
                sq += q[e];
            }
            s = lanes_sum(s);
            sq = lanes_sum(sq);
            if (lane == 0) {
                wave_top[0][wave] = wt, wave_sum[0][wave] = s;
                wave_top[1][wave] = wq, wave_sum[1][wave] = sq;
            }
            __syncthreads();
            if (wave == 0 || (wave == 1 && inner)) {
                const bool mine = lane < WAVES;
                const float m = mine ? (pass == kRows ? wave_top[wave][lane] : 0.f) : -INFINITY, mm = lanes_max(m);
                const double part = m > -INFINITY ? wave_sum[wave][lane] * exp2_of(((double)m - mm) * (wave ? draft_heat : heat)) : 0.0;
                const double sum = lanes_sum(part);
                const int best = greedy && wave == 0 ? lanes_min(mine && m == mm ? wave_best[lane] : kNone) : kNone;
                if (alone || !told) {
                    if (lane == 0) {
                        part_top[wave][slice] = mm, part_sum[wave][slice] = sum;
                        if (wave == 0) part_best[slice] = best;
                        heard_sh[wave] = 1;
                    }
                } else {
                    const uint64_t bits = __builtin_bit_cast(uint64_t, sum);
                    ex.tell(wave, lane, lane == 0 ? __float_as_uint(mm) : lane == 1 ? (uint32_t)bits : lane == 2 ? (uint32_t)(bits >> 32) : (uint32_t)best);
                    uint32_t value[4];
                    const bool all = ex.hear(wave, lane, value);
                    if (lane < a.slices) {
                        part_top[wave][lane] = __uint_as_float(value[0]);
                        part_sum[wave][lane] = from_words(value[1], value[2]);
                        if (wave == 0) part_best[lane] = (int)value[3];
                    }
                    if (lane == 0) heard_sh[wave] = all;
                }
            }
            __syncthreads();
            heard = heard_sh[0] && (!inner || heard_sh[1]);
        }

        if (!heard) {  // the first one to give up goes on alone, from the root
            if (tid == 0) {
                unsigned long long expected = 0;
                first_sh = __hip_atomic_compare_exchange_strong((unsigned long long *)ex.state, &expected, 1ull, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                                                __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (!first_sh) return;
            alone = true;
            pass = kRows;
            cur = 0, len = 1;
            if (is_node) path[tid] = tid == 0 ? 0 : -1;
            __syncthreads();
            continue;
        }

        if (pass == kDraw) {
            double s = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                const double r = p[e] - taken * q[e];
                p[e] = r > 0 ? r : 0.0;
                s += p[e];
            }
            s = lanes_sum(s);
            if (lane == 0) wave_sum[0][wave] = s;
            if (tid == 0) first_sh = kNone, last_sh = -1;
            __syncthreads();
            double before = 0;  // of the entries before this wave's, then before this run
            for (int w = 0; w < wave; ++w) before += wave_sum[0][w];
            int first = kNone, last = -1;
#pragma unroll
            for (int r = 0; r < RUNS; ++r) {
                double run = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) run += p[r * 8 + e];
                const double upto = lanes_scan(run);
                double c = before + (upto - run);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int v = writer * SLICE + own + r * kWave * 8 + e;
                    c += p[r * 8 + e];
                    if (p[r * 8 + e] > 0) {
                        last = v;
                        if (first == kNone && c > rest) first = v;
                    }
                }
                before += of_lane(upto, 63);
            }
            if (first != kNone) atomicMin(&first_sh, first);
            if (last >= 0) atomicMax(&last_sh, last);
            __syncthreads();
            next = first_sh != kNone ? first_sh : last_sh;
            break;
        }

        // What the sums say
        const double per_temp = 1.0 / (greedy ? 1.0 : (double)temp);
        const bool mine = lane < a.slices;
        double part = mine ? part_sum[0][lane] : 0.0;
        int best = kNone;
        if (pass == kRows) {
            const float m = mine ? part_top[0][lane] : -INFINITY;
            top = lanes_max(m);
            part = m > -INFINITY ? part * exp2_of(((double)m - top) * heat) : 0.0;
            total = lanes_sum(part);
            if (greedy && total > 0) best = lanes_min(mine && m == top ? part_best[lane] : kNone);
            if (total > 0) part /= total;
            if (inner) {
                const float mq = mine ? part_top[1][lane] : -INFINITY;
                draft_top = lanes_max(mq);
                draft_total = lanes_sum(mq > -INFINITY ? part_sum[1][lane] * exp2_of(((double)mq - draft_top) * draft_heat) : 0.0);
            }
            // the children's probabilities, each in its own thread; a token that comes again has been refused before
            if (my_parent == cur && tid > cur) {
                const float l = cleaned(Elem<TT>::load(target + cur * a.t_stride[1] + my_tok));
                double px = total > 0 ? weight(l, top, heat) / total : 0.0, qx = 1.0;
                kid_logit[tid] = ((double)l - top) * per_temp;
                if (inner) {
                    const float lq = cleaned(Elem<TD>::load(draft + cur * a.d_stride[1] + my_tok));
                    qx = draft_total > 0 ? weight(lq, draft_top, draft_heat) / draft_total : 0.0;
                }
                for (int w = 0; w <= wave; ++w)
                    for (uint64_t k = kid_mask[w]; k; k &= k - 1) {
                        const int i = w * kWave + __builtin_ctzll(k);
                        if (i >= tid) break;
                        if (tok[i] == my_tok) px = 0.0, qx = inner ? 0.0 : 1.0;
                    }
                kid_p[tid] = px, kid_q[tid] = qx;
            }
            __syncthreads();
        }
        mass = lanes_sum(part);
        if (pass == kResidual && inner && !a.with_replacement) left = lanes_sum(mine ? part_sum[1][lane] : 0.0);

        // the children that have not been tried
        int found = -1;
        bool again = false;
        for (int w = refused / kWave; w < LS_MAX_TREE / kWave && found < 0 && !again; ++w) {
            uint64_t m = kid_mask[w];
            if (w == refused / kWave) m &= ~0ull << (refused % kWave);
            for (; m && found < 0 && !again; m &= m - 1) {
                const int k = w * kWave + __builtin_ctzll(m);
                const double px = kid_p[k], qx = kid_q[k], u = accept_u[k];
                const bool ok = greedy ? tok[k] == best : (px - (inner ? taken * qx : 0.0)) * left > u * qx * mass;
                if (ok) {
                    found = k;
                } else {
                    refused = k + 1;
                    again = !greedy;
                }
            }
        }
        if (found >= 0) {
            if (tid == 0) path[len] = found, new_logit[len - 1] = kid_logit[found], new_total[len - 1] = total;
            ++len;
            cur = found;
            pass = kRows;
            __syncthreads();  // children and parts are read before the next node's are written
            continue;
        }
        if (again) {
            if (inner) taken = uniform(left > 0 ? fmin(taken + mass / left, 1e300) : 1e300);  // (finite: q(v) = 0 stays out of it)
            pass = kResidual;
            continue;
        }
        // the path ends here
        if (greedy) {
            next = best == kNone ? -1 : best;
        } else if (mass > 0) {
            const double upto = lanes_scan(part), point = (double)a.sample_uniforms[b] * mass;
            const uint64_t passed = __ballot(part > 0 && upto > point), some = __ballot(part > 0);
            writer = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some);
            rest = uniform(point - of_lane(upto - part, writer));
            pass = kDraw;
        }
        if (!alone && writer != ex.slice) return;
        if (pass != kDraw) break;
        __syncthreads();
    }
    if (tid == 0) {
        if (next >= 0) {
            const float l = cleaned(Elem<TT>::load(target + cur * a.t_stride[1] + next));
            new_logit[len - 1] = ((double)l - top) / (greedy ? 1.0 : (double)temp), new_total[len - 1] = total;
        } else {
            new_logit[len - 1] = -INFINITY, new_total[len - 1] = 1.0;
            err |= 4;
        }
        a.len[b] = len;
        a.next[b] = next;
        if (a.err_flag) a.err_flag[b] = err;
    }
    __syncthreads();
    if (is_node) {
        const int64_t at = (int64_t)b * a.n_tree + tid;
        a.path[at] = path[tid];
        if (a.logprobs) a.logprobs[at] = tid < len ? (float)(new_logit[tid] - log(new_total[tid])) : 0.f;
    }
}

template <typename TT, typename TD> hipError_t launch_types(const SampleArgs &a, hipStream_t stream)
{
    const dim3 grid((uint32_t)a.batch * a.slices), block(NT);
    if (a.slice == NT * 8) hipLaunchKernelGGL((tree_sample_kernel<TT, TD, 8>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((tree_sample_kernel<TT, TD, 16>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_for(const SampleArgs &a, int draft_dtype, hipStream_t stream)
{
    if (draft_dtype == LS_F32) return launch_types<TT, float>(a, stream);
    if (draft_dtype == LS_F16) return launch_types<TT, half_t>(a, stream);
    return launch_types<TT, uint16_t>(a, stream);
}

}  // namespace

hipError_t launch_tree_sample(const SampleArgs &a, int target_dtype, int draft_dtype, hipStream_t stream)
{
    if (a.slices > 1) {
        const int64_t words = (int64_t)sample_record_bytes(a.batch, a.slices) / 8;
        const int64_t groups = (words + 255) / 256;
        hipLaunchKernelGGL(sample_clear_kernel, dim3(groups < 1024 ? groups : 1024), dim3(256), 0, stream, a.records, words);
    }
    if (!a.draft) draft_dtype = target_dtype;
    if (target_dtype == LS_F32) return launch_for<float>(a, draft_dtype, stream);
    if (target_dtype == LS_F16) return launch_for<half_t>(a, draft_dtype, stream);
    return launch_for<uint16_t>(a, draft_dtype, stream);
}

}  // namespace ls
