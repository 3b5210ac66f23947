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

// a b + c with c in scalar registers: for a constant c the compiler takes the form whose result is its third operand, and moves the constant there
// before each of them.
__device__ __forceinline__ double fma_scalar(double a, double b, double c)
{
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
    return d;
}

// 2^y for y <= 0, to 4e-14 of its value: y = n + f, |f| <= 1/2, and 2^f = 1 + f g(f) with the polynomial g of degree 8 that meets
// (2^f - 1) / f at the zeros of the Chebyshev polynomial of degree 9.  Less than 2^-1074, and NaN, give 0.
__device__ __forceinline__ double exp2_of(double y)
{
    y = __builtin_fmax(y, -1100.0);
    const double n = __builtin_rint(y), f = y - n;
    double r = fma_scalar(f, 1.0203121047189341e-07, 1.3255224879317324e-06);
    r = fma_scalar(r, f, 1.525268684635191e-05);
    r = fma_scalar(r, f, 1.540345585244999e-04);
    r = fma_scalar(r, f, 1.3333558179042969e-03);
    r = fma_scalar(r, f, 9.618129159402565e-03);
    r = fma_scalar(r, f, 5.5504108664760424e-02);
    r = fma_scalar(r, f, 2.402265069581299e-01);
    r = fma_scalar(r, f, 6.931471805599453e-01);
    r = __builtin_fma(r, f, 1.0);
    return __builtin_ldexp(r, (int)n);
}

// exp((logit - top) / temperature), heat = log2(e) / temperature; 0 for -inf and NaN, also where top is -inf
__device__ __forceinline__ double weight(float logit, double top, double heat) { return exp2_of(((double)logit - top) * heat); }

// The same of four logits, step by step, so that no step waits for the one before it.  (Left to itself the compiler takes one after the other, or starts
// all of a thread's at once and runs out of registers.)
__device__ __forceinline__ void weights(const float (&logit)[4], double top, double heat, double (&w)[4])
{
    double n[4], f[4];
#define LS_STEP(...)                        \
    _Pragma("unroll") for (int i = 0; i < 4; ++i) __VA_ARGS__; \
    __builtin_amdgcn_sched_barrier(0);
    LS_STEP(f[i] = (double)logit[i] - top)
    LS_STEP(f[i] = __builtin_fmax(f[i] * heat, -1100.0))
    LS_STEP(n[i] = __builtin_rint(f[i]))
    LS_STEP(f[i] = f[i] - n[i])
    LS_STEP(w[i] = fma_scalar(f[i], 1.0203121047189341e-07, 1.3255224879317324e-06))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 1.525268684635191e-05))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 1.540345585244999e-04))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 1.3333558179042969e-03))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 9.618129159402565e-03))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 5.5504108664760424e-02))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 2.402265069581299e-01))
    LS_STEP(w[i] = fma_scalar(w[i], f[i], 6.931471805599453e-01))
    LS_STEP(w[i] = __builtin_fma(w[i], f[i], 1.0))
    LS_STEP(w[i] = __builtin_ldexp(w[i], (int)n[i]))
#undef LS_STEP
}

// The largest finite number of a type, which +inf counts as
template <typename T> constexpr float kLargest = std::is_same_v<T, half_t> ? 65504.f : sizeof(T) == 4 ? FLT_MAX : 3.38953139e38f;
template <typename T> __device__ __forceinline__ float entry_of(const T *row, int at)
{
    const float x = Elem<T>::load(row + at);
    return x > kLargest<T> ? kLargest<T> : x;
}

// Eight entries of a row as they are stored
template <typename T> struct Run {
    static constexpr int WORDS = 2 * sizeof(T);
    uint32_t w[WORDS];
    __device__ __forceinline__ float entry(int e) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        const uint32_t u = w[e / 2];
        if constexpr (std::is_same_v<T, half_t>) return half_to_float((uint16_t)(e & 1 ? u >> 16 : u));
        else return __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void set(int e, bool set, uint32_t bits)
    {
        if constexpr (sizeof(T) == 4) w[e] = set ? bits : w[e];
        else w[e / 2] = set ? (e & 1 ? (w[e / 2] & 0xffffu) | bits << 16 : (w[e / 2] & 0xffff0000u) | bits) : w[e / 2];
    }
    // Entries are unpacked anew from here on, and not kept apart: the compiler would hold all of them, and all the exponentials that it can start with them.
    __device__ __forceinline__ void stay_packed()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) asm volatile("" : "+v"(w[i]));
    }
    static constexpr uint32_t kMinusInf = sizeof(T) == 4 ? 0xff800000u : std::is_same_v<T, half_t> ? 0xfc00u : 0xff80u;
    static constexpr uint32_t kLargestBits = sizeof(T) == 4 ? 0x7f7fffffu : std::is_same_v<T, half_t> ? 0x7bffu : 0x7f7fu;
};
struct __attribute__((packed, aligned(2))) Words16 {
    uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) Words32 {
    uint32_t w[8];
};

// Entries at .. at + 7 of a row; -inf behind its end
template <typename T> __device__ __forceinline__ void load_run(const T *row, int at, int vocab, Run<T> &x)
{
    if (at + 8 <= vocab) {
        const auto r = *(const std::conditional_t<sizeof(T) == 4, Words32, Words16> *)(row + at);
#pragma unroll
        for (int i = 0; i < Run<T>::WORDS; ++i) x.w[i] = r.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < Run<T>::WORDS; ++i) x.w[i] = Run<T>::kMinusInf * (sizeof(T) == 4 ? 1u : 0x10001u);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < vocab) {
                const T v = row[at + e];
                if constexpr (sizeof(T) == 4) x.set(e, true, __float_as_uint(v));
                else x.set(e, true, *(const uint16_t *)&v);
            }
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
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
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
__device__ __forceinline__ int lanes_min(int x)
{
    auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const int y = from_lane<decltype(ctrl)::value, decltype(rows)::value>(x, kNone);
        x = y < x ? y : x;
    };
    step(Const<0x111>{}, Const<0xf>{});
    step(Const<0x112>{}, Const<0xf>{});
    step(Const<0x114>{}, Const<0xf>{});
    step(Const<0x118>{}, Const<0xf>{});
    step(Const<0x142>{}, Const<0xa>{});
    step(Const<0x143>{}, Const<0xc>{});
    return __builtin_amdgcn_readlane(x, 63);
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

// The kernel's arguments, read where they are needed: held in scalar registers from the start, as the compiler would have it, they
// leave too few for the polynomial's coefficients, which then take vector registers.
typedef const __attribute__((address_space(4))) SampleArgs *ArgsHere;
__device__ __forceinline__ ArgsHere args_here()
{
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return (ArgsHere)p;
}

// add(r, w): the weights of a thread's entries, in order, four at a time of run r
template <typename R, int RUNS, typename F>
__device__ __forceinline__ void each_four(R (&runs)[RUNS], double top, double heat, const F &add)
{
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        runs[r].stay_packed();
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const float l[4] = {runs[r].entry(h), runs[r].entry(h + 1), runs[r].entry(h + 2), runs[r].entry(h + 3)};
            double w[4];
            weights(l, top, heat, w);
            add(r, w);
        }
    }
}
// residual(r, v): max(p - a q, 0) of the same, and the weights of q
template <typename P, typename Q, int RUNS, typename F>
__device__ __forceinline__ void each_four(P (&x)[RUNS], Q (&y)[RUNS], double top, double heat, double draft_top, double draft_heat, double per_total,
                                          double takes, const F &add)
{
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        x[r].stay_packed();
        y[r].stay_packed();
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const float l[4] = {x[r].entry(h), x[r].entry(h + 1), x[r].entry(h + 2), x[r].entry(h + 3)};
            const float m[4] = {y[r].entry(h), y[r].entry(h + 1), y[r].entry(h + 2), y[r].entry(h + 3)};
            double v[4], w[4];
            weights(l, top, heat, v);
            weights(m, draft_top, draft_heat, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_fmax(__builtin_fma(-takes, w[i], v[i] * per_total), 0.0);
            add(r, v, w);
        }
    }
}
// A sum that is worked out here, and not where it is used
__device__ __forceinline__ void add_four(double &sum, const double (&w)[4])
{
    sum += (w[0] + w[1]) + (w[2] + w[3]);
    asm volatile("" : "+v"(sum));
}

// The walk is a sequence of passes over a slice (over all of them, one after the other, where a workgroup is alone): the weights of a node's
// rows and their sums; the sums of max(p - a q, 0) after a refusal; the search for the next token.
enum Pass { kRows, kResidual, kDraw };

template <typename TT, typename TD, int EPT>
__global__ void __launch_bounds__(NT, 4)
tree_sample_kernel(SampleArgs)
{
    const ArgsHere a = args_here();
    constexpr int RUNS = EPT / 8;  // a thread's entries: runs of 8, the lanes' runs side by side; a wave's are contiguous
    constexpr int SLICE = NT * EPT;
    static_assert(LS_MAX_TREE <= NT, "a thread per node");
    __shared__ int32_t tok[LS_MAX_TREE], path[LS_MAX_TREE], has_kids[LS_MAX_TREE];
    __shared__ float accept_u[LS_MAX_TREE], kid_x[LS_MAX_TREE], kid_y[LS_MAX_TREE];  // kid: logits of both models
    __shared__ double new_logit[LS_MAX_TREE], new_total[LS_MAX_TREE];  // of the new tokens: logit / temperature below the largest, and the sum of the weights
    __shared__ uint64_t kid_mask[LS_MAX_TREE / kWave];
    __shared__ float wave_top[2][WAVES];
    __shared__ double wave_sum[2][WAVES];
    __shared__ int32_t wave_best[WAVES];
    // of the slices: largest entry, sum of the weights relative to it, and where the largest of p is first; then the sums of max(p - a q, 0) and of q
    __shared__ float part_top[2][kSampleSlices];
    __shared__ double part_sum[2][kSampleSlices];
    __shared__ int32_t part_best[kSampleSlices];
    __shared__ int32_t first_sh, heard_sh[2];

    const int b = (int)(blockIdx.x / (uint32_t)a->slices), tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    Exchange ex;
    ex.slices = a->slices, ex.slice = (int)(blockIdx.x % (uint32_t)a->slices), ex.spin_limit = a->spin_limit, ex.number = 0;
    ex.state = a->records + (int64_t)b * (2 * a->slices + 1) * kRecordWords;
    ex.records = ex.state + kRecordWords;
    bool alone = false;  // this workgroup does all slices
    const bool told = a->slices > 1;
    // node's rows of logits
    auto target_row = [&](int node) __attribute__((always_inline)) {
        const ArgsHere h = args_here();
        return (const TT *)h->target + b * h->t_stride[0] + node * h->t_stride[1];
    };
    auto draft_row = [&](int node) __attribute__((always_inline)) {
        const ArgsHere h = args_here();
        return (const TD *)h->draft + b * h->d_stride[0] + node * h->d_stride[1];
    };

    // thread i has node i
    const bool is_node = tid < a->n_tree;
    int my_parent = -1, my_tok = -1, bad = 0;
    if (is_node) {
        my_parent = a->parents[(int64_t)b * a->n_tree + tid];
        my_tok = a->draft_tokens[(int64_t)b * a->n_tree + tid];
        accept_u[tid] = a->accept_uniforms[(int64_t)b * a->n_tree + tid];
        tok[tid] = my_tok;
        path[tid] = tid == 0 ? 0 : -1;
        has_kids[tid] = 0;
        if (my_parent < -1 || my_parent >= tid) bad = 1, my_parent = -1;
        if ((uint32_t)my_tok >= (uint32_t)a->vocab) my_parent = -1;  // nobody's child
    }
    if (tid == 0) heard_sh[0] = 0, heard_sh[1] = told && __hip_atomic_load(ex.state, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0;
    __syncthreads();
    if (bad) heard_sh[0] = 1;
    if (my_parent >= 0) has_kids[my_parent] = 1;
    __syncthreads();
    int err = uniform(heard_sh[0]);
    if (uniform(heard_sh[1])) return;  // somebody walks alone already

    float temp = a->temperature[b], draft_temp = a->draft_temperature ? a->draft_temperature[b] : temp;
    if (!(temp >= 0.f && temp <= FLT_MAX)) err |= 2, temp = 0.f;
    if (!(draft_temp >= 0.f && draft_temp <= FLT_MAX)) err |= 2, draft_temp = 0.f;
    const bool greedy = temp == 0.f;
    const bool drawn = a->draft && !greedy && draft_temp > 0.f;
    const double heat = uniform(1.4426950408889634074 / (greedy ? 1.0 : (double)temp));
    const double draft_heat = uniform(drawn ? 1.4426950408889634074 / (double)draft_temp : 0.0);

    Pass pass = kRows;
    int cur = 0, len = 1, next = -1;
    int writer = 0;                     // the slice whose workgroup draws the token and writes the outputs
    bool inner = false;                 // the node has children, and what they were drawn from counts
    float wt = 0.f, wq = 0.f;           // the wave's largest entries
    float top = 0.f, draft_top = 0.f;   // the largest of the rows
    double total = 0, per_total = 0, per_draft_total = 0;  // sum of the weights relative to it; inverse sums
    double part = 0;                    // lane i: slice i's share of `mass`
    double taken = 0, mass = 1, left = 1;  // a, S, W
    double rest = 0;                    // what the sum has to pass in the writer's slice
    int refused = 0, removed = 0;       // the children before these nodes have been refused, and taken out of the rows
    Run<TT> x[RUNS];
    Run<TD> y[RUNS];

    const int own = wave * (kWave * EPT) + lane * 8;  // this thread's first entry in a slice

    while (true) {
        float my_x = -INFINITY, my_y = -INFINITY;  // this thread's node is a child: its token's logits
        const bool kid = my_parent == cur && tid > cur;
        if (pass == kRows) {
            inner = drawn && uniform(has_kids[cur]);
            if (kid) {
                my_x = entry_of(target_row(cur), my_tok);
                if (inner) my_y = entry_of(draft_row(cur), my_tok);
            }
            taken = 0, mass = left = 1;
            refused = 0;
        }
        ++ex.number;
        bool heard = true;
        int slice = alone ? 0 : ex.slice, end = alone ? a->slices : ex.slice + 1;
        if (pass == kDraw) slice = writer, end = writer + 1;
        for (; slice < end && heard; ++slice) {
            if (pass == kRows || alone) {
                const TT *row = target_row(cur);
                const int at = slice * SLICE + own;
#pragma unroll
                for (int r = 0; r < RUNS; ++r) load_run(row, at + r * kWave * 8, a->vocab, x[r]);
                if (inner) {
                    const TD *drow = draft_row(cur);
#pragma unroll
                    for (int r = 0; r < RUNS; ++r) load_run(drow, at + r * kWave * 8, a->vocab, y[r]);
                }
                // the largest entries; +inf counts as the largest finite number (of its type), which is what it is from here on
                auto largest = [&](auto &runs) __attribute__((always_inline)) {
                    float m = -INFINITY;
#pragma unroll
                    for (int r = 0; r < RUNS; ++r) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) m = fmaxf(m, runs[r].entry(e));
                        runs[r].stay_packed();
                    }
                    m = lanes_max(m);
                    if (m == INFINITY) {
                        m = -INFINITY;
#pragma unroll
                        for (int r = 0; r < RUNS; ++r)
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                runs[r].set(e, runs[r].entry(e) == INFINITY, runs[r].kLargestBits);
                                m = fmaxf(m, runs[r].entry(e));
                            }
                        m = lanes_max(m);
                    }
                    return m;
                };
                wt = largest(x);
                wq = inner ? largest(y) : -INFINITY;
                removed = 0;
            }
            // refused tokens have no weight any more
            if (pass != kRows) {
                for (int w = removed / kWave; w * kWave < refused; ++w)
                    for (uint64_t m = uniform(kid_mask[w]); m; m &= m - 1) {
                        const int k = w * kWave + __builtin_ctzll(m);
                        if (k >= refused) break;
                        const int at = __builtin_amdgcn_readfirstlane(tok[k] - slice * SLICE - wave * (kWave * EPT));
                        if (k < removed || (uint32_t)at >= (uint32_t)(kWave * EPT)) continue;
                        const bool my_run = lane == (at >> 3) % kWave;
#pragma unroll
                        for (int r = 0; r < RUNS; ++r) {
                            if (r != at / (8 * kWave)) continue;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                x[r].set(e, my_run && e == at % 8, x[r].kMinusInf);
                                if (inner) y[r].set(e, my_run && e == at % 8, y[r].kMinusInf);
                            }
                        }
                    }
                removed = refused;
            }
            if (pass == kDraw) break;
            // sums over the thread, the wave, the slice (in waves 0 and 1); then to everybody
            double s = 0, sq = 0;
            if (pass == kRows) {  // of the weights relative to the wave's largest entries
                each_four(x, wt, heat, [&](int, const double (&w)[4]) __attribute__((always_inline)) { add_four(s, w); });
                if (inner) each_four(y, wq, draft_heat, [&](int, const double (&w)[4]) __attribute__((always_inline)) { add_four(sq, w); });
            } else if (inner) {   // of max(p - a q, 0), and of q
                each_four(x, y, top, heat, draft_top, draft_heat, per_total, taken * per_draft_total,
                          [&](int, const double (&v)[4], const double (&w)[4]) __attribute__((always_inline)) { add_four(s, v), add_four(sq, w); });
                sq *= per_draft_total;
            } else {
                each_four(x, top, heat, [&](int, const double (&w)[4]) __attribute__((always_inline)) { add_four(s, w); });
                s *= per_total;
            }
            s = lanes_sum(s);
            if (inner) sq = lanes_sum(sq);
            if (greedy && pass == kRows) {
                int best = kNone;
                const int at = slice * SLICE + own;
#pragma unroll
                for (int r = RUNS - 1; r >= 0; --r)
#pragma unroll
                    for (int e = 7; e >= 0; --e)
                        if (x[r].entry(e) == wt) best = at + r * kWave * 8 + e;
                best = wt > -INFINITY ? lanes_min(best) : kNone;
                if (lane == 0) wave_best[wave] = best;
            }
            if (lane == 0) {
                wave_top[0][wave] = wt, wave_sum[0][wave] = s;
                wave_top[1][wave] = wq, wave_sum[1][wave] = sq;
            }
            __syncthreads();
            if (pass == kRows) {
                const uint64_t kids = __ballot(kid);
                if (lane == 0) kid_mask[wave] = kids;
                if (kid) kid_x[tid] = my_x, kid_y[tid] = my_y;
            }
            if (wave == 0 || (wave == 1 && inner)) {
                const bool mine = lane < WAVES;
                double sum = mine ? wave_sum[wave][lane] : 0.0;
                float mm = 0.f;
                int best = kNone;
                if (pass == kRows) {
                    const float m = mine ? wave_top[wave][lane] : -INFINITY;
                    mm = lanes_max(m);
                    sum *= weight(m, mm, wave ? draft_heat : heat);
                    if (greedy) best = lanes_min(mine && m == mm ? wave_best[lane] : kNone);
                }
                sum = lanes_sum(sum);
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
                    if (lane < a->slices) {
                        part_top[wave][lane] = __uint_as_float(value[0]);
                        part_sum[wave][lane] = from_words(value[1], value[2]);
                        if (wave == 0) part_best[lane] = (int)value[3];
                    }
                    if (lane == 0) heard_sh[wave] = all;
                }
            }
            __syncthreads();
            heard = uniform(heard_sh[0]) && (!inner || uniform(heard_sh[1]));
        }

        if (!heard) {  // the first one to give up goes on alone, from the root
            if (tid == 0) {
                unsigned long long expected = 0;
                first_sh = __hip_atomic_compare_exchange_strong((unsigned long long *)ex.state, &expected, 1ull, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                                                __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (!uniform(first_sh)) return;
            alone = true;
            pass = kRows;
            cur = 0, len = 1;
            path[tid] = tid == 0 ? 0 : -1;
            __syncthreads();
            continue;
        }

        if (pass == kDraw) {
            // The first entry at which the sum of max(p - a q, 0) passes `rest`: its wave, run, lane, place.  Where roundings let none pass, the last one
            // that has any weight.
            const double takes = inner ? taken * per_draft_total : 0.0;
            double run[RUNS], all = 0;
#pragma unroll
            for (int r = 0; r < RUNS; ++r) run[r] = 0;
            if (inner)
                each_four(x, y, top, heat, draft_top, draft_heat, per_total, takes,
                          [&](int r, const double (&v)[4], const double (&)[4]) __attribute__((always_inline)) { add_four(run[r], v); });
            else
                each_four(x, top, heat, [&](int r, const double (&w)[4]) __attribute__((always_inline)) { add_four(run[r], w); });
#pragma unroll
            for (int r = 0; r < RUNS; ++r) {
                run[r] = lanes_sum(inner ? run[r] : run[r] * per_total);
                all += run[r];
            }
            if (lane == 0) wave_sum[0][wave] = all;
            if (tid == 0) first_sh = -1;
            __syncthreads();
            double before = 0, upto = 0;  // of the entries before the wave's; before what has been looked at
            int at_wave = -1;
            bool passed = false;
            for (int w = 0; w < WAVES && !passed; ++w) {
                const double sum = uniform(wave_sum[0][w]);
                if (sum > 0) at_wave = w, before = upto, passed = upto + sum > rest;
                upto += sum;
            }
            if (wave == at_wave) {
                upto = before;
                passed = false;
                int at_run = 0;
                Run<TT> rx = x[0];
                Run<TD> ry = y[0];
#pragma unroll
                for (int r = 0; r < RUNS; ++r) {
                    if (run[r] > 0 && !passed) {
                        rx = x[r], ry = y[r];
                        at_run = r, before = upto, passed = upto + run[r] > rest;
                    }
                    upto += run[r];
                }
                double v[8], sum = 0;
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    const float l[4] = {rx.entry(h), rx.entry(h + 1), rx.entry(h + 2), rx.entry(h + 3)};
                    double w[4];
                    weights(l, top, heat, w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[h + i] = w[i] * per_total;
                }
                if (inner)
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const float l[4] = {ry.entry(h), ry.entry(h + 1), ry.entry(h + 2), ry.entry(h + 3)};
                        double w[4];
                        weights(l, draft_top, draft_heat, w);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[h + i] = __builtin_fmax(__builtin_fma(-takes, w[i], v[h + i]), 0.0);
                    }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[e];
                const double scan = lanes_scan(sum);
                const uint64_t some = __ballot(sum > 0), over = __ballot(sum > 0 && before + scan > rest);
                if (lane == (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some))) {
                    double c = before + (scan - sum);
                    int place = 0;
                    passed = false;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        c += v[e];
                        if (v[e] > 0 && !passed) place = e, passed = c > rest;
                    }
                    first_sh = writer * SLICE + own + at_run * kWave * 8 + place;
                }
            }
            __syncthreads();
            next = uniform(first_sh);
            break;
        }

        // What the sums say
        const bool mine = lane < a->slices;
        part = mine ? part_sum[0][lane] : 0.0;
        int best = kNone;
        if (pass == kRows) {
            const float m = mine ? part_top[0][lane] : -INFINITY;
            top = lanes_max(m);
            part *= weight(m, top, heat);
            total = lanes_sum(part);
            per_total = uniform(total > 0 ? 1.0 / total : 0.0);
            if (greedy && total > 0) best = lanes_min(mine && m == top ? part_best[lane] : kNone);
            part *= per_total;
            if (inner) {
                const float mq = mine ? part_top[1][lane] : -INFINITY;
                draft_top = lanes_max(mq);
                const double draft_total = lanes_sum(mine ? part_sum[1][lane] * weight(mq, draft_top, draft_heat) : 0.0);
                per_draft_total = uniform(draft_total > 0 ? 1.0 / draft_total : 0.0);
            }
        }
        mass = lanes_sum(part);
        if (pass == kResidual && inner && !args_here()->with_replacement) left = lanes_sum(mine ? part_sum[1][lane] : 0.0);

        // the children that have not been tried
        int found = -1;
        bool again = false;
        for (int w = refused / kWave; w < LS_MAX_TREE / kWave && found < 0 && !again; ++w) {
            uint64_t m = uniform(kid_mask[w]);
            if (w == refused / kWave) m &= ~0ull << (refused % kWave);
            for (; m && found < 0 && !again; m &= m - 1) {
                const int k = w * kWave + __builtin_ctzll(m);
                bool ok;
                if (greedy) {
                    ok = tok[k] == best;
                } else {
                    const double px = weight(kid_x[k], top, heat) * per_total, u = accept_u[k];
                    if (inner) {
                        const double qx = weight(kid_y[k], draft_top, draft_heat) * per_draft_total;
                        ok = (px - taken * qx) * left > u * qx * mass;
                    } else {
                        ok = px > u * mass;
                    }
                }
                ok = uniform((int)ok);
                if (ok) found = k;
                else refused = k + 1, again = !greedy;
            }
        }
        if (found >= 0) {
            if (tid == 0) path[len] = found, new_logit[len - 1] = ((double)kid_x[found] - top) / (greedy ? 1.0 : (double)temp), new_total[len - 1] = total;
            ++len;
            cur = found;
            pass = kRows;
            continue;
        }
        if (again) {
            if (inner) taken = uniform(left > 0 ? fmin(taken + mass / left, 1e300) : 1e300);  // (finite: q(v) = 0 stays out of it)
            // the same token once more has no weight either
            if (kid && tid >= refused && my_tok == tok[refused - 1]) kid_x[tid] = kid_y[tid] = -INFINITY;
            pass = kResidual;
            continue;
        }
        // the path ends here
        if (greedy) {
            next = best == kNone ? -1 : best;
        } else if (mass > 0) {
            const double upto = lanes_scan(part), point = (double)args_here()->sample_uniforms[b] * mass;
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
            const float l = entry_of(target_row(cur), next);
            new_logit[len - 1] = ((double)l - top) / (greedy ? 1.0 : (double)temp), new_total[len - 1] = total;
        } else {
            new_logit[len - 1] = -INFINITY, new_total[len - 1] = 1.0;
            err |= 4;
        }
        const ArgsHere h = args_here();
        h->len[b] = len;
        h->next[b] = next;
        if (h->err_flag) h->err_flag[b] = err;
    }
    __syncthreads();
    const ArgsHere h = args_here();
    if (tid < h->n_tree) {
        const int64_t at = (int64_t)b * h->n_tree + tid;
        h->path[at] = path[tid];
        if (h->logprobs) h->logprobs[at] = tid < len ? (float)(new_logit[tid] - log(new_total[tid])) : 0.f;
    }
}

template <typename TT, typename TD> hipError_t launch_types(const SampleArgs &a, hipStream_t stream)
{
    const dim3 grid((uint32_t)a.batch * a.slices), block(NT);
    if (a.slice == NT * 8) hipLaunchKernelGGL((tree_sample_kernel<TT, TD, 8>), grid, block, 0, stream, a);
    else if (a.slice == NT * 16) hipLaunchKernelGGL((tree_sample_kernel<TT, TD, 16>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((tree_sample_kernel<TT, TD, 32>), grid, block, 0, stream, a);
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
