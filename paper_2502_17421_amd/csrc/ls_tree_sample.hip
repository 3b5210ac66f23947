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
// A sequence belongs to a group of workgroups, one per slice of the vocabulary, which walk its tree together: each reads its slice of both rows into
// LDS, as they are stored (weights as doubles would take four times the room, and let one workgroup on a compute unit where these let four), and works out the weights
// anew in each pass over it; it tells the others its sums, and the first wave of each decides what all of them decide, from all sums in the
// same order.  See Exchange.
//
// What bounds it: one request and few trees, the passes' chain: each waits for a row (1 us), its sums, the others' sums (1 us) and the decision (1.5 us).
// One request, 22 nodes of 32000 in half: 22 to 28 us by how far its path goes (one workgroup by itself 189).  Four beam trees of 69 nodes of 32000 in float 17 to 23.
// Many requests, the weights: 18 instructions of 64 bits each, 2 ns for a wave on a SIMD, and waits that four workgroups on a compute unit do not all cover.  48 chains
// of 5 tokens over 128256 in bf16: 87 to 91 us, of which the vector ALUs are busy 45 to 50 (107 MB: 21 us at the rate of a copy); 16 trees over 152064: 58 to 73 us.  The walk
// of a group and that of a workgroup alone are code of their own, from one source; together they spill 75 to 80 scalar registers, into lanes of vector
// registers and never to memory.
// Tried, and not faster than the form of the time: the next child's rows asked for ahead (chains 95.0 us for 93.4), two polls in flight (16 trees 73.5 for
// 69.8), eight weights of a thread at a time (chains 116 for 98).
#include <float.h>

#include <type_traits>

#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = kSampleThreads;
constexpr int WAVES = NT / kWave;
constexpr int kNone = INT32_MAX;
constexpr int RUN = 4;  // entries that a thread takes at a time
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

// The same of a run, step by step, so that no step waits for the one before it.  (Left to itself the compiler takes one after the other, or starts
// all of a thread's at once and runs out of registers.)
__device__ __forceinline__ void weights(const float (&logit)[RUN], double top, double heat, double (&w)[RUN])
{
    double n[RUN], f[RUN];
#define LS_STEP(...)                        \
    _Pragma("unroll") for (int i = 0; i < RUN; ++i) __VA_ARGS__; \
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

// Four entries of a row as they are stored
template <typename T> struct Run {
    static constexpr int WORDS = RUN * sizeof(T) / 4;
    alignas(16) uint32_t w[WORDS];
    __device__ __forceinline__ float entry(int e) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        const uint32_t u = w[e / 2];
        if constexpr (std::is_same_v<T, half_t>) return half_to_float((uint16_t)(e & 1 ? u >> 16 : u));
        else return __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void entries(float (&l)[RUN]) const
    {
#pragma unroll
        for (int e = 0; e < RUN; ++e) l[e] = entry(e);
    }
};
struct __attribute__((packed, aligned(2))) Words16 {
    uint32_t w[2];
};
struct __attribute__((packed, aligned(4))) Words32 {
    uint32_t w[4];
};
template <typename T> __device__ __forceinline__ Run<T> run_of_row(const T *at)  // (any alignment)
{
    Run<T> x;
    const auto r = *(const std::conditional_t<sizeof(T) == 4, Words32, Words16> *)at;
#pragma unroll
    for (int i = 0; i < Run<T>::WORDS; ++i) x.w[i] = r.w[i];
    return x;
}
template <typename T> __device__ __forceinline__ Run<T> run_of_lds(const T *at)
{
    Run<T> x;
    using W = std::conditional_t<sizeof(T) == 4, uint4, uint2>;
    *(W *)x.w = *(const W *)at;
    return x;
}
template <typename T> __device__ __forceinline__ void run_to_lds(const Run<T> &x, T *at)
{
    using W = std::conditional_t<sizeof(T) == 4, uint4, uint2>;
    *(W *)at = *(const W *)x.w;
}
template <typename T> __device__ __forceinline__ T from_bits(uint32_t bits)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
    else if constexpr (std::is_same_v<T, half_t>) return half_t{(uint16_t)bits};
    else return (T)bits;
}
template <typename T> __device__ __forceinline__ T minus_inf() { return from_bits<T>(sizeof(T) == 4 ? 0xff800000u : std::is_same_v<T, half_t> ? 0xfc00u : 0xff80u); }
template <typename T> __device__ __forceinline__ T largest_bits() { return from_bits<T>(sizeof(T) == 4 ? 0x7f7fffffu : std::is_same_v<T, half_t> ? 0x7bffu : 0x7f7fu); }

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
// Sums and largest values of all lanes: rotations within rows of 16, then the four rows'
template <int BY> __device__ __forceinline__ int rotated(int x)  // by BY lanes of the row
{
    return __builtin_amdgcn_update_dpp(x, x, 0x120 + BY, 0xf, 0xf, false);
}
template <int BY> __device__ __forceinline__ double rotated(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)rotated<BY>((int)(u >> 32)) << 32 | (uint32_t)rotated<BY>((int)u));
}
__device__ __forceinline__ double lanes_sum(double x)
{
    x += rotated<8>(x);
    x += rotated<4>(x);
    x += rotated<2>(x);
    x += rotated<1>(x);
    return (of_lane(x, 0) + of_lane(x, 16)) + (of_lane(x, 32) + of_lane(x, 48));
}
__device__ __forceinline__ float lanes_max(float x)
{
    x = fmaxf(x, __int_as_float(rotated<8>(__float_as_int(x))));
    x = fmaxf(x, __int_as_float(rotated<4>(__float_as_int(x))));
    x = fmaxf(x, __int_as_float(rotated<2>(__float_as_int(x))));
    x = fmaxf(x, __int_as_float(rotated<1>(__float_as_int(x))));
    auto row = [&](int lane) __attribute__((always_inline)) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); };
    return fmaxf(fmaxf(row(0), row(16)), fmaxf(row(32), row(48)));
}
// The same over WAVES neighbouring lanes, in all of these: of the lane next to it, of two lanes on
__device__ __forceinline__ double waves_sum(double x)
{
    x += from_lane<0xb1, 0xf>(x);
    x += from_lane<0x4e, 0xf>(x);
    return x;
}
__device__ __forceinline__ float waves_max(float x)
{
    auto step = [&](auto ctrl) __attribute__((always_inline)) {
        x = fmaxf(x, __int_as_float(from_lane<decltype(ctrl)::value, 0xf>(__float_as_int(x), __float_as_int(-INFINITY))));
    };
    step(Const<0xb1>{});
    step(Const<0x4e>{});
    return x;
}
// 1 / x to the last bit or two, for x of the size of such sums
__device__ __forceinline__ double inverse(double x)
{
    double r = __builtin_amdgcn_rcp(x);
    r = __builtin_fma(__builtin_fma(-x, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-x, r, 1.0), r, r);
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

// What the workgroups of a group tell each other: per exchange a record each, half of it about p and half about q, of four 32-bit values with a
// tag each in the upper half of 64 bits.  A word is written and read at once, so its tag says that its value is there, and no fence is needed; two
// sets of records take turns, since nobody is at exchange n + 2 before everybody has read those of n.
//
// Tags are the halves of a 64-bit number of the call's own, in turns, plus the number of the exchange; that of a half record's last word with a checksum of its
// values.  What the workspace held before does not pass for a record (with a chance of 2^-64).  A graph that is replayed has the same number again, so no record
// may be there when a launch ends:
// - Whoever writes the outputs clears all records at the end, once the others have left their marks that they have read all they need.
// - Whoever gives up on the group clears its own first of all, so that what it has told late does not stay.
// That is enough.  A workgroup that gets to the end with the group, and does not write, has heard the others in its last exchange after it has told them.  If
// the writer got there too, it has heard this one, and clears it.  If not, it gave up in that same exchange, and its record was heard before it cleared it; whoever
// walked alone for it cleared everything after that.  (Marks may stay, of late ones.  They let the writer of a replay clear too early; who has not
// read by then gives up and walks alone.)  A kernel that cleared the records beforehand took 5 us of each call.
//
// The workgroups of a group are next to each other in the launch, so that all of the first group that is not done yet are on the card, or
// will be when what else runs there is done.  No wait is unbounded all the same: who has polled spin_limit times gives up on
// the group, and the first of them (the state word says so) walks the tree alone, slice after slice, with the same sums in the same order.
// What it writes are the bits that the group writes if it gets to the end after all.
constexpr int kRecordWords = 8;  // of p: 0 largest entry, 1-2 sum, 3 where the largest is; 4-7 the same of q

struct Half {
    uint32_t value[4];
    __device__ __forceinline__ uint32_t check() const
    {
        return value[0] ^ value[1] * 0x85ebca6bu ^ value[2] * 0xc2b2ae35u ^ value[3] * 0x27d4eb2fu;
    }
};

struct Exchange {
    uint64_t *words;  // of the sequence: [8] state, [slices up to a multiple of 8] marks, [2][slices][kRecordWords] records
    int slices, slice;
    uint64_t call;
    uint32_t number;

    __device__ __forceinline__ uint64_t *marks() const { return words + 8; }
    __device__ __forceinline__ uint64_t *record(int of) const
    {
        return words + 8 + (slices + 7) / 8 * 8 + ((number & 1) * slices + of) * kRecordWords;
    }
    __device__ __forceinline__ int n_words() const { return 8 + (slices + 7) / 8 * 8 + 2 * slices * kRecordWords; }
    static __device__ __forceinline__ void put(uint64_t *at, uint64_t word)
    {
        __hip_atomic_store(at, word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    static __device__ __forceinline__ uint64_t get(const uint64_t *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

    __device__ __forceinline__ bool somebody_alone() const { return get(words) == call; }
    // true for the first one of the call
    __device__ __forceinline__ bool go_alone() const
    {
        unsigned long long now = get(words);
        while (now != call)
            if (__hip_atomic_compare_exchange_strong((unsigned long long *)words, &now, (unsigned long long)call, __ATOMIC_RELAXED,
                                                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
                return true;
        return false;
    }
    // lanes first .. first + 3 have the values of half `which`, lane by lane
    __device__ __forceinline__ void tell(int which, int lane_of_four, uint32_t value, uint32_t check) const
    {
        const uint32_t tag = ((lane_of_four & 1 ? (uint32_t)(call >> 32) : (uint32_t)call) + number) ^ (lane_of_four == 3 ? check : 0u);
        if (lane_of_four >= 0 && lane_of_four < 4) put(record(slice) + 4 * which + lane_of_four, (uint64_t)tag << 32 | value);
    }
    // (by the lanes that have told it) this workgroup's records, before anything that follows
    __device__ __forceinline__ void take_back(int lane) const
    {
        uint64_t *const mine = words + 8 + (slices + 7) / 8 * 8 + slice * kRecordWords + lane;
        if (lane < kRecordWords) put(mine, 0), put(mine + slices * kRecordWords, 0);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    }
    // lane i reads what slice i says (of q only if `both`); false: given up
    __device__ __forceinline__ bool hear(int lane, bool both, int spin_limit, Half &p, Half &q) const
    {
        const uint64_t *from = record(lane < slices ? lane : 0);
        const uint32_t tag = (uint32_t)call + number, odd_tag = (uint32_t)(call >> 32) + number;
        for (int poll = 0; poll < spin_limit; ++poll) {
            uint64_t word[8] = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) word[i] = get(from + i);
            if (both) {
#pragma unroll
                for (int i = 4; i < 8; ++i) word[i] = get(from + i);
            }
            bool there = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) p.value[i] = (uint32_t)word[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) there &= (uint32_t)(word[i] >> 32) == ((i & 1 ? odd_tag : tag) ^ (i == 3 ? p.check() : 0u));
            if (both) {
#pragma unroll
                for (int i = 0; i < 4; ++i) q.value[i] = (uint32_t)word[4 + i];
#pragma unroll
                for (int i = 0; i < 4; ++i) there &= (uint32_t)(word[4 + i] >> 32) == ((i & 1 ? odd_tag : tag) ^ (i == 3 ? q.check() : 0u));
            }
            if (__all(there)) return true;
            if ((poll & 15) == 15 && somebody_alone()) return false;
        }
        return false;
    }
    __device__ __forceinline__ void leave_mark() const { put(marks() + slice, call); }
    // (by a wave) the others' marks are there, or it has been long enough: then they find nothing and walk alone
    __device__ __forceinline__ void wait_for_marks(int lane, int spin_limit) const
    {
        for (int poll = 0; poll < spin_limit; ++poll)
            if (__all(lane >= slices || lane == slice || get(marks() + lane) == call)) return;
    }
};

__device__ __forceinline__ double from_words(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }

// A value that the compiler takes for a new one: it works out what follows from it where that is needed, and not before a loop for all its
// turns, where it would hold it in registers or even scratch.
__device__ __forceinline__ int here(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ int here_scalar(int x)
{
    asm volatile("" : "+s"(x));
    return x;
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

__device__ __forceinline__ double sum_of(const double (&w)[RUN]) { return (w[0] + w[1]) + (w[2] + w[3]); }

// The walk is a sequence of passes over a slice (over all of them, one after the other, where a workgroup is alone): the weights of a node's
// rows and their sums; the sums of max(p - a q, 0) after a refusal; the search for the next token.  Between two passes the first wave joins
// the sums of the waves, exchanges them with the group, and decides what comes next (all of it in Walk, in LDS).
enum Pass { kRows, kResidual, kDraw, kEnd, kGiveUp };

struct Walk {
    int32_t pass, cur, len, next, writer;  // writer: the slice whose workgroup draws the token and writes the outputs
    int32_t refused, removed, newest;      // the children before these nodes have been refused, and taken out of the rows in LDS; the last one's token
    float top, draft_top;                  // the largest entries of the rows
    double total;                          // the sum of the target's weights relative to its largest entry
    double per_total, per_draft_total;     // inverse sums
    double taken, mass, left;              // a, S, W
    double rest;                           // what the sum (of weights times the inverse sum) has to pass in the writer's slice
};

// What there is per node in LDS.  new_: of the path's n-th token in node n, its logit less the largest, and the sum of the weights.  kid_: the logits
// of both models at a child's token.
struct Node {
    double new_logit, new_total;
    int32_t tok, path, first_kid;
    float accept_u, kid_x, kid_y;
};
static_assert(sizeof(Node) == kSampleNode, "what the launch reserves");

template <typename TT, typename TD>
__global__ void __launch_bounds__(NT, 4)
tree_sample_kernel(SampleArgs)
{
    constexpr int NODES = LS_MAX_TREE / NT;  // of a thread: tid, tid + NT
    static_assert(WAVES == 4, "their sums are joined in as many lanes");
    // what there is per node, then the slice's entries of both rows
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ uint64_t kid_mask[LS_MAX_TREE / kWave];
    __shared__ float wave_top[2][WAVES];
    __shared__ double wave_sum[2][WAVES];
    __shared__ int32_t wave_best[WAVES];
    // of the slices, where there is no group: largest entries, sums, and where the largest of p is first
    __shared__ float part_top[2][kSampleSlices];
    __shared__ double part_sum[2][kSampleSlices];
    __shared__ int32_t part_best[kSampleSlices];
    __shared__ Walk walk;
    __shared__ int32_t flag_sh;

    const ArgsHere a = args_here();
    const int slices = a->slices, vocab = a->vocab;
    const int b = blockIdx.y, tid = threadIdx.x, wave = uniform(tid >> 6);
    Exchange ex;
    ex.slices = slices, ex.slice = blockIdx.x, ex.call = a->call, ex.number = 0;
    ex.words = a->records + (int64_t)b * ex.n_words();
    const int n_nodes = (a->n_tree + kWave - 1) / kWave * kWave, slice_size = a->slice;
    Node *const nodes = (Node *)lds;
    TT *const x_lds = (TT *)(nodes + n_nodes);
    TD *const y_lds = (TD *)(x_lds + slice_size);
    const bool told = slices > 1;
    // node's rows of logits
    const TT *const target = (const TT *)a->target + b * a->t_stride[0];
    const TD *const draft = (const TD *)a->draft + (a->draft ? b * a->d_stride[0] : 0);
    const int64_t t_node = a->t_stride[1], d_node = a->d_stride[1];
    auto target_row = [&](int node) __attribute__((always_inline)) { return target + node * t_node; };
    auto draft_row = [&](int node) __attribute__((always_inline)) { return draft + node * d_node; };
    int my_parent[NODES], my_tok[NODES];
    float my_u[NODES];
#pragma unroll
    for (int n = 0; n < NODES; ++n) {
        const int node = tid + n * NT;
        const int64_t at = (int64_t)b * a->n_tree + node;
        my_parent[n] = my_tok[n] = -1, my_u[n] = 0.f;
        if (node < a->n_tree) my_parent[n] = a->parents[at], my_tok[n] = a->draft_tokens[at], my_u[n] = a->accept_uniforms[at];
    }
    float temp = a->temperature[b], draft_temp = a->draft_temperature ? a->draft_temperature[b] : temp;
    bool bad = false;
#pragma unroll
    for (int n = 0; n < NODES; ++n) {
        const int node = tid + n * NT;
        if (node < n_nodes) nodes[node] = {0.0, 0.0, my_tok[n], node == 0 ? 0 : -1, kNone, my_u[n], 0.f, 0.f};
        if (my_parent[n] < -1 || my_parent[n] >= node) bad = true, my_parent[n] = -1;
        if ((uint32_t)my_tok[n] >= (uint32_t)vocab) my_parent[n] = -1;  // nobody's child
    }
    if (tid == 0) {
        flag_sh = 0;
        walk.pass = kRows, walk.cur = 0, walk.len = 1, walk.next = -1, walk.writer = 0;
    }
    __syncthreads();
    if (bad) flag_sh = 1;
#pragma unroll
    for (int n = 0; n < NODES; ++n)
        if (my_parent[n] >= 0) atomicMin(&nodes[my_parent[n]].first_kid, tid + n * NT);
    int err = 0;
    if (!(temp >= 0.f && temp <= FLT_MAX)) err = 2, temp = 0.f;
    if (!(draft_temp >= 0.f && draft_temp <= FLT_MAX)) err = 2, draft_temp = 0.f;
    const bool greedy = temp == 0.f;
    const bool drawn = a->draft && !greedy && draft_temp > 0.f;
    const double heat = 1.4426950408889634074 / (greedy ? 1.0 : (double)temp);
    const double draft_heat = drawn ? 1.4426950408889634074 / (double)draft_temp : 0.0;
    __syncthreads();
    err |= uniform(flag_sh);

    // A thread's entries: runs of 4, the lanes' runs side by side; a wave's are contiguous.  What a thread reads of its runs in LDS it has written itself.
    const int wave_size = slice_size / WAVES, runs = wave_size / (kWave * RUN);

    // The walk, over this workgroup's slice of each row, or over all of them.  false: given up
    auto walk_tree = [&](auto by_itself) __attribute__((always_inline)) {
        constexpr bool ALONE = decltype(by_itself)::value;
        int pass = kEnd;
        while (true) {
            const int lane = here(tid) & 63, own = wave * wave_size + lane * RUN;
            const bool summed = pass == kResidual;
            const int cur = uniform(walk.cur);
            pass = uniform(walk.pass);
            if (pass == kEnd) return true;
            if (pass == kGiveUp) return false;
            const int kid = uniform(nodes[cur].first_kid);
            const bool inner = drawn && kid != kNone;  // the node has children, and what they were drawn from counts
            if (!ALONE && pass == kDraw && uniform(walk.writer) != ex.slice) return true;
            const float top = walk.top, draft_top = walk.draft_top;
            const double per_total = walk.per_total, per_draft_total = walk.per_draft_total, takes = walk.taken * per_draft_total;
            int slice = ALONE ? 0 : ex.slice;
            const int end = ALONE ? slices : slice + 1;
            if (ALONE && pass == kDraw) slice = uniform(walk.writer);
            ++ex.number;
            float wt = -INFINITY, wq = -INFINITY;  // the wave's largest entries
            TT my_x[NODES];                        // logits of nodes that are children, as they are stored: asked for after the rows, and first looked at
            TD my_y[NODES];                        // when the sums of these are done
            do {
                const int lane = here(tid) & 63, own = wave * wave_size + lane * RUN;
                if (pass == kRows || ALONE) {
                    const TT *row = target_row(cur);
                    const TD *drow = inner ? draft_row(cur) : nullptr;
                    float m = -INFINITY, mq = -INFINITY;
                    auto fetch = [&](auto *from, auto *to, int at, float &most) __attribute__((always_inline)) {  // entries behind the row's end, one by one
                        using T = std::remove_reference_t<decltype(*to)>;
#pragma unroll 1
                        for (int e = 0; e < RUN; ++e) {
                            const T v = at + e < vocab ? from[at + e] : minus_inf<T>();
                            to[e] = v;
                            most = fmaxf(most, Elem<T>::load(&v));
                        }
                    };
#pragma unroll 1
                    for (int r0 = 0; r0 < runs; r0 += 4) {
                        Run<TT> x[4] = {};
                        Run<TD> y[4] = {};
                        const int at = slice * slice_size + own + r0 * kWave * RUN;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (r0 + i < runs && at + i * kWave * RUN + RUN <= vocab) x[i] = run_of_row(row + at + i * kWave * RUN);
                        if (inner)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (r0 + i < runs && at + i * kWave * RUN + RUN <= vocab) y[i] = run_of_row(drow + at + i * kWave * RUN);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (r0 + i < runs) {
                                const int in = own + (r0 + i) * kWave * RUN;
                                if (at + i * kWave * RUN + RUN <= vocab) {
                                    run_to_lds(x[i], x_lds + in);
#pragma unroll
                                    for (int e = 0; e < RUN; ++e) m = fmaxf(m, x[i].entry(e));
                                } else {
                                    fetch(row, x_lds + in, slice * slice_size + in, m);
                                }
                            }
                        if (inner)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (r0 + i < runs) {
                                    const int in = own + (r0 + i) * kWave * RUN;
                                    if (at + i * kWave * RUN + RUN <= vocab) {
                                        run_to_lds(y[i], y_lds + in);
#pragma unroll
                                        for (int e = 0; e < RUN; ++e) mq = fmaxf(mq, y[i].entry(e));
                                    } else {
                                        fetch(drow, y_lds + in, slice * slice_size + in, mq);
                                    }
                                }
                    }
#pragma unroll
                    for (int n = 0; n < NODES; ++n) {
                        my_x[n] = minus_inf<TT>(), my_y[n] = minus_inf<TD>();
                        if (pass == kRows && my_parent[n] == cur) {
                            my_x[n] = target_row(cur)[my_tok[n]];
                            if (inner) my_y[n] = draft_row(cur)[my_tok[n]];
                        }
                    }
                    // +inf counts as the largest finite number of its type, which is what it is from here on
                    auto whole = [&](auto *entries, float most) __attribute__((always_inline)) {
                        using T = std::remove_reference_t<decltype(*entries)>;
                        most = lanes_max(most);
                        if (most != INFINITY) return most;
                        most = -INFINITY;
#pragma unroll 1
                        for (int r = 0; r < runs; ++r)
#pragma unroll 1
                            for (int e = 0; e < RUN; ++e) {
                                T *const at = entries + own + r * kWave * RUN + e;
                                if (Elem<T>::load(at) == INFINITY) *at = largest_bits<T>();
                                most = fmaxf(most, Elem<T>::load(at));
                            }
                        return lanes_max(most);
                    };
                    wt = whole(x_lds, m);
                    wq = inner ? whole(y_lds, mq) : -INFINITY;
                }
                // refused tokens have no weight any more
                if (pass != kRows) {
                    auto remove = [&](int token) __attribute__((always_inline)) {
                        const int at = token - slice * slice_size, in_wave = at - wave * wave_size;
                        if ((uint32_t)in_wave < (uint32_t)wave_size && in_wave / RUN % kWave == lane) {
                            x_lds[at] = minus_inf<TT>();
                            if (inner) y_lds[at] = minus_inf<TD>();
                        }
                    };
                    if (pass == kResidual && inner && !ALONE) {
                        remove(walk.newest);
                    } else {
                        const int refused = uniform(walk.refused), removed = ALONE ? 0 :  // (the rows have been read again)
                            uniform(walk.removed);
                        for (int w = removed / kWave; w * kWave < refused; ++w) {
                            uint64_t m = uniform(kid_mask[w]);
                            if (w == removed / kWave) m &= ~0ull << (removed % kWave);
                            for (; m; m &= m - 1) {
                                const int k = w * kWave + __builtin_ctzll(m);
                                if (k >= refused) break;
                                remove(nodes[k].tok);
                            }
                        }
                    }
                }
                if (pass == kDraw) break;
                // sums over the thread and the wave: of the weights relative to the wave's largest entries, or of max(p - a q, 0) and of q
                double s = 0, sq = 0;
                auto sum_weights = [&](const auto *entries, double most, double h) __attribute__((always_inline)) {
                    double sum = 0;
#pragma unroll 1
                    for (int r = 0; r < runs; ++r) {
                        float l[RUN];
                        double w[RUN];
                        run_of_lds(entries + own + r * kWave * RUN).entries(l);
                        weights(l, most, h, w);
                        sum += sum_of(w);
                    }
                    return sum;
                };
                if (pass == kRows) {
                    s = sum_weights(x_lds, wt, heat);
                    if (inner) sq = sum_weights(y_lds, wq, draft_heat);
                } else if (inner) {
#pragma unroll 1
                    for (int r = 0; r < runs; ++r) {
                        float l[RUN];
                        double v[RUN], w[RUN];
                        run_of_lds(x_lds + own + r * kWave * RUN).entries(l);
                        weights(l, top, heat, v);
                        run_of_lds(y_lds + own + r * kWave * RUN).entries(l);
                        weights(l, draft_top, draft_heat, w);
#pragma unroll
                        for (int e = 0; e < RUN; ++e) v[e] = __builtin_fmax(__builtin_fma(-takes, w[e], v[e] * per_total), 0.0);
                        s += sum_of(v);
                        sq += sum_of(w);
                    }
                    sq *= per_draft_total;
                } else {
                    s = sum_weights(x_lds, top, heat) * per_total;
                }
                if (inner) sq = lanes_sum(sq);
                s = lanes_sum(s);
                if (pass == kRows) {
                    if (lane == 0) wave_top[0][wave] = wt, wave_top[1][wave] = wq;
                    if (greedy) {
                        int best = kNone;
#pragma unroll 1
                        for (int r = runs - 1; r >= 0; --r) {
                            const Run<TT> x = run_of_lds(x_lds + own + r * kWave * RUN);
#pragma unroll
                            for (int e = RUN - 1; e >= 0; --e)
                                if (x.entry(e) == wt) best = slice * slice_size + own + r * kWave * RUN + e;
                        }
                        best = wt > -INFINITY ? lanes_min(best) : kNone;
                        if (lane == 0) wave_best[wave] = best;
                    }
                }
                if (lane == 0) wave_sum[0][wave] = s, wave_sum[1][wave] = sq;
                if (pass == kRows) {
#pragma unroll
                    for (int n = 0; n < NODES; ++n) {
                        const bool is_kid = my_parent[n] == cur;
                        const uint64_t kids = __ballot(is_kid);
                        if (lane == 0) kid_mask[wave + n * WAVES] = kids;
                        if (is_kid) nodes[tid + n * NT].kid_x = entry_of(&my_x[n], 0), nodes[tid + n * NT].kid_y = entry_of(&my_y[n], 0);
                    }
                }
                __syncthreads();
                if (wave == 0) {
                    const int lane = here(tid) & 63, slices = here_scalar(ex.slices);  // (what follows from them is not worked out before,
                    // for every pass and wave)
                    // The waves' sums to the slice's: the first WAVES lanes have p's, the next ones q's
                    const bool mine = lane < 2 * WAVES;
                    const int which = lane / WAVES;
                    double sum = mine ? wave_sum[which][lane % WAVES] : 0.0;
                    float mm = 0.f;
                    int best = kNone;
                    if (pass == kRows) {
                        const float m = mine ? wave_top[which][lane % WAVES] : -INFINITY;
                        mm = waves_max(m);
                        sum *= weight(m, mm, which == 0 ? heat : draft_heat);
                        if (greedy) best = lanes_min(lane < WAVES && m == mm ? wave_best[lane] : kNone);
                    }
                    sum = waves_sum(sum);
                    Half p = {}, q = {};
                    if (ALONE) {
                        if (lane % WAVES == 0 && mine) {
                            part_top[which][slice] = mm, part_sum[which][slice] = sum;
                            if (lane == 0) part_best[slice] = best;
                        }
                        if (slice + 1 < end) goto next_slice;
                    } else {
                        const uint64_t bits = __builtin_bit_cast(uint64_t, sum);
                        Half own_half = {{__float_as_uint(mm), (uint32_t)bits, (uint32_t)(bits >> 32), (uint32_t)best}};
                        const int i = lane % WAVES;
                        const uint32_t value = i == 0 ? own_half.value[0] : i == 1 ? own_half.value[1] : i == 2 ? own_half.value[2] : own_half.value[3];
                        if (told) {
                            if (lane < (inner ? 2 : 1) * WAVES) ex.tell(which, i, value, own_half.check());
                            if (!ex.hear(lane, inner, args_here()->spin_limit, p, q)) {
                                if (lane == 0) walk.pass = kGiveUp;
                                goto next_slice;
                            }
                        } else {
                            p = own_half;
#pragma unroll
                            for (int k = 0; k < 4; ++k) q.value[k] = (uint32_t)__builtin_amdgcn_readlane((int)own_half.value[k], WAVES);
                        }
                    }
                    {
                        // What the sums say
                        const bool there = lane < slices;
                        float m = -INFINITY, mq = -INFINITY;
                        double part = 0, part_q = 0;
                        int part_b = kNone;
                        if (there) {
                            m = ALONE ? part_top[0][lane] : __uint_as_float(p.value[0]);
                            part = ALONE ? part_sum[0][lane] : from_words(p.value[1], p.value[2]);
                            part_b = ALONE ? part_best[lane] : (int)p.value[3];
                            if (inner) {
                                mq = ALONE ? part_top[1][lane] : __uint_as_float(q.value[0]);
                                part_q = ALONE ? part_sum[1][lane] : from_words(q.value[1], q.value[2]);
                            }
                        }
                        double taken = 0, left = 1, pt = per_total, pd = per_draft_total;
                        float t = top, dt = draft_top;
                        int at_best = kNone, refused = 0, newest = -1;
                        double mass = 1;
                        if (pass == kRows) {  // (both rows, step by step together, also where there is no draft's)
                            t = lanes_max(m), dt = lanes_max(mq);
                            part *= weight(m, t, heat), part_q *= weight(mq, dt, draft_heat);
                            const double total = lanes_sum(part), draft_total = lanes_sum(part_q);
                            pt = inverse(total), pd = inverse(draft_total);
                            pt = total > 0 ? pt : 0.0, pd = draft_total > 0 ? pd : 0.0;
                            part *= pt;
                            mass = total > 0 ? 1.0 : 0.0;
                            if (greedy && total > 0) at_best = lanes_min(there && m == t ? part_b : kNone);
                            if (lane == 0) walk.top = t, walk.draft_top = dt, walk.total = total, walk.per_total = pt, walk.per_draft_total = pd;
                        } else {
                            taken = walk.taken, refused = uniform(walk.refused);
                            const double q_left = lanes_sum(part_q);
                            mass = lanes_sum(part);
                            // (a draft whose tokens have all been refused has q = 0 for the others: 1 in place of the 0 that would hide it)
                            if (inner && !args_here()->with_replacement) left = q_left > 0 ? q_left : 1.0;
                        }

                        const double whole = part;

                        // The children that have not been tried.  Of tokens that were chosen the refused ones' probabilities are taken off the sums as long
                        // as much is left (then a pass over the rows makes the sums anew).
                        int found = -1;
                        bool again = false;
                        const int len = uniform(walk.len);
                        for (int w = refused / kWave; w * kWave < n_nodes && found < 0 && !again; ++w) {
                            uint64_t k = uniform(kid_mask[w]);
                            if (w == refused / kWave) k &= ~0ull << (refused % kWave);
                            if (!k) continue;
                            const int node = w * kWave + lane, my_token = nodes[node].tok;
                            const double u = nodes[node].accept_u;
                            const bool is_kid = k >> lane & 1;
                            double px = weight(is_kid ? nodes[node].kid_x : -INFINITY, t, heat) * pt, qx = weight(is_kid ? nodes[node].kid_y : -INFINITY, dt, draft_heat) * pd;
                            if (!inner) qx = 1.0;
                            for (; k && found < 0 && !again; k &= k - 1) {
                                const int i = __builtin_ctzll(k);
                                const int token = __builtin_amdgcn_readlane(my_token, i);
                                bool ok;
                                if (greedy) ok = token == at_best;
                                else ok = __ballot((px - (inner ? taken * qx : 0.0)) * left > u * qx * mass) >> i & 1;
                                if (ok) {
                                    found = w * kWave + i;
                                    break;
                                }
                                refused = w * kWave + i + 1, newest = token;
                                if (greedy) continue;
                                // the same token once more has no weight either
                                const bool same = my_token == token;
                                const double off = of_lane(px, i);
                                px = same ? 0.0 : px;
                                if (inner && same) qx = 0.0;
                                for (int v = w; v * kWave < n_nodes; ++v) {
                                    Node &other = nodes[v * kWave + lane];
                                    if (uniform(kid_mask[v]) >> lane & 1 && v * kWave + lane >= refused && other.tok == token) other.kid_x = other.kid_y = -INFINITY;
                                }
                                if (inner) {
                                    again = true;
                                } else {
                                    mass -= off;
                                    if ((uint32_t)(token - lane * slice_size) < (uint32_t)slice_size) part = __builtin_fmax(part - off, 0.0);
                                    again = mass < 0x1p-10;
                                }
                            }
                        }
                        int next_pass = kRows, writer = 0;
                        if (found >= 0) {
                            if (lane == 0) {
                                nodes[len].path = found;
                                nodes[len - 1].new_logit = (double)nodes[found].kid_x - t, nodes[len - 1].new_total = walk.total;
                                walk.len = len + 1, walk.cur = found;
                            }
                        } else if (again) {
                            if (inner && lane == 0) walk.taken = fmin(taken + mass / left, 1e300);  // (finite: q(v) = 0 stays out of it)
                            if (!inner && lane == 0) walk.taken = 0;
                            next_pass = kResidual;
                        } else {  // the path ends here
                            next_pass = kEnd;
                            int next = -1;
                            double rest = 0;
                            if (greedy) {
                                next = at_best == kNone ? -1 : at_best;
                            } else if (mass > 0) {
                                const double upto = lanes_scan(part), point = (double)args_here()->sample_uniforms[b] * mass;
                                const uint64_t passed = __ballot(part > 0 && upto > point), some = __ballot(part > 0);
                                if (some) {
                                    writer = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some);
                                    rest = point - of_lane(upto - part, writer);
                                    next_pass = kDraw;
                                    // Whether a slice has any weight at all is said by sums that are made after the refusals, of the weights that the draw looks
                                    // at (what is left of a sum that a refusal has been taken off may be a rounding of nothing, or 0 where something is left;
                                    // sums relative to other entries may be the least numbers there are without any weight being one).
                                    const bool made = pass == kResidual && refused == uniform(walk.refused);
                                    if (!inner && !made && (__any(part < whole * 0x1p-32) || of_lane(part, writer) < 0x1p-900)) next_pass = kResidual;
                                }
                            }
                            if (lane == 0) {
                                walk.next = next, walk.rest = rest, walk.writer = writer;
                                if (pass == kRows) walk.taken = 0;
                            }
                        }
                        if (lane == 0) {
                            walk.pass = next_pass;
                            walk.removed = pass == kRows ? 0 : uniform(walk.refused);
                            walk.refused = refused, walk.newest = newest;
                        }
                    }
                next_slice:;
                }
                __syncthreads();
            } while (ALONE && ++slice < end);
            if (pass != kDraw) continue;

            // The first entry at which the sum of max(p - a q, 0) passes `rest`: its wave, run, lane, place.  Where roundings let none pass, the last one
            // that has any weight.  Of the target's weights alone, which are summed as they are: a product with the inverse sum could round the least of them to 0.
            const double rest = inner ? walk.rest : walk.rest * walk.total;
            // the entries of a run, and their sum
            auto residual_run = [&](int r, double (&v)[RUN]) __attribute__((always_inline)) {
                float l[RUN];
                run_of_lds(x_lds + own + r * kWave * RUN).entries(l);
                weights(l, top, heat, v);
                if (inner) {
                    double w[RUN];
                    run_of_lds(y_lds + own + r * kWave * RUN).entries(l);
                    weights(l, draft_top, draft_heat, w);
#pragma unroll
                    for (int e = 0; e < RUN; ++e) v[e] = __builtin_fmax(__builtin_fma(-takes, w[e], v[e] * per_total), 0.0);
                }
                return sum_of(v);
            };
            double v[RUN], sum = 0;
            const bool sums_there = !ALONE && summed && inner;  // (those of the pass before)
            if (!sums_there) {
                double all = 0;
#pragma unroll 1
                for (int r = 0; r < runs; ++r) all += sum = residual_run(r, v);
                all = lanes_sum(all);
                if (lane == 0) wave_sum[0][wave] = all;
            }
            __syncthreads();
            double before = 0, upto = 0;  // of the entries before the wave's; before what has been looked at
            int at_wave = -1;
            bool passed = false;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const double of_wave = uniform(wave_sum[0][w]);
                if (of_wave > 0 && !passed) at_wave = w, before = upto, passed = upto + of_wave > rest;
                upto += of_wave;
            }
            if (wave == at_wave) {
                // runs in turn, until one passes; where roundings let none, the last that has any weight
                upto = before;
                int last_run = -1;
#pragma unroll 1
                for (int r = 0;; ++r) {
                    const bool again = r == runs;
                    if (again) r = last_run, upto = before;
                    if (again || runs > 1 || sums_there) sum = residual_run(r, v);
                    const double scan = lanes_scan(sum), of_run = of_lane(scan, 63);
                    if (!again && of_run > 0) last_run = r, before = upto;
                    const uint64_t over = __ballot(sum > 0 && upto + scan > rest), some = __ballot(sum > 0);
                    if (over || again) {
                        if (lane == (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some))) {
                            double c = upto + (scan - sum);
                            int place = 0;
                            passed = false;
#pragma unroll
                            for (int e = 0; e < RUN; ++e) {
                                c += v[e];
                                if (v[e] > 0 && !passed) place = e, passed = c > rest;
                            }
                            walk.next = uniform(walk.writer) * slice_size + own + r * kWave * RUN + place;
                        }
                        break;
                    }
                    upto += of_run;
                }
            }
            __syncthreads();
            return true;
        }
    };

    bool alone = false;
    if (!walk_tree(std::false_type{})) {  // the first one to give up goes on alone, from the root
        if (wave == 0) ex.take_back(tid);
        __syncthreads();
        if (tid == 0) {
            flag_sh = ex.go_alone();
            walk.pass = kRows, walk.cur = 0, walk.len = 1, walk.next = -1, walk.writer = 0;
        }
        for (int i = tid; i < n_nodes; i += NT) nodes[i].path = i == 0 ? 0 : -1;
        __syncthreads();
        if (!uniform(flag_sh)) return;
        alone = true;
        walk_tree(std::true_type{});
    }

    // The outputs
    const ArgsHere h = args_here();
    if (!alone && uniform(walk.writer) != ex.slice) {
        if (tid == 0) ex.leave_mark();
        return;
    }
    const int len = uniform(walk.len), next = uniform(walk.next);
    if (tid == 0) {
        if (next >= 0) {
            nodes[len - 1].new_logit = (double)entry_of(target_row(walk.cur), next) - walk.top;
            nodes[len - 1].new_total = walk.total;
        } else {
            nodes[len - 1].new_logit = -INFINITY, nodes[len - 1].new_total = 1.0;
            err |= 4;
        }
        h->len[b] = len;
        h->next[b] = next;
        if (h->err_flag) h->err_flag[b] = err;
    }
    __syncthreads();
    if (told && !alone && wave == WAVES - 1) ex.wait_for_marks(tid & 63, h->spin_limit);
    for (int i = tid; i < h->n_tree; i += NT) {
        const int64_t at = (int64_t)b * h->n_tree + i;
        h->path[at] = nodes[i].path;
        if (h->logprobs) h->logprobs[at] = i < len ? (float)(nodes[i].new_logit / (greedy ? 1.0 : (double)temp) - log(nodes[i].new_total)) : 0.f;
    }
    if (!told) return;
    __syncthreads();
    for (int i = tid; i < ex.n_words(); i += NT) Exchange::put(ex.words + i, 0);
}

template <typename TT, typename TD> hipError_t launch_types(const SampleArgs &a, hipStream_t stream)
{
    const int bytes = sample_lds_bytes(a.n_tree, a.slice, sizeof(TT), a.draft ? sizeof(TD) : 0);
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_dynamic_lds((const void *)tree_sample_kernel<TT, TD>, kSampleLds, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((tree_sample_kernel<TT, TD>), dim3(a.slices, a.batch), dim3(NT), bytes, stream, a);
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
    if (!a.draft) draft_dtype = target_dtype;
    if (target_dtype == LS_F32) return launch_for<float>(a, draft_dtype, stream);
    if (target_dtype == LS_F16) return launch_for<half_t>(a, draft_dtype, stream);
    return launch_for<uint16_t>(a, draft_dtype, stream);
}

}  // namespace ls
