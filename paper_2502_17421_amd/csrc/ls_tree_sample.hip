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
// One workgroup per sequence, which goes through the vocabulary in slices of 16 entries a thread.
#include <float.h>

#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = kSampleThreads;
constexpr int WAVES = NT / kWave;
constexpr int EPT = kSampleSlice / NT;  // entries of a thread
constexpr int RUNS = EPT / 8;           // in runs of 8, the lanes' runs side by side; a wave's entries are contiguous
constexpr int kNone = INT32_MAX;

// 2^y for y <= 0, to 1e-14 of its value: the Taylor series of exp(f ln 2), |f| <= 1/2, whose first term left out is
// (ln 2 / 2)^12 / 12! = 6e-15.
__device__ __forceinline__ double exp2_of(double y)
{
    if (y < -1000.0) return 0.0;  // (a lowest finite number that stands for a mask, say)
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

__device__ __forceinline__ double lanes_sum(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
    return v;
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
// Sums of the lanes up to this one, this one included
__device__ __forceinline__ double lanes_scan(double v, int lane)
{
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double y = __shfl_up(v, off, kWave);
        v += lane >= off ? y : 0.0;
    }
    return v;
}

template <typename TT, typename TD>
__global__ void __launch_bounds__(NT)
tree_sample_kernel(SampleArgs a)
{
    __shared__ int32_t tok[LS_MAX_TREE], path[LS_MAX_TREE], refused[LS_MAX_TREE];
    __shared__ float accept_u[LS_MAX_TREE], logp[LS_MAX_TREE], kid_logp[LS_MAX_TREE];
    __shared__ double kid_p[LS_MAX_TREE], kid_q[LS_MAX_TREE];
    __shared__ uint64_t kid_mask[LS_MAX_TREE / kWave];
    __shared__ float wave_top[2][WAVES];
    __shared__ double wave_sum[2][WAVES];
    __shared__ int32_t wave_best[WAVES];
    // of the slices: largest entry, sum of the weights relative to it, and where the largest of p is first; then the sums of max(p - a q, 0) and of q
    __shared__ float part_top[2][kSampleSlices];
    __shared__ double part_sum[2][kSampleSlices];
    __shared__ int32_t part_best[kSampleSlices];
    __shared__ int32_t found_sh, last_sh;
    static_assert(LS_MAX_TREE <= NT, "a thread per node");

    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const TT *target = (const TT *)a.target + b * a.t_stride[0];
    const TD *draft = (const TD *)a.draft + (a.draft ? b * a.d_stride[0] : 0);

    // thread i has node i
    const bool is_node = tid < a.n_tree;
    int my_parent = -1, bad = 0;
    if (is_node) {
        my_parent = a.parents[(int64_t)b * a.n_tree + tid];
        if (my_parent < -1 || my_parent >= tid) bad = 1, my_parent = -1;
        tok[tid] = a.draft_tokens[(int64_t)b * a.n_tree + tid];
        accept_u[tid] = a.accept_uniforms[(int64_t)b * a.n_tree + tid];
        logp[tid] = 0.f;
        path[tid] = tid == 0 ? 0 : -1;
    }
    int err = __syncthreads_or(bad) ? 1 : 0;
    const int my_tok = is_node ? tok[tid] : -1;
    const bool my_tok_ok = (uint32_t)my_tok < (uint32_t)a.vocab;

    float temp = a.temperature[b], draft_temp = a.draft_temperature ? a.draft_temperature[b] : temp;
    if (!(temp >= 0.f && temp <= FLT_MAX)) err |= 2, temp = 0.f;
    if (!(draft_temp >= 0.f && draft_temp <= FLT_MAX)) err |= 2, draft_temp = 0.f;
    const bool greedy = temp == 0.f;
    const bool drawn = a.draft && !greedy && draft_temp > 0.f;
    const double heat = 1.4426950408889634074 / (greedy ? 1.0 : (double)temp);
    const double draft_heat = drawn ? 1.4426950408889634074 / (double)draft_temp : 0.0;

    int cur = 0, len = 1, n_refused = 0;
    bool inner = false;  // the node has children, and what they were drawn from counts
    float top = 0.f, draft_top = 0.f;  // of the rows of p and q
    double total = 0, draft_total = 0; // of the weights relative to them
    double p[EPT], q[EPT];

    const int own = wave * (kWave * EPT) + lane * 8;  // this thread's first entry in a slice

    // The slice's weights into p and q: relative to the wave's largest entries, which are returned.
    auto load_slice = [&](int slice, float &wt, float &wq) __attribute__((always_inline)) {
        const TT *row = target + cur * a.t_stride[1];
        const int at = slice * kSampleSlice + own;
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
            for (int e = 0; e < 8; ++e) {
                m = fmaxf(m, x[r][e]);
                if (inner) mq = fmaxf(mq, y[r][e]);
            }
        int best = kNone;
        wt = lanes_max(m);
        if (greedy) {
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
            for (int e = 0; e < 8; ++e) p[r * 8 + e] = weight(x[r][e], wt, heat);
        if (inner) {
            wq = lanes_max(mq);
#pragma unroll
            for (int r = 0; r < RUNS; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) q[r * 8 + e] = weight(y[r][e], wq, draft_heat);
        }
    };

    // From weights relative to the wave's largest entry to probabilities, refused tokens at zero
    auto normalise = [&](int slice, float wt, float wq) __attribute__((always_inline)) {
        const double f = wt > -INFINITY && total > 0 ? exp2_of(((double)wt - top) * heat) / total : 0.0;
        const double fq = inner && wq > -INFINITY && draft_total > 0 ? exp2_of(((double)wq - draft_top) * draft_heat) / draft_total : 0.0;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            p[e] *= f;
            q[e] = inner ? q[e] * fq : 0.0;
        }
        for (int i = 0; i < n_refused; ++i) {
            const int at = refused[i] - (slice * kSampleSlice + own);
#pragma unroll
            for (int e = 0; e < EPT; ++e)
                if (at == (e >> 3) * kWave * 8 + (e & 7)) p[e] = q[e] = 0.0;
        }
    };

    // Largest entries and sums over all of a node's rows
    auto sum_rows = [&]() __attribute__((always_inline)) {
        for (int slice = 0; slice < a.slices; ++slice) {
            float wt, wq = -INFINITY;
            load_slice(slice, wt, wq);
            double s = 0, sq = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                s += p[e];
                if (inner) sq += q[e];
            }
            s = lanes_sum(s);
            if (inner) sq = lanes_sum(sq);
            if (lane == 0) {
                wave_top[0][wave] = wt, wave_sum[0][wave] = s;
                wave_top[1][wave] = wq, wave_sum[1][wave] = sq;
            }
            __syncthreads();
            if (wave < 2) {  // the first wave joins the parts of p, the second those of q
                const float m = lane < WAVES ? wave_top[wave][lane] : -INFINITY;
                const float mm = lanes_max(m);
                const double part = m > -INFINITY ? wave_sum[wave][lane] * exp2_of(((double)m - mm) * (wave ? draft_heat : heat)) : 0.0;
                const double ss = lanes_sum(part);
                const int best = greedy && wave == 0 ? lanes_min(m == mm && lane < WAVES ? wave_best[lane] : kNone) : kNone;
                if (lane == 0) {
                    part_top[wave][slice] = mm, part_sum[wave][slice] = ss;
                    if (wave == 0) part_best[slice] = best;
                }
            }
            __syncthreads();
        }
        auto join = [&](int which, double h, float &t, double &sum) __attribute__((always_inline)) {
            const float m = lane < a.slices ? part_top[which][lane] : -INFINITY;
            t = lanes_max(m);
            sum = lanes_sum(m > -INFINITY ? part_sum[which][lane] * exp2_of(((double)m - t) * h) : 0.0);
        };
        join(0, heat, top, total);
        if (inner) join(1, draft_heat, draft_top, draft_total);
    };

    // Sums of max(p - a q, 0) and of q into part_sum
    auto sum_residual = [&](double taken, double &s_all, double &w_all) __attribute__((always_inline)) {
        __syncthreads();
        for (int slice = 0; slice < a.slices; ++slice) {
            float wt, wq = -INFINITY;
            load_slice(slice, wt, wq);
            normalise(slice, wt, wq);
            double s = 0, w = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                const double r = p[e] - taken * q[e];
                s += r > 0 ? r : 0.0;
                w += q[e];
            }
            s = lanes_sum(s);
            w = lanes_sum(w);
            if (lane == 0) wave_sum[0][wave] = s, wave_sum[1][wave] = w;
            __syncthreads();
            if (wave < 2) {
                const double all = lanes_sum(lane < WAVES ? wave_sum[wave][lane] : 0.0);
                if (lane == 0) part_sum[wave][slice] = all;
            }
            __syncthreads();
        }
        s_all = lanes_sum(lane < a.slices ? part_sum[0][lane] : 0.0);
        w_all = lanes_sum(lane < a.slices ? part_sum[1][lane] : 0.0);
    };

    int next = -1;
    float next_logp = -INFINITY;
    while (true) {
        const uint64_t kids = __ballot(is_node && my_parent == cur && my_tok_ok);
        if (lane == 0) kid_mask[wave] = kids;
        const bool any_kid = __syncthreads_or(kids != 0);
        inner = any_kid && drawn;
        n_refused = 0;
        sum_rows();
        const double log_total = log(total);
        int best = kNone;
        if (greedy) {
            best = lanes_min(lane < a.slices && part_top[0][lane] == top ? part_best[lane] : kNone);
            if (!(total > 0)) best = kNone;
        }
        // the children's probabilities, each in its own thread
        if (is_node && my_parent == cur && my_tok_ok) {
            const float l = cleaned(Elem<TT>::load(target + cur * a.t_stride[1] + my_tok));
            kid_p[tid] = total > 0 ? weight(l, top, heat) / total : 0.0;
            kid_logp[tid] = total > 0 && l > -INFINITY ? (float)(((double)l - top) / (greedy ? 1.0 : (double)temp) - log_total) : -INFINITY;
            kid_q[tid] = 1.0;
            if (inner) {
                const float lq = cleaned(Elem<TD>::load(draft + cur * a.d_stride[1] + my_tok));
                kid_q[tid] = draft_total > 0 ? weight(lq, draft_top, draft_heat) / draft_total : 0.0;
            }
        }
        __syncthreads();
        double taken = 0, mass = 1, left = 1;  // a, S, W
        int found = -1;
        for (int w = 0; w < LS_MAX_TREE / kWave && found < 0; ++w) {
            for (uint64_t m = kid_mask[w]; m && found < 0; m &= m - 1) {
                const int k = w * kWave + __builtin_ctzll(m);
                const int t = tok[k];
                bool again = false;  // a token that has been refused has no weight any more
                for (int i = 0; i < n_refused; ++i) again |= refused[i] == t;
                const double px = again ? 0.0 : kid_p[k], qx = again && inner ? 0.0 : kid_q[k], u = accept_u[k];
                const bool ok = greedy ? t == best : (px - (inner ? taken * qx : 0.0)) * left > u * qx * mass;
                if (ok) {
                    found = k;
                } else {
                    __syncthreads();  // everybody has read the list
                    if (tid == 0) refused[n_refused] = t;
                    ++n_refused;
                    __syncthreads();
                    if (!greedy) {
                        if (inner) taken = left > 0 ? fmin(taken + mass / left, 1e300) : 1e300;  // (finite: q(v) = 0 stays out of it)
                        double w_all;
                        sum_residual(inner ? taken : 0.0, mass, w_all);
                        if (inner && !a.with_replacement) left = w_all;
                    }
                }
            }
        }
        if (found >= 0) {
            if (tid == 0) {
                path[len] = found;
                logp[len - 1] = kid_logp[found];
            }
            ++len;
            cur = found;
            __syncthreads();  // children and parts are read before the next node's are written
            continue;
        }

        // The path ends here
        if (greedy) {
            next = best == kNone ? -1 : best;
        } else if (total > 0) {
            if (n_refused == 0) {  // the parts are of weights still
                double s = 0;
                if (lane < a.slices && part_top[0][lane] > -INFINITY)
                    s = part_sum[0][lane] * exp2_of(((double)part_top[0][lane] - top) * heat) / total;
                __syncthreads();
                if (wave == 0 && lane < a.slices) part_sum[0][lane] = s;
                __syncthreads();
                mass = lanes_sum(lane < a.slices ? part_sum[0][lane] : 0.0);
            }
            if (mass > 0) {
                const float u = a.sample_uniforms[b];
                const double mine = lane < a.slices ? part_sum[0][lane] : 0.0;
                const double upto = lanes_scan(mine, lane);
                const double point = (double)u * mass;
                const uint64_t passed = __ballot(mine > 0 && upto > point), some = __ballot(mine > 0);
                const int slice = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some);
                const double rest = point - __shfl(upto - mine, slice, kWave);
                if (tid == 0) found_sh = kNone, last_sh = -1;
                float wt, wq = -INFINITY;
                load_slice(slice, wt, wq);
                normalise(slice, wt, wq);
                double s = 0;
#pragma unroll
                for (int e = 0; e < EPT; ++e) {
                    const double r = p[e] - (inner ? taken : 0.0) * q[e];
                    p[e] = r > 0 ? r : 0.0;
                    s += p[e];
                }
                s = lanes_sum(s);
                if (lane == 0) wave_sum[0][wave] = s;
                __syncthreads();
                double before = 0;  // of the entries before this wave's, then before this run
                for (int w = 0; w < wave; ++w) before += wave_sum[0][w];
                int first = kNone, last = -1;
#pragma unroll
                for (int r = 0; r < RUNS; ++r) {
                    double run = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) run += p[r * 8 + e];
                    const double end = lanes_scan(run, lane);
                    double c = before + (end - run);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int v = slice * kSampleSlice + own + r * kWave * 8 + e;
                        c += p[r * 8 + e];
                        if (p[r * 8 + e] > 0) {
                            last = v;
                            if (first == kNone && c > rest) first = v;
                        }
                    }
                    before += __shfl(end, 63, kWave);
                }
                if (first != kNone) atomicMin(&found_sh, first);
                if (last >= 0) atomicMax(&last_sh, last);
                __syncthreads();
                next = found_sh != kNone ? found_sh : last_sh;
            }
        }
        if (next >= 0) {
            const float l = cleaned(Elem<TT>::load(target + cur * a.t_stride[1] + next));
            next_logp = (float)(((double)l - top) / (greedy ? 1.0 : (double)temp) - log_total);
        } else {
            err |= 4;
        }
        break;
    }
    __syncthreads();
    if (is_node) {
        const int64_t at = (int64_t)b * a.n_tree + tid;
        a.path[at] = path[tid];
        if (a.logprobs) a.logprobs[at] = tid == len - 1 ? next_logp : logp[tid];
    }
    if (tid == 0) {
        a.len[b] = len;
        a.next[b] = next;
        if (a.err_flag) a.err_flag[b] = err;
    }
}

template <typename TT> hipError_t launch_for(const SampleArgs &a, int draft_dtype, hipStream_t stream)
{
    const dim3 grid(a.batch), block(NT);
    if (draft_dtype == LS_F32) hipLaunchKernelGGL((tree_sample_kernel<TT, float>), grid, block, 0, stream, a);
    else if (draft_dtype == LS_F16) hipLaunchKernelGGL((tree_sample_kernel<TT, half_t>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((tree_sample_kernel<TT, uint16_t>), grid, block, 0, stream, a);
    return hipGetLastError();
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
