// Rotary positions of packed tokens, with the write of keys and values into pages.
//
// Pair (x, y) of a head becomes (x cos - y sin, x sin + y cos); the cosines and sines of a token are a row of a table (several
// axes: pieces of several rows).  Products and differences in fp32, rounded once.
//
// A thread owns one unit of 16 elements of a token, 8 pairs, and goes through the token's heads: cosines and sines are read
// once and stay in registers, queries, keys and values pass through once, 16 bytes a lane.  A rotated unit is two pieces of 8
// elements rotary_dim/2 apart, or 16 neighbouring elements (interleaved).
//
// Bound by HBM for prompts (8192 tokens of 56 heads of 128, bf16: 48 us, 5.0 TB/s read and written), by latency for a few
// tokens (24 tokens: 4 us).
#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int NT = 256;   // threads per workgroup
constexpr int BATCH = 2;  // heads whose loads are in flight together
constexpr int kFewTokens = 2048;

// 16-byte pieces of 8 elements
template <typename T> constexpr int kPieces = sizeof(T) * 8 / 16;

template <typename T> __device__ __forceinline__ void unpack(const uint4 (&raw)[kPieces<T>], float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 f = __builtin_bit_cast(float4, raw[i]);
            x[4 * i] = f.x, x[4 * i + 1] = f.y, x[4 * i + 2] = f.z, x[4 * i + 3] = f.w;
        }
    } else {
        const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T lo, hi;
            *(uint16_t *)&lo = (uint16_t)w[i];
            *(uint16_t *)&hi = (uint16_t)(w[i] >> 16);
            x[2 * i] = Elem<T>::load(&lo);
            x[2 * i + 1] = Elem<T>::load(&hi);
        }
    }
}

template <typename T> __device__ __forceinline__ void pack(const float (&x)[8], uint4 (&raw)[kPieces<T>])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) raw[i] = __builtin_bit_cast(uint4, make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T lo, hi;
            Elem<T>::store(&lo, x[2 * i]);
            Elem<T>::store(&hi, x[2 * i + 1]);
            w[i] = (uint32_t) * (uint16_t *)&lo | (uint32_t) * (uint16_t *)&hi << 16;
        }
        raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// SLOTS: heads of a token in work at a time (threads per token: SLOTS * D / 16)
template <typename T, int D, int SLOTS, bool INTERLEAVED>
__global__ void __launch_bounds__(NT)
rope_kernel(RopeArgs a)
{
    constexpr int UNITS = D / 16;
    constexpr int PIECES = kPieces<T>;
    constexpr int TOKENS = NT / (UNITS * SLOTS);  // per workgroup
    const int unit = threadIdx.x % UNITS;
    const int head0 = threadIdx.x / UNITS % SLOTS;
    const int t = blockIdx.x * TOKENS + threadIdx.x / (UNITS * SLOTS);
    if (t >= a.n_tokens) return;

    const bool rotates = unit * 8 < a.pairs;
    // byte offsets of the unit's two pieces of 8 elements
    const int at0 = (int)sizeof(T) * (rotates && !INTERLEAVED ? 8 * unit : 16 * unit);
    const int at1 = (int)sizeof(T) * (rotates && !INTERLEAVED ? 8 * unit + a.pairs : 16 * unit + 8);
    const int n_k = a.k ? a.n_kv_heads : 0, n_v = a.v ? a.n_kv_heads : 0;
    const int last_k = a.n_q_heads + n_k, n_heads = last_k + n_v;  // queries, then keys, then values

    uint4 raw[BATCH][2][PIECES];
    auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = h0 + i * SLOTS;
            if (h >= n_heads) continue;
            const uint8_t *src = h < a.n_q_heads ? a.q + t * a.q_s[0] + h * a.q_s[1]
                                 : h < last_k    ? a.k + t * a.k_s[0] + (h - a.n_q_heads) * a.k_s[1]
                                                 : a.v + t * a.v_s[0] + (h - last_k) * a.v_s[1];
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                raw[i][0][j] = *(const uint4 *)(src + at0 + 16 * j);
                raw[i][1][j] = *(const uint4 *)(src + at1 + 16 * j);
            }
        }
    };
    load(head0);  // on their way while the token's position and its row of the table are read, one after the other

    int32_t slot = a.slots ? a.slots[t] : 0;
    float cs[8], sn[8];  // this unit's cosines and sines
    if (rotates) {
        const int i0 = unit * 8;
        int32_t place[LS_MAX_AXES];
#pragma unroll
        for (int x = 0; x < LS_MAX_AXES; ++x) {
            const int p = x < a.n_axes ? a.positions[x * a.positions_stride + t] : 0;
            place[x] = p < 0 ? 0 : (p < a.n_positions ? p : a.n_positions - 1);
        }
        // the position by which pair i goes
        auto place_of = [&](int i) __attribute__((always_inline)) {
            int p = place[0];
#pragma unroll
            for (int x = 1; x < LS_MAX_AXES; ++x) p = x < a.n_axes && i >= a.axis_end[x - 1] ? place[x] : p;
            return p;
        };
        bool whole = true;  // no axis ends inside the unit
#pragma unroll
        for (int x = 0; x + 1 < LS_MAX_AXES; ++x) whole &= x + 1 >= a.n_axes || a.axis_end[x] <= i0 || a.axis_end[x] >= i0 + 8;
        if (whole) {
            const float *row = a.cos_sin + (int64_t)place_of(i0) * (2 * a.pairs) + i0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 c = *(const float4 *)(row + 4 * i), s = *(const float4 *)(row + a.pairs + 4 * i);
                cs[4 * i] = c.x, cs[4 * i + 1] = c.y, cs[4 * i + 2] = c.z, cs[4 * i + 3] = c.w;
                sn[4 * i] = s.x, sn[4 * i + 1] = s.y, sn[4 * i + 2] = s.z, sn[4 * i + 3] = s.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float *row = a.cos_sin + (int64_t)place_of(i0 + i) * (2 * a.pairs) + i0 + i;
                cs[i] = row[0];
                sn[i] = row[a.pairs];
            }
        }
    }
    const bool stored = !a.slots || (uint32_t)slot < (uint32_t)a.n_slots;
    const int64_t page = slot >> a.page_shift, row = slot & ((1 << a.page_shift) - 1);
    const int64_t k_dst = a.slots ? page * a.ko_s[0] + row * a.ko_s[2] : t * a.ko_s[0];
    const int64_t v_dst = page * a.vo_s[0] + row * a.vo_s[2];

    for (int h0 = head0; h0 < n_heads; h0 += BATCH * SLOTS) {
        if (h0 != head0) load(h0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = h0 + i * SLOTS;
            if (h >= n_heads || (h >= a.n_q_heads && !stored)) continue;
            uint8_t *dst = h < a.n_q_heads ? a.q_out + t * a.qo_s[0] + h * a.qo_s[1]
                           : h < last_k    ? a.k_out + k_dst + (h - a.n_q_heads) * a.ko_s[1]
                                           : a.v_out + v_dst + (h - last_k) * a.vo_s[1];
            if (rotates && h < last_k) {
                float x[2][8], y[2][8];
                unpack<T>(raw[i][0], x[0]);
                unpack<T>(raw[i][1], x[1]);
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    // pair p of the unit: elements p of both pieces, or 2p and 2p + 1 of the two in a row
                    const int e0 = INTERLEAVED ? (2 * p) / 8 : 0, i0 = INTERLEAVED ? (2 * p) % 8 : p;
                    const int e1 = INTERLEAVED ? e0 : 1, i1 = INTERLEAVED ? i0 + 1 : p;
                    y[e0][i0] = x[e0][i0] * cs[p] - x[e1][i1] * sn[p];
                    y[e1][i1] = x[e0][i0] * sn[p] + x[e1][i1] * cs[p];
                }
                pack<T>(y[0], raw[i][0]);
                pack<T>(y[1], raw[i][1]);
            }
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                *(uint4 *)(dst + at0 + 16 * j) = raw[i][0][j];
                *(uint4 *)(dst + at1 + 16 * j) = raw[i][1][j];
            }
        }
    }
}

template <typename T, int D, int SLOTS> hipError_t launch_form(const RopeArgs &a, hipStream_t stream)
{
    constexpr int TOKENS = NT / (D / 16 * SLOTS);
    const dim3 grid((a.n_tokens + TOKENS - 1) / TOKENS);
    if (a.interleaved) hipLaunchKernelGGL((rope_kernel<T, D, SLOTS, true>), grid, dim3(NT), 0, stream, a);
    else hipLaunchKernelGGL((rope_kernel<T, D, SLOTS, false>), grid, dim3(NT), 0, stream, a);
    return hipGetLastError();
}

template <typename T> hipError_t launch_type(const RopeArgs &a, int head_dim, hipStream_t stream)
{
    // head_dim 128: a token's heads go through one workgroup, so that its reads and writes are in one place (8000 tokens of 32 + 8 + 8
    // heads: 16 threads a token 60 us, 32 48, 64 46, 128 43, 256 42).  head_dim 64: 32 slots up to 2048 tokens, beyond by 8, of which
    // none is idle where heads come in eights.  us by 32 and by 8 slots, bf16, all of a head turned:
    //   tokens               1500          2000          3000          4000          8000
    //   16 + 4 + 4 heads   4.7   5.7     5.6   6.9     7.5   8.2     9.3   8.8    13.6  11.9
    //   8 + 8 + 8          4.7   5.3     5.4   6.2     7.0   7.7     8.9   8.2    13.0  11.3
    //   32 + 8 + 8         7.0  10.2     8.3  10.6    10.4  11.9    12.6  12.9    25.5  25.0
    //   4 + 1 + 1          3.6   3.4     3.6   3.5     4.3   3.8     5.4   4.0     9.3   6.1
    // (16 + 4 + 4 with three axes, neighbouring pairs, half a head: 6.9 and 7.3 at 2000, 9.4 and 8.9 at 3000.)  Where the two cross
    // goes by the heads, from below 1500 to past 4500 tokens; just past 2048 the 8 slots cost 2.3 us more at most.
    if (head_dim == 128) return launch_form<T, 128, 32>(a, stream);
    return a.n_tokens <= kFewTokens ? launch_form<T, 64, 32>(a, stream) : launch_form<T, 64, 8>(a, stream);
}

}  // namespace

hipError_t launch_rope(const RopeArgs &all, int dtype, int head_dim, hipStream_t stream)
{
    constexpr int32_t kMostTokens = 1 << 23;  // of a launch, which has fewer than 2^32 threads: up to 256 a token
    for (int64_t done = 0; done < all.n_tokens; done += kMostTokens) {
        RopeArgs a = all;
        a.n_tokens = all.n_tokens - done < kMostTokens ? (int32_t)(all.n_tokens - done) : kMostTokens;
        a.q += done * a.q_s[0];
        a.q_out += done * a.qo_s[0];
        a.positions += done;
        if (a.k) a.k += done * a.k_s[0];
        if (a.v) a.v += done * a.v_s[0];
        if (a.slots) a.slots += done;
        else if (a.k) a.k_out += done * a.ko_s[0];
        const hipError_t e = dtype == LS_BF16  ? launch_type<uint16_t>(a, head_dim, stream)
                             : dtype == LS_F16 ? launch_type<half_t>(a, head_dim, stream)
                                               : launch_type<float>(a, head_dim, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ls
