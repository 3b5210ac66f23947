// Causal attention of a step's new tokens over a paged cache (16-bit inputs, matrix cores).
//
// Request b has n new tokens, the last of its kv rows; token i stands at row p = kv - n + i and sees rows
// max(0, p - window + 1) .. p.  The n * G query rows that share a KV head (G query heads a KV head) are ordered token
// first, row r = token r / G, head r % G, so that what a row sees grows with r.
//
// One wave per 32 query rows of a request and KV head; it walks the rows they see in tiles of 32 keys.
//   S^T = K Q^T, softmax with a running maximum, O^T += V^T P^T   (operand layouts: ls_mfma.hpp)
// so a lane holds 16 scores of ONE query row, and the numerators go from the accumulators of the first product to the operand of the
// second without leaving the lane.
#include "ls_mfma.hpp"
#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int TK = 32;  // keys per tile

template <int D, bool F16>
__global__ void __launch_bounds__(64)
chunk_attn_kernel(ChunkArgs a)
{
    constexpr int KSTEPS = D / 16, MT = D / 32, CH = D / 8, ROWB = D * 2, TILEB = TK * ROWB;
    typedef __attribute__((address_space(3))) const uint4 *lds_u4;
    typedef __attribute__((address_space(3))) shortx4 *lds_s4;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * TILEB];
    const int lane = threadIdx.x, li = lane & 31, lh = lane >> 5;
    const int g = blockIdx.x % a.n_kv_heads;
    int block = blockIdx.x / a.n_kv_heads;

    // the request whose row block this is
    int b = 0, first = 0, n = 0;
    for (; b < a.batch; ++b) {
        first = a.cu_new[b];
        first = first < 0 ? 0 : (first > a.n_tokens ? a.n_tokens : first);
        int end = a.cu_new[b + 1];
        end = end < first ? first : (end > a.n_tokens ? a.n_tokens : end);
        n = end - first;
        const int rows = (n < a.max_new_len ? n : a.max_new_len) * a.group, blocks = (rows + 31) / 32;
        if (block < blocks) break;
        block -= blocks;
    }
    if (b == a.batch) return;
    int kv = a.kv_lens[b];
    kv = kv < 0 ? 0 : (kv > a.max_kv_len ? a.max_kv_len : kv);
    const int rows = (n < a.max_new_len ? n : a.max_new_len) * a.group;
    const int r = block * 32 + li;
    const bool ok = r < rows;
    const int token = first + (ok ? r : rows - 1) / a.group, head = g * a.group + (ok ? r : rows - 1) % a.group;
    const int place = kv - n + (token - first);  // the row this query stands at
    const int seen_lo = a.window > 0 && place - a.window + 1 > 0 ? place - a.window + 1 : 0;
    // rows that some query of the block sees
    const int lo = __builtin_amdgcn_readfirstlane(seen_lo);
    int hi = kv - n + (block * 32 + 31 < rows ? block * 32 + 31 : rows - 1) / a.group + 1;

    const uint8_t *q_ptr = a.q + token * a.q_s[0] + head * a.q_s[1];
    bf16x8 q_reg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) q_reg[kk] = __builtin_bit_cast(bf16x8, *(const uint4 *)(q_ptr + kk * 32 + lh * 16));

    floatx16 o[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[mt][e] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float c = a.scale_log2;
    const int32_t *tab = a.block_table + (int64_t)b * a.bt_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const uint32_t base = lds_offset(smem);
    const uint32_t k_off = base + li * ROWB + ((lh ^ (li & (CH - 1))) * 16);
    const int tr_s = lane & 15, tr_row = 4 * lh + (tr_s >> 2);
    const int tr_dchunk = 2 * ((lane >> 4) & 1) + ((tr_s & 3) >> 1);
    const uint32_t v_off = base + TILEB + tr_row * ROWB + ((tr_dchunk ^ (vswz(tr_row) & (CH - 1))) * 16) + (tr_s & 1) * 8;

    for (int k0 = lo & ~(TK - 1); k0 < hi; k0 += TK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TK * CH / 64; ++i) {
            const int row = (i * 64 + lane) / CH, pos = lane % CH;
            const int src = k0 + row < kv ? k0 + row : kv - 1;  // rows past the end repeat the last; their scores are masked
            const int64_t page = tab[src >> a.page_shift];
            const int in_page = src & page_mask;
            const uint8_t *kr = a.k_pages + page * a.kc_s[0] + g * a.kc_s[1] + in_page * a.kc_s[2];
            const uint8_t *vr = a.v_pages + page * a.vc_s[0] + g * a.vc_s[1] + in_page * a.vc_s[2];
            *(uint4 *)(smem + row * ROWB + (pos ^ (row & (CH - 1))) * 16) = *(const uint4 *)(kr + pos * 16);
            *(uint4 *)(smem + TILEB + row * ROWB + (pos ^ (vswz(row) & (CH - 1))) * 16) = *(const uint4 *)(vr + pos * 16);
        }
        __syncthreads();
        floatx16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk)
            s = mfma32<F16>(__builtin_bit_cast(bf16x8, *(lds_u4)(uintptr_t)(k_off ^ (uint32_t)(kk << 5))), q_reg[kk], s);
        float mx = -INFINITY;
        uint32_t seen = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int key = k0 + 8 * (e >> 2) + 4 * lh + (e & 3);
            const bool sees = key >= seen_lo && key <= place;
            seen |= (uint32_t)sees << e;
            s[e] = sees ? s[e] : -INFINITY;
            mx = fmaxf(mx, s[e]);
        }
        mx = half_max(mx);
        const float m_new = fmaxf(m, mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * c);
        m = m_new;
        l *= alpha;
        const float mc = m == -INFINITY ? 0.f : m * c;
        uint32_t pp[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -mc)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], c, -mc));
            l += p0 + p1;
            pp[e >> 1] = pack16<F16>(p0, p1);
        }
        bf16x8 frag[KSTEPS];
#pragma unroll
        for (int f = 0; f < KSTEPS; ++f) {
            const uint32_t at = (v_off ^ (uint32_t)((f % MT) << 6)) + ((f / MT) * 16) * ROWB;
            const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)at));
            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)(at + 8 * ROWB)));
            frag[f] = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
        }
        // infinities and NaN among the values reach the rows that see them, and no others (0 * inf in the product)
        const bool not_finite = __any(seen != 0xffffu) && drop_not_finite<F16>(frag);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[mt][e] *= alpha;
#pragma unroll
        for (int f = 0; f < KSTEPS; ++f) {
            const uint32_t *u = pp + 4 * (f / MT);
            o[f % MT] = mfma32<F16>(frag[f], __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3])), o[f % MT]);
        }
        if (not_finite)
            for (int key = k0; key < k0 + TK && key < kv; ++key)
                if (key >= seen_lo && key <= place)
                    add_not_finite<F16>(o, a.v_pages + (int64_t)tab[key >> a.page_shift] * a.vc_s[0] + g * a.vc_s[1] + (key & page_mask) * a.vc_s[2], lh);
    }
    if (!ok) return;
    l = half_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint8_t *dst = a.out + token * a.o_s[0] + head * a.o_s[1];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg)
            *(uint2 *)(dst + (mt * 32 + rg * 8 + 4 * lh) * 2) = make_uint2(pack16<F16>(o[mt][4 * rg] * inv, o[mt][4 * rg + 1] * inv),
                                                                         pack16<F16>(o[mt][4 * rg + 2] * inv, o[mt][4 * rg + 3] * inv));
    if (lh == 0) a.lse[(int64_t)token * a.n_q_heads + head] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkArgs &a, int dtype, int head_dim, hipStream_t stream)
{
    // row blocks: each request rounds up by less than one
    const int64_t rows = (int64_t)a.n_tokens * a.group, most = (int64_t)a.max_new_len * a.group;
    int64_t blocks = (rows + 31 * (int64_t)(a.batch < a.n_tokens ? a.batch : a.n_tokens)) / 32;
    if (blocks > a.batch * ((most + 31) / 32)) blocks = a.batch * ((most + 31) / 32);
    const dim3 grid((unsigned)(blocks * a.n_kv_heads));
    auto kernel = head_dim == 128 ? (dtype == LS_F16 ? chunk_attn_kernel<128, true> : chunk_attn_kernel<128, false>)
                                  : (dtype == LS_F16 ? chunk_attn_kernel<64, true> : chunk_attn_kernel<64, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ls
