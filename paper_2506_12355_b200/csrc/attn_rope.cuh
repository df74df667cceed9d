// Per-head normalisation and rotation of queries and keys in one pass over a projection's output, its gradient, and the
// same pass for new tokens whose keys and values go into a paged cache.
//
//     n = x rsqrt(mean(x^2) + eps) w   (over one head's D values),     y = R_pos n :
//     pair i < R/2 of the first R values turns by the angle whose cosine and sine are row pos of the table.
//     Gradient, with g = R_pos^T dy, r = rsqrt(mean(x^2) + eps):  dx = r (g w) - x r^3 mean(g w x),   dw = sum g x r.
//
// Memory-bound: each value is read and written once, ~11 operations per value.  A row (one head of one token) lies on
// D / 8 lanes, 16 bytes each, so that the mean and (for pairs R/2 apart) the partner values move by warp shuffles and
// nothing is staged.  A warp stays with one token: position, cosines and sines are read once and kept in registers while
// it walks the token's heads, four rows deep.  The eight warps of a block take eight neighbouring tokens, so that
// the head-major outputs are written in runs of 8 rows.  fp32 inside, one rounding on output.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "attn_paged.cuh"
#include "sm100_ptx.cuh"

namespace attn_rope {

using attn_paged::report_bad_index;

constexpr int kWarps = 8;      // warps of a block
constexpr int kDeep = 4;       // rows of a lane in flight

struct Strides { int64_t batch, token, head; };   // elements

struct RopeParams {
    const void* in[3];          // q, k, v: [B, S, heads, D] (paged: [tokens, heads, D]) through strides
    void* out[3];               // head-major (or, paged, q_out and the two caches)
    Strides is[3], os[3];       // paged: of a cache batch = page, token = slot
    int heads[3];
    const void* weight[3];      // NULL: not normalised
    int weight_f32;
    const float* table;         // [table_len][R]: R/2 cosines, R/2 sines
    int table_len, R, interleaved;
    const int* positions;       // [B, S]; NULL: the token's index in its sequence
    float eps;
    int64_t tokens;             // B * S, or tokens of the batch
    int S;
    int unit_end[3];            // running sums of the units of kDeep * rows-per-warp heads of q, k, v
    int* status;
    // paged
    const int* cu_seqlens;      // [n_seqs + 1]; NULL: token t belongs to sequence t
    const int* seq_lens;        // lengths, the new tokens included
    const int* block_table;
    int64_t table_stride;
    int n_seqs, max_len, num_pages, page_shift;
    // gradient
    const void* dy[3];
    Strides ds[3];
    float* partial;             // [blocks][2][D] sums of the weight gradients
};

template <int DTYPE>
__device__ __forceinline__ void unpack8(const uint4& w, float* f) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DTYPE == 0) {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            f[2 * i] = h.x;
            f[2 * i + 1] = h.y;
        } else {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}

template <int DTYPE>
__device__ __forceinline__ uint4 pack8(const float* f) {
    return make_uint4(sm100::pack2<DTYPE>(f[0], f[1]), sm100::pack2<DTYPE>(f[2], f[3]), sm100::pack2<DTYPE>(f[4], f[5]),
                      sm100::pack2<DTYPE>(f[6], f[7]));
}

template <int DTYPE>
__device__ __forceinline__ void load_weight(const void* w, int f32, int d0, float* f) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 1.f;
    } else if (f32) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + d0));
        const float4 b = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + d0 + 4));
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
        unpack8<DTYPE>(__ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(w) + d0 * 2)), f);
    }
}

// One token's rotation, as a lane (8 values of a row, from value d0) needs it: y_e = n_e cs_e + partner_e sn_e.
struct Turn {
    float cs[8], sn[8];
    int partner;          // lane that holds the partner values (own lane: pairs are neighbours, or not rotated)
    __device__ __forceinline__ void load(const RopeParams& p, int pos, int d0, int lane, bool back) {
        partner = lane;
        const float flip = back ? -1.f : 1.f;
        if (d0 >= p.R) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
            return;
        }
        const int half = p.R >> 1;
        const float* row = p.table + static_cast<int64_t>(pos) * p.R;
        if (p.interleaved) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(row + (d0 >> 1)));
            const float4 b = __ldg(reinterpret_cast<const float4*>(row + half + (d0 >> 1)));
            const float cc[4] = {a.x, a.y, a.z, a.w}, ss[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                cs[e] = cc[e >> 1];
                sn[e] = (e & 1) ? flip * ss[e >> 1] : -flip * ss[e >> 1];
            }
        } else {
            const bool first = d0 < half;
            const int i0 = first ? d0 : d0 - half;
            partner = first ? lane + (half >> 3) : lane - (half >> 3);
            const float sgn = first ? -flip : flip;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = __ldg(reinterpret_cast<const float4*>(row + i0 + 4 * h));
                const float4 b = __ldg(reinterpret_cast<const float4*>(row + half + i0 + 4 * h));
                cs[4 * h] = a.x; cs[4 * h + 1] = a.y; cs[4 * h + 2] = a.z; cs[4 * h + 3] = a.w;
                sn[4 * h] = sgn * b.x; sn[4 * h + 1] = sgn * b.y; sn[4 * h + 2] = sgn * b.z; sn[4 * h + 3] = sgn * b.w;
            }
        }
    }
    // executed by all lanes of the warp
    __device__ __forceinline__ void apply(float* f, int R, int interleaved) const {
        if (R == 0) return;
        float o[8];
        if (interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = f[e ^ 1];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = __shfl_sync(0xffffffffu, f[e], partner);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = fmaf(o[e], sn[e], f[e] * cs[e]);
    }
};

__device__ __forceinline__ void make_nan(float* f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __int_as_float(0x7fffffff);
}

template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int off = LPR / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Where one token's rows go in the paged form.  Returns the position, or -1 when the token is not written (padding behind
// the last sequence, or an entry that is out of range).
__device__ __forceinline__ int place_token(const RopeParams& p, int64_t token, int& page, int& slot) {
    int seq, pos;
    const int t = static_cast<int>(token);
    if (p.cu_seqlens) {
        // last sequence that begins at or before t (empty sequences share a begin; the last of them is not empty or is the end)
        if (t >= __ldg(p.cu_seqlens + p.n_seqs)) return -1;
        int lo = 0, hi = p.n_seqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(p.cu_seqlens + mid) <= t) lo = mid; else hi = mid;
        }
        seq = lo;
        const int len = __ldg(p.seq_lens + seq);
        pos = len - (__ldg(p.cu_seqlens + seq + 1) - t);
        if (len <= 0) return -1;
    } else {
        seq = t;
        const int len = __ldg(p.seq_lens + seq);
        if (len <= 0) return -1;      // a padded row of a batch
        pos = len - 1;
    }
    if (pos < 0 || pos >= p.max_len || (p.R > 0 && pos >= p.table_len)) {
        report_bad_index(p.status);
        return -1;
    }
    page = __ldg(p.block_table + static_cast<int64_t>(seq) * p.table_stride + (pos >> p.page_shift));
    slot = pos & ((1 << p.page_shift) - 1);
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) {
        report_bad_index(p.status);
        return -1;
    }
    return pos;
}

// grid: (blocks of 8 tokens, parts of the unit list)
template <int D, int DTYPE, bool PAGED>
__global__ void __launch_bounds__(kWarps * 32)
attn_rope_kernel(const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPR, d0 = (lane % LPR) * 8;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
    if (token >= p.tokens) return;
    int64_t b = 0, s = token;
    int pos, page = 0, slot = 0;
    bool bad = false;
    if constexpr (PAGED) {
        pos = place_token(p, token, page, slot);
        if (pos < 0) return;
    } else {
        b = token / p.S;
        s = token - b * p.S;
        pos = p.positions ? __ldg(p.positions + token) : static_cast<int>(s);
        if (p.R > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(p.table_len)) {
            report_bad_index(p.status);
            bad = true;      // the token's q and k rows become NaN
            pos = 0;
        }
    }
    Turn turn;
    turn.load(p, pos, d0, lane, false);
    for (int u = blockIdx.y; u < p.unit_end[2]; u += gridDim.y) {
        const int kind = u < p.unit_end[0] ? 0 : (u < p.unit_end[1] ? 1 : 2);
        const int h0 = (u - (kind == 0 ? 0 : p.unit_end[kind - 1])) * (kDeep * RPW) + sub;
        const int heads = p.heads[kind];
        const uint8_t* src = static_cast<const uint8_t*>(p.in[kind]) + (b * p.is[kind].batch + s * p.is[kind].token + d0) * 2;
        const bool cache = PAGED && kind > 0;
        uint8_t* dst = static_cast<uint8_t*>(p.out[kind]) +
                       ((cache ? page * p.os[kind].batch + slot * p.os[kind].token : b * p.os[kind].batch + s * p.os[kind].token) + d0) * 2;
        uint4 raw[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int h = h0 + i * RPW;
            if (h < heads) raw[i] = *reinterpret_cast<const uint4*>(src + h * p.is[kind].head * 2);
        }
        if (kind < 2) {
            float w[8];
            const bool norm = p.weight[kind] != nullptr;
            load_weight<DTYPE>(p.weight[kind], p.weight_f32, d0, w);
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                if (h0 - sub + i * RPW >= heads) break;      // uniform over the warp
                float f[8];
                if (h0 + i * RPW >= heads) raw[i] = make_uint4(0u, 0u, 0u, 0u);
                unpack8<DTYPE>(raw[i], f);
                if (bad) make_nan(f);
                if (norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
                    const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + p.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= r * w[e];
                }
                turn.apply(f, p.R, p.interleaved);
                raw[i] = pack8<DTYPE>(f);
            }
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int h = h0 + i * RPW;
            if (h < heads) *reinterpret_cast<uint4*>(dst + h * p.os[kind].head * 2) = raw[i];
        }
    }
}

// Gradient.  dy: head-major gradients of the outputs; in: q, k as the forward pass read them; out: gradients laid out like
// the inputs.  Blocks walk the tokens with a stride and keep the weight gradients of their rows in registers; each
// leaves its sum in `partial`, and attn_rope_weight_grad_kernel adds those in a fixed order.
template <int D, int DTYPE>
__global__ void __launch_bounds__(kWarps * 32)
attn_rope_bwd_kernel(const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    __shared__ float sums[2][kWarps * RPW][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPR, d0 = (lane % LPR) * 8;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float dw[2][8], w[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        load_weight<DTYPE>(p.weight[k], p.weight_f32, d0, w[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[k][e] = 0.f;
    }
    for (int64_t token = static_cast<int64_t>(blockIdx.x) * kWarps + warp; token < p.tokens; token += static_cast<int64_t>(gridDim.x) * kWarps) {
        const int64_t b = token / p.S, s = token - b * p.S;
        int pos = p.positions ? __ldg(p.positions + token) : static_cast<int>(s);
        bool bad = false;
        if (p.R > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(p.table_len)) {
            report_bad_index(p.status);
            bad = true;
            pos = 0;
        }
        Turn turn;
        turn.load(p, pos, d0, lane, true);
#pragma unroll
        for (int kind = 0; kind < 3; ++kind) {
            const int heads = p.heads[kind];
            const uint8_t* gsrc = static_cast<const uint8_t*>(p.dy[kind]) + (b * p.ds[kind].batch + s * p.ds[kind].token + d0) * 2;
            const uint8_t* xsrc = static_cast<const uint8_t*>(p.in[kind]) + (b * p.is[kind].batch + s * p.is[kind].token + d0) * 2;
            uint8_t* dst = static_cast<uint8_t*>(p.out[kind]) + (b * p.os[kind].batch + s * p.os[kind].token + d0) * 2;
            const bool norm = kind < 2 && p.weight[kind] != nullptr;
            for (int hw = 0; hw < heads; hw += kDeep * RPW) {
                uint4 gr[kDeep], xr[kDeep];
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    const int h = hw + i * RPW + sub;
                    gr[i] = xr[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (h < heads) {
                        gr[i] = *reinterpret_cast<const uint4*>(gsrc + h * p.ds[kind].head * 2);
                        if (norm) xr[i] = *reinterpret_cast<const uint4*>(xsrc + h * p.is[kind].head * 2);
                    }
                }
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    if (hw + i * RPW >= heads) break;
                    if (kind < 2) {
                        float f[8];
                        unpack8<DTYPE>(gr[i], f);
                        if (bad) make_nan(f);
                        turn.apply(f, p.R, p.interleaved);
                        if (norm) {
                            float x[8];
                            unpack8<DTYPE>(xr[i], x);
                            float ss = 0.f, gx = 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                ss = fmaf(x[e], x[e], ss);
                                gx = fmaf(f[e] * w[kind & 1][e], x[e], gx);
                            }
                            const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + p.eps);
                            const float k = row_sum<LPR>(gx) * (1.f / D) * r * r;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                dw[kind & 1][e] = fmaf(f[e], x[e] * r, dw[kind & 1][e]);
                                f[e] = r * fmaf(-k, x[e], f[e] * w[kind & 1][e]);
                            }
                        }
                        gr[i] = pack8<DTYPE>(f);
                    }
                    const int h = hw + i * RPW + sub;
                    if (h < heads) *reinterpret_cast<uint4*>(dst + h * p.os[kind].head * 2) = gr[i];
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[k][warp * RPW + sub][d0 + e] = dw[k][e];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kWarps * 32) {
        const int k = i / D, d = i % D;
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < kWarps * RPW; ++r) x += sums[k][r][d];
        p.partial[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = x;
    }
}

// dq_weight, dk_weight [D] fp32 from the blocks' sums; 32 columns per block, 32 warps.
__global__ void __launch_bounds__(1024)
attn_rope_weight_grad_kernel(const float* partial, int blocks, int D, float* dqw, float* dkw) {
    __shared__ float sums[32][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = blockIdx.x * 32 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float x = 0.f;
    for (int r = warp; r < blocks; r += 32) x += __ldcg(partial + static_cast<int64_t>(r) * 2 * D + col);
    sums[warp][lane] = x;
    __syncthreads();
    if (warp == 0) {
        x = 0.f;
#pragma unroll
        for (int w = 0; w < 32; ++w) x += sums[w][lane];
        float* out = col < D ? dqw : dkw;
        if (out) out[col < D ? col : col - D] = x;
    }
}

}  // namespace attn_rope
