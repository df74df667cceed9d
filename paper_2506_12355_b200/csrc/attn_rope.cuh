// Per-head normalisation and rotation of queries and keys in one pass over a projection's output, its gradient, and the
// same pass for new tokens whose keys and values go into a paged cache.
//
//     n = x rsqrt(mean(x^2) + eps) w   (over one head's D values),     y = R_pos n :
//     pair i < R/2 of the first R values turns by the angle whose cosine and sine are row pos of the table.
//     With several position axes (time, height, width, ..) each pair belongs to one of them, and turns by the row of that axis'
//     position.
//     Gradient, with g = R_pos^T dy, r = rsqrt(mean(x^2) + eps):  dx = r (g w) - x r^3 mean(g w x),   dw = sum g x r.
//
// Memory-bound: each value is read and written once.  The limit on the way there is the issue rate, so the arithmetic per
// 512 bytes is what the code is shaped by (a first form with a warp shuffle per partner value took 145 instructions):
//   * A row (one head of one token) lies on D / 8 lanes, and a lane holds two runs of four values, chosen so that both halves
//     of its pairs are its own (4 l and R/2 + 4 l for pairs R/2 apart): no shuffles but those of the mean.
//   * A warp stays with one token while it walks its heads, several rows deep, and the weights are folded into the cosines
//     and sines once per token: y = r (x_e A_e + x_p B_e), A_e = w_e cos, B_e = +- w_p sin.
//   * fp32 arithmetic is two-wide (f32x2); rows are addressed by stepping pointers.
// The eight warps of a block take eight neighbouring tokens, so that the head-major side is read or written in runs of 8
// rows.  fp32 inside, one rounding on output.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "attn_paged.cuh"
#include "sm100_ptx.cuh"

namespace attn_rope {

using attn_paged::report_bad_index;

constexpr int kWarps = 8;      // warps of a block
constexpr int kDeep = 4;       // rows of a lane in flight
constexpr int kBwdBlocks = 2;  // resident blocks per SM of the gradient kernel (its grid is one wave)

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
    const int* positions;       // [B, S]; NULL: the token's index in its sequence.  With several axes [axes][B, S] (paged: [axes][tokens])
    int n_axes;                 // several axes: their number, and the axis of each pair: four pairs to a byte, 2 bits each
    uint8_t pair_axes[32];
    float eps;
    int tokens;                 // B * S, or tokens of the batch
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
    float* partial;             // [blocks][D] sums of the weight gradients
    int q_blocks;               // blocks that take q; the others take k, then v
};

// Two-wide fp32.
struct F2 {
    uint64_t v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(uint64_t x) : v(x) {}
    __device__ __forceinline__ F2(float lo, float hi) : v(sm100::pack_f32x2(lo, hi)) {}
    __device__ __forceinline__ void get(float& lo, float& hi) const { sm100::unpack_f32x2(v, lo, hi); }
    __device__ __forceinline__ float sum() const {
        float lo, hi;
        get(lo, hi);
        return lo + hi;
    }
};
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { return F2(sm100::mul_f32x2(a.v, b.v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { return F2(sm100::fma_f32x2(a.v, b.v, c.v)); }

template <int DTYPE>
__device__ __forceinline__ F2 unpack2(uint32_t u) {
    if constexpr (DTYPE == 0) {
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&u));
        return F2(h.x, h.y);
    } else {
        return F2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
}

// The eight values of a row that a lane holds: two runs of four, from value a and from value b.
// Pairs R/2 apart: both halves of four pairs; neighbouring pairs, and the values that are not rotated: eight in a row.
struct Place {
    int a, b;
    bool turns;           // these values are rotated
    __device__ __forceinline__ Place(const RopeParams& p, int l) {
        turns = 8 * l < p.R;
        const bool split = turns && !p.interleaved;
        a = split ? 4 * l : 8 * l;
        b = split ? (p.R >> 1) + 4 * l : 8 * l + 4;
    }
};

// Rows as a lane sees them, 16-bit: .x, .y the run from a, .z, .w the run from b.
__device__ __forceinline__ uint4 load_row(const uint8_t* row, const Place& at) {
    const uint2 u = *reinterpret_cast<const uint2*>(row + 2 * at.a), v = *reinterpret_cast<const uint2*>(row + 2 * at.b);
    return make_uint4(u.x, u.y, v.x, v.y);
}
__device__ __forceinline__ void store_row(uint8_t* row, const Place& at, const uint4& x) {
    *reinterpret_cast<uint2*>(row + 2 * at.a) = make_uint2(x.x, x.y);
    *reinterpret_cast<uint2*>(row + 2 * at.b) = make_uint2(x.z, x.w);
}
template <int DTYPE>
__device__ __forceinline__ void unpack_row(const uint4& x, F2* f) {
    f[0] = unpack2<DTYPE>(x.x);
    f[1] = unpack2<DTYPE>(x.y);
    f[2] = unpack2<DTYPE>(x.z);
    f[3] = unpack2<DTYPE>(x.w);
}
template <int DTYPE>
__device__ __forceinline__ uint4 pack_row(const F2* f) {
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo, hi;
        f[e].get(lo, hi);
        y[e] = sm100::pack2<DTYPE>(lo, hi);
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}
template <int DTYPE>
__device__ __forceinline__ void load_weight(const void* w, int f32, const Place& at, F2* f) {
    if (f32) {
        const float4 u = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + at.a));
        const float4 v = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + at.b));
        f[0] = F2(u.x, u.y); f[1] = F2(u.z, u.w); f[2] = F2(v.x, v.y); f[3] = F2(v.z, v.w);
    } else {
        unpack_row<DTYPE>(load_row(static_cast<const uint8_t*>(w), at), f);
    }
}

// The other value of each pair.
template <bool INTER>
__device__ __forceinline__ F2 partner(const F2* x, int e) {
    if constexpr (INTER) {
        float lo, hi;
        x[e].get(lo, hi);
        return F2(hi, lo);
    } else {
        return x[e ^ 2];
    }
}

// The kernels' arithmetic in four forms, chosen once per row group by branches that all threads take alike: neighbouring pairs
// or not, the whole head rotated or not (then a lane's values may be unrotated, and an unrotated value must not meet a
// "partner": 0 times infinity is no number).  As run-time selects inside the arithmetic these cost a third of its instructions.
template <class Work>
__device__ __forceinline__ void by_form(const RopeParams& p, int D, Work&& work) {
    if (p.interleaved) {
        if (p.R == D) work(std::true_type{}, std::true_type{}); else work(std::true_type{}, std::false_type{});
    } else {
        if (p.R == D) work(std::false_type{}, std::true_type{}); else work(std::false_type{}, std::false_type{});
    }
}

// x turned by (cs, sn)
template <bool INTER, bool WHOLE>
__device__ __forceinline__ void turn_values(F2* y, const F2* x, const F2* cs, const F2* sn, bool turns) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = x[e] * cs[e];
        if (WHOLE || turns) y[e] = fma2(partner<INTER>(x, e), sn[e], y[e]);
    }
}

// The axes of a lane's four pairs, 2 bits each.  `same`: in every lane of the warp the four pairs belong to one axis (runs of pairs
// per axis whose lengths are multiples of 4): two 16-byte loads of the table per lane and token, as with one axis.  Axes that
// take turns need eight single loads.  (With one axis nothing is asked: the vote cost the gradient half a us of 60.)
struct PairAxes {
    unsigned of;
    bool same;
    template <bool AXES>
    static __device__ __forceinline__ PairAxes of_lane(const RopeParams& p, int l) {
        PairAxes a = {0u, true};
        if constexpr (AXES) {
            a.of = 8 * l < p.R ? p.pair_axes[l] : 0u;
            a.same = __all_sync(0xffffffffu, a.of == (a.of & 3u) * 0x55u);
        }
        return a;
    }
};

// One token's positions on all axes.
struct AxisPositions {
    int at[4];
    // false: one of them is out of range (all are 0 then)
    __device__ __forceinline__ bool load(const RopeParams& p, int64_t token) {
        bool ok = true;
#pragma unroll
        for (int a = 0; a < 4; ++a) at[a] = a < p.n_axes ? __ldg(p.positions + a * static_cast<int64_t>(p.tokens) + token) : 0;
#pragma unroll
        for (int a = 0; a < 4; ++a) ok = ok && (p.R == 0 || static_cast<unsigned>(at[a]) < static_cast<unsigned>(p.table_len));
        if (!ok) at[0] = at[1] = at[2] = at[3] = 0;
        return ok;
    }
    // the position of pair i of a lane's four
    __device__ __forceinline__ int of_pair(const PairAxes& axes, int i) const {
        const unsigned a = axes.of >> (2 * i);
        return a & 2u ? (a & 1u ? at[3] : at[2]) : (a & 1u ? at[1] : at[0]);
    }
};

// One token's rotation, for the values of a lane: y_e = n_e cs_e + partner_e sn_e.
struct Turn {
    F2 cs[4], sn[4];
    // back: the transposed rotation
    __device__ __forceinline__ void load(const RopeParams& p, int pos, int l, const Place& at, bool back) {
        if (!at.turns) {
            none();
            return;
        }
        const float* row = p.table + static_cast<int64_t>(pos) * p.R;     // either way pairs 4 l .. 4 l + 3
        set(p, __ldg(reinterpret_cast<const float4*>(row + 4 * l)), __ldg(reinterpret_cast<const float4*>(row + (p.R >> 1) + 4 * l)), back);
    }
    __device__ __forceinline__ void load_axes(const RopeParams& p, const AxisPositions& pos, const PairAxes& axes, int l, const Place& at, bool back) {
        if (!at.turns) {
            none();
            return;
        }
        const int half = p.R >> 1;
        auto row = [&](int i) { return p.table + static_cast<int64_t>(pos.of_pair(axes, i)) * p.R + 4 * l; };
        if (axes.same) {
            set(p, __ldg(reinterpret_cast<const float4*>(row(0))), __ldg(reinterpret_cast<const float4*>(row(0) + half)), back);
        } else {
            const float *r0 = row(0), *r1 = row(1), *r2 = row(2), *r3 = row(3);
            const float4 c = make_float4(__ldg(r0), __ldg(r1 + 1), __ldg(r2 + 2), __ldg(r3 + 3));
            const float4 s = make_float4(__ldg(r0 + half), __ldg(r1 + half + 1), __ldg(r2 + half + 2), __ldg(r3 + half + 3));
            set(p, c, s, back);
        }
    }
    // The transposed rotation of token `token` of all, the s-th of its sequence.  False: a position is out of range (and reported).
    template <bool AXES>
    __device__ __forceinline__ bool load_token(const RopeParams& p, int64_t token, int s, const PairAxes& axes, int l, const Place& at) {
        bool ok = true;
        if constexpr (AXES) {
            AxisPositions pos;
            ok = pos.load(p, token);
            load_axes(p, pos, axes, l, at, true);
        } else {
            int pos = p.positions ? __ldg(p.positions + token) : s;
            if (p.R > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(p.table_len)) {
                ok = false;
                pos = 0;
            }
            load(p, pos, l, at, true);
        }
        if (!ok) report_bad_index(p.status);
        return ok;
    }
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int e = 0; e < 4; ++e) { cs[e] = F2(1.f, 1.f); sn[e] = F2(0.f, 0.f); }
    }
    __device__ __forceinline__ void set(const RopeParams& p, const float4& c, float4 s, bool back) {
        const float flip = back ? -1.f : 1.f;
        s.x *= flip; s.y *= flip; s.z *= flip; s.w *= flip;
        if (p.interleaved) {
            cs[0] = F2(c.x, c.x); cs[1] = F2(c.y, c.y); cs[2] = F2(c.z, c.z); cs[3] = F2(c.w, c.w);
            sn[0] = F2(-s.x, s.x); sn[1] = F2(-s.y, s.y); sn[2] = F2(-s.z, s.z); sn[3] = F2(-s.w, s.w);
        } else {
            cs[0] = cs[2] = F2(c.x, c.y);
            cs[1] = cs[3] = F2(c.z, c.w);
            sn[0] = F2(-s.x, -s.y); sn[1] = F2(-s.z, -s.w);
            sn[2] = F2(s.x, s.y); sn[3] = F2(s.z, s.w);
        }
    }
};

template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int off = LPR / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Where one token's rows go in the paged form.  Returns the position, or -1 when the token is not written (padding before the
// first sequence's new tokens or behind the last one's, or an entry that is out of range).
// AXES: the rotation has positions of its own.
template <bool AXES>
__device__ __forceinline__ int place_token(const RopeParams& p, int t, int& page, int& slot) {
    int seq, pos;
    if (p.cu_seqlens) {
        // last sequence that begins at or before t (empty sequences share a begin; the last of them is not empty or is the end)
        if (t < __ldg(p.cu_seqlens) || t >= __ldg(p.cu_seqlens + p.n_seqs)) return -1;
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
    if (pos < 0 || pos >= p.max_len || (!AXES && p.R > 0 && pos >= p.table_len)) {
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
template <int D, int DTYPE, bool PAGED, bool AXES>
__global__ void __launch_bounds__(kWarps * 32, 4)
attn_rope_kernel(const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPR, l = lane % LPR;
    const int token = blockIdx.x * kWarps + warp;
    if (token >= p.tokens) return;
    int b = 0, s = token;
    if constexpr (!PAGED) {
        b = static_cast<unsigned>(token) / static_cast<unsigned>(p.S);
        s = token - b * p.S;
    }
    const Place at(p, l);
    int u = blockIdx.y;
    // The rows of unit u: asked for before the position, the page and the rotation's factors, whose loads depend on one another.
    uint4 raw[kDeep];
    int left;                    // this lane's rows are those i with i * RPW < left
    auto load_unit = [&](int kind) {
        const int h0 = (u - (kind == 0 ? 0 : p.unit_end[kind - 1])) * (kDeep * RPW);
        left = p.heads[kind] - h0 - sub;
        const int64_t head = p.is[kind].head * 2;
        const uint8_t* src = static_cast<const uint8_t*>(p.in[kind]) + (b * p.is[kind].batch + s * p.is[kind].token) * 2 + (h0 + sub) * head;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if (i * RPW < left) raw[i] = load_row(src, at);
            src += RPW * head;
        }
    };
    load_unit(u < p.unit_end[0] ? 0 : (u < p.unit_end[1] ? 1 : 2));
    bool loaded = true;
    int pos, page = 0, slot = 0;
    float bad = 1.f;             // NaN: the token's q and k rows become NaN
    if constexpr (PAGED) {
        pos = place_token<AXES>(p, token, page, slot);
        if (pos < 0) return;
    } else if constexpr (!AXES) {
        pos = p.positions ? __ldg(p.positions + token) : s;
        if (p.R > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(p.table_len)) {
            report_bad_index(p.status);
            bad = __int_as_float(0x7fffffff);
            pos = 0;
        }
    }
    AxisPositions axis_pos;
    const PairAxes axes = PairAxes::of_lane<AXES>(p, l);
    if constexpr (AXES) {
        if (!axis_pos.load(p, token)) {
            report_bad_index(p.status);
            if (PAGED) return;   // skipped, like a token whose place in the cache is out of range
            bad = __int_as_float(0x7fffffff);
        }
    }
#pragma unroll
    for (int kind = 0; kind < 3; ++kind) {
        if (u >= p.unit_end[kind]) continue;
        if (!loaded) load_unit(kind);
        const bool cache = PAGED && kind > 0, norm = kind < 2 && p.weight[kind] != nullptr;
        const int64_t dst_head = p.os[kind].head * 2;
        uint8_t* dst0 = static_cast<uint8_t*>(p.out[kind]) + sub * dst_head +
                        (cache ? page * p.os[kind].batch + slot * p.os[kind].token : b * p.os[kind].batch + s * p.os[kind].token) * 2;
        Turn f;                  // the rotation with the weights folded in
        if (kind < 2) {
            if constexpr (AXES) f.load_axes(p, axis_pos, axes, l, at, false); else f.load(p, pos, l, at, false);
            if (norm) {
                F2 w[4];
                load_weight<DTYPE>(p.weight[kind], p.weight_f32, at, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f.cs[e] = f.cs[e] * w[e];
                    f.sn[e] = f.sn[e] * (p.interleaved ? partner<true>(w, e) : partner<false>(w, e));
                }
            }
        }
        for (;;) {
            if (kind < 2)
                by_form(p, D, [&](auto inter, auto whole_head) {
#pragma unroll
                    for (int i = 0; i < kDeep; ++i) {
                        if (i * RPW >= left + sub) break;      // uniform over the warp
                        F2 x[4], y[4];
                        unpack_row<DTYPE>(raw[i], x);
                        float r = bad;
                        if (norm) {
                            F2 ss = x[0] * x[0];
#pragma unroll
                            for (int e = 1; e < 4; ++e) ss = fma2(x[e], x[e], ss);
                            r *= rsqrtf(row_sum<LPR>(ss.sum()) * (1.f / D) + p.eps);
                        }
                        turn_values<decltype(inter)::value, decltype(whole_head)::value>(y, x, f.cs, f.sn, at.turns);
                        const F2 rr(r, r);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = y[e] * rr;
                        raw[i] = pack_row<DTYPE>(y);
                    }
                });
            uint8_t* dst = dst0 + (u - (kind == 0 ? 0 : p.unit_end[kind - 1])) * (kDeep * RPW) * dst_head;
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                if (i * RPW < left) store_row(dst, at, raw[i]);
                dst += RPW * dst_head;
            }
            u += gridDim.y;
            if (u >= p.unit_end[kind]) break;
            load_unit(kind);
        }
        loaded = false;
    }
}

// Gradient.  dy: head-major gradients of the outputs; in: q, k as the forward pass read them; out: gradients laid out like
// the inputs.  One wave of blocks, shared out between q and (k, v) by their bytes; an item is a token and kDeep x
// rows-per-warp of its heads, eight neighbouring tokens to a block, so that even a few thousand tokens are many items per
// warp (with whole tokens as items the last round is mostly empty); 70 us for 4 x 2048 tokens x 48 heads of 128.  A warp
// keeps the weight gradients of its rows in registers; each block leaves its sum in `partial`, and
// attn_rope_weight_grad_kernel adds those in a fixed order.
template <int D, int DTYPE, bool AXES>
__global__ void __launch_bounds__(kWarps * 32, kBwdBlocks)
attn_rope_bwd_kernel(const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    __shared__ float sums[kWarps * RPW][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPR, l = lane % LPR;
    const Place at(p, l);
    const PairAxes axes = PairAxes::of_lane<AXES>(p, l);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const bool is_q = static_cast<int>(blockIdx.x) < p.q_blocks;
    const unsigned block = is_q ? blockIdx.x : blockIdx.x - p.q_blocks, blocks = is_q ? p.q_blocks : gridDim.x - p.q_blocks;
    for (int kind = is_q ? 0 : 1; kind < (is_q ? 1 : 3); ++kind) {
        const int heads = p.heads[kind];
        const unsigned units = (heads + kDeep * RPW - 1) / (kDeep * RPW);
        const bool norm = kind < 2 && p.weight[kind] != nullptr;
        const int64_t g_head = p.ds[kind].head * 2, x_head = p.is[kind].head * 2, o_head = p.os[kind].head * 2;
        F2 dw[4], w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[e] = w[e] = F2(0.f, 0.f);
        if (norm) load_weight<DTYPE>(p.weight[kind], p.weight_f32, at, w);
        const unsigned items = static_cast<unsigned>((p.tokens + kWarps - 1) / kWarps) * units;      // of eight tokens, one per warp
        for (unsigned item = block; item < items; item += blocks) {
            const unsigned eight = item / units;
            const int token = eight * kWarps + warp, h0 = (item - eight * units) * (kDeep * RPW);
            if (token >= p.tokens) continue;
            const int b = static_cast<unsigned>(token) / static_cast<unsigned>(p.S), s = token - b * p.S;
            const int left = heads - h0 - sub;
            const uint8_t* gsrc = static_cast<const uint8_t*>(p.dy[kind]) + (b * p.ds[kind].batch + s * p.ds[kind].token) * 2 + (h0 + sub) * g_head;
            const uint8_t* xsrc = static_cast<const uint8_t*>(p.in[kind]) + (b * p.is[kind].batch + s * p.is[kind].token) * 2 + (h0 + sub) * x_head;
            uint8_t* dst = static_cast<uint8_t*>(p.out[kind]) + (b * p.os[kind].batch + s * p.os[kind].token) * 2 + (h0 + sub) * o_head;
            uint4 gr[kDeep], xr[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                gr[i] = xr[i] = make_uint4(0u, 0u, 0u, 0u);
                if (i * RPW < left) {
                    gr[i] = load_row(gsrc, at);
                    if (norm) xr[i] = load_row(xsrc, at);
                }
                gsrc += RPW * g_head;
                xsrc += RPW * x_head;
            }
            Turn turn;
            if (kind < 2) {
                const bool bad = !turn.load_token<AXES>(p, token, s, axes, l, at);
                if (bad) {       // the token's gradients, and with them the weights', become NaN
#pragma unroll
                    for (int e = 0; e < 4; ++e) turn.cs[e] = F2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
                }
            }
            if (kind < 2)
                by_form(p, D, [&](auto inter, auto whole_head) {
#pragma unroll
                    for (int i = 0; i < kDeep; ++i) {
                        if (i * RPW >= left + sub) break;      // uniform over the warp
                        F2 g[4], h[4];       // h: g, turned back
                        unpack_row<DTYPE>(gr[i], g);
                        turn_values<decltype(inter)::value, decltype(whole_head)::value>(h, g, turn.cs, turn.sn, at.turns);
                        if (norm) {
                            F2 x[4], hx[4], ss(0.f, 0.f), gx(0.f, 0.f);
                            unpack_row<DTYPE>(xr[i], x);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                ss = fma2(x[e], x[e], ss);
                                hx[e] = h[e] * x[e];
                                gx = fma2(hx[e], w[e], gx);
                            }
                            const float r = rsqrtf(row_sum<LPR>(ss.sum()) * (1.f / D) + p.eps);
                            const float k = -row_sum<LPR>(gx.sum()) * (1.f / D) * r * r * r;
                            // (lanes past the last head hold zeros in x and g: at eps 0 their r is infinite)
                            const float rd = i * RPW < left ? r : 0.f;
                            const F2 rr(r, r), kk(k, k), rrd(rd, rd);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                dw[e] = fma2(hx[e], rrd, dw[e]);
                                h[e] = fma2(h[e], w[e] * rr, kk * x[e]);
                            }
                        }
                        gr[i] = pack_row<DTYPE>(h);
                    }
                });
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                if (i * RPW < left) store_row(dst, at, gr[i]);
                dst += RPW * o_head;
            }
        }
        if (kind < 2) {
            float* mine = sums[warp * RPW + sub];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                dw[e].get(mine[at.a + 2 * e], mine[at.a + 2 * e + 1]);
                dw[2 + e].get(mine[at.b + 2 * e], mine[at.b + 2 * e + 1]);
            }
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += kWarps * 32) {
                float x = 0.f;
#pragma unroll
                for (int r = 0; r < kWarps * RPW; ++r) x += sums[r][d];
                p.partial[static_cast<int64_t>(blockIdx.x) * D + d] = x;
            }
            __syncthreads();
        }
    }
}

// dq_weight, dk_weight [D] fp32 from the blocks' sums: q's are nq rows from q_sums, k's nk rows from k_sums, `stride` floats
// apart.  32 columns of one of them per block, 32 warps.
__global__ void __launch_bounds__(1024)
attn_rope_weight_grad_kernel(const float* q_sums, int nq, const float* k_sums, int nk, int stride, int D, float* dqw, float* dkw) {
    __shared__ float sums[32][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool is_q = static_cast<int>(blockIdx.x) * 32 < D;
    const int col = blockIdx.x * 32 + lane - (is_q ? 0 : D);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float* from = (is_q ? q_sums : k_sums) + col;
    const int n = is_q ? nq : nk;
    float x = 0.f;
#pragma unroll 4
    for (int r = warp; r < n; r += 32) x += __ldcg(from + static_cast<int64_t>(r) * stride);
    sums[warp][lane] = x;
    __syncthreads();
    if (warp == 0) {
        x = 0.f;
#pragma unroll
        for (int w = 0; w < 32; ++w) x += sums[w][lane];
        float* out = is_q ? dqw : dkw;
        if (out) out[col] = x;
    }
}

}  // namespace attn_rope
