// C ABI of the operators around the attention kernels (declared in include/attn_fwd.h): sliding windows, normalisation and
// rotation of queries and keys, the paged cache.  Included at the end of attn_api.cu; host-side validation and launches only.

namespace {

#ifdef ATTN_TEST_HOOKS
int g_test_skip_step = -1;
#endif

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

bool misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// The status word's address, looked up once per device.
int* cached_status_ptr() {
    static std::mutex mu;
    static int* ptr[kMaxDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!ptr[dev]) ptr[dev] = device_status_ptr();
    return ptr[dev];
}

bool strides_ok(const long long* s, int n) {
    for (int i = 0; i < n; ++i)
        if (s[i] % 8 != 0) return false;
    return true;
}

bool head_dim_ok(int D) { return D == 64 || D == 128 || D == 256; }
bool dtype_ok(int dtype) { return dtype == ATTN_DTYPE_FP16 || dtype == ATTN_DTYPE_BF16; }

constexpr int kRopeBwdBlocks = 148 * attn_rope::kBwdBlocks;   // blocks of the gradient kernel at most: one wave (each leaves D partial sums)

// What the three entry points of the rotation share.
int validate_rope(const void* q_weight, const void* k_weight, const float* cos_sin, int table_len, int R, float eps, int D, int dtype) {
    if (!head_dim_ok(D)) return ATTN_ERR_UNSUPPORTED_HEAD_DIM;
    if (!dtype_ok(dtype)) return ATTN_ERR_UNSUPPORTED_DTYPE;
    if (R < 0 || R > D || R % 16 != 0 || (R > 0 && table_len < 1)) return ATTN_ERR_BAD_SHAPE;
    if (R > 0 && !cos_sin) return ATTN_ERR_NULL_POINTER;
    if (misaligned(q_weight, 16) || misaligned(k_weight, 16) || (R > 0 && misaligned(cos_sin, 16))) return ATTN_ERR_MISALIGNED;
    if (!isfinite(eps) || eps < 0.f) return ATTN_ERR_BAD_SCALE;
    return ATTN_OK;
}

int validate_cache(const void* k_cache, const void* v_cache, const long long* cache_strides, int num_pages, int page_size,
                   const int* block_table, int max_pages, const int* seq_lens) {
    if (num_pages < 0 || max_pages < 0 || page_size < 1 || (page_size & (page_size - 1)) != 0) return ATTN_ERR_BAD_SHAPE;
    if (static_cast<int64_t>(max_pages) * page_size > 2147483647LL) return ATTN_ERR_BAD_SHAPE;
    if (!cache_strides || !seq_lens || (max_pages > 0 && !block_table) || (num_pages > 0 && (!k_cache || !v_cache))) return ATTN_ERR_NULL_POINTER;
    if (misaligned(k_cache, 16) || misaligned(v_cache, 16) || !strides_ok(cache_strides, 6)) return ATTN_ERR_MISALIGNED;
    if (misaligned(block_table, 4) || misaligned(seq_lens, 4)) return ATTN_ERR_MISALIGNED;
    return ATTN_OK;
}

// log2 of the heads that a tile of the decode kernel covers side by side: all warps' worth where the number of heads has that
// power of two, else as many as it has.
int tile_heads_shift(int64_t heads, int D) {
    const int warps = D == 256 ? 4 : 8;
    int s = 0;
    while ((2 << s) <= warps && heads % (2 << s) == 0) ++s;
    return s;
}

// Rank-4 tensor map of 16-bit elements: D contiguous columns, then three axes of n[i] elements at stride[i] (in elements, any
// order); box[0] columns, box[1 + i] of axis i.  A map is a pure function of these arguments; encoded maps are kept in a small
// per-thread cache, as a training or serving loop passes the same tensors again (see make_map).
struct Map4Key {
    const void* base;
    int64_t stride[3];
    int dtype, D, n[3], box[4], swizzle;
    bool operator==(const Map4Key& o) const {
        bool same = base == o.base && dtype == o.dtype && D == o.D && box[0] == o.box[0] && swizzle == o.swizzle;
        for (int i = 0; i < 3; ++i) same = same && stride[i] == o.stride[i] && n[i] == o.n[i] && box[1 + i] == o.box[1 + i];
        return same;
    }
};

// Strides that a map can have: above 0 (an axis of one element may have any) and, in bytes, below 2^40.
bool mappable(const int64_t* stride, const int* n) {
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (stride[i] <= 0 || stride[i] >= (1LL << 39))) return false;
    return true;
}

bool make_map4(CUtensorMap* map, const Map4Key& key) {
    struct Entry {
        bool valid = false;
        Map4Key key;
        CUtensorMap map;
    };
    constexpr int kEntries = 256;
    thread_local Entry cache[kEntries];
    const uint64_t h = ((reinterpret_cast<uintptr_t>(key.base) >> 7) + static_cast<uint64_t>(key.stride[0] + 3 * key.stride[1]) * 31 + key.n[0]) *
                       0x9E3779B97F4A7C15ull;
    Entry& e = cache[(h >> 40) % kEntries];
    if (!e.valid || !(e.key == key)) {
        EncodeTiledFn enc = get_encode_fn();
        if (!enc) return false;
        cuuint64_t dims[4] = {static_cast<cuuint64_t>(key.D)}, strides[3];
        cuuint32_t box[4] = {static_cast<cuuint32_t>(key.box[0])}, estr[4] = {1, 1, 1, 1};
        for (int i = 0; i < 3; ++i) {
            dims[1 + i] = static_cast<cuuint64_t>(key.n[i]);
            strides[i] = static_cast<cuuint64_t>(key.n[i] > 1 ? key.stride[i] : key.D) * 2;
            box[1 + i] = static_cast<cuuint32_t>(key.box[1 + i]);
        }
        const CUtensorMapDataType type = key.dtype == ATTN_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
        e.valid = enc(&e.map, type, 4, const_cast<void*>(key.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      key.swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
        if (!e.valid) return false;
        e.key = key;
    }
    *map = e.map;
    return true;
}

// Map over one cache for the decode kernel: the slot, head and page axes by ascending stride; box = 64 columns x `rows` slots,
// 128-byte swizzle.  `axes` receives the coordinate number of the slot, head and page axis (2 bits each).
bool make_cache_map(CUtensorMap* map, int* axes, const void* base, const long long* cache_strides, int dtype, int D, int num_pages, int Hkv,
                    int page_size, int rows) {
    const int64_t stride[3] = {cache_strides[2], cache_strides[1], cache_strides[0]};     // slot, head, page
    const int n[3] = {page_size, Hkv, num_pages};
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (stride[order[j]] > stride[order[j + 1]]) {
                const int x = order[j];
                order[j] = order[j + 1];
                order[j + 1] = x;
            }
    Map4Key key{base, {}, dtype, D, {}, {64, 1, 1, 1}, 1};
    *axes = 0;
    for (int i = 0; i < 3; ++i) {
        key.stride[i] = stride[order[i]];
        key.n[i] = n[order[i]];
        if (order[i] == 0) key.box[1 + i] = rows;
        *axes |= (i + 1) << (2 * order[i]);
    }
    return make_map4(map, key);
}

// Tokens, and items of a token and a few heads, are counted in 32 bits (more would not fit any GPU's memory).
bool rope_tokens_ok(int64_t tokens, int H, int Hkv) {
    return tokens < (1LL << 31) - 64 && H < (1 << 20) && Hkv < (1 << 20) && (tokens / 8 + 1) * ((H > Hkv ? H : Hkv) / 4 + 1) < (1LL << 32);
}

void rope_units(attn_rope::RopeParams& p, int D) {
    const int per = attn_rope::kDeep * (256 / D);
    int end = 0;
    for (int i = 0; i < 3; ++i) {
        end += (p.heads[i] + per - 1) / per;
        p.unit_end[i] = end;
    }
}

template <bool PAGED>
int launch_rope(attn_rope::RopeParams& p, int D, int dtype, cudaStream_t st) {
    rope_units(p, D);
    if (p.tokens == 0 || p.unit_end[2] == 0) return ATTN_OK;
    const int64_t gx = (static_cast<int64_t>(p.tokens) + attn_rope::kWarps - 1) / attn_rope::kWarps;
    // few tokens: their heads are spread over blocks until the GPU has eight blocks per SM
    int64_t gy = (148 * 8 + gx - 1) / gx;
    if (gy > p.unit_end[2]) gy = p.unit_end[2];
    if (gy > 65535) gy = 65535;
    const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>(gy));
#define ATTN_ROPE_CASE(DD, TT) \
    if (D == DD && dtype == TT) attn_rope::attn_rope_kernel<DD, TT, PAGED><<<grid, attn_rope::kWarps * 32, 0, st>>>(p);
    ATTN_ROPE_CASE(64, 0)
    ATTN_ROPE_CASE(64, 1)
    ATTN_ROPE_CASE(128, 0)
    ATTN_ROPE_CASE(128, 1)
    ATTN_ROPE_CASE(256, 0)
    ATTN_ROPE_CASE(256, 1)
#undef ATTN_ROPE_CASE
    return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

// The TMA form of the gradient.  *launched false: a stride that a tensor map cannot have (0, for a broadcast input), the caller
// takes the register form.  p: as for that form.
int launch_rope_bwd_tma(const attn_rope::RopeParams& p, int B, int D, int dtype, cudaStream_t st, bool* launched, int* ctas) {
    *launched = false;
    const int most = log2_of(1024 / D);      // log2 of the heads of a tile of 8 tokens
    attn_rope::TmaMaps maps;
    attn_rope::TmaParams tp = {};
    tp.r = p;
    tp.partial = p.partial;
#ifdef ATTN_TEST_HOOKS
    tp.test_skip_tile = g_test_skip_step;
    g_test_skip_step = -1;
#endif
    tp.block_shift = 3;
    for (int i = 0; i < 3; ++i) {
        int hb = 0;
        while (hb < most && (1 << hb) < p.heads[i]) ++hb;
        tp.hb_shift[i] = hb;
        tp.tb_shift[i] = 3 + most - hb;
        tp.units[i] = (p.heads[i] + (1 << hb) - 1) >> hb;
        if (p.heads[i] == 0) continue;
        if (tp.tb_shift[i] > tp.block_shift) tp.block_shift = tp.tb_shift[i];
        const int n[3] = {p.S, p.heads[i], B}, box_t = 1 << tp.tb_shift[i], box_h = 1 << hb;
        auto make = [&](CUtensorMap* map, const void* base, const attn_rope::Strides& s) {
            const Map4Key key{base, {s.token, s.head, s.batch}, dtype, D, {n[0], n[1], n[2]}, {D, box_t, box_h, 1}, 0};
            return mappable(key.stride, n) && make_map4(map, key);
        };
        if (!make(&maps.dy[i], p.dy[i], p.ds[i]) || !make(&maps.out[i], p.out[i], p.os[i])) return ATTN_OK;
        if (i < 2 && p.weight[i] && !make(&maps.x[i], p.in[i], p.is[i])) return ATTN_OK;
    }
    const bool packed = (p.heads[0] > 0 && tp.tb_shift[0] != 3) || (p.heads[1] > 0 && tp.tb_shift[1] != 3);
    tp.token_blocks = static_cast<int>((static_cast<int64_t>(p.S) + (1 << tp.block_shift) - 1) >> tp.block_shift);
    for (int i = 0; i < 3; ++i)
        if (p.heads[i] > 0) tp.per_block += tp.units[i] << (tp.block_shift - tp.tb_shift[i]);
    DeviceInfo di;
    if (device_info(&di) != ATTN_OK) return ATTN_ERR_CUDA;
    tp.tiles = static_cast<int64_t>(B) * tp.token_blocks * tp.per_block;
    if (tp.tiles / di.sm_count >= 2147483647LL) return ATTN_OK;
    int grid = di.sm_count < kRopeBwdBlocks / 2 ? di.sm_count : kRopeBwdBlocks / 2;      // (a CTA leaves 2 D partial sums)
    if (tp.tiles < grid) grid = static_cast<int>(tp.tiles);
    *ctas = grid;
#define ATTN_ROPE_CASE(DD, TT)                                                                                       \
    if (D == DD && dtype == TT) {                                                                                     \
        using C = attn_rope::TmaCfg<DD>;                                                                              \
        auto kern = packed ? attn_rope::attn_rope_bwd_tma_kernel<DD, TT, true> : attn_rope::attn_rope_bwd_tma_kernel<DD, TT, false>; \
        if (!allow_dynamic_smem(reinterpret_cast<const void*>(kern), C::SMEM)) return ATTN_ERR_CUDA;                  \
        kern<<<grid, C::THREADS, C::SMEM, st>>>(maps, tp);                                                            \
    }
    ATTN_ROPE_CASE(64, 0)
    ATTN_ROPE_CASE(64, 1)
    ATTN_ROPE_CASE(128, 0)
    ATTN_ROPE_CASE(128, 1)
    ATTN_ROPE_CASE(256, 0)
    ATTN_ROPE_CASE(256, 1)
#undef ATTN_ROPE_CASE
    *launched = true;
    return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

// The row strides of [B, heads, S, D], contiguous.
attn_rope::Strides head_major(int heads, int S, int D) {
    return attn_rope::Strides{static_cast<int64_t>(heads) * S * D, D, static_cast<int64_t>(S) * D};
}

// The window arguments: window 0 stands for one without an end.
int validate_window(int Sq, int* window, int sinks, int q_offset) {
    if (*window < 0 || sinks < 0 || q_offset < 0 || static_cast<int64_t>(q_offset) + (Sq > 0 ? Sq : 0) > kMaxSeq) return ATTN_ERR_BAD_SHAPE;
    if (*window == 0) *window = 2147483647;
    return ATTN_OK;
}


}  // namespace

extern "C" {

#ifdef ATTN_TEST_HOOKS
// Test build only (never part of libattn_fwd.so): the next launch of the decode kernel (of the rotation's gradient) leaves out the
// copies of this step of every warp (tile of every CTA), so that the wait for them runs out.
void attn_test_skip_step(int step) { g_test_skip_step = step; }
#endif

int attn_fwd_window(const void* q, const void* k, const void* v, void* o, float* lse, int B, int H, int Hkv, int Sq, int Sk,
                    int D, float scale, int window, int sinks, int q_offset, int dtype, void* stream) {
    if (D != 64 && D != 128) {
        if (B < 0 || H < 0 || Hkv < 0 || Sq < 0 || Sk < 0 || D < 0) return ATTN_ERR_BAD_SHAPE;
        return ATTN_ERR_UNSUPPORTED_HEAD_DIM;
    }
    int rc = validate(q, k, v, o, lse, B, H, Hkv, Sq, Sk, D, scale, dtype, true);
    if (rc == ATTN_OK) rc = validate_window(Sq, &window, sinks, q_offset);
    if (rc != ATTN_OK) return rc;
    if (static_cast<int64_t>(B) * H * Sq == 0) return ATTN_OK;
    rc = check_arch();
    if (rc != ATTN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (Sk == 0) return fill_empty(o, lse, static_cast<int64_t>(B) * H * Sq * D, static_cast<int64_t>(B) * H * Sq, st);
#define ATTN_WINDOW_CASE(DD, TT) \
    if (D == DD && dtype == TT)  \
        return launch_tc_pipe<DD, TT, true>(q, k, v, o, lse, B, H, Hkv, Sq, Sk, scale, 1, -q_offset, st, 1.f, -1, 1, window, sinks);
    ATTN_WINDOW_CASE(64, 0)
    ATTN_WINDOW_CASE(64, 1)
    ATTN_WINDOW_CASE(128, 0)
    ATTN_WINDOW_CASE(128, 1)
#undef ATTN_WINDOW_CASE
    return ATTN_ERR_UNSUPPORTED_DTYPE;
}

size_t attn_bwd_window_workspace_bytes(int B, int H, int Hkv, int Sq, int Sk, int D, int window, int sinks, int q_offset) {
    if (B < 0 || H < 0 || Hkv < 0 || Sq < 0 || Sk < 0 || D < 0 || (H > 0 && (Hkv == 0 || H % Hkv != 0))) return 0;
    if (validate_window(Sq, &window, sinks, q_offset) != ATTN_OK) return 0;
    return attn_bwd_workspace_bytes(B, H, Sq) + sink_plan(B, H, Hkv, Sq, Sk, D, window, sinks, q_offset).part_floats * sizeof(float);
}

int attn_bwd_window(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* dout, void* dq,
                    void* dk, void* dv, int B, int H, int Hkv, int Sq, int Sk, int D, float scale, int window, int sinks,
                    int q_offset, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = validate_window(Sq, &window, sinks, q_offset);
    if (rc != ATTN_OK) return rc;
    return bwd<true>(q, k, v, o, lse, dout, dq, dk, dv, B, H, Hkv, Sq, Sk, D, scale, 1, dtype, workspace, workspace_bytes, stream,
                     window, sinks, q_offset);
}

int attn_qk_norm_rope(const void* q, const void* k, const void* v, const long long* in_strides, const void* q_weight,
                      const void* k_weight, int weight_f32, const float* cos_sin, int table_len, int R, int interleaved,
                      const int* positions, float eps, void* q_out, void* k_out, void* v_out, int B, int S, int H, int Hkv,
                      int D, int dtype, void* stream) {
    if (B < 0 || S < 0 || H < 0 || Hkv < 0 || S > kMaxSeq) return ATTN_ERR_BAD_SHAPE;
    int rc = validate_rope(q_weight, k_weight, cos_sin, table_len, R, eps, D, dtype);
    if (rc != ATTN_OK) return rc;
    if (R > 0 && !positions && S > table_len) return ATTN_ERR_BAD_SHAPE;
    const int64_t tokens = static_cast<int64_t>(B) * S;
    if (tokens == 0 || (H == 0 && Hkv == 0)) return ATTN_OK;
    if (!rope_tokens_ok(tokens, H, Hkv)) return ATTN_ERR_BAD_SHAPE;
    if (!in_strides || (H > 0 && (!q || !q_out)) || (Hkv > 0 && (!k || !k_out || !v != !v_out))) return ATTN_ERR_NULL_POINTER;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(q_out, 16) || misaligned(k_out, 16) ||
        misaligned(v_out, 16) || misaligned(positions, 4) || !strides_ok(in_strides, 9))
        return ATTN_ERR_MISALIGNED;
    rc = check_arch();
    if (rc != ATTN_OK) return rc;
    attn_rope::RopeParams p = {};
    const void* in[3] = {q, k, v};
    void* out[3] = {q_out, k_out, v_out};
    const int heads[3] = {H, Hkv, v ? Hkv : 0};
    for (int i = 0; i < 3; ++i) {
        p.in[i] = in[i];
        p.out[i] = out[i];
        p.heads[i] = heads[i];
        p.is[i] = attn_rope::Strides{in_strides[3 * i], in_strides[3 * i + 1], in_strides[3 * i + 2]};
        p.os[i] = head_major(heads[i], S, D);
    }
    p.weight[0] = q_weight;
    p.weight[1] = k_weight;
    p.weight_f32 = weight_f32;
    p.table = cos_sin;
    p.table_len = table_len;
    p.R = R;
    p.interleaved = interleaved;
    p.positions = positions;
    p.eps = eps;
    p.tokens = static_cast<int>(tokens);
    p.S = S;
    p.status = cached_status_ptr();
    if (!p.status) return ATTN_ERR_CUDA;
    return launch_rope<false>(p, D, dtype, static_cast<cudaStream_t>(stream));
}

size_t attn_qk_norm_rope_bwd_workspace_bytes(int D) {
    return head_dim_ok(D) ? static_cast<size_t>(kRopeBwdBlocks) * D * sizeof(float) : 0;
}

int attn_qk_norm_rope_bwd(const void* dq, const void* dk, const void* dv, const void* q, const void* k,
                          const long long* in_strides, const void* q_weight, const void* k_weight, int weight_f32,
                          const float* cos_sin, int table_len, int R, int interleaved, const int* positions, float eps,
                          void* dq_in, void* dk_in, void* dv_in, const long long* out_strides, float* dq_weight,
                          float* dk_weight, int B, int S, int H, int Hkv, int D, int dtype, void* workspace,
                          size_t workspace_bytes, void* stream) {
    if (B < 0 || S < 0 || H < 0 || Hkv < 0 || S > kMaxSeq) return ATTN_ERR_BAD_SHAPE;
    int rc = validate_rope(q_weight, k_weight, cos_sin, table_len, R, eps, D, dtype);
    if (rc != ATTN_OK) return rc;
    if (R > 0 && !positions && S > table_len) return ATTN_ERR_BAD_SHAPE;
    const int64_t tokens = static_cast<int64_t>(B) * S;
    if (!rope_tokens_ok(tokens, H, Hkv)) return ATTN_ERR_BAD_SHAPE;
    if ((q_weight && !dq_weight) || (k_weight && !dk_weight)) return ATTN_ERR_NULL_POINTER;
    if (misaligned(dq_weight, 4) || misaligned(dk_weight, 4)) return ATTN_ERR_MISALIGNED;
    if (tokens > 0) {
        if (!in_strides || !out_strides) return ATTN_ERR_NULL_POINTER;
        if (H > 0 && (!dq || !dq_in || (q_weight && !q))) return ATTN_ERR_NULL_POINTER;
        if (Hkv > 0 && (!dk || !dk_in || (k_weight && !k) || !dv != !dv_in)) return ATTN_ERR_NULL_POINTER;
        if (misaligned(dq, 16) || misaligned(dk, 16) || misaligned(dv, 16) || misaligned(q, 16) || misaligned(k, 16) ||
            misaligned(dq_in, 16) || misaligned(dk_in, 16) || misaligned(dv_in, 16) || misaligned(positions, 4) ||
            !strides_ok(in_strides, 6) || !strides_ok(out_strides, 9))
            return ATTN_ERR_MISALIGNED;
        const int heads[3] = {H, Hkv, dv ? Hkv : 0};
        for (int i = 0; i < 3; ++i) {   // an output whose rows lie on top of each other
            const long long* s = out_strides + 3 * i;
            if (heads[i] > 0 && ((B > 1 && s[0] == 0) || (S > 1 && s[1] == 0) || (heads[i] > 1 && s[2] == 0))) return ATTN_ERR_BAD_SHAPE;
        }
    }
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < attn_qk_norm_rope_bwd_workspace_bytes(D)) return ATTN_ERR_WORKSPACE;
    rc = check_arch();
    if (rc != ATTN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0 || (H == 0 && Hkv == 0)) {
        if (dq_weight && cudaMemsetAsync(dq_weight, 0, D * sizeof(float), st) != cudaSuccess) return ATTN_ERR_CUDA;
        if (dk_weight && cudaMemsetAsync(dk_weight, 0, D * sizeof(float), st) != cudaSuccess) return ATTN_ERR_CUDA;
        return ATTN_OK;
    }
    attn_rope::RopeParams p = {};
    const void* in[3] = {q, k, nullptr};
    const void* dy[3] = {dq, dk, dv};
    void* out[3] = {dq_in, dk_in, dv_in};
    const int heads[3] = {H, Hkv, dv ? Hkv : 0};
    for (int i = 0; i < 3; ++i) {
        p.in[i] = in[i];
        p.dy[i] = dy[i];
        p.out[i] = out[i];
        p.heads[i] = heads[i];
        if (i < 2) p.is[i] = attn_rope::Strides{in_strides[3 * i], in_strides[3 * i + 1], in_strides[3 * i + 2]};
        p.os[i] = attn_rope::Strides{out_strides[3 * i], out_strides[3 * i + 1], out_strides[3 * i + 2]};
        p.ds[i] = head_major(heads[i], S, D);
    }
    p.weight[0] = q_weight;
    p.weight[1] = k_weight;
    p.weight_f32 = weight_f32;
    p.table = cos_sin;
    p.table_len = table_len;
    p.R = R;
    p.interleaved = interleaved;
    p.positions = positions;
    p.eps = eps;
    p.tokens = static_cast<int>(tokens);
    p.S = S;
    p.partial = static_cast<float*>(workspace);
    p.status = cached_status_ptr();
    if (!p.status) return ATTN_ERR_CUDA;
    bool launched;
    int ctas;
    rc = launch_rope_bwd_tma(p, B, D, dtype, st, &launched, &ctas);
    if (rc != ATTN_OK) return rc;
    const bool sums = dq_weight || dk_weight;
    if (launched)
        return !sums || launch_dependent(attn_rope::attn_rope_weight_grad_kernel, dim3(2 * D / 32), dim3(1024), 0, st, p.partial, ctas,
                                         p.partial + D, ctas, 2 * D, D, dq_weight, dk_weight)
                   ? ATTN_OK
                   : ATTN_ERR_CUDA;
    // blocks of q and of (k, v): by their bytes (a row of q or k is read twice and written, of v read and written), each at
    // least one where it has heads, and no more than it has items
    const int per_unit = attn_rope::kDeep * (256 / D);
    const int64_t steps = (tokens + attn_rope::kWarps - 1) / attn_rope::kWarps;
    const int64_t q_items = steps * ((H + per_unit - 1) / per_unit), k_items = steps * ((Hkv + per_unit - 1) / per_unit);
    const double q_cost = 3.0 * H, kv_cost = (dv ? 5.0 : 3.0) * Hkv;
    int64_t q_blocks = H == 0 ? 0 : static_cast<int64_t>(kRopeBwdBlocks * q_cost / (q_cost + kv_cost) + 0.5);
    if (H > 0 && q_blocks < 1) q_blocks = 1;
    if (Hkv > 0 && q_blocks > kRopeBwdBlocks - 1) q_blocks = kRopeBwdBlocks - 1;
    int64_t kv_blocks = Hkv == 0 ? 0 : kRopeBwdBlocks - q_blocks;
    if (q_blocks > q_items) q_blocks = q_items;
    if (kv_blocks > k_items) kv_blocks = k_items;
    const int64_t blocks = q_blocks + kv_blocks;
    p.q_blocks = static_cast<int>(q_blocks);
#define ATTN_ROPE_CASE(DD, TT) \
    if (D == DD && dtype == TT) attn_rope::attn_rope_bwd_kernel<DD, TT><<<static_cast<unsigned>(blocks), attn_rope::kWarps * 32, 0, st>>>(p);
    ATTN_ROPE_CASE(64, 0)
    ATTN_ROPE_CASE(64, 1)
    ATTN_ROPE_CASE(128, 0)
    ATTN_ROPE_CASE(128, 1)
    ATTN_ROPE_CASE(256, 0)
    ATTN_ROPE_CASE(256, 1)
#undef ATTN_ROPE_CASE
    if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
    return !sums || launch_dependent(attn_rope::attn_rope_weight_grad_kernel, dim3(2 * D / 32), dim3(1024), 0, st, p.partial, p.q_blocks,
                                     p.partial + static_cast<int64_t>(p.q_blocks) * D, static_cast<int>(kv_blocks), D, D, dq_weight,
                                     dk_weight)
               ? ATTN_OK
               : ATTN_ERR_CUDA;
}

int attn_paged_append(const void* q, const void* k, const void* v, const long long* in_strides, const void* q_weight,
                      const void* k_weight, int weight_f32, const float* cos_sin, int table_len, int R, int interleaved,
                      float eps, void* q_out, void* k_cache, void* v_cache, const long long* cache_strides, int num_pages,
                      int page_size, const int* block_table, long long table_stride, int max_pages, const int* seq_lens,
                      const int* cu_seqlens, int n_seqs, int tokens, int H, int Hkv, int D, int dtype, void* stream) {
    if (n_seqs < 0 || tokens < 0 || H < 0 || Hkv < 0 || (!cu_seqlens && tokens != n_seqs)) return ATTN_ERR_BAD_SHAPE;
    int rc = validate_rope(q_weight, k_weight, cos_sin, table_len, R, eps, D, dtype);
    if (rc != ATTN_OK) return rc;
    if (tokens == 0 || n_seqs == 0 || (H == 0 && Hkv == 0)) return ATTN_OK;
    if (!in_strides || !q != !q_out || (Hkv > 0 && (!k || !v)) || (H > 0 && !q && Hkv == 0)) return ATTN_ERR_NULL_POINTER;
    rc = validate_cache(k_cache, v_cache, cache_strides, num_pages, page_size, block_table, max_pages, seq_lens);
    if (rc != ATTN_OK) return rc;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(q_out, 16) || misaligned(cu_seqlens, 4) ||
        !strides_ok(in_strides, 6))
        return ATTN_ERR_MISALIGNED;
    for (int i = 0; i < 2; ++i) {   // cache rows that lie on top of each other
        const long long* s = cache_strides + 3 * i;
        if (Hkv > 0 && ((num_pages > 1 && s[0] == 0) || (Hkv > 1 && s[1] == 0) || (page_size > 1 && s[2] == 0))) return ATTN_ERR_BAD_SHAPE;
    }
    rc = check_arch();
    if (rc != ATTN_OK) return rc;
    attn_rope::RopeParams p = {};
    const void* in[3] = {q, k, v};
    void* out[3] = {q_out, k_cache, v_cache};
    const int heads[3] = {q ? H : 0, Hkv, Hkv};
    for (int i = 0; i < 3; ++i) {
        p.in[i] = in[i];
        p.out[i] = out[i];
        p.heads[i] = heads[i];
        p.is[i] = attn_rope::Strides{0, in_strides[2 * i], in_strides[2 * i + 1]};
    }
    p.os[0] = attn_rope::Strides{0, static_cast<int64_t>(H) * D, D};
    for (int i = 0; i < 2; ++i) p.os[1 + i] = attn_rope::Strides{cache_strides[3 * i], cache_strides[3 * i + 2], cache_strides[3 * i + 1]};
    p.weight[0] = q_weight;
    p.weight[1] = k_weight;
    p.weight_f32 = weight_f32;
    p.table = cos_sin;
    p.table_len = table_len;
    p.R = R;
    p.interleaved = interleaved;
    p.eps = eps;
    p.tokens = tokens;
    p.S = tokens;
    p.cu_seqlens = cu_seqlens;
    p.seq_lens = seq_lens;
    p.block_table = block_table;
    p.table_stride = table_stride;
    p.n_seqs = n_seqs;
    p.max_len = max_pages * page_size;
    p.num_pages = num_pages;
    p.page_shift = log2_of(page_size);
    p.status = cached_status_ptr();
    if (!p.status) return ATTN_ERR_CUDA;
    return launch_rope<true>(p, D, dtype, static_cast<cudaStream_t>(stream));
}

size_t attn_paged_decode_workspace_bytes(int H, int Hkv, int D) {
    if (H < 0 || Hkv < 1 || H % Hkv != 0 || !head_dim_ok(D)) return 0;
    const int group = H / Hkv, rows = group <= 8 ? 8 : 16;
    const size_t parts = static_cast<size_t>(2) * attn_paged::kMaxCtas << tile_heads_shift(Hkv * ((group + 15) / 16), D);
    return align256(parts * rows * (D + 2) * sizeof(float));
}

int attn_paged_decode(const void* q, const void* k_cache, const void* v_cache, const long long* cache_strides, int num_pages,
                      int page_size, const int* block_table, long long table_stride, int max_pages, const int* seq_lens,
                      void* o, float* lse, int B, int H, int Hkv, int D, float scale, int window, int sinks, int dtype,
                      void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || H < 0 || Hkv < 0 || window < 0 || sinks < 0) return ATTN_ERR_BAD_SHAPE;
    if (H > 0 && (Hkv == 0 || H % Hkv != 0)) return ATTN_ERR_BAD_SHAPE;
    if (!head_dim_ok(D)) return ATTN_ERR_UNSUPPORTED_HEAD_DIM;
    if (!dtype_ok(dtype)) return ATTN_ERR_UNSUPPORTED_DTYPE;
    if (static_cast<int64_t>(B) * H > 2147483647LL) return ATTN_ERR_BAD_SHAPE;
    if (!isfinite(scale) || scale < 0.f) return ATTN_ERR_BAD_SCALE;
    if (B == 0 || H == 0) return ATTN_OK;
    if (!q || !o || !lse) return ATTN_ERR_NULL_POINTER;
    int rc = validate_cache(k_cache, v_cache, cache_strides, num_pages, page_size, block_table, max_pages, seq_lens);
    if (rc != ATTN_OK) return rc;
    if (misaligned(q, 16) || misaligned(o, 16) || misaligned(lse, 4)) return ATTN_ERR_MISALIGNED;
    for (int i = 0; i < 2; ++i) {
        const int64_t stride[3] = {cache_strides[3 * i], cache_strides[3 * i + 1], cache_strides[3 * i + 2]};
        const int n[3] = {num_pages, Hkv, page_size};
        if (!mappable(stride, n)) return ATTN_ERR_BAD_SHAPE;
    }
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < attn_paged_decode_workspace_bytes(H, Hkv, D)) return ATTN_ERR_WORKSPACE;
    rc = check_arch();
    if (rc != ATTN_OK) return rc;
    DeviceInfo di;
    if (device_info(&di) != ATTN_OK) return ATTN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (num_pages == 0) return fill_empty(o, lse, static_cast<int64_t>(B) * H * D, static_cast<int64_t>(B) * H, st);
    attn_paged::DecodeParams p = {};
    p.q = q;
    p.o = o;
    p.lse = lse;
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.parts = static_cast<float*>(workspace);
    p.table_stride = table_stride;
    p.B = B;
    p.H = H;
    p.Hkv = Hkv;
    p.group = H / Hkv;
    p.sub = (p.group + 15) / 16;
    p.heads = Hkv * p.sub;
    p.hpt_shift = tile_heads_shift(p.heads, D);
    p.max_len = max_pages * page_size;
    p.num_pages = num_pages;
    p.page_shift = log2_of(page_size);
    p.window = window;
    p.sinks = sinks;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.status = cached_status_ptr();
    if (!p.status) return ATTN_ERR_CUDA;
    const int64_t pairs = static_cast<int64_t>(B) * p.heads;
    const int64_t join_blocks = (H + attn_paged::kJoinWarps - 1) / attn_paged::kJoinWarps;
    if (pairs > 2147483647LL || B * join_blocks > 2147483647LL) return ATTN_ERR_BAD_SHAPE;
    // one CTA per SM, and no more than there can be tiles (16 keys are the smallest tile)
    const int64_t most = pairs * ((static_cast<int64_t>(p.max_len) + 15) / 16 + 2);
    int grid = di.sm_count < attn_paged::kMaxCtas ? di.sm_count : attn_paged::kMaxCtas;
    if (most < grid) grid = static_cast<int>(most);
    p.grid = grid;
    // Few pairs whose sequences cannot be long: clusters (see attn_paged.cuh), of as many CTAs as let all of them be resident at
    // once (16 clusters of 8); and a CTA should not have more than 8 tiles while other SMs have none.  8 heads of 128, against
    // the list and its second kernel: 4 sequences of 1000 keys (clusters of 4) 9 us instead of 14, 8 of 1000 (2) 12 instead of
    // 17, 16 of 1000 (1) 18 instead of 21.
    const int64_t tile_keys = D == 256 ? 4 * 16 : (D == 128 ? 8 * 16 : 8 * 32);
    int cluster = attn_paged::kCluster;
    while (cluster > 1 && pairs * cluster > 128) cluster >>= 1;
#ifdef ATTN_TEST_HOOKS
    p.test_skip_step = g_test_skip_step;
    g_test_skip_step = -1;
#endif
    p.cluster = pairs * cluster <= di.sm_count && p.max_len <= cluster * 8 * tile_keys ? cluster : 0;
#define ATTN_DECODE_CASE(DD, TT, GG)                                                                                     \
    if (D == DD && dtype == TT && (p.group <= 8) == (GG == 8)) {                                                         \
        using C = attn_paged::DecodeCfg<DD, GG>;                                                                         \
        auto kern = attn_paged::attn_paged_decode_kernel<DD, TT, GG>;                                                    \
        if (!allow_dynamic_smem(reinterpret_cast<const void*>(kern), C::SMEM_BYTES)) return ATTN_ERR_CUDA;               \
        const int rows = page_size < C::CK ? page_size : C::CK;                                                          \
        p.box_shift = log2_of(rows);                                                                                     \
        CUtensorMap mk, mv;                                                                                              \
        if (!make_cache_map(&mk, &p.k_axes, k_cache, cache_strides, TT, DD, num_pages, Hkv, page_size, rows) ||          \
            !make_cache_map(&mv, &p.v_axes, v_cache, cache_strides + 3, TT, DD, num_pages, Hkv, page_size, rows))        \
            return ATTN_ERR_CUDA;                                                                                        \
        if (p.cluster)                                                                                                   \
            return launch_cluster(kern, dim3(static_cast<unsigned>(pairs * cluster)), dim3(C::THREADS), C::SMEM_BYTES, \
                                  static_cast<unsigned>(cluster), st, mk, mv, p)                                                   \
                       ? ATTN_OK                                                                                         \
                       : ATTN_ERR_CUDA;                                                                                  \
        kern<<<grid, C::THREADS, C::SMEM_BYTES, st>>>(mk, mv, p);                                                        \
        if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;                                                     \
        return launch_dependent(attn_paged::attn_paged_join_kernel<DD, TT, GG>, dim3(static_cast<unsigned>(B * join_blocks)), \
                                dim3(attn_paged::kJoinWarps * 32), 0, st, p, static_cast<int>(join_blocks)) \
                   ? ATTN_OK                                                                                             \
                   : ATTN_ERR_CUDA;                                                                                      \
    }
    ATTN_DECODE_CASE(64, 0, 8)
    ATTN_DECODE_CASE(64, 1, 8)
    ATTN_DECODE_CASE(128, 0, 8)
    ATTN_DECODE_CASE(128, 1, 8)
    ATTN_DECODE_CASE(256, 0, 8)
    ATTN_DECODE_CASE(256, 1, 8)
    ATTN_DECODE_CASE(64, 0, 16)
    ATTN_DECODE_CASE(64, 1, 16)
    ATTN_DECODE_CASE(128, 0, 16)
    ATTN_DECODE_CASE(128, 1, 16)
    ATTN_DECODE_CASE(256, 0, 16)
    ATTN_DECODE_CASE(256, 1, 16)
#undef ATTN_DECODE_CASE
    return ATTN_ERR_UNSUPPORTED_DTYPE;
}

}  // extern "C"
