// C-ABI entry points of the serving calls: host-side validation, then kernel launches.
#include "../../include/sage.h"
#include "sage_serving.h"
#include <cmath>

namespace {

using sage::RowStrides;

// a launch counts its threads, 256 per workgroup here, in 32 bits
constexpr long long MOST_WORKGROUPS = (1ll << 24) - 1;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool fp16_or_bf16(int type) { return type == SAGE_F16 || type == SAGE_BF16; }

int check_shape(int B, int H, int N) {
    if (B <= 0 || H <= 0 || N <= 0 || N > (1 << 23)) return SAGE_ERR_SHAPE;
    if ((long long)B * H > 65535) return SAGE_ERR_SHAPE;
    return SAGE_OK;
}

// The strides of a [B, H, N, D] tensor: the caller's three, or those of a contiguous one.  Where there is one index only
// its stride says nothing.  ok turns false where a row would not start on a 16-byte boundary; written: or where two rows would
// be the same memory.
RowStrides strides(const int64_t* s, int B, int H, int N, int D, int size, bool written, bool& ok) {
    RowStrides r = {(long)H * N * D, (long)N * D, D};
    if (s != nullptr) r = {(long)s[0], (long)s[1], (long)s[2]};
    if (B == 1) r.b = 0;
    if (H == 1) r.h = 0;
    if (N == 1) r.n = 0;
    const int unit = 16 / size;
    ok = ok && r.b % unit == 0 && r.h % unit == 0 && r.n % unit == 0;
    if (written) ok = ok && (B == 1 || r.b) && (H == 1 || r.h) && (N == 1 || r.n);
    return r;
}

bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128 || page == 256; }
bool form_ok(int D, int page, int group) {
    return (D == 64 || D == 128) && page_ok(page) && (group == 32 || group == 64 || group == 128) && group <= D;
}
int check_cache(const void* cache, const int32_t* pages, int B, int Hkv, int D, int num_pages, int columns, int page, int group) {
    if (!cache || !pages) return SAGE_ERR_NULL;
    if (int e = check_shape(B, Hkv, 1)) return e;
    if (!form_ok(D, page, group)) return SAGE_ERR_UNSUPPORTED;
    if (num_pages <= 0 || columns <= 0 || (long long)columns * page > (1 << 23)) return SAGE_ERR_SHAPE;
    if (!aligned(cache, 16) || !aligned(pages, 4)) return SAGE_ERR_ALIGN;
    return SAGE_OK;
}
sage::Cache4 view(const void* cache, const int32_t* pages, int Hkv, int D, int num_pages, int columns, int page, int group) {
    // (at most 65535 heads of 256 rows of 144 bytes: below 2^32)
    const unsigned block = (unsigned)sage_cache4_block_bytes(D, page, group);
    return {(unsigned char*)cache, pages, num_pages, columns, Hkv, __builtin_ctz((unsigned)page), D, D / group, block, block * (unsigned)Hkv};
}
int check_queries(int B, int Hq, int Hkv, int Nq, int type, float sm_scale) {
    if (int e = check_shape(B, Hq, Nq)) return e;
    if (Hq % Hkv != 0 || !fp16_or_bf16(type)) return SAGE_ERR_UNSUPPORTED;
    // query rows are counted in an int
    if ((long long)Hq * Nq > (1 << 30) || (long long)B * Hq * Nq > 0x7fffffffLL) return SAGE_ERR_SHAPE;
    if (!std::isfinite(sm_scale) || !(sm_scale > 0.0f)) return SAGE_ERR_VALUE;
    return SAGE_OK;
}
int status(hipError_t e) { return e == hipSuccess ? SAGE_OK : SAGE_ERR_LAUNCH; }

int rope(const void* q, const int64_t* q_strides, void* q_out, const int64_t* q_out_strides, const void* k, const int64_t* k_strides,
         void* k_out, const int64_t* k_out_strides, const int32_t* positions, int64_t position_stride, const double* inv_freq,
         float amplitude, int B, int Hq, int Hk, int N, int D, int rotated, int type, int interleaved, bool backward, void* stream) {
    if (!q || !q_out || !positions || !inv_freq || (Hk > 0 && (!k || !k_out))) return SAGE_ERR_NULL;
    if (Hk < 0 || position_stride < 0 || D <= 0) return SAGE_ERR_SHAPE;
    if (int e = check_shape(B, Hq, N)) return e;
    if (int e = check_shape(B, Hq + Hk, N)) return e;
    if ((long long)B * N * D > 512 * MOST_WORKGROUPS) return SAGE_ERR_SHAPE;         // (a thread per pair of channels)
    if (type != SAGE_F16 && type != SAGE_BF16 && type != SAGE_F32) return SAGE_ERR_UNSUPPORTED;
    if (D % 8 != 0 || D > 512 || rotated < 2 || rotated > D || rotated % 2 != 0) return SAGE_ERR_UNSUPPORTED;
    if (!std::isfinite(amplitude)) return SAGE_ERR_VALUE;
    bool ok = aligned(q, 16) && aligned(q_out, 16) && aligned(positions, 4) && aligned(inv_freq, 8);
    const int size = type == SAGE_F32 ? 4 : 2;
    sage::RopeTensor tq = {q, q_out, strides(q_strides, B, Hq, N, D, size, false, ok), strides(q_out_strides, B, Hq, N, D, size, true, ok), Hq};
    sage::RopeTensor tk = {};
    if (Hk > 0) {
        ok = ok && aligned(k, 16) && aligned(k_out, 16);
        tk = {k, k_out, strides(k_strides, B, Hk, N, D, size, false, ok), strides(k_out_strides, B, Hk, N, D, size, true, ok), Hk};
    }
    if (!ok) return SAGE_ERR_ALIGN;
    return status(sage::launch_rope(tq, tk, positions, position_stride, inv_freq, amplitude, B, N, D, rotated, type, interleaved != 0,
                                    backward, (hipStream_t)stream));
}

}  // namespace

extern "C" {

int sage_rope(const void* q, const int64_t* q_strides, void* q_out, const int64_t* q_out_strides, const void* k, const int64_t* k_strides,
              void* k_out, const int64_t* k_out_strides, const int32_t* positions, int64_t position_stride, const double* inv_freq,
              float amplitude, int B, int Hq, int Hk, int N, int D, int rotated, int type, int interleaved, void* stream) {
    return rope(q, q_strides, q_out, q_out_strides, k, k_strides, k_out, k_out_strides, positions, position_stride, inv_freq, amplitude,
                B, Hq, Hk, N, D, rotated, type, interleaved, false, stream);
}

int sage_rope_bwd(const void* dq, const int64_t* dq_strides, void* dq_out, const int64_t* dq_out_strides, const void* dk, const int64_t* dk_strides,
                  void* dk_out, const int64_t* dk_out_strides, const int32_t* positions, int64_t position_stride, const double* inv_freq,
                  float amplitude, int B, int Hq, int Hk, int N, int D, int rotated, int type, int interleaved, void* stream) {
    return rope(dq, dq_strides, dq_out, dq_out_strides, dk, dk_strides, dk_out, dk_out_strides, positions, position_stride, inv_freq,
                amplitude, B, Hq, Hk, N, D, rotated, type, interleaved, true, stream);
}

size_t sage_cache4_block_bytes(int D, int page, int group) {
    return form_ok(D, page, group) ? (size_t)page * (D + 4 * (D / group)) : 0;
}

int sage_cache4_append(const void* k, const int64_t* k_strides, const void* v, const int64_t* v_strides, const float* k_mean, void* cache,
                       const int32_t* pages, const int32_t* start, const int32_t* count, int B, int Hkv, int N, int D, int type,
                       int num_pages, int columns, int page, int group, void* stream) {
    if (!k || !v || !start) return SAGE_ERR_NULL;
    if (int e = check_cache(cache, pages, B, Hkv, D, num_pages, columns, page, group)) return e;
    if (int e = check_shape(B, Hkv, N)) return e;
    if (!fp16_or_bf16(type)) return SAGE_ERR_UNSUPPORTED;
    bool ok = aligned(k, 16) && aligned(v, 16) && aligned(k_mean, 16) && aligned(start, 4) && aligned(count, 4);
    const RowStrides ks = strides(k_strides, B, Hkv, N, D, 2, false, ok), vs = strides(v_strides, B, Hkv, N, D, 2, false, ok);
    if (!ok) return SAGE_ERR_ALIGN;
    return status(sage::launch_cache4_append(view(cache, pages, Hkv, D, num_pages, columns, page, group), k, ks, v, vs, k_mean, start, count,
                                             B, N, type, (hipStream_t)stream));
}

int sage_cache4_load(const void* cache, const int32_t* pages, const int32_t* start, const int32_t* count, const float* k_mean, void* k, void* v,
                     int B, int Hkv, int N, int D, int type, int num_pages, int columns, int page, int group, void* stream) {
    if (!k || !v) return SAGE_ERR_NULL;
    if (int e = check_cache(cache, pages, B, Hkv, D, num_pages, columns, page, group)) return e;
    if (int e = check_shape(B, Hkv, N)) return e;
    if (!fp16_or_bf16(type)) return SAGE_ERR_UNSUPPORTED;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_mean, 16) || !aligned(start, 4) || !aligned(count, 4)) return SAGE_ERR_ALIGN;
    return status(sage::launch_cache4_load(view(cache, pages, Hkv, D, num_pages, columns, page, group), start, count, k_mean, k, v, B, N, type,
                                           (hipStream_t)stream));
}

size_t sage_cache4_attn_workspace(int B, int Hq, int Hkv, int Nq, int D, int columns, int page, int n_splits) {
    if (check_shape(B, Hq, Nq) || check_shape(B, Hkv, 1) || Hq % Hkv != 0 || (D != 64 && D != 128) || !page_ok(page)) return 0;
    if (columns <= 0 || (long long)columns * page > (1 << 23) || n_splits < 0) return 0;
    if ((long long)Hq * Nq > (1 << 30) || (long long)B * Hq * Nq > 0x7fffffffLL) return 0;
    return sage::cache4_attn_workspace(B, Hq, Hkv, Nq, D, columns * page, n_splits);
}

int sage_cache4_attn(const void* q, const int64_t* q_strides, const void* cache, const int32_t* pages, const int32_t* lengths, const int32_t* count,
                     void* out, const int64_t* out_strides, float* lse, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int Nq,
                     int D, int type, int num_pages, int columns, int page, int group, int causal, float sm_scale, int n_splits, void* stream) {
    if (!q || !lengths || !out) return SAGE_ERR_NULL;
    if (int e = check_cache(cache, pages, B, Hkv, D, num_pages, columns, page, group)) return e;
    if (int e = check_queries(B, Hq, Hkv, Nq, type, sm_scale)) return e;
    if (n_splits < 0) return SAGE_ERR_VALUE;
    if (sage::cache4_attn_workgroups(B, Hq, Hkv, Nq, D, columns * page, n_splits) > MOST_WORKGROUPS) return SAGE_ERR_SHAPE;
    const size_t need = sage_cache4_attn_workspace(B, Hq, Hkv, Nq, D, columns, page, n_splits);
    if (need > 0 && !workspace) return SAGE_ERR_NULL;
    if (workspace_bytes < need) return SAGE_ERR_WORKSPACE;
    bool ok = aligned(q, 16) && aligned(out, 16) && aligned(lengths, 4) && aligned(count, 4) && aligned(lse, 4) && (need == 0 || aligned(workspace, 16));
    const RowStrides qs = strides(q_strides, B, Hq, Nq, D, 2, false, ok), os = strides(out_strides, B, Hq, Nq, D, 2, true, ok);
    if (!ok) return SAGE_ERR_ALIGN;
    return status(sage::launch_cache4_attn(view(cache, pages, Hkv, D, num_pages, columns, page, group),
                                           {q, qs, lengths, count, B, Hq, Nq, type, causal ? 1 : 0, sm_scale}, out, os, lse, workspace, n_splits,
                                           (hipStream_t)stream));
}

int sage_cache4_weights(const void* q, const int64_t* q_strides, const void* cache, const int32_t* pages, const int32_t* lengths, const int32_t* count,
                        const float* lse, const float* weights, float* out, int width, int B, int Hq, int Hkv, int Nq, int D, int type,
                        int num_pages, int columns, int page, int group, int causal, float sm_scale, void* stream) {
    if (!q || !lengths || !lse || !out) return SAGE_ERR_NULL;
    if (int e = check_cache(cache, pages, B, Hkv, D, num_pages, columns, page, group)) return e;
    if (int e = check_queries(B, Hq, Hkv, Nq, type, sm_scale)) return e;
    if (width < columns * page || width > (1 << 23)) return SAGE_ERR_SHAPE;
    bool ok = aligned(q, 16) && aligned(lengths, 4) && aligned(count, 4) && aligned(lse, 4) && aligned(weights, 4) && aligned(out, 4);
    const RowStrides qs = strides(q_strides, B, Hq, Nq, D, 2, false, ok);
    if (!ok) return SAGE_ERR_ALIGN;
    return status(sage::launch_cache4_weights(view(cache, pages, Hkv, D, num_pages, columns, page, group),
                                              {q, qs, lengths, count, B, Hq, Nq, type, causal ? 1 : 0, sm_scale}, lse, weights, out, width,
                                              (hipStream_t)stream));
}

int sage_cache4_evict(const void* cache, int num_pages, const int32_t* pages, int columns, const int32_t* lengths, const float* weights, int width,
                      void* out_cache, int out_num_pages, const int32_t* out_pages, int out_columns, float* out_weights, int out_width,
                      int32_t* kept, int32_t* out_lengths, int B, int Hkv, int D, int page, int group, int keep, int recent, void* stream) {
    if (!lengths || !weights || !out_weights || !kept || !out_lengths) return SAGE_ERR_NULL;
    if (int e = check_cache(cache, pages, B, Hkv, D, num_pages, columns, page, group)) return e;
    if (int e = check_cache(out_cache, out_pages, B, Hkv, D, out_num_pages, out_columns, page, group)) return e;
    if (keep <= 0 || keep > out_columns * page || width < columns * page || width > (1 << 23) || out_width < keep || out_width > (1 << 23))
        return SAGE_ERR_SHAPE;
    // in place, or the old accumulators under the new ones: rows would be overwritten before they are read
    const bool in_place = cache == out_cache && pages == out_pages;
    if (recent < 0 || recent > keep || in_place || weights == out_weights || lengths == out_lengths) return SAGE_ERR_VALUE;
    if (!aligned(lengths, 4) || !aligned(weights, 4) || !aligned(out_weights, 4) || !aligned(kept, 4) || !aligned(out_lengths, 4)) return SAGE_ERR_ALIGN;
    return status(sage::launch_cache4_evict(view(cache, pages, Hkv, D, num_pages, columns, page, group), lengths, weights, width,
                                            view(out_cache, out_pages, Hkv, D, out_num_pages, out_columns, page, group), out_weights, out_width,
                                            kept, out_lengths, B, keep, recent, (hipStream_t)stream));
}

}  // extern "C"
