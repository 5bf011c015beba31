// Attention over the cache held in 4 bits, and the weight that each of its keys is given.
//
//   S = sm_scale q K^T,  out = softmax(S) V,  lse = ln sum exp S,   K, V = code * scale;
//   weights[key] += sum over the queries of the key's heads of exp(S - lse).
//
// Query t of the n that a sequence has is its token number length - n + t; with the causal mask it sees the tokens up to itself.
#include "sage_serving.h"
#include "sage_device.h"

namespace sage {

namespace {
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float element(const void* p, long at, int type) {
    if (type == TYPE_F16) return (float)((const _Float16*)p)[at];
    return __builtin_bit_cast(float, (unsigned)((const unsigned short*)p)[at] << 16);
}
// channel d of token `row` of a block
__device__ __forceinline__ float key_value(const Cache4& c, const unsigned char* block, int row, int d) {
    const int word = (d & 31) / 8 * (c.D / 32) + d / 32, e = d & 7;
    const unsigned w = ((const unsigned*)(block + c.k_codes(row)))[word];
    return (float)((int)(w >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8) * (float)((const _Float16*)(block + c.k_scales(row)))[d / c.group];
}
__device__ __forceinline__ float value_value(const Cache4& c, const unsigned char* block, int row, int d) {
    const unsigned w = ((const unsigned*)(block + c.v_codes(row)))[d / 8];
    return (float)((int)(w >> 4 * (d & 7) & 15u) - 8) * (float)((const _Float16*)(block + c.v_scales(row)))[d / c.group];
}
__device__ __forceinline__ float wg_reduce(float x, bool sum, float* red) {
    for (int off = 32; off; off >>= 1) {
        const float y = __shfl_xor(x, off, 64);
        x = sum ? x + y : __builtin_fmaxf(x, y);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    return sum ? red[0] + red[1] + red[2] + red[3] : __builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3]));
}
}  // namespace

// The simple form: a workgroup per query row, 256 keys at a time.
__global__ void __launch_bounds__(256) cache4_attn_kernel(Cache4 c, CacheQueries q, void* __restrict__ out, RowStrides os, float* __restrict__ lse) {
    __shared__ float s_q[128], s_p[256], red[4];
    const int t = threadIdx.x;
    const int n = blockIdx.x % q.Nq, hq = blockIdx.x / q.Nq % q.Hq, b = blockIdx.x / (q.Nq * q.Hq), h = hq / (q.Hq / c.heads);
    const int length = min(max(q.lengths[b], 0), c.capacity()), count = q.count != nullptr ? min(max(q.count[b], 0), q.Nq) : q.Nq;
    const int end = n >= count ? 0 : (q.causal ? min(length, length - count + n + 1) : length);
    if (t < c.D) s_q[t] = element(q.q, b * q.strides.b + hq * q.strides.h + n * q.strides.n + t, q.type) * q.sm_scale;
    __syncthreads();
    float top = -__builtin_inff(), sum = 0.0f, acc = 0.0f;
    for (int j0 = 0; j0 < end; j0 += 256) {
        const int j = j0 + t;
        const unsigned char* block = j < end ? c.block(b, h, j) : nullptr;
        float s = -__builtin_inff();
        if (block != nullptr) {
            s = 0.0f;
            for (int d = 0; d < c.D; ++d) s = __builtin_fmaf(s_q[d], key_value(c, block, j & (c.page() - 1), d), s);
        }
        const float most = __builtin_fmaxf(top, wg_reduce(s, false, red));
        const float sub = most == -__builtin_inff() ? 0.0f : most;
        const float p = expf(s - sub), keep = expf(top - sub);
        top = most;
        sum = sum * keep + wg_reduce(p, true, red);
        acc *= keep;
        s_p[t] = p;
        __syncthreads();
        if (t < c.D)
            for (int i = 0; i < min(256, end - j0); ++i) {
                const unsigned char* at = c.block(b, h, j0 + i);
                if (at != nullptr) acc = __builtin_fmaf(s_p[i], value_value(c, at, (j0 + i) & (c.page() - 1), t), acc);
            }
        __syncthreads();
    }
    const float r = sum == 0.0f ? 0.0f : acc / sum;
    if (t < c.D) {
        const long at = b * os.b + hq * os.h + n * os.n + t;
        if (q.type == TYPE_F16) ((_Float16*)out)[at] = (_Float16)r;
        else ((__bf16*)out)[at] = (__bf16)r;
    }
    if (t == 0 && lse != nullptr) lse[((long)b * q.Hq + hq) * q.Nq + n] = sum == 0.0f ? -__builtin_inff() : top + logf(sum);
}

// A thread per key.
__global__ void __launch_bounds__(256) cache4_weights_kernel(Cache4 c, CacheQueries q, const float* __restrict__ lse, const float* __restrict__ weights,
                                                             float* __restrict__ out, int width) {
    const int bh = blockIdx.y, b = bh / c.heads, h = bh - b * c.heads, j = blockIdx.x * 256 + threadIdx.x;
    if (j >= width) return;
    const int length = min(max(q.lengths[b], 0), c.capacity()), count = q.count != nullptr ? min(max(q.count[b], 0), q.Nq) : q.Nq;
    const unsigned char* block = j < length ? c.block(b, h, j) : nullptr;
    const int share = q.Hq / c.heads;
    float sum = 0.0f;
    for (int g = 0; g < share; ++g)
        for (int n = 0; n < count; ++n) {
            if (block == nullptr || (q.causal && j > length - count + n)) continue;
            const long at = b * q.strides.b + (h * share + g) * q.strides.h + n * q.strides.n;
            float s = 0.0f;
            for (int d = 0; d < c.D; ++d) s = __builtin_fmaf(element(q.q, at + d, q.type), key_value(c, block, j & (c.page() - 1), d), s);
            const float l = lse[((long)b * q.Hq + h * share + g) * q.Nq + n];
            if (l != -__builtin_inff()) sum += expf(s * q.sm_scale - l);
        }
    const size_t at = (size_t)bh * width + j;
    out[at] = (weights != nullptr ? weights[at] : 0.0f) + sum;
}

size_t cache4_attn_workspace(int B, int Hq, int Hkv, int Nq, int D, int capacity, int n_splits) { return 0; }

hipError_t launch_cache4_attn(const Cache4& c, const CacheQueries& q, void* out, const RowStrides& os, float* lse, void* workspace,
                              int n_splits, hipStream_t st) {
    cache4_attn_kernel<<<q.B * q.Hq * q.Nq, 256, 0, st>>>(c, q, out, os, lse);
    return hipGetLastError();
}

hipError_t launch_cache4_weights(const Cache4& c, const CacheQueries& q, const float* lse, const float* weights, float* out, int width,
                                 hipStream_t st) {
    cache4_weights_kernel<<<dim3((width + 255) / 256, q.B * c.heads), 256, 0, st>>>(c, q, lse, weights, out, width);
    return hipGetLastError();
}

}  // namespace sage
