// Rotary positions: pairs of channels turned by position * frequency, and the gradient of it (the turn back).
//
//   (x, y) -> (x c - y s, y c + x s),   c = amplitude cos(p f_i), s = amplitude sin(p f_i),
//
// pair i being channels (i, i + R/2) or (2 i, 2 i + 1) of the first R; the others pass.  The turn is orthogonal up to the
// amplitude, so the gradient is the same with -s.  Bound by memory.
#include "sage_serving.h"
#include "sage_device.h"

namespace sage {

template <class T> struct RopeType;
template <> struct RopeType<_Float16> {
    static __device__ __forceinline__ float get(_Float16 x) { return (float)x; }
    static __device__ __forceinline__ _Float16 put(float x) { return (_Float16)x; }
};
template <> struct RopeType<__bf16> {
    static __device__ __forceinline__ float get(__bf16 x) { return (float)x; }
    static __device__ __forceinline__ __bf16 put(float x) { return (__bf16)x; }
};
template <> struct RopeType<float> {
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
};

// One thread per pair of channels (and per pair of channels that pass).
template <class T>
__global__ void __launch_bounds__(256) rope_kernel(RopeTensor q, RopeTensor k, const int* __restrict__ positions, long position_stride,
                                                   const double* __restrict__ inv_freq, float amplitude, int N, int D, int R,
                                                   int interleaved, float sign, long total) {
    const int pairs = D / 2, H = q.H + k.H;
    for (long w = blockIdx.x * 256l + threadIdx.x; w < total; w += gridDim.x * 256l) {
        const int i = (int)(w % pairs);
        long r = w / pairs;
        const int h = (int)(r % H);
        r /= H;
        const int n = (int)(r % N), b = (int)(r / N);
        const RopeTensor& t = h < q.H ? q : k;
        const int ht = h < q.H ? h : h - q.H;
        const T* x = (const T*)t.x + b * t.xs.b + ht * t.xs.h + n * t.xs.n;
        T* y = (T*)t.y + b * t.ys.b + ht * t.ys.h + n * t.ys.n;
        if (2 * i >= R) {
            const T u = x[2 * i], v = x[2 * i + 1];
            y[2 * i] = u;
            y[2 * i + 1] = v;
            continue;
        }
        // turns, in fp64: far positions are many of them, and only the fraction counts
        const double turns = positions[b * position_stride + n] * (inv_freq[i] * 0.15915494309189535);
        const float part = (float)(turns - __builtin_rint(turns));
        const float c = amplitude * cospif(2.0f * part), s = sign * amplitude * sinpif(2.0f * part);
        const int c0 = interleaved ? 2 * i : i, c1 = interleaved ? 2 * i + 1 : i + R / 2;
        const float u = RopeType<T>::get(x[c0]), v = RopeType<T>::get(x[c1]);
        y[c0] = RopeType<T>::put(u * c - v * s);
        y[c1] = RopeType<T>::put(v * c + u * s);
    }
}

hipError_t launch_rope(const RopeTensor& q, const RopeTensor& k, const int* positions, long position_stride, const double* inv_freq,
                       float amplitude, int B, int N, int D, int rotated, int type, bool interleaved, bool backward, hipStream_t st) {
    const long total = (long)B * N * (q.H + k.H) * (D / 2);
    const long want = (total + 255) / 256;
    const dim3 grid((unsigned)(want < (1 << 20) ? want : (1 << 20)));
    const float sign = backward ? -1.0f : 1.0f;
#define SAGE_ROPE(T) rope_kernel<T><<<grid, 256, 0, st>>>(q, k, positions, position_stride, inv_freq, amplitude, N, D, rotated, interleaved, sign, total)
    if (type == TYPE_F32) SAGE_ROPE(float);
    else if (type == TYPE_BF16) SAGE_ROPE(__bf16);
    else SAGE_ROPE(_Float16);
#undef SAGE_ROPE
    return hipGetLastError();
}

}  // namespace sage
