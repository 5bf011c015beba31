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

// Sine and cosine of a number of turns, times amplitude (the sine also times sign): the fraction is what counts, in fp64, as far positions are
// many turns.  Rounded to fp32 it is off by up to 2^-26 of a turn, 9e-8 of an angle: next to nothing beside a 16-bit type's step.  In fp32
// that would be half of a result's error, so there the rest is put back, by the first two terms of the sum of two angles.
template <class T>
__device__ __forceinline__ void turn_of(double turns, float amplitude, float sign, float& c, float& s) {
    const double fraction = turns - __builtin_rint(turns);
    const float near = (float)fraction;
    sincospif(2.0f * near, &s, &c);
    if constexpr (sizeof(T) == 4) {
        const float rest = (float)(fraction - near) * 6.2831853071795865f, c0 = c;
        c = __builtin_fmaf(-rest, s, c);
        s = __builtin_fmaf(rest, c0, s);
    }
    c *= amplitude;
    s *= sign * amplitude;
}

// VEC pairs of a token for HEADS heads: both halves of the pairs as vectors of 8 bytes (interleaved: 2 VEC neighbouring channels),
// the angles made once for all heads while the rows are on their way.  Vectors past the rotated channels are copied.  168 MB read
// and written (2 x 4096 tokens, 40 heads of 128, bf16) take 37-41 us, 4.1-4.6 TB/s, where a training step's tensors come from memory (a
// copy of 1 GiB reaches 5.2), and 29 where the same ones are rotated again and again; fp32, twice the bytes, 72 there.  Beside 34-36 in
// one comparison: vectors of 16 bytes 44, one head per thread 43-47.
template <class T, int VEC, int HEADS>
__global__ void __launch_bounds__(256) rope_kernel(RopeTensor q, RopeTensor k, const int* __restrict__ positions, long position_stride,
                                                   const double* __restrict__ inv_freq, float amplitude, int N, int D, int R,
                                                   int interleaved, float sign, long tokens) {
    typedef T vec __attribute__((ext_vector_type(VEC)));
    const int units = D / (2 * VEC), turned = R / (2 * VEC);
    const long w = blockIdx.x * 256l + threadIdx.x, token = w / units;
    if (token >= tokens) return;
    const int j = (int)(w - token * units), b = (int)(token / N), n = (int)(token - (long)b * N);
    const bool turn = j < turned;
    // the two vectors of the unit
    const int first = turn && !interleaved ? VEC * j : 2 * VEC * j, second = turn && !interleaved ? R / 2 + VEC * j : 2 * VEC * j + VEC;
    vec x0[HEADS], x1[HEADS];
    T* to[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = blockIdx.y * HEADS + i;
        to[i] = nullptr;
        if (h >= q.H + k.H) continue;
        const RopeTensor& t = h < q.H ? q : k;
        const int ht = h < q.H ? h : h - q.H;
        const T* const x = (const T*)t.x + b * t.xs.b + ht * t.xs.h + n * t.xs.n;
        to[i] = (T*)t.y + b * t.ys.b + ht * t.ys.h + n * t.ys.n;
        x0[i] = *(const vec*)(x + first);
        x1[i] = *(const vec*)(x + second);
    }
    if (turn) {
        float c[VEC], s[VEC];
        const double position = positions[b * position_stride + n] * 0.15915494309189535;
#pragma unroll
        for (int e = 0; e < VEC; ++e) turn_of<T>(position * inv_freq[VEC * j + e], amplitude, sign, c[e], s[e]);
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            if (interleaved) {
                vec y0, y1;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float u = RopeType<T>::get(2 * e < VEC ? x0[i][2 * e % VEC] : x1[i][2 * e % VEC]);
                    const float v = RopeType<T>::get(2 * e < VEC ? x0[i][(2 * e + 1) % VEC] : x1[i][(2 * e + 1) % VEC]);
                    const T a = RopeType<T>::put(u * c[e] - v * s[e]), d = RopeType<T>::put(v * c[e] + u * s[e]);
                    if (2 * e < VEC) {
                        y0[2 * e % VEC] = a;
                        y0[(2 * e + 1) % VEC] = d;
                    } else {
                        y1[2 * e % VEC] = a;
                        y1[(2 * e + 1) % VEC] = d;
                    }
                }
                x0[i] = y0;
                x1[i] = y1;
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float u = RopeType<T>::get(x0[i][e]), v = RopeType<T>::get(x1[i][e]);
                    x0[i][e] = RopeType<T>::put(u * c[e] - v * s[e]);
                    x1[i][e] = RopeType<T>::put(v * c[e] + u * s[e]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
        if (to[i] != nullptr) {
            *(vec*)(to[i] + first) = x0[i];
            *(vec*)(to[i] + second) = x1[i];
        }
}

// Pairs that no vector fits: one thread per pair of channels of a head (and per pair of channels that pass).
template <class T>
__global__ void __launch_bounds__(256) rope_pair_kernel(RopeTensor q, RopeTensor k, const int* __restrict__ positions, long position_stride,
                                                        const double* __restrict__ inv_freq, float amplitude, int N, int D, int R,
                                                        int interleaved, float sign, long total) {
    const int pairs = D / 2, h = blockIdx.y;
    const long w = blockIdx.x * 256l + threadIdx.x, token = w / pairs;
    if (w >= total) return;
    const int i = (int)(w - token * pairs), b = (int)(token / N), n = (int)(token - (long)b * N);
    const RopeTensor& t = h < q.H ? q : k;
    const int ht = h < q.H ? h : h - q.H;
    const T* x = (const T*)t.x + b * t.xs.b + ht * t.xs.h + n * t.xs.n;
    T* y = (T*)t.y + b * t.ys.b + ht * t.ys.h + n * t.ys.n;
    if (2 * i >= R) {
        const T u = x[2 * i], v = x[2 * i + 1];
        y[2 * i] = u;
        y[2 * i + 1] = v;
        return;
    }
    float s, c;
    turn_of<T>(positions[b * position_stride + n] * 0.15915494309189535 * inv_freq[i], amplitude, sign, c, s);
    const int c0 = interleaved ? 2 * i : i, c1 = interleaved ? 2 * i + 1 : i + R / 2;
    const float u = RopeType<T>::get(x[c0]), v = RopeType<T>::get(x[c1]);
    y[c0] = RopeType<T>::put(u * c - v * s);
    y[c1] = RopeType<T>::put(v * c + u * s);
}

template <class T>
static void launch_rope_type(const RopeTensor& q, const RopeTensor& k, const int* positions, long position_stride, const double* inv_freq,
                             float amplitude, int B, int N, int D, int R, bool interleaved, float sign, hipStream_t st) {
    const long tokens = (long)B * N;
    const int H = q.H + k.H;
#define SAGE_ROPE(VEC, HEADS) rope_kernel<T, VEC, HEADS><<<dim3((unsigned)((tokens * (D / (2 * VEC)) + 255) / 256), (H + HEADS - 1) / HEADS), 256, 0, st>>>( \
        q, k, positions, position_stride, inv_freq, amplitude, N, D, R, interleaved, sign, tokens)
    constexpr int VEC = 8 / sizeof(T);
    if (R % (2 * VEC) == 0) {
        // one head per thread while there is too little work to fill the chip with four (a decoding step of 64 tokens and 40 heads)
        if (tokens * H * (D / 16) < (1l << 17)) SAGE_ROPE(VEC, 1);
        else SAGE_ROPE(VEC, 4);
    } else {
        const long total = tokens * (D / 2);
        rope_pair_kernel<T><<<dim3((unsigned)((total + 255) / 256), H), 256, 0, st>>>(q, k, positions, position_stride, inv_freq, amplitude, N, D, R,
                                                                                      interleaved, sign, total);
    }
#undef SAGE_ROPE
}

hipError_t launch_rope(const RopeTensor& q, const RopeTensor& k, const int* positions, long position_stride, const double* inv_freq,
                       float amplitude, int B, int N, int D, int rotated, int type, bool interleaved, bool backward, hipStream_t st) {
    const float sign = backward ? -1.0f : 1.0f;
    if (type == TYPE_F32) launch_rope_type<float>(q, k, positions, position_stride, inv_freq, amplitude, B, N, D, rotated, interleaved, sign, st);
    else if (type == TYPE_BF16) launch_rope_type<__bf16>(q, k, positions, position_stride, inv_freq, amplitude, B, N, D, rotated, interleaved, sign, st);
    else launch_rope_type<_Float16>(q, k, positions, position_stride, inv_freq, amplitude, B, N, D, rotated, interleaved, sign, st);
    return hipGetLastError();
}

}  // namespace sage
