// The cache held in 4 bits: tokens quantized into their pages, read back, and the least used ones left behind.
//
// The quantizer is Section 3.2's with 7 in place of 127, one scale per token, head and group of channels:
//   delta = fp16(amax / 7),  code = clamp(round_half_even(x / delta), -7, 7),
// the division by the scale as it is stored, so that the code is the nearest one for the reader.  x is v, or k - k_mean (Section
// 4.2: a vector added to every key of a head does not change the softmax, and K's channels carry large ones).
#include "sage_serving.h"
#include "sage_device.h"

namespace sage {

namespace {
constexpr float MAX_SCALE = 65504.0f;       // fp16's largest: values beyond 7 of it saturate

// 8 channels of a row as fp32
template <int TYPE>
__device__ __forceinline__ void row8(const void* p, long at, float (&x)[8]) {
    if constexpr (TYPE == TYPE_F16) {
        const half8 v = *(const half8*)((const _Float16*)p + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    } else {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        const u4 v = *(const u4*)((const unsigned short*)p + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __builtin_bit_cast(float, v[e] << 16);
            x[2 * e + 1] = __builtin_bit_cast(float, v[e] & 0xffff0000u);
        }
    }
}
template <int TYPE>
__device__ __forceinline__ void put_row8(void* p, long at, const float (&x)[8]) {
    if constexpr (TYPE == TYPE_F16) {
        half8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (_Float16)x[e];
        *(half8*)((_Float16*)p + at) = v;
    } else {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        b8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
        *(b8*)((__bf16*)p + at) = v;
    }
}
// The quotient z / d, rounded as a division rounds it, by three instructions instead of ten: with y within 2^-22 of 1 / d, q = z y
// is off by three ulp at most, its remainder z - q d is exact in an FMA where d has few bits (a scale in fp16, 7), and q +
// remainder y rounds to the quotient -- which lies 2^-12 ulp and more from where two fp32 numbers meet, or on one of them.
__device__ __forceinline__ float quotient(float z, float d, float y) {
    const float q = z * y;
    return __builtin_fmaf(__builtin_fmaf(-q, d, z), y, q);
}
// the scale of a group from its largest magnitude (infinite: the quotient is no number, and the minimum passes over it)
__device__ __forceinline__ _Float16 scale_of(float amax) { return (_Float16)__builtin_fminf(quotient(amax, 7.0f, 1.0f / 7.0f), MAX_SCALE); }
// where channel e of 8 stands in its word
template <bool IS_K> __device__ __forceinline__ int nibble_shift(int e) { return IS_K ? 4 * (e >> 1) + 16 * (e & 1) : 4 * e; }
// the word of octet o (channels 8 o .. 8 o + 7) in its row
template <bool IS_K> __device__ __forceinline__ int octet_word(int o, int D) { return IS_K ? (o & 3) * (D / 32) + (o >> 2) : o; }

template <int GROUP>
__device__ __forceinline__ float group_max(const float (&x)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, __builtin_fabsf(x[e]));
    return lanes_max<GROUP / 8>(m);
}
// The codes of 8 channels in their word: limited to 7 steps before the quotient, so that infinities saturate and nothing
// overflows; the addition of 1.5 * 2^23 + 8 rounds to whole numbers, ties to even, and leaves code + 8 in the low bits.
template <bool IS_K>
__device__ __forceinline__ unsigned pack8(const float (&x)[8], float delta) {
    const float y = delta > 0.0f ? __builtin_amdgcn_rcpf(delta) : 0.0f, most = 7.0f * delta;
    unsigned n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        n[e] = __builtin_bit_cast(unsigned, quotient(__builtin_amdgcn_fmed3f(x[e], -most, most), delta, y) + 12582920.0f);
    // two nibbles in the low byte of a word (1 .. 15 is all of it), four of those to a word
    auto pair = [&n](int i, int j) { return n[j] << 4 | n[i]; };
    const unsigned b0 = IS_K ? pair(0, 2) : pair(0, 1), b1 = IS_K ? pair(4, 6) : pair(2, 3);
    const unsigned b2 = IS_K ? pair(1, 3) : pair(4, 5), b3 = IS_K ? pair(5, 7) : pair(6, 7);
    return __builtin_amdgcn_perm(b1, b0, 0x0c0c0400u) | __builtin_amdgcn_perm(b3, b2, 0x04000c0cu);
}
// NaN to 0
__device__ __forceinline__ void numbers(float (&x)[8]) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; e += 2) odd |= __builtin_isunordered(x[e], x[e + 1]);
    if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] == x[e] ? x[e] : 0.0f;
    }
}
template <bool IS_K>
__device__ __forceinline__ void unpack8(unsigned w, float delta, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)((int)(w >> nibble_shift<IS_K>(e) & 15u) - 8) * delta;
}
}  // namespace

// A thread takes 8 channels of K and of V of a token, D / 8 adjacent threads the token's row.  24.6K tokens of 8 heads of 128 in bf16,
// 166 MB read and written: 43 us; the same loads and stores without the arithmetic 34.  (Two tokens per thread, or the heads of a
// token next to each other in the grid: no change.)
template <int D, int GROUP, int TYPE>
__global__ void __launch_bounds__(256) cache4_append_kernel(Cache4 c, const void* __restrict__ k, RowStrides ks, const void* __restrict__ v,
                                                            RowStrides vs, const float* __restrict__ k_mean, const int* __restrict__ start,
                                                            const int* __restrict__ count, int N) {
    constexpr int OCTETS = D / 8, ROWS = 256 / OCTETS;
    const int o = threadIdx.x % OCTETS, bh = blockIdx.y, b = bh / c.heads, h = bh - b * c.heads;
    const int first = blockIdx.x * ROWS, row = threadIdx.x / OCTETS, n = first + row;
    const int there = count != nullptr ? min(count[b], N) : N;
    // (a row's threads stay or leave together: group_max looks at no other row's)
    if (n >= there) return;
    // the rows are on their way while the page is looked up
    float x[8], y[8];
    row8<TYPE>(k, (b * ks.b + h * ks.h + first * ks.n) + row * ks.n + 8 * o, x);
    row8<TYPE>(v, (b * vs.b + h * vs.h + first * vs.n) + row * vs.n + 8 * o, y);
    float mean[8] = {};
    if (k_mean != nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) mean[e] = k_mean[(size_t)bh * D + 8 * o + e];
    }
    const long slot = (long)start[b] + n;
    if (slot < 0 || slot >= c.capacity()) return;
    unsigned char* block = c.block(b, h, (int)slot);
    if (block == nullptr) return;
    const int r = (int)slot & (c.page() - 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] -= mean[e];
    numbers(x);
    numbers(y);
    const _Float16 dk = scale_of(group_max<GROUP>(x)), dv = scale_of(group_max<GROUP>(y));
    ((unsigned*)(block + c.k_codes(r)))[octet_word<true>(o, D)] = pack8<true>(x, (float)dk);
    ((unsigned*)(block + c.v_codes(r)))[octet_word<false>(o, D)] = pack8<false>(y, (float)dv);
    if (o % (GROUP / 8) == 0) {
        ((_Float16*)(block + c.k_scales(r)))[o / (GROUP / 8)] = dk;
        ((_Float16*)(block + c.v_scales(r)))[o / (GROUP / 8)] = dv;
    }
}

template <int D, int GROUP, int TYPE>
__global__ void __launch_bounds__(256) cache4_load_kernel(Cache4 c, const int* __restrict__ start, const int* __restrict__ count,
                                                          const float* __restrict__ k_mean, void* __restrict__ k, void* __restrict__ v, int N) {
    constexpr int OCTETS = D / 8, ROWS = 256 / OCTETS;
    const int o = threadIdx.x % OCTETS, bh = blockIdx.y, b = bh / c.heads, h = bh - b * c.heads;
    const int n = blockIdx.x * ROWS + threadIdx.x / OCTETS;
    if (n >= N) return;
    const int there = count != nullptr ? min(count[b], N) : N;
    const long slot = (start != nullptr ? (long)start[b] : 0l) + n;
    const unsigned char* block = n < there && slot >= 0 && slot < c.capacity() ? c.block(b, h, (int)slot) : nullptr;
    float x[8] = {}, y[8] = {};
    if (block != nullptr) {
        const int r = (int)slot & (c.page() - 1);
        unpack8<true>(((const unsigned*)(block + c.k_codes(r)))[octet_word<true>(o, D)],
                      (float)((const _Float16*)(block + c.k_scales(r)))[o / (GROUP / 8)], x);
        unpack8<false>(((const unsigned*)(block + c.v_codes(r)))[octet_word<false>(o, D)],
                       (float)((const _Float16*)(block + c.v_scales(r)))[o / (GROUP / 8)], y);
        if (k_mean != nullptr) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += k_mean[(size_t)bh * D + 8 * o + e];
        }
    }
    const long at = ((long)bh * N + n) * D + 8 * o;
    put_row8<TYPE>(k, at, x);
    put_row8<TYPE>(v, at, y);
}

#define SAGE_CACHE4_SHAPE(KERNEL, TYPE, ...)                                                                       \
    do {                                                                                                            \
        if (c.D == 64 && c.groups == 2) KERNEL<64, 32, TYPE><<<grid, 256, 0, st>>>(__VA_ARGS__);                    \
        else if (c.D == 64) KERNEL<64, 64, TYPE><<<grid, 256, 0, st>>>(__VA_ARGS__);                                \
        else if (c.groups == 4) KERNEL<128, 32, TYPE><<<grid, 256, 0, st>>>(__VA_ARGS__);                           \
        else if (c.groups == 2) KERNEL<128, 64, TYPE><<<grid, 256, 0, st>>>(__VA_ARGS__);                           \
        else KERNEL<128, 128, TYPE><<<grid, 256, 0, st>>>(__VA_ARGS__);                                             \
    } while (0)

hipError_t launch_cache4_append(const Cache4& c, const void* k, const RowStrides& ks, const void* v, const RowStrides& vs,
                                const float* k_mean, const int* start, const int* count, int B, int N, int type, hipStream_t st) {
    const int rows = 256 / (c.D / 8);
    const dim3 grid((N + rows - 1) / rows, B * c.heads);
    if (type == TYPE_BF16) SAGE_CACHE4_SHAPE(cache4_append_kernel, TYPE_BF16, c, k, ks, v, vs, k_mean, start, count, N);
    else SAGE_CACHE4_SHAPE(cache4_append_kernel, TYPE_F16, c, k, ks, v, vs, k_mean, start, count, N);
    return hipGetLastError();
}

hipError_t launch_cache4_load(const Cache4& c, const int* start, const int* count, const float* k_mean, void* k, void* v, int B, int N,
                              int type, hipStream_t st) {
    const int rows = 256 / (c.D / 8);
    const dim3 grid((N + rows - 1) / rows, B * c.heads);
    if (type == TYPE_BF16) SAGE_CACHE4_SHAPE(cache4_load_kernel, TYPE_BF16, c, start, count, k_mean, k, v, N);
    else SAGE_CACHE4_SHAPE(cache4_load_kernel, TYPE_F16, c, start, count, k_mean, k, v, N);
    return hipGetLastError();
}

// ---- eviction
// The slots that stay, in order: the last `recent` of n and, of the m before them, the need = keep - recent with the largest
// weights, of equal ones the lowest slots.  One workgroup per (sequence, head); a wavefront has a share of the slots of its
// own, the first 1024 of them in registers.  The need-th largest weight is closed in on: [low, high] holds it, at first the smallest and
// the largest weight; 2048 bins over it are counted, summed from the largest down, and one of them is the next [low, high].  At most
// 64 weights left are compared each with each.  (Bins over what is there, not over fixed bits: weights of a softmax
// share most of their upper bits, and one pass leaves a handful: 64 heads of 16K slots 17 us, 12 if all are equal, 25 if most are; by
// 11, 11 and 10 bits from the top 23.)  Then every wavefront counts those of its share above it and equal
// to it, and writes its share.
namespace {
// larger weight, larger key; a NaN below all numbers, -0 with 0; 0 is no weight's
__device__ __forceinline__ unsigned rank_key(float w) {
    const unsigned u = __builtin_bit_cast(unsigned, w + 0.0f);
    return w != w ? 1u : (u >> 31 ? ~u : u | 0x80000000u);
}
__device__ __forceinline__ int popcount(unsigned long long x) { return __builtin_popcountll(x); }
// bits of x below the lane's own
__device__ __forceinline__ int before(unsigned long long x) {
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(x >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)x, 0u));
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ unsigned moved(unsigned otherwise, unsigned x) {
    return (unsigned)__builtin_amdgcn_update_dpp((int)otherwise, (int)x, CTRL, ROWS, 0xF, false);
}
// over 16 lanes, in all of them
template <class F>
__device__ __forceinline__ unsigned over16(unsigned x, F&& f) {
    x = f(x, moved<0xB1>(x, x));                // lane ^ 1
    x = f(x, moved<0x4E>(x, x));                // lane ^ 2
    x = f(x, moved<0x141>(x, x));               // the other half of 8, mirrored
    return f(x, moved<0x140>(x, x));            // the other half of 16, mirrored
}
// the sum over the lanes up to the own
__device__ __forceinline__ int running_sum(int x) {
    x += (int)moved<0x111>(0u, (unsigned)x);            // from the lane 1, 2, 4, 8 before, of 16
    x += (int)moved<0x112>(0u, (unsigned)x);
    x += (int)moved<0x114>(0u, (unsigned)x);
    x += (int)moved<0x118>(0u, (unsigned)x);
    x += (int)moved<0x142, 0xA>(0u, (unsigned)x);       // the 16 before's last to the second and fourth 16
    x += (int)moved<0x143, 0xC>(0u, (unsigned)x);       // the first 32's last to the others
    return x;
}
}  // namespace

constexpr int SELECT_NT = 1024, SELECT_WAVES = SELECT_NT / 64, SELECT_HELD = 16, SELECT_BINS = 2 * SELECT_NT, SELECT_COPIES = 4, SELECT_LIST = 64;
static_assert(SELECT_WAVES == 16 && SELECT_LIST == 64, "a value per wavefront in 16 lanes, a listed weight per lane");
__global__ void __launch_bounds__(SELECT_NT) cache4_select_kernel(const int* __restrict__ lengths, const float* __restrict__ weights, int width,
                                                                  int capacity, int heads, int* __restrict__ kept,
                                                                  int* __restrict__ out_lengths, int keep, int recent) {
    // (copies, one for every fourth lane: weights of like size fall into few bins, and additions to one word wait for each other)
    __shared__ __attribute__((aligned(16))) int histogram[SELECT_COPIES][SELECT_BINS + 8];
    __shared__ unsigned s_low[SELECT_WAVES], s_high[SELECT_WAVES], s_list[SELECT_LIST];
    __shared__ int s_digit, s_above, s_count, s_listed, s_rank[SELECT_LIST], s_total[SELECT_WAVES], s_gt[SELECT_WAVES], s_eq[SELECT_WAVES];
    const int bh = blockIdx.x, b = bh / heads, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int n = min(max(lengths[b], 0), capacity);
    int* const to = kept + (size_t)bh * keep;
    if (bh == b * heads && t == 0) out_lengths[b] = min(n, keep);
    if (n <= keep) {
        for (int i = t; i < keep; i += SELECT_NT) to[i] = i < n ? i : -1;
        return;
    }
    const float* const w = weights + (size_t)bh * width;
    const int m = n - recent, need = keep - recent;
    for (int i = t; i < recent; i += SELECT_NT) to[need + i] = m + i;
    if (need == 0) return;
    const int share = (m + SELECT_NT - 1) / SELECT_NT * 64, first = min(wave * share, m), last = min(first + share, m);
    unsigned held[SELECT_HELD];
#pragma unroll
    for (int j = 0; j < SELECT_HELD; ++j) {
        const int i = first + 64 * j + lane;
        held[j] = i < last ? rank_key(w[i]) : 0u;
    }
    // f(key, slot) for the lane's slots, 64 neighbouring ones of the wavefront at a time; key 0: none there
    auto walk = [&](auto&& f) {
#pragma unroll
        for (int j = 0; j < SELECT_HELD; ++j)
            if (first + 64 * j < last) f(held[j], first + 64 * j + lane);
        for (int i0 = first + 64 * SELECT_HELD; i0 < last; i0 += 64 * 4) {
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = w[min(i0 + 64 * j + lane, m - 1)];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i0 + 64 * j < last) f(i0 + 64 * j + lane < last ? rank_key(x[j]) : 0u, i0 + 64 * j + lane);
        }
    };
    auto smaller = [](unsigned x, unsigned y) { return x < y ? x : y; };
    auto larger = [](unsigned x, unsigned y) { return x > y ? x : y; };
    auto sum = [](unsigned x, unsigned y) { return x + y; };
    // of the wavefronts' values those before this one's, added up
    auto sum_before = [&](const int* of) { return (int)over16((lane & 15) < wave ? (unsigned)of[lane & 15] : 0u, sum); };
    typedef int pair_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < SELECT_COPIES; ++i) *(pair_t*)&histogram[i][2 * t] = (pair_t){0, 0};
    if (t < SELECT_LIST) s_rank[t] = 0;
    if (t == 0) s_listed = 0;
    unsigned low = ~0u, high = 0u;
    walk([&](unsigned u, int) {
        low = smaller(low, u - 1u);
        high = larger(high, u);
    });
    low = over16(low, smaller);
    high = over16(high, larger);
    low = smaller(low, __shfl_xor(low, 16, 64));
    high = larger(high, __shfl_xor(high, 16, 64));
    low = smaller(low, __shfl_xor(low, 32, 64));
    high = larger(high, __shfl_xor(high, 32, 64));
    if (lane == 0) {
        s_low[wave] = low;
        s_high[wave] = high;
    }
    __syncthreads();
    low = __builtin_amdgcn_readfirstlane(over16(s_low[lane & 15], smaller)) + 1u;
    high = __builtin_amdgcn_readfirstlane(over16(s_high[lane & 15], larger));
    int left = need, count = m;         // of the `count` keys in [low, high], how many stay
    while (left < count && low < high) {
        const unsigned span = high - low;
        if (count <= SELECT_LIST) {
            walk([&](unsigned u, int) {
                if (u - low <= span) s_list[atomicAdd(&s_listed, 1)] = u;
            });
            __syncthreads();
            const unsigned x = lane < count ? s_list[lane] : 0u;
            int rank = 0;               // larger ones, and 2^16 times the equal ones
#pragma unroll
            for (int i = 0; i < SELECT_LIST / SELECT_WAVES; ++i) {
                const int at = wave * (SELECT_LIST / SELECT_WAVES) + i;
                const unsigned y = at < count ? __builtin_amdgcn_readlane(x, at) : 0u;
                rank += y > x ? 1 : y == x ? 1 << 16 : 0;
            }
            atomicAdd(&s_rank[lane], rank);
            __syncthreads();
            rank = s_rank[lane];
            const int above = rank & 0xffff, equal = rank >> 16;
            const int one = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < count && above < left && left <= above + equal));
            low = __builtin_amdgcn_readlane(x, one);
            left -= __builtin_amdgcn_readlane(above, one);
            count = __builtin_amdgcn_readlane(equal, one);
            break;
        }
        const int shift = max(21 - (int)__builtin_clz(span), 0);
        walk([&](unsigned u, int) {
            const unsigned d = u - low;
            if (d <= span) atomicAdd(&histogram[lane % SELECT_COPIES][d >> shift], 1);
        });
        __syncthreads();
        // thread t: two bins, from the largest down; `above`: keys in the bins before them
        const int bin = SELECT_BINS - 2 - 2 * t;
        pair_t h = {0, 0};
#pragma unroll
        for (int i = 0; i < SELECT_COPIES; ++i) {
            h += *(const pair_t*)&histogram[i][bin];
            *(pair_t*)&histogram[i][bin] = (pair_t){0, 0};
        }
        int above = running_sum(h[0] + h[1]);
        if (lane == 63) s_total[wave] = above;
        __syncthreads();
        above += sum_before(s_total) - h[0] - h[1];
        if (above < left && left <= above + h[0] + h[1]) {
            const bool upper = left <= above + h[1];
            s_digit = upper ? bin + 1 : bin;
            s_above = upper ? above : above + h[1];
            s_count = upper ? h[1] : h[0];
        }
        __syncthreads();
        low += (unsigned)__builtin_amdgcn_readfirstlane(s_digit) << shift;
        high = smaller(high, low + ((1u << shift) - 1u));
        left -= __builtin_amdgcn_readfirstlane(s_above);
        count = __builtin_amdgcn_readfirstlane(s_count);
    }
    const unsigned found = low;
    if (left == count) left = m;        // all keys in [low, high] stay: whatever is there from low on
    int gt = 0, eq = 0;
    walk([&](unsigned u, int) {
        gt += popcount(__builtin_amdgcn_ballot_w64(u > found));
        eq += popcount(__builtin_amdgcn_ballot_w64(u == found));
    });
    if (lane == 0) {
        s_gt[wave] = gt;
        s_eq[wave] = eq;
    }
    __syncthreads();
    int ties = __builtin_amdgcn_readfirstlane(sum_before(s_eq));        // equal ones before this share
    int at = __builtin_amdgcn_readfirstlane(sum_before(s_gt)) + min(ties, left);
    walk([&](unsigned u, int i) {
        const unsigned long long equal = __builtin_amdgcn_ballot_w64(u == found);
        const bool stays = u > found || (u == found && ties + before(equal) < left);
        const unsigned long long all = __builtin_amdgcn_ballot_w64(stays);
        if (stays) to[at + before(all)] = i;
        at += popcount(all);
        ties += popcount(equal);
    });
}

// The kept rows copied: D / 32 threads for 16 bytes each of the K codes, as many for V's; each also one of the 2 D / group
// scales.  A row whose page holds no tokens becomes zeros.  A thread has GATHER_ROWS rows: index, pages and bytes are three
// round trips to memory, one after the other.
constexpr int GATHER_ROWS = 4;
template <int D>
__global__ void __launch_bounds__(256) cache4_gather_kernel(Cache4 c, Cache4 to, const int* __restrict__ kept, const float* __restrict__ weights,
                                                            int width, float* __restrict__ out_weights, int out_width, int keep) {
    constexpr int TPR = D / 16, ROWS = 256 / TPR;
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    const int bh = blockIdx.y, b = bh / c.heads, h = bh - b * c.heads, i = threadIdx.x % TPR;
    const int j0 = blockIdx.x * ROWS * GATHER_ROWS + threadIdx.x / TPR, S = c.groups, half = D / 32;
    const bool is_v = i >= half;
    const int chunk = is_v ? i - half : i;
    int from[GATHER_ROWS];
#pragma unroll
    for (int r = 0; r < GATHER_ROWS; ++r) {
        const int j = j0 + r * ROWS;
        from[r] = j < keep ? kept[(size_t)bh * keep + j] : -1;
    }
    const unsigned char* src[GATHER_ROWS];
    unsigned char* dst[GATHER_ROWS];
#pragma unroll
    for (int r = 0; r < GATHER_ROWS; ++r) {
        src[r] = from[r] >= 0 ? c.block(b, h, from[r]) : nullptr;
        dst[r] = from[r] >= 0 ? to.block(b, h, j0 + r * ROWS) : nullptr;
    }
    u4 x[GATHER_ROWS];
    unsigned short s[GATHER_ROWS];
    float w[GATHER_ROWS];
#pragma unroll
    for (int r = 0; r < GATHER_ROWS; ++r) {
        x[r] = (u4){0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u};
        s[r] = 0;
        w[r] = 0.0f;
        const int row = from[r] & (c.page() - 1);
        if (src[r] != nullptr) {
            x[r] = ((const u4*)(src[r] + (is_v ? c.v_codes(row) : c.k_codes(row))))[chunk];
            if (chunk < S) s[r] = ((const unsigned short*)(src[r] + (is_v ? c.v_scales(row) : c.k_scales(row))))[chunk];
        }
        if (i == 0 && from[r] >= 0) w[r] = weights[(size_t)bh * width + from[r]];
    }
#pragma unroll
    for (int r = 0; r < GATHER_ROWS; ++r) {
        const int j = j0 + r * ROWS, row = j & (to.page() - 1);
        if (i == 0 && j < out_width) out_weights[(size_t)bh * out_width + j] = w[r];
        if (dst[r] != nullptr) {
            ((u4*)(dst[r] + (is_v ? to.v_codes(row) : to.k_codes(row))))[chunk] = x[r];
            if (chunk < S) ((unsigned short*)(dst[r] + (is_v ? to.v_scales(row) : to.k_scales(row))))[chunk] = s[r];
        }
    }
}

hipError_t launch_cache4_evict(const Cache4& c, const int* lengths, const float* weights, int width, const Cache4& to, float* out_weights,
                               int out_width, int* kept, int* out_lengths, int B, int keep, int recent, hipStream_t st) {
    cache4_select_kernel<<<B * c.heads, SELECT_NT, 0, st>>>(lengths, weights, width, c.capacity(), c.heads, kept, out_lengths, keep, recent);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int rows = 256 / (c.D / 16) * GATHER_ROWS;
    const dim3 grid((out_width + rows - 1) / rows, B * c.heads);
    if (c.D == 64) cache4_gather_kernel<64><<<grid, 256, 0, st>>>(c, to, kept, weights, width, out_weights, out_width, keep);
    else cache4_gather_kernel<128><<<grid, 256, 0, st>>>(c, to, kept, weights, width, out_weights, out_width, keep);
    return hipGetLastError();
}

}  // namespace sage
