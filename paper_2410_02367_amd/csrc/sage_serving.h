// Internal interface of the serving calls: rotary positions, and the cache held in 4 bits with what works on it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sage {

enum { TYPE_F16 = 0, TYPE_BF16 = 1, TYPE_F32 = 2 };

// element strides of a [B, H, N, D] tensor whose channels are next to each other
struct RowStrides {
    long b, h, n;
};

// A pool of pages and the table of the pages that a batch of sequences holds.  Block (page, head) of the pool is
//   K codes [page][D / 2], V codes [page][D / 2], K scales [page][D / group], V scales [page][D / group] (fp16).
// A code c of -7 .. 7 is the nibble c + 8.  V's nibbles are in the order of the channels, the low one first.  K's row holds
// channel 32 i + 8 h + e in word h * D / 32 + i, nibble e / 2 + 4 (e % 2): a lane of the matrix instruction that takes
// channels 8 h .. 8 h + 7 of every 32 finds all its words next to each other, and the halves of a word masked with 0x000f000f
// are a pair of its operand.
struct Cache4 {
    unsigned char* data;
    const int* table;           // [B, columns]; an entry outside 0 .. num_pages - 1 holds no tokens
    int num_pages, columns, heads;
    int shift;                  // log2 of the tokens per page
    int D, groups;              // channels, and groups of them with a scale
    unsigned block_bytes, page_bytes;           // of a head of a page, of a page: (D + 4 groups) << shift, times the heads
    __host__ __device__ int page() const { return 1 << shift; }
    __host__ __device__ int capacity() const { return columns << shift; }
    // the block that holds token `slot` of sequence b, or null
    __device__ unsigned char* block(int b, int h, int slot) const {
        const int p = table[(size_t)b * columns + (slot >> shift)];
        if ((unsigned)p >= (unsigned)num_pages) return nullptr;
        return data + (size_t)h * block_bytes + (unsigned long long)(unsigned)p * page_bytes;
    }
    // byte offsets in a block of the parts of row r (of its page)
    __device__ int k_codes(int r) const { return r * (D / 2); }
    __device__ int v_codes(int r) const { return ((D / 2) << shift) + r * (D / 2); }
    __device__ int k_scales(int r) const { return (D << shift) + r * 2 * groups; }
    __device__ int v_scales(int r) const { return ((D + 2 * groups) << shift) + r * 2 * groups; }
};

// [b][h][n] rows of a tensor rotated; x and y may be the same.  All return the hipError_t of the launch.
struct RopeTensor {
    const void* x;
    void* y;
    RowStrides xs, ys;
    int H;
};
hipError_t launch_rope(const RopeTensor& q, const RopeTensor& k, const int* positions, long position_stride, const double* inv_freq,
                       float amplitude, int B, int N, int D, int rotated, int type, bool interleaved, bool backward, hipStream_t st);

hipError_t launch_cache4_append(const Cache4& c, const void* k, const RowStrides& ks, const void* v, const RowStrides& vs,
                                const float* k_mean, const int* start, const int* count, int B, int N, int type, hipStream_t st);
hipError_t launch_cache4_load(const Cache4& c, const int* start, const int* count, const float* k_mean, void* k, void* v, int B, int N,
                              int type, hipStream_t st);

// queries of an attention call over a cache: [B, Hq, Nq, D], the first count[b] of a sequence's rows are there
struct CacheQueries {
    const void* q;
    RowStrides strides;
    const int *lengths, *count;
    int B, Hq, Nq, type, causal;
    float sm_scale;
};
long long cache4_attn_workgroups(int B, int Hq, int Hkv, int Nq, int D, int capacity, int n_splits);
size_t cache4_attn_workspace(int B, int Hq, int Hkv, int Nq, int D, int capacity, int n_splits);
hipError_t launch_cache4_attn(const Cache4& c, const CacheQueries& q, void* out, const RowStrides& os, float* lse, void* workspace,
                              int n_splits, hipStream_t st);
hipError_t launch_cache4_weights(const Cache4& c, const CacheQueries& q, const float* lse, const float* weights, float* out, int width,
                                 hipStream_t st);

hipError_t launch_cache4_evict(const Cache4& c, const int* lengths, const float* weights, int width, const Cache4& to, float* out_weights,
                               int out_width, int* kept, int* out_lengths, int B, int keep, int recent, hipStream_t st);

}  // namespace sage
