// Attention over the cache held in 4 bits, and the weight that each of its keys is given.
//
//   S = sm_scale q K^T,  out = softmax(S) V,  lse = ln sum exp S,   K, V = code * scale;
//   weights[key] += sum over the queries of the key's heads of exp(S - lse).
//
// Query t of the n that a sequence has is its token number length - n + t; with the causal mask it sees the tokens up to itself.
//
// One pass over the cache.  A row is a (query, head of the key head's group) pair, row t * share + g; a workgroup takes 16 QT rows
// of one (sequence, key head) and its four wavefronts take tiles of 64 keys in turn, each with its own running reference, sum
// and O, without a barrier, and add up at the end; long caches are cut into chunks for several workgroups and merged.
//
// Codes go to the matrix pipe as whole numbers, scales are applied to sums: 9 vector instructions turn 8 codes into 4 operand
// registers (operand()), every other pair 16 times too large, for which the other operand makes up.
//   S^T = K q^T: contraction steps of 32 channels, so a group's sum is finished after group / 32 of them and is scaled there.
//   O^T = V^T P^T: the sums run over keys, whose scales are the weights' business: P is formed once per group of channels as
//         fp16(exp2(s - M) * scale).  V is transposed by the LDS read that transposes nibbles; the keys of an operand are in
//         the order in which the score tiles leave them, so P never leaves its registers.
//
// What is rounded to fp16, a weight times its key's scale, is bounded by a reference R per row and group of channels: it is
// exp2(s - R) * scale, and where one passes 2^15 (or the weights of 8 keys 2^50) R is raised to the largest s + log2(scale) less 10, rounded up
// to a whole number.  So the range of fp16 is spent on what reaches the group's output, whatever the scales are: neither a key with large
// values and next to no weight nor a group of larger values leaves others less precision, down to 2^-100 of a row's largest, below which the
// exponentials leave fp32.  M is the largest R of a row, and its largest s less 46 at least.  Groups that ask for up to 7 less, or have had
// no value but 0, share it (their largest is 2^2 at least, so that what rounds to a subnormal number is off by 2^-23 of it), and as
// long as all rows of a wavefront have nothing but M, which is the rule, a weight is one product.  Where they have not, 32 keys are weighed
// again with a product more per group, and R follows the largest: 108 -> 129 us for 256 slabs of 8K to 16K keys with four rows and one group of
// four 2^8 times the others, 118 -> 194 with 16 rows, 912 -> 2680 for 1024 queries of 32 heads on 32K keys.  (A product with a power of two
// per row and group in any case: 719 us for 717 for those 1024 with two groups, 979 for 915 with four, 119 for 117 with the 16 rows.)
// The weights in fp16 are a choice: with half a step of 2^-11 each they take the error of an fp16 output against 64 bits from 2.1e-4, its own
// rounding, to 2.9e-4 (a bf16 output's stays 1.7e-3).  With what the rounding leaves as a second operand it is 2.1e-4 again, at 109 us for 102
// for a decoding step of 32 sequences and at 1014 for 715 for 1024 queries on 32K keys.  The sums l (with M) and O (each group with its R) are fp32.
#include "sage_serving.h"
#include "sage_device.h"

namespace sage {

typedef float c4f __attribute__((ext_vector_type(4)));
typedef unsigned c4u __attribute__((ext_vector_type(4)));
typedef unsigned c2u __attribute__((ext_vector_type(2)));
typedef int c2i __attribute__((ext_vector_type(2)));

namespace {
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float UNSET = -1e30f;             // a reference below every score: the first key that is seen raises it
constexpr _Float16 W_LIMIT = 32768.0f;
constexpr float P_LIMIT = 0x1p50f;
constexpr float RAISE = 10.0f, ALIKE = 7.0f, FARTHEST = 120.0f, FLOOR = 46.0f;
constexpr int TILE = 64, WAVES = 4, FEW_CHUNK = 2048;

// 8 codes of a word -> operand registers: element 2 m + s is the code of nibble m + 4 s, times 16 where m is odd.  A nibble in the
// low mantissa bits of 1024 is 1024 + nibble (or + 16 nibble); the packed subtraction is exact and leaves a small whole number.
// (The nibbles as subnormal numbers would need no exponent and, with the 8 in the other terms, no subtraction: 9 -> 5
// instructions.  But the matrix pipe aligns a subnormal operand's products as if it were 2^-14, which costs the sums 7 bits.)
// (No inline assembly beside matrix instructions: the compiler keeps no distance between one's registers and what such a line writes.
// An AND and an OR with two scalar constants are two instructions, so that one constant comes from a register, out of its sight.)
__device__ __forceinline__ unsigned thousands() {
    unsigned x;
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(x));
    return x;
}
__device__ __forceinline__ half8 operand(unsigned w, unsigned thousand) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const unsigned x = w >> 8;
    const h2 even = {(_Float16)1032.0f, (_Float16)1032.0f}, odd = {(_Float16)1152.0f, (_Float16)1152.0f};
    const h2 a = __builtin_bit_cast(h2, (w & 0x000f000fu) | thousand) - even, b = __builtin_bit_cast(h2, (w & 0x00f000f0u) | thousand) - odd;
    const h2 c = __builtin_bit_cast(h2, (x & 0x000f000fu) | thousand) - even, d = __builtin_bit_cast(h2, (x & 0x00f000f0u) | thousand) - odd;
    return (half8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What a row of queries sees.
struct RowRange {
    int length, count;          // of the sequence, limited to what there is
    int rows;                   // rows that are there: count * share
    __device__ __forceinline__ RowRange(const Cache4& c, const CacheQueries& q, int b, int share) {
        length = min(max(q.lengths[b], 0), c.capacity());
        count = q.count != nullptr ? min(max(q.count[b], 0), q.Nq) : q.Nq;
        rows = count * share;
    }
    // slots [0, end) for query t
    __device__ __forceinline__ int end(int t, int causal) const { return causal ? max(min(length, length - count + t + 1), 0) : length; }
};

// 16 rows of queries as the second operand of the score product: lane (column lane % 16, h = lane / 16) holds channels 32 i + 8 h
// .. of the row at `at`.  A row is brought to a largest magnitude of 2^13 .. 2^14 by a power of two, so that every element that
// matters beside the largest is exact in fp16, bf16's range and the 2^-4 of those that meet 16-fold codes included.
// -> what turns a scaled sum into the exponent of 2.
template <int D>
struct Queries4 {
    c4u raw[D / 32];
    half8 op[D / 32];
    __device__ __forceinline__ void request(const CacheQueries& q, long at, int h) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) raw[i] = *(const c4u*)((const unsigned short*)q.q + at + 32 * i + 8 * h);
    }
    __device__ __forceinline__ float load(const CacheQueries& q, long at, int h) {
        request(q, at, h);
        return convert(q);
    }
    __device__ __forceinline__ float convert(const CacheQueries& q) {
        float x[D / 32][8], m = 0.0f;
        if (q.type == TYPE_F16) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const half8 v = __builtin_bit_cast(half8, raw[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = (float)v[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned w = raw[i][e];
                    x[i][2 * e] = word_f32(w << 16);
                    x[i][2 * e + 1] = word_f32(w & 0xffff0000u);
                }
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, __builtin_fabsf(x[i][e]));
        m = __builtin_fmaxf(m, __shfl_xor(m, 16, 64));
        m = __builtin_fmaxf(m, __shfl_xor(m, 32, 64));
        const int exponent = __builtin_amdgcn_frexp_expf(m);        // (0 of 0 and of infinity)
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) op[i][e] = (_Float16)ldexpf(x[i][e], 14 - exponent - (e & 2 ? 4 : 0));
        // (never 0 or infinite: a score of 0 or -infinity times it stays one)
        return __builtin_fminf(__builtin_fmaxf(ldexpf(q.sm_scale * LOG2E, exponent - 14), 1e-37f), 1e37f);
    }
};

// The pages of a tile's four 16-key pieces (of the whole tile where a page holds 64 tokens or more: id[0]), uniform over the
// wavefront; looked up a tile before they are used.  -1: none.
struct PageIds {
    int id[4];
    __device__ __forceinline__ void look_up(const Cache4& c, const int* table, int k0) {
        const int n = c.shift >= 6 ? 1 : 4;
        const int col = k0 >> c.shift;
        id[0] = col < c.columns ? table[col] : -1;
        if (n == 1) return;
#pragma unroll
        for (int j = 1; j < 4; ++j) {
            const int cj = (k0 + 16 * j) >> c.shift;
            id[j] = cj < c.columns ? table[cj] : -1;
        }
    }
};

template <int NG> struct ScaleWord;
template <> struct ScaleWord<4> { typedef c2u type; };
template <> struct ScaleWord<2> { typedef unsigned type; };
template <> struct ScaleWord<1> { typedef unsigned short type; };

// A tile of 64 keys on its way: K's words as operands want them, V's rows, a key's scales per lane.  A piece without a page
// reads block 0 instead, and is masked.
template <int D, int NG, bool VALUES>
struct KeyTile {
    typedef typename ScaleWord<NG>::type scale_t;
    typedef unsigned words __attribute__((ext_vector_type(D / 32)));
    static constexpr int ROW = D / 2;
    words k[4];
    c4u v[VALUES ? D / 32 : 1];
    scale_t ks, vs;
    unsigned bad;               // bit j: piece j has no page
    // head: the block of the key head in page 0
    static __device__ __forceinline__ const unsigned char* block(const Cache4& c, const unsigned char* head, int id, bool& ok) {
        ok = (unsigned)id < (unsigned)c.num_pages;
        return head + (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane(ok ? id : 0) * c.page_bytes;
    }
    __device__ __forceinline__ void request(const Cache4& c, const unsigned char* head, const PageIds& pages, int k0, int lane) {
        const int col = lane & 15, h = lane >> 4, mask = c.page() - 1;
        if (c.shift >= 6) {
            bool ok;
            const unsigned char* const at = block(c, head, pages.id[0], ok);
            const int row = k0 & mask;
            bad = ok ? 0u : 15u;
            const unsigned char* const kp = at + row * ROW;
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = *(const words*)(kp + col * ROW + h * (D / 8) + 16 * j * ROW);
            const unsigned char* const sp = at + (D << c.shift) + row * 2 * NG;
            ks = *(const scale_t*)(sp + lane * 2 * NG);
            if constexpr (VALUES) {
                vs = *(const scale_t*)(sp + (2 * NG << c.shift) + lane * 2 * NG);
                const unsigned char* const vp = kp + (ROW << c.shift);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) v[i] = *(const c4u*)(vp + lane * 16 + 1024 * i);
            }
            return;
        }
        const unsigned char* at[4];
        int row[4];
        bad = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bool ok;
            at[j] = block(c, head, pages.id[j], ok);
            row[j] = (k0 + 16 * j) & mask;
            if (!ok) bad |= 1u << j;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = *(const words*)(at[j] + (row[j] + col) * ROW + h * (D / 8));
        const unsigned char* mine = at[0];
        int r = row[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) {
            mine = h == j ? at[j] : mine;
            r = h == j ? row[j] : r;
        }
        r += col;
        ks = *(const scale_t*)(mine + (D << c.shift) + r * 2 * NG);
        if constexpr (VALUES) {
            vs = *(const scale_t*)(mine + ((D + 2 * NG) << c.shift) + r * 2 * NG);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                // 1 KB at a time: 16 rows of 64 bytes, or 32 of 32
                if constexpr (D == 128) v[i] = *(const c4u*)(at[i] + (ROW << c.shift) + row[i] * ROW + lane * 16);
                else {
                    const unsigned char* half = lane < 32 ? at[2 * i] : at[2 * i + 1];
                    v[i] = *(const c4u*)(half + (ROW << c.shift) + (lane < 32 ? row[2 * i] : row[2 * i + 1]) * ROW + (lane & 31) * 16);
                }
            }
        }
    }
};

// The LDS of a wavefront: K's words, each lane's own (so that the registers are free for the next tile at once); V's rows in
// 16-byte chunks, exchanged so that the 16 rows a transposing read takes lie in different banks; a key's scales.
template <int D, int NG>
struct WaveLds {
    unsigned char k[TILE * D / 2], v[TILE * D / 2];
    _Float16 ks[TILE * NG], vs[TILE * NG];
};
template <int D> __device__ __forceinline__ int v_chunk(int key, int chunk) {
    return key * (D / 2) + ((chunk ^ (((key >> 4) + (key >> 2)) & (D / 32 - 1))) * 16);
}

// the larger of three, of both halves (a NaN stays)
__device__ __forceinline__ unsigned max3_pairs(unsigned a, unsigned b, unsigned c) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_bit_cast(h2, a), __builtin_bit_cast(h2, b)),
                                                                      __builtin_bit_cast(h2, c)));
}
__device__ __forceinline__ _Float16 half_of(unsigned w, int hi) { return __builtin_bit_cast(_Float16, (unsigned short)(hi ? w >> 16 : w)); }

// x, and the compiler does not know that: what is seldom needed is not made ahead and kept in registers
template <class T>
__device__ __forceinline__ T anew(T x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Groups of a wavefront's keys that had no value but 0 so far, a bit each.  (Such a group asks for no reference: channels that only fill
// up a head would have one of their own for nothing.)
template <int NG>
struct EmptyGroups {
    unsigned empty = (1u << NG) - 1u;
    // scales: those of the lane's key of a tile -> whether a group of them is no longer empty (the same in all lanes)
    template <class S>
    __device__ __forceinline__ bool look(S scales) {
        unsigned seen = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            unsigned short own;
            if constexpr (NG == 4) own = (unsigned short)(scales[g / 2] >> 16 * (g & 1));
            else own = (unsigned short)(scales >> 16 * g);
            if (__builtin_amdgcn_ballot_w64((own & 0x7fff) != 0) != 0ull) seen |= 1u << g;
        }
        const unsigned fresh = empty & seen;
        empty &= ~seen;
        return fresh != 0;
    }
};
// The references of a row: M, and how far below it those of the groups are, whole numbers in 8 bits each; NONE: the row has seen no value
// of the group but 0, so that the group's sums are 0.
template <int NG>
struct References {
    static constexpr unsigned NONE = 255;
    float M;
    unsigned below;
    __device__ __forceinline__ void clear() {
        M = UNSET;
        below = ~0u;
    }
    __device__ __forceinline__ unsigned byte(int g) const { return below >> 8 * g & 255u; }
    __device__ __forceinline__ int distance(int g) const { return NG == 1 || byte(g) == NONE ? 0 : (int)byte(g); }
    // what brings sums of group g to M
    __device__ __forceinline__ float back(int g) const { return ldexpf(1.0f, -distance(g)); }
    // raised to what the row's keys ask for, M to their largest score less FLOOR at least, which bounds the sum of the weights; alpha: what the groups'
    // sums so far are multiplied by -> what l is (whole powers of two)
    __device__ __forceinline__ float raise(const float (&most)[NG], float score, float (&alpha)[NG]) {
        const float M_old = M;
        float R[NG];
        M = __builtin_fmaxf(M, __builtin_ceilf(score - FLOOR));
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            R[g] = __builtin_fmaxf(NG > 1 && byte(g) == NONE ? UNSET : M_old - (float)distance(g), __builtin_ceilf(most[g]));
            M = __builtin_fmaxf(M, R[g]);
        }
        unsigned now = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            // (a row that is no number has nothing but M)
            const float d = NG > 1 && M - R[g] > ALIKE ? __builtin_fminf(M - R[g], FARTHEST) : 0.0f;
            alpha[g] = __builtin_amdgcn_exp2f((M_old - M) + (d - (float)distance(g)));
            now |= (R[g] == UNSET ? NONE : (unsigned)d) << 8 * g;
        }
        below = now;
        return __builtin_amdgcn_exp2f(M_old - M);
    }
    // whether the rows of the wavefront have nothing but M for the groups that are not empty (the same in all lanes)
    __device__ __forceinline__ bool alike(const EmptyGroups<NG>& groups) const {
        if constexpr (NG == 1) return true;
        unsigned others = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) others |= groups.empty >> g & 1 ? 0u : 255u << 8 * g;
        return __builtin_amdgcn_ballot_w64((below & others) != 0u) == 0ull;
    }
};

// The weights of 32 keys for 16 rows: register r of the two score tiles is keys 4 h + r and 16 + 4 h + r, element 2 r and 2 r + 1
// of an operand; those of odd r meet 16-fold codes and are 2^-4 of the others.  PLAIN: with M for all groups.  -> whether a reference is too low.
template <bool PLAIN, int NG, class S>
__device__ __forceinline__ bool weigh(const float (&s)[2][4], float sc, const References<NG>& ref, const S (&vs)[2], half8 (&w)[NG], float& sum) {
    unsigned x[NG][4];
    const float M = ref.M, M_odd = M + 4.0f;
    float factor[NG];
    if constexpr (!PLAIN) {
#pragma unroll
        for (int g = 0; g < NG; ++g) factor[g] = ldexpf(1.0f, ref.distance(g));
    }
    sum = 0.0f;
    auto one = [&](auto R) {
        constexpr int r = decltype(R)::value;
        float p[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][r], sc, r & 1 ? -M_odd : -M));
            sum = r & 1 ? __builtin_fmaf(p[j], 16.0f, sum) : sum + p[j];
        }
        auto group = [&](auto G) {
            constexpr int g = decltype(G)::value, at = r * NG + g;
            // (two products and a conversion: the instructions that multiply into half a register take twice as long)
            if constexpr (g < NG) {
                typedef float f2 __attribute__((ext_vector_type(2)));
                typedef _Float16 h2 __attribute__((ext_vector_type(2)));
                f2 y = {__builtin_fmaf(p[0], (float)half_of(vs[0][at / 2], at & 1), 0.0f), __builtin_fmaf(p[1], (float)half_of(vs[1][at / 2], at & 1), 0.0f)};
                // (last: a weight without a value may be large, and infinite times 0 is no number)
                if constexpr (!PLAIN) y *= factor[g];
                x[g][r] = __builtin_bit_cast(unsigned, __builtin_convertvector(y, h2));
            }
        };
        group(std::integral_constant<int, 0>{});
        group(std::integral_constant<int, 1>{});
        group(std::integral_constant<int, 2>{});
        group(std::integral_constant<int, 3>{});
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
    unsigned top = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        top = max3_pairs(top, x[g][0], x[g][1]);
        top = max3_pairs(top, x[g][2], x[g][3]);
        w[g] = __builtin_bit_cast(half8, (c4u){x[g][0], x[g][1], x[g][2], x[g][3]});
    }
    return __builtin_amdgcn_ballot_w64(sum > P_LIMIT || half_of(top, 0) > W_LIMIT || half_of(top, 1) > W_LIMIT) != 0ull;
}
__device__ __forceinline__ void wave_order() {       // LDS written by other lanes of the wavefront: in program order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ void store4(void* out, long at, int type, c4f x) {
    if (type == TYPE_F16) {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        *(h4*)((_Float16*)out + at) = __builtin_convertvector(x, h4);
    } else {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        *(b4*)((__bf16*)out + at) = __builtin_convertvector(x, b4);
    }
}
__device__ __forceinline__ float over_h(float x, bool sum) {
    const float y = __shfl_xor(x, 16, 64);
    x = sum ? x + y : __builtin_fmaxf(x, y);
    const float z = __shfl_xor(x, 32, 64);
    return sum ? x + z : __builtin_fmaxf(x, z);
}
// All references of a row raised to what the 32 keys of a lane and the three others of its column ask for, the sums l and O with them.  (The
// logarithm of a scale of 0 is -infinity: that key does not ask.)
template <int NG, int CT, class S>
__device__ __forceinline__ void raise_references(const float (&s)[2][4], float sc, const S (&vs)[2], References<NG>& ref, float& l, c4f (&o)[CT]) {
    float most[NG], alpha[NG], score = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) score = __builtin_fmaxf(score, s[j][r] * sc);
    score = over_h(score, false);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        most[g] = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                most[g] = __builtin_fmaxf(most[g], __builtin_fmaf(s[j][r], sc, __builtin_amdgcn_logf((float)half_of(vs[j][(r * NG + g) / 2], (r * NG + g) & 1)) - RAISE));
        most[g] = over_h(most[g], false);
    }
    l *= ref.raise(most, score, alpha);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) o[ct] *= alpha[ct * NG / CT];
}
}  // namespace

namespace {
// Which (sequence, head), tile of rows and chunk of keys a workgroup has.  One tile of rows: nothing is shared, the first chunks of
// all slabs come first and the last ones, which short sequences do not have, fill up behind them.  Several: slabs dealt out to the
// XCDs, so that the workgroups of one share its keys in one L2; the tiles that see most first.
struct RowsPlace {
    int slab, tile, split, slabs;
    __device__ __forceinline__ RowsPlace(const Cache4& c, const CacheQueries& q, int tiles, int n_splits) {
        slabs = q.B * c.heads;
        if (tiles == 1) {
            slab = blockIdx.x % slabs;
            split = blockIdx.x / slabs;
            tile = 0;
            return;
        }
        const int per_slab = tiles * n_splits;
        int rest;
        if (slabs % 8 == 0) {
            const int i = blockIdx.x >> 3;
            slab = (i / per_slab) * 8 + (blockIdx.x & 7);
            rest = i % per_slab;
        } else {
            slab = blockIdx.x / per_slab;
            rest = blockIdx.x % per_slab;
        }
        split = rest % n_splits;
        tile = tiles - 1 - rest / n_splits;
    }
};
// Where a row's result goes: the output, or the partial results of a chunk, [chunk][slab][row][D] normalized fp32 and the base-2
// logarithm of their sums.
struct RowResult {
    float norm, log_sum;
    size_t part_row, lse_at;
    long b, hq;
    int tq;
    // live: the row is there; M, total: reference and sum of its weights
    __device__ __forceinline__ RowResult(const RowsPlace& at, const CacheQueries& q, int head, int share, int row, bool live, float M, float total,
                                         int all_rows) {
        live = live && total != 0.0f;
        norm = live ? 1.0f / total : 0.0f;
        // (M and the sum's exponent are whole numbers that nearly cancel where V's scales are small: their sum first, without rounding)
        log_sum = live ? (M + (float)__builtin_amdgcn_frexp_expf(total)) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(total)) : -__builtin_inff();
        part_row = ((size_t)at.split * at.slabs + at.slab) * all_rows + row;
        tq = row / share;
        b = at.slab / (q.Hq / share);
        hq = head * share + row - tq * share;
        lse_at = ((size_t)b * q.Hq + hq) * q.Nq + tq;
    }
    __device__ __forceinline__ void put_sum(const CacheQueries& q, float* lse, float* part_lse, bool partial) const {
        if (partial) part_lse[part_row] = log_sum;
        else if (lse != nullptr) lse[lse_at] = log_sum * LN2;
    }
    // channels d .. d + 3
    template <int D>
    __device__ __forceinline__ void put(const CacheQueries& q, void* out, const RowStrides& os, float* part, c4f x, int d) const {
        x = norm == 0.0f ? (c4f){0.0f, 0.0f, 0.0f, 0.0f} : x * norm;
        if (part != nullptr) *(c4f*)(part + part_row * D + d) = x;
        else store4(out, b * os.b + hq * os.h + tq * os.n + d, q.type, x);
    }
};
}  // namespace

// grid: (tile of rows, chunk of keys, (sequence, head)) from one index.  part != nullptr: partial results, [chunk][slab][row][D]
// normalized fp32 and the base-2 logarithm of their sums.
// (Three wavefronts per SIMD where 168 registers are enough: with four scales of 128 channels they are not, 119 us for 117.)
template <int D, int NG, int QT>
__global__ void __launch_bounds__(WAVES * 64, (QT == 1 ? NG * D < 512 : D == 64) ? 3 : 2)
cache4_attn_kernel(Cache4 c, CacheQueries q, void* __restrict__ out, RowStrides os, float* __restrict__ lse, float* __restrict__ part,
                   float* __restrict__ part_lse, int tiles, int n_splits, int chunk) {
    constexpr int CT = D / 16, STEPS = D / 32 / NG;
    typedef WaveLds<D, NG> Lds;
    constexpr int MERGE = WAVES * CT * 64 * 16, STAGE = WAVES * (int)sizeof(Lds);
    __shared__ __attribute__((aligned(16))) unsigned char lds[MERGE > STAGE ? MERGE : STAGE];
    __shared__ float s_m[WAVES][16], s_l[WAVES][16];
    // (32 rows and four scales of 128 channels: no registers for the second tile's queries, which all wavefronts have alike; there, and with 16
    // rows and two scales where three wavefronts fit on a SIMD, nor for addresses from one tile to the next)
    constexpr bool STAGED = QT == 2 && NG * D == 512, ADDRESSES_ANEW = STAGED || (QT == 1 && NG == 2);
    __shared__ half8 s_query[STAGED ? D / 32 : 1][64];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const RowsPlace at(c, q, tiles, n_splits);
    const int b = at.slab / c.heads, head = at.slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int row0 = at.tile * 16 * QT, all_rows = q.Nq * share;
    const int there = min(range.rows - row0, 16 * QT);               // rows of this workgroup that are there
    const int first_end = there > 0 ? range.end(row0 / share, q.causal) : 0;
    const int last_end = there > 0 ? range.end((row0 + there - 1) / share, q.causal) : 0;
    const int k_begin = at.split * chunk, k_end = min(k_begin + chunk, last_end);
    if (part != nullptr && k_begin >= last_end) return;              // (the merge knows)

    Queries4<D> query[QT];
    float sc[QT], l[QT];
    References<NG> ref[QT];
    int end[QT];
    c4f o[QT][CT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int row = row0 + min(16 * i + col, max(there - 1, 0)), tq = row / share, g = row - tq * share;
        sc[i] = query[i].load(q, b * q.strides.b + (head * share + g) * q.strides.h + tq * q.strides.n, h);
        end[i] = range.end(tq, q.causal);
        ref[i].clear();
        l[i] = 0.0f;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[i][ct] = (c4f){0.0f, 0.0f, 0.0f, 0.0f};
    }

    if constexpr (STAGED) {
        if (wave == 0) {
#pragma unroll
            for (int n = 0; n < D / 32; ++n) s_query[n][lane] = query[1].op[n];
        }
        __syncthreads();
    }
    Lds& mine = *(Lds*)(lds + wave * sizeof(Lds));
    const int* const table = c.table + (size_t)b * c.columns;
    const unsigned char* const head_at = c.data + (size_t)head * c.block_bytes;
    typedef KeyTile<D, NG, true> Tile;
    typedef typename Tile::words words;
    constexpr int NEXT = TILE * WAVES;
    Tile tile;
    PageIds pages;
    int k0 = k_begin + TILE * wave;
    if (k0 < k_end) {
        pages.look_up(c, table, k0);
        tile.request(c, head_at, pages, k0, lane);
        pages.look_up(c, table, k0 + NEXT);
    }
    EmptyGroups<NG> groups;
    bool plain = true;                  // the wavefront's rows have nothing but M
    for (; k0 < k_end; k0 += NEXT) {
        wave_order();
        // ---- the tile to LDS.  The scales of a row past the last key are perhaps no numbers: 0 instead.
        const unsigned bad = tile.bad;
        const bool absent = k0 + lane >= last_end || (bad >> h & 1);
        *(typename Tile::scale_t*)(mine.ks + lane * NG) = absent ? (typename Tile::scale_t)(0) : tile.ks;
        const typename Tile::scale_t v_scale = absent ? (typename Tile::scale_t)(0) : tile.vs;
        *(typename Tile::scale_t*)(mine.vs + lane * NG) = v_scale;
        if (NG > 1 && groups.empty != 0 && groups.look(v_scale)) plain = false;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) *(c4u*)(mine.v + v_chunk<D>((i * 1024 + lane * 16) / (D / 2), lane % (D / 32))) = tile.v[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) ((words*)mine.k)[j * 64 + lane] = tile.k[j];
        wave_order();
        if (k0 + NEXT < k_end) {
            tile.request(c, head_at, pages, k0 + NEXT, ADDRESSES_ANEW ? anew(lane) : lane);
            pages.look_up(c, table, k0 + 2 * NEXT);
        }
        const int v_key = 16 * (col >> 2) + 4 * h + (col & 3);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // ---- 32 keys: pieces 2 u and 2 u + 1.  An operand is made when its products are due and feeds all tiles of rows.
            typedef unsigned scales_t __attribute__((ext_vector_type(2 * NG)));
            scales_t vs[2];
            float s[QT][2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const words kw = ((const words*)mine.k)[(2 * u + j) * 64 + lane];
                const scales_t ks = *(const scales_t*)(mine.ks + (16 * (2 * u + j) + 4 * h) * NG);
                vs[j] = *(const scales_t*)(mine.vs + (16 * (2 * u + j) + 4 * h) * NG);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    c4f a[QT];
#pragma unroll
                    for (int n = 0; n < STEPS; ++n) {
                        const half8 k = operand(kw[g * STEPS + n], thousand);
#pragma unroll
                        for (int i = 0; i < QT; ++i) {
                            const half8 row = STAGED && i == 1 ? s_query[g * STEPS + n][lane] : query[i].op[g * STEPS + n];
                            a[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, row, n == 0 ? (c4f){0.0f, 0.0f, 0.0f, 0.0f} : a[i], 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < QT; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float scale = (float)half_of(ks[(r * NG + g) / 2], (r * NG + g) & 1);
                            s[i][j][r] = __builtin_fmaf(scale, a[i][r], g == 0 ? 0.0f : s[i][j][r]);
                        }
                }
            }
            if (k0 + 32 * u + 32 > first_end || (bad >> 2 * u & 3) != 0) {
#pragma unroll
                for (int i = 0; i < QT; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int last = bad >> (2 * u + j) & 1 ? 0 : end[i];
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (k0 + 16 * (2 * u + j) + 4 * h + r >= last) s[i][j][r] = -__builtin_inff();
                    }
            }
            half8 w[QT][NG];
            const bool again = !plain;
            // (no reference yet: no need to weigh twice, 2 us of 30 where a wavefront has one tile.  One tile of rows has no registers for the
            // branch: 108 us instead of 135)
            const bool first = QT > 1 && u == 0 && k0 == k_begin + TILE * wave;
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                float sum;
                if (first || weigh<true, NG>(s[i], sc[i], ref[i], vs, w[i], sum) || again) {
                    const scales_t own[2] = {anew(vs[0]), anew(vs[1])};
                    raise_references<NG>(s[i], sc[i], own, ref[i], l[i], o[i]);
                    plain = ref[0].alike(groups) && ref[QT - 1].alike(groups);
                    weigh<NG == 1, NG>(s[i], sc[i], ref[i], vs, w[i], sum);
                }
                l[i] += sum;
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                // V transposed: channel 16 ct + lane % 16, nibble i of the words: key 16 (i / 4) + 4 h + i % 4
                const c2i vt = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
                    (__attribute__((address_space(3))) c2i*)(mine.v + v_chunk<D>(v_key, ct >> 1) + 8 * (ct & 1)));
                const half8 v = operand((unsigned)vt[u], thousand);
#pragma unroll
                for (int i = 0; i < QT; ++i) o[i][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[i][ct * NG / CT], o[i][ct], 0, 0, 0);
            }
        }
    }

    // ---- the wavefronts' results: O = sum f_w O_w / sum f_w l_w, f_w = 2^(M_w - max M)
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const float lw = over_h(l[i], true);
        __syncthreads();                // the tiles, or the query tile before, have been read
        if (h == 0) {
            s_m[wave][col] = ref[i].M;
            s_l[wave][col] = lw;
        }
        __syncthreads();
        float top = s_m[0][col], total = 0.0f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = __builtin_fmaxf(top, s_m[w][col]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) total = __builtin_fmaf(s_l[w][col], __builtin_amdgcn_exp2f(s_m[w][col] - top), total);
        const float f = __builtin_amdgcn_exp2f(ref[i].M - top);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) *(c4f*)(lds + ((wave * CT + ct) * 64 + lane) * 16) = o[i][ct] * (f * ref[i].back(ct * NG / CT));
        __syncthreads();
        const int row = row0 + 16 * i + col;
        if (row >= all_rows) continue;
        const RowResult r(at, q, head, share, row, row < range.rows, top, total, all_rows);
        if (wave == 0 && h == 0) r.put_sum(q, lse, part_lse, part != nullptr);
#pragma unroll
        for (int n = 0; n < CT / WAVES; ++n) {
            const int ct = wave + WAVES * n;
            c4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) x += *(const c4f*)(lds + ((w * CT + ct) * 64 + lane) * 16);
            r.template put<D>(q, out, os, part, x, 16 * ct + 4 * h);
        }
    }
}

// ---- at most four rows (a decoding step of up to four query heads per key head)
namespace {
// the sum over the lanes 4 apart of 16, in all of them
__device__ __forceinline__ float over_fours(float x) {
    const auto turned = [](float v, auto ctrl) {
        const int i = __builtin_bit_cast(int, v);
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, false));
    };
    x += turned(x, std::integral_constant<int, 0x128>{});        // the lane 8 before, round 16
    return x + turned(x, std::integral_constant<int, 0x124>{});  // 4 before
}
}  // namespace

// With four rows a quarter of the score products' columns would be of use.  Column 4 j + c of them is row c for the keys of piece j: the
// queries of piece j's product are zero in the other columns, and the four products of a tile add up into one.  A lane has 4
// scores per tile instead of 16 and weighs those; its weights stand, in its column of the second product, at the keys of its
// piece beside zeros, and the columns of a row are added up at the end.  Some 490 vector instructions per tile for 650; 256 slabs of 8K to 16K
// keys of 128 channels with four scales 108 us for 117, the same loads alone 82.  (The queries in LDS, for three wavefronts per
// SIMD instead of two: no change.)
template <int D, int NG>
__global__ void __launch_bounds__(WAVES * 64, D == 64 ? 3 : 2)
cache4_attn_few_kernel(Cache4 c, CacheQueries q, void* __restrict__ out, RowStrides os, float* __restrict__ lse, float* __restrict__ part,
                       float* __restrict__ part_lse, int n_splits, int chunk) {
    constexpr int CT = D / 16, STEPS = D / 32 / NG;
    typedef WaveLds<D, NG> Lds;
    constexpr int MERGE = WAVES * CT * 16 * 16, STAGE = WAVES * (int)sizeof(Lds);
    __shared__ __attribute__((aligned(16))) unsigned char lds[MERGE > STAGE ? MERGE : STAGE];
    __shared__ float s_m[WAVES][4], s_l[WAVES][4];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const int own = col & 3, piece = col >> 2;                      // the column's row, and the keys it has
    const RowsPlace at(c, q, 1, n_splits);
    const int b = at.slab / c.heads, head = at.slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int all_rows = q.Nq * share;
    const int first_end = range.rows > 0 ? range.end(0, q.causal) : 0, last_end = range.rows > 0 ? range.end(range.count - 1, q.causal) : 0;
    const int k_begin = at.split * chunk, k_end = min(k_begin + chunk, last_end);
    if (part != nullptr && k_begin >= last_end) return;              // (the merge knows)

    half8 query[4][D / 32];
    float sc, l = 0.0f;
    References<NG> ref;
    ref.clear();
    int end;
    {
        const int row = min(own, max(range.rows - 1, 0)), tq = row / share, g = row - tq * share;
        Queries4<D> mine;
        sc = mine.load(q, b * q.strides.b + (head * share + g) * q.strides.h + tq * q.strides.n, h);
        end = range.end(tq, q.causal);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) query[j][i] = piece == j ? mine.op[i] : (half8){};
    }
    // what brings half r % 2 of a register to where the weights of keys r of the pieces 2 u (low) and 2 u + 1 (high) stand
    unsigned place[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const unsigned bytes = r ? 0x0302u : 0x0100u;
            place[u][r] = piece == 2 * u ? 0x0c0c0000u | bytes : piece == 2 * u + 1 ? bytes << 16 | 0x0c0cu : 0x0c0c0c0cu;
        }
    c4f o[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) o[ct] = (c4f){0.0f, 0.0f, 0.0f, 0.0f};

    Lds& mine = *(Lds*)(lds + wave * sizeof(Lds));
    const int* const table = c.table + (size_t)b * c.columns;
    const unsigned char* const head_at = c.data + (size_t)head * c.block_bytes;
    typedef KeyTile<D, NG, true> Tile;
    typedef typename Tile::words words;
    typedef unsigned scales_t __attribute__((ext_vector_type(2 * NG)));
    constexpr int NEXT = TILE * WAVES;
    Tile tile;
    PageIds pages;
    int k0 = k_begin + TILE * wave;
    if (k0 < k_end) {
        pages.look_up(c, table, k0);
        tile.request(c, head_at, pages, k0, lane);
        pages.look_up(c, table, k0 + NEXT);
    }
    EmptyGroups<NG> groups;
    bool plain = true;                  // the wavefront's rows have nothing but M
    for (; k0 < k_end; k0 += NEXT) {
        wave_order();
        // ---- the tile to LDS.  The scales of a row past the last key are perhaps no numbers: 0 instead.
        const unsigned bad = tile.bad;
        const bool absent = k0 + lane >= last_end || (bad >> h & 1);
        *(typename Tile::scale_t*)(mine.ks + lane * NG) = absent ? (typename Tile::scale_t)(0) : tile.ks;
        const typename Tile::scale_t v_scale = absent ? (typename Tile::scale_t)(0) : tile.vs;
        *(typename Tile::scale_t*)(mine.vs + lane * NG) = v_scale;
        if (NG > 1 && groups.empty != 0 && groups.look(v_scale)) plain = false;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) *(c4u*)(mine.v + v_chunk<D>((i * 1024 + lane * 16) / (D / 2), lane % (D / 32))) = tile.v[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) ((words*)mine.k)[j * 64 + lane] = tile.k[j];
        wave_order();
        if (k0 + NEXT < k_end) {
            tile.request(c, head_at, pages, k0 + NEXT, lane);
            pages.look_up(c, table, k0 + 2 * NEXT);
        }
        // ---- scores of keys 16 piece + 4 h + r for row `own`
        const int key = 16 * piece + 4 * h;
        const scales_t ks = *(const scales_t*)(mine.ks + key * NG), vs = *(const scales_t*)(mine.vs + key * NG);
        c4f a[NG];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const words kw = ((const words*)mine.k)[j * 64 + lane];
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int n = 0; n < STEPS; ++n)
                    a[g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(kw[g * STEPS + n], thousand), query[j][g * STEPS + n],
                                                                  j == 0 && n == 0 ? (c4f){0.0f, 0.0f, 0.0f, 0.0f} : a[g], 0, 0, 0);
        }
        float s[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int g = 0; g < NG; ++g) s[r] = __builtin_fmaf((float)half_of(ks[(r * NG + g) / 2], (r * NG + g) & 1), a[g][r], g == 0 ? 0.0f : s[r]);
        if (k0 + TILE > first_end || bad != 0) {
            const int last = bad >> piece & 1 ? 0 : end;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (k0 + key + r >= last) s[r] = -__builtin_inff();
        }
        // ---- weights, as weigh() forms them: two keys to a register
        unsigned x[NG][2];
        float sum;
        auto weights = [&](auto P) {
            constexpr bool PLAIN = decltype(P)::value;
            typedef float f2 __attribute__((ext_vector_type(2)));
            typedef _Float16 h2 __attribute__((ext_vector_type(2)));
            float p[4];
            sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, r & 1 ? -(ref.M + 4.0f) : -ref.M));
                sum = r & 1 ? __builtin_fmaf(p[r], 16.0f, sum) : sum + p[r];
            }
            unsigned top = 0;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float factor = PLAIN ? 1.0f : ldexpf(1.0f, ref.distance(g));
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    f2 y = {__builtin_fmaf(p[r], (float)half_of(vs[(r * NG + g) / 2], (r * NG + g) & 1), 0.0f),
                            __builtin_fmaf(p[r + 1], (float)half_of(vs[((r + 1) * NG + g) / 2], ((r + 1) * NG + g) & 1), 0.0f)};
                    if constexpr (!PLAIN) y *= factor;
                    x[g][r / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(y, h2));
                }
                top = max3_pairs(top, x[g][0], x[g][1]);
            }
            return __builtin_amdgcn_ballot_w64(sum > P_LIMIT || half_of(top, 0) > W_LIMIT || half_of(top, 1) > W_LIMIT) != 0ull;
        };
        if (__builtin_expect(weights(std::true_type{}) || !plain, 0)) {
            const auto over_keys = [](float x) {
                x = __builtin_fmaxf(x, __shfl_xor(x, 4, 64));
                return over_h(__builtin_fmaxf(x, __shfl_xor(x, 8, 64)), false);
            };
            float most[NG], alpha[NG], score = -__builtin_inff();
#pragma unroll
            for (int r = 0; r < 4; ++r) score = __builtin_fmaxf(score, s[r] * sc);
            score = over_keys(score);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                most[g] = -__builtin_inff();
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    most[g] = __builtin_fmaxf(most[g], __builtin_fmaf(s[r], sc, __builtin_amdgcn_logf((float)half_of(vs[(r * NG + g) / 2], (r * NG + g) & 1)) - RAISE));
                most[g] = over_keys(most[g]);
            }
            l *= ref.raise(most, score, alpha);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct] *= alpha[ct * NG / CT];
            plain = ref.alike(groups);
            weights(std::integral_constant<bool, NG == 1>{});
        }
        l += sum;
        half8 w[2][NG];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int g = 0; g < NG; ++g)
                w[u][g] = __builtin_bit_cast(half8, (c4u){__builtin_amdgcn_perm(0u, x[g][0], place[u][0]), __builtin_amdgcn_perm(0u, x[g][0], place[u][1]),
                                                         __builtin_amdgcn_perm(0u, x[g][1], place[u][0]), __builtin_amdgcn_perm(0u, x[g][1], place[u][1])});
        const int v_key = 16 * (col >> 2) + 4 * h + (col & 3);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            // V transposed: channel 16 ct + lane % 16, nibble i of the words: key 16 (i / 4) + 4 h + i % 4
            const c2i vt = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
                (__attribute__((address_space(3))) c2i*)(mine.v + v_chunk<D>(v_key, ct >> 1) + 8 * (ct & 1)));
#pragma unroll
            for (int u = 0; u < 2; ++u)
                o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand((unsigned)vt[u], thousand), w[u][ct * NG / CT], o[ct], 0, 0, 0);
        }
    }

    // ---- the columns' and the wavefronts' results: O = sum f_w O_w / sum f_w l_w, f_w = 2^(M_w - max M)
    const float lw = over_fours(over_h(l, true));
    __syncthreads();                    // the tiles have been read
    if (lane < 4) {
        s_m[wave][own] = ref.M;
        s_l[wave][own] = lw;
    }
    __syncthreads();
    float top = s_m[0][own], total = 0.0f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = __builtin_fmaxf(top, s_m[w][own]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total = __builtin_fmaf(s_l[w][own], __builtin_amdgcn_exp2f(s_m[w][own] - top), total);
    const float f = __builtin_amdgcn_exp2f(ref.M - top);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        c4f x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = over_fours(o[ct][r]) * (f * ref.back(ct * NG / CT));
        if (piece == 0) *(c4f*)(lds + ((wave * CT + ct) * 16 + 4 * h + own) * 16) = x;
    }
    __syncthreads();
    if (piece != 0 || own >= all_rows) return;
    const RowResult r(at, q, head, share, own, own < range.rows, top, total, all_rows);
    if (wave == 0 && h == 0) r.put_sum(q, lse, part_lse, part != nullptr);
#pragma unroll
    for (int n = 0; n < CT / WAVES; ++n) {
        const int ct = wave + WAVES * n;
        c4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += *(const c4f*)(lds + ((w * CT + ct) * 16 + 4 * h + own) * 16);
        r.template put<D>(q, out, os, part, x, 16 * ct + 4 * h);
    }
}

// ---- many rows: operands made once for all of a workgroup's wavefronts
namespace {
// A wavefront's share of a tile of 64 keys, as it comes from memory: K's words of piece `wave`, a quarter of every V row, the
// scales (wavefront 0: K's, 1: V's; a key per lane).
template <int D, int NG>
struct TileShare {
    typedef typename ScaleWord<NG>::type scale_t;
    typedef unsigned words __attribute__((ext_vector_type(D / 32)));
    static constexpr int ROW = D / 2;
    words k, v;
    scale_t scale;
    unsigned bad;
    __device__ __forceinline__ void request(const Cache4& c, const unsigned char* head, const PageIds& pages, int k0, int lane, int wave) {
        const int col = lane & 15, h = lane >> 4, mask = c.page() - 1;
        const unsigned char *piece, *mine;          // the blocks of piece `wave` and of the lane's key
        int piece_row, row;
        if (c.shift >= 6) {
            bool ok;
            piece = mine = KeyTile<D, NG, true>::block(c, head, pages.id[0], ok);
            bad = ok ? 0u : 15u;
            piece_row = (k0 & mask) + 16 * wave;
            row = (k0 & mask) + lane;
        } else {
            const unsigned char* at[4];
            bad = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bool ok;
                at[j] = KeyTile<D, NG, true>::block(c, head, pages.id[j], ok);
                if (!ok) bad |= 1u << j;
            }
            piece = mine = at[0];
#pragma unroll
            for (int j = 1; j < 4; ++j) {
                piece = wave == j ? at[j] : piece;
                mine = h == j ? at[j] : mine;
            }
            piece_row = (k0 + 16 * wave) & mask;
            row = (k0 + lane) & mask;
        }
        k = *(const words*)(piece + (piece_row + col) * ROW + h * (D / 8));
        v = *(const words*)(mine + (ROW << c.shift) + row * ROW + wave * (ROW / 4));
        if (wave < 2) scale = *(const scale_t*)(mine + ((D + 2 * NG * wave) << c.shift) + row * 2 * NG);
    }
};
// A tile as operands: [piece][step] of K, [half][channels of 16] of V, 16 bytes per lane each; the scales.
template <int D, int NG>
struct TileStage {
    half8 k[4][D / 32][64], v[2][D / 16][64];
    _Float16 ks[TILE * NG], vs[TILE * NG];
};
}  // namespace

// 128 rows per workgroup, 32 per wavefront; the wavefronts walk the tiles together.  Each makes a quarter of a tile's operands
// in LDS, one tile ahead, in two buffers, a barrier per tile.  The 18 vector instructions that a word of K and a word of V cost are
// spent once for 128 rows instead of once for 32; the price is the LDS, 128 KB read per tile and 128 rows.
template <int D, int NG>
__global__ void __launch_bounds__(WAVES * 64, 2)
cache4_attn_rows_kernel(Cache4 c, CacheQueries q, void* __restrict__ out, RowStrides os, float* __restrict__ lse, float* __restrict__ part,
                        float* __restrict__ part_lse, int tiles, int n_splits, int chunk) {
    constexpr int QT = 2, CT = D / 16, STEPS = D / 32 / NG, RAW = TILE * D / 8;
    __shared__ TileStage<D, NG> stage[2];
    __shared__ __attribute__((aligned(16))) unsigned char raw_v[WAVES][RAW];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const RowsPlace at(c, q, tiles, n_splits);
    const int b = at.slab / c.heads, head = at.slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int all_rows = q.Nq * share, group0 = at.tile * WAVES * 16 * QT, row0 = group0 + wave * 16 * QT;
    // what the wavefront's first and last rows see, and the workgroup's last
    const int there = min(range.rows - row0, 16 * QT), last_there = min(range.rows - group0, WAVES * 16 * QT);
    const int first_end = there > 0 ? range.end(row0 / share, q.causal) : 0;
    const int wave_end = there > 0 ? range.end((row0 + there - 1) / share, q.causal) : 0;
    const int last_end = last_there > 0 ? range.end((group0 + last_there - 1) / share, q.causal) : 0;
    const int k_begin = at.split * chunk, k_end = min(k_begin + chunk, last_end);
    if (part != nullptr && k_begin >= last_end) return;              // (the merge knows)

    Queries4<D> query[QT];
    float sc[QT], l[QT];
    References<NG> ref[QT];
    int end[QT];
    c4f o[QT][CT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int row = min(row0 + 16 * i + col, max(range.rows - 1, 0)), tq = row / share, g = row - tq * share;
        sc[i] = query[i].load(q, b * q.strides.b + (head * share + g) * q.strides.h + tq * q.strides.n, h);
        end[i] = range.end(tq, q.causal);
        ref[i].clear();
        l[i] = 0.0f;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[i][ct] = (c4f){0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int* const table = c.table + (size_t)b * c.columns;
    const unsigned char* const head_at = c.data + (size_t)head * c.block_bytes;
    TileShare<D, NG> own;
    PageIds pages;
    // the share that has arrived, the tile from k0 on, into a buffer
    auto put = [&](TileStage<D, NG>& to, int k0) {
        typedef typename TileShare<D, NG>::words words;
        typedef typename TileShare<D, NG>::scale_t scale_t;
        wave_order();
        *(words*)(raw_v[wave] + lane * (D / 8)) = own.v;
        if (wave < 2) {
            // (a row past the last key holds anything, its scale is no number perhaps: 0 instead)
            const bool absent = k0 + lane >= last_end || (own.bad >> h & 1);
            *(scale_t*)((wave == 0 ? to.ks : to.vs) + lane * NG) = absent ? (scale_t)(0) : own.scale;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) to.k[wave][i][lane] = operand(own.k[i], thousand);
        wave_order();
        // V transposed: lane's channel, nibble i of the words: key 16 (i / 4) + 4 h + i % 4
        const int v_key = 16 * (col >> 2) + 4 * h + (col & 3);
#pragma unroll
        for (int n = 0; n < D / 64; ++n) {
            const c2i x = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) c2i*)(raw_v[wave] + v_key * (D / 8) + 8 * n));
            to.v[0][D / 64 * wave + n][lane] = operand((unsigned)x[0], thousand);
            to.v[1][D / 64 * wave + n][lane] = operand((unsigned)x[1], thousand);
        }
    };
    unsigned bad = 0;
    if (k_begin < k_end) {
        pages.look_up(c, table, k_begin);
        own.request(c, head_at, pages, k_begin, lane, wave);
        pages.look_up(c, table, k_begin + TILE);
        put(stage[0], k_begin);
        bad = own.bad;
        if (k_begin + TILE < k_end) {
            own.request(c, head_at, pages, k_begin + TILE, lane, wave);
            pages.look_up(c, table, k_begin + 2 * TILE);
        }
    }
    __syncthreads();
    typedef unsigned scales_t __attribute__((ext_vector_type(2 * NG)));
    struct Half {               // 32 keys: scores, V's scales, weights
        float s[QT][2][4];
        scales_t vs[2];
        half8 w[QT][NG];
        float sum[QT];
    };
    auto score = [&](Half& x, const TileStage<D, NG>& now, int u) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const scales_t ks = *(const scales_t*)(now.ks + (16 * (2 * u + j) + 4 * h) * NG);
            x.vs[j] = *(const scales_t*)(now.vs + (16 * (2 * u + j) + 4 * h) * NG);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                c4f a[QT];
#pragma unroll
                for (int n = 0; n < STEPS; ++n) {
                    const half8 k = now.k[2 * u + j][g * STEPS + n][lane];
#pragma unroll
                    for (int i = 0; i < QT; ++i)
                        a[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, query[i].op[g * STEPS + n], n == 0 ? (c4f){0.0f, 0.0f, 0.0f, 0.0f} : a[i], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < QT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float scale = (float)half_of(ks[(r * NG + g) / 2], (r * NG + g) & 1);
                        x.s[i][j][r] = __builtin_fmaf(scale, a[i][r], g == 0 ? 0.0f : x.s[i][j][r]);
                    }
            }
        }
    };
    auto hide = [&](Half& x, int k0, int u) {
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int last = bad >> (2 * u + j) & 1 ? 0 : end[i];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (k0 + 16 * (2 * u + j) + 4 * h + r >= last) x.s[i][j][r] = -__builtin_inff();
            }
    };
    EmptyGroups<NG> groups;
    bool plain = true;                  // the wavefront's rows have nothing but M
    auto weighed = [&](Half& x, auto P) {
        bool low = false;
#pragma unroll
        for (int i = 0; i < QT; ++i) low |= weigh<decltype(P)::value, NG>(x.s[i], sc[i], ref[i], x.vs, x.w[i], x.sum[i]);
        return low;
    };
    // the references are too low, or groups have references of their own, which may be too low as well
    auto again = [&](Half& x) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            const scales_t own[2] = {anew(x.vs[0]), anew(x.vs[1])};
            raise_references<NG>(x.s[i], sc[i], own, ref[i], l[i], o[i]);
        }
        plain = ref[0].alike(groups) && ref[QT - 1].alike(groups);
        weighed(x, std::integral_constant<bool, NG == 1>{});
    };
    auto values = [&](const Half& x, const TileStage<D, NG>& now, int u) {
#pragma unroll
        for (int i = 0; i < QT; ++i) l[i] += x.sum[i];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const half8 v = now.v[u][ct][lane];
#pragma unroll
            for (int i = 0; i < QT; ++i) o[i][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, x.w[i][ct * NG / CT], o[i][ct], 0, 0, 0);
        }
    };
    for (int k0 = k_begin, turn = 0; k0 < k_end; k0 += TILE, turn ^= 1) {
        const TileStage<D, NG>& now = stage[turn];
        const unsigned now_bad = bad;
        const bool more = k0 + TILE < k_end;
        if (k0 < wave_end) {
            // products of one half beside the other half's weights
            const bool masked = k0 + TILE > first_end || now_bad != 0;
            if (NG > 1 && groups.empty != 0 && groups.look(((const typename ScaleWord<NG>::type*)now.vs)[lane])) plain = false;
            if constexpr (NG <= 2) {
                Half x, y;
                score(x, now, 0);
                if (masked) hide(x, k0, 0);
                score(y, now, 1);
                if (__builtin_expect(weighed(x, std::true_type{}) || !plain, 0)) again(x);
                if (masked) hide(y, k0, 1);
                values(x, now, 0);
                if (__builtin_expect(weighed(y, std::true_type{}) || !plain, 0)) again(y);
                values(y, now, 1);
            } else {
                // (four groups' operands and scales: no registers for two halves)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    Half x;
                    score(x, now, u);
                    if (masked) hide(x, k0, u);
                    if (__builtin_expect(weighed(x, std::true_type{}) || !plain, 0)) again(x);
                    values(x, now, u);
                }
            }
        }
        if (more) {
            put(stage[turn ^ 1], k0 + TILE);
            bad = own.bad;
            if (k0 + 2 * TILE < k_end) {
                own.request(c, head_at, pages, k0 + 2 * TILE, lane, wave);
                pages.look_up(c, table, k0 + 3 * TILE);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const float total = over_h(l[i], true);
        const int row = row0 + 16 * i + col;
        if (row >= all_rows) continue;
        const RowResult r(at, q, head, share, row, row < range.rows, ref[i].M, total, all_rows);
        if (h == 0) r.put_sum(q, lse, part_lse, part != nullptr);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) r.template put<D>(q, out, os, part, o[i][ct] * ref[i].back(ct * NG / CT), 16 * ct + 4 * h);
    }
}

// O = sum_s w_s O_s / sum_s w_s, w_s = 2^(lse_s - max lse).  D / 4 threads hold a row, 4 channels each; LANES such groups take
// every LANES-th chunk, BATCH of them requested before the first is used, and add up through LDS.  Few rows of many chunks
// (a decoding step) have the whole workgroup on a row, many rows one group each.
template <int D, int LANES, int BATCH>
__global__ void __launch_bounds__(256) cache4_merge_kernel(Cache4 c, CacheQueries q, void* __restrict__ out, RowStrides os, float* __restrict__ lse,
                                                           const float* __restrict__ part, const float* __restrict__ part_lse, int chunk) {
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * LANES);
    __shared__ c4f s_x[LANES > 1 ? 256 : 1];
    __shared__ float s_top[LANES > 1 ? LANES : 1], s_sum[LANES > 1 ? LANES : 1];
    const int share = q.Hq / c.heads, all_rows = q.Nq * share, slabs = q.B * c.heads;
    const long at_row = (long)blockIdx.x * ROWS + (LANES > 1 ? 0 : threadIdx.x / TPR);
    if (at_row >= (long)slabs * all_rows) return;                    // (with several groups on a row: all of them)
    const int slab = (int)(at_row / all_rows), row = (int)(at_row - (long)slab * all_rows), d = threadIdx.x % TPR * 4;
    const int b = slab / c.heads, head = slab - b * c.heads, tq = row / share, g = row - tq * share;
    const RowRange range(c, q, b, share);
    const int end = row < range.rows ? range.end(tq, q.causal) : 0, n = (end + chunk - 1) / chunk;
    const int first = LANES > 1 ? threadIdx.x / TPR : 0;
    const long step = (long)slabs * all_rows;
    float top = UNSET, total = 0.0f;
    c4f x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = first; s0 < n; s0 += LANES * BATCH) {
        float ls[BATCH];
        c4f y[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            // (past the last chunk: the last one again, with weight 0)
            const int s = s0 + i * LANES, sc = s < n ? s : n - 1;
            const float v = part_lse[sc * step + at_row];
            y[i] = *(const c4f*)(part + (sc * step + at_row) * D + d);
            ls[i] = s < n ? v : -__builtin_inff();
        }
        __builtin_amdgcn_sched_barrier(0);
        float most = top;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) most = __builtin_fmaxf(most, ls[i]);
        const float keep = __builtin_amdgcn_exp2f(top - most);
        top = most;
        total *= keep;
        x *= keep;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float w = __builtin_amdgcn_exp2f(ls[i] - top);
            total += w;
            x += y[i] * w;
        }
    }
    if constexpr (LANES > 1) {
        s_x[threadIdx.x] = x;
        if (threadIdx.x % TPR == 0) {
            s_top[first] = top;
            s_sum[first] = total;
        }
        __syncthreads();
        if (first != 0) return;
        float most = s_top[0];
#pragma unroll
        for (int i = 1; i < LANES; ++i) most = __builtin_fmaxf(most, s_top[i]);
        total = 0.0f;
        x = (c4f){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < LANES; ++i) {
            const float f = __builtin_amdgcn_exp2f(s_top[i] - most);
            total = __builtin_fmaf(s_sum[i], f, total);
            x += s_x[i * TPR + threadIdx.x] * f;
        }
        top = most;
    }
    if (total != 0.0f) x *= 1.0f / total;
    if (d == 0 && lse != nullptr)
        lse[((size_t)b * q.Hq + head * share + g) * q.Nq + tq] = total != 0.0f ? (top + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
    store4(out, b * os.b + (head * share + g) * os.h + tq * os.n + d, q.type, x);
}

// ---- the weights of the keys
// The products are turned round: rows of queries times columns of keys, so that a key's sum runs over a lane's registers and the
// four lanes of a column (over 16 columns of rows: 192 vector instructions per tile, here 28).
namespace {
// a row's lse as the base-2 reference its weights are relative to; of a row that saw nothing one that leaves no weight
__device__ __forceinline__ float row_reference(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * LOG2E; }

// what the rows 4 h + r of a lane need: scale of the exponent, reference, slots seen
struct LaneRows {
    float sc[4], reference[4];
    int end[4];
};
// 16 rows from `first` on, on their way: queries, lse, slots seen by row lane % 16; of those behind the last the last one's query, which sees
// none here
template <int D>
struct SomeRows {
    Queries4<D> query;
    float lse;
    int end;
    __device__ __forceinline__ void request(const Cache4& c, const CacheQueries& q, const float* from, const RowRange& range, int b, int head, int first,
                                            int lane) {
        const int share = q.Hq / c.heads, at = first + (lane & 15), row = min(at, range.rows - 1), tq = row / share, g = row - tq * share;
        query.request(q, b * q.strides.b + (head * share + g) * q.strides.h + tq * q.strides.n, lane >> 4);
        lse = from[((size_t)b * q.Hq + head * share + g) * q.Nq + tq];
        end = at < range.rows ? range.end(tq, q.causal) : 0;
    }
    __device__ __forceinline__ float reference() const { return end > 0 ? row_reference(lse) : __builtin_inff(); }
};
template <int NG> using LaneScales = unsigned[(NG + 1) / 2];
// -> the weights that 16 rows give to the lane's key, the first R of the rows 4 h .. 4 h + 3; key: the slot.  whole: every row sees it
template <int D, int NG, int R = 4>
__device__ __forceinline__ float piece_weights(const half8 (&q)[D / 32], const half8 (&k)[D / 32], const LaneScales<NG>& ks, const LaneRows& rows, int key,
                                               bool whole) {
    constexpr int STEPS = D / 32 / NG;
    c4f s;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        c4f a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < STEPS; ++i) a = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[g * STEPS + i], k[g * STEPS + i], a, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = __builtin_fmaf((float)half_of(ks[g / 2], g & 1), a[r], g == 0 ? 0.0f : s[r]);
    }
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], rows.sc[r], -rows.reference[r]));
        sum += whole || key < rows.end[r] ? p : 0.0f;
    }
    return sum;
}
// the scales of a key, staged as [key][group]
template <int NG>
__device__ __forceinline__ void lane_scales(const _Float16* staged, int key, LaneScales<NG>& ks) {
    const typename ScaleWord<NG>::type w = *(const typename ScaleWord<NG>::type*)(staged + key * NG);
    if constexpr (NG == 4) {
        ks[0] = w[0];
        ks[1] = w[1];
    } else {
        ks[0] = w;
    }
}
// the sums of a tile's 64 keys over the lanes of a column, in LDS; pieces without a page get none
__device__ __forceinline__ void put_sums(const float (&sum)[4], unsigned bad, float* to, int lane) {
    const int col = lane & 15, h = lane >> 4;
    float mine = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = over_h(sum[j], true);
        mine = h == j ? x : mine;
    }
    to[16 * h + col] = bad >> h & 1 ? 0.0f : mine;
}
// a workgroup's sums for the slots [begin, end), of which no query sees those from `seen` on, added to what they had (which may
// be where they go)
__device__ __forceinline__ void add_sums(const float* sums, const float* had, float* to, int begin, int end, int seen) {
    __syncthreads();
    for (int key = begin + threadIdx.x; key < end; key += WAVES * 64)
        to[key] = (had != nullptr ? had[key] : 0.0f) + (key < seen ? sums[key - begin] : 0.0f);
}
}  // namespace

// At most 4 R rows (a decoding step): their operands stay in registers, a wavefront walks tiles of keys, the next one on its way.  Row i
// is row 4 (i / R) + i % R of the product, so that a lane has R of them and none of its arithmetic is for rows that are not there.
template <int D, int NG, int R>
__global__ void __launch_bounds__(WAVES * 64, 4) cache4_weights_few_kernel(Cache4 c, CacheQueries q, const float* __restrict__ lse,
                                                                        const float* weights, float* out, int width, int chunk) {
    __shared__ __attribute__((aligned(16))) _Float16 s_ks[WAVES][TILE * NG];
    // (the sums wait here for one pass at the end: stores between the tiles would be waited for with the next tile's loads)
    __shared__ __attribute__((aligned(16))) float s_sum[FEW_CHUNK];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const int slab = blockIdx.y, b = slab / c.heads, head = slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int last_end = range.rows > 0 ? range.end(range.count - 1, q.causal) : 0;
    constexpr int NEXT = TILE * WAVES;
    const int k_begin = blockIdx.x * chunk, k_end = min(k_begin + chunk, width), seen = min(k_end, last_end);
    int k0 = k_begin + TILE * wave;
    typedef KeyTile<D, NG, false> Tile;
    Tile tile;
    PageIds pages;
    const int* const table = c.table + (size_t)b * c.columns;
    const unsigned char* const head_at = c.data + (size_t)head * c.block_bytes;
    if (k0 < seen) {
        pages.look_up(c, table, k0);
        tile.request(c, head_at, pages, k0, lane);
        pages.look_up(c, table, k0 + NEXT);
        const int at = (col >> 2) * R + (col & 3), row = min(at, range.rows - 1), tq = row / share, g = row - tq * share;
        const bool is = (col & 3) < R && at < range.rows;
        const int first_end = range.end(0, q.causal);
        Queries4<D> query;
        const float sc = query.load(q, b * q.strides.b + (head * share + g) * q.strides.h + tq * q.strides.n, h);
        // (of 16 rows those that are not there leave no weight either)
        const float reference = is ? row_reference(lse[((size_t)b * q.Hq + head * share + g) * q.Nq + tq]) : __builtin_inff();
        const int end = is ? range.end(tq, q.causal) : 0;
        LaneRows rows;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rows.sc[r] = __shfl(sc, 4 * h + r, 64);
            rows.reference[r] = __shfl(reference, 4 * h + r, 64);
            rows.end[r] = __shfl(end, 4 * h + r, 64);
        }
        for (; k0 < seen; k0 += NEXT) {
            wave_order();
            *(typename Tile::scale_t*)(s_ks[wave] + lane * NG) = tile.ks;
            wave_order();
            typename Tile::words words[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) words[j] = tile.k[j];
            const unsigned bad = tile.bad;
            if (k0 + NEXT < seen) {
                tile.request(c, head_at, pages, k0 + NEXT, lane);
                pages.look_up(c, table, k0 + 2 * NEXT);
            }
            // (a piece at a time: with the operands of all 64 keys in registers two wavefronts fit on a SIMD instead of four)
            float sum[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                half8 k[D / 32];
                LaneScales<NG> ks;
                lane_scales<NG>(s_ks[wave], 16 * j + col, ks);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) k[i] = operand(words[j][i], thousand);
                sum[j] = piece_weights<D, NG, R>(query.op, k, ks, rows, k0 + 16 * j + col, k0 + TILE <= first_end);
            }
            put_sums(sum, bad, s_sum + (k0 - k_begin), lane);
        }
    }
    add_sums(s_sum, weights != nullptr ? weights + (size_t)slab * width : nullptr, out + (size_t)slab * width, k_begin, k_end, seen);
}

// More rows: a workgroup takes 256 keys, a wavefront 64 of them, whose operands stay in its registers.  The rows come 64 at a time:
// each wavefront makes the operands of 16 of them in LDS, and all use them.
template <int D, int NG>
__global__ void __launch_bounds__(WAVES * 64, 2) cache4_weights_kernel(Cache4 c, CacheQueries q, const float* __restrict__ lse,
                                                                       const float* weights, float* out, int width) {
    __shared__ __attribute__((aligned(16))) _Float16 s_ks[WAVES][TILE * NG];
    __shared__ half8 s_q[WAVES][D / 32][64];
    __shared__ __attribute__((aligned(16))) float s_sum[WAVES * TILE];
    __shared__ __attribute__((aligned(16))) float s_sc[WAVES][16], s_reference[WAVES][16];
    __shared__ __attribute__((aligned(16))) int s_end[WAVES][16];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const int slab = blockIdx.y, b = slab / c.heads, head = slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int last_end = range.rows > 0 ? range.end(range.count - 1, q.causal) : 0;
    const int k_first = blockIdx.x * WAVES * TILE, k0 = k_first + wave * TILE;
    float sum[4] = {};
    unsigned bad = 0;
    if (k_first < last_end) {                   // (the same for the whole workgroup)
        half8 k[4][D / 32];
        LaneScales<NG> ks[4];
        {
            PageIds pages;
            pages.look_up(c, c.table + (size_t)b * c.columns, k0);
            KeyTile<D, NG, false> tile;
            tile.request(c, c.data + (size_t)head * c.block_bytes, pages, k0, lane);
            *(typename ScaleWord<NG>::type*)(s_ks[wave] + lane * NG) = tile.ks;
            bad = tile.bad;
            wave_order();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lane_scales<NG>(s_ks[wave], 16 * j + col, ks[j]);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) k[j][i] = operand(tile.k[j][i], thousand);
            }
        }
        // the first row that sees a key of the workgroup
        int row0 = 0;
        if (q.causal) row0 = max(0, k_first + 1 - (range.length - range.count + 1)) * share / 64 * 64;
        SomeRows<D> some;
        some.request(c, q, lse, range, b, head, row0 + 16 * wave, lane);
        for (; row0 < range.rows; row0 += 64) {
            {
                const float sc = some.query.convert(q), reference = some.reference();
                const int end = some.end;
                __syncthreads();                // the rows before have been read
#pragma unroll
                for (int i = 0; i < D / 32; ++i) s_q[wave][i][lane] = some.query.op[i];
                if (h == 0) {
                    s_sc[wave][col] = sc;
                    s_reference[wave][col] = reference;
                    s_end[wave][col] = end;
                }
                some.request(c, q, lse, range, b, head, row0 + 64 + 16 * wave, lane);
                __syncthreads();
            }
#pragma unroll 1
            for (int w = 0; w < WAVES; ++w) {
                if (row0 + 16 * w >= range.rows) break;
                const int first_end = range.end((row0 + 16 * w) / share, q.causal);
                half8 op[D / 32];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) op[i] = s_q[w][i][lane];
                LaneRows rows;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    rows.sc[r] = s_sc[w][4 * h + r];
                    rows.reference[r] = s_reference[w][4 * h + r];
                    rows.end[r] = s_end[w][4 * h + r];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[j] += piece_weights<D, NG>(op, k[j], ks[j], rows, k0 + 16 * j + col, k0 + TILE <= first_end);
            }
        }
    }
    put_sums(sum, bad, s_sum + wave * TILE, lane);
    add_sums(s_sum, weights != nullptr ? weights + (size_t)slab * width : nullptr, out + (size_t)slab * width, k_first, min(k_first + WAVES * TILE, width),
             last_end);
}

// More rows where 256 keys at a time would leave the chip idle: a workgroup takes 64 keys, whose operands each of its NW wavefronts has
// in its registers, and a wavefront every NW-th 16 rows; the sums of a key are added in the wavefronts' order.  The price: the
// rows' operands are made for 64 keys instead of for 256.
template <int D, int NG, int NW>
__global__ void __launch_bounds__(NW * 64, 2) cache4_weights_rows_kernel(Cache4 c, CacheQueries q, const float* __restrict__ lse,
                                                                            const float* weights, float* out, int width) {
    __shared__ __attribute__((aligned(16))) _Float16 s_ks[NW][TILE * NG];
    __shared__ __attribute__((aligned(16))) float s_sum[NW][TILE];
    const unsigned thousand = thousands();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, h = lane >> 4;
    const int slab = blockIdx.y, b = slab / c.heads, head = slab - b * c.heads, share = q.Hq / c.heads;
    const RowRange range(c, q, b, share);
    const int last_end = range.rows > 0 ? range.end(range.count - 1, q.causal) : 0, k0 = blockIdx.x * TILE;
    float sum[4] = {};
    unsigned bad = 0;
    int row0 = 16 * wave;
    // (of the first rows those that see no key of the workgroup are passed over; where some row sees one they are fewer than all)
    if (q.causal && k0 < last_end) row0 += max(0, k0 + 1 - (range.length - range.count + 1)) * share / (16 * NW) * (16 * NW);
    if (k0 < last_end && row0 < range.rows) {
        half8 k[4][D / 32];
        LaneScales<NG> ks[4];
        {
            PageIds pages;
            pages.look_up(c, c.table + (size_t)b * c.columns, k0);
            KeyTile<D, NG, false> tile;
            tile.request(c, c.data + (size_t)head * c.block_bytes, pages, k0, lane);
            *(typename ScaleWord<NG>::type*)(s_ks[wave] + lane * NG) = tile.ks;
            bad = tile.bad;
            wave_order();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lane_scales<NG>(s_ks[wave], 16 * j + col, ks[j]);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) k[j][i] = operand(tile.k[j][i], thousand);
            }
        }
        SomeRows<D> some;
        some.request(c, q, lse, range, b, head, row0, lane);
        for (; row0 < range.rows; row0 += 16 * NW) {
            const float sc = some.query.convert(q), reference = some.reference();
            const int end = some.end, first_end = range.end(row0 / share, q.causal);
            half8 op[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) op[i] = some.query.op[i];
            some.request(c, q, lse, range, b, head, row0 + 16 * NW, lane);
            LaneRows rows;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                rows.sc[r] = __shfl(sc, 4 * h + r, 64);
                rows.reference[r] = __shfl(reference, 4 * h + r, 64);
                rows.end[r] = __shfl(end, 4 * h + r, 64);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum[j] += piece_weights<D, NG>(op, k[j], ks[j], rows, k0 + 16 * j + col, k0 + TILE <= first_end);
        }
    }
    put_sums(sum, bad, s_sum[wave], lane);
    __syncthreads();
    const int key = k0 + lane;
    if (wave != 0 || key >= width) return;
    float* const to = out + (size_t)slab * width;
    const float had = weights != nullptr ? weights[(size_t)slab * width + key] : 0.0f;
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) x += s_sum[w][lane];
    to[key] = had + (key < last_end ? x : 0.0f);
}

namespace {
// How a call is cut.  Keys: chunks of a multiple of 256, as many as it takes to have WANTED workgroups, two per compute unit (us with
// 256 / 512 / 1024 workgroups: 256 slabs of 16K keys 146 / 112 / 110, 8 of 128K 40 / 36 / 40, 64 of 16K with 64 rows 110 / 90 / 98), none
// shorter than 512 unless the caller asks for it or even those are fewer than the compute units (512 / 256: 20 slabs of 2.4K 14.8 / 13.1, 8 of
// 16K 15.3 / 13.4; but 6 of 24K, 276 of them, 16.7 / 17.3), and none at all where the walk is shorter than the merge's launch (one chunk /
// the best cut, 2 slabs: 768 keys of 128 channels 10.0 / 10.4, 1024 11.8 / 10.1; 1280 of 64 channels 9.8 / 10.1, 2048 13.2 / 10.0).  Sequences of a batch differ in length: up to four times as many chunks, of
// 2048 keys at least, even that out (256 slabs of 8K to 16K keys: 2 chunks 117, 8 chunks 106; all of 16K: 126 and 122; 80 of 18K to 36K
// with 52 rows: 3 chunks 238, 12 chunks 190; 32 of 16K to 32K with 1024 rows: 2 chunks 729, 8 chunks 646; 16 of 8K to 16K with
// 1024 rows: 4 chunks 195, 8 chunks 201).  Rows: 16 or 32 per workgroup, whose wavefronts share the keys; or 128, whose
// wavefronts share the operands, where there are that many and the chunks are long (us with 32 / 128, four scales per key: 4096 rows of 8
// slabs of 32K keys 1067 / 911, of 8K 270 / 253, of 4K 139 / 141, 2048 of 32 of 2K 151 / 131, 128 of 64 of 16K 170 / 140; chunks of 512
// keys: 512 rows of 32 slabs of 2K 47 / 56).
struct AttnPlan {
    int rows, tiles, n_splits, chunk;       // rows of a workgroup
};
constexpr long UNCUT = 768 * 128 * 16;
constexpr int COMPUTE_UNITS = 256, WANTED = 512, WANTED_FEW = 1024, MANY_ROWS = 128, LONG_CHUNK = 2048;
AttnPlan plan(int B, int Hq, int Hkv, int Nq, int D, int capacity, int requested) {
    const int rows = Hq / Hkv * Nq;
    auto cut = [&](int per) {
        AttnPlan p;
        p.rows = per;
        p.tiles = (rows + per - 1) / per;
        const long groups = (long)B * Hkv * p.tiles;
        long n = requested > 0 ? requested : WANTED / groups;
        const int least = requested > 0 || groups * (capacity / 512) < COMPUTE_UNITS ? 256 : 512;
        if (n > capacity / least) n = capacity / least;
        if (requested == 0 && B > 1) {
            const long more = 4 * WANTED / groups, most = capacity / LONG_CHUNK;
            n = n > more || n > most ? n : more < most ? more : most;
        }
        if (n < 1 || (requested == 0 && (long)capacity * D * per <= UNCUT)) n = 1;
        p.chunk = (int)(((capacity + n - 1) / n + 255) / 256 * 256);
        p.n_splits = (capacity + p.chunk - 1) / p.chunk;
        return p;
    };
    if (rows > 96) {
        const AttnPlan p = cut(MANY_ROWS);
        if (p.chunk >= LONG_CHUNK) return p;
    }
    return cut(rows <= 16 ? 16 : 32);
}
}  // namespace

// the merge: few rows of many chunks have a workgroup each
static bool wide_merge(size_t rows, int n_splits) { return rows <= 2048 && n_splits > 4; }

// of the larger of the call's launches
long long cache4_attn_workgroups(int B, int Hq, int Hkv, int Nq, int D, int capacity, int n_splits) {
    const AttnPlan p = plan(B, Hq, Hkv, Nq, D, capacity, n_splits);
    const long long attn = (long long)B * Hkv * p.tiles * p.n_splits;
    if (p.n_splits <= 1) return attn;
    const long long rows = (long long)B * Hq * Nq, per = wide_merge(rows, p.n_splits) ? 1 : 1024 / D, merge = (rows + per - 1) / per;
    return attn > merge ? attn : merge;
}

size_t cache4_attn_workspace(int B, int Hq, int Hkv, int Nq, int D, int capacity, int n_splits) {
    const AttnPlan p = plan(B, Hq, Hkv, Nq, D, capacity, n_splits);
    return p.n_splits <= 1 ? 0 : (size_t)p.n_splits * B * Hq * Nq * (D + 1) * sizeof(float);
}

template <int D, int NG>
static void launch_attn_form(const AttnPlan& p, const Cache4& c, const CacheQueries& q, void* out, const RowStrides& os, float* lse, float* part,
                             float* part_lse, hipStream_t st) {
    const unsigned grid = (unsigned)(q.B * c.heads * p.tiles * p.n_splits);
#define SAGE_CACHE4_ATTN(QT) cache4_attn_kernel<D, NG, QT><<<grid, WAVES * 64, 0, st>>>(c, q, out, os, lse, part, part_lse, p.tiles, p.n_splits, p.chunk)
    if (q.Hq / c.heads * q.Nq <= 4) cache4_attn_few_kernel<D, NG><<<grid, WAVES * 64, 0, st>>>(c, q, out, os, lse, part, part_lse, p.n_splits, p.chunk);
    else if (p.rows == 16) SAGE_CACHE4_ATTN(1);
    else if (p.rows == 32) SAGE_CACHE4_ATTN(2);
    else cache4_attn_rows_kernel<D, NG><<<grid, WAVES * 64, 0, st>>>(c, q, out, os, lse, part, part_lse, p.tiles, p.n_splits, p.chunk);
#undef SAGE_CACHE4_ATTN
}

hipError_t launch_cache4_attn(const Cache4& c, const CacheQueries& q, void* out, const RowStrides& os, float* lse, void* workspace,
                              int n_splits, hipStream_t st) {
    const AttnPlan p = plan(q.B, q.Hq, c.heads, q.Nq, c.D, c.capacity(), n_splits);
    const size_t rows = (size_t)q.B * q.Hq * q.Nq;
    float* const part = p.n_splits > 1 ? (float*)workspace : nullptr;
    float* const part_lse = p.n_splits > 1 ? part + p.n_splits * rows * c.D : nullptr;
    const int ng = c.groups;
    if (c.D == 64) {
        if (ng == 1) launch_attn_form<64, 1>(p, c, q, out, os, lse, part, part_lse, st);
        else launch_attn_form<64, 2>(p, c, q, out, os, lse, part, part_lse, st);
    } else {
        if (ng == 1) launch_attn_form<128, 1>(p, c, q, out, os, lse, part, part_lse, st);
        else if (ng == 2) launch_attn_form<128, 2>(p, c, q, out, os, lse, part, part_lse, st);
        else launch_attn_form<128, 4>(p, c, q, out, os, lse, part, part_lse, st);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.n_splits <= 1) return e;
#define SAGE_CACHE4_MERGE(D, LANES, BATCH) cache4_merge_kernel<D, LANES, BATCH><<<(unsigned)((rows * (D / 4) * LANES + 255) / 256), 256, 0, st>>>(c, q, out, os, lse, part, part_lse, p.chunk)
    const bool wide = wide_merge(rows, p.n_splits);
    if (c.D == 64) { if (wide) SAGE_CACHE4_MERGE(64, 16, 4); else SAGE_CACHE4_MERGE(64, 1, 4); }
    else { if (wide) SAGE_CACHE4_MERGE(128, 8, 4); else SAGE_CACHE4_MERGE(128, 1, 4); }
#undef SAGE_CACHE4_MERGE
    return hipGetLastError();
}

// 64 keys per workgroup where 256 would make fewer workgroups than there are compute units and the rows are several rounds of 64 (us with 64 /
// 256 keys: 828 rows of 12 slabs of 338 keys 10 / 34, 197 of 48 of 777 10 / 12, 512 of 16 of 2048 17 / 24; not 128 of 16 of 4096, 16 / 9,
// nor 48 of 8 of 4096, 7 / 6); 8 wavefronts where those are few as well (8192 rows of one slab of 16K: 4 / 8 wavefronts 150 / 102, 828
// of 12 of 338 15 / 10; not 512 of 16 of 2048, 17 / 19).
constexpr int NARROW = 256;
hipError_t launch_cache4_weights(const Cache4& c, const CacheQueries& q, const float* lse, const float* weights, float* out, int width,
                                 hipStream_t st) {
    const int slabs = q.B * c.heads, ng = c.groups, tiles = (width + WAVES * TILE - 1) / (WAVES * TILE);
    const int rows = q.Hq / c.heads * q.Nq;
    const bool few = rows <= 16;
    const bool narrow = (long)tiles * slabs < NARROW && rows > 64, eight = (long)tiles * slabs <= NARROW / 4;
    // few rows: as many workgroups as the attention has, so that a wavefront has tiles to walk
    int chunks = few ? WANTED_FEW / slabs : tiles;
    if (chunks < 1) chunks = 1;
    if (chunks > tiles) chunks = tiles;
    const int longest = few ? FEW_CHUNK : WAVES * TILE, even = (tiles + chunks - 1) / chunks * WAVES * TILE, chunk = even < longest ? even : longest;
    const dim3 grid((width + chunk - 1) / chunk, slabs), by_64((width + TILE - 1) / TILE, slabs);
#define SAGE_CACHE4_WEIGHTS(D, NG)                                                                                          \
    do {                                                                                                                     \
        if (rows <= 4) cache4_weights_few_kernel<D, NG, 1><<<grid, WAVES * 64, 0, st>>>(c, q, lse, weights, out, width, chunk);      \
        else if (rows <= 8) cache4_weights_few_kernel<D, NG, 2><<<grid, WAVES * 64, 0, st>>>(c, q, lse, weights, out, width, chunk); \
        else if (few) cache4_weights_few_kernel<D, NG, 4><<<grid, WAVES * 64, 0, st>>>(c, q, lse, weights, out, width, chunk);       \
        else if (narrow && eight) cache4_weights_rows_kernel<D, NG, 8><<<by_64, 8 * 64, 0, st>>>(c, q, lse, weights, out, width); \
        else if (narrow) cache4_weights_rows_kernel<D, NG, 4><<<by_64, 4 * 64, 0, st>>>(c, q, lse, weights, out, width);      \
        else cache4_weights_kernel<D, NG><<<grid, WAVES * 64, 0, st>>>(c, q, lse, weights, out, width);                       \
    } while (0)
    if (c.D == 64 && ng == 1) SAGE_CACHE4_WEIGHTS(64, 1);
    else if (c.D == 64) SAGE_CACHE4_WEIGHTS(64, 2);
    else if (ng == 1) SAGE_CACHE4_WEIGHTS(128, 1);
    else if (ng == 2) SAGE_CACHE4_WEIGHTS(128, 2);
    else SAGE_CACHE4_WEIGHTS(128, 4);
#undef SAGE_CACHE4_WEIGHTS
    return hipGetLastError();
}

}  // namespace sage
