// Linear layers of all learners, forward and backward (gfx950).
//
//     y = act(x W' + b) + residual                                   dz = dy act'(z),  dx = dz W,  dW = dz' x,  db = sum_t dz
//
// All three products are C[m, n] = sum_k P[m, k] Q[n, k] with C's columns next to each other:
//     forward  m token, n output, k input    P = x  [m][k]   Q = W [n][k]
//     dx       m token, n input,  k output   P = dz [m][k]   Q = W [k][n]
//     dW       m output, n input, k token    P = dz [k][m]   Q = x [k][n]
// so an operand comes with k along its rows or down its columns, and one kernel serves them all: it brings either into the same LDS tile,
// rows of 128 bytes of k, and multiplies from there with the matrix instructions of the type (bf16 32x32x16, float 32x32x2, both summing
// in fp32).  2 m n k operations against (m + n) k elements: bound by the matrix cores on batches, by reading W at a few tokens.
//
// Tiles of 256 x 256 (eight wavefronts), 128 x 128, 64 x 64 and for narrow float products 128 x 32 and 32 x 128 (four each) by 128 bytes of k, twice in
// LDS: one is multiplied while the next is put beside it and the one behind is on its way in registers.  Large tiles read least; what then
// keeps the matrix cores from their rate is the operands' way through registers and LDS (without it the same loop multiplies at 1200 to 1380
// TFLOP/s in bf16; waiting for memory is not it: k read again and again from one place is 0 to 5 % faster).  Measured, TFLOP/s forward / dx / dW: bf16
// 8192^3 1091 / 1157 / 1155 (a library's product of that size here: 1517 / 1384 / 1192), 4096^3 1143 / 1111 / 1089, 4 x 2048 x 2048 -> 8192
// 1052 / 1118 / 1031, 4096 x 1024 -> 32 000 929 / 822 / 1016; float 4096^3 140 / 141 / 139 (154).  The epilogue of large tiles has the chip to itself, one
// workgroup to a compute unit: bias, GELU and a second array of 134 MB are 42 of 303 us for 4 x 2048 x 2048 -> 8192.
#include "psgd_rows.h"

#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

namespace psgd {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

struct Operand {          // element (row, col) of learner i at p + i * learner + row * pitch + col
    const char* p;
    int64_t learner, pitch;
};

constexpr float kLog2E = 1.44269504088896341f;

// The activations z Phi(z) and z / (1 + exp(-z)) and their slopes, each as exact as its outputs' type can hold, however far z is from zero.  Phi by fitted
// polynomials: with a = |z|, t = 1 / (1 + a / 4),
//     Phi(-a) = exp(-a^2 / 2) t (c1 + t (c2 + ...)),      Phi(z) = 1/2 + z (d0 + d1 z^2 + ...).
// bf16: the first alone, seven terms, fitted to 1e-7 and to 2e-5 of itself on a <= 14.5 (beyond, the exponential is zero in float), with the hardware's
// exponential and reciprocal: 2e-7 in float arithmetic, which is what an output whose residual cancels z Phi(z) shows, and a hundredth of what rounding
// costs any other.  (Five terms, off by 4e-5 of itself, are no faster: 4 x 2048 x 2048 -> 8192 292.5 / 291.7 us.)
// Float: the first with eight terms from 1.25 on, below it the second with six, both off by 1e-8 of themselves; with their roundings Phi is off by at most
// 12 units of 2^-24 of itself up to a = 3, and by a^2 / 2 more beyond, for the square's.  No branches: erfcf, the same to a few units, has them.  us, by
// an approximation of erf (whose error stays while Phi falls) / erfcf / this: 3 x 257 x 1000 -> 771 backward 42.1 / 45.8 / 43.3, 4096 x 1024 -> 4096
// forward 260 / 269 / 265, 4 x 64 x 512 -> 2048 15.2 / - / 15.9.  SiLU by the exact exponential and quotient, the hardware's before: the first 41.4 / 42.7,
// the last 14.8 / 15.5.
template <typename T> __device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(T) == 4) return expf(x);
    else return __builtin_amdgcn_exp2f(x * kLog2E);
}
template <typename T> __device__ __forceinline__ float bell_of(float z) {       // exp(-z^2 / 2)
    if constexpr (sizeof(T) == 4) return expf(-0.5f * z * z);
    else return __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E));
}
template <int N> __device__ __forceinline__ float polynomial(float x, const float (&c)[N]) {
    float p = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) p = __builtin_fmaf(p, x, c[i]);
    return p;
}
// Phi(-|z|); float: |z| from 1.25 on.
template <typename T> __device__ __forceinline__ float tail_of(float z, float bell) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, __builtin_fabsf(z), 1.0f));
    if constexpr (sizeof(T) == 4)
        return t * polynomial(t, {0.0997423306f, 0.0995698348f, 0.0952199996f, 0.0711945444f, 0.0975557044f, -0.0292390473f, 0.114079773f,
                                  -0.0481649525f}) * bell;
    else
        return t * polynomial(t, {0.0990288705f, 0.109893471f, 0.0344877355f, 0.260672182f, -0.243641973f, 0.327903092f, -0.0883433446f}) * bell;
}
template <typename T> __device__ __forceinline__ float normal_cdf(float z, float bell) {
    const float tail = tail_of<T>(z, bell), far = z < 0.0f ? tail : 1.0f - tail;
    if constexpr (sizeof(T) == 2) return far;
    const float slope = polynomial(z * z, {0.398942262f, -0.0664902106f, 0.00997228269f, -0.00118383719f, 0.000111041125f, -6.80949188e-06f});
    const float near = __builtin_fmaf(z, slope, 0.5f);
    return __builtin_fabsf(z) < 1.25f ? near : far;
}
template <int ACT, typename T> __device__ __forceinline__ float act_of(float z) {
    if (ACT == PSGD_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == PSGD_ACT_GELU) {
        if constexpr (sizeof(T) == 4) return z * normal_cdf<T>(z, bell_of<T>(z));
        // max(z, 0) - |z| Phi(-|z|); the least value keeps +inf times 0 out
        else return __builtin_fmaf(-__builtin_fabsf(fminf(z, 1e30f)), tail_of<T>(z, bell_of<T>(z)), fmaxf(z, 0.0f));
    }
    if (ACT == PSGD_ACT_SILU) {
        const float d = 1.0f + exp_of<T>(-z);
        return sizeof(T) == 4 ? z / d : z * __builtin_amdgcn_rcpf(d);
    }
    return z;
}
template <int ACT, typename T> __device__ __forceinline__ float slope_of(float z) {
    if (ACT == PSGD_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == PSGD_ACT_GELU) {
        const float bell = bell_of<T>(z);
        return normal_cdf<T>(z, bell) + z * bell * 0.39894228040143268f;
    }
    if (ACT == PSGD_ACT_SILU) {
        const float d = 1.0f + exp_of<T>(-z), p = sizeof(T) == 4 ? 1.0f / d : __builtin_amdgcn_rcpf(d);
        return p * (1.0f + z * (1.0f - p));
    }
    return 1.0f;
}

// ------------------------------------------------------------------------------------------------ the product
// What follows the sum over k: y = act(z) + residual, z = sum + bias.
struct Epilogue {
    Operand y, z, residual, bias;
    int act;
};
struct GemmArgs {
    Operand p, q;
    Epilogue out;
    float* partial;         // split > 1: [split][learners][m][n] sums of parts of k, without an epilogue
    int64_t m, n, k;
    int learners, split;
    int tiles_m, tiles_n;
};

template <typename T> constexpr int kDepth = kRowBytes / (int)sizeof(T);

// Where chunk c of row r lies.  LDS serves 16 lanes of a 16-byte access at a time, from 64 banks: two rows.  Lanes that read one chunk of 16 rows
// next to each other, that write the eight chunks of two rows, or four chunks of four rows eight or four apart (turned blocks) find them in
// 16 different places.  (Chunk c at place c ^ (r & 7), which serves eight lanes at a time: twice the time for each read.)  Rows 32 apart differ
// by a constant.
__device__ __forceinline__ int tile_place(int r, int c) {
    const int pair = r >> 1, half = (r ^ (pair >> 1) ^ (pair >> 2)) & 1;
    return pair * (2 * kRowBytes) + half * kRowBytes + (((c ^ pair ^ (r >> 2 & 4)) & 7) << 4);
}

// What is left of an output's 16 bytes of columns after the sum over k.
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& a, int64_t learner, int64_t m, int64_t n, int64_t left, const float (&bias)[kPer<T>],
                                       float (&v)[kPer<T>]) {
    constexpr int E = kPer<T>;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += bias[e];
    if (a.z.p) store_cols<T>(reinterpret_cast<T*>(const_cast<char*>(a.z.p)) + learner * a.z.learner + m * a.z.pitch + n, v, left);
    if (a.act == PSGD_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = act_of<PSGD_ACT_RELU, T>(v[e]);
    } else if (a.act == PSGD_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = act_of<PSGD_ACT_GELU, T>(v[e]);
    } else if (a.act == PSGD_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = act_of<PSGD_ACT_SILU, T>(v[e]);
    }
    if (a.residual.p) {
        float r[E];
        widen<T>(load_cols(reinterpret_cast<const T*>(a.residual.p) + learner * a.residual.learner + m * a.residual.pitch + n, left), r);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += r[e];
    }
    store_cols<T>(reinterpret_cast<T*>(const_cast<char*>(a.y.p)) + learner * a.y.learner + m * a.y.pitch + n, v, left);
}

// Up to four words of elements, any alignment.
typedef uint32_t u32_any __attribute__((aligned(2)));
template <int WORDS, typename T> __device__ __forceinline__ u32x4 load_words(const T* p) {
    if constexpr (WORDS == 4) {
        return load_raw(p);
    } else if constexpr (WORDS == 2) {
        const u32x2 r = *reinterpret_cast<const u32x2_any*>(p);
        return (u32x4){r.x, r.y, 0u, 0u};
    } else {
        return (u32x4){*reinterpret_cast<const u32_any*>(p), 0u, 0u, 0u};
    }
}
// The same element by element, none beyond p[last]: the ones behind it repeat it.  No branches: loads that wait for one another would cost more.
template <int WORDS> __device__ __forceinline__ u32x4 load_words_to(const float* p, int last) {
    u32x4 v = {};
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v[i] = __float_as_uint(p[i < last ? i : last]);
    return v;
}
template <int WORDS> __device__ __forceinline__ u32x4 load_words_to(const uint16_t* p, int last) {
    u32x4 v = {};
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v[i] = (uint32_t)p[2 * i < last ? 2 * i : last] | (uint32_t)p[2 * i + 1 < last ? 2 * i + 1 : last] << 16;
    return v;
}
// A chunk from its element `by` on, zeros behind.
template <typename T> __device__ __forceinline__ u32x4 chunk_from(u32x4 v, int by) {
    const int words = by * (int)sizeof(T) / 4;
    if (words & 1) v = (u32x4){v.y, v.z, v.w, 0u};
    if (words & 2) v = (u32x4){v.z, v.w, 0u, 0u};
    if (words & 4) v = (u32x4){};
    if (sizeof(T) == 2 && by % 2) v = (u32x4){v.x >> 16 | v.y << 16, v.y >> 16 | v.z << 16, v.z >> 16 | v.w << 16, v.w >> 16};
    return v;
}
// `left` < kPer<T> elements of a row that has no more, one after the other, zeros behind.
template <typename T> __device__ __forceinline__ u32x4 chunk_of_few(const T* p, int left) {
    u32x4 v = {};
#pragma unroll 1
    for (int e = 0; e < left; ++e) {
        const uint32_t x = sizeof(T) == 4 ? __float_as_uint(load_1(p + e)) : __float_as_uint(load_1(p + e)) >> 16 << e % 2 * 16;
        const int word = e * (int)sizeof(T) / 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] |= i == word ? x : 0u;
    }
    return v;
}

// One operand's way into LDS: ROWS rows by a tile's depth of k, through the registers of LANES lanes (half of the workgroup; the other half brings
// the other operand).  ALONG: memory has k along its rows; then a lane brings chunks.  Otherwise memory's rows are k: a lane brings blocks of E
// values of k (E elements to 16 bytes) by WIDE rows of the tile, and turns them.  Rows of the tile beyond the operand's last are not stored by
// anyone, so they may hold anything: chunks of the last row again, or what LDS held before.  A block that would reach beyond the last row
// is one that ends there.
//
// Where a chunk or block starts is one 32-bit offset a lane behind an address that is the same for all lanes, and its place in LDS one exclusive or:
// the products leave little time for anything else on the vector unit, and the float ones run on its own multipliers.  (64-bit addresses a lane,
// computed where they were used, 24 instructions a load: bf16 8192^3 929 TFLOP/s forward and 1030 for dx and dW, now 1071 and 1100; float 4096^3
// 125 to 131, now 136 to 139; float tiles of 64, 100.)
template <typename T, int ROWS, int LANES> struct Bring {
    static constexpr int E = kPer<T>, COUNT = ROWS * kRowBytes / 16 / LANES, LINES = LANES / 8;      // chunks a lane brings; rows or blocks side by side
    static constexpr int WIDE = COUNT < E ? COUNT : E, BLOCKS = COUNT / WIDE, WORDS = WIDE * (int)sizeof(T) / 4;
    static_assert(COUNT > 0 && WORDS > 0 && COUNT % WIDE == 0 && BLOCKS <= 2, "whole chunks and blocks a lane");

    const T* base;             // of the tile's first row, or column
    int64_t pitch;
    int line, c;               // the lane's first chunk or block, and its chunk of k
    int rows;                  // of the operand from the tile's first on, at most INT_MAX / 2
    int few;                   // rows of an operand that has fewer than a block, else 0
    int last;                  // ALONG: the last LINES rows of which there is one, and
    uint32_t off[2];           // where the lane's chunk is in LINES rows, and in the last ones; else where its blocks are, and WIDE behind
    int place;                 // of the first chunk in the tile
    bool cut;                  // a block ends with the operand's last row instead of beginning at a multiple of WIDE

    template <bool ALONG> __device__ __forceinline__ void start(const T* p, int64_t pitch_, int64_t row0, int64_t all) {
        const int tid = threadIdx.x % LANES;
        if (ALONG) {
            line = tid / 8;
            c = tid % 8;
        } else {      // four lanes side by side along memory's rows: lanes that jump from row to row are served one a cycle
            const int w = tid / kWave;
            line = tid % 4 + tid / 16 % 4 * 4 + w % (LANES / 128) * 16;
            c = tid / 4 % 4 + w / (LANES / 128) * 4;
        }
        pitch = pitch_;
        rows = (int)(all - row0 < (1 << 30) ? all - row0 : (1 << 30));
        few = !ALONG && all < WIDE ? (int)all : 0;
        base = ALONG ? p + row0 * pitch : p + row0;
        const int size = (int)sizeof(T);
        if (ALONG) {
            last = (rows < ROWS ? rows - 1 : ROWS - 1) / LINES;
            const int end = rows - 1 - last * LINES;
            off[0] = (uint32_t)line * (uint32_t)pitch * size + c * 16;
            off[1] = (uint32_t)(line < end ? line : end) * (uint32_t)pitch * size + c * 16;
            place = tile_place(line, c);
        } else {
            cut = rows < ROWS && rows % WIDE;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = k < BLOCKS ? k : 0;
                off[k] = (uint32_t)(c * E) * (uint32_t)pitch * size + (uint32_t)(row_of<false>(j) + WIDE) * size;
            }
            place = tile_place(line * WIDE, c);
        }
    }
    // Rows so long that 32-bit offsets of a tile could end are brought by fetch_upto alone.
    static __device__ __forceinline__ bool too_long(int64_t pitch) { return pitch > 1 << 24; }
    // The row of chunk or block j.
    template <bool ALONG> __device__ __forceinline__ int row_of(int j) const {
        const int r = ALONG ? line + j * LINES : (line + j * LINES) * WIDE;
        return ALONG || few || r + WIDE <= rows ? r : rows - WIDE;
    }
    template <bool ALONG> __device__ __forceinline__ const T* from(int j) const {
        if (ALONG) {
            const int r = row_of<ALONG>(j);
            return base + (r < rows ? r : rows - 1) * pitch + c * E;
        }
        return base + c * E * pitch + (few ? 0 : row_of<ALONG>(j));
    }
    // The whole depth from k0 is there.  Chunks, or lines, first to end - 1.
    static constexpr int loads(bool along) { return along ? COUNT : BLOCKS * E; }
    template <bool ALONG> __device__ __forceinline__ void fetch(u32x4 (&raw)[COUNT], int64_t k0, int first = 0, int end = loads(ALONG)) {
        asm volatile("" : "+v"(off[0]), "+v"(off[1]));      // no sums with them, and no choice between them, are made outside of the loop
#pragma unroll
        for (int l = first; l < end; ++l) {
            if constexpr (ALONG) {
                const char* at = reinterpret_cast<const char*>(base + (int64_t)((l < last ? l : last) * LINES) * pitch + k0);
                raw[l] = load_raw(reinterpret_cast<const T*>(at + (l < last ? off[0] : off[1])));
            } else {
                const char* at = reinterpret_cast<const char*>(base + (k0 + l % E) * pitch - WIDE);
                keep(raw, l, load_words<WORDS>(reinterpret_cast<const T*>(at + off[l / E])));
            }
            __builtin_amdgcn_sched_barrier(0);      // one address at a time
        }
    }
    // Only k < end is there, the rest counts as zero; or the operand has fewer rows than a block.
    template <bool ALONG> __device__ __forceinline__ void fetch_upto(u32x4 (&raw)[COUNT], int64_t k0, int64_t end) {
        const int left = (int)(end - k0) - c * E;       // of the lane's E values of k
#pragma unroll
        for (int s = 0; s < (ALONG ? COUNT : BLOCKS); ++s) {
            const T* p = from<ALONG>(s);
            if constexpr (ALONG) {
                if (end < E) {
                    raw[s] = chunk_of_few(p + k0, left);
                } else {                                                      // the row's last whole chunk, moved up
                    const int by = left >= E ? 0 : left <= 0 ? E : E - left;
                    raw[s] = chunk_from<T>(load_raw(p + k0 - (left >= E ? 0 : E - left)), by);
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const T* q = p + (k0 + (j < left ? j : left - 1)) * pitch;      // the last line again, possibly of another chunk
                    const u32x4 v = few ? load_words_to<WORDS>(q, few - 1) : load_words<WORDS>(q);
                    keep(raw, s * E + j, j < left ? v : (u32x4){});
                }
            }
        }
    }
    // Lines of WORDS words, one after the other in the registers.
    static __device__ __forceinline__ void keep(u32x4 (&raw)[COUNT], int n, u32x4 v) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) raw[(n * WORDS + w) / 4][(n * WORDS + w) % 4] = v[w];
    }
    static __device__ __forceinline__ uint32_t word(const u32x4 (&raw)[COUNT], int n, int w) { return raw[(n * WORDS + w) / 4][(n * WORDS + w) % 4]; }

    // tile_place is made of exclusive ors of the bits of r and c: the place of r ^ e is that of r, exclusive or that of e.
    template <bool ALONG> __device__ __forceinline__ void put(const u32x4 (&raw)[COUNT], char* tile, int first = 0, int end = COUNT) {
        asm volatile("" : "+v"(place), "+v"(line));      // places are made where they are used: kept, they would cost registers that the products need
        if constexpr (ALONG) {
#pragma unroll
            for (int n = first; n < end; ++n) *reinterpret_cast<u32x4*>(tile + (place ^ tile_place(n * LINES, 0))) = raw[n];
        } else if (!cut && !few) {
#pragma unroll
            for (int n = first; n < end; ++n) {
                *reinterpret_cast<u32x4*>(tile + (place ^ tile_place(n / WIDE * LINES * WIDE + n % WIDE, 0))) = turned(raw, n);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {      // a block that ends with the operand's last row may begin before the tile's first: to rows that are beyond the last
#pragma unroll
            for (int n = first; n < end; ++n) {
                *reinterpret_cast<u32x4*>(tile + tile_place(((few ? 0 : row_of<false>(n / WIDE)) + n % WIDE) & (ROWS - 1), c)) = turned(raw, n);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    // Row n of the lane's blocks.
    static __device__ __forceinline__ u32x4 turned(const u32x4 (&raw)[COUNT], int n) {
        const int s = n / WIDE, e = n % WIDE;
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if constexpr (sizeof(T) == 4)
                v[j] = word(raw, s * 4 + j, e);
            else      // the upper or lower halves of two words
                v[j] = __builtin_amdgcn_perm(word(raw, s * 8 + 2 * j + 1, e / 2), word(raw, s * 8 + 2 * j, e / 2), e % 2 ? 0x07060302u : 0x05040100u);
        return v;
    }
    // Slot `slot` of `slots` in a tile's products: this lane's part of putting the next tile, which is in `raw`, into LDS, and of sending for the
    // one behind it, so that what is sent for travels for the time of a tile.  Chunks go one after the other, spread over the tile (2 % faster than
    // all at once); blocks are turned, which takes all of their lines, so they go together (in quarters: 4 % slower).
    template <bool ALONG> __device__ __forceinline__ void turn_over(u32x4 (&raw)[COUNT], char* tile, bool more, int64_t k0, int slot, int slots) {
        if constexpr (ALONG) {
            const int first = slot * COUNT / slots, end = (slot + 1) * COUNT / slots;
            put<true>(raw, tile, first, end);
            if (more) fetch<true>(raw, k0, first, end);
        } else if (slot == slots / 3) {
            put<false>(raw, tile);
            if (more) fetch<false>(raw, k0);
        }
    }
};

// A wavefront's part of bringing a tile of k: one operand of a square tile (half of the wavefronts bring the other), or its share of both.
template <bool ALONG, typename Bring> struct BringOne {
    Bring& b;
    u32x4 (&raw)[Bring::COUNT];
    char* at;
    __device__ __forceinline__ void fetch(int64_t k0) { b.template fetch<ALONG>(raw, k0); }
    __device__ __forceinline__ void fetch_upto(int64_t k0, int64_t end) { b.template fetch_upto<ALONG>(raw, k0, end); }
    __device__ __forceinline__ void put(int side) { b.template put<ALONG>(raw, at + side); }
    __device__ __forceinline__ void turn_over(int side, bool more, int64_t k0, int slot, int slots) {
        b.template turn_over<ALONG>(raw, at + side, more, k0, slot, slots);
    }
};
template <typename One, typename Other> struct BringBoth {
    One& p;
    Other& q;
    __device__ __forceinline__ void fetch(int64_t k0) { p.fetch(k0), q.fetch(k0); }
    __device__ __forceinline__ void fetch_upto(int64_t k0, int64_t end) { p.fetch_upto(k0, end), q.fetch_upto(k0, end); }
    __device__ __forceinline__ void put(int side) { p.put(side), q.put(side); }
    __device__ __forceinline__ void turn_over(int side, bool more, int64_t k0, int slot, int slots) {
        p.turn_over(side, more, k0, slot, slots);
        q.turn_over(side, more, k0, slot, slots);
    }
};

__device__ __forceinline__ void multiply(u32x4 a, u32x4 b, f32x16& c, uint16_t) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Sixteen bytes of a lane are four values of k; the halves of the wavefront hold different ones, so instruction j sums two values of k.
__device__ __forceinline__ void multiply(u32x4 a, u32x4 b, f32x16& c, float) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
}

// The tile that workgroup `id` of `total` takes.  Consecutive workgroups go to the eight dies in turn; this gives each die a contiguous stretch
// of tiles, and walks eight tiles of m for each of n, so that the tiles a die works on at a time share operands in its L2.
struct Tile {
    int learner, part, tm, tn;
};
__device__ __forceinline__ Tile tile_of(const GemmArgs& a, uint32_t id, uint32_t total) {
    const uint32_t q = total / 8, r = total % 8, die = id % 8;
    uint32_t t = die * q + (die < r ? die : r) + id / 8;
    const uint32_t each = (uint32_t)a.tiles_m * a.tiles_n;
    Tile o;
    o.part = (int)(t / each) % a.split;
    o.learner = (int)(t / each) / a.split;
    t %= each;
    const uint32_t band = 8u * a.tiles_n, first = t / band * 8, high = min(8u, (uint32_t)a.tiles_m - first);
    t %= band;
    o.tm = (int)(first + t % high);
    o.tn = (int)(t / high);
    return o;
}

extern __shared__ __attribute__((aligned(128))) char lds[];

// The wavefronts of a workgroup, along m and along n.
template <int BM, int BN> struct TileShape {
    static constexpr int ACROSS_M = BM > BN ? 4 : BM < BN ? 1 : 2, ACROSS_N = BM > BN ? 1 : BM < BN || BM == 256 ? 4 : 2;
    static constexpr int LANES = kWave * ACROSS_M * ACROSS_N;
};

// Workgroup `id` of `total` that this product has.
template <typename T, int BM, int BN, bool P_ALONG, bool Q_ALONG>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, uint32_t id, uint32_t total) {
    using Shape = TileShape<BM, BN>;
    constexpr int NT = Shape::LANES, ACROSS_M = Shape::ACROSS_M, WM = BM / ACROSS_M, WN = BN / Shape::ACROSS_N, TM = WM / 32, TN = WN / 32, BK = kDepth<T>;
    constexpr int kP = BM * kRowBytes, kBoth = (BM + BN) * kRowBytes;
    const Tile t = tile_of(a, id, total);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const T* p = reinterpret_cast<const T*>(a.p.p) + t.learner * a.p.learner;
    const T* q = reinterpret_cast<const T*>(a.q.p) + t.learner * a.q.learner;
    const int64_t m0 = (int64_t)t.tm * BM, n0 = (int64_t)t.tn * BN;
    // this part's stretch of k, in whole tiles
    const int64_t tiles = (a.k + BK - 1) / BK;
    const int from = (int)(tiles * t.part / a.split), to = (int)(tiles * (t.part + 1) / a.split);
    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = (f32x16){};
    // which operand the wavefront brings, if one
    constexpr bool SQUARE = BM == BN;
    const bool first = __builtin_amdgcn_readfirstlane(threadIdx.x) < NT / 2;
    using BringP = Bring<T, BM, SQUARE ? NT / 2 : NT>;
    using BringQ = Bring<T, BN, SQUARE ? NT / 2 : NT>;
    const bool slow = (!P_ALONG && a.m < BringP::WIDE) || (!Q_ALONG && a.n < BringQ::WIDE) ||      // the same for the whole workgroup
                      BringP::too_long(a.p.pitch) || BringQ::too_long(a.q.pitch);
    const int mw = wave % ACROSS_M * WM + lane % 32, nw = wave / ACROSS_M * WN + lane % 32;
    // The chunks of one step of 16 bytes of k, and its products.
    struct Step {
        u32x4 p[TM], q[TN];
    };
    int at_p = tile_place(mw, lane / 32), at_q = kP + tile_place(nw, lane / 32);      // step s: place ^ (s << 5)
    auto read = [&](const char* now, int s, Step& f) {
        asm volatile("" : "+v"(at_p), "+v"(at_q));      // one register each, not one a step
#pragma unroll
        for (int j = 0; j < TM; ++j) f.p[j] = *reinterpret_cast<const u32x4*>(now + (at_p ^ (s << 5)) + 32 * j * kRowBytes);
#pragma unroll
        for (int i = 0; i < TN; ++i) f.q[i] = *reinterpret_cast<const u32x4*>(now + (at_q ^ (s << 5)) + 32 * i * kRowBytes);
    };
    // A tile of k: each step's chunks are read while the one before is multiplied, and the next tile is brought in during the first three steps
    // (turn_over).  The workgroup meets before the last step, so that the next tile's first chunks are read during it: met after it, the matrix
    // cores would wait for them.  The fences keep the compiler from sinking loads to their uses.
    Step f[2];
    auto multiply_tile = [&](const char* now, auto more, const char* next, auto meanwhile) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) {
                read(now, s + 1, f[(s + 1) % 2]);
            } else if constexpr (decltype(more)::value) {
                __syncthreads();
                read(next, 0, f[0]);
            }
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if (s < 3) meanwhile(s * TN + i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < TM; ++j) multiply(f[s % 2].q[i], f[s % 2].p[j], acc[i][j], T{});
            }
        }
    };
    // Tiles of k that are there to their end, then what is cut off.
    auto walk = [&](auto& bring) {
        const int last = (int)(a.k / BK), whole = slow ? from : to < last ? to : last;
        int tile = from;
        if (tile < whole) {
            bring.fetch((int64_t)tile * BK);
            bring.put(0);
            if (tile + 1 < whole) bring.fetch((int64_t)(tile + 1) * BK);
            __syncthreads();
            read(lds, 0, f[0]);
            int side = 0;
            for (; tile + 2 < whole; ++tile) {
                multiply_tile(lds + side, std::true_type{}, lds + (kBoth - side), [&](int slot) { bring.turn_over(kBoth - side, true, (int64_t)(tile + 2) * BK, slot, 3 * TN); });
                side = kBoth - side;
            }
            if (tile + 1 < whole) {
                multiply_tile(lds + side, std::true_type{}, lds + (kBoth - side), [&](int slot) { bring.turn_over(kBoth - side, false, 0, slot, 3 * TN); });
                side = kBoth - side;
                ++tile;
            }
            multiply_tile(lds + side, std::false_type{}, nullptr, [](int) {});
            ++tile;
            __syncthreads();
        }
        for (; tile < to; ++tile) {
            bring.fetch_upto((int64_t)tile * BK, a.k);
            bring.put(0);
            __syncthreads();
            const int64_t left = a.k - (int64_t)tile * BK;      // no products of the zeros behind it
            const int steps = left < BK ? (int)((left * (int)sizeof(T) + 31) / 32) : 4;
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                read(lds, s, f[0]);
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j) multiply(f[0].q[i], f[0].p[j], acc[i][j], T{});
            }
            __syncthreads();
        }
    };
    if constexpr (SQUARE) {      // the same loop for both halves of the workgroup, each with its operand's way
        BringP bring;
        u32x4 raw[BringP::COUNT];
        char* const at = first ? lds : lds + kP;
        if (first) bring.template start<P_ALONG>(p, a.p.pitch, m0, a.m);
        else bring.template start<Q_ALONG>(q, a.q.pitch, n0, a.n);
        BringOne<P_ALONG, BringP> one{bring, raw, at};
        BringOne<Q_ALONG, BringP> other{bring, raw, at};
        if (P_ALONG == Q_ALONG || first) walk(one);
        else walk(other);
    } else {
        BringP bring_p;
        BringQ bring_q;
        u32x4 raw_p[BringP::COUNT], raw_q[BringQ::COUNT];
        bring_p.template start<P_ALONG>(p, a.p.pitch, m0, a.m);
        bring_q.template start<Q_ALONG>(q, a.q.pitch, n0, a.n);
        BringOne<P_ALONG, BringP> one{bring_p, raw_p, lds};
        BringOne<Q_ALONG, BringQ> other{bring_q, raw_q, lds + kP};
        BringBoth<decltype(one), decltype(other)> both{one, other};
        walk(both);
    }
    // Lane l holds column l % 32 of m and, of each 32 of n, four stretches of four: 8 g + 4 (l / 32) .. + 3.  Through LDS, 32 rows of m at a time, so that
    // C's rows are read and written side by side.
    constexpr int E = kPer<T>, PITCH = WN + 4, ACROSS = WN / E;          // a lane takes 16 bytes of C's columns: 64 / ACROSS rows at a time
    float* mine = reinterpret_cast<float*>(lds) + wave * 32 * PITCH;
    const int64_t n = n0 + wave / ACROSS_M * WN + lane % ACROSS * E, left = a.n - n;
    float bias[E] = {};
    if (a.out.bias.p && left > 0 && !a.partial)
        widen<T>(load_cols(reinterpret_cast<const T*>(a.out.bias.p) + t.learner * a.out.bias.learner + n, left), bias);
#pragma unroll
    for (int j = 0; j < TM; ++j) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(mine + lane % 32 * PITCH + 32 * i + 8 * g + lane / 32 * 4) =
                    (f32x4){acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // each wavefront has a place of its own
        if (left > 0) {
#pragma unroll 2
            for (int r = lane / ACROSS; r < 32; r += kWave / ACROSS) {
                const int64_t m = m0 + wave % ACROSS_M * WM + 32 * j + r;
                float v[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f32x4 sum = *reinterpret_cast<const f32x4*>(mine + r * PITCH + lane % ACROSS * E + e);
                    v[e] = sum.x, v[e + 1] = sum.y, v[e + 2] = sum.z, v[e + 3] = sum.w;
                }
                if (m >= a.m) break;
                if (a.partial) {
                    float* to = a.partial + (((int64_t)t.part * a.learners + t.learner) * a.m + m) * a.n + n;
#pragma unroll
                    for (int e = 0; e < E; e += 4) {
                        const float w[4] = {v[e], v[e + 1], v[e + 2], v[e + 3]};
                        store_cols<float>(to + e, w, left - e);
                    }
                } else {
                    finish<T>(a.out, t.learner, m, n, left, bias, v);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <typename T, int BM, int BN, bool P_ALONG, bool Q_ALONG>
__global__ __launch_bounds__((TileShape<BM, BN>::LANES)) void gemm_kernel(GemmArgs a) {
    gemm_tile<T, BM, BN, P_ALONG, Q_ALONG>(a, blockIdx.x, gridDim.x);
}
// The backward pass' two products side by side, dx's workgroups first: neither fills the chip then, and a workgroup alone on its compute unit waits for
// most of its time.  Float, 3 x 257 x 1000 -> 771: 38 us for both, one after the other 22 each.
template <typename T, int TILE> __global__ __launch_bounds__(256) void gemm_pair_kernel(GemmArgs dx, GemmArgs dw, uint32_t first) {
    if (blockIdx.x < first) gemm_tile<T, TILE, TILE, true, false>(dx, blockIdx.x, first);
    else gemm_tile<T, TILE, TILE, false, false>(dw, blockIdx.x - first, gridDim.x - first);
}

// ------------------------------------------------------------------------------------------------ a few tokens
// The forward product of up to TOK tokens: W is read once, 1 KB of one row at a time, which is all it costs; the tokens come from the first-level
// cache.  A wavefront takes R rows of W (outputs) and keeps R x TOK sums a lane, joined at the end.  Bound by HBM: eight learners' bf16 4096 x 4096 for
// one token 47 us, 268 MB at 5.7 TB/s.
struct FewArgs {
    Operand x, w;
    Epilogue out;
    int64_t t, k, n;
};
template <typename T, int TOK, int R> __global__ __launch_bounds__(256) void few_tokens_kernel(FewArgs a) {
    constexpr int E = kPer<T>, U = R == 1 ? 4 : 2;
    const int lane = threadIdx.x % kWave;
    const int64_t i = blockIdx.y, row0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * R;
    if (row0 >= a.n) return;
    const T* w[R];
    const T* x[TOK];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = reinterpret_cast<const T*>(a.w.p) + i * a.w.learner + (row0 + r < a.n ? row0 + r : a.n - 1) * a.w.pitch;
#pragma unroll
    for (int t = 0; t < TOK; ++t) x[t] = reinterpret_cast<const T*>(a.x.p) + i * a.x.learner + (t < a.t ? t : a.t - 1) * a.x.pitch;
    float acc[R][TOK];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < TOK; ++t) acc[r][t] = 0.0f;
    auto add = [&](const u32x4 (&rw)[R], const u32x4 (&rx)[TOK]) {
        float v[R][E];
#pragma unroll
        for (int r = 0; r < R; ++r) widen<T>(rw[r], v[r]);
#pragma unroll
        for (int t = 0; t < TOK; ++t) {
            float u[E];
            widen<T>(rx[t], u);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][t] = __builtin_fmaf(v[r][e], u[e], acc[r][t]);
        }
    };
    const int64_t whole = a.k / E;
    int64_t g = lane;
    for (; g - lane + U * kWave <= whole; g += U * kWave) {
        u32x4 rw[U][R], rx[TOK];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) rw[u][r] = load_raw(w[r] + (g + u * kWave) * E);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int t = 0; t < TOK; ++t) rx[t] = load_raw(x[t] + (g + u * kWave) * E);
            add(rw[u], rx);
        }
    }
    for (; g * E < a.k; g += kWave) {
        u32x4 rw[R], rx[TOK];
#pragma unroll
        for (int r = 0; r < R; ++r) rw[r] = load_cols(w[r] + g * E, a.k - g * E);
#pragma unroll
        for (int t = 0; t < TOK; ++t) rx[t] = load_cols(x[t] + g * E, a.k - g * E);
        add(rw, rx);
    }
    // lane r * TOK + t finishes output r of token t
    float v = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < TOK; ++t) {
            const float sum = wave_all<Sum>(acc[r][t]);
            v = lane == r * TOK + t ? sum : v;
        }
    const int64_t t = lane % TOK, n = row0 + lane / TOK;
    if (lane >= R * TOK || t >= a.t || n >= a.n) return;
    const Epilogue& o = a.out;
    if (o.bias.p) v += load_1(reinterpret_cast<const T*>(o.bias.p) + i * o.bias.learner + n);
    if (o.z.p) store_1(reinterpret_cast<T*>(const_cast<char*>(o.z.p)) + i * o.z.learner + t * o.z.pitch + n, v);
    v = o.act == PSGD_ACT_RELU   ? act_of<PSGD_ACT_RELU, T>(v)
        : o.act == PSGD_ACT_GELU ? act_of<PSGD_ACT_GELU, T>(v)
        : o.act == PSGD_ACT_SILU ? act_of<PSGD_ACT_SILU, T>(v)
                                 : v;
    if (o.residual.p) v += load_1(reinterpret_cast<const T*>(o.residual.p) + i * o.residual.learner + t * o.residual.pitch + n);
    store_1(reinterpret_cast<T*>(const_cast<char*>(o.y.p)) + i * o.y.learner + t * o.y.pitch + n, v);
}

// dW = dz' x of up to TOK tokens: little more than writing dW, which is done in rows.  A lane keeps 16 bytes of columns of x; a wavefront takes up to 64
// rows (outputs), whose dz it reads at once, a row a lane.  Bound by HBM: 4 float tokens of eight learners, 6400 x 4096, 155 us, 839 MB at 5.4 TB/s.
// (dx of so few tokens is left to the tiles: 1 to 8 tokens of eight learners, 4096 x 4096, 44 us in bf16, W at 6.1 TB/s, and 98 to 102 in float, 5.3 to 5.5;
// of one learner 13 and 20.  W read in rows, with its sums beside it, was slower at every size but one, 8 to 200 % at four tokens.)
struct FewGradArgs {
    Operand dz, x, dw;
    int64_t t, in, out;
    int rows;                      // of dW to a wavefront, at most 64
};
template <typename T, int TOK> __global__ __launch_bounds__(256) void few_tokens_grad_kernel(FewGradArgs a) {
    constexpr int E = kPer<T>;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t i = blockIdx.z, col0 = (int64_t)blockIdx.x * kWave * E, col = col0 + lane * E, left = a.in - col;
    const int64_t first = ((int64_t)blockIdx.y * 4 + wave) * a.rows;
    if (first >= a.out) return;
    const int count = (int)(a.out - first < a.rows ? a.out - first : a.rows);
    const T* dz = reinterpret_cast<const T*>(a.dz.p) + i * a.dz.learner + first;
    T* dw = reinterpret_cast<T*>(const_cast<char*>(a.dw.p)) + i * a.dw.learner + first * a.dw.pitch + col;
    float x[TOK][E] = {}, d[TOK];
#pragma unroll
    for (int t = 0; t < TOK; ++t) {
        d[t] = t < a.t && lane < count ? load_1(dz + t * a.dz.pitch + lane) : 0.0f;
        if (t < a.t && left > 0) widen<T>(load_cols(reinterpret_cast<const T*>(a.x.p) + i * a.x.learner + t * a.x.pitch + col, left), x[t]);
    }
    auto walk = [&](auto inside) {
        for (int r = 0; r < count; ++r) {
            float v[E] = {};
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(d[t]), r));
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = __builtin_fmaf(f, x[t][e], v[e]);
            }
            if (inside) store_cols<T>(dw + r * a.dw.pitch, v, E);
            else if (left > 0) store_cols<T>(dw + r * a.dw.pitch, v, left);
        }
    };
    if (col0 + kWave * E <= a.in) walk(std::true_type{});
    else walk(std::false_type{});
}

// ------------------------------------------------------------------------------------------------ dz and db
struct SlopeArgs {
    Operand dy, z;
    char* dz;              // [n][t][pitch] elements of T, or NULL
    int64_t dz_pitch;
    float* partial;        // [n][slabs][o] column sums, or NULL
    int64_t t, o;
};
// dz = dy act'(z) and its sums down the columns.  In bf16 dz is rounded once, for the matrix instructions take bf16; db sums what was not rounded.  The
// rounding is as large as the one of the outputs: dx and dW are 0.0023 of themselves from the formula's instead of 0.0017 (4 x 2048 x 8192 -> 2048), and
// equal the product of the rounded dz but for 0.05 % of their values.  Kept whole as the sum of two bf16, dz would make both products twice, 540 us more
// on 570 there; without an activation nothing is rounded but the outputs, and float layers have no such choice to make.
// Bound by HBM: 4 x 2048 x 2048 bf16 22 us, 100 MB at 4.6 TB/s.  64 lanes side by side, four rows at a time, a slab of one learner's rows a workgroup.
template <typename T, int ACT> __global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a) {
    constexpr int E = kPer<T>;
    __shared__ float rest[4][kWave * E];
    const int lane = threadIdx.x % kWave, line = threadIdx.x / kWave;
    const int64_t i = blockIdx.z, col = ((int64_t)blockIdx.x * kWave + lane) * E, left = a.o - col;
    const int64_t r0 = a.t * blockIdx.y / gridDim.y, r1 = a.t * (blockIdx.y + 1) / gridDim.y;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    if (left > 0) {
        for (int64_t r = r0 + line; r < r1; r += 4) {
            float v[E];
            widen<T>(load_cols(reinterpret_cast<const T*>(a.dy.p) + i * a.dy.learner + r * a.dy.pitch + col, left), v);
            if (ACT != PSGD_ACT_NONE) {
                float z[E];
                widen<T>(load_cols(reinterpret_cast<const T*>(a.z.p) + i * a.z.learner + r * a.z.pitch + col, left), z);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] *= slope_of<ACT, T>(z[e]);
                store_cols<T>(reinterpret_cast<T*>(a.dz) + (i * a.t + r) * a.dz_pitch + col, v, left);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += v[e];
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int e = 0; e < E; ++e) rest[line][e * kWave + lane] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < kWave * E; c += 256) {
        const int at = c % E * kWave + c / E;
        const int64_t column = (int64_t)blockIdx.x * kWave * E + c;
        if (column < a.o) a.partial[(i * gridDim.y + blockIdx.y) * a.o + column] = (rest[0][at] + rest[1][at]) + (rest[2][at] + rest[3][at]);
    }
}

// Adds the slabs of db up: 64 columns a workgroup the first of them 64 `first`, its sixteen wavefronts every sixteenth slab each.
constexpr int kSumWaves = 16;
template <typename T> __global__ __launch_bounds__(kSumWaves* kWave) void sum_slabs_kernel(const float* partial, int64_t slabs, int64_t o, Operand db, int64_t first) {
    __shared__ float rest[kSumWaves][kWave];
    const int64_t i = blockIdx.y, col = (first + blockIdx.x) * kWave + threadIdx.x % kWave;
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
    float sum = 0.0f;
    if (col < o) {
#pragma unroll 4
        for (int64_t s = w; s < slabs; s += kSumWaves) sum += partial[(i * slabs + s) * o + col];
    }
    rest[w][l] = sum;
    __syncthreads();
    if (w || col >= o) return;
    float v = rest[0][l];
#pragma unroll
    for (int k = 1; k < kSumWaves; ++k) v += rest[k][l];
    store_1(reinterpret_cast<T*>(const_cast<char*>(db.p)) + i * db.learner + col, v);
}

// Adds up `parts` arrays of [learners][rows][cols] floats in order, parts of k, with the product's epilogue.
struct JoinArgs {
    const float* partial;
    int64_t parts, part_stride, learner_stride;
    Epilogue out;
    int64_t rows, cols;
};
template <typename T> __global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
    constexpr int E = kPer<T>;
    const int64_t i = blockIdx.z, across = (a.cols + E - 1) / E, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.rows * across) return;
    const int64_t r = at / across, c = at % across * E, left = a.cols - c;
    const float* p = a.partial + i * a.learner_stride + r * a.cols + c;
    float v[E] = {};
#pragma unroll 4
    for (int64_t s = 0; s < a.parts; ++s) {
        float w[4];
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            widen<float>(load_cols(p + s * a.part_stride + e, left - e), w);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[e + k] += w[k];
        }
    }
    float bias[E] = {};
    if (a.out.bias.p) widen<T>(load_cols(reinterpret_cast<const T*>(a.out.bias.p) + i * a.out.bias.learner + c, left), bias);
    finish<T>(a.out, i, r, c, left, bias, v);
}

// ------------------------------------------------------------------------------------------------ launches
inline Operand operand(const psgd_view* v) {
    return v ? Operand{static_cast<const char*>(v->data), v->learner, v->row} : Operand{nullptr, 0, 0};
}

inline Operand moved(Operand o, int64_t elements, int bytes) { return o.p ? Operand{o.p + elements * bytes, o.learner, o.pitch} : o; }
inline Epilogue moved(const Epilogue& e, int64_t m, int64_t n, int bytes) {
    return Epilogue{moved(e.y, m * e.y.pitch + n, bytes), moved(e.z, m * e.z.pitch + n, bytes), moved(e.residual, m * e.residual.pitch + n, bytes),
                    moved(e.bias, n, bytes), e.act};
}

template <typename T, int BM, int BN, bool P_ALONG, bool Q_ALONG> int launch_tiles(GemmArgs a, hipStream_t s) {
    a.tiles_m = (int)parts_of(a.m, BM);
    a.tiles_n = (int)parts_of(a.n, BN);
    const int64_t grid = (int64_t)a.tiles_m * a.tiles_n * a.learners * a.split;
    if (grid > kMostGroups) {       // more than a launch counts: one half of C after the other
        if (a.split > 1 || (a.tiles_m == 1 && a.tiles_n == 1)) return fail(PSGD_EINVAL, "psgd_linear: too many tiles");
        const int64_t m = a.tiles_m > 1 ? (int64_t)(a.tiles_m / 2) * BM : 0, n = a.tiles_m > 1 ? 0 : (int64_t)(a.tiles_n / 2) * BN;
        GemmArgs low = a, high = a;
        low.m = m ? m : a.m, low.n = n ? n : a.n;
        high.m = a.m - m, high.n = a.n - n;
        high.p = moved(a.p, P_ALONG ? m * a.p.pitch : m, sizeof(T));
        high.q = moved(a.q, Q_ALONG ? n * a.q.pitch : n, sizeof(T));
        high.out = moved(a.out, m, n, sizeof(T));
        if (int rc = launch_tiles<T, BM, BN, P_ALONG, Q_ALONG>(low, s)) return rc;
        return launch_tiles<T, BM, BN, P_ALONG, Q_ALONG>(high, s);
    }
    using Shape = TileShape<BM, BN>;
    constexpr size_t tile = (size_t)(BM + BN) * kRowBytes, rows = (size_t)Shape::LANES / kWave * 32 * (BN / Shape::ACROSS_N + 4) * sizeof(float);
    auto fn = gemm_kernel<T, BM, BN, P_ALONG, Q_ALONG>;
    if (2 * tile >= 64 * 1024) {
        static LdsRecord record;
        if (int rc = allow_lds(reinterpret_cast<const void*>(fn), 2 * tile, record)) return rc;
    }
    const size_t lds = short_k(a.k, sizeof(T)) ? std::max(tile, rows) : 2 * tile;
    hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(TileShape<BM, BN>::LANES), lds, s, a);
    return PSGD_OK;
}

template <typename T, bool P_ALONG, bool Q_ALONG>
int launch_gemm(GemmArgs a, const Plan& plan, float* room, hipStream_t s) {
    a.split = plan.split;
    a.partial = plan.split > 1 ? room : nullptr;
    int rc;
    if (plan.rows == 256) {
        rc = launch_tiles<T, 256, 256, P_ALONG, Q_ALONG>(a, s);
    } else if (plan.rows == 128 && plan.cols == 128) {
        rc = launch_tiles<T, 128, 128, P_ALONG, Q_ALONG>(a, s);
    } else if (plan.rows == plan.cols) {
        rc = launch_tiles<T, 64, 64, P_ALONG, Q_ALONG>(a, s);
    } else if constexpr (sizeof(T) == 4) {
        if (plan.rows == 128) rc = launch_tiles<T, 128, 32, P_ALONG, Q_ALONG>(a, s);
        else rc = launch_tiles<T, 32, 128, P_ALONG, Q_ALONG>(a, s);
    } else {
        return fail(PSGD_EINVAL, "psgd_linear: no such tile");
    }
    if (rc || plan.split == 1) return rc;
    const JoinArgs j{room, plan.split, a.learners * a.m * a.n, a.m * a.n, a.out, a.m, a.n};
    hipLaunchKernelGGL((join_kernel<T>), dim3((unsigned)parts_of(a.m * parts_of(a.n, kPer<T>), 256), 1, a.learners), dim3(256), 0, s, j);
    return PSGD_OK;
}

template <typename T, int TILE> int launch_pair(GemmArgs dx, GemmArgs dw, hipStream_t s) {
    int64_t count[2];
    int k = 0;
    for (GemmArgs* a : {&dx, &dw}) {
        a->tiles_m = (int)parts_of(a->m, TILE);
        a->tiles_n = (int)parts_of(a->n, TILE);
        count[k++] = (int64_t)a->tiles_m * a->tiles_n * a->learners;
    }
    constexpr size_t bytes = (size_t)4 * TILE * kRowBytes;
    auto fn = gemm_pair_kernel<T, TILE>;
    if (bytes >= 64 * 1024) {
        static LdsRecord record;
        if (int rc = allow_lds(reinterpret_cast<const void*>(fn), bytes, record)) return rc;
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)(count[0] + count[1])), dim3(256), bytes, s, dx, dw, (uint32_t)count[0]);
    return PSGD_OK;
}

inline int check_linear_sizes(const char* name, int n, int64_t t, int64_t in, int64_t out, int act) {
    if (int rc = check_counts(name, n, t, in)) return rc;
    if (int rc = check_counts(name, n, t, out)) return rc;
    if (act < PSGD_ACT_NONE || act > PSGD_ACT_SILU) return fail(PSGD_EINVAL, "%s: act=%d", name, act);
    // arrays of all learners that have to be there, or that a workspace may hold, counted in elements
    for (const auto& [rows, cols] : {std::pair<int64_t, int64_t>{t, in}, {t, out}, {out, in}})
        if (rows > 0 && cols > kMostElements / n / rows) return fail(PSGD_EINVAL, "%s: the layer is too large", name);
    return PSGD_OK;
}
inline int check_room(const char* name, void* workspace, size_t have, size_t need) {
    if (need && (!workspace || have < need || reinterpret_cast<uintptr_t>(workspace) % 256))
        return fail(PSGD_EINVAL, "%s: %zu bytes of workspace are needed, at a multiple of 256", name, need);
    return PSGD_OK;
}

template <typename T, int TOK, int R> void launch_few(const FewArgs& all, int learners, hipStream_t s) {
    in_slices(parts_of(all.n, 4 * R), [&](int64_t first, unsigned count) {
        FewArgs f = all;
        const int64_t n = first * 4 * R;
        f.w = moved(all.w, n * all.w.pitch, sizeof(T));
        f.out = moved(all.out, 0, n, sizeof(T));
        f.n = all.n - n;
        hipLaunchKernelGGL((few_tokens_kernel<T, TOK, R>), dim3(count, learners), dim3(256), 0, s, f);
    });
}
template <typename T> int linear_of(const GemmArgs& a, const Plan& plan, void* workspace, int cus, hipStream_t s) {
    if (a.m > most_few(a.learners, a.n, sizeof(T), cus)) return launch_gemm<T, true, true>(a, plan, static_cast<float*>(workspace), s);
    const FewArgs all{a.p, a.q, a.out, a.m, a.k, a.n};
    const bool four = four_outputs(a.learners, a.n, cus);
#define PSGD_FEW(TOK)                                                                                                       \
    do {                                                                                                                    \
        if (four) launch_few<T, TOK, 4>(all, a.learners, s);                                                                \
        else launch_few<T, TOK, 1>(all, a.learners, s);                                                                     \
    } while (0)
    if (a.m <= 1) PSGD_FEW(1);
    else if (a.m <= 2) PSGD_FEW(2);
    else if (a.m <= 4) PSGD_FEW(4);
    else if constexpr (sizeof(T) == 4) launch_few<T, 8, 1>(all, a.learners, s);
#undef PSGD_FEW
    return PSGD_OK;
}

template <typename T>
int linear_grad_of(const psgd_view* dy, const psgd_view* z, const psgd_view* x, const psgd_view* w, const psgd_view* dx, const psgd_view* dw,
                   const psgd_view* db, int act, int n, int64_t t, int64_t in, int64_t out, char* room, int cus, hipStream_t s) {
    const GradRoom r = grad_room(act, n, t, in, out, sizeof(T), cus, dx, dw, db);
    float* sums = reinterpret_cast<float*>(room + r.dz);
    float* product = reinterpret_cast<float*>(room + r.dz + r.sums);
    Operand dz = operand(dy);
    // nobody asks for what it makes, or there is nothing to make it of: a grid of no workgroups is an error to the runtime
    if (out > 0 && (db || (act != PSGD_ACT_NONE && (dx || dw)))) {
        const SlopeArgs a{operand(dy), operand(z), act != PSGD_ACT_NONE ? room : nullptr, r.dz_pitch, db ? sums : nullptr, t, out};
        const int64_t slabs = slope_slabs(n, t, out, sizeof(T), cus);
        const dim3 grid((unsigned)parts_of(out, kWave * kPer<T>), (unsigned)slabs, n);
        if (act == PSGD_ACT_NONE) hipLaunchKernelGGL((slope_kernel<T, PSGD_ACT_NONE>), grid, dim3(256), 0, s, a);
        else if (act == PSGD_ACT_RELU) hipLaunchKernelGGL((slope_kernel<T, PSGD_ACT_RELU>), grid, dim3(256), 0, s, a);
        else if (act == PSGD_ACT_GELU) hipLaunchKernelGGL((slope_kernel<T, PSGD_ACT_GELU>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((slope_kernel<T, PSGD_ACT_SILU>), grid, dim3(256), 0, s, a);
        if (act != PSGD_ACT_NONE) dz = Operand{room, t * r.dz_pitch, r.dz_pitch};
        if (db) {
            in_slices(parts_of(out, kWave), [&](int64_t first, unsigned count) {
                hipLaunchKernelGGL((sum_slabs_kernel<T>), dim3(count, n), dim3(kSumWaves * kWave), 0, s, sums, slabs, out, operand(db), first);
            });
        }
    }
    GemmArgs ax{dz, operand(w), Epilogue{operand(dx), {}, {}, {}, PSGD_ACT_NONE}, nullptr, t, in, out, n, 1, 0, 0};
    GemmArgs aw{dz, operand(x), Epilogue{operand(dw), {}, {}, {}, PSGD_ACT_NONE}, nullptr, out, in, t, n, 1, 0, 0};
    const GradPlan g = grad_plan(n, t, in, out, sizeof(T), cus, dx, dw);
    if (g.pair) {
        if constexpr (sizeof(T) == 2)
            if (g.dx.rows == 128) return launch_pair<T, 128>(ax, aw, s);
        return launch_pair<T, 64>(ax, aw, s);
    }
    if (dx)
        if (int rc = launch_gemm<T, true, false>(ax, g.dx, product, s)) return rc;
    if (dw && g.few) {
        const FewGradArgs f{dz, operand(x), operand(dw), t, in, out, g.few_rows};
        const dim3 grid((unsigned)parts_of(in, kWave * kPer<T>), (unsigned)parts_of(out, 4 * g.few_rows), n);
        if (t <= 2) hipLaunchKernelGGL((few_tokens_grad_kernel<T, 2>), grid, dim3(256), 0, s, f);
        else if (t <= 4) hipLaunchKernelGGL((few_tokens_grad_kernel<T, 4>), grid, dim3(256), 0, s, f);
        else if (t <= 8) hipLaunchKernelGGL((few_tokens_grad_kernel<T, 8>), grid, dim3(256), 0, s, f);
        else if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((few_tokens_grad_kernel<T, 16>), grid, dim3(256), 0, s, f);
    } else if (dw) {
        if (int rc = launch_gemm<T, false, false>(aw, g.dw, product, s)) return rc;
    }
    return PSGD_OK;
}

}  // namespace
}  // namespace psgd

extern "C" {

size_t psgd_linear_workspace(const psgd_view* x, const psgd_view* w, int n, int64_t t, int64_t in, int64_t out) {
    using namespace psgd;
    int cus = 0;
    if (!x || !w || check_linear_sizes("psgd_linear_workspace", n, t, in, out, 0) || t == 0 || out == 0 || compute_units(&cus)) return 0;
    return forward_plan(n, t, out, in, elem_bytes(x->type), cus).bytes(n, t, out);
}

int psgd_linear(const psgd_view* x, const psgd_view* w, const psgd_view* bias, const psgd_view* residual, const psgd_view* y,
                const psgd_view* z, int act, int n, int64_t t, int64_t in, int64_t out, void* workspace, size_t workspace_bytes,
                void* stream) {
    using namespace psgd;
    const char* name = "psgd_linear";
    clear_error();
    if (!x || !w || !y) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_linear_sizes(name, n, t, in, out, act)) return rc;
    for (const psgd_view* v : {x, w, y, bias, residual, z})
        if (v && (!float_type(v->type) || v->type != x->type)) return fail(PSGD_EINVAL, "%s: all operands must be float or bf16 alike", name);
    if (t == 0 || out == 0) return PSGD_OK;
    const Extent ex{"x", x, n, t, in}, ew{"w", w, n, out, in}, ey{"y", y, n, t, out};
    const Extent eb{"bias", bias ? bias : w, n, 1, bias ? out : 0}, er{"residual", residual ? residual : x, n, t, residual ? out : 0};
    const Extent ez{"z", z ? z : y, n, t, z ? out : 0};
    for (const Extent* e : {&ex, &ew, &eb, &er})
        if (int rc = check_operand(name, *e, false)) return rc;
    for (const Extent* e : {&ey, &ez})
        if (int rc = check_operand(name, *e, true)) return rc;
    for (const Extent* e : {&ex, &ew, &eb}) {
        if (int rc = refuse_overlap(name, ey, *e)) return rc;
        if (int rc = refuse_overlap(name, ez, *e)) return rc;
    }
    if (int rc = refuse_overlap(name, ey, er, true)) return rc;
    if (int rc = refuse_overlap(name, ez, er)) return rc;
    if (int rc = refuse_overlap(name, ez, ey)) return rc;
    int cus = 0;
    if (int rc = compute_units(&cus)) return rc;
    const Plan plan = forward_plan(n, t, out, in, elem_bytes(x->type), cus);
    const size_t need = plan.bytes(n, t, out);
    if (int rc = check_room(name, workspace, workspace_bytes, need)) return rc;
    psgd_view vw;
    const Extent room = flat("the workspace", workspace, (int64_t)(need / 4), &vw);
    for (const Extent* e : {&ex, &ew, &eb, &er, &ey, &ez})
        if (int rc = refuse_overlap(name, room, *e)) return rc;
    const GemmArgs a{operand(x), operand(w), Epilogue{operand(y), operand(z), operand(residual), operand(bias), act}, nullptr, t, out, in, n, 1, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (int rc = x->type == PSGD_F32 ? linear_of<float>(a, plan, workspace, cus, s) : linear_of<uint16_t>(a, plan, workspace, cus, s)) return rc;
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

size_t psgd_linear_grad_workspace(const psgd_view* dy, const psgd_view* x, const psgd_view* w, const psgd_view* dx, const psgd_view* dw,
                                  const psgd_view* db, int act, int n, int64_t t, int64_t in, int64_t out) {
    using namespace psgd;
    int cus = 0;
    if (!dy || !x || !w || check_linear_sizes("psgd_linear_grad_workspace", n, t, in, out, act) || compute_units(&cus)) return 0;
    return grad_room(act, n, t, in, out, elem_bytes(x->type), cus, dx, dw, db).total;
}

int psgd_linear_grad(const psgd_view* dy, const psgd_view* z, const psgd_view* x, const psgd_view* w, const psgd_view* dx,
                     const psgd_view* dw, const psgd_view* db, int act, int n, int64_t t, int64_t in, int64_t out, void* workspace,
                     size_t workspace_bytes, void* stream) {
    using namespace psgd;
    const char* name = "psgd_linear_grad";
    clear_error();
    if (!dy || !x || !w) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_linear_sizes(name, n, t, in, out, act)) return rc;
    if (act != PSGD_ACT_NONE && !z) return fail(PSGD_EINVAL, "%s: z is needed for the activation's slope", name);
    if (act == PSGD_ACT_NONE) z = nullptr;
    for (const psgd_view* v : {dy, x, w, z, dx, dw, db})
        if (v && (!float_type(v->type) || v->type != x->type)) return fail(PSGD_EINVAL, "%s: all operands must be float or bf16 alike", name);
    if (!dx && !dw && !db) return PSGD_OK;
    const Extent edy{"dy", dy, n, t, out}, ex{"x", x, n, t, in}, ew{"w", w, n, out, in}, ez{"z", z ? z : dy, n, t, z ? out : 0};
    const Extent edx{"dx", dx ? dx : x, n, t, dx ? in : 0}, edw{"dw", dw ? dw : w, n, out, dw ? in : 0}, edb{"db", db ? db : w, n, 1, db ? out : 0};
    for (const Extent* e : {&edy, &ex, &ew, &ez})
        if (int rc = check_operand(name, *e, false)) return rc;
    for (const Extent* e : {&edx, &edw, &edb}) {
        if (int rc = check_operand(name, *e, true)) return rc;
        for (const Extent* o : {&edy, &ex, &ew, &ez})
            if (int rc = refuse_overlap(name, *e, *o)) return rc;
    }
    if (int rc = refuse_overlap(name, edx, edw)) return rc;
    if (int rc = refuse_overlap(name, edx, edb)) return rc;
    if (int rc = refuse_overlap(name, edw, edb)) return rc;
    int cus = 0;
    if (int rc = compute_units(&cus)) return rc;
    const size_t need = grad_room(act, n, t, in, out, elem_bytes(x->type), cus, dx, dw, db).total;
    if (int rc = check_room(name, workspace, workspace_bytes, need)) return rc;
    psgd_view vw;
    const Extent room = flat("the workspace", workspace, (int64_t)(need / 4), &vw);
    for (const Extent* e : {&edy, &ex, &ew, &ez, &edx, &edw, &edb})
        if (int rc = refuse_overlap(name, room, *e)) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* p = static_cast<char*>(workspace);
    if (t == 0) dx = nullptr;
    if (in == 0) dx = dw = nullptr;
    if (out == 0) dw = db = nullptr;
    if (int rc = x->type == PSGD_F32 ? linear_grad_of<float>(dy, z, x, w, dx, dw, db, act, n, t, in, out, p, cus, s)
                                     : linear_grad_of<uint16_t>(dy, z, x, w, dx, dw, db, act, n, t, in, out, p, cus, s))
        return rc;
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

}  // extern "C"
