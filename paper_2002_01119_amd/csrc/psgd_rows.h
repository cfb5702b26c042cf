// What the layers' and losses' translation units share (gfx950): operands as the kernels get them, 128-bit accesses to rows that start at any
// element, wavefront reductions, and the host's checks of operands.
#ifndef PSGD_ROWS_H
#define PSGD_ROWS_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "psgd_internal.h"
#include "psgd_layers.h"
#include "psgd_layers_plan.h"

namespace psgd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------------ elements
// A lane's access is 16 bytes: four floats or eight bf16.  Rows start at any element: gfx950 takes such accesses unaligned.
template <typename T> constexpr int kPer = 16 / (int)sizeof(T);

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {      // round to nearest even, one instruction
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

template <typename T> __device__ __forceinline__ float load_1(const T* p);
template <> __device__ __forceinline__ float load_1(const float* p) { return *p; }
template <> __device__ __forceinline__ float load_1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_1(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

template <typename T> __device__ __forceinline__ u32x4 load_raw(const T* p) { return *reinterpret_cast<const u32x4_any*>(p); }
// The same where the row ends inside: `left` elements are there (possibly none), the others read as `fill`, a pattern of T.
__device__ __forceinline__ u32x4 load_raw_upto(const float* p, int64_t left, uint32_t fill) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = i < left ? __float_as_uint(p[i]) : fill;
    return r;
}
__device__ __forceinline__ u32x4 load_raw_upto(const uint16_t* p, int64_t left, uint32_t fill) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = 2 * i < left ? p[2 * i] : fill, b = 2 * i + 1 < left ? p[2 * i + 1] : fill;
        r[i] = a | b << 16;
    }
    return r;
}
template <typename T> __device__ __forceinline__ u32x4 load_cols(const T* p, int64_t left, uint32_t fill = 0) {
    return left >= kPer<T> ? load_raw(p) : load_raw_upto(p, left, fill);
}
template <typename T> __device__ __forceinline__ void widen(u32x4 r, float (&v)[kPer<T>]);
template <> __device__ __forceinline__ void widen<float>(u32x4 r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
template <> __device__ __forceinline__ void widen<uint16_t>(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = low_bf16(r[i]);
        v[2 * i + 1] = high_bf16(r[i]);
    }
}
__device__ __forceinline__ u32x4 narrow(const float (&v)[4], float) {
    return (u32x4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}
__device__ __forceinline__ u32x4 narrow(const float (&v)[8], uint16_t) {
    return (u32x4){two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
}
template <typename T> __device__ __forceinline__ void store_cols(T* p, const float (&v)[kPer<T>], int64_t left) {
    if (left >= kPer<T>) {
        *reinterpret_cast<u32x4_any*>(p) = narrow(v, T{});
    } else {
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i)
            if (i < left) store_1(p + i, v[i]);
    }
}
// kPer<T> parameters of either type, as floats.
template <typename T, typename P> __device__ __forceinline__ void load_params(const P* p, int64_t left, float (&v)[kPer<T>]) {
    if constexpr (sizeof(P) == sizeof(T)) {
        widen<P>(load_cols(p, left), v);
    } else if constexpr (sizeof(P) == 4) {          // T is bf16: eight floats
        float a[4], b[4];
        widen<float>(load_cols(p, left), a);
        widen<float>(load_cols(p + 4, left - 4), b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    } else {                                        // T is float: four bf16
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? load_1(p + i) : 0.0f;
    }
}

// ------------------------------------------------------------------------------------------------ wavefront reductions
struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct Max {   // NaN if either is
    static __device__ __forceinline__ float of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
};
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// Over the 64 lanes, in every lane: neighbours, pairs, halves of a row of 16 mirrored, then rows and halves exchanged.  All of it in the
// vector unit; the order is the same in every lane, so all hold the same bits.
// LANES: over 16 or 32 lanes that belong together instead.
template <typename OP, int LANES = kWave> __device__ __forceinline__ float wave_all(float v) {
    static_assert(LANES == 16 || LANES == 32 || LANES == kWave, "rows of 16 lanes");
    v = OP::of(v, dpp<0xB1>(v));    // quad_perm 1 0 3 2
    v = OP::of(v, dpp<0x4E>(v));    // quad_perm 2 3 0 1
    v = OP::of(v, dpp<0x141>(v));   // row_half_mirror
    v = OP::of(v, dpp<0x140>(v));   // row_mirror
    if constexpr (LANES == 16) return v;
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = OP::of(__uint_as_float(a[0]), __uint_as_float(a[1]));
    if constexpr (LANES == 32) return v;
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return OP::of(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Over a workgroup of W wavefronts, in every lane.  `room`: W floats of LDS that nothing else reads until the next barrier after this call's own.
template <typename OP, int W> __device__ __forceinline__ float group_all(float v, float* room) {
    v = wave_all<OP>(v);
    if constexpr (W == 1) return v;
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = v;
    __syncthreads();
    float r = room[0];
#pragma unroll
    for (int i = 1; i < W; ++i) r = OP::of(r, room[i]);
    return r;
}

// Two of them behind one barrier.
template <typename OP, int W> __device__ __forceinline__ void group_all_2(float& a, float& b, float* room) {
    a = wave_all<OP>(a);
    b = wave_all<OP>(b);
    if constexpr (W == 1) return;
    if (threadIdx.x % kWave == 0) {
        room[threadIdx.x / kWave] = a;
        room[W + threadIdx.x / kWave] = b;
    }
    __syncthreads();
    a = room[0];
    b = room[W];
#pragma unroll
    for (int i = 1; i < W; ++i) {
        a = OP::of(a, room[i]);
        b = OP::of(b, room[W + i]);
    }
}

// ------------------------------------------------------------------------------------------------ host: operands and checks
inline int hip_error(hipError_t e, const char* what) { return fail(PSGD_EHIP, "%s: %s", what, hipGetErrorString(e)); }

// A kernel that is launched with more than 64 KB of LDS is opted in, once a device (`done`: its own record).
struct LdsRecord {
    bool done[64];
};
inline int allow_lds(const void* fn, size_t bytes, LdsRecord& record) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_error(e, "hipGetDevice");
    if (dev >= 0 && dev < 64 && __atomic_load_n(&record.done[dev], __ATOMIC_RELAXED)) return PSGD_OK;
    e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return hip_error(e, "hipFuncSetAttribute(MaxDynamicSharedMemorySize)");
    if (dev >= 0 && dev < 64) __atomic_store_n(&record.done[dev], true, __ATOMIC_RELAXED);
    return PSGD_OK;
}

inline int elem_bytes(int type) { return type == PSGD_BF16 ? 2 : 4; }

// Compute units of the current device, asked for once a device.
inline int compute_units(int* cus) {
    static int known[64] = {0};
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_error(e, "hipGetDevice");
    if (dev < 0 || dev >= 64) return fail(PSGD_EHIP, "device index %d unsupported", dev);
    int c = __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
    if (c == 0) {
        e = hipDeviceGetAttribute(&c, hipDeviceAttributeMultiprocessorCount, dev);
        if (e != hipSuccess) return hip_error(e, "hipDeviceGetAttribute");
        c = c > 0 ? c : 1;
        __atomic_store_n(&known[dev], c, __ATOMIC_RELAXED);
    }
    *cus = c;
    return PSGD_OK;
}

// An operand with its extent: n learners of `rows` rows of `cols` elements.
struct Extent {
    const char* what;
    const psgd_view* v;
    int64_t n, rows, cols;
    int64_t span() const { return (n - 1) * v->learner + (rows - 1) * v->row + cols; }      // elements from the first to behind the last
    uintptr_t begin() const { return reinterpret_cast<uintptr_t>(v->data); }
    uintptr_t end() const { return begin() + (uintptr_t)span() * elem_bytes(v->type); }
    bool empty() const { return n == 0 || rows == 0 || cols == 0; }
};

constexpr int64_t kMostElements = (int64_t)1 << 48;

// Pointer, type and strides of one operand.  `written`: no two of its elements may share an address.
inline int check_operand(const char* name, const Extent& x, bool written) {
    const psgd_view& v = *x.v;
    if (x.empty()) return PSGD_OK;
    if (!v.data) return fail(PSGD_EINVAL, "%s: %s is a null pointer", name, x.what);
    const uintptr_t unit = (uintptr_t)elem_bytes(v.type);
    if (x.begin() % unit) return fail(PSGD_EALIGN, "%s: %s is not aligned to its element size", name, x.what);
    if (v.learner < 0 || v.row < 0) return fail(PSGD_EINVAL, "%s: a stride of %s is negative", name, x.what);
    if (v.learner > kMostElements / x.n || v.row > kMostElements / x.rows || x.cols > kMostElements)
        return fail(PSGD_EINVAL, "%s: %s is too large", name, x.what);
    if (written) {
        const bool rows_in = x.rows == 1 || v.row >= x.cols, learners_in = x.n == 1 || v.learner >= x.cols;
        const bool learner_outer = rows_in && (x.n == 1 || v.learner >= (x.rows - 1) * v.row + x.cols);
        const bool row_outer = learners_in && (x.rows == 1 || v.row >= (x.n - 1) * v.learner + x.cols);
        if (!learner_outer && !row_outer) return fail(PSGD_EALIAS, "%s: rows of the output %s overlap", name, x.what);
    }
    return PSGD_OK;
}

inline bool same_place(const Extent& a, const Extent& b) {
    return a.v->data == b.v->data && a.v->type == b.v->type && (a.n == 1 || a.v->learner == b.v->learner) &&
           (a.rows == 1 || a.v->row == b.v->row);
}

// Blocks of `ra` bytes every `pitch` bytes from a and blocks of `rb` bytes as far apart from b: whether any two meet.  A block of a may
// also meet one of b a whole number of pitches away, so only the distance modulo the pitch counts; said to meet if the blocks are
// longer than the pitch.
inline bool combs_meet(uintptr_t a, int64_t ra, uintptr_t b, int64_t rb, int64_t pitch) {
    if (ra > pitch || rb > pitch || pitch <= 0) return true;
    int64_t off = (int64_t)(b - a) % pitch;
    if (off < 0) off += pitch;
    return off < ra || off + rb > pitch;
}

// Whether two operands may share a byte: their ranges meet, and they are not shown to be apart as blocks of learners a common distance
// apart (layers in the rows of one [n, d] array) or as rows a common distance apart (column slices of one activation).
inline bool may_overlap(const Extent& a, const Extent& b) {
    if (a.empty() || b.empty()) return false;
    if (a.begin() >= b.end() || b.begin() >= a.end()) return false;
    const int ea = elem_bytes(a.v->type), eb = elem_bytes(b.v->type);
    const int64_t pa = a.v->learner * ea, pb = b.v->learner * eb, qa = a.v->row * ea, qb = b.v->row * eb;
    const int64_t block_a = ((a.rows - 1) * a.v->row + a.cols) * ea, block_b = ((b.rows - 1) * b.v->row + b.cols) * eb;
    const bool one_a = a.n == 1, one_b = b.n == 1;
    if (!(one_a && one_b) && (pa == pb || one_a || one_b)) {
        if (!combs_meet(a.begin(), block_a, b.begin(), block_b, one_a ? pb : pa)) return false;
    }
    // rows a common distance apart through all learners
    if (qa == qb && qa > 0 && (one_a || pa % qa == 0) && (one_b || pb % qa == 0) &&
        !combs_meet(a.begin(), a.cols * ea, b.begin(), b.cols * eb, qa))
        return false;
    return true;
}

inline Extent flat(const char* what, const void* p, int64_t count, psgd_view* room, int type = PSGD_F32) {
    *room = psgd_view{const_cast<void*>(p), 0, 0, type};
    return Extent{what, room, 1, 1, count};
}

inline int refuse_overlap(const char* name, const Extent& out, const Extent& other, bool same_allowed = false) {
    if (same_allowed && same_place(out, other)) return PSGD_OK;
    if (may_overlap(out, other)) return fail(PSGD_EALIAS, "%s: the output %s overlaps %s", name, out.what, other.what);
    return PSGD_OK;
}

inline int check_counts(const char* name, int n, int64_t t, int64_t c) {
    if (n < 1 || n > PSGD_MAX_N) return fail(PSGD_EINVAL, "%s: n=%d outside 1..%d", name, n, (int)PSGD_MAX_N);
    if (t < 0 || c < 0) return fail(PSGD_EINVAL, "%s: a negative size", name);
    if (t > INT32_MAX || c > INT32_MAX) return fail(PSGD_EINVAL, "%s: a size beyond 2^31 - 1", name);
    return PSGD_OK;
}

inline bool float_type(int type) { return type == PSGD_F32 || type == PSGD_BF16; }

}  // namespace
}  // namespace psgd
#endif
