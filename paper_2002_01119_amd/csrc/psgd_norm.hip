// Layer norm of all learners, forward and backward (gfx950).
//
//     y = (x - m) r g + b,   m = mean_c x,   r = (mean_c (x - m)^2 + eps)^-1/2
//     dx = r (u - mean_c u - h mean_c(u h)) [+ add],   u = dy g,   h = (x - m) r
//     dg = sum_t dy h,   db = sum_t dy
//
// About ten vector operations an element against 4 bytes (forward, bf16) to 16 (backward, float, add): bound by HBM.  So every array is
// touched once: a row stays in the registers of 16 to 1024 lanes (a lane holds NV groups of 16 bytes) between the load and the
// store, the variance is taken from there in a second pass, and a lane keeps the gain's and bias's columns for all rows
// it walks.  The gradients of gain and bias are sums down the columns, which those same lanes own: each workgroup walks a slab of one
// learner's rows with running sums in registers and leaves one partial row, and a second kernel adds the slabs up in a fixed order.
//
// Measured: forward 4 x 4096 x 4096 bf16 56.5 us (268 MB, 4.75 TB/s; a copy of that size 5.3); backward 8 x 4096 x 2048 bf16 with `add` 106 us (537 MB, 5.1) and
// 4.9 for its slabs; 16 x 257 x 1001 float 13 and 4, where a row of 1001 keeps 251 of 256 lanes busy and a workgroup has eight or nine rows to hide
// its start behind; one row of 512 for each of eight learners 2.7 us, the launch and one trip to memory.
#include "psgd_rows.h"

#include <initializer_list>

namespace psgd {
namespace {

struct Rows {       // [n, t, c] in the kernels
    char* p;
    int64_t learner, row;   // in elements
};
struct Vecs {       // [n, c]
    char* p;
    int64_t learner;
};
template <typename T> __device__ __forceinline__ T* at(const Rows& a, int64_t i, int64_t r) {
    return reinterpret_cast<T*>(a.p) + i * a.learner + r * a.row;
}
template <typename T> __device__ __forceinline__ T* at(const Vecs& a, int64_t i) { return reinterpret_cast<T*>(a.p) + i * a.learner; }

struct NormArgs {
    Rows x, y;
    Vecs gain, bias;
    float *mean, *rstd;
    int64_t t, c;
    float eps, count;       // count: c, divided by (a row of one value has that value for its mean)
};

// A row takes 16, 32, 64, 256 or 1024 lanes; a workgroup has 256 lanes or 1024, and a row or as many as that makes.
template <int LANES> constexpr int kGroupThreads = LANES < 256 ? 256 : LANES;
template <int LANES> constexpr int kGroupRows = kGroupThreads<LANES> / LANES;
template <int LANES> constexpr int kRowWaves = LANES < kWave ? 1 : LANES / kWave;

// Sums over a row's lanes, in every one of them.  `room`: LDS for the wavefronts of a row, which nothing else reads until the next barrier after this call's own.
template <int LANES> __device__ __forceinline__ float row_sum(float v, float* room) {
    if constexpr (LANES <= kWave) return wave_all<Sum, LANES>(v);
    else return group_all<Sum, LANES / kWave>(v, room);
}
template <int LANES> __device__ __forceinline__ void row_sums(float& a, float& b, float* room) {
    if constexpr (LANES <= kWave) {
        a = wave_all<Sum, LANES>(a);
        b = wave_all<Sum, LANES>(b);
    } else {
        group_all_2<Sum, LANES / kWave>(a, b, room);
    }
}

template <typename T, typename P, int LANES, int NV>
__global__ __launch_bounds__(kGroupThreads<LANES>) void norm_kernel(NormArgs a) {
    constexpr int E = kPer<T>;
    __shared__ float room[2][kRowWaves<LANES>];
    const int lane = threadIdx.x % LANES;
    const int64_t i = blockIdx.y;
    float g[NV][E], b[NV][E];
    int left[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int64_t col = (int64_t)(j * LANES + lane) * E;
        left[j] = (int)(a.c - col);
        load_params<T, P>(at<P>(a.gain, i) + col, left[j], g[j]);
        if (a.bias.p) {
            load_params<T, P>(at<P>(a.bias, i) + col, left[j], b[j]);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) b[j][k] = 0.0f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * kGroupRows<LANES>;
    for (int64_t r = (int64_t)blockIdx.x * kGroupRows<LANES> + threadIdx.x / LANES; r < a.t; r += step) {
        const T* x = at<T>(a.x, i, r) + lane * E;
        float v[NV][E];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) widen<T>(load_cols(x + j * LANES * E, left[j]), v[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < E; ++k) sum += v[j][k];
        const float m = row_sum<LANES>(sum, room[0]) / a.count;
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                v[j][k] = k < left[j] ? v[j][k] - m : 0.0f;
                sq += v[j][k] * v[j][k];
            }
        const float var = row_sum<LANES>(sq, room[1]) / a.count;
        const float rs = 1.0f / sqrtf(var + a.eps);
        if (a.mean && lane == 0) {
            a.mean[i * a.t + r] = m;
            a.rstd[i * a.t + r] = rs;
        }
        T* y = at<T>(a.y, i, r) + lane * E;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < E; ++k) v[j][k] = __builtin_fmaf(v[j][k] * rs, g[j][k], b[j][k]);
            store_cols<T>(y + j * LANES * E, v[j], left[j]);
        }
    }
}

// Rows that no workgroup's registers hold: read three times, from the caches where they fit.
template <typename T, typename P> __global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
    constexpr int E = kPer<T>;
    __shared__ float room[2][16];
    const int64_t i = blockIdx.y;
    for (int64_t r = blockIdx.x; r < a.t; r += gridDim.x) {
        const T* x = at<T>(a.x, i, r);
        float v[E], g[E], b[E], sum = 0.0f, sq = 0.0f;
        for (int64_t col = (int64_t)threadIdx.x * E; col < a.c; col += 1024 * E) {
            widen<T>(load_cols(x + col, a.c - col), v);
#pragma unroll
            for (int k = 0; k < E; ++k) sum += v[k];
        }
        const float m = group_all<Sum, 16>(sum, room[0]) / a.count;
        for (int64_t col = (int64_t)threadIdx.x * E; col < a.c; col += 1024 * E) {
            widen<T>(load_cols(x + col, a.c - col), v);
#pragma unroll
            for (int k = 0; k < E; ++k) sq += k < a.c - col ? (v[k] - m) * (v[k] - m) : 0.0f;
        }
        const float rs = 1.0f / sqrtf(group_all<Sum, 16>(sq, room[1]) / a.count + a.eps);
        if (a.mean && threadIdx.x == 0) {
            a.mean[i * a.t + r] = m;
            a.rstd[i * a.t + r] = rs;
        }
        for (int64_t col = (int64_t)threadIdx.x * E; col < a.c; col += 1024 * E) {
            const int64_t left = a.c - col;
            widen<T>(load_cols(x + col, left), v);
            load_params<T, P>(at<P>(a.gain, i) + col, left, g);
            if (a.bias.p) load_params<T, P>(at<P>(a.bias, i) + col, left, b);
#pragma unroll
            for (int k = 0; k < E; ++k) v[k] = a.bias.p ? __builtin_fmaf((v[k] - m) * rs, g[k], b[k]) : (v[k] - m) * rs * g[k];
            store_cols<T>(at<T>(a.y, i, r) + col, v, left);
        }
    }
}

struct NormGradArgs {
    Rows dy, x, add, dx;
    Vecs gain;
    const float *mean, *rstd;
    float* partial;      // [n][gridDim.x][2][c]: a slab's sums for the gain and for the bias; NULL: nobody asks for them
    int64_t t, c;
    float inv_c;
};

template <typename T, typename P, int LANES, int NV, bool ADD>
__global__ __launch_bounds__(kGroupThreads<LANES>) void norm_grad_kernel(NormGradArgs a) {
    constexpr int E = kPer<T>, ROWS = kGroupRows<LANES>;
    __shared__ float room[2][2 * kRowWaves<LANES>];
    extern __shared__ float sums[];      // several rows at a time: [2][NV * E * LANES], to join their lanes' sums
    const int lane = threadIdx.x % LANES;
    const int64_t i = blockIdx.y;
    // 1024 lanes have 128 registers each: they fetch the gain again for each use, and `add` when it is wanted
    constexpr bool HELD = LANES < 1024;
    float g[HELD ? NV : 1][E], dg[NV][E], db[NV][E];
    int left[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int64_t col = (int64_t)(j * LANES + lane) * E;
        left[j] = (int)(a.c - col);
        if (HELD) load_params<T, P>(at<P>(a.gain, i) + col, left[j], g[HELD ? j : 0]);
#pragma unroll
        for (int k = 0; k < E; ++k) dg[j][k] = db[j][k] = 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * kGroupRows<LANES>;
    int turn = 0;
    for (int64_t r = (int64_t)blockIdx.x * kGroupRows<LANES> + threadIdx.x / LANES; r < a.t; r += step, turn ^= 1) {
        const T *px = at<T>(a.x, i, r) + lane * E, *pdy = at<T>(a.dy, i, r) + lane * E;
        const T* padd = ADD ? at<T>(a.add, i, r) + lane * E : nullptr;
        u32x4 rx[NV], rdy[NV], radd[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            rx[j] = load_cols(px + j * LANES * E, left[j]);
            rdy[j] = load_cols(pdy + j * LANES * E, left[j]);
            if (ADD && HELD) radd[j] = load_cols(padd + j * LANES * E, left[j]);
        }
        const float m = a.mean[i * a.t + r], rs = a.rstd[i * a.t + r];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[E], dy[E];
            if (!HELD) load_params<T, P>(at<P>(a.gain, i) + (j * LANES + lane) * E, left[j], g[0]);
            widen<T>(rx[j], x);
            widen<T>(rdy[j], dy);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float h = (x[k] - m) * rs, u = dy[k] * g[HELD ? j : 0][k];
                s1 += u;
                s2 = __builtin_fmaf(u, h, s2);
                dg[j][k] = __builtin_fmaf(dy[k], h, dg[j][k]);     // columns past the row's end: dy reads as zero
                db[j][k] += dy[k];
            }
        }
        // two rooms in turn: a wavefront may be a row ahead of one that still reads
        row_sums<LANES>(s1, s2, room[turn]);
        const float mu = s1 * a.inv_c, muh = s2 * a.inv_c;
        T* pdx = at<T>(a.dx, i, r) + lane * E;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[E], dy[E], out[E];
            if (!HELD) load_params<T, P>(at<P>(a.gain, i) + (j * LANES + lane) * E, left[j], g[0]);
            widen<T>(rx[j], x);
            widen<T>(rdy[j], dy);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float h = (x[k] - m) * rs;
                out[k] = rs * (__builtin_fmaf(dy[k], g[HELD ? j : 0][k], -mu) - h * muh);
            }
            if (ADD) {
                float e[E];
                widen<T>(HELD ? radd[j] : load_cols(padd + j * LANES * E, left[j]), e);
#pragma unroll
                for (int k = 0; k < E; ++k) out[k] += e[k];
            }
            store_cols<T>(pdx + j * LANES * E, out, left[j]);
        }
    }
    if (!a.partial) return;
    float* part = a.partial + (i * gridDim.x + blockIdx.x) * 2 * a.c;
    if constexpr (ROWS > 1) {
        for (int w = 0; w < ROWS; ++w) {                // one row's lanes after the other: a fixed order
            if ((int)threadIdx.x / LANES == w) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int k = 0; k < E; ++k) {
                        float *q0 = &sums[(j * E + k) * LANES + lane], *q1 = q0 + NV * E * LANES;
                        *q0 = w ? *q0 + dg[j][k] : dg[j][k];
                        *q1 = w ? *q1 + db[j][k] : db[j][k];
                    }
            }
            __syncthreads();
        }
        for (int e = threadIdx.x; e < NV * E * LANES; e += kGroupThreads<LANES>) {
            const int k = e % E, l = e / E % LANES, j = e / (E * LANES);      // column (j * LANES + l) * E + k
            if (e < a.c) {
                part[e] = sums[(j * E + k) * LANES + l];
                part[a.c + e] = sums[(NV * E + j * E + k) * LANES + l];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t col = (int64_t)(j * LANES + lane) * E;
#pragma unroll
            for (int h = 0; h < E; h += 4) {
                float u[4] = {dg[j][h], dg[j][h + 1], dg[j][h + 2], dg[j][h + 3]}, v[4] = {db[j][h], db[j][h + 1], db[j][h + 2], db[j][h + 3]};
                store_cols<float>(part + col + h, u, left[j] - h);
                store_cols<float>(part + a.c + col + h, v, left[j] - h);
            }
        }
    }
}

// The input's gradient of rows that no workgroup's registers hold.
template <typename T, typename P, bool ADD> __global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a) {
    constexpr int E = kPer<T>;
    __shared__ float room[2][32];
    const int64_t i = blockIdx.y;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.t; r += gridDim.x, turn ^= 1) {
        const T *px = at<T>(a.x, i, r), *pdy = at<T>(a.dy, i, r);
        const float m = a.mean[i * a.t + r], rs = a.rstd[i * a.t + r];
        float x[E], dy[E], g[E], s1 = 0.0f, s2 = 0.0f;
        for (int64_t col = (int64_t)threadIdx.x * E; col < a.c; col += 1024 * E) {
            const int64_t left = a.c - col;
            widen<T>(load_cols(px + col, left), x);
            widen<T>(load_cols(pdy + col, left), dy);
            load_params<T, P>(at<P>(a.gain, i) + col, left, g);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float u = dy[k] * g[k];
                s1 += u;
                s2 = __builtin_fmaf(u, (x[k] - m) * rs, s2);
            }
        }
        group_all_2<Sum, 16>(s1, s2, room[turn]);
        const float mu = s1 * a.inv_c, muh = s2 * a.inv_c;
        for (int64_t col = (int64_t)threadIdx.x * E; col < a.c; col += 1024 * E) {
            const int64_t left = a.c - col;
            widen<T>(load_cols(px + col, left), x);
            widen<T>(load_cols(pdy + col, left), dy);
            load_params<T, P>(at<P>(a.gain, i) + col, left, g);
            float out[E];
#pragma unroll
            for (int k = 0; k < E; ++k) out[k] = rs * (__builtin_fmaf(dy[k], g[k], -mu) - (x[k] - m) * rs * muh);
            if (ADD) {
                float e[E];
                widen<T>(load_cols(at<T>(a.add, i, r) + col, left), e);
#pragma unroll
                for (int k = 0; k < E; ++k) out[k] += e[k];
            }
            store_cols<T>(at<T>(a.dx, i, r) + col, out, left);
        }
    }
}

// The parameters' partial sums of such rows: a lane owns a group of columns and walks a slab of rows.  It runs before the input's gradient, which
// may be written over dy.
template <typename T> __global__ __launch_bounds__(256) void norm_slab_kernel(NormGradArgs a, int slabs) {
    constexpr int E = kPer<T>;
    const int64_t i = blockIdx.z, col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E, left = a.c - col;
    if (left <= 0) return;
    const int slab = blockIdx.y;
    const int64_t r0 = a.t * slab / slabs, r1 = a.t * (slab + 1) / slabs;
    float dg[E], db[E], x[E], dy[E];
#pragma unroll
    for (int k = 0; k < E; ++k) dg[k] = db[k] = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float m = a.mean[i * a.t + r], rs = a.rstd[i * a.t + r];
        widen<T>(load_cols(at<T>(a.x, i, r) + col, left), x);
        widen<T>(load_cols(at<T>(a.dy, i, r) + col, left), dy);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            dg[k] = __builtin_fmaf(dy[k], (x[k] - m) * rs, dg[k]);
            db[k] += dy[k];
        }
    }
    float* part = a.partial + (i * slabs + slab) * 2 * a.c;
#pragma unroll
    for (int k = 0; k < E; ++k)
        if (k < left) {
            part[col + k] = dg[k];
            part[a.c + col + k] = db[k];
        }
}

// Adds the slabs up: 64 columns a workgroup, the first of them 64 `first`, its sixteen wavefronts every sixteenth slab each.
constexpr int kSumWaves = 16;
template <typename G>
__global__ __launch_bounds__(kSumWaves* kWave) void norm_params_kernel(const float* partial, int64_t slabs, Vecs dgain, Vecs dbias, int64_t c, int64_t first) {
    __shared__ float rest[kSumWaves][kWave];
    const int64_t i = blockIdx.y, col = (first + blockIdx.x) * kWave + threadIdx.x % kWave;     // of 2 c: gain's, then bias's
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
    float sum = 0.0f;
    if (col < 2 * c) {
        const float* p = partial + i * slabs * 2 * c + col;
#pragma unroll 4
        for (int64_t s = w; s < slabs; s += kSumWaves) sum += p[s * 2 * c];
    }
    rest[w][l] = sum;
    __syncthreads();
    if (w == 0 && col < 2 * c) {
        float v = rest[0][l];
#pragma unroll
        for (int k = 1; k < kSumWaves; ++k) v += rest[k][l];
        if (col < c) {
            if (dgain.p) store_1(at<G>(dgain, i) + col, v);
        } else if (dbias.p) {
            store_1(at<G>(dbias, i) + (col - c), v);
        }
    }
}

// How a row of c columns is held: so many lanes, NV 16-byte groups each; none: not at all.
struct Hold {
    int lanes, nv;
};
inline Hold forward_hold(int64_t c, int bytes) {
    const int64_t groups = (c * bytes + 15) / 16;
    if (groups <= 16) return {16, 1};
    if (groups <= 32) return {32, 1};
    if (groups <= 64) return {64, 1};
    if (groups <= 128) return {64, 2};
    if (groups <= 256) return {64, 4};            // bf16 32 768 x 2048: 44.6 us, by 256 lanes 51.6; backward 120 / 114
    if (groups <= 512) return {256, 2};
    if (groups <= 1024) return {256, 4};
    if (groups <= 2048) return {1024, 2};
    if (groups <= 4096 && bytes == 4) return {1024, 4};
    return {0, 0};
}
inline Hold backward_hold(int64_t c, int bytes) {
    const Hold h = forward_hold(c, bytes);
    return h.lanes == 64 && h.nv == 4 ? Hold{256, 1} : h;
}

// Workgroups for each learner: enough rows at a time to fill the chip, no more than there are.
inline int64_t groups_per_learner(int64_t t, int rows, int n, int64_t chip) {
    const int64_t most = (t + rows - 1) / rows, fair = (chip + n - 1) / n;
    const int64_t g = most < fair ? most : fair;
    return g < 1 ? 1 : g;
}
// Slabs of the backward pass: two workgroups a compute unit, which leave as many partial rows behind; narrow rows, whose partial sums are little, as many as
// are resident; the widest one.  us, slabs of all learners 256 / 512 / 1024: bf16 32 768 x 2048 164 / 114 / 130, float 1024 x 16 384 54 / 64 / 83.
inline int64_t backward_slabs(int n, int64_t t, int64_t c, int bytes) {
    const Hold h = backward_hold(c, bytes);
    const int rows = h.lanes && h.lanes < 256 ? 256 / h.lanes : 1;
    const int64_t chip = h.lanes && h.lanes <= 64 && h.nv == 1 ? 2048 : h.lanes == 1024 ? 256 : 512;
    const int64_t g = groups_per_learner(t, rows, n, chip), turns = (t + rows - 1) / rows;
    return g > 64 && 4 * g > turns ? (turns > 256 ? turns / 4 : 64) : g;      // four turns each, or the sums cost more than the rows
}

inline Rows rows_of(const psgd_view* v) {
    return v ? Rows{static_cast<char*>(v->data), v->learner, v->row} : Rows{nullptr, 0, 0};
}
inline Vecs vecs_of(const psgd_view* v) { return v ? Vecs{static_cast<char*>(v->data), v->learner} : Vecs{nullptr, 0}; }

template <typename T, typename P> void launch_norm(const NormArgs& a, int n, int cus, hipStream_t s) {
    const Hold h = forward_hold(a.c, sizeof(T));
#define PSGD_NORM(L_, NV_)                                                                                                  \
    if (h.lanes == L_ && h.nv == NV_) {                                                                                     \
        const int64_t g = groups_per_learner(a.t, kGroupRows<L_>, n, (int64_t)cus * 2048 / kGroupThreads<L_>);              \
        hipLaunchKernelGGL((norm_kernel<T, P, L_, NV_>), dim3((unsigned)g, n), dim3(kGroupThreads<L_>), 0, s, a);           \
        return;                                                                                                             \
    }
    PSGD_NORM(16, 1) PSGD_NORM(32, 1) PSGD_NORM(64, 1) PSGD_NORM(64, 2) PSGD_NORM(64, 4) PSGD_NORM(256, 2) PSGD_NORM(256, 4) PSGD_NORM(1024, 2)
    if constexpr (sizeof(T) == 4) PSGD_NORM(1024, 4)
#undef PSGD_NORM
    const int64_t g = groups_per_learner(a.t, 1, n, (int64_t)cus * 2);
    hipLaunchKernelGGL((norm_long_kernel<T, P>), dim3((unsigned)g, n), dim3(1024), 0, s, a);
}

template <typename T, typename P, bool ADD> void launch_norm_grad(const NormGradArgs& a, int n, int slabs, hipStream_t s) {
    const Hold h = backward_hold(a.c, sizeof(T));
#define PSGD_NORM_GRAD(L_, NV_)                                                                                             \
    if (h.lanes == L_ && h.nv == NV_) {                                                                                     \
        const size_t lds = kGroupRows<L_> > 1 && a.partial ? (size_t)2 * NV_ * kPer<T> * L_ * sizeof(float) : 0;            \
        hipLaunchKernelGGL((norm_grad_kernel<T, P, L_, NV_, ADD>), dim3(slabs, n), dim3(kGroupThreads<L_>), lds, s, a);      \
        return;                                                                                                             \
    }
    PSGD_NORM_GRAD(16, 1) PSGD_NORM_GRAD(32, 1) PSGD_NORM_GRAD(64, 1) PSGD_NORM_GRAD(64, 2) PSGD_NORM_GRAD(256, 1) PSGD_NORM_GRAD(256, 2)
    PSGD_NORM_GRAD(256, 4) PSGD_NORM_GRAD(1024, 2)
    if constexpr (sizeof(T) == 4) PSGD_NORM_GRAD(1024, 4)
#undef PSGD_NORM_GRAD
    if (a.partial) {
        const int64_t across = (a.c + 256 * kPer<T> - 1) / (256 * kPer<T>);
        hipLaunchKernelGGL((norm_slab_kernel<T>), dim3((unsigned)across, slabs, n), dim3(256), 0, s, a, slabs);
    }
    hipLaunchKernelGGL((norm_grad_long_kernel<T, P, ADD>), dim3(slabs, n), dim3(1024), 0, s, a);
}

}  // namespace
}  // namespace psgd

extern "C" {

int psgd_layer_norm(const psgd_view* x, const psgd_view* gain, const psgd_view* bias, const psgd_view* y, float* mean, float* rstd, int n,
                    int64_t t, int64_t c, float eps, void* stream) {
    using namespace psgd;
    const char* name = "psgd_layer_norm";
    clear_error();
    if (!x || !gain || !y) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_counts(name, n, t, c)) return rc;
    if (!float_type(x->type) || y->type != x->type) return fail(PSGD_EINVAL, "%s: x and y must be float or bf16 alike", name);
    if (!float_type(gain->type) || (bias && bias->type != gain->type))
        return fail(PSGD_EINVAL, "%s: gain and bias must be float or bf16 alike", name);
    if ((mean == nullptr) != (rstd == nullptr)) return fail(PSGD_EINVAL, "%s: mean and rstd go together", name);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(PSGD_EINVAL, "%s: eps=%g", name, (double)eps);
    if (t == 0 || c == 0) return PSGD_OK;
    const Extent ex{"x", x, n, t, c}, ey{"y", y, n, t, c}, eg{"gain", gain, n, 1, c}, eb{"bias", bias ? bias : gain, n, 1, c};
    if (int rc = check_operand(name, ex, false)) return rc;
    if (int rc = check_operand(name, ey, true)) return rc;
    if (int rc = check_operand(name, eg, false)) return rc;
    if (int rc = check_operand(name, eb, false)) return rc;
    if (int rc = refuse_overlap(name, ey, ex, true)) return rc;
    for (const Extent* p : {&eg, &eb})
        if (int rc = refuse_overlap(name, ey, *p)) return rc;
    psgd_view vm, vr;
    if (mean) {
        const Extent em = flat("mean", mean, n * t, &vm), er = flat("rstd", rstd, n * t, &vr);
        if (int rc = check_operand(name, em, true)) return rc;
        if (int rc = check_operand(name, er, true)) return rc;
        if (int rc = refuse_overlap(name, em, er)) return rc;
        for (const Extent* e : {&em, &er})
            for (const Extent* o : {&ex, &ey, &eg, &eb})
                if (int rc = refuse_overlap(name, *e, *o)) return rc;
    }
    int cus = 0;
    if (int rc = compute_units(&cus)) return rc;
    const NormArgs a{rows_of(x), rows_of(y), vecs_of(gain), vecs_of(bias), mean, rstd, t, c, eps, (float)c};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (x->type == PSGD_F32) {
        if (gain->type == PSGD_F32) launch_norm<float, float>(a, n, cus, s);
        else launch_norm<float, uint16_t>(a, n, cus, s);
    } else {
        if (gain->type == PSGD_F32) launch_norm<uint16_t, float>(a, n, cus, s);
        else launch_norm<uint16_t, uint16_t>(a, n, cus, s);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

size_t psgd_layer_norm_grad_workspace(int n, int64_t t, int64_t c) {
    if (n < 1 || n > PSGD_MAX_N || t < 0 || c < 1 || t > INT32_MAX || c > INT32_MAX) return 0;
    // rows of the two types have different numbers of slabs; the larger serves either
    const int64_t a = psgd::backward_slabs(n, t, c, 2), b = psgd::backward_slabs(n, t, c, 4);
    return psgd::up256((size_t)n * (a > b ? a : b) * 2 * c * sizeof(float));
}

int psgd_layer_norm_grad(const psgd_view* dy, const psgd_view* x, const psgd_view* gain, const float* mean, const float* rstd,
                         const psgd_view* add, const psgd_view* dx, const psgd_view* dgain, const psgd_view* dbias, int n, int64_t t,
                         int64_t c, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace psgd;
    const char* name = "psgd_layer_norm_grad";
    clear_error();
    if (!dy || !x || !gain || !dx) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_counts(name, n, t, c)) return rc;
    if (!float_type(x->type) || dy->type != x->type || dx->type != x->type || (add && add->type != x->type))
        return fail(PSGD_EINVAL, "%s: dy, x, dx and add must be float or bf16 alike", name);
    if (!float_type(gain->type)) return fail(PSGD_EINVAL, "%s: gain must be float or bf16", name);
    const psgd_view* params = dgain ? dgain : dbias;
    if (params && (!float_type(params->type) || (dgain && dbias && dbias->type != dgain->type)))
        return fail(PSGD_EINVAL, "%s: dgain and dbias must be float or bf16 alike", name);
    if (c == 0) return PSGD_OK;
    if (t > 0 && (!mean || !rstd)) return fail(PSGD_EINVAL, "%s: mean and rstd are needed", name);
    const Extent edy{"dy", dy, n, t, c}, ex{"x", x, n, t, c}, edx{"dx", dx, n, t, c}, eadd{"add", add ? add : dy, n, t, c};
    const Extent eg{"gain", gain, n, 1, c};
    // what is not asked for has no column to overlap
    const Extent edg{"dgain", dgain ? dgain : gain, n, 1, dgain ? c : 0}, edb{"dbias", dbias ? dbias : gain, n, 1, dbias ? c : 0};
    psgd_view vm, vr, vw;
    const Extent em = flat("mean", mean, n * t, &vm), er = flat("rstd", rstd, n * t, &vr);
    const size_t need = params ? psgd_layer_norm_grad_workspace(n, t, c) : 0;
    const Extent ew = flat("the workspace", workspace, (int64_t)(need / 4), &vw);
    for (const Extent* e : {&edy, &ex, &eadd, &eg, &em, &er})
        if (int rc = check_operand(name, *e, false)) return rc;
    if (int rc = check_operand(name, edx, true)) return rc;
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256))
        return fail(PSGD_EINVAL, "%s: %zu bytes of workspace are needed, at a multiple of 256", name, need);
    if (int rc = refuse_overlap(name, edx, edy, true)) return rc;
    if (add)
        if (int rc = refuse_overlap(name, edx, eadd, true)) return rc;
    for (const Extent* e : {&ex, &eg, &em, &er})
        if (int rc = refuse_overlap(name, edx, *e)) return rc;
    for (const Extent* e : {&edg, &edb}) {
        if (int rc = check_operand(name, *e, true)) return rc;
        for (const Extent* o : {&edy, &ex, &eadd, &edx, &eg, &em, &er})
            if (int rc = refuse_overlap(name, *e, *o)) return rc;
    }
    if (dgain && dbias)
        if (int rc = refuse_overlap(name, edg, edb)) return rc;
    if (need) {
        for (const Extent* o : {&edy, &ex, &eadd, &edx, &eg, &edg, &edb, &em, &er})
            if (int rc = refuse_overlap(name, ew, *o)) return rc;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t slabs = backward_slabs(n, t, c, elem_bytes(x->type));
    const NormGradArgs a{rows_of(dy),   rows_of(x), rows_of(add), rows_of(dx), vecs_of(gain), mean, rstd,
                         params ? static_cast<float*>(workspace) : nullptr, t, c, 1.0f / (float)c};
    if (t > 0) {
#define PSGD_NORM_GRAD_TYPES(T, P)                                                                                          \
    if (add) launch_norm_grad<T, P, true>(a, n, (int)slabs, s);                                                             \
    else launch_norm_grad<T, P, false>(a, n, (int)slabs, s)
        if (x->type == PSGD_F32) {
            if (gain->type == PSGD_F32) PSGD_NORM_GRAD_TYPES(float, float);
            else PSGD_NORM_GRAD_TYPES(float, uint16_t);
        } else {
            if (gain->type == PSGD_F32) PSGD_NORM_GRAD_TYPES(uint16_t, float);
            else PSGD_NORM_GRAD_TYPES(uint16_t, uint16_t);
        }
#undef PSGD_NORM_GRAD_TYPES
    }
    if (params) {
        const int64_t count = t > 0 ? slabs : 0;
        auto sum = params->type == PSGD_F32 ? norm_params_kernel<float> : norm_params_kernel<uint16_t>;
        in_slices(parts_of(2 * c, kWave), [&](int64_t first, unsigned groups) {
            hipLaunchKernelGGL(sum, dim3(groups, n), dim3(kSumWaves * kWave), 0, s, a.partial, count, vecs_of(dgain), vecs_of(dbias), c, first);
        });
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

}  // extern "C"
