// What the learners' logits say of tokens (gfx950): log probabilities with entropy and top alternatives, and distillation from a teacher's
// top logits with its gradient.
//
// Both are softmax statistics of rows of v logits: m = max x, S = sum exp(x - m).  A logit costs 4 or 2 bytes to read and about ten vector
// operations (widen, maximum, difference, exponential at a quarter of the rate, sums), which on bf16 rows is close to what a compute unit does
// while its share of the HBM delivers them: so each row is read once, and nothing is computed twice where it is not also stored.
// A workgroup takes a row.  Statistics that need no second look at the row run online: a lane keeps the maximum of its logits so far and the
// sums relative to it, brought to a new maximum once a batch of four 16-byte groups; lanes are joined at the end.  The gradient needs the
// row again, and finds it in the workgroup's registers (up to 256 KB: 64 registers of each of 1024 lanes).
#include "psgd_rows.h"

namespace psgd {
namespace {

__device__ int g_token_status = 0;
constexpr int kTokenFlag = 2;            // bit 1 of psgd_device_status()

struct Rows {
    char* p;
    int64_t learner, row;
};
template <typename T> __device__ __forceinline__ T* at(const Rows& a, int64_t i, int64_t r) {
    return reinterpret_cast<T*>(a.p) + i * a.learner + r * a.row;
}
template <typename T> constexpr uint32_t kMasked = sizeof(T) == 4 ? 0xFF800000u : 0xFF80u;      // -inf

constexpr float kLog2E = 1.44269504088896341f;
constexpr float kNoLess = -200.0f;       // exp of it is 0 in float, and a product with it stays finite

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// Sums relative to a running maximum.  An empty one has m = -inf; differences that are not numbers (-inf from -inf) count as kNoLess.
struct Online {
    float m = -INFINITY, s = 0.0f, a = 0.0f;      // a: sum (x - m) exp(x - m)
    template <bool ENTROPY> __device__ __forceinline__ void move(float to) {
        const float d = fmaxf(m - to, kNoLess), f = exp_of(d);
        if (ENTROPY) a = f * __builtin_fmaf(d, s, a);
        s *= f;
        m = to;
    }
    template <bool ENTROPY> __device__ __forceinline__ void add(float x, float scale) {
        const float c = fmaxf(x - m, kNoLess), e = __builtin_amdgcn_exp2f(c * scale);
        s += e;
        if (ENTROPY) a = __builtin_fmaf(c, e, a);
    }
};

// Logits in ascending order as unsigned numbers: NaN above all, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
// Larger first, then lower place first.
__device__ __forceinline__ uint64_t rank_of(uint32_t order, uint32_t place) { return (uint64_t)order << 32 | (uint32_t)~place; }

template <typename T> __device__ __forceinline__ float largest(const float (&v)[kPer<T>]) {
    float a = Max::of(Max::of(v[0], v[1]), v[2]);
    if constexpr (kPer<T> == 4) return Max::of(a, v[3]);
    else return Max::of(Max::of(Max::of(a, v[3]), v[4]), Max::of(Max::of(v[5], v[6]), v[7]));
}

struct LogArgs {
    Rows logits, tokens;
    float *logp, *entropy, *top_logp;
    int32_t* top_idx;
    int k;
    int64_t t;
    int32_t v;
};

constexpr int kGroupsRanked = 256;       // groups of lanes whose largest logits give the threshold
constexpr int kCandidates = 2048;

// The k largest of a row, ties by ascending column.  Every lane knows the largest of its logits and the first 16-byte group that
// holds it.  Of kGroupsRanked groups of lanes the k-th best such pair is a threshold that at least k logits reach, and no logit
// outside of the lanes that reach it can be among the k: only those lanes look at their logits again and put what reaches the threshold
// into a list in LDS, whose members are ranked by counting.  Typically that is k lanes of 1024 and little more than k logits.  A row
// that overflows the list (long runs in order within one lane's groups) or holds NaN is searched k times instead.
template <typename T, int B>
__device__ void top_of_row(const LogArgs& a, const T* x, int64_t row, float best, uint32_t best_at, float m, float log_s, bool bad) {
    constexpr int E = kPer<T>;
    __shared__ uint64_t group[kGroupsRanked], list[kCandidates];
    __shared__ uint64_t limit, wave_best[B / kWave];
    __shared__ int count;
    const int tid = threadIdx.x;
    const uint32_t v = (uint32_t)a.v, groups = (v + E - 1) / E;      // 16-byte groups of the row: lane `tid` has tid, tid + B, ...
    const uint64_t own = (uint32_t)tid < groups ? rank_of(order_of(best), best_at) : rank_of(0, (uint32_t)tid);
    auto emit = [&](int place, uint64_t r) {
        const float z = logit_of((uint32_t)(r >> 32));
        a.top_idx[row * a.k + place] = (int32_t) ~(uint32_t)r;
        a.top_logp[row * a.k + place] = bad ? NAN : (m == -INFINITY ? -INFINITY : (z - m) - log_s);
    };
    bool listed = !bad;
    if (listed) {
        uint64_t g = own;
        constexpr int PART = B / kGroupsRanked;
#pragma unroll
        for (int d = 1; d < PART; d *= 2) {
            const uint64_t o = __shfl_xor((unsigned long long)g, d);
            g = o > g ? o : g;
        }
        if (tid % PART == 0) group[tid / PART] = g;
        if (tid == 0) count = 0;
        __syncthreads();
        int above = 0;
        const int from = tid % PART * (kGroupsRanked / PART);
#pragma unroll 8
        for (int j = 0; j < kGroupsRanked / PART; ++j) above += group[from + j] > g;
#pragma unroll
        for (int d = 1; d < PART; d *= 2) above += __shfl_xor(above, d);
        if (above == a.k - 1 && tid % PART == 0) limit = g;
        __syncthreads();
        const uint64_t lim = limit;
        const uint32_t lim_order = (uint32_t)(lim >> 32), lim_at = ~(uint32_t)lim;
        if (own >= lim && (uint32_t)tid < groups) {
            for (uint32_t q = tid; q < groups; q += B) {
                float z[E];
                widen<T>(load_cols(x + (int64_t)q * E, (int64_t)v - (int64_t)q * E, kMasked<T>), z);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t o = order_of(z[e]), col = q * E + e;
                    if (col < v && (o > lim_order || (o == lim_order && q <= lim_at))) {
                        const int p = atomicAdd(&count, 1);       // the order in the list does not matter
                        if (p < kCandidates) list[p] = rank_of(o, col);
                    }
                }
            }
        }
        __syncthreads();
        const int found = count;
        listed = found <= kCandidates;
        if (listed) {
            for (int c = tid; c < found; c += B) {
                const uint64_t r = list[c];
                int place = 0;
                for (int j = 0; j < found; ++j) place += list[j] > r;
                if (place < a.k) emit(place, r);
            }
        }
    }
    if (listed) return;
    uint64_t last = ~(uint64_t)0;
    for (int place = 0; place < a.k; ++place) {
        uint64_t most = 0;
        for (uint32_t q = tid; q < groups; q += B) {
            float z[E];
            widen<T>(load_cols(x + (int64_t)q * E, (int64_t)v - (int64_t)q * E, kMasked<T>), z);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t col = q * E + e;
                const uint64_t r = rank_of(order_of(z[e]), col);
                if (col < v && r < last && r > most) most = r;
            }
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const uint64_t o = __shfl_xor((unsigned long long)most, d);
            most = o > most ? o : most;
        }
        __syncthreads();
        if (tid % kWave == 0) wave_best[tid / kWave] = most;
        __syncthreads();
        most = wave_best[0];
        for (int w = 1; w < B / kWave; ++w) most = wave_best[w] > most ? wave_best[w] : most;
        if (tid == 0) emit(place, most);
        last = most;
    }
}

template <typename T, int B, bool ENTROPY, bool TOP> __global__ __launch_bounds__(B) void logprobs_kernel(LogArgs a) {
    constexpr int E = kPer<T>, U = 4, W = B / kWave;
    __shared__ float room[W], room2[2 * W];
    const int64_t row = blockIdx.x, i = row / a.t, r = row % a.t;
    const T* x = at<T>(a.logits, i, r);
    const int32_t v = a.v;
    const uint32_t tid = threadIdx.x, groups = ((uint32_t)v + E - 1) / E, whole = (uint32_t)v / E;
    Online o;
    float best = -INFINITY;
    uint32_t best_at = tid;
    auto batch = [&](const u32x4 (&raw)[U], uint32_t q) {
        float z[U][E], m = o.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            widen<T>(raw[u], z[u]);
            const float l = largest<T>(z[u]);
            if (TOP) {
                const bool up = l > best;
                best = up ? l : best;
                best_at = up ? q + u * B : best_at;
            }
            m = Max::of(m, l);
        }
        o.move<ENTROPY>(m);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) o.add<ENTROPY>(z[u][e], kLog2E);
    };
    uint32_t q = tid;
    for (; q + (U - 1) * B < whole; q += U * B) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_raw(x + (int64_t)(q + u * B) * E);
        batch(raw, q);
    }
    if (q < groups) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t col = (int64_t)(q + u * B) * E;
            raw[u] = load_cols(x + col, v - col, kMasked<T>);
        }
        batch(raw, q);
    }
    const float m = group_all<Max, W>(o.m, room);
    o.move<ENTROPY>(m);
    group_all_2<Sum, W>(o.s, o.a, room2);
    const bool bad = m != m || m == INFINITY, empty = m == -INFINITY;
    const float log_s = logf(o.s);
    if (tid == 0) {
        const int32_t token = *at<int32_t>(a.tokens, i, r);
        float lp = 0.0f;
        if (token >= v) {
            lp = NAN;
            atomicOr(&g_token_status, kTokenFlag);
        } else if (token >= 0) {
            lp = bad ? NAN : empty ? -INFINITY : (load_1(x + token) - m) - log_s;
        }
        a.logp[row] = lp;
        if (ENTROPY) a.entropy[row] = bad ? NAN : empty ? 0.0f : log_s - o.a / o.s;
    }
    if (TOP) top_of_row<T, B>(a, x, row, best, best_at, m, log_s, bad);
}

struct DistillArgs {
    Rows logits, idx, top, dlogits;
    const float* weight;
    float* loss;
    float tau, inv_tau;
    int k;
    int64_t t;
    int32_t v;
};

// What a lane keeps of its row stays as it was loaded: without this the compiler carries the widened values, twice the registers, from one pass to
// the next.
template <int N> __device__ __forceinline__ void stay_narrow(u32x4 (&raw)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(raw[j]));
}

// NV: groups of 16 bytes a lane keeps of the row, 0 for a row that is read again instead.
template <typename T, int B, int NV, bool GRAD> __global__ __launch_bounds__(B) void distill_kernel(DistillArgs a) {
    constexpr int E = kPer<T>, W = B / kWave, U = 4;
    __shared__ float room[W], room2[2][2 * W];
    extern __shared__ float slots[];
    float *p = slots, *z = slots + a.k;
    int32_t* at_col = reinterpret_cast<int32_t*>(slots + 2 * a.k);
    const int64_t row = blockIdx.x, i = row / a.t, r = row % a.t;
    const T* x = at<T>(a.logits, i, r);
    T* g = GRAD ? at<T>(a.dlogits, i, r) : nullptr;
    const int32_t v = a.v;
    const int tid = threadIdx.x;
    const int whole = v / E, cut = v % E;       // 16-byte groups of the row, and what is left behind them
    const float scale = a.inv_tau * kLog2E;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    bool off = weight == 0.0f;
    float amax = -INFINITY, m = -INFINITY;
    u32x4 raw[NV > 0 ? NV : 1];
    Online o;
    if (!off) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t masked = sizeof(T) == 4 ? kMasked<T> : kMasked<T> * 0x10001u;
                raw[j] = (u32x4){masked, masked, masked, masked};
                if (j * B + tid < whole) raw[j] = load_raw(x + (int64_t)(j * B + tid) * E);
            }
            if (cut) {
                const u32x4 part = load_raw_upto(x + (int64_t)whole * E, cut, kMasked<T>);      // of one lane, at a time of its own
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (j * B + tid == whole) raw[j] = part;
            }
        }
        for (int s = tid; s < a.k; s += B) {
            int32_t col = at<int32_t>(a.idx, i, r)[s];
            const float l = at<float>(a.top, i, r)[s] * a.inv_tau;
            if (col >= v) {
                atomicOr(&g_token_status, kTokenFlag);
                col = -1;
            }
            if (l == -INFINITY) col = -1;
            at_col[s] = col;
            p[s] = col >= 0 ? l : -INFINITY;
            z[s] = col >= 0 ? load_1(x + col) : 0.0f;
            amax = Max::of(amax, p[s]);
        }
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float c[E];
                widen<T>(raw[j], c);
                m = Max::of(m, largest<T>(c));
            }
        } else {
            for (int64_t col = (int64_t)tid * E; col < v; col += U * B * E) {
                float c[U][E];
                float to = o.m;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    widen<T>(load_cols(x + col + u * B * E, v - col - u * B * E, kMasked<T>), c[u]);
                    to = Max::of(to, largest<T>(c[u]));
                }
                const float f = __builtin_amdgcn_exp2f(fmaxf(o.m - to, -1e30f) * scale);
                o.s *= f;
                o.m = to;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) o.s += __builtin_amdgcn_exp2f(fmaxf(c[u][e] - to, -1e30f) * scale);
            }
            m = o.m;
        }
        group_all_2<Max, W>(m, amax, room2[0]);
        off = amax == -INFINITY;
    }
    if (off) {       // the whole workgroup: no weight, or no slot
        if (GRAD) {
            const float none[E] = {};
            for (int64_t col = (int64_t)tid * E; col < v; col += B * E) store_cols<T>(g + col, none, v - col);
        }
        if (tid == 0) a.loss[row] = 0.0f;
        return;
    }
    float sum = 0.0f, psum = 0.0f;
    if constexpr (NV > 0) {
        if (E == 8) stay_narrow(raw);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float c[E];
            widen<T>(raw[j], c);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f((c[e] - m) * scale);
        }
    } else {
        // a lane without logits has m = -inf and s = 0; a row of nothing but -inf has no distribution: NaN, as the formula has it
        sum = m == -INFINITY ? NAN : o.s * __builtin_amdgcn_exp2f(fmaxf(o.m - m, -1e30f) * scale);
        if (m == INFINITY) sum = NAN;
    }
    for (int s = tid; s < a.k; s += B)
        if (at_col[s] >= 0) psum += exp_of(p[s] - amax);
    group_all_2<Sum, W>(sum, psum, room2[1]);
    const float log_s = logf(sum), log_p = logf(psum), by_p = 1.0f / psum;
    float loss = 0.0f;
    for (int s = tid; s < a.k; s += B) {
        if (at_col[s] < 0) {
            p[s] = 0.0f;
            continue;
        }
        const float l = p[s] - amax, q = exp_of(l) * by_p;
        if (q != 0.0f) loss += q * ((l - log_p) - ((z[s] - m) * a.inv_tau - log_s));
        p[s] = q;
    }
    loss = group_all<Sum, W>(loss, room);
    if (tid == 0) a.loss[row] = weight * a.tau * a.tau * loss;
    if constexpr (GRAD) {
        const float share = weight * a.tau / sum;
        if constexpr (NV > 0) {
            u32x4 part = {};
            if (E == 8) stay_narrow(raw);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float c[E];
                widen<T>(raw[j], c);
#pragma unroll
                for (int e = 0; e < E; ++e) c[e] = __builtin_amdgcn_exp2f((c[e] - m) * scale) * share;
                const u32x4 out = narrow(c, T{});
                if (j * B + tid < whole) *reinterpret_cast<u32x4_any*>(g + (int64_t)(j * B + tid) * E) = out;
                if (j * B + tid == whole) part = out;
            }
            if (cut && tid == whole % B) {
                float c[E];
                widen<T>(part, c);
                store_cols<T>(g + (int64_t)whole * E, c, cut);
            }
        } else {
            for (int64_t col = (int64_t)tid * E; col < v; col += B * E) {
                float c[E];
                widen<T>(load_cols(x + col, v - col, kMasked<T>), c);
#pragma unroll
                for (int e = 0; e < E; ++e) c[e] = __builtin_amdgcn_exp2f((c[e] - m) * scale) * share;
                store_cols<T>(g + col, c, v - col);
            }
        }
        __syncthreads();          // the teacher's columns are written once more, with the whole value, so that it is rounded once
        for (int s = tid; s < a.k; s += B) {
            const int32_t col = at_col[s];
            if (col < 0) continue;
            float given = 0.0f;
            for (int j = 0; j < a.k; ++j) given += at_col[j] == col ? p[j] : 0.0f;
            store_1(g + col, __builtin_amdgcn_exp2f((z[s] - m) * scale) * share - weight * a.tau * given);
        }
    }
}

inline Rows rows_of(const psgd_view* v) {
    return v ? Rows{static_cast<char*>(v->data), v->learner, v->row} : Rows{nullptr, 0, 0};
}

template <typename T> void launch_logprobs(const LogArgs& a, int64_t rows, hipStream_t s) {
#define PSGD_LOG(B, EN, TOP) hipLaunchKernelGGL((logprobs_kernel<T, B, EN, TOP>), dim3((unsigned)rows), dim3(B), 0, s, a)
#define PSGD_LOG_B(B)                                                                                                       \
    do {                                                                                                                    \
        if (a.entropy && a.k) PSGD_LOG(B, true, true);                                                                      \
        else if (a.entropy) PSGD_LOG(B, true, false);                                                                       \
        else if (a.k) PSGD_LOG(B, false, true);                                                                             \
        else PSGD_LOG(B, false, false);                                                                                     \
    } while (0)
    if (a.v > 256 * 16 * kPer<T>) PSGD_LOG_B(1024);
    else PSGD_LOG_B(256);
#undef PSGD_LOG_B
#undef PSGD_LOG
}

template <typename T> void launch_distill(const DistillArgs& a, int64_t rows, hipStream_t s) {
    const size_t lds = (size_t)a.k * 12;
#define PSGD_DISTILL(B, NV, GRAD) hipLaunchKernelGGL((distill_kernel<T, B, NV, GRAD>), dim3((unsigned)rows), dim3(B), lds, s, a)
    const int64_t groups = ((int64_t)a.v + kPer<T> - 1) / kPer<T>;
    if (!a.dlogits.p) {
        if (groups > 256 * 16) PSGD_DISTILL(1024, 0, false);
        else PSGD_DISTILL(256, 0, false);
    } else if (groups <= 256) PSGD_DISTILL(256, 1, true);
    else if (groups <= 256 * 2) PSGD_DISTILL(256, 2, true);
    else if (groups <= 256 * 4) PSGD_DISTILL(256, 4, true);
    else if (groups <= 256 * 8) PSGD_DISTILL(256, 8, true);
    else if (groups <= 1024 * 4) PSGD_DISTILL(1024, 4, true);
    else if (groups <= 1024 * 8) PSGD_DISTILL(1024, 8, true);
    else if (groups <= 1024 * 16) PSGD_DISTILL(1024, 16, true);
    else PSGD_DISTILL(1024, 0, true);
#undef PSGD_DISTILL
}

inline int check_rows(const char* name, int n, int64_t t, int64_t v) {
    if (int rc = check_counts(name, n, t, v)) return rc;
    if (v < 1) return fail(PSGD_EINVAL, "%s: a row has no column", name);
    if ((int64_t)n * t > INT32_MAX) return fail(PSGD_EINVAL, "%s: n * t beyond 2^31 - 1", name);
    return PSGD_OK;
}

}  // namespace

int token_status(int clear, int* word) {
    hipError_t e = hipMemcpyFromSymbol(word, HIP_SYMBOL(g_token_status), sizeof(int));
    if (e != hipSuccess) return hip_error(e, "hipMemcpyFromSymbol");
    if (clear && *word) {
        const int zero = 0;
        e = hipMemcpyToSymbol(HIP_SYMBOL(g_token_status), &zero, sizeof(int));
        if (e != hipSuccess) return hip_error(e, "hipMemcpyToSymbol");
    }
    return PSGD_OK;
}

}  // namespace psgd

extern "C" {

size_t psgd_token_logprobs_workspace(int n, int64_t t, int64_t v, int k) {
    (void)n;
    (void)t;
    (void)v;
    (void)k;
    return 0;
}

int psgd_token_logprobs(const psgd_view* logits, const psgd_view* tokens, float* logp, float* entropy, float* top_logp, int32_t* top_idx,
                        int k, int n, int64_t t, int64_t v, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace psgd;
    const char* name = "psgd_token_logprobs";
    clear_error();
    (void)workspace;
    (void)workspace_bytes;
    if (!logits || !tokens) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_rows(name, n, t, v)) return rc;
    if (!float_type(logits->type) || tokens->type != PSGD_I32) return fail(PSGD_EINVAL, "%s: logits must be float or bf16, tokens int32", name);
    if (k < 0 || k > PSGD_MAX_TOP || k > v) return fail(PSGD_EINVAL, "%s: k=%d outside 0..min(v, %d)", name, k, (int)PSGD_MAX_TOP);
    if (t == 0) return PSGD_OK;
    if (!logp || (k > 0) != (top_logp != nullptr) || (k > 0) != (top_idx != nullptr))
        return fail(PSGD_EINVAL, "%s: logp is needed, top_logp and top_idx go with k > 0", name);
    const Extent el{"logits", logits, n, t, v}, et{"tokens", tokens, n, t, 1};
    if (int rc = check_operand(name, el, false)) return rc;
    if (int rc = check_operand(name, et, false)) return rc;
    psgd_view room[4];
    const int64_t rows = n * t;
    const Extent outs[4] = {flat("logp", logp, rows, &room[0]), flat("entropy", entropy, entropy ? rows : 0, &room[1]),
                            flat("top_logp", top_logp, rows * k, &room[2]), flat("top_idx", top_idx, rows * k, &room[3], PSGD_I32)};
    for (int p = 0; p < 4; ++p) {
        if (int rc = check_operand(name, outs[p], true)) return rc;
        if (int rc = refuse_overlap(name, outs[p], el)) return rc;
        if (int rc = refuse_overlap(name, outs[p], et)) return rc;
        for (int q = 0; q < p; ++q)
            if (int rc = refuse_overlap(name, outs[p], outs[q])) return rc;
    }
    const LogArgs a{rows_of(logits), rows_of(tokens), logp, entropy, top_logp, top_idx, k, t, (int32_t)v};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (logits->type == PSGD_F32) launch_logprobs<float>(a, rows, s);
    else launch_logprobs<uint16_t>(a, rows, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

int psgd_distill(const psgd_view* logits, const psgd_view* top_idx, const psgd_view* top_logit, const float* weight, float* loss,
                 const psgd_view* dlogits, float tau, int k, int n, int64_t t, int64_t v, void* stream) {
    using namespace psgd;
    const char* name = "psgd_distill";
    clear_error();
    if (!logits || !top_idx || !top_logit) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_rows(name, n, t, v)) return rc;
    if (!float_type(logits->type) || (dlogits && dlogits->type != logits->type))
        return fail(PSGD_EINVAL, "%s: logits and dlogits must be float or bf16 alike", name);
    if (top_idx->type != PSGD_I32 || top_logit->type != PSGD_F32) return fail(PSGD_EINVAL, "%s: top_idx must be int32, top_logit float", name);
    if (k < 1 || k > PSGD_MAX_SLOTS) return fail(PSGD_EINVAL, "%s: k=%d outside 1..%d", name, k, (int)PSGD_MAX_SLOTS);
    if (!(tau > 0.0f) || !std::isfinite(tau) || !std::isfinite(1.0f / tau)) return fail(PSGD_EINVAL, "%s: tau=%g", name, (double)tau);
    if (t == 0) return PSGD_OK;
    if (!loss) return fail(PSGD_EINVAL, "%s: loss is needed", name);
    const int64_t rows = n * t;
    psgd_view rw, rl;
    const Extent el{"logits", logits, n, t, v}, ei{"top_idx", top_idx, n, t, k}, et{"top_logit", top_logit, n, t, k};
    const Extent ew = flat("weight", weight, weight ? rows : 0, &rw), eo = flat("loss", loss, rows, &rl);
    for (const Extent* e : {&el, &ei, &et, &ew})
        if (int rc = check_operand(name, *e, false)) return rc;
    if (int rc = check_operand(name, eo, true)) return rc;
    for (const Extent* e : {&el, &ei, &et, &ew})
        if (int rc = refuse_overlap(name, eo, *e)) return rc;
    if (dlogits) {
        const Extent eg{"dlogits", dlogits, n, t, v};
        if (int rc = check_operand(name, eg, true)) return rc;
        if (int rc = refuse_overlap(name, eg, el, true)) return rc;
        for (const Extent* e : {&ei, &et, &ew, &eo})
            if (int rc = refuse_overlap(name, eg, *e)) return rc;
    }
    const DistillArgs a{rows_of(logits), rows_of(top_idx), rows_of(top_logit), rows_of(dlogits), weight, loss, tau, 1.0f / tau, k, t, (int32_t)v};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (logits->type == PSGD_F32) launch_distill<float>(a, rows, s);
    else launch_distill<uint16_t>(a, rows, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

}  // extern "C"
