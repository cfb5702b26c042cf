// What the learners' logits say of tokens (gfx950): log probabilities with entropy and top alternatives, and distillation from a teacher's
// top logits with its gradient.
//
// Both are softmax statistics of rows of v logits: m = max x, S = sum exp(x - m).  A logit costs 4 or 2 bytes to read and about ten vector
// operations (widen, maximum, difference, exponential at a quarter of the rate, sums), which on bf16 rows is close to what a compute unit does
// while its share of the HBM delivers them: so each row is read once, and nothing is computed twice where it is not also stored.
// A workgroup takes a row.  Statistics that need no second look at the row run online: a lane keeps the maximum of its logits so far and the
// sums relative to it, brought to a new maximum once a batch of four 16-byte groups; lanes are joined at the end.  The gradient needs the
// row again, and finds it in the workgroup's registers (up to 256 KB: 64 registers of each of 1024 lanes).
//
// Measured: log probabilities, entropy and 20 alternatives of 4096 rows of 32 000 floats 119 us (524 MB, 4.4 TB/s), of one row of 131 072 bf16 with 8
// alternatives 15 (one compute unit reads it, then the search); distillation of 8192 rows of 131 072 bf16 880 us (4.3 GB, 4.9 TB/s; a copy of that
// size reaches 4.74), of 592 rows of 10 007 floats 12.8; its loss alone of 2048 rows of 131 072 bf16 90 (537 MB, 6.0 TB/s).  Rows that no workgroup's
// registers hold, beyond 131 072 bf16 or 65 536 floats, are read twice for the gradient: 2048 rows of 200 000 bf16 434 us, 3.8 TB/s of what they cannot do
// without.
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

// 2^x of a difference that is at most 0, zero where it is not a number (-inf from -inf).
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(fmaxf(x, kNoLess)); }
// The product's rounding is |x| 2^-24 of the exponential, as much as the difference of two logits that x is: where it enters sums, of terms that are at
// most 0.37 / |x|; where it is an output, the gradient's q, no more than its logit was known to.
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

template <int B> constexpr int kRowsOf = rows_of_group(B);
// Between the lanes of a row.  A wavefront's own accesses to LDS are in order, so there only the compiler has to keep them.
template <int B> __device__ __forceinline__ void row_sync() {
    if constexpr (B == kWave) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

struct LogArgs {
    Rows logits, tokens;
    float *logp, *entropy, *top_logp;
    int32_t* top_idx;
    int k, keep;            // keep: floats of LDS for a row's batches' maxima, 0 if they do not fit
    int64_t t, rows, first;      // first: the row this launch begins with
    int32_t v;
};

// What finding the k largest takes of LDS, for rows of B lanes.  Lanes are joined to at most 256 groups.
template <int B> struct TopRoom {
    static constexpr int GROUPS = B < 256 ? B : 256, LIST = B < 256 ? 512 : B < 1024 ? 1024 : 2048;
    static constexpr int BATCHES = B < 256 ? 128 : 256;
    uint64_t group[GROUPS], list[LIST], best[B / kWave];
    uint32_t batch[BATCHES];         // first 16-byte groups of the batches to read again
    uint64_t limit;
    int count, batches;
};
// The k largest of a row, ties by ascending column.  Every lane knows the largest of its logits and the first 16-byte group that
// holds it, and in LDS the largest of each of its batches.  Of up to 256 groups of lanes the k-th best is a threshold that at least k logits
// reach, and no logit outside of the batches that reach it can be among the k: only those are read again, all lanes' at once, and what
// reaches the threshold goes into a list in LDS, whose members are ranked by counting.  Typically that is k batches and little more than k
// logits.  A row that overflows the list (long runs in order within one lane's groups) or holds NaN is searched k times instead.
// (Before the batches' maxima were kept, and with the threshold by counting in every lane, this took as long as reading the row: 4096 rows of 32 000
// floats 158 us, 84 without it.)
template <typename T, int B, typename EMIT>
__device__ void top_of_row(const LogArgs& a, TopRoom<B>& room, const float* batch_max, const T* x, uint32_t v, float m, float best, uint32_t best_at, bool bad,
                           const EMIT& emit) {
    constexpr int E = kPer<T>, U = kUnroll, GROUPS = TopRoom<B>::GROUPS, PART = B / GROUPS;
    const int tid = threadIdx.x % B;
    const uint32_t groups = (v + E - 1) / E;      // 16-byte groups of the row: lane `tid` has tid, tid + B, ...
    bool listed = !bad;
    if (listed) {
        uint64_t g = (uint32_t)tid < groups ? rank_of(order_of(best), best_at) : rank_of(0, (uint32_t)tid);
#pragma unroll
        for (int d = 1; d < PART; d *= 2) {
            const uint64_t o = __shfl_xor((unsigned long long)g, d);
            g = o > g ? o : g;
        }
        if (tid % PART == 0) room.group[tid / PART] = g;
        if (tid == 0) room.count = room.batches = 0;
        row_sync<B>();
        if (tid < kWave) {
            // one wavefront: the largest order that k groups reach, bit by bit, and no further than to a few more than k
            constexpr int HELD = GROUPS / kWave;
            uint32_t o[HELD];
#pragma unroll
            for (int h = 0; h < HELD; ++h) o[h] = (uint32_t)(room.group[h * kWave + tid] >> 32);
            uint32_t t = 0;
            int reach = GROUPS;
            const uint32_t top = order_of(m);
            for (uint32_t bit = 0x80000000u; bit && reach > a.k + 8; bit >>= 1) {
                if ((t | bit) > top) continue;                 // nobody
                int c = 0;
#pragma unroll
                for (int h = 0; h < HELD; ++h) c += __popcll(__ballot(o[h] >= (t | bit)));
                if (c >= a.k) {
                    t |= bit;
                    reach = c;
                }
            }
            uint64_t lim = (uint64_t)t << 32;                  // every place
            if (reach > 2 * a.k + 16) {                        // equal ones: the k-th with its place
                for (int h = 0; h < HELD; ++h) {
                    const uint64_t mine = room.group[h * kWave + tid];
                    int above = 0;
                    for (int j = 0; j < GROUPS; ++j) above += room.group[j] > mine;
                    if (above == a.k - 1) room.limit = mine;
                }
            } else if (tid == 0) {
                room.limit = lim;
            }
        }
        row_sync<B>();
        const uint64_t lim = room.limit;
        const uint32_t lim_order = (uint32_t)(lim >> 32), lim_at = ~(uint32_t)lim, whole = v / E;
        // the threshold as a logit: there is no NaN here, and below -inf's order there is nothing
        const float lim_logit = lim_order <= order_of(-INFINITY) ? -INFINITY : logit_of(lim_order);
        auto look = [&](uint32_t q) {
            u32x4 raw[U];
            if (q + (U - 1) * B < whole) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = load_raw(x + (int64_t)(q + u * B) * E);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t col = (int64_t)(q + u * B) * E;
                    raw[u] = load_cols(x + col, v - col, kMasked<T>);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t at = q + u * B;
                float z[E];
                widen<T>(raw[u], z);
                if (at >= groups || !(largest<T>(z) >= lim_logit)) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t o = order_of(z[e]), col = at * E + e;
                    if (z[e] >= lim_logit && (o > lim_order || at <= lim_at) && col < v) {
                        const int p = atomicAdd(&room.count, 1);       // the order in the list does not matter
                        if (p < TopRoom<B>::LIST) room.list[p] = rank_of(o, col);
                    }
                }
            }
        };
        // The batches are listed first, so that all of them are read at once: a wavefront that reads as it finds them waits for each.
        bool all = batch_max == nullptr;
        if (!all) {
            int b = 0;
            for (uint32_t q = tid; q < groups; q += U * B, ++b) {
                if (!(batch_max[b * B + tid] >= lim_logit)) continue;
                const int p = atomicAdd(&room.batches, 1);
                if (p < TopRoom<B>::BATCHES) room.batch[p] = q;
            }
            row_sync<B>();
            const int listed_batches = room.batches;
            all = listed_batches > TopRoom<B>::BATCHES;
            if (!all)
                for (int p = tid; p < listed_batches; p += B) look(room.batch[p]);
        }
        if (all)
            for (uint32_t q = tid; q < groups; q += U * B) look(q);
        row_sync<B>();
        const int found = room.count;
        listed = found <= TopRoom<B>::LIST;
        if (listed) {
            for (int c = tid; c < found; c += B) {
                const uint64_t r = room.list[c];
                int place = 0;
#pragma unroll 8
                for (int j = 0; j < found; ++j) place += room.list[j] > r;
                if (place < a.k) emit(place, r);
            }
        }
    }
    if (listed) return;
    uint64_t last = 0;               // of the place before; the first takes any: NaN in column 0 has the largest rank there is
    for (int place = 0; place < a.k; ++place) {
        uint64_t most = 0;
        for (uint32_t q = tid; q < groups; q += B) {
            float z[E];
            widen<T>(load_cols(x + (int64_t)q * E, (int64_t)v - (int64_t)q * E, kMasked<T>), z);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t col = q * E + e;
                const uint64_t r = rank_of(order_of(z[e]), col);
                if (col < v && (place == 0 || r < last) && r > most) most = r;
            }
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const uint64_t o = __shfl_xor((unsigned long long)most, d);
            most = o > most ? o : most;
        }
        row_sync<B>();
        if (tid % kWave == 0) room.best[tid / kWave] = most;
        row_sync<B>();
        most = room.best[0];
        for (int w = 1; w < B / kWave; ++w) most = room.best[w] > most ? room.best[w] : most;
        if (tid == 0) emit(place, most);
        last = most;
    }
}

// What a row's statistics say, once they are whole.
struct Said {
    float m, s, a, log_s;
    bool bad, empty;
    __device__ __forceinline__ Said(float m_, float s_, float a_)
        : m(m_), s(s_), a(a_), log_s(logf(s_)), bad(m_ != m_ || m_ == INFINITY), empty(m_ == -INFINITY) {}
    __device__ __forceinline__ float of(float z) const { return bad ? NAN : empty ? -INFINITY : (z - m) - log_s; }
    __device__ __forceinline__ float entropy() const { return bad ? NAN : empty ? 0.0f : log_s - a / s; }
};
template <typename T, int B, bool ENTROPY, bool TOP> __global__ __launch_bounds__(B * kRowsOf<B>) void logprobs_kernel(LogArgs a) {
    constexpr int E = kPer<T>, U = kUnroll, W = B / kWave, ROWS = kRowsOf<B>;
    __shared__ float room[W], room2[2 * W];
    extern __shared__ float batches[];               // TOP: [row][batch][B], if a.keep says that they fit
    const int slot = ROWS > 1 ? threadIdx.x / B : 0;
    const int64_t row = a.first + (int64_t)blockIdx.x * ROWS + slot;
    if (ROWS > 1 && row >= a.rows) return;
    const int64_t i = row / a.t, r = row % a.t;
    const T* x = at<T>(a.logits, i, r);
    const int32_t v = a.v;
    float* batch_max = batches + slot * a.keep;
    const uint32_t tid = threadIdx.x % B, groups = ((uint32_t)v + E - 1) / E, whole = (uint32_t)v / E;
    Online o;
    float best = -INFINITY;
    uint32_t best_at = tid;
    float* mine = TOP && a.keep ? batch_max + tid : nullptr;
    auto batch = [&](const u32x4 (&raw)[U], uint32_t q) {
        float z[U][E], m = -INFINITY;
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
        if (TOP && mine) {
            *mine = m;
            mine += B;
        }
        o.move<ENTROPY>(Max::of(o.m, m));
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
    const Said said(m, o.s, o.a);
    if (tid == 0) {
        const int32_t token = *at<int32_t>(a.tokens, i, r);
        float lp = 0.0f;
        if (token >= v) {
            lp = NAN;
            atomicOr(&g_token_status, kTokenFlag);
        } else if (token >= 0) {
            lp = said.of(load_1(x + token));
        }
        a.logp[row] = lp;
        if (ENTROPY) a.entropy[row] = said.entropy();
    }
    if constexpr (TOP) {
        __shared__ TopRoom<B> top[ROWS];
        top_of_row<T, B>(a, top[slot], a.keep ? batch_max : nullptr, x, (uint32_t)v, m, best, best_at, said.bad, [&](int place, uint64_t rank) {
            a.top_idx[row * a.k + place] = (int32_t) ~(uint32_t)rank;
            a.top_logp[row * a.k + place] = said.of(logit_of((uint32_t)(rank >> 32)));
        });
    }
}

struct DistillArgs {
    Rows logits, idx, top, dlogits;
    const float* weight;
    float* loss;
    float tau, inv_tau;
    int k;
    int64_t t, rows, first;      // first: the row this launch begins with
    int32_t v;
};

// What a lane keeps of its row stays as it was loaded: without this the compiler carries the widened values, twice the registers, from one pass to
// the next.
template <int N> __device__ __forceinline__ void stay_narrow(u32x4 (&raw)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(raw[j]));
}

// NV: groups of 16 bytes a lane keeps of the row, 0 for a row that is read again instead.
template <typename T, int B, int NV, bool GRAD> __global__ __launch_bounds__(B * kRowsOf<B>) void distill_kernel(DistillArgs a) {
    constexpr int E = kPer<T>, W = B / kWave, U = 4, ROWS = kRowsOf<B>;
    __shared__ float room[W], room2[2][2 * W];
    extern __shared__ float slots[];                 // of each row: p, z and the columns
    const int slot = ROWS > 1 ? threadIdx.x / B : 0;
    const int64_t row = a.first + (int64_t)blockIdx.x * ROWS + slot;
    if (ROWS > 1 && row >= a.rows) return;
    const int64_t i = row / a.t, r = row % a.t;
    float *p = slots + slot * 3 * a.k, *z = p + a.k;
    int32_t* at_col = reinterpret_cast<int32_t*>(p + 2 * a.k);
    const T* x = at<T>(a.logits, i, r);
    T* g = GRAD ? at<T>(a.dlogits, i, r) : nullptr;
    const int32_t v = a.v;
    const int tid = threadIdx.x % B;
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
            const float l = at<float>(a.top, i, r)[s];       // divided by tau once the maximum is off: alone it may leave float
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
                const float f = exp_below((o.m - to) * scale);
                o.s *= f;
                o.m = to;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) o.s += exp_below((c[u][e] - to) * scale);
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
        sum = m == -INFINITY ? NAN : o.s * exp_below((o.m - m) * scale);
        if (m == INFINITY) sum = NAN;
    }
    for (int s = tid; s < a.k; s += B)
        if (at_col[s] >= 0) psum += exp_of((p[s] - amax) * a.inv_tau);
    group_all_2<Sum, W>(sum, psum, room2[1]);
    const float log_s = logf(sum), log_p = logf(psum), by_p = 1.0f / psum;
    float loss = 0.0f;
    for (int s = tid; s < a.k; s += B) {
        if (at_col[s] < 0) {
            p[s] = 0.0f;
            continue;
        }
        const float l = (p[s] - amax) * a.inv_tau, q = exp_of(l) * by_p;
        // tau (log p - log q): neither difference is divided by tau, with which it may leave float
        if (q != 0.0f) loss += q * (((p[s] - amax) - (z[s] - m)) + a.tau * (log_s - log_p));
        p[s] = q;
    }
    loss = group_all<Sum, W>(loss, room);
    if (tid == 0) a.loss[row] = weight * a.tau * loss;
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
        row_sync<B>();            // the teacher's columns are written once more, with the whole value, so that it is rounded once
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

template <typename T> int launch_logprobs(LogArgs a, int cus, hipStream_t s) {
    const int64_t groups = ((int64_t)a.v + kPer<T> - 1) / kPer<T>;
    const int lanes = lanes_of_row(a.rows, groups, a.k, cus);
#define PSGD_LOG(B, EN, TOP)                                                                                                \
    do {                                                                                                                    \
        if (B == 1024 && TOP && lds > 40 * 1024) {                                                                          \
            static LdsRecord record;                                                                                        \
            if (int rc = allow_lds(reinterpret_cast<const void*>(logprobs_kernel<T, B, EN, TOP>), batch_room(B), record)) return rc; \
        }                                                                                                                   \
        in_slices(parts_of(a.rows, kRowsOf<B>), [&](int64_t first, unsigned count) {                                        \
            a.first = first * kRowsOf<B>;                                                                                   \
            hipLaunchKernelGGL((logprobs_kernel<T, B, EN, TOP>), dim3(count), dim3(B * kRowsOf<B>), lds, s, a);             \
        });                                                                                                                 \
    } while (0)
#define PSGD_LOG_B(B)                                                                                                       \
    do {                                                                                                                    \
        a.keep = a.k > 0 ? batches_kept(groups, B) : 0;                                                                     \
        const size_t lds = (size_t)a.keep * kRowsOf<B> * sizeof(float);                                                     \
        if (a.entropy && a.k) PSGD_LOG(B, true, true);                                                                      \
        else if (a.entropy) PSGD_LOG(B, true, false);                                                                       \
        else if (a.k) PSGD_LOG(B, false, true);                                                                             \
        else PSGD_LOG(B, false, false);                                                                                     \
    } while (0)
    if (lanes == 1024) PSGD_LOG_B(1024);
    else if (lanes == 256) PSGD_LOG_B(256);
    else PSGD_LOG_B(64);
#undef PSGD_LOG_B
#undef PSGD_LOG
    return PSGD_OK;
}

template <typename T> void launch_distill(DistillArgs a, int cus, hipStream_t s) {
    const DistillHold h = distill_hold(a.rows, ((int64_t)a.v + kPer<T> - 1) / kPer<T>, a.dlogits.p, cus);
#define PSGD_DISTILL(B, NV, GRAD)                                                                                           \
    if (h.lanes == B && h.held == NV && (a.dlogits.p != nullptr) == GRAD)                                                   \
    in_slices(parts_of(a.rows, kRowsOf<B>), [&](int64_t first, unsigned count) {                                            \
        a.first = first * kRowsOf<B>;                                                                                       \
        hipLaunchKernelGGL((distill_kernel<T, B, NV, GRAD>), dim3(count), dim3(B * kRowsOf<B>), (size_t)a.k * 12 * kRowsOf<B>, s, a); \
    })
    PSGD_DISTILL(64, 0, false);
    PSGD_DISTILL(256, 0, false);
    PSGD_DISTILL(1024, 0, false);
    PSGD_DISTILL(64, 1, true);
    PSGD_DISTILL(64, 2, true);
    PSGD_DISTILL(64, 4, true);
    PSGD_DISTILL(256, 2, true);
    PSGD_DISTILL(256, 4, true);
    PSGD_DISTILL(256, 8, true);
    PSGD_DISTILL(256, 16, true);
    PSGD_DISTILL(1024, 4, true);
    PSGD_DISTILL(1024, 8, true);
    PSGD_DISTILL(1024, 16, true);
    PSGD_DISTILL(1024, 0, true);
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

int psgd_token_logprobs(const psgd_view* logits, const psgd_view* tokens, float* logp, float* entropy, float* top_logp, int32_t* top_idx,
                        int k, int n, int64_t t, int64_t v, void* stream) {
    using namespace psgd;
    const char* name = "psgd_token_logprobs";
    clear_error();
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
    int cus = 0;
    if (int rc = compute_units(&cus)) return rc;
    const LogArgs a{rows_of(logits), rows_of(tokens), logp, entropy, top_logp, top_idx, k, 0, t, rows, 0, (int32_t)v};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (int rc = logits->type == PSGD_F32 ? launch_logprobs<float>(a, cus, s) : launch_logprobs<uint16_t>(a, cus, s)) return rc;
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
    if (!(tau > 0.0f) || !std::isfinite(tau) || !std::isfinite(1.0f / tau * kLog2E)) return fail(PSGD_EINVAL, "%s: tau=%g", name, (double)tau);
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
    int cus = 0;
    if (int rc = compute_units(&cus)) return rc;
    const DistillArgs a{rows_of(logits), rows_of(top_idx), rows_of(top_logit), rows_of(dlogits), weight, loss, tau, 1.0f / tau, k, t, rows, 0, (int32_t)v};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (logits->type == PSGD_F32) launch_distill<float>(a, cus, s);
    else launch_distill<uint16_t>(a, cus, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}

}  // extern "C"
