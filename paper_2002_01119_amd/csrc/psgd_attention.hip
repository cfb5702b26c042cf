// Causal attention in packed sequences, with a sliding window and first tokens that stay visible, forward and backward (gfx950).
//
//     s_ij = scale q_i . k_j,   p_ij = exp(s_ij - lse_i),   o_i = sum_j p_ij v_j
//     D_i = do_i . o_i,   ds_ij = p_ij (do_i . v_j - D_i),   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i
//
// Forward a workgroup owns a tile of one head's queries and walks the keys that they see, a tile at a time, with the running maximum and sum of the
// softmax; the wavefronts share the tile in LDS and own 16 or 32 queries each.  Scores are computed as keys times queries, so a lane has four
// keys of one query: maximum, sum and scale of a query are a lane's own, and the exponentials are the next product's operand as they stand.  Two products,
// 4 pairs head operations.
//
// Backward in two kernels, so that every sum has one owner and a fixed order: the first owns queries and makes dq (and D, which the second reads), the second owns keys, walks
// the queries that see them, of all heads that share the key head, and makes dk and dv.  Both compute s and p again from lse: seven products, of which five are
// what the gradients cannot do without.
//
// A tile never reaches beyond its sequence: rows there are read as zero.
#include "psgd_attention_core.h"

#include <algorithm>

namespace psgd {
namespace {

__device__ int g_attention_status = 0;
constexpr int kAttentionFlag = 2;            // bit 1 of psgd_device_status()

struct AttentionArgs {
    HeadsView q, k, v, o, dout, dq, dk, dv;
    float *lse, *along;          // [n, heads, t]; along: D
    const int32_t* starts;
    int64_t starts_learner, t, first, total, places;      // first, total: workgroups of this launch and of all
    int sequences, heads, kv, head, window, sinks, n;
    float scale;
};

// Which learner, head and tile a workgroup has.  Workgroups that read the same keys follow each other on one die: dies take workgroups in turn, so where
// the pairs of learner and key head are a multiple of eight each die keeps its own.
struct Work {
    int learner, kv_head, member, lo, hi, tile;      // member: of the heads that share the key head; lo, hi: the sequence's rows
    bool there;
};
template <int ROWS> __device__ __forceinline__ Work find_work(const AttentionArgs& a, int members, bool last_first) {
    const int64_t id = a.first + blockIdx.x, inner = members * a.places;
    const int units = a.n * a.kv;
    int64_t unit, in;
    if (units % 8 == 0) {
        unit = id / (8 * inner) * 8 + id % 8;
        in = id / 8 % inner;
    } else {
        unit = id / inner;
        in = id % inner;
    }
    Work w{(int)(unit / a.kv), (int)(unit % a.kv), (int)(in % members), 0, (int)a.t, 0, true};
    int64_t place = in / members;
    if (last_first) place = a.places - 1 - place;
    if (!a.starts) {
        w.tile = (int)place;
    } else {
        const int32_t* starts = a.starts + w.learner * a.starts_learner;
        const int lane = threadIdx.x % kWave, t = (int)a.t;
        if (place == 0 && in % members == 0 && w.kv_head == 0) {
            bool bad = false;
            for (int s = threadIdx.x; s <= a.sequences; s += blockDim.x) bad |= starts[s] < 0 || starts[s] > t || (s > 0 && starts[s] < starts[s - 1]);
            if (bad) atomicOr(&g_attention_status, kAttentionFlag);
        }
        // the last sequence whose places start here or before: 64 candidates at a time
        int lo = 0, hi = a.sequences;          // it is in [lo, hi), if any is
        while (hi - lo > kWave) {
            const int mid = lo + (hi - lo) / 2;
            const int at = std::min(std::max(starts[mid], 0), t);
            if (at / ROWS + mid <= place) lo = mid;
            else hi = mid;
        }
        const int s = lo + lane, at = s < hi ? std::min(std::max(starts[s], 0), t) : 0;
        const int found = __popcll(__ballot(s < hi && at / ROWS + s <= place)) - 1;
        if (found < 0) {
            w.there = false;
            return w;
        }
        const int seq = lo + found;
        w.lo = std::min(std::max(starts[seq], 0), t);
        w.hi = std::min(std::max(starts[seq + 1], 0), t);
        w.tile = (int)(place - (w.lo / ROWS + seq));
    }
    w.there = w.tile >= 0 && (int64_t)w.tile * ROWS < w.hi - w.lo;
    return w;
}

// Moves a tile of rows row0 ... of a sequence (first row `lo`, `len` rows) from memory through registers to LDS.
template <typename T, int H, int ROWS, int THREADS> struct Mover {
    using Lds = Tile<T, H, ROWS>;
    static constexpr int kEach = (ROWS * Lds::kGroups + THREADS - 1) / THREADS;
    static_assert(ROWS * Lds::kGroups % THREADS == 0, "every lane moves as much");
    u32x4 held[kEach];
    __device__ __forceinline__ void fetch(const T* seq, int64_t row_stride, int row0, int len, int head, bool whole) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = threadIdx.x + j * THREADS, row = row0 + at / Lds::kGroups, col = at % Lds::kGroups * kPer<T>;
            held[j] = load_group(seq + row * row_stride + col, row < len ? head - col : 0, whole);
        }
    }
    __device__ __forceinline__ void put(char* tile) const {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = threadIdx.x + j * THREADS;
            Lds::put(tile, at / Lds::kGroups, at % Lds::kGroups, held[j]);
        }
    }
};

// Tiles of keys that a tile of queries sees: those of the first tokens, then from the window on.
struct KeyWalk {
    int sink_tiles, first, count;
    __device__ __forceinline__ KeyWalk(int row0, int row1, int window, int sinks, int rows) {      // queries [row0, row1)
        const int from = window ? std::max(0, row0 - window + 1) / rows : 0, to = (row1 + rows - 1) / rows;
        sink_tiles = std::min((sinks + rows - 1) / rows, from);
        first = from;
        count = sink_tiles + to - from;
    }
    __device__ __forceinline__ int tile(int step) const { return step < sink_tiles ? step : first + step - sink_tiles; }
};
__device__ __forceinline__ bool sees(int i, int j, int window, int sinks) { return j <= i && (window == 0 || i - j < window || j < sinks); }
// Whether rows [i0, i1] see all, and whether any of them sees one, of [j0, j1].
__device__ __forceinline__ bool all_see(int i0, int i1, int j0, int j1, int window, int sinks) {
    return j1 <= i0 && (window == 0 || i1 - j0 < window || j1 < sinks);
}
__device__ __forceinline__ bool any_sees(int i0, int i1, int j0, int j1, int window, int sinks) {
    return j0 <= i1 && (window == 0 || i0 - j1 < window || j0 < sinks);
}

template <typename T, int H> struct Shape {
    static constexpr int kOwnBlocks = own_blocks(H, sizeof(T)), kOwn = own_rows(H, sizeof(T)), kWalked = walked_rows(H, sizeof(T));
    static constexpr int kThreads = kAttentionWaves * kWave, kBlocks = kWalked / 16, kSteps = H / 32, kCols = H / 16;
    static constexpr bool kAhead = H * sizeof(T) < 1024;       // whether registers hold the next tile beside dk and dv
    using Lds = Tile<T, H, kWalked>;
};

template <typename T, int H> __global__ __launch_bounds__(kAttentionWaves* kWave) void attention_kernel(AttentionArgs a) {
    using S = Shape<T, H>;
    using Lds = typename S::Lds;
    extern __shared__ __attribute__((aligned(16))) char lds[];       // two of keys, two of values
    const int members = a.heads / a.kv;
    const Work w = find_work<S::kOwn>(a, members, true);
    if (!w.there) return;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = lane % 16, g = lane / 16, len = w.hi - w.lo;
    const int h = w.kv_head * members + w.member, row0 = w.tile * S::kOwn, row1 = std::min(row0 + S::kOwn, len);
    const bool whole = a.head % kPer<T> == 0;
    const int mine = row0 + wave * 16 * S::kOwnBlocks;               // the wavefront's first query
    const float to_log2 = a.scale * kLog2E;

    Eight<T> q[S::kOwnBlocks][S::kSteps];
    f32x4 o[S::kOwnBlocks][S::kCols];
    float top[S::kOwnBlocks], sum[S::kOwnBlocks];
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col;
        const T* p = at<T>(a.q, w.learner, w.lo + row, (int64_t)h * a.head);
#pragma unroll
        for (int kc = 0; kc < S::kSteps; ++kc) q[b][kc] = load_eight(p, kc, g, row < len ? a.head : 0, whole);
#pragma unroll
        for (int d = 0; d < S::kCols; ++d) o[b][d] = (f32x4){0, 0, 0, 0};
        top[b] = -INFINITY;
        sum[b] = 0.0f;
    }
    const T *keys = at<T>(a.k, w.learner, w.lo, (int64_t)w.kv_head * a.head), *values = at<T>(a.v, w.learner, w.lo, (int64_t)w.kv_head * a.head);
    const KeyWalk walk(row0, row1, a.window, a.sinks, S::kWalked);
    Mover<T, H, S::kWalked, S::kThreads> mk, mv;
    mk.fetch(keys, a.k.row, walk.tile(0) * S::kWalked, len, a.head, whole);
    mv.fetch(values, a.v.row, walk.tile(0) * S::kWalked, len, a.head, whole);
    mk.put(lds);
    mv.put(lds + Lds::kBytes);
    __syncthreads();
    for (int step = 0; step < walk.count; ++step) {
        const int key0 = walk.tile(step) * S::kWalked;
        const char *tk = lds + (step & 1) * 2 * Lds::kBytes, *tv = tk + Lds::kBytes;
        if (step + 1 < walk.count) {
            mk.fetch(keys, a.k.row, walk.tile(step + 1) * S::kWalked, len, a.head, whole);
            mv.fetch(values, a.v.row, walk.tile(step + 1) * S::kWalked, len, a.head, whole);
        }
        if (mine < len && any_sees(mine, mine + 16 * S::kOwnBlocks - 1, key0, key0 + S::kWalked - 1, a.window, a.sinks)) {
            f32x4 s[S::kOwnBlocks][S::kBlocks];
#pragma unroll
            for (int kb = 0; kb < S::kBlocks; ++kb) {
#pragma unroll
                for (int b = 0; b < S::kOwnBlocks; ++b) s[b][kb] = (f32x4){0, 0, 0, 0};
#pragma unroll
                for (int kc = 0; kc < S::kSteps; ++kc) {
                    const Eight<T> k = Lds::along(tk, kb, kc, lane);
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) s[b][kb] = mma(k, q[b][kc], s[b][kb]);
                }
            }
            const bool full = all_see(mine, mine + 16 * S::kOwnBlocks - 1, key0, key0 + S::kWalked - 1, a.window, a.sinks);
#pragma unroll
            for (int b = 0; b < S::kOwnBlocks; ++b) {
                float m = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < S::kBlocks; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[b][kb][e] *= to_log2;
                        if (!full && !sees(mine + 16 * b + col, key0 + 16 * kb + 4 * g + e, a.window, a.sinks)) s[b][kb][e] = -INFINITY;
                        m = fmaxf(m, s[b][kb][e]);
                    }
                m = fmaxf(top[b], column_all<Larger>(m));
                const float safe = m == -INFINITY ? 0.0f : m, less = exp_2(top[b] - safe);
                top[b] = m;
                float part = 0.0f;
#pragma unroll
                for (int kb = 0; kb < S::kBlocks; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[b][kb][e] = exp_2(s[b][kb][e] - safe);
                        part += s[b][kb][e];
                    }
                sum[b] = sum[b] * less + part;
#pragma unroll
                for (int d = 0; d < S::kCols; ++d) o[b][d] *= less;
            }
#pragma unroll
            for (int kc = 0; kc < S::kBlocks / 2; ++kc) {
                Eight<T> p[S::kOwnBlocks];
#pragma unroll
                for (int b = 0; b < S::kOwnBlocks; ++b) p[b] = as_operand<T>(s[b][2 * kc], s[b][2 * kc + 1]);
#pragma unroll
                for (int d = 0; d < S::kCols; ++d) {
                    const Eight<T> v = Lds::across(tv, d, kc, lane);
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) o[b][d] = mma(v, p[b], o[b][d]);
                }
            }
        }
        if (step + 1 < walk.count) {
            char* next = lds + (~step & 1) * 2 * Lds::kBytes;
            mk.put(next);
            mv.put(next + Lds::kBytes);
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col;
        const float all = column_all<Sum>(sum[b]), by = 1.0f / all;
        if (row >= len) continue;
        T* p = at<T>(a.o, w.learner, w.lo + row, (int64_t)h * a.head);
#pragma unroll
        for (int d = 0; d < S::kCols; ++d) store_four(p, 16 * d + 4 * g, a.head, o[b][d] * by);
        if (a.lse && g == 0) a.lse[((int64_t)w.learner * a.heads + h) * a.t + w.lo + row] = (top[b] + __builtin_amdgcn_logf(all)) * kLn2;
    }
}

// dq and D.  Queries and their gradients stay in registers, keys and values are walked as above, 32 rows of a tile at a time.
template <typename T, int H> __global__ __launch_bounds__(kAttentionWaves* kWave) void attention_dq_kernel(AttentionArgs a) {
    using S = Shape<T, H>;
    using Lds = typename S::Lds;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int members = a.heads / a.kv;
    const Work w = find_work<S::kOwn>(a, members, true);
    if (!w.there) return;
    int lane = threadIdx.x % kWave;
    const int wave = threadIdx.x / kWave, col = lane % 16, g = lane / 16, len = w.hi - w.lo;
    const int h = w.kv_head * members + w.member, row0 = w.tile * S::kOwn, row1 = std::min(row0 + S::kOwn, len);
    const bool whole = a.head % kPer<T> == 0;
    const int mine = row0 + wave * 16 * S::kOwnBlocks;
    const float to_log2 = a.scale * kLog2E;
    const int64_t stat = ((int64_t)w.learner * a.heads + h) * a.t + w.lo;

    Eight<T> q[S::kOwnBlocks][S::kSteps], dy[S::kOwnBlocks][S::kSteps];
    f32x4 dq[S::kOwnBlocks][S::kCols];
    float lse[S::kOwnBlocks], along[S::kOwnBlocks];
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col, left = row < len ? a.head : 0;
        const T *pq = at<T>(a.q, w.learner, w.lo + row, (int64_t)h * a.head), *pd = at<T>(a.dout, w.learner, w.lo + row, (int64_t)h * a.head),
                *po = at<T>(a.o, w.learner, w.lo + row, (int64_t)h * a.head);
        float d = 0.0f;
#pragma unroll
        for (int kc = 0; kc < S::kSteps; ++kc) {
            q[b][kc] = load_eight(pq, kc, g, left, whole);
            dy[b][kc] = load_eight(pd, kc, g, left, whole);
            d += dot(dy[b][kc], load_eight(po, kc, g, left, whole));
        }
        along[b] = column_all<Sum>(d);
        lse[b] = row < len ? a.lse[stat + row] * kLog2E : INFINITY;       // rows that are not there: p = 0
        if (row < len && g == 0) a.along[stat + row] = along[b];
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) dq[b][c] = (f32x4){0, 0, 0, 0};
    }
    const T *keys = at<T>(a.k, w.learner, w.lo, (int64_t)w.kv_head * a.head), *values = at<T>(a.v, w.learner, w.lo, (int64_t)w.kv_head * a.head);
    const KeyWalk walk(row0, row1, a.window, a.sinks, S::kWalked);
    Mover<T, H, S::kWalked, S::kThreads> mk, mv;
    mk.fetch(keys, a.k.row, walk.tile(0) * S::kWalked, len, a.head, whole);
    mv.fetch(values, a.v.row, walk.tile(0) * S::kWalked, len, a.head, whole);
    mk.put(lds);
    mv.put(lds + Lds::kBytes);
    __syncthreads();
    for (int step = 0; step < walk.count; ++step) {
        const int key0 = walk.tile(step) * S::kWalked;
        const char *tk = lds + (step & 1) * 2 * Lds::kBytes, *tv = tk + Lds::kBytes;
        if (!S::kAhead) asm("" : "+v"(lane));       // addresses in LDS are made anew: as many as are kept for a whole walk do not fit
        if (step + 1 < walk.count) {
            mk.fetch(keys, a.k.row, walk.tile(step + 1) * S::kWalked, len, a.head, whole);
            mv.fetch(values, a.v.row, walk.tile(step + 1) * S::kWalked, len, a.head, whole);
        }
        if (mine < len && any_sees(mine, mine + 16 * S::kOwnBlocks - 1, key0, key0 + S::kWalked - 1, a.window, a.sinks)) {
            const bool full = all_see(mine, mine + 16 * S::kOwnBlocks - 1, key0, key0 + S::kWalked - 1, a.window, a.sinks);
#pragma unroll
            for (int half = 0; half < S::kBlocks / 2; ++half) {
                f32x4 s[S::kOwnBlocks][2], dp[S::kOwnBlocks][2];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) s[b][kb] = dp[b][kb] = (f32x4){0, 0, 0, 0};
#pragma unroll
                    for (int kc = 0; kc < S::kSteps; ++kc) {
                        const Eight<T> k = Lds::along(tk, 2 * half + kb, kc, lane), v = Lds::along(tv, 2 * half + kb, kc, lane);
#pragma unroll
                        for (int b = 0; b < S::kOwnBlocks; ++b) {
                            s[b][kb] = mma(k, q[b][kc], s[b][kb]);
                            dp[b][kb] = mma(v, dy[b][kc], dp[b][kb]);
                        }
                    }
                }
                Eight<T> ds[S::kOwnBlocks];
#pragma unroll
                for (int b = 0; b < S::kOwnBlocks; ++b) {
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = exp_2(__builtin_fmaf(s[b][kb][e], to_log2, -lse[b]));
                            const float v = p * (dp[b][kb][e] - along[b]);
                            s[b][kb][e] = full || sees(mine + 16 * b + col, key0 + 16 * (2 * half + kb) + 4 * g + e, a.window, a.sinks) ? v : 0.0f;
                        }
                    ds[b] = as_operand<T>(s[b][0], s[b][1]);
                }
#pragma unroll
                for (int c = 0; c < S::kCols; ++c) {
                    const Eight<T> k = Lds::across(tk, c, half, lane);
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) dq[b][c] = mma(k, ds[b], dq[b][c]);
                }
            }
        }
        if (step + 1 < walk.count) {
            char* next = lds + (~step & 1) * 2 * Lds::kBytes;
            mk.put(next);
            mv.put(next + Lds::kBytes);
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col;
        if (row >= len) continue;
        T* p = at<T>(a.dq, w.learner, w.lo + row, (int64_t)h * a.head);
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) store_four(p, 16 * c + 4 * g, a.head, dq[b][c] * a.scale);
    }
}

// dk and dv.  Keys and values stay in registers; the queries that see them and their gradients are walked, one head that shares the key head after
// the other, with lse and D of a tile's rows beside it.
template <typename T, int H> __global__ __launch_bounds__(kAttentionWaves* kWave) void attention_dkv_kernel(AttentionArgs a) {
    using S = Shape<T, H>;
    using Lds = typename S::Lds;
    extern __shared__ __attribute__((aligned(16))) char lds[];       // two of queries, two of gradients, two of [2][rows] statistics
    const Work w = find_work<S::kOwn>(a, 1, false);
    if (!w.there) return;
    int lane = threadIdx.x % kWave;
    const int wave = threadIdx.x / kWave, col = lane % 16, g = lane / 16, len = w.hi - w.lo, members = a.heads / a.kv;
    const int key0 = w.tile * S::kOwn, key1 = std::min(key0 + S::kOwn, len);
    const bool whole = a.head % kPer<T> == 0;
    const int mine = key0 + wave * 16 * S::kOwnBlocks;               // the wavefront's first key
    const float to_log2 = a.scale * kLog2E;
    float* const stats = reinterpret_cast<float*>(lds + 4 * Lds::kBytes);

    Eight<T> k[S::kOwnBlocks][S::kSteps], v[S::kOwnBlocks][S::kSteps];
    f32x4 dk[S::kOwnBlocks][S::kCols], dv[S::kOwnBlocks][S::kCols];
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col, left = row < len ? a.head : 0;
        const T *pk = at<T>(a.k, w.learner, w.lo + row, (int64_t)w.kv_head * a.head), *pv = at<T>(a.v, w.learner, w.lo + row, (int64_t)w.kv_head * a.head);
#pragma unroll
        for (int kc = 0; kc < S::kSteps; ++kc) {
            k[b][kc] = load_eight(pk, kc, g, left, whole);
            v[b][kc] = load_eight(pv, kc, g, left, whole);
        }
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) dk[b][c] = dv[b][c] = (f32x4){0, 0, 0, 0};
    }
    // the tiles of queries: from the keys' own on, to the last that the window leaves them
    const int first = key0 / S::kWalked;
    const int64_t behind = a.window == 0 || key0 < a.sinks ? len : std::min((int64_t)len, (int64_t)key1 - 1 + a.window);
    const int tiles = (int)((behind + S::kWalked - 1) / S::kWalked) - first, count = tiles * members;
    Mover<T, H, S::kWalked, S::kThreads> mq, md;
    float held[2];
    auto fetch = [&](int step) {
        const int h = w.kv_head * members + step / tiles, row0 = (first + step % tiles) * S::kWalked, row = row0 + threadIdx.x;
        mq.fetch(at<T>(a.q, w.learner, w.lo, (int64_t)h * a.head), a.q.row, row0, len, a.head, whole);
        md.fetch(at<T>(a.dout, w.learner, w.lo, (int64_t)h * a.head), a.dout.row, row0, len, a.head, whole);
        const int64_t stat = ((int64_t)w.learner * a.heads + h) * a.t + w.lo + row;
        const bool there = threadIdx.x < S::kWalked && row < len;
        held[0] = there ? a.lse[stat] * kLog2E : INFINITY;
        held[1] = there ? a.along[stat] : 0.0f;
    };
    auto put = [&](int buffer) {
        mq.put(lds + buffer * 2 * Lds::kBytes);
        md.put(lds + buffer * 2 * Lds::kBytes + Lds::kBytes);
        if (threadIdx.x < S::kWalked) {
            stats[buffer * 2 * S::kWalked + threadIdx.x] = held[0];
            stats[(buffer * 2 + 1) * S::kWalked + threadIdx.x] = held[1];
        }
    };
    fetch(0);
    put(0);
    __syncthreads();
    for (int step = 0; step < count; ++step) {
        const int row0 = (first + step % tiles) * S::kWalked;
        const char *tq = lds + (step & 1) * 2 * Lds::kBytes, *td = tq + Lds::kBytes;
        const float* st = stats + (step & 1) * 2 * S::kWalked;
        if (S::kAhead && step + 1 < count) fetch(step + 1);
        if (!S::kAhead) asm("" : "+v"(lane));       // addresses in LDS are made anew: as many as are kept for a whole walk do not fit
        if (mine < len && any_sees(row0, row0 + S::kWalked - 1, mine, mine + 16 * S::kOwnBlocks - 1, a.window, a.sinks)) {
            const bool full = all_see(row0, row0 + S::kWalked - 1, mine, mine + 16 * S::kOwnBlocks - 1, a.window, a.sinks);
#pragma unroll
            for (int half = 0; half < S::kBlocks / 2; ++half) {
                f32x4 s[S::kOwnBlocks][2], dp[S::kOwnBlocks][2];
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) {
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) s[b][qb] = dp[b][qb] = (f32x4){0, 0, 0, 0};
#pragma unroll
                    for (int kc = 0; kc < S::kSteps; ++kc) {
                        const Eight<T> q = Lds::along(tq, 2 * half + qb, kc, lane), dy = Lds::along(td, 2 * half + qb, kc, lane);
#pragma unroll
                        for (int b = 0; b < S::kOwnBlocks; ++b) {
                            s[b][qb] = mma(q, k[b][kc], s[b][qb]);
                            dp[b][qb] = mma(dy, v[b][kc], dp[b][qb]);
                        }
                    }
                    const int row = 16 * (2 * half + qb) + 4 * g;
                    const f32x4 lse = *reinterpret_cast<const f32x4*>(st + row), along = *reinterpret_cast<const f32x4*>(st + S::kWalked + row);
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool seen = full || sees(row0 + row + e, mine + 16 * b + col, a.window, a.sinks);
                            const float p = exp_2(__builtin_fmaf(s[b][qb][e], to_log2, -lse[e])), ds = p * (dp[b][qb][e] - along[e]);
                            s[b][qb][e] = seen ? p : 0.0f;
                            dp[b][qb][e] = seen ? ds : 0.0f;
                        }
                }
                Eight<T> p[S::kOwnBlocks], ds[S::kOwnBlocks];
#pragma unroll
                for (int b = 0; b < S::kOwnBlocks; ++b) {
                    p[b] = as_operand<T>(s[b][0], s[b][1]);
                    ds[b] = as_operand<T>(dp[b][0], dp[b][1]);
                }
#pragma unroll
                for (int c = 0; c < S::kCols; ++c) {
                    const Eight<T> dy = Lds::across(td, c, half, lane), q = Lds::across(tq, c, half, lane);
#pragma unroll
                    for (int b = 0; b < S::kOwnBlocks; ++b) {
                        dv[b][c] = mma(dy, p[b], dv[b][c]);
                        dk[b][c] = mma(q, ds[b], dk[b][c]);
                    }
                }
            }
        }
        if (step + 1 < count) {
            if (!S::kAhead) fetch(step + 1);
            put(~step & 1);
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
        const int row = mine + 16 * b + col;
        if (row >= len) continue;
        T *pk = at<T>(a.dk, w.learner, w.lo + row, (int64_t)w.kv_head * a.head), *pv = at<T>(a.dv, w.learner, w.lo + row, (int64_t)w.kv_head * a.head);
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) {
            store_four(pk, 16 * c + 4 * g, a.head, dk[b][c] * a.scale);
            store_four(pv, 16 * c + 4 * g, a.head, dv[b][c]);
        }
    }
}

template <typename T, int H> constexpr size_t kTileLds = 4 * (size_t)Tile<T, H, walked_rows(H, sizeof(T))>::kBytes;
template <typename T, int H> constexpr size_t kStatLds = 4 * (size_t)walked_rows(H, sizeof(T)) * sizeof(float);

using AttentionKernel = void (*)(AttentionArgs);
template <typename T, int H> int launch_forward(const char* name, AttentionArgs a, hipStream_t s) {
    static LdsRecord record = {};
    const AttentionKernel fn = attention_kernel<T, H>;
    if (int rc = allow_lds(reinterpret_cast<const void*>(fn), kTileLds<T, H>, record)) return rc;
    a.places = tile_places(a.t, a.sequences, own_rows(H, sizeof(T)));
    in_slices(a.places * a.n * a.heads, [&](int64_t first, unsigned groups) {
        a.first = first;
        hipLaunchKernelGGL(fn, dim3(groups), dim3(kAttentionWaves * kWave), (kTileLds<T, H>), s, a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}
template <typename T, int H> int launch_backward(const char* name, AttentionArgs a, hipStream_t s) {
    static LdsRecord record_q = {}, record_kv = {};
    const AttentionKernel fq = attention_dq_kernel<T, H>, fkv = attention_dkv_kernel<T, H>;
    const size_t lds = kTileLds<T, H>, more = lds + kStatLds<T, H>;
    if (int rc = allow_lds(reinterpret_cast<const void*>(fq), lds, record_q)) return rc;
    if (int rc = allow_lds(reinterpret_cast<const void*>(fkv), more, record_kv)) return rc;
    a.places = tile_places(a.t, a.sequences, own_rows(H, sizeof(T)));
    in_slices(a.places * a.n * a.heads, [&](int64_t first, unsigned groups) {
        a.first = first;
        hipLaunchKernelGGL(fq, dim3(groups), dim3(kAttentionWaves * kWave), lds, s, a);
    });
    in_slices(a.places * a.n * a.kv, [&](int64_t first, unsigned groups) {
        a.first = first;
        hipLaunchKernelGGL(fkv, dim3(groups), dim3(kAttentionWaves * kWave), more, s, a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PSGD_OK : hip_error(e, name);
}
template <typename T> int forward_of(const char* name, const AttentionArgs& a, hipStream_t s) {
    switch (held_head(a.head)) {
        case 64: return launch_forward<T, 64>(name, a, s);
        case 128: return launch_forward<T, 128>(name, a, s);
        default: return launch_forward<T, 256>(name, a, s);
    }
}
template <typename T> int backward_of(const char* name, const AttentionArgs& a, hipStream_t s) {
    switch (held_head(a.head)) {
        case 64: return launch_backward<T, 64>(name, a, s);
        case 128: return launch_backward<T, 128>(name, a, s);
        default: return launch_backward<T, 256>(name, a, s);
    }
}

inline int check_shape(const char* name, int heads, int kv, int head, int window, int sinks, float scale, int sequences, const psgd_view* starts, int n, int64_t t) {
    if (heads < 1 || kv < 1 || heads % kv) return fail(PSGD_EINVAL, "%s: kv=%d does not divide heads=%d", name, kv, heads);
    if (head < 1 || head > PSGD_MAX_HEAD) return fail(PSGD_EINVAL, "%s: head=%d outside 1..%d", name, head, (int)PSGD_MAX_HEAD);
    if (int rc = check_counts(name, n, t, (int64_t)heads * head)) return rc;
    if (window < 0 || sinks < 0 || (sinks && !window)) return fail(PSGD_EINVAL, "%s: window=%d with sinks=%d", name, window, sinks);
    if (!std::isfinite(scale)) return fail(PSGD_EINVAL, "%s: scale=%g", name, (double)scale);
    if (sequences < 0 || (sequences > 0) != (starts != nullptr)) return fail(PSGD_EINVAL, "%s: sequences=%d %s starts", name, sequences, starts ? "with" : "without");
    if (starts && starts->type != PSGD_I32) return fail(PSGD_EINVAL, "%s: starts must be int32", name);
    // a row's number and a tile's end are counted in 32 bits, and so are all learners' heads
    if (t > INT32_MAX - 1024 || (int64_t)n * heads > INT32_MAX || sequences > INT32_MAX - 1024 || (double)n * heads * ((double)t + sequences) > 1e15)
        return fail(PSGD_EINVAL, "%s: a size beyond 2^31 - 1", name);
    return PSGD_OK;
}

}  // namespace

int attention_status(int clear, int* word) {
    hipError_t e = hipMemcpyFromSymbol(word, HIP_SYMBOL(g_attention_status), sizeof(int));
    if (e != hipSuccess) return hip_error(e, "hipMemcpyFromSymbol");
    if (clear && *word) {
        const int zero = 0;
        e = hipMemcpyToSymbol(HIP_SYMBOL(g_attention_status), &zero, sizeof(int));
        if (e != hipSuccess) return hip_error(e, "hipMemcpyToSymbol");
    }
    return PSGD_OK;
}

}  // namespace psgd

extern "C" {

int psgd_attention(const psgd_view* q, const psgd_view* k, const psgd_view* v, const psgd_view* starts, const psgd_view* out, float* lse, int heads,
                   int kv, int head, int window, int sinks, float scale, int sequences, int n, int64_t t, void* stream) {
    using namespace psgd;
    const char* name = "psgd_attention";
    clear_error();
    if (!q || !k || !v || !out) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_shape(name, heads, kv, head, window, sinks, scale, sequences, starts, n, t)) return rc;
    for (const psgd_view* x : {q, k, v, out})
        if (!float_type(x->type) || x->type != q->type) return fail(PSGD_EINVAL, "%s: q, k, v and out must be float or bf16 alike", name);
    if (t == 0) return PSGD_OK;
    psgd_view vl;
    const int64_t cq = (int64_t)heads * head, ck = (int64_t)kv * head;
    const Extent eq{"q", q, n, t, cq}, ek{"k", k, n, t, ck}, ev{"v", v, n, t, ck}, eo{"out", out, n, t, cq},
        es{"starts", starts ? starts : q, n, 1, starts ? (int64_t)sequences + 1 : 0}, el = flat("lse", lse, lse ? (int64_t)n * heads * t : 0, &vl);
    for (const Extent* e : {&eq, &ek, &ev, &es})
        if (int rc = check_operand(name, *e, false)) return rc;
    for (const Extent* e : {&eo, &el})
        if (int rc = check_operand(name, *e, true)) return rc;
    for (const Extent* o : {&eo, &el})
        for (const Extent* e : {&eq, &ek, &ev, &es})
            if (int rc = refuse_overlap(name, *o, *e)) return rc;
    if (int rc = refuse_overlap(name, eo, el)) return rc;
    AttentionArgs a{};
    a.q = heads_view(q);
    a.k = heads_view(k);
    a.v = heads_view(v);
    a.o = heads_view(out);
    a.lse = lse;
    if (starts) {
        a.starts = static_cast<const int32_t*>(starts->data);
        a.starts_learner = starts->learner;
    }
    a.t = t;
    a.sequences = sequences;
    a.heads = heads;
    a.kv = kv;
    a.head = head;
    a.window = window < t ? window : 0;                  // a window that leaves nothing out is none
    a.sinks = a.window ? (int)std::min<int64_t>(sinks, t) : 0;
    a.n = n;
    a.scale = scale;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return q->type == PSGD_F32 ? forward_of<float>(name, a, s) : forward_of<uint16_t>(name, a, s);
}

size_t psgd_attention_grad_workspace(int heads, int kv, int head, int window, int sinks, int sequences, int n, int64_t t) {
    (void)kv, (void)head, (void)window, (void)sinks, (void)sequences;
    if (n < 1 || n > PSGD_MAX_N || t < 1 || t > INT32_MAX || heads < 1) return 0;
    return psgd::up256((size_t)n * heads * t * sizeof(float));
}

int psgd_attention_grad(const psgd_view* dout, const psgd_view* q, const psgd_view* k, const psgd_view* v, const psgd_view* out, const float* lse,
                        const psgd_view* starts, const psgd_view* dq, const psgd_view* dk, const psgd_view* dv, int heads, int kv, int head, int window,
                        int sinks, float scale, int sequences, int n, int64_t t, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace psgd;
    const char* name = "psgd_attention_grad";
    clear_error();
    if (!dout || !q || !k || !v || !out || !dq || !dk || !dv) return fail(PSGD_EINVAL, "%s: null operand", name);
    if (int rc = check_shape(name, heads, kv, head, window, sinks, scale, sequences, starts, n, t)) return rc;
    for (const psgd_view* x : {dout, q, k, v, out, dq, dk, dv})
        if (!float_type(x->type) || x->type != q->type) return fail(PSGD_EINVAL, "%s: dout, q, k, v, out, dq, dk and dv must be float or bf16 alike", name);
    if (t == 0) return PSGD_OK;
    if (!lse) return fail(PSGD_EINVAL, "%s: lse is needed", name);
    const size_t need = psgd_attention_grad_workspace(heads, kv, head, window, sinks, sequences, n, t);
    psgd_view vl, vw;
    const int64_t cq = (int64_t)heads * head, ck = (int64_t)kv * head;
    const Extent ed{"dout", dout, n, t, cq}, eq{"q", q, n, t, cq}, ek{"k", k, n, t, ck}, ev{"v", v, n, t, ck}, eo{"out", out, n, t, cq},
        es{"starts", starts ? starts : q, n, 1, starts ? (int64_t)sequences + 1 : 0}, el = flat("lse", lse, (int64_t)n * heads * t, &vl),
        edq{"dq", dq, n, t, cq}, edk{"dk", dk, n, t, ck}, edv{"dv", dv, n, t, ck}, ew = flat("the workspace", workspace, (int64_t)(need / 4), &vw);
    for (const Extent* e : {&ed, &eq, &ek, &ev, &eo, &es, &el})
        if (int rc = check_operand(name, *e, false)) return rc;
    for (const Extent* e : {&edq, &edk, &edv})
        if (int rc = check_operand(name, *e, true)) return rc;
    if (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail(PSGD_EINVAL, "%s: %zu bytes of workspace are needed, at a multiple of 256", name, need);
    for (const Extent* o : {&edq, &edk, &edv, &ew})
        for (const Extent* e : {&ed, &eq, &ek, &ev, &eo, &es, &el})
            if (int rc = refuse_overlap(name, *o, *e)) return rc;
    if (int rc = refuse_overlap(name, edq, edk)) return rc;
    if (int rc = refuse_overlap(name, edq, edv)) return rc;
    if (int rc = refuse_overlap(name, edk, edv)) return rc;
    for (const Extent* e : {&edq, &edk, &edv})
        if (int rc = refuse_overlap(name, ew, *e)) return rc;
    AttentionArgs a{};
    a.dout = heads_view(dout);
    a.q = heads_view(q);
    a.k = heads_view(k);
    a.v = heads_view(v);
    a.o = heads_view(out);
    a.dq = heads_view(dq);
    a.dk = heads_view(dk);
    a.dv = heads_view(dv);
    a.lse = const_cast<float*>(lse);
    a.along = static_cast<float*>(workspace);
    if (starts) {
        a.starts = static_cast<const int32_t*>(starts->data);
        a.starts_learner = starts->learner;
    }
    a.t = t;
    a.sequences = sequences;
    a.heads = heads;
    a.kv = kv;
    a.head = head;
    a.window = window < t ? window : 0;                  // a window that leaves nothing out is none
    a.sinks = a.window ? (int)std::min<int64_t>(sinks, t) : 0;
    a.n = n;
    a.scale = scale;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return q->type == PSGD_F32 ? backward_of<float>(name, a, s) : backward_of<uint16_t>(name, a, s);
}

}  // extern "C"
