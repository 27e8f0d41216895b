// Rules on the logits of new tokens, and the choice of a token under them.
//
// With c the number of times that token v stands in its sequence's history,
// and one list of biases a sequence, every step rounded to float32:
//   z = x                                               c = 0
//   z = (x > 0 ? x / r : x r) - (f c + p)               c > 0
//   z = z + bias[v]                                     v in the list
//   y = z (1 / T),  -inf where the mask does not allow v
// logits_apply_rules writes y; logits_pick reads x once and keeps a row's
// best token, its probability (or the margin to the second best, or the
// distribution's negative entropy) and the log-sum-exp. The order of tokens
// is that of z: a temperature does not change it, but its rounding could
// make two tokens equal.
//
// With d_v = (z_v - m) / T, m a running maximum, l = sum e^d:
//   probability 1 / l, margin (1 - e^(d_second)) / l,
//   entropy -sum p ln p = ln l - (sum e^d d) / l,  ln sum e^y = m / T + ln l.
//
// Bound by memory: x once (and y once), a mask's bit a token. A history and
// a list of biases name few tokens, so they are not spread over the
// vocabulary: a CTA sets a bit for each named token of its slice in shared
// memory. Eight warps stream the slice and leave the named tokens out (a few
// bit operations for 16 bytes); four others meanwhile number the bits and list
// the named tokens with their penalties and biases, and take them one a lane,
// which the eight join when the stream has ended. (Looked up in the stream
// itself, a warp met a named token in most of its pieces and spent most of its
// time on them; before the stream, it stood still for as long.) A CTA takes up to eight rows of a
// sequence, which share the tables; a warp takes a row or parts of it, its
// maximum is one number for all lanes and moves only when a batch of tokens
// passes it. A cluster shares the slices; its first CTA joins the results, in
// their order.
#include <algorithm>

#include "logits.cuh"

namespace starq {
namespace {

constexpr int STREAM = 8, HELP = 4;    // warps
constexpr int WARPS = STREAM + HELP, THREADS = 32 * WARPS;
constexpr int SLICE = 16384;           // most tokens of a slice
constexpr int NAMED = 8192;            // named tokens that a CTA has room for (then a slice is no longer than that)
constexpr int MAX_CLUSTER = 8;
constexpr int ROWS = 8;                // rows of a CTA
constexpr int AHEAD = 3;               // tokens of the history that a thread asks for at once
constexpr int NAMES = 4;               // named tokens of a thread on their way
// Tokens of a thread that are worked on together (a chain of dependent
// operations a batch: four batches of 4 took 640 cycles each), and 16-byte
// loads on their way beside them.
constexpr int BATCH = 16, FLIGHT = 4;
constexpr int CHUNK = 32 * NAMES, CHUNKS = NAMED / CHUNK;      // of named tokens
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

enum { APPLY = -1 };                   // else a starq_confidence

// How the work is cut.
struct Cut {
    int rows;                          // of a CTA
    int groups;                        // CTAs' row groups of a sequence
    int parts, parts_log;              // of a row's slice: 1, 2, 4 or 8
    int cluster;                       // CTAs that share the slices
    int len;                           // tokens of a slice, a multiple of 32
    int room;                          // named tokens of a slice at most
};

// What is known of some of a row's tokens: largest z (its lowest index), and
// with d = (z - m) kk, kk = log2(e) / T, sum of 2^d and the second largest z or
// sum of 2^d d. (z kk - m kk would be one operation less, but the products of
// large logits overflow.)
struct Best {
    float m;
    int at;
    float l, s;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 A, B, D;\n\t"
        "mov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\t"
        "mul.rn.f32x2 D, A, B;\n\tmov.b64 {%0, %1}, D;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// The largest of z, NaN if one is.
template <int N> __device__ __forceinline__ float largest(const float (&z)[N]) {
    float top = z[0];
    #pragma unroll
    for (int k = 1; k + 1 < N; k += 2) top = max_nan(top, z[k], z[k + 1]);
    return N % 2 == 0 ? max_nan(top, z[N - 1]) : top;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 A, B, C, D;\n\t"
        "mov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\tmov.b64 C, {%6, %7};\n\t"
        "fma.rn.f32x2 D, A, B, C;\n\tmov.b64 {%0, %1}, D;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 A, B, D;\n\t"
        "mov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\t"
        "add.rn.f32x2 D, A, B;\n\tmov.b64 {%0, %1}, D;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float warp_max_nan(float a) {
    float d;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(a));
    return d;
}

// Adds b to a (kk: log2(e) / T). NaN is above everything.
template <int KIND>
__device__ __forceinline__ void join(Best& a, const Best& b, float kk) {
    const bool nan_a = a.m != a.m, nan_b = b.m != b.m;
    const bool other = nan_b ? !nan_a || b.at < a.at : !nan_a && (b.m > a.m || (b.m == a.m && b.at < a.at));
    const float top = other ? b.m : a.m;
    const float da = a.m == NEG_INF ? NEG_INF : a.m == top ? 0.f : (a.m - top) * kk;
    const float db = b.m == NEG_INF ? NEG_INF : b.m == top ? 0.f : (b.m - top) * kk;
    const float fa = ex2(da), fb = ex2(db);
    if (KIND == STARQ_CONFIDENCE_MARGIN) a.s = fmaxf(fminf(a.m, b.m), fmaxf(a.s, b.s));
    if (KIND == STARQ_CONFIDENCE_ENTROPY)
        a.s = (fa > 0.f ? fa * fmaf(a.l, da, a.s) : 0.f) + (fb > 0.f ? fb * fmaf(b.l, db, b.s) : 0.f);
    a.l = fa * a.l + fb * b.l;
    a.m = top;
    if (other) a.at = b.at;
}

template <int KIND>
__device__ __forceinline__ Best nothing() {
    return Best{NEG_INF, 0x7fffffff, 0.f, KIND == STARQ_CONFIDENCE_MARGIN ? NEG_INF : 0.f};
}

template <int KIND>
__device__ __forceinline__ void join_lanes(Best& a, float kk) {
    #pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
        Best b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, m);
        b.at = __shfl_xor_sync(0xffffffffu, a.at, m);
        b.l = __shfl_xor_sync(0xffffffffu, a.l, m);
        b.s = __shfl_xor_sync(0xffffffffu, a.s, m);
        join<KIND>(a, b, kk);
    }
}

// The warp's part of a row: m and at are the same in all lanes, and s of a
// margin; l and s of an entropy are the lane's.
template <int KIND> constexpr bool MARGIN = KIND == STARQ_CONFIDENCE_MARGIN;
template <int KIND> constexpr bool ENTROPY = KIND == STARQ_CONFIDENCE_ENTROPY;

// The N tokens of every lane, token(k) the k-th, may move the maximum (or the
// second largest). The whole warp comes here.
template <int KIND, int N, typename F>
__device__ __forceinline__ void move_best(Best& a, const float (&z)[N], float lane_top, F&& token, float kk) {
    const float top = warp_max_nan(lane_top);
    const bool nan = top != top;
    unsigned first = 0x7fffffffu;                            // the lowest token that has the top
    #pragma unroll
    for (int k = N - 1; k >= 0; --k)
        if (nan ? z[k] != z[k] : z[k] == top) first = min(first, (unsigned)token(k));
    first = __reduce_min_sync(0xffffffffu, first);
    if (a.m != a.m) {                                        // NaN stays, the lowest of them
        if (nan) a.at = min(a.at, (int)first);
        return;
    }
    if (!nan && top <= a.m) {
        if (top == a.m && top != NEG_INF) a.at = min(a.at, (int)first);
        if (MARGIN<KIND>) a.s = fmaxf(a.s, top);
        return;
    }
    if (MARGIN<KIND>) {
        float second = NEG_INF;
        #pragma unroll
        for (int k = 0; k < N; ++k)
            if ((unsigned)token(k) != first) second = fmaxf(second, z[k]);
        a.s = fmaxf(a.m, warp_max_nan(second));
    }
    const float d = a.m == NEG_INF ? NEG_INF : (a.m - top) * kk, f = ex2(d);
    if (ENTROPY<KIND>) a.s = f > 0.f ? f * fmaf(a.l, d, a.s) : 0.f;
    a.l *= f;
    a.m = top;
    a.at = (int)first;
}

template <int KIND, int N>
__device__ __forceinline__ void add_weights(Best& a, const float (&z)[N], float kk) {
    const float c = a.m == NEG_INF ? 0.f : -a.m;
    if constexpr (N == 1) {
        const float d = (z[0] + c) * kk, e = ex2(d);
        a.l += e;
        if (ENTROPY<KIND>) a.s = fmaf(e, fmaxf(d, -1000.f), a.s);
    } else {
        float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, s[2] = {l[0], l[0]};
        #pragma unroll
        for (int k = 0; k < N; k += 2) {
            const float2 d = mul2(add2(make_float2(z[k], z[k + 1]), make_float2(c, c)), make_float2(kk, kk));
            const float2 e = make_float2(ex2(d.x), ex2(d.y));
            l[k / 2 & 1] = add2(l[k / 2 & 1], e);
            // (a weight of 0 adds nothing, though its d may be -inf)
            if (ENTROPY<KIND>) s[k / 2 & 1] = fma2(e, make_float2(fmaxf(d.x, -1000.f), fmaxf(d.y, -1000.f)), s[k / 2 & 1]);
        }
        a.l += (l[0].x + l[1].x) + (l[0].y + l[1].y);
        if (ENTROPY<KIND>) a.s += (s[0].x + s[1].x) + (s[0].y + s[1].y);
    }
}

// A 16-byte piece of a row.
template <typename T> constexpr int SE = 16 / (int)sizeof(T);
template <typename T> __device__ __forceinline__ void open_as(const uint4& w, float (&z)[SE<T>]) {
    if constexpr (sizeof(T) == 4) {
        z[0] = __uint_as_float(w.x); z[1] = __uint_as_float(w.y); z[2] = __uint_as_float(w.z); z[3] = __uint_as_float(w.w);
    } else {
        Eight<T>::load(reinterpret_cast<const T*>(&w), z);
    }
}

template <typename T, int KIND, bool TABLES>
__global__ void __launch_bounds__(THREADS, 2) logits_kernel(const LogitsArgs a, const Cut cut) {
    constexpr int E = SE<T>, U = BATCH / E, BUFFERS = FLIGHT / U + 1;
    constexpr bool PICK = KIND != APPLY;
    constexpr uint32_t FULL = (1u << E) - 1;
    constexpr uint32_t COUNTED = 1u << 29, LISTED = 1u << 30, NONE = 1u << 31;
    // by number: the named tokens of the slice (and which rules name them), penalties, list entries that become biases
    // [room]; counts [len]; the named tokens' bits [len / 32 + 1], the numbers before them [len / 32]; for each row the
    // bits of the tokens that the stream may take [len / 32]
    extern __shared__ __align__(16) uint32_t tables[];
    __shared__ Best s_item[ROWS][STREAM + 1 + CHUNKS], s_row[ROWS][MAX_CLUSTER];
    __shared__ int s_sum[HELP], s_next, s_names;
    const int words = cut.len / 32;
    uint32_t* const token_of = tables;
    float* const penalty = reinterpret_cast<float*>(token_of + cut.room);
    uint32_t* const entry = token_of + 2 * cut.room;
    uint32_t* const count = token_of + 3 * cut.room;
    uint32_t* const named = count + cut.len;
    uint32_t* const before = named + (words + 1);
    uint32_t* const free_bits = TABLES ? before + words : tables;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool streams = warp < STREAM;
    const int unit = (int)(blockIdx.x / (unsigned)cut.cluster), rank = (int)(blockIdx.x % (unsigned)cut.cluster);
    const int b = unit / cut.groups, first = (unit - b * cut.groups) * cut.rows;

    grid_dependency_wait();
    // What does not wait for anything else is asked for first: the lengths, the settings, the first tokens of the
    // history and of the list.
    const int row0 = __ldg(a.seq_start + b), n = __ldg(a.seq_start + b + 1) - row0;
    const int32_t* const history = a.r.history + (size_t)b * a.r.history_ld;
    const int32_t* const ids = a.r.bias_ids + (size_t)b * a.r.bias_ld;
    const float* const values = a.r.bias_values + (size_t)b * a.r.bias_ld;
    const bool told_any = TABLES && a.r.history != nullptr, listed_any = TABLES && a.r.bias_ids != nullptr;
    int told = told_any ? __ldg(a.r.history_len + b) : 0, entries = listed_any ? __ldg(a.r.bias_len + b) : 0;
    int told0[AHEAD];
    #pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        told0[k] = told_any && tid + k * THREADS < a.r.history_ld ? __ldg(history + tid + k * THREADS) : 0;
    const int listed0 = listed_any && tid < a.r.bias_ld ? __ldg(ids + tid) : 0;
    float temperature = 1.f, repetition = 1.f, presence = 0.f, frequency = 0.f;
    if (a.r.params != nullptr) {
        const float* p = a.r.params + 4 * (size_t)b;
        temperature = __ldg(p); repetition = __ldg(p + 1); presence = __ldg(p + 2); frequency = __ldg(p + 3);
    }
    if (n < 0 || n > a.max_new || row0 < 0 || row0 > a.T - n) {
        if (tid == 0) atomicOr(a.status, STATUS_RANGE);
        return;                                              // (the whole cluster does)
    }
    if (first >= n) return;
    if (PICK && cut.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    const int rows = min(cut.rows, n - first), items = rows << cut.parts_log;

    // A row's slice: 16-byte pieces, aligned; the tokens before and behind them are its edges.
    struct Slice {
        const T* x; T* y;
        const uint32_t* mask;
        int lead, pieces, here;                              // tokens before the pieces, pieces, all tokens
    };
    auto slice_of = [&](int r, int v0) {
        Slice t;
        t.here = min(cut.len, a.V - v0);
        const size_t row = (size_t)row0 + first + r;
        t.x = static_cast<const T*>(a.X) + row * a.ldx + v0;
        t.y = PICK ? nullptr : static_cast<T*>(a.Y) + row * a.ldy + v0;
        t.mask = a.r.allowed;
        if (t.mask != nullptr) t.mask += (a.r.allowed_by_row ? row : (size_t)b) * a.r.allowed_ld + (v0 >> 5);
        t.lead = min(t.here, -((int)(reinterpret_cast<uintptr_t>(t.x) / sizeof(T))) & (E - 1));
        t.pieces = (t.here - t.lead) / E;
        return t;
    };
    // rows whose bits are the same (their masks and alignments are)
    const bool bits = TABLES || a.r.allowed != nullptr;
    const bool one = !(a.r.allowed != nullptr && a.r.allowed_by_row) && (size_t)a.ldx * sizeof(T) % 16 == 0;

    // A warp's items, parts of rows, one after the other: the place of a batch.
    struct Place {
        const T* x; T* y;                                    // the row's first piece
        int item, row, lead, j, j_end;
    };
    auto settle = [&](Place& p, int v0) {                    // the first item from p.item on that has pieces
        for (; p.item < items; p.item += STREAM) {
            p.row = p.item >> cut.parts_log;
            const Slice t = slice_of(p.row, v0);
            const int share = (t.pieces + cut.parts - 1) >> cut.parts_log;
            p.j = (p.item & (cut.parts - 1)) * share;
            p.j_end = min(t.pieces, p.j + share);
            p.lead = t.lead;
            p.x = t.x + t.lead;
            p.y = PICK ? nullptr : t.y + t.lead;
            if (p.j < p.j_end) return;
        }
    };
    struct Batch { uint4 w[U]; };
    // Pieces j + 32 u + lane; what is behind the item's last one is read as the last one and not used.
    auto load = [&](Place& p, int v0, Batch& q) {
        if (p.item >= items) return;
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint4* from = reinterpret_cast<const uint4*>(p.x) + min(p.j + 32 * u + lane, p.j_end - 1);
            q.w[u] = PICK ? __ldcs(from) : *from;
        }
        p.j += 32 * U;
        if (p.j >= p.j_end) {
            p.item += STREAM;
            settle(p, v0);
        }
    };

    const bool t_ok = temperature >= 1e-30f && temperature <= 1e30f, r_ok = repetition >= 1e-30f && repetition <= 1e30f;
    if (PICK)
        for (int i = tid; i < ROWS * (STREAM + 1 + CHUNKS); i += THREADS) s_item[0][i] = nothing<KIND>();
    float warm = 0.f, kk = 0.f;

    for (int v0 = rank * cut.len; v0 < a.V; v0 += cut.cluster * cut.len) {
        const int here = min(cut.len, a.V - v0);
        Batch q[BUFFERS];
        Place at{nullptr, nullptr, streams ? warp : items, 0, 0, 0, 0};
        settle(at, v0);
        Place next = at;
        #pragma unroll
        for (int k = 0; k < BUFFERS - 1; ++k) load(next, v0, q[k]);       // on their way beside the tables
        if (v0 == rank * cut.len) {
            const bool odd = !(t_ok && r_ok) || told < 0 || told > a.r.history_ld || entries < 0 || entries > a.r.bias_ld;
            if (!t_ok) temperature = 1.f;
            if (!r_ok) repetition = 1.f;
            if (told < 0 || told > a.r.history_ld) told = 0;
            if (entries < 0 || entries > a.r.bias_ld) entries = 0;
            if (odd && tid == 0) atomicOr(a.status, STATUS_RANGE);
            warm = __fdiv_rn(1.f, temperature);
            kk = warm * LOG2E;
        }
        __syncthreads();                                     // the tables of the slice before are done with
        if (tid == 0) { s_next = 0; s_names = 0; }
        if (TABLES) {
            // counts, then bits; list entries before them
            const int zeros = 3 * cut.room + cut.len + words + 1;
            for (int i = 4 * (2 * cut.room / 4 + tid); i < zeros; i += 4 * THREADS)
                *reinterpret_cast<uint4*>(tables + i) = make_uint4(0, 0, 0, 0);
            __syncthreads();
            auto name = [&](int v, bool told_one) {
                const int p = v - v0;
                if (v < 0 || v >= a.V) {
                    atomicOr(a.status, STATUS_RANGE);
                } else if (p >= 0 && p < here) {
                    if (told_one) atomicAdd(count + p, 1u);
                    atomicOr(named + (p >> 5), 1u << (p & 31));
                }
            };
            #pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (tid + k * THREADS < told) name(told0[k], true);
            #pragma unroll 4
            for (int i = tid + AHEAD * THREADS; i < told; i += THREADS) name(__ldg(history + i), true);
            if (tid < entries) name(listed0, false);
            for (int i = tid + THREADS; i < entries; i += THREADS) name(__ldg(ids + i), false);
            __syncthreads();
        }
        if (bits) {                                          // bit i of a row: token lead + i is allowed and not named
            const int some = (here + 31) / 32;
            for (int r = one ? 0 : warp; r < (one ? 1 : rows); r += WARPS) {
                const Slice t = slice_of(r, v0);
                #pragma unroll 4
                for (int k = one ? tid : lane; k < some; k += one ? THREADS : 32) {
                    const int e = t.lead + 32 * k, w = e >> 5;
                    uint32_t free = ~0u;
                    if (t.mask != nullptr) {
                        const uint32_t lo = __ldg(t.mask + min(w, some - 1)), hi = __ldg(t.mask + min(w + 1, some - 1));
                        free = __funnelshift_r(lo, hi, e);
                    }
                    if (TABLES) free &= ~__funnelshift_r(named[min(w, words)], named[min(w + 1, words)], e);
                    free_bits[r * words + k] = free;
                }
            }
            __syncthreads();
        }

        Best best = nothing<KIND>();
        auto work = [&](const Place& p, const Batch& q) {
            float z[BATCH];
            uint32_t good[U];
            #pragma unroll
            for (int u = 0; u < U; ++u) {
                const int jj = p.j + 32 * u + lane;
                float f[E];
                open_as<T>(q.w[u], f);
                good[u] = jj < p.j_end ? FULL : 0u;
                if (bits) good[u] &= free_bits[(one ? 0 : p.row * words) + (min(jj, p.j_end - 1) * E >> 5)] >> (jj * E & 31);
                #pragma unroll
                for (int k = 0; k < E; ++k) z[u * E + k] = good[u] >> k & 1 ? f[k] : NEG_INF;
            }
            if constexpr (!PICK) {
                const bool wide = reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
                #pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int jj = p.j + 32 * u + lane;
                    T o[E];
                    #pragma unroll
                    for (int k = 0; k < E; ++k) o[k] = (T)(__fmul_rn(z[u * E + k], warm));
                    if (jj >= p.j_end) continue;
                    uint32_t mine = FULL;                     // tokens that are not named
                    const int e = p.lead + jj * E;
                    if (TABLES && good[u] != FULL) mine &= ~__funnelshift_r(named[e >> 5], named[(e >> 5) + 1], e);
                    if (wide && mine == FULL) {
                        uint4 v;
                        memcpy(&v, o, 16);
                        reinterpret_cast<uint4*>(p.y)[jj] = v;
                    } else {
                        #pragma unroll
                        for (int k = 0; k < E; ++k)
                            if (mine >> k & 1) p.y[jj * E + k] = o[k];
                    }
                }
            } else {
                const float top = largest(z);
                if (__any_sync(0xffffffffu, !(top <= (MARGIN<KIND> ? best.s : best.m))))
                    move_best<KIND>(best, z, top, [&](int k) {
                        return v0 + p.lead + (p.j + 32 * (k / E) + lane) * E + k % E;
                    }, kk);
                add_weights<KIND, BATCH>(best, z, kk);
            }
        };
        auto finish = [&](Best& to) {                        // what the warp knows of some tokens of a row
            #pragma unroll
            for (int m = 16; m > 0; m >>= 1) {
                best.l += __shfl_xor_sync(0xffffffffu, best.l, m);
                if (ENTROPY<KIND>) best.s += __shfl_xor_sync(0xffffffffu, best.s, m);
            }
            if (lane == 0) {
                Best sum = to;
                join<KIND>(sum, best, kk);
                to = sum;
            }
            best = nothing<KIND>();
        };
        #pragma unroll 1
        while (at.item < items) {
            #pragma unroll
            for (int k = 0; k < BUFFERS; ++k) {
                load(next, v0, q[(k + BUFFERS - 1) % BUFFERS]);
                work(at, q[k]);
                at.j += 32 * U;
                if (at.j >= at.j_end) {
                    if (PICK) finish(s_item[at.row][warp]);
                    at.item += STREAM;
                    settle(at, v0);
                    if (at.item >= items) break;
                }
            }
        }

        // --- the other warps: the list of the named tokens --------------------------------
        constexpr int HELPERS = 32 * HELP;
        if (TABLES && !streams) {
            const int hid = tid - 32 * STREAM, help = warp - STREAM;
            auto meet = [] { asm volatile("bar.sync 1, %0;" :: "n"(32 * HELP) : "memory"); };
            // the bits' numbers, in the order of the tokens: a thread takes a run of words
            const int per = (words + HELPERS - 1) / HELPERS, w0 = hid * per, w1 = min(words, w0 + per);
            int sum = 0;
            for (int w = w0; w < w1; ++w) sum += __popc(named[w]);
            int upto = sum;
            #pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, upto, m);
                if (lane >= m) upto += u;
            }
            if (lane == 31) s_sum[help] = upto;
            meet();
            int number0 = upto - sum, names = 0;
            #pragma unroll
            for (int w = 0; w < HELP; ++w) {
                if (w < help) number0 += s_sum[w];
                names += s_sum[w];
            }
            for (int w = w0; w < w1; ++w) {
                before[w] = number0;
                number0 += __popc(named[w]);
            }
            if (hid == 0) s_names = names;
            meet();
            // four bits of a word a thread (named tokens lie close together)
            for (int i = hid; i < 8 * words; i += HELPERS) {
                const uint32_t word = named[i >> 3], low = word & ((1u << 4 * (i & 7)) - 1);
                uint32_t m = word >> 4 * (i & 7) & 15;
                for (int to = (int)before[i >> 3] + __popc(low); m != 0; m &= m - 1, ++to) {
                    const int p = 4 * i + __ffs(m) - 1;
                    const uint32_t c = count[p];
                    token_of[to] = (uint32_t)p | (c ? COUNTED : 0u);
                    penalty[to] = __fadd_rn(__fmul_rn(frequency, (float)c), presence);
                }
            }
            for (int i = hid; i < entries; i += HELPERS) {   // the last of a token's entries counts
                const int p = __ldg(ids + i) - v0;
                if (p >= 0 && p < here)
                    atomicMax(entry + before[p >> 5] + __popc(named[p >> 5] & ((1u << (p & 31)) - 1)), (uint32_t)i + 1);
            }
            meet();
            if (entries > 0)
                for (int i = hid; i < names; i += HELPERS) {
                    const uint32_t k = entry[i];
                    if (k != 0) {
                        token_of[i] |= LISTED;
                        entry[i] = __float_as_uint(__ldg(values + (k - 1)));
                    }
                }
        }
        // --- the named tokens and the edges of the rows, by whoever is free ----------------
        // (the helpers wait for one another, the streaming warps for them)
        if (streams) asm volatile("bar.sync 2, %0;" :: "n"(32 * WARPS) : "memory");
        else {
            asm volatile("bar.arrive 2, %0;" :: "n"(32 * WARPS) : "memory");
            asm volatile("bar.sync 1, %0;" :: "n"(32 * HELP) : "memory");
        }
        const int names = TABLES ? *static_cast<volatile int*>(&s_names) : 0;
        const int chunks = (names + CHUNK - 1) / CHUNK;
        for (;;) {
            int i = 0;
            if (lane == 0) i = atomicAdd(&s_next, 1);
            i = __shfl_sync(0xffffffffu, i, 0);
            if (i >= rows * (chunks + 1)) break;
            const int r = i / (chunks + 1), chunk = i - r * (chunks + 1) - 1;        // -1: the edges
            const Slice t = slice_of(r, v0);
            uint32_t by[NAMES], word[NAMES];
            T x[NAMES];
            if (chunk >= 0) {
                #pragma unroll
                for (int k = 0; k < NAMES; ++k) {
                    const int m = chunk * CHUNK + 32 * k + lane;
                    by[k] = token_of[min(m, names - 1)] | (m < names ? 0u : NONE);
                }
            } else {
                const int ends = t.here - t.pieces * E;
                if (ends == 0) continue;
                const int p = lane < t.lead ? lane : lane + t.pieces * E;
                by[0] = lane < ends ? (uint32_t)p : NONE;
                if (TABLES && lane < ends && (named[p >> 5] >> (p & 31) & 1)) by[0] = NONE;          // it is in the list
                #pragma unroll
                for (int k = 1; k < NAMES; ++k) by[k] = NONE;
            }
            #pragma unroll
            for (int k = 0; k < NAMES; ++k) {                // (where there is none, token 0)
                const uint32_t p = by[k] & (COUNTED - 1);
                x[k] = t.x[p];
                word[k] = t.mask != nullptr ? __ldg(t.mask + (p >> 5)) : ~0u;
            }
            float z[NAMES];
            #pragma unroll
            for (int k = 0; k < NAMES; ++k) {
                const uint32_t p = by[k] & (COUNTED - 1);
                z[k] = (float)x[k];
                if (TABLES && chunk >= 0) {
                    const int m = min(chunk * CHUNK + 32 * k + lane, names - 1);
                    const float scaled = z[k] > 0.f ? __fdiv_rn(z[k], repetition) : __fmul_rn(z[k], repetition);
                    if (by[k] & COUNTED) z[k] = __fsub_rn(scaled, penalty[m]);
                    if (by[k] & LISTED) z[k] = __fadd_rn(z[k], __uint_as_float(entry[m]));
                }
                if ((by[k] & NONE) || !(word[k] >> (p & 31) & 1)) z[k] = NEG_INF;
                if (!PICK && !(by[k] & NONE)) t.y[p] = (T)(__fmul_rn(z[k], warm));
            }
            if constexpr (PICK) {
                const float top = largest(z);
                if (__any_sync(0xffffffffu, !(top < (MARGIN<KIND> ? best.s : best.m)) && top != NEG_INF))
                    move_best<KIND>(best, z, top, [&](int k) { return v0 + (int)(by[k] & (COUNTED - 1)); }, kk);
                add_weights<KIND, NAMES>(best, z, kk);
                finish(s_item[r][STREAM + 1 + chunk]);
            }
        }
    }
    if constexpr (PICK) {
        __syncthreads();
        // a warp a row: the CTA's result to the cluster's first CTA, then all of them
        Best best = nothing<KIND>();
        if (warp < rows) {
            for (int i = lane; i < STREAM + 1 + CHUNKS; i += 32) join<KIND>(best, s_item[warp][i], kk);
            join_lanes<KIND>(best, kk);
        }
        if (cut.cluster > 1) {
            asm volatile("barrier.cluster.wait;" ::: "memory");               // the first CTA runs
            if (lane == 0 && warp < rows)
                asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};"
                             :: "r"(mapa_shared(smem_addr(&s_row[warp][rank]), 0)),
                                "r"(__float_as_uint(best.m)), "r"(best.at), "r"(__float_as_uint(best.l)),
                                "r"(__float_as_uint(best.s)) : "memory");
            __syncwarp();
            asm volatile("barrier.cluster.arrive.release;" ::: "memory");
            if (rank != 0) return;
            asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
            if (warp >= rows) return;
            best = nothing<KIND>();
            if (lane < cut.cluster) best = s_row[warp][lane];
            join_lanes<KIND>(best, kk);
        }
        if (warp >= rows || lane != 0) return;
        const size_t to = (size_t)row0 + first + warp;
        const bool none = best.m == NEG_INF;
        a.token[to] = none ? -1 : best.at;
        if (a.confidence != nullptr) {
            float c = __fdiv_rn(1.f, best.l);
            if (MARGIN<KIND>) c = __fdiv_rn(-expm1f((best.s - best.m) * warm), best.l);
            if (ENTROPY<KIND>) c = __fdiv_rn(best.s, best.l) * LN2 - logf(best.l);
            a.confidence[to] = none ? 0.f : c;
        }
        // (an infinite maximum has no differences to it: l is NaN, the sum of the exponentials is not)
        if (a.lse != nullptr)
            a.lse[to] = none || best.m == -NEG_INF ? best.m : fmaf(best.m, warm, logf(best.l));
    }
}

template <typename T, int KIND, bool TABLES>
cudaError_t launch_kernel(const LogitsArgs& a, cudaStream_t s) {
    // Up to eight rows of a sequence a CTA, and as many slices as fill the
    // GPU or leave a CTA 1024 tokens of each row.
    Cut c;
    c.groups = (a.max_new + ROWS - 1) / ROWS;
    c.rows = (a.max_new + c.groups - 1) / c.groups;
    c.parts_log = c.rows % 8 == 0 ? 0 : c.rows % 4 == 0 ? 1 : c.rows % 2 == 0 ? 2 : 3;      // every warp has as many
    c.parts = 1 << c.parts_log;
    const long long units = (long long)a.B * c.groups, target = 2ll * num_sms();
    c.cluster = 1;
    if (KIND == APPLY) c.cluster = (int)std::max<long long>(1, std::min<long long>(target / units, (a.V + 2047) / 2048));
    else
        while (c.cluster < MAX_CLUSTER && units * c.cluster < target && a.V > 2048 * c.cluster) c.cluster *= 2;
    const long long names = TABLES ? (long long)a.r.history_ld + a.r.bias_ld : 0;
    const int longest = names > NAMED ? NAMED : SLICE;
    const int rounds = (a.V + c.cluster * longest - 1) / (c.cluster * longest), cuts = c.cluster * rounds;
    c.len = std::min(longest, ((a.V + cuts - 1) / cuts + 31) / 32 * 32);
    c.room = (int)std::min<long long>(c.len, (names + 3) / 4 * 4);
    if (units * c.cluster >= (1ll << 31)) return cudaErrorInvalidValue;
    size_t smem = 0;
    if (TABLES || a.r.allowed != nullptr) smem = (size_t)c.rows * (c.len / 32) * 4;
    if (TABLES) smem += (size_t)c.room * 12 + (size_t)c.len * 4 + (c.len / 32) * 8 + 16;
    static DeviceCache<int> ready;
    int dummy = 0;
    cudaError_t e = ready.get(&dummy, [](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(logits_kernel<T, KIND, TABLES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    NAMED * 12 + SLICE * 4 + (SLICE / 32) * (8 + 4 * ROWS) + 16);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * c.cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2] = {pdl_attribute(), {}};
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)c.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = KIND != APPLY && c.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, logits_kernel<T, KIND, TABLES>, a, c);
}

template <typename T, int KIND>
cudaError_t launch_tables(const LogitsArgs& a, cudaStream_t s) {
    return a.r.history != nullptr || a.r.bias_ids != nullptr ? launch_kernel<T, KIND, true>(a, s)
                                                             : launch_kernel<T, KIND, false>(a, s);
}

template <typename T>
cudaError_t launch_typed(const LogitsArgs& a, cudaStream_t s) {
    switch (a.kind) {
        case APPLY: return launch_tables<T, APPLY>(a, s);
        case STARQ_CONFIDENCE_PROBABILITY: return launch_tables<T, STARQ_CONFIDENCE_PROBABILITY>(a, s);
        case STARQ_CONFIDENCE_MARGIN: return launch_tables<T, STARQ_CONFIDENCE_MARGIN>(a, s);
        default: return launch_tables<T, STARQ_CONFIDENCE_ENTROPY>(a, s);
    }
}

}  // namespace

cudaError_t launch_logits(const LogitsArgs& a, cudaStream_t s) {
    switch (a.dtype) {
        case STARQ_F16: return launch_typed<__half>(a, s);
        case STARQ_BF16: return launch_typed<__nv_bfloat16>(a, s);
        default: return launch_typed<float>(a, s);
    }
}

}  // namespace starq
