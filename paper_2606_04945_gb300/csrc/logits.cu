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
// vocabulary in memory: a CTA counts its slice's tokens in shared memory
// (counters, list entries, and a bit for each token that has either), and
// only tokens whose bit is set look at them. A CTA takes up to eight rows of
// a sequence, which share the tables of a slice, a row or part of it a warp.
// A cluster shares the slices; its first CTA joins the warps' results, in
// their order. A thread moves its maximum only when 16 bytes of values pass
// it, so a value costs an exponential and a few operations.
#include <algorithm>

#include "logits.cuh"

namespace starq {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int SLICE = 8192;            // tokens of a table
constexpr int MAX_CLUSTER = 8;
constexpr int UNROLL = 4;              // 16-byte loads of a thread on their way
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

enum { APPLY = -1 };                   // else a starq_confidence

// What is known of some of a row's tokens: largest z (its lowest index), sum
// of 2^d, and the second largest z or sum of 2^d d.
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

// A 16-byte piece of a row.
template <typename T> constexpr int SE = 16 / (int)sizeof(T);
__device__ __forceinline__ void open(const uint4& w, float (&z)[4]) {
    z[0] = __uint_as_float(w.x); z[1] = __uint_as_float(w.y); z[2] = __uint_as_float(w.z); z[3] = __uint_as_float(w.w);
}
template <typename T> __device__ __forceinline__ void open_as(const uint4& w, float (&z)[SE<T>]) {
    if constexpr (sizeof(T) == 4) open(w, z);
    else Eight<T>::load(reinterpret_cast<const T*>(&w), z);
}

// Bits e .. e + 31 of a row of bits that starts at e = 0 (e > -32), words
// behind `count` read as 0.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int count, int e) {
    if (e < 0) return words[0] << -e;
    const int w = e >> 5, sh = e & 31;
    uint32_t b = words[w] >> sh;
    if (sh > 24 && w + 1 < count) b |= words[w + 1] << (32 - sh);        // (8 bits are asked for)
    return b;
}

template <typename T, int KIND, bool TABLES>
__global__ void __launch_bounds__(THREADS) logits_kernel(const LogitsArgs a, int rows_per_cta, int cluster, int groups,
                                                        int len) {
    constexpr int E = SE<T>;
    constexpr bool PICK = KIND != APPLY;
    constexpr uint32_t FULL = (1u << E) - 1;
    extern __shared__ __align__(16) uint32_t tables[];       // counters [len], list entries [len], bits [len / 32 + 1]
    __shared__ Best s_best[MAX_CLUSTER * WARPS];
    uint32_t* const count = tables;
    uint32_t* const entry = tables + len;
    uint32_t* const named = tables + 2 * len;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int unit = (int)(blockIdx.x / (unsigned)cluster), rank = (int)(blockIdx.x % (unsigned)cluster);
    const int b = unit / groups, first = (unit - b * groups) * rows_per_cta;

    grid_dependency_wait();
    const int row0 = __ldg(a.seq_start + b), n = __ldg(a.seq_start + b + 1) - row0;
    if (n < 0 || n > a.max_new || row0 < 0 || row0 > a.T - n) {
        if (tid == 0) atomicOr(a.status, STATUS_RANGE);
        return;                                              // (the whole cluster does)
    }
    if (first >= n) return;
    if (PICK && cluster > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");

    float temperature = 1.f, repetition = 1.f, presence = 0.f, frequency = 0.f;
    if (a.r.params != nullptr) {
        const float* p = a.r.params + 4 * (size_t)b;
        temperature = __ldg(p); repetition = __ldg(p + 1); presence = __ldg(p + 2); frequency = __ldg(p + 3);
        const bool t_ok = temperature >= 1e-30f && temperature <= 1e30f, r_ok = repetition >= 1e-30f && repetition <= 1e30f;
        if (!(t_ok && r_ok)) {
            if (tid == 0) atomicOr(a.status, STATUS_RANGE);
            if (!t_ok) temperature = 1.f;
            if (!r_ok) repetition = 1.f;
        }
    }
    const float warm = __fdiv_rn(1.f, temperature), kk = warm * LOG2E;
    int told = 0, entries = 0;                               // tokens of the history, entries of the list
    if (TABLES) {
        if (a.r.history != nullptr) {
            told = __ldg(a.r.history_len + b);
            if (told < 0 || told > a.r.history_ld) {
                if (tid == 0) atomicOr(a.status, STATUS_RANGE);
                told = 0;
            }
        }
        if (a.r.bias_ids != nullptr) {
            entries = __ldg(a.r.bias_len + b);
            if (entries < 0 || entries > a.r.bias_ld) {
                if (tid == 0) atomicOr(a.status, STATUS_RANGE);
                entries = 0;
            }
        }
    }
    const int32_t* history = a.r.history + (size_t)b * a.r.history_ld;
    const int32_t* ids = a.r.bias_ids + (size_t)b * a.r.bias_ld;
    const float* values = a.r.bias_values + (size_t)b * a.r.bias_ld;

    const int share = WARPS / rows_per_cta;                  // warps of a row
    const int mine = first + warp / share, part = warp % share;
    const bool live = mine < n;
    const size_t row = (size_t)row0 + (live ? mine : 0);
    const uint32_t* mask = nullptr;
    if (a.r.allowed != nullptr) mask = a.r.allowed + (a.r.allowed_by_row ? row : (size_t)b) * a.r.allowed_ld;
    Best best = nothing<KIND>();

    for (int v0 = rank * len; v0 < a.V; v0 += cluster * len) {
        const int here = min(len, a.V - v0);
        if (TABLES) {
            __syncthreads();                                 // the tables of the slice before are done with
            for (int i = tid; i < len / 2; i += THREADS) reinterpret_cast<uint4*>(tables)[i] = make_uint4(0, 0, 0, 0);
            for (int i = tid; i < len / 32 + 1; i += THREADS) named[i] = 0;
            __syncthreads();
            #pragma unroll 4
            for (int i = tid; i < told; i += THREADS) {
                const int v = __ldg(history + i), p = v - v0;
                if (v < 0 || v >= a.V) atomicOr(a.status, STATUS_RANGE);
                else if (p >= 0 && p < here) {
                    atomicAdd(count + p, 1u);
                    atomicOr(named + (p >> 5), 1u << (p & 31));
                }
            }
            for (int i = tid; i < entries; i += THREADS) {
                const int v = __ldg(ids + i), p = v - v0;
                if (v < 0 || v >= a.V) atomicOr(a.status, STATUS_RANGE);
                else if (p >= 0 && p < here) {
                    atomicMax(entry + p, (uint32_t)i + 1);   // the last of a token's entries counts
                    atomicOr(named + (p >> 5), 1u << (p & 31));
                }
            }
            __syncthreads();
        }
        if (!live) continue;
        const T* x = static_cast<const T*>(a.X) + row * a.ldx + v0;
        T* y = PICK ? nullptr : static_cast<T*>(a.Y) + row * a.ldy + v0;
        // pieces are 16-byte aligned; the first begins up to E - 1 tokens before the slice
        const int ahead = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T)) & (E - 1);
        const bool wide = !PICK && ((int)(reinterpret_cast<uintptr_t>(y) / sizeof(T)) & (E - 1)) == ahead;
        const int pieces = (here + ahead + E - 1) / E;
        const uint32_t* words = mask != nullptr ? mask + (v0 >> 5) : nullptr;
        const int word_count = (here + 31) >> 5;
        for (int j0 = part * 32 + lane; j0 - lane < pieces; j0 += share * 32 * UNROLL) {
            uint4 w[UNROLL];
            uint32_t ok[UNROLL];
            #pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int e0 = (j0 + u * share * 32) * E - ahead;
                ok[u] = 0;
                w[u] = make_uint4(0, 0, 0, 0);
                if (e0 >= 0 && e0 + E <= here) {
                    w[u] = *reinterpret_cast<const uint4*>(x + e0);
                    ok[u] = FULL;
                } else if (e0 < here) {                      // the slice's ends, token by token
                    T t[E];
                    #pragma unroll
                    for (int k = 0; k < E; ++k) {
                        t[k] = T(0.f);
                        if (e0 + k >= 0 && e0 + k < here) { t[k] = x[e0 + k]; ok[u] |= 1u << k; }
                    }
                    memcpy(&w[u], t, 16);
                }
            }
            if (words != nullptr) {
                #pragma unroll
                for (int u = 0; u < UNROLL; ++u)
                    if (ok[u]) ok[u] &= bits_at(words, word_count, (j0 + u * share * 32) * E - ahead);
            }
            #pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int e0 = (j0 + u * share * 32) * E - ahead;
                if (e0 >= here) break;
                float z[E];
                open_as<T>(w[u], z);
                if (TABLES) {
                    const uint32_t touched = bits_at(named, len / 32 + 1, e0) & ok[u];
                    if (touched) {
                        #pragma unroll
                        for (int k = 0; k < E; ++k)
                            if (touched >> k & 1) {
                                const uint32_t c = count[e0 + k], i = entry[e0 + k];
                                if (c) {
                                    z[k] = z[k] > 0.f ? __fdiv_rn(z[k], repetition) : __fmul_rn(z[k], repetition);
                                    z[k] = __fsub_rn(z[k], __fadd_rn(__fmul_rn(frequency, (float)c), presence));
                                }
                                if (i) z[k] = __fadd_rn(z[k], __ldg(values + (i - 1)));
                            }
                    }
                }
                #pragma unroll
                for (int k = 0; k < E; ++k)
                    if (!(ok[u] >> k & 1)) z[k] = NEG_INF;
                if constexpr (!PICK) {
                    T t[E];
                    #pragma unroll
                    for (int k = 0; k < E; ++k) t[k] = (T)(__fmul_rn(z[k], warm));
                    if (wide && e0 >= 0 && e0 + E <= here) {
                        uint4 o;
                        memcpy(&o, t, 16);
                        *reinterpret_cast<uint4*>(y + e0) = o;
                    } else {
                        #pragma unroll
                        for (int k = 0; k < E; ++k)
                            if (e0 + k >= 0 && e0 + k < here) y[e0 + k] = t[k];
                    }
                } else {
                    float top = z[0];
                    #pragma unroll
                    for (int k = 1; k < E; ++k) top = max_nan(top, z[k]);
                    if (!(top <= (KIND == STARQ_CONFIDENCE_MARGIN ? best.s : best.m))) {
                        const float old = best.m;
                        #pragma unroll
                        for (int k = 0; k < E; ++k) {
                            if (z[k] > best.m || (z[k] != z[k] && best.m == best.m)) {
                                if (KIND == STARQ_CONFIDENCE_MARGIN) best.s = best.m;
                                best.m = z[k];
                                best.at = v0 + e0 + k;
                            } else if (KIND == STARQ_CONFIDENCE_MARGIN) {
                                best.s = fmaxf(best.s, z[k]);
                            }
                        }
                        if (old != NEG_INF) {
                            const float d = old == best.m ? 0.f : (old - best.m) * kk, f = ex2(d);
                            if (KIND == STARQ_CONFIDENCE_ENTROPY) best.s = f > 0.f ? f * fmaf(best.l, d, best.s) : 0.f;
                            best.l *= f;
                        }
                    }
                    const float ref = best.m == NEG_INF ? 0.f : best.m;
                    #pragma unroll
                    for (int k = 0; k < E; ++k) {
                        const float d = (z[k] - ref) * kk, e = ex2(d);
                        best.l += e;
                        if (KIND == STARQ_CONFIDENCE_ENTROPY) best.s = fmaf(e, fmaxf(d, -1000.f), best.s);
                    }
                }
            }
        }
    }
    if constexpr (PICK) {
        if (live) join_lanes<KIND>(best, kk);
        // every warp's result to the cluster's first CTA: [row][rank][part]
        const int slot = (warp / share) * (cluster * share) + rank * share + part;
        if (cluster > 1) {
            asm volatile("barrier.cluster.wait;" ::: "memory");               // it runs
            if (lane == 0)
                asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};"
                             :: "r"(mapa_shared(smem_addr(&s_best[slot]), 0)), "r"(__float_as_uint(best.m)), "r"(best.at),
                                "r"(__float_as_uint(best.l)), "r"(__float_as_uint(best.s)) : "memory");
            __syncwarp();
            asm volatile("barrier.cluster.arrive.release;" ::: "memory");
            if (rank != 0) return;
            asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        } else {
            if (lane == 0) s_best[slot] = best;
            __syncthreads();
        }
        const int i = first + warp;
        if (warp >= rows_per_cta || i >= n) return;
        const int results = cluster * share;
        best = nothing<KIND>();
        for (int q = lane; q < results; q += 32) join<KIND>(best, s_best[warp * results + q], kk);
        join_lanes<KIND>(best, kk);
        if (lane != 0) return;
        const size_t to = (size_t)row0 + i;
        const bool none = best.m == NEG_INF;
        a.token[to] = none ? -1 : best.at;
        if (a.confidence != nullptr) {
            float c = __fdiv_rn(1.f, best.l);
            if (KIND == STARQ_CONFIDENCE_MARGIN) c = __fdiv_rn(-expm1f((best.s - best.m) * warm), best.l);
            if (KIND == STARQ_CONFIDENCE_ENTROPY) c = __fdiv_rn(best.s, best.l) * LN2 - logf(best.l);
            a.confidence[to] = none ? 0.f : c;
        }
        // (an infinite maximum has no differences to it: l is NaN, the sum of the exponentials is not)
        if (a.lse != nullptr) a.lse[to] = none || best.m == -NEG_INF ? best.m : fmaf(best.m, warm, logf(best.l));
    }
}

template <typename T, int KIND, bool TABLES>
cudaError_t launch_kernel(const LogitsArgs& a, cudaStream_t s) {
    // How the rows and the vocabulary are cut. A sequence's rows share a
    // CTA's tables, so with tables a CTA takes as many rows as leave enough
    // CTAs; a cluster as large as leaves a CTA 1024 tokens.
    const long long target = 4ll * num_sms();
    auto units = [&](int rows) { return (long long)a.B * ((a.max_new + rows - 1) / rows); };
    int rows = 1, cluster = 1;
    if (TABLES)
        while (rows < WARPS && rows < a.max_new && units(2 * rows) * MAX_CLUSTER >= target) rows *= 2;
    while (cluster < MAX_CLUSTER && units(rows) * cluster < target && a.V > 2048 * cluster) cluster *= 2;
    const int rounds = (a.V + cluster * SLICE - 1) / (cluster * SLICE);
    const int len = std::min(SLICE, ((a.V + cluster * rounds - 1) / (cluster * rounds) + 31) / 32 * 32);
    if (units(rows) * cluster >= (1ll << 31)) return cudaErrorInvalidValue;
    const size_t smem = TABLES ? (size_t)len * 8 + (len / 32 + 1) * 4 : 0;
    static DeviceCache<int> ready;
    int dummy = 0;
    cudaError_t e = ready.get(&dummy, [](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(logits_kernel<T, KIND, TABLES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    SLICE * 8 + (SLICE / 32 + 1) * 4);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units(rows) * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2] = {pdl_attribute(), {}};
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = KIND != APPLY && cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, logits_kernel<T, KIND, TABLES>, a, rows, cluster,
                              (a.max_new + rows - 1) / rows, len);
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
