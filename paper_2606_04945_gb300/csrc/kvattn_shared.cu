// Attention over the cache for sequences that share a prefix: the prefix is
// read once for all rows of its sequences.
//
//   o_i = (sum over the shared slots + sum over the sequence's own) p_ij v_j / l_i
//
// Two passes of the attention kernels (KV_SPLIT) and a join. In the first the
// rows of a group's sequences are the rows of one: with S sequences of n new
// tokens a key meets S n G rows at once, so the cache's bytes fall by S and
// the tensor cores are filled (one token of 32 sequences with 7 query heads a
// key/value head: 224 of a unit's 256 rows, where each sequence by itself has
// 7 of 16). The second takes each sequence's slots behind the prefix. Both
// leave sums relative to a row's running maximum; the join adds a row's runs of
// both, in their order.
#include <algorithm>

#include "kvattn.cuh"

namespace starq {
namespace {

constexpr int TILE = 128;              // keys of a tile of either kernel

// One row's runs in one pass.
struct Runs {
    const float* acc;                  // of the first run, this row
    const float* ml;
    size_t step;                       // from a run's slot to the next run's
    size_t second;                     // 1: the first run's slot is its CTA's second (else 0)
    int count;
};

template <int D>
__device__ __forceinline__ Runs runs_of(const KvAttnArgs& a, const KvCut& cut, int G, const SeqShape& s, int b, int i,
                                        int head) {
    Runs r = {nullptr, nullptr, 0, 0, 0};
    if (s.n <= 0 || s.nt <= 0) return r;
    const int h = head / G, row = i * G + (head - h * G);
    const size_t at = (size_t)(s.row0 + i) * a.H + head;
    r.acc = a.sums + at * D;
    r.ml = a.sums + (size_t)a.T * a.H * D + 2 * at;
    r.count = 1;
    if (cut.whole) return r;
    const int tile = row / cut.rows, rr = row - tile * cut.rows, tiles = (s.n * G + cut.rows - 1) / cut.rows;
    const long long total = cut.prefix[a.B], share = quotient(total + cut.ctas - 1, cut.ctas);
    const long long u0 = cut.prefix[b] + ((long long)h * tiles + tile) * s.nt;
    int c0, c1;
    if (total < (1ll << 31)) {
        c0 = (int)((unsigned)u0 / (unsigned)share);
        c1 = (int)((unsigned)(u0 + s.nt - 1) / (unsigned)share);
    } else {
        c0 = (int)(u0 / share);
        c1 = (int)((u0 + s.nt - 1) / share);
    }
    if (c0 == c1) return r;                               // one run covered the unit
    r.count = c1 - c0 + 1;
    r.step = 2 * slot_floats(cut.slot_rows, D);
    r.second = u0 > (long long)c0 * share ? slot_floats(cut.slot_rows, D) : 0;
    r.acc = cut.slots + c0 * r.step + (size_t)rr * D;
    r.ml = cut.slots + c0 * r.step + (size_t)cut.slot_rows * D + 2 * rr;
    return r;
}

template <typename T, int D, int SHARE>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
kv_attention_split_join_kernel(const KvAttnArgs pre, const KvCut pre_cut, const KvAttnArgs own, const KvCut own_cut, int G) {
    constexpr int PER = D / 32, AT_ONCE = 4;
    __shared__ float s_acc[SHARE > 1 ? SHARE : 1][D];
    __shared__ float2 s_ml[SHARE > 1 ? SHARE : 1];
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % SHARE;
    const int b = blockIdx.y;
    const SeqShape s = seq_shape<16, TILE, KV_SPLIT>(own, G, b, false);
    const int idx = blockIdx.x * (JOIN_WARPS / SHARE) + warp / SHARE;      // token * H + head
    const int i = idx / own.H, head = idx - i * own.H;
    if (i >= s.n) return;
    const size_t row = (size_t)(s.row0 + i);
    Runs from[2] = {{nullptr, nullptr, 0, 0, 0}, runs_of<D>(own, own_cut, G, s, b, i, head)};
    const int g = group_of(own, b);
    if (g >= 0) {
        const SeqShape p = seq_shape<16, TILE, KV_SPLIT>(pre, G, g, false);
        const int at = s.row0 + i - p.row0;               // (outside only where the starts are not in order)
        if (at >= 0 && at < p.n) from[0] = runs_of<D>(pre, pre_cut, G, p, g, at, head);
    }
    float top = NEG_INF, l = 0.f, acc[PER];
    #pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] = 0.f;
    #pragma unroll 1
    for (int q = 0; q < 2; ++q) {
        const Runs& r = from[q];
        for (int c = part; c < r.count; c += AT_ONCE * SHARE) {
            float2 ml[AT_ONCE];
            float v[AT_ONCE][PER];
            #pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int cu = c + u * SHARE;
                ml[u] = make_float2(NEG_INF, 0.f);
                #pragma unroll
                for (int k = 0; k < PER; ++k) v[u][k] = 0.f;
                if (cu < r.count) {
                    const size_t off = cu * r.step + (cu == 0 ? r.second : 0);
                    ml[u] = *reinterpret_cast<const float2*>(r.ml + off);
                    #pragma unroll
                    for (int k = 0; k < PER; k += 2) {
                        const float2 w = *reinterpret_cast<const float2*>(r.acc + off + lane * PER + k);
                        v[u][k] = w.x; v[u][k + 1] = w.y;
                    }
                }
            }
            float to = top;
            #pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) to = fmaxf(to, ml[u].x);
            const float f0 = top == to ? 1.f : ex2(top - to);
            top = to;
            l *= f0;
            #pragma unroll
            for (int k = 0; k < PER; ++k) acc[k] *= f0;
            #pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const float f = ml[u].x == top ? 1.f : ex2(ml[u].x - top);
                l = fmaf(ml[u].y, f, l);
                #pragma unroll
                for (int k = 0; k < PER; ++k) acc[k] = fmaf(v[u][k], f, acc[k]);
            }
        }
    }
    if (SHARE > 1) {                                      // one row a CTA: the warps' results
        #pragma unroll
        for (int k = 0; k < PER; ++k) s_acc[part][lane * PER + k] = acc[k];
        if (lane == 0) s_ml[part] = make_float2(top, l);
        __syncthreads();
        if (part != 0) return;
        float to = NEG_INF;
        #pragma unroll
        for (int w = 0; w < SHARE; ++w) to = fmaxf(to, s_ml[w].x);
        top = to;
        l = 0.f;
        #pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] = 0.f;
        #pragma unroll
        for (int w = 0; w < SHARE; ++w) {
            const float2 ml = s_ml[w];
            const float f = ml.x == top ? 1.f : ex2(ml.x - top);
            l = fmaf(ml.y, f, l);
            #pragma unroll
            for (int k = 0; k < PER; ++k) acc[k] = fmaf(s_acc[w][lane * PER + k], f, acc[k]);
        }
    }
    const float inv = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
    T* out = static_cast<T*>(own.Out) + row * own.ldo + (size_t)head * D + lane * PER;
    #pragma unroll
    for (int k = 0; k < PER; ++k) out[k] = (T)(l == 0.f ? 0.f : acc[k] * inv);
    if (lane == 0 && own.lse != nullptr)
        own.lse[row * own.H + head] = l == 0.f ? NEG_INF : (log2f(l) + (top - HEAD)) * 0.6931471805599453f;
}

template <typename T, int D>
cudaError_t launch_split_join(const KvAttnArgs& pre, const KvCut& pc, const KvAttnArgs& own, const KvCut& oc,
                              cudaStream_t s) {
    const int G = own.H / own.c.Hkv;
    const size_t rows = (size_t)own.max_new * own.H;
    if (rows * own.B <= 4 * (size_t)num_sms())            // up to four CTAs an SM
        return launch_overlapped(kv_attention_split_join_kernel<T, D, JOIN_WARPS>, dim3((unsigned)rows, (unsigned)own.B),
                                 JOIN_WARPS * 32, 0, s, pre, pc, own, oc, G);
    return launch_overlapped(kv_attention_split_join_kernel<T, D, 1>,
                             dim3((unsigned)((rows + JOIN_WARPS - 1) / JOIN_WARPS), (unsigned)own.B), JOIN_WARPS * 32, 0,
                             s, pre, pc, own, oc, G);
}

constexpr size_t align256(size_t n) { return (n + 255) / 256 * 256; }
size_t sums_bytes(int T, int H, int D) { return align256((size_t)T * H * (D + 2) * 4); }

}  // namespace

// The two passes' own workspaces, then their rows' sums.
size_t kv_attention_shared_workspace_bytes(int T, int B, int max_new, int groups, int max_rows, int H, int Hkv, int D) {
    return align256(kv_attention_workspace_bytes(B, max_new, H, Hkv, D)) +
           align256(kv_attention_workspace_bytes(groups, max_rows, H, Hkv, D)) + 2 * sums_bytes(T, H, D);
}

cudaError_t launch_kv_attention_shared(const KvAttnArgs& a, int max_rows, int max_shared, cudaStream_t s) {
    // nothing is shared, as far as the bounds tell
    if (a.groups == 0 || max_rows <= a.max_new || max_shared == 0) return launch_kv_attention(a, s);
    const int H = a.H, Hkv = a.c.Hkv, D = a.c.D;
    uint8_t* w = static_cast<uint8_t*>(a.workspace);
    KvAttnArgs own = a, pre = a;
    own.sequences = pre.sequences = a.B;
    own.prefix = 0;
    own.likely_len = std::max(1, a.max_len - max_shared);
    w += align256(kv_attention_workspace_bytes(a.B, a.max_new, H, Hkv, D));
    pre.workspace = w;
    w += align256(kv_attention_workspace_bytes(a.groups, max_rows, H, Hkv, D));
    own.sums = reinterpret_cast<float*>(w);
    pre.sums = reinterpret_cast<float*>(w + sums_bytes(a.T, H, D));
    pre.prefix = 1;
    pre.B = a.groups;
    pre.max_new = max_rows;
    pre.max_len = pre.likely_len = max_shared;
    pre.causal = 0;                                       // a shared slot lies before all new tokens
    auto pass = [&](KvAttnArgs& p, KvCut* cut) {
        const cudaError_t e = kv_attention_by_warps(p) ? launch_kv_attention_warp<KV_SPLIT>(p, cut, s)
                                                       : launch_kv_attention_tc<KV_SPLIT>(p, cut, s);
        p.whole = cut->whole;
        return e;
    };
    KvCut pc, oc;
    cudaError_t e = pass(pre, &pc);
    if (e != cudaSuccess || (e = pass(own, &oc)) != cudaSuccess) return e;
    if (a.dtype == STARQ_BF16)
        return D == 64 ? launch_split_join<__nv_bfloat16, 64>(pre, pc, own, oc, s)
                       : launch_split_join<__nv_bfloat16, 128>(pre, pc, own, oc, s);
    return D == 64 ? launch_split_join<__half, 64>(pre, pc, own, oc, s) : launch_split_join<__half, 128>(pre, pc, own, oc, s);
}

}  // namespace starq
