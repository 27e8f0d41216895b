// Launcher interface of the cached-decoding operators (rope.cu, kvcache.cu,
// kvattn.cu, w4g.cu), called by the C ABI (api_decode.cu) after validation,
// and the device helpers that they share.
#pragma once

#include "common.cuh"

namespace starq {

// Status bit: a kernel met an index outside the array it indexes (a position
// beyond the rotary table, a page beyond the cache, lengths that do not fit
// their bounds) and skipped the access.
constexpr unsigned STATUS_RANGE = 1u << 8;

// A block's scale is at least this: log2 and reciprocal of every scale are
// then finite normal numbers.
constexpr float KV_SCALE_FLOOR = 7.888609052210118e-31f;   // 2^-100

struct RopeArgs {
    const void* X; void* Y; int dtype; int L; int ldx; int ldy; int heads; int D; int rot;
    int interleaved; int inverse;
    const int32_t* pos; const float2* table; int positions;
    unsigned* status;
};
cudaError_t launch_rope_table(float2* table, int positions, int rot, double theta, int scaling, double factor,
                              double original, double beta_fast, double beta_slow, double mscale, cudaStream_t s);
double rope_parts_mscale(double factor);   // 0.1 ln(factor) + 1
cudaError_t launch_rope_apply(const RopeArgs& a, cudaStream_t s);

struct KvAppendArgs {
    starq_kv_cache c;
    const void* K; int ldk; const void* V; int ldv;
    const void* Q; int ldq; void* Qo; int ldqo; int H;
    int dtype; int T;
    const int32_t* seq_start; const int32_t* past; int B; int max_new;
    const int32_t* page_table; int table_ld;
    const int32_t* pos; const float2* table; int positions; int rot; int interleaved;
    unsigned* status;
};
cudaError_t launch_kv_append(const KvAppendArgs& a, cudaStream_t s);

struct KvReadArgs {
    starq_kv_cache c;
    const int32_t* page_table; int table_ld;
    const int32_t* first; const int32_t* out_start; int B; int max_rows; int T;
    void* K; void* V; int ld; int dtype;
    unsigned* status;
};
cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s);

struct KvAttnArgs {
    starq_kv_cache c;
    const void* Q; int ldq; int dtype; int T;
    const int32_t* seq_start; int B; int max_new; int H;
    const int32_t* page_table; int table_ld;
    const int32_t* kv_len; int max_len;
    int causal; const uint8_t* key_mask; int mask_ld;
    float scale;
    void* Out; int ldo; float* lse;
    void* workspace;
    unsigned* status;
    int whole;                       // units are not cut (set by the launcher)
};
size_t kv_attention_workspace_bytes(int B, int max_new, int H, int Hkv, int D);
cudaError_t launch_kv_attention(const KvAttnArgs& a, cudaStream_t s);

struct W4gArgs {
    const void* X; int ldx; int dtype; int L; int K;
    const uint8_t* Wq; const float* scales; int group; int N; const float* bias;
    void* Y; int ldy; int y_dtype;
};
cudaError_t launch_w4g_linear(const W4gArgs& a, cudaStream_t s);

// A launch whose kernel begins with grid_dependency_wait(): its CTAs are
// brought up while the kernel before it drains. (These kernels do not let
// their own dependents start early: measured slower, the waiting CTAs take
// room and issue slots.)
template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at = pdl_attribute();
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Eight values of an element type to and from float32 (one rounding).
template <typename T> struct Eight;
template <> struct Eight<__half> {
    static __device__ __forceinline__ void load(const __half* p, float (&f)[8]) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const __half2* h = reinterpret_cast<const __half2*>(&w);
        #pragma unroll
        for (int k = 0; k < 4; ++k) { const float2 v = __half22float2(h[k]); f[2 * k] = v.x; f[2 * k + 1] = v.y; }
    }
    static __device__ __forceinline__ void store(__half* p, const float (&f)[8]) {
        uint4 w;
        __half2* h = reinterpret_cast<__half2*>(&w);
        #pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
        *reinterpret_cast<uint4*>(p) = w;
    }
};
template <> struct Eight<__nv_bfloat16> {
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&f)[8]) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
        #pragma unroll
        for (int k = 0; k < 4; ++k) { const float2 v = __bfloat1622float2(h[k]); f[2 * k] = v.x; f[2 * k + 1] = v.y; }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&f)[8]) {
        uint4 w;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
        #pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
        *reinterpret_cast<uint4*>(p) = w;
    }
};
template <> struct Eight<float> {
    static __device__ __forceinline__ void load(const float* p, float (&f)[8]) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
};

// Eight values as they lie in memory: half the registers of Eight's floats
// while loads are on their way.
template <typename T> struct Packed8 {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
        #pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void open(float (&f)[8]) const { Eight<T>::load(reinterpret_cast<const T*>(w), f); }
};

// One rotation unit: 16 channels of a head that hold eight rotation pairs,
// i = 8 u .. 8 u + 7. Half layout: the vectors at 8 u and rot / 2 + 8 u
// (pair (lo[k], hi[k])); interleaved: the 16 channels from 16 u on (pairs of
// neighbours). Channels of unit u start at unit_lo / unit_hi.
__device__ __forceinline__ int rope_unit_lo(int u, int interleaved) { return interleaved ? 16 * u : 8 * u; }
__device__ __forceinline__ int rope_unit_hi(int u, int rot, int interleaved) {
    return interleaved ? 16 * u + 8 : rot / 2 + 8 * u;
}

// (a, b) -> (a c - b s, b c + a s), products and sums each rounded to
// float32, so that the result is the plain formula's bit for bit.
__device__ __forceinline__ void rope_pair(float& a, float& b, float c, float s) {
    const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
    const float y = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
    a = x; b = y;
}
__device__ __forceinline__ void rope_unit(float (&lo)[8], float (&hi)[8], const float2 (&cs)[8], int interleaved) {
    if (interleaved) {
        #pragma unroll
        for (int k = 0; k < 4; ++k) rope_pair(lo[2 * k], lo[2 * k + 1], cs[k].x, cs[k].y);
        #pragma unroll
        for (int k = 0; k < 4; ++k) rope_pair(hi[2 * k], hi[2 * k + 1], cs[4 + k].x, cs[4 + k].y);
    } else {
        #pragma unroll
        for (int k = 0; k < 8; ++k) rope_pair(lo[k], hi[k], cs[k].x, cs[k].y);
    }
}
// cos and sin of the unit's eight pairs at position p; identity (and the
// status bit) for a position outside the table.
__device__ __forceinline__ void rope_load(float2 (&cs)[8], const float2* __restrict__ table, int positions, int rot,
                                          int p, int u, int inverse, unsigned* status) {
    if (p < 0 || p >= positions) {
        atomicOr(status, STATUS_RANGE);
        #pragma unroll
        for (int k = 0; k < 8; ++k) cs[k] = make_float2(1.f, 0.f);
        return;
    }
    const float4* t = reinterpret_cast<const float4*>(table + (size_t)p * (rot / 2) + 8 * u);
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 v = __ldg(t + k);
        cs[2 * k] = make_float2(v.x, inverse ? -v.y : v.y);
        cs[2 * k + 1] = make_float2(v.z, inverse ? -v.w : v.w);
    }
}

}  // namespace starq
