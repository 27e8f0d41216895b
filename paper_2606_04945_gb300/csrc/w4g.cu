// Products of a few rows with 4-bit weights that carry one scale per group
// of input channels (weight-only quantisation: the activations stay 16-bit).
//
//   Y[i][n] = sum_k x[i][k] s[n][k / group] q[n][k] (+ bias[n])
//
// Bound by memory: the weights are read once for all rows (K / 2 + 4 K /
// group bytes a channel) and one row needs two operations a weight. The
// products run on the 16-bit MMA, weights as the 16-row operand and eight
// activation rows as the columns: with one row the MMA is idle seven
// eighths of the time and still far from the bound, and the CUDA cores are
// left to turn codes into 16-bit numbers. Codes are exact in fp16 and bf16,
// a group's sum is accumulated in float32 and only then multiplied by its
// scale, so no product is rounded before the float32 sums.
//
// A CTA owns 16 output channels; its warps take 128-channel blocks of K in
// turn and meet once at the end in shared memory, in warp order. The k order
// inside an MMA is free: a thread takes the eight nibbles of one word, pairs
// nibble i with nibble i + 4 (one AND puts both into the halves of a
// register), and the activations are paired the same way.
#include <type_traits>

#include "decode.cuh"

namespace starq {
namespace {

constexpr int WARPS = 8;
constexpr int THREADS = WARPS * 32;
constexpr int TILE_N = 16;             // output channels of a CTA
constexpr int KB = 128;                // input channels of a warp's block
constexpr int AHEAD = 4;               // blocks in flight per warp

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
    if (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Nibbles I and I + 4 of a word (two's complement) as a pair of 16-bit
// numbers: the nibble with its sign bit flipped is c + 8; put under the
// exponent of 1024 (fp16) or 128 (bf16), whose last place is 1, it reads
// 1024 + c + 8, and one exact subtraction leaves c.
template <typename T, int I>
__device__ __forceinline__ uint32_t nibble_pair(uint32_t w) {
    constexpr uint32_t magic = std::is_same<T, __half>::value ? 0x64086408u : 0x43084308u;
    const uint32_t u = ((w >> (4 * I)) & 0x000f000fu) ^ magic;
    uint32_t r;
    if (std::is_same<T, __half>::value) {
        const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&u),
                                  __half2half2(__ushort_as_half((unsigned short)0x6408)));       // 1032
        r = *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u),
                                         __bfloat162bfloat162(__ushort_as_bfloat16((unsigned short)0x4308)));   // 136
        r = *reinterpret_cast<const uint32_t*>(&v);
    }
    return r;
}

// Words of one weight row in a 128-channel block: sub-block j (of GROUP
// channels) gives thread t the GROUP / 32 words at channel GROUP j +
// GROUP / 4 t. Sub-blocks past K stay 0.
template <int GROUP>
__device__ __forceinline__ void load_words(uint32_t (&w)[4], const uint8_t* row, int k0, int K, int t) {
    #pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0;
    if (row == nullptr) return;
    #pragma unroll
    for (int j = 0; j < KB / GROUP; ++j) {
        const int k = k0 + GROUP * j;
        if (k < K) {
            const uint8_t* p = row + (k + GROUP / 4 * t) / 2;
            if (GROUP == 128) {
                const uint4 v = ld_global_nc_v4(p);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else if (GROUP == 64) {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
                w[2 * j] = v.x; w[2 * j + 1] = v.y;
            } else {
                w[j] = __ldg(reinterpret_cast<const uint32_t*>(p));
            }
        }
    }
}

// NT tiles of 8 activation rows.
template <typename T, int GROUP, int NT>
__global__ void __launch_bounds__(THREADS) w4g_linear_kernel(const W4gArgs a) {
    __shared__ float part[WARPS][NT][TILE_N][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * TILE_N;
    const int blocks = (a.K + KB - 1) / KB, groups = a.K / GROUP;
    const uint8_t* row[2];
    const float* srow[2];
    #pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int n = n0 + g + 8 * r;
        row[r] = n < a.N ? a.Wq + (size_t)n * (a.K / 2) : nullptr;
        srow[r] = a.scales + (size_t)(n < a.N ? n : 0) * groups;
    }
    float acc[NT][4];
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;

    for (int kb0 = warp; kb0 < blocks; kb0 += WARPS * AHEAD) {
        uint32_t w[AHEAD][2][4];
        float sc[AHEAD][2][KB / GROUP];
        #pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
            const int kb = kb0 + p * WARPS;
            #pragma unroll
            for (int r = 0; r < 2; ++r) {
                load_words<GROUP>(w[p][r], kb < blocks ? row[r] : nullptr, kb * KB, a.K, t);
                #pragma unroll
                for (int j = 0; j < KB / GROUP; ++j) {
                    const int grp = kb * (KB / GROUP) + j;
                    sc[p][r][j] = kb < blocks && grp < groups ? __ldg(srow[r] + grp) : 0.f;
                }
            }
        }
        #pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
            const int kb = kb0 + p * WARPS;
            if (kb >= blocks) break;
            #pragma unroll
            for (int j = 0; j < KB / GROUP; ++j) {
                const int k = kb * KB + GROUP * j + GROUP / 4 * t;
                if (kb * KB + GROUP * j >= a.K) break;
                float d[NT][4];
                #pragma unroll
                for (int i = 0; i < NT; ++i)
                    #pragma unroll
                    for (int c = 0; c < 4; ++c) d[i][c] = 0.f;
                #pragma unroll
                for (int e = 0; e < GROUP / 32; ++e) {
                    const uint32_t w0 = w[p][0][j * (GROUP / 32) + e], w1 = w[p][1][j * (GROUP / 32) + e];
                    const uint32_t p0 = nibble_pair<T, 0>(w0), p1 = nibble_pair<T, 1>(w0);
                    const uint32_t p2 = nibble_pair<T, 2>(w0), p3 = nibble_pair<T, 3>(w0);
                    const uint32_t q0 = nibble_pair<T, 0>(w1), q1 = nibble_pair<T, 1>(w1);
                    const uint32_t q2 = nibble_pair<T, 2>(w1), q3 = nibble_pair<T, 3>(w1);
                    #pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (8 * i + g < a.L)
                            x = ld_global_nc_v4(static_cast<const T*>(a.X) + (size_t)(8 * i + g) * a.ldx + k + 8 * e);
                        mma_16816<T>(d[i], p0, q0, p1, q1, prmt(x.x, x.z, 0x5410u), prmt(x.x, x.z, 0x7632u));
                        mma_16816<T>(d[i], p2, q2, p3, q3, prmt(x.y, x.w, 0x5410u), prmt(x.y, x.w, 0x7632u));
                    }
                }
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    acc[i][0] = fmaf(d[i][0], sc[p][0][j], acc[i][0]);
                    acc[i][1] = fmaf(d[i][1], sc[p][0][j], acc[i][1]);
                    acc[i][2] = fmaf(d[i][2], sc[p][1][j], acc[i][2]);
                    acc[i][3] = fmaf(d[i][3], sc[p][1][j], acc[i][3]);
                }
            }
        }
    }
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int c = 0; c < 4; ++c) part[warp][i][g + 8 * (c >> 1)][2 * t + (c & 1)] = acc[i][c];
    __syncthreads();
    for (int e = threadIdx.x; e < NT * 8 * TILE_N; e += THREADS) {
        const int n = e % TILE_N, i = e / TILE_N;
        if (i >= a.L || n0 + n >= a.N) continue;
        float y = 0.f;
        #pragma unroll
        for (int w = 0; w < WARPS; ++w) y += part[w][i >> 3][n][i & 7];
        if (a.bias != nullptr) y += __ldg(a.bias + n0 + n);
        const size_t at = (size_t)i * a.ldy + n0 + n;
        if (a.y_dtype == STARQ_F16) static_cast<__half*>(a.Y)[at] = __float2half_rn(y);
        else if (a.y_dtype == STARQ_BF16) static_cast<__nv_bfloat16*>(a.Y)[at] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.Y)[at] = y;
    }
}

template <typename T, int GROUP>
cudaError_t launch_group(const W4gArgs& a, cudaStream_t s) {
    const unsigned grid = (unsigned)((a.N + TILE_N - 1) / TILE_N);
    switch ((a.L + 7) / 8) {
        case 1: w4g_linear_kernel<T, GROUP, 1><<<grid, THREADS, 0, s>>>(a); break;
        case 2: w4g_linear_kernel<T, GROUP, 2><<<grid, THREADS, 0, s>>>(a); break;
        case 3: w4g_linear_kernel<T, GROUP, 3><<<grid, THREADS, 0, s>>>(a); break;
        default: w4g_linear_kernel<T, GROUP, 4><<<grid, THREADS, 0, s>>>(a); break;
    }
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_typed(const W4gArgs& a, cudaStream_t s) {
    switch (a.group) {
        case 32: return launch_group<T, 32>(a, s);
        case 64: return launch_group<T, 64>(a, s);
        default: return launch_group<T, 128>(a, s);
    }
}

}  // namespace

cudaError_t launch_w4g_linear(const W4gArgs& a, cudaStream_t s) {
    return a.dtype == STARQ_BF16 ? launch_typed<__nv_bfloat16>(a, s) : launch_typed<__half>(a, s);
}

}  // namespace starq
