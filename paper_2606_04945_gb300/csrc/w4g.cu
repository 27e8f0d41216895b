// Products of a few rows with 4-bit weights that carry one scale per group
// of input channels (weight-only quantisation: the activations stay 16-bit).
//
//   Y[i][n] = sum_k x[i][k] s[n][k / group] q[n][k] (+ bias[n])
//
// Bound by memory: the weights are read once for all rows (K / 2 + 4 K /
// group bytes a channel) and one row needs two operations a weight. The
// products run on the 16-bit MMA, weights as the 16-row operand and eight
// activation rows as the columns: with one row the MMA is idle seven eighths
// of the time and still far from the bound.
//
// A code c enters the MMA as the fp16 subnormal c 2^-24: one three-input
// operation takes two codes out of a word and flips their sign bits, which is
// (c + 8) 2^-24, and one subtraction is exact; the result is multiplied by
// 2^24 at the end. The upper codes of a byte come out as c 2^-20 and have a
// sum of their own that is divided by 16. The products are exact as well,
// a group's sum is accumulated in float32 and only then multiplied by its
// scale. bf16 activations become fp16, a row's 128 channels of a block scaled
// by a power of two that puts the largest at 2^14: what lies 2^-29 below
// that one loses its last bits, which is under the float32 sum's own.
// The k order inside an MMA is free: a thread takes the eight codes of a word
// and the activations are paired to match.
//
// A warp owns 16 output channels and a slice of K, and nothing in its loop
// waits for another warp: codes and scales come into a ring of its own by
// asynchronous 16- and 4-byte copies. A cluster of CTAs shares the slices and
// adds up at its end, through each other's shared memory, in the order of the
// slices. So a CTA brings and converts its slice of the activations only,
// once. Measured at K = 12288, N = 4096, groups of 32, 12 rows (31.8 MB):
// 13.9 us, 2.3 TB/s; with the warps of one CTA taking the blocks of K in turn
// for 16 channels, all of them needing all activations, 25.7 us with the
// codes in registers, 31 us with 512-byte bulk copies. One row at K = 3584,
// N = 37888, groups of 64 (76.5 MB): 17.8 us, 4.3 TB/s, against 22.3 and 29
// us. About 5 us of each call are its start, the activations and the joining:
// K = N = 4096 (8.9 MB) takes 5.7 us. Four stages of two CTAs an SM suffice:
// 6 or 8 of them, or a third CTA, changed nothing. 32 rows at K = 3584, N =
// 37888 take 43 us, 200 TFLOP/s: there the loads of the activations from
// shared memory and the conversions are the bound, not the MMA. (Leaving the
// 8 of c + 8 in the products and starting each sum from -8 sum x takes an
// operation a pair less, but loads more, is not exact, and took 50 us there.)
#include <algorithm>
#include <type_traits>

#include "decode.cuh"

namespace starq {
namespace {

constexpr int TILE = 16;               // output channels of a warp
constexpr int KB = 128;                // input channels of a block
constexpr int STAGES = 4;              // blocks of a warp on their way
constexpr int MAX_SLICES = 8;          // CTAs of a cluster
constexpr int X_ROW = KB * 2;          // bytes of an activation row in a block
constexpr int CODES = TILE * KB / 2;   // bytes of a stage's codes
template <int GROUP> constexpr int STAGE = CODES + TILE * (KB / GROUP) * 4;       // and of its scales behind them

// A CTA of W warps: 16 instead of 8 where several tiles of activations make
// their conversion, which the warps share, a large part of the work.
template <int W> struct Cta {
    static constexpr int THREADS = W * 32;
    static constexpr int N = W * TILE;               // output channels
    static constexpr int PER_SM = 16 / W;
    static constexpr int SMEM = 220 * 1024 / PER_SM;
    static constexpr int PART_ROW = N + 4;           // floats of a row of partial sums
};
template <int GROUP, int W> constexpr int RING = W * STAGES * STAGE<GROUP>;

template <typename T> constexpr bool IS_HALF = std::is_same<T, __half>::value;

// d = a b + c (c may be d).
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0,
                                          float c1, float c2, float c3) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                 "{%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// Two codes of a word as fp16 numbers c 2^-24 (c 2^-20 with the fields four
// bits up): (w & mask) ^ flip in one operation is the subnormal (c + 8) 2^-24,
// and `flip` is also the pair of subnormals to subtract. Both steps are exact.
// (With constants as immediates the compiler makes two operations of the
// first: a third of all instructions were these.)
__device__ __forceinline__ uint32_t codes(uint32_t w, uint32_t mask, uint32_t flip) {
    uint32_t r;
    asm("{\n\t.reg .b32 u;\n\tlop3.b32 u, %1, %2, %3, 0x6a;\n\tsub.rn.f16x2 %0, u, %3;\n\t}"
        : "=r"(r) : "r"(w), "r"(mask), "r"(flip));
    return r;
}

// Eight activations as four fp16 pairs (x0, x4), (x2, x6), (x1, x5), (x3, x7).
__device__ __forceinline__ uint4 paired(const float (&f)[8]) {
    uint4 v;
    const __half2 a = __floats2half2_rn(f[0], f[4]), b = __floats2half2_rn(f[2], f[6]);
    const __half2 c = __floats2half2_rn(f[1], f[5]), d = __floats2half2_rn(f[3], f[7]);
    v.x = *reinterpret_cast<const uint32_t*>(&a);
    v.y = *reinterpret_cast<const uint32_t*>(&b);
    v.z = *reinterpret_cast<const uint32_t*>(&c);
    v.w = *reinterpret_cast<const uint32_t*>(&d);
    return v;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory");
}

// 16-byte chunk c (of 4) of row r of a stage: rows that are read together
// fall into different banks.
template <int GROUP> __device__ __forceinline__ int w_offset(int r, int c) {
    const int key = GROUP == 128 ? 0 : GROUP == 64 ? r & 2 : (r >> 1) & 3;
    return r * (KB / 2) + ((c ^ key) << 4);
}

// 16-byte chunk c (of 16) of activation row i of a block; the four threads
// and the two rows that are read together fall into different chunks of 128
// bytes. A reader's row is one of 8 next to each other: its parity is the
// thread's, and with it the chunks' order.
template <int GROUP> __device__ __forceinline__ uint32_t x_offset(int i, int c) {
    const int odd = i & 1;
    const int key = GROUP == 128 ? 2 * odd ^ ((c >> 3) & 1) : GROUP == 64 ? odd : 4 * odd;
    return i * X_ROW + ((c ^ key) << 4);
}
// Activation rows that a block has room for: with one tile the rows there
// are, or else whole tiles (rows past L are read and not stored).
template <int NT> __host__ __device__ __forceinline__ int x_rows(int L) { return NT == 1 ? L : 8 * NT; }

template <int NT> constexpr int POW_ROW = 8 * NT * 4;                              // powers of two of a block, bytes

// NT tiles of 8 activation rows. A cluster of `slices` CTAs takes Cta::N output
// channels, each CTA `per` blocks of K; the activations of `chunk` of them are
// in shared memory at a time.
template <typename T, int GROUP, int NT, int W>
__global__ void __launch_bounds__(Cta<W>::THREADS, Cta<W>::PER_SM) w4g_linear_kernel(const W4gArgs a, int slices, int per, int chunk) {
    constexpr int GB = KB / GROUP;                   // groups of a block
    constexpr int GW = GROUP / 32;                   // words of a thread in a group
    constexpr int COLS = 8 * NT, THREADS = Cta<W>::THREADS, CTA_N = Cta<W>::N;
    constexpr int PART_ROW = Cta<W>::PART_ROW;
    extern __shared__ __align__(128) uint8_t smem[];
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int blocks = (a.K + KB - 1) / KB, groups = a.K / GROUP;
    const int rank = blockIdx.x % slices, n0 = blockIdx.x / slices * CTA_N, nw = n0 + warp * TILE;
    const int k0 = min(rank * per, blocks), k1 = min(k0 + per, blocks);
    uint8_t* const ring = smem + warp * STAGES * STAGE<GROUP>;
    const int xblock = x_rows<NT>(a.L) * X_ROW;      // bytes of a block's activations
    uint8_t* const xs = smem + RING<GROUP, W>;
    float* const pows = reinterpret_cast<float*>(xs + chunk * xblock);               // [chunk][COLS]

    // --- a warp's weights: 16 rows of 64 bytes and their scales a block ---------
    const uint8_t* src[2];
    #pragma unroll
    for (int h = 0; h < 2; ++h)
        src[h] = a.Wq + (size_t)min(nw + 8 * h + g, a.N - 1) * (size_t)(a.K / 2) + 16 * t;
    const float* ssrc[(GB + 1) / 2];
    #pragma unroll
    for (int h = 0; h < (GB + 1) / 2; ++h)
        ssrc[h] = a.scales + (size_t)min(nw + (lane + 32 * h) / GB % TILE, a.N - 1) * groups + lane % GB;
    auto fetch = [&](int kb, int st) {
        const uint32_t to = smem_addr(ring + st * STAGE<GROUP>);
        if (kb < k1) {
            const bool real = kb * KB + 32 * t < a.K;          // K is a multiple of 32: a chunk is in or out
            #pragma unroll
            for (int h = 0; h < 2; ++h)
                copy16(to + w_offset<GROUP>(8 * h + g, t), src[h] + (real ? (size_t)kb * (KB / 2) : 0), real);
            const bool group = kb * GB + lane % GB < groups;
            #pragma unroll
            for (int h = 0; h < (GB + 1) / 2; ++h)
                if (GB > 1 || lane < TILE)
                    copy4(to + CODES + 4 * (lane + 32 * h), ssrc[h] + (group ? kb * GB : 0), group);
        }
        copies_commit();
    };
    #pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(k0 + i, i);

    // --- the chunk's activations: 16 threads a row of a block ------------------
    auto bring = [&](int c0) {
        constexpr int BATCH = 4;                     // loads of a thread on their way together
        const int pieces = min(chunk, k1 - c0) * a.L * 16;
        const int hop = THREADS / 16 / a.L, skip = THREADS / 16 - hop * a.L;       // blocks and rows of a step
        int b0 = (int)threadIdx.x / 16 / a.L, i0 = (int)threadIdx.x / 16 - b0 * a.L;
        for (int e0 = threadIdx.x; e0 < pieces; e0 += BATCH * THREADS) {
            uint4 raw[BATCH];
            int blk[BATCH], tok[BATCH];
            #pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int e = e0 + u * THREADS, c = e & 15;
                blk[u] = b0;
                tok[u] = i0;
                b0 += hop;
                i0 += skip;
                if (i0 >= a.L) { i0 -= a.L; ++b0; }
                const int k = (c0 + blk[u]) * KB + 8 * c;
                raw[u] = make_uint4(0, 0, 0, 0);
                if (e < pieces && k < a.K) raw[u] = ld_global_nc_v4(static_cast<const T*>(a.X) + (size_t)tok[u] * a.ldx + k);
            }
            #pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (e0 + u * THREADS >= pieces) break;
                const int c = e0 & 15, b = blk[u], i = tok[u];
                float f[8];
                Eight<T>::load(reinterpret_cast<const T*>(&raw[u]), f);
                float down = 1.f;
                // the 16 threads of a row are half a warp (the last round may have one half only)
                const unsigned half = 0xffffu << (lane & 16);
                if (!IS_HALF<T>) {
                    float top = 0.f;
                    #pragma unroll
                    for (int v = 0; v < 8; ++v) top = fmaxf(top, fabsf(f[v]));
                    #pragma unroll
                    for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(half, top, d));
                    const int ex = max((int)(__float_as_uint(top) >> 23) - 127, -112);
                    const float up = __uint_as_float((uint32_t)(14 - ex + 127) << 23);          // 2^(14 - ex)
                    down = __uint_as_float((uint32_t)(ex - 14 + 127) << 23);
                    #pragma unroll
                    for (int v = 0; v < 8; ++v) f[v] *= up;
                }
                *reinterpret_cast<uint4*>(xs + b * xblock + x_offset<GROUP>(i, c)) = paired(f);
                if (!IS_HALF<T> && c == 0) pows[b * COLS + i] = down;
            }
        }
    };
    // constants of the fields, kept in registers
    uint32_t m0 = 0x000f000fu, f0 = 0x00080008u, m1 = 0x00f000f0u, f1 = 0x00800080u;
    asm volatile("" : "+r"(m0), "+r"(f0), "+r"(m1), "+r"(f1));

    float acc[NT][4];
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][c] = 0.f;
    // this thread's activations: row g of a tile; chunks of the first group,
    // word by word (of the first two groups, where a group is one word)
    const int xrow = NT == 1 ? min(g, a.L - 1) : g;
    constexpr int XO = GW == 1 ? 2 : GW;
    uint32_t xo[XO];
    #pragma unroll
    for (int e = 0; e < XO; ++e) xo[e] = x_offset<GROUP>(xrow, GW == 1 ? t + 4 * e : GW * t + e);
    int st = 0, to = STAGES - 1;
    for (int c0 = k0; c0 < k1; c0 += chunk) {
        if (c0 != k0) __syncthreads();               // the last chunk is done with
        bring(c0);
        __syncthreads();
        const int c1 = min(c0 + chunk, k1);
        for (int kb = c0; kb < c1; ++kb) {
            copies_wait<STAGES - 2>();
            __syncwarp();                            // everyone's copies are in, and the stage before is done with
            fetch(kb + STAGES - 1, to);
            if (++to == STAGES) to = 0;
            const uint8_t* const ws = ring + st * STAGE<GROUP>;
            if (++st == STAGES) st = 0;
            const uint8_t* const xb = xs + (kb - c0) * xblock;
            float sc[2][GB];
            #pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float* p = reinterpret_cast<const float*>(ws + CODES) + (8 * h + g) * GB;
                if (GB == 4) *reinterpret_cast<float4*>(sc[h]) = *reinterpret_cast<const float4*>(p);
                else if (GB == 2) *reinterpret_cast<float2*>(sc[h]) = *reinterpret_cast<const float2*>(p);
                else sc[h][0] = *p;
            }
            float sum[NT][4];                        // of the block, before the powers of two
            #pragma unroll
            for (int j = 0; j < GB; ++j) {
                uint32_t w[2][4];
                #pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // bytes GROUP / 2 j + GROUP / 8 t of the row
                    const int at = GROUP / 2 * j + GROUP / 8 * t;
                    const uint8_t* p = ws + w_offset<GROUP>(8 * h + g, at >> 4) + (at & 15);
                    if (GROUP == 128) *reinterpret_cast<uint4*>(w[h]) = *reinterpret_cast<const uint4*>(p);
                    else if (GROUP == 64) *reinterpret_cast<uint2*>(w[h]) = *reinterpret_cast<const uint2*>(p);
                    else w[h][0] = *reinterpret_cast<const uint32_t*>(p);
                }
                float lo[NT][4], hi[NT][4];
                #pragma unroll
                for (int e = 0; e < GW; ++e) {
                    const uint32_t w0 = w[0][e], w1 = w[1][e], v0 = w0 >> 8, v1 = w1 >> 8;
                    const uint32_t ev[4] = {codes(w0, m0, f0), codes(w1, m0, f0), codes(v0, m0, f0), codes(v1, m0, f0)};
                    const uint32_t od[4] = {codes(w0, m1, f1), codes(w1, m1, f1), codes(v0, m1, f1), codes(v1, m1, f1)};
                    #pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const uint4 x = *reinterpret_cast<const uint4*>(
                            xb + 8 * i * X_ROW + (GW == 1 ? xo[j & 1] + 128 * (j >> 1) : xo[e] + GROUP * 2 * j));
                        float(&l)[4] = lo[i], (&h)[4] = hi[i];
                        if (e == 0) {
                            mma_16816(l, ev, x.x, x.y, 0.f, 0.f, 0.f, 0.f);
                            mma_16816(h, od, x.z, x.w, 0.f, 0.f, 0.f, 0.f);
                        } else {
                            mma_16816(l, ev, x.x, x.y, l[0], l[1], l[2], l[3]);
                            mma_16816(h, od, x.z, x.w, h[0], h[1], h[2], h[3]);
                        }
                    }
                }
                #pragma unroll
                for (int i = 0; i < NT; ++i)
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float v = fmaf(hi[i][k], 0.0625f, lo[i][k]), s = sc[k >> 1][j];
                        if (IS_HALF<T>) acc[i][k] = fmaf(v, s, acc[i][k]);
                        else sum[i][k] = j == 0 ? v * s : fmaf(v, s, sum[i][k]);
                    }
            }
            if (!IS_HALF<T>)
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const float2 pw = *reinterpret_cast<const float2*>(pows + (kb - c0) * COLS + 8 * i + 2 * t);
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][k] = fmaf(sum[i][k], k & 1 ? pw.y : pw.x, acc[i][k]);
                }
        }
    }

    // --- the cluster adds up, in the order of the slices -------------------------
    copies_wait<0>();
    __syncthreads();                                 // the rings are done with
    float* const part = reinterpret_cast<float*>(smem);          // [L][PART_ROW]
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = 8 * i + 2 * t + (k & 1);
            if (row < a.L) part[row * PART_ROW + warp * TILE + g + 8 * (k >> 1)] = acc[i][k];
        }
    if (slices > 1) cluster_sync();
    else __syncthreads();
    for (int e = rank * THREADS + threadIdx.x; e < a.L * CTA_N; e += slices * THREADS) {
        const int row = e / CTA_N, nn = e % CTA_N, n = n0 + nn;
        if (n >= a.N) continue;
        float y = 0.f;
        if (slices == 1) y = part[row * PART_ROW + nn];
        else {
            const uint32_t at = smem_addr(part + row * PART_ROW + nn);
            for (int q = 0; q < slices; ++q) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa_shared(at, q)) : "memory");
                y += v;
            }
        }
        y *= 16777216.f;                                         // 2^24
        if (a.bias != nullptr) y += __ldg(a.bias + n);
        const size_t at = (size_t)row * a.ldy + n;
        if (a.y_dtype == STARQ_F16) static_cast<__half*>(a.Y)[at] = __float2half_rn(y);
        else if (a.y_dtype == STARQ_BF16) static_cast<__nv_bfloat16*>(a.Y)[at] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.Y)[at] = y;
    }
    if (slices > 1) cluster_sync();                  // the sums stay until every CTA has read them
}

template <typename T, int GROUP, int NT, int W>
cudaError_t launch_ctas(const W4gArgs& a, cudaStream_t s) {
    using C = Cta<W>;
    const int blocks = (a.K + KB - 1) / KB, tiles = (a.N + C::N - 1) / C::N, slots = C::PER_SM * num_sms();
    // Slices of K: as few as fill the SMs, counted in blocks of
    // the busiest SM slot, a CTA's start and end counting as 4.
    int slices = 1, best = 0;
    for (int q = 1; q <= MAX_SLICES && q <= blocks; q *= 2) {
        const long long waves = ((long long)tiles * q + slots - 1) / slots;
        const long long cost = waves * ((blocks + q - 1) / q + 4);
        if (q == 1 || cost < best) { best = (int)std::min(cost, 0x7fffffffLL); slices = q; }
    }
    const int per = (blocks + slices - 1) / slices;
    const int xb = x_rows<NT>(a.L) * X_ROW + POW_ROW<NT>;       // bytes of a block's activations
    const int chunk = std::min(per, (C::SMEM - RING<GROUP, W>) / xb);
    const int smem = RING<GROUP, W> + chunk * xb;
    static DeviceCache<int> ready;
    int dummy = 0;
    cudaError_t e = ready.get(&dummy, [](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(w4g_linear_kernel<T, GROUP, NT, W>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    C::SMEM);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * slices));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)slices;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = slices > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, w4g_linear_kernel<T, GROUP, NT, W>, a, slices, per, chunk);
}

// Several tiles of activations and channels that fill the SMs without
// slices: 16 warps (measured at 32 rows, K = 3584, N = 37888: 50 us against
// 59 with 8, in an earlier form). With fewer channels the slices keep 8
// (clusters of whole SMs do not pack: 12 rows, K = 12288, N = 4096, in that
// form: 16 us against 30 with 16).
template <typename T, int GROUP, int NT>
cudaError_t launch_tiles(const W4gArgs& a, cudaStream_t s) {
    if constexpr (NT > 1)
        if (a.N >= num_sms() * Cta<16>::N * 3 / 4) return launch_ctas<T, GROUP, NT, 16>(a, s);
    return launch_ctas<T, GROUP, NT, 8>(a, s);
}

template <typename T, int GROUP>
cudaError_t launch_group(const W4gArgs& a, cudaStream_t s) {
    switch ((a.L + 7) / 8) {
        case 1: return launch_tiles<T, GROUP, 1>(a, s);
        case 2: return launch_tiles<T, GROUP, 2>(a, s);
        case 3: return launch_tiles<T, GROUP, 3>(a, s);
        default: return launch_tiles<T, GROUP, 4>(a, s);
    }
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
