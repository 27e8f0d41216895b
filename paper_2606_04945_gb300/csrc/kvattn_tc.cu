// Attention over the paged 8-bit cache for more than 16 query rows of a
// key/value head (blocks of positions under denoising, drafted runs with
// grouped heads): both products on tcgen05. The mathematics is kvattn.cu's.
//
// With R rows a cached key costs 4 R D operations for 2 D bytes, so from
// about 100 rows on the tensor cores' work outweighs the cache's bytes; the
// warp-level MMA would be the bound from 24 rows on. What has to be fed is
// fp16 tiles: four warps read a tile's codes (128 keys) straight from their
// pages, turn them into fp16 and store them as 128-byte-swizzled tiles, keys
// and values alike; the value product takes its tile as an MN-major operand,
// so no transposition is needed.
//
// A unit is up to 256 rows. Two streams, each with 128 TMEM lanes of rows,
// its own scores, weights and accumulators, and four softmax warps (one
// thread a row), run half a step apart, so that one stream's products hide
// behind the other's exponentials. With more than 128 rows the streams are
// the unit's two row tiles and share every key tile; otherwise they take the
// key tiles in turn, with the same rows, and their results are joined in
// shared memory at the end. Weights replace the scores they came from in
// TMEM (A operand from tensor memory). Warps without rows skip the softmax.
#include <algorithm>

#include "kvattn.cuh"

namespace starq {
namespace {

constexpr unsigned STATUS_TIMEOUT_KVATTN = 1u << 5;
constexpr int ROWS = 256;                          // rows of a unit
constexpr int TILE = 128;                          // keys of a tile, rows of a stream
constexpr int SOFT_WARPS = 8, CONV_WARPS = 4;
constexpr int MMA_WARP = SOFT_WARPS + CONV_WARPS;
constexpr int THREADS = (MMA_WARP + 1) * 32;
constexpr int CONV_THREADS = CONV_WARPS * 32;
constexpr int STAGES = 2;
constexpr uint32_t TM_S = 0, TM_O = 256;           // TMEM columns: two score tiles, two accumulators
constexpr int BLOCKS = TILE / 16;                  // 16-key blocks of a tile (each inside one page)

struct TileInfo {                                  // what the softmax needs of a key tile
    float4 blk[BLOCKS];                            // log2(e) scale s_k, log2 s_v, 1 / s_v
    float bias[TILE];                              // with a key mask: 0, or -inf for a key that is not seen
    int key0, edge;                                // first key; whether keys past the length or a mask concern it
};

struct Shared {
    uint64_t k_full[STAGES], k_empty[STAGES], v_full[STAGES], v_empty[STAGES], info[STAGES];
    uint64_t q_full, s_full[2], p_full[2], pv_done[2], meet;
    uint32_t tmem_base;
    int abort;
    alignas(16) TileInfo tile[STAGES];
    float2 ml[TILE];                               // the odd stream's (m, l) for the join of the two
};

template <int D> struct Layout {
    static constexpr int TILE_BYTES = TILE * D * 2;                  // fp16, 64-channel halves of 16 KB
    static constexpr int HALF = TILE * 128;
    static constexpr int Q = 0, K = 2 * TILE_BYTES, V = K + STAGES * TILE_BYTES, END = V + STAGES * TILE_BYTES;
    // the join of the two streams uses a 128 x D float32 area over Q (and, for
    // D = 64, exactly Q's two tiles)
    static constexpr int SMEM = END + 1024 + (int)sizeof(Shared);
};

// D (+)= A B, f16 inputs, A in TMEM, B in shared memory.
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// Descriptor of an MN-major operand in the 128-byte swizzle layout: each k
// (a key) is a row of 64 values (128 bytes), eight of them an atom; `half`
// bytes lead to the next 64 values.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr, uint32_t half) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(half >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 A, B, C, D;\n\t"
        "mov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\tmov.b64 C, {%6, %7};\n\t"
        "fma.rn.f32x2 D, A, B, C;\n\tmov.b64 {%0, %1}, D;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 16 codes of a row, channels 16 c .. 16 c + 15, as fp16 into row r of a
// tile. Threads whose channels lie in the upper half store their two chunks
// in the other order, so that a quarter warp covers all banks.
template <int D>
__device__ __forceinline__ void store_codes(uint32_t tile, int r, int c, const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t h[8];
    #pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[2 * i] = codes_half2(prmt(w[i], 0x64646464u, 0x4140u));
        h[2 * i + 1] = codes_half2(prmt(w[i], 0x64646464u, 0x4342u));
    }
    const uint32_t base = tile + (c >> 2) * (TILE * 128);
    const uint32_t lo = base + sw128_offset(r, 2 * (c & 3)), hi = base + sw128_offset(r, 2 * (c & 3) + 1);
    if (c >> 2) {
        st_shared_v4(hi, h[4], h[5], h[6], h[7]);
        st_shared_v4(lo, h[0], h[1], h[2], h[3]);
    } else {
        st_shared_v4(lo, h[0], h[1], h[2], h[3]);
        st_shared_v4(hi, h[4], h[5], h[6], h[7]);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 1) kv_attention_tc_kernel(const KvAttnArgs a, int G, int slot_rows,
                                                                    long long* prefix, float* slots) {
    using L = Layout<D>;
    using Cur = Cursor<ROWS, TILE>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    Shared* sh = reinterpret_cast<Shared*>(smem + L::END);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort = &sh->abort;
    auto B = [](const uint64_t& bar) { return smem_addr(&bar); };

    const Run run = find_run<ROWS, TILE, THREADS>(a, G, prefix);
    if (run.tau0 >= run.tau1) return;
    const int count = (int)(run.tau1 - run.tau0);

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(B(sh->k_full[i]), CONV_WARPS);
            mbar_init(B(sh->v_full[i]), CONV_WARPS);
            mbar_init(B(sh->info[i]), 1);
            mbar_init(B(sh->k_empty[i]), 1);
            mbar_init(B(sh->v_empty[i]), 1);
        }
        mbar_init(B(sh->q_full), SOFT_WARPS);
        mbar_init(B(sh->meet), SOFT_WARPS);
        for (int s = 0; s < 2; ++s) {
            mbar_init(B(sh->s_full[s]), 1);
            mbar_init(B(sh->p_full[s]), 4);
            mbar_init(B(sh->pv_done[s]), 1);
        }
        sh->abort = 0;
        mbar_fence_init();
    }
    if (warp == MMA_WARP) {
        tmem_alloc(smem_addr(&sh->tmem_base), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    bool ok = true;

    // Every role walks the run segment by segment (a segment is the run's
    // part of one unit). In a segment of n key tiles the streams' steps are
    // items: shared = 1 (more than 128 rows): item u is key tile u / 2 for
    // stream u & 1; shared = 0: key tile u for stream u & 1.
    Cur cur;
    cur.start(a, G, run);
    auto unit_rows = [&](const Cur& c) { return min(ROWS, c.s.n * G - c.rt * ROWS); };
    auto segment = [&](const Cur& c, int left) { return min(left, c.s.nt - c.kt); };

    if (warp >= SOFT_WARPS && warp < MMA_WARP) {
        // --- codes to fp16 tiles ------------------------------------------------
        const int ct = threadIdx.x - SOFT_WARPS * 32, cw = warp - SOFT_WARPS;
        constexpr int CPR = D / 16;                          // 16-code chunks of a row
        constexpr int PER = TILE * CPR / CONV_THREADS;       // chunks of a thread
        const int c = ct % CPR, r0 = ct / CPR;               // its channels, its rows r0 + RSTEP i
        constexpr int RSTEP = CONV_THREADS / CPR;
        uint4 kreg[PER], vreg[PER];
        const int shift = __ffs(a.c.page) - 1;
        const size_t row_of_head = (size_t)a.c.page * D;
        // page number of a key of the cursor's tile, -1 past the length or outside the cache
        auto page_of = [&](const Cur& q, int key) {
            if (key >= q.s.len) return -1;
            const int i = key >> shift;
            if (i >= a.table_ld) return -2;
            const int p = __ldg(a.page_table + (size_t)q.b * a.table_ld + i);
            return p < 0 || p >= a.c.pages ? -2 : p;
        };
        auto load = [&](const Cur& q, const uint8_t* src, uint4 (&reg)[PER]) {
            #pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int key = q.kt * TILE + r0 + RSTEP * i, p = page_of(q, key);
                reg[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);   // codes 0
                if (p >= 0)
                    reg[i] = ld_global_nc_v4(src + ((size_t)p * a.c.Hkv + q.h) * row_of_head +
                                             (size_t)(key & (a.c.page - 1)) * D + 16 * c);
            }
        };
        Cur nxt = cur;
        int left = count;
        load(nxt, a.c.K, kreg);
        load(nxt, a.c.V, vreg);
        for (int it = 0; it < count && ok; ++it) {
            const int st = it % STAGES;
            const uint32_t parity = (uint32_t)(it / STAGES) & 1u;
            cur = nxt;
            --left;
            if (++nxt.kt == nxt.s.nt && left > 0) nxt.next_unit(a, G);
            ok = mbar_wait_bounded_warp(B(sh->k_empty[st]), parity ^ 1u, abort);
            if (!ok) break;
            #pragma unroll
            for (int i = 0; i < PER; ++i) store_codes<D>(base + L::K + st * L::TILE_BYTES, r0 + RSTEP * i, c, kreg[i]);
            if (left > 0) load(nxt, a.c.K, kreg);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->k_full[st]));
            ok = mbar_wait_bounded_warp(B(sh->v_empty[st]), parity ^ 1u, abort);
            if (!ok) break;
            if (cw == 0) {
                // the tile's scales and mask (the values' stage is free, so the softmax is done with the last ones)
                TileInfo& ti = sh->tile[st];
                const int key0 = cur.kt * TILE;
                bool none = true;                            // this lane's 4 keys are all masked or past the length
                if (a.key_mask != nullptr) {
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + 4 * lane + i;
                        const bool see = key < cur.s.len &&
                                         __ldg(a.key_mask + (size_t)cur.b * a.mask_ld + key) != 0;
                        ti.bias[4 * lane + i] = see ? 0.f : NEG_INF;
                        none = none && !see;
                    }
                } else {
                    none = key0 + (lane & ~3) * 4 >= cur.s.len;
                }
                const unsigned hidden = __ballot_sync(0xffffffffu, none);
                if (lane < BLOCKS) {
                    float4 b = make_float4(0.f, 0.f, 1.f, 0.f);
                    if ((hidden >> (4 * lane) & 0xf) != 0xf) {   // some key counts
                        const int p = page_of(cur, key0 + 16 * lane);
                        if (p >= 0) {
                            const size_t blk = (size_t)p * a.c.Hkv + cur.h;
                            const float sv = __ldg(a.c.v_scale + blk), vs = sv < KV_SCALE_FLOOR ? KV_SCALE_FLOOR : sv;
                            b = make_float4(__ldg(a.c.k_scale + blk) * (a.scale * 1.4426950408889634f), __log2f(vs),
                                            __fdividef(1.f, vs), 0.f);
                        } else {
                            atomicOr(a.status, STATUS_RANGE);
                            b.x = __uint_as_float(0x7fffffffu);
                        }
                    }
                    ti.blk[lane] = b;
                }
                if (lane == 0) {
                    ti.key0 = key0;
                    ti.edge = a.key_mask != nullptr || key0 + TILE > cur.s.len ||
                              (a.causal && key0 + TILE > cur.s.len - cur.s.n + 1);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(B(sh->info[st]));
            }
            #pragma unroll
            for (int i = 0; i < PER; ++i) store_codes<D>(base + L::V + st * L::TILE_BYTES, r0 + RSTEP * i, c, vreg[i]);
            if (left > 0) load(nxt, a.c.V, vreg);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->v_full[st]));
        }
        // the last use of every stage has been given back, so no commit lands after this CTA has exited
        for (int st = 0; st < STAGES && ok; ++st) {
            const int uses = (count - st + STAGES - 1) / STAGES;
            if (uses > 0)
                ok = mbar_wait_bounded_warp(B(sh->k_empty[st]), (uint32_t)(uses - 1) & 1u, abort) &&
                     mbar_wait_bounded_warp(B(sh->v_empty[st]), (uint32_t)(uses - 1) & 1u, abort);
        }
        if (!ok && lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
    } else if (warp == MMA_WARP) {
        // --- the products ---------------------------------------------------------
        constexpr uint32_t IDESC_QK = (1u << 4) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
        constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
        int left = count, tile0 = 0, steps[2] = {0, 0};      // key tiles and stream steps before the segment
        int seg = 0;
        while (left > 0 && ok) {
            const int n = segment(cur, left);
            const int shared = unit_rows(cur) > TILE;
            const int items = shared ? 2 * n : n;
            ok = mbar_wait_bounded_warp(B(sh->q_full), (uint32_t)seg & 1u, abort);
            auto qk = [&](int u) {
                const int kt = tile0 + (shared ? u >> 1 : u), st = kt % STAGES, s = u & 1;
                if (!mbar_wait_bounded_warp(B(sh->k_full[st]), (uint32_t)(kt / STAGES) & 1u, abort)) return false;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t qd = smem_desc_sw128(base + L::Q + (shared ? s : 0) * L::TILE_BYTES);
                    const uint64_t kd = smem_desc_sw128(base + L::K + st * L::TILE_BYTES);
                    #pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t off = (uint64_t)(((k >> 2) * L::HALF + (k & 3) * 32) >> 4);
                        mma_f16(tmem + TM_S + s * TILE, qd + off, kd + off, IDESC_QK, k > 0);
                    }
                    if (!shared || s == 1) tc_commit(B(sh->k_empty[st]));
                    tc_commit(B(sh->s_full[s]));
                }
                __syncwarp();
                return true;
            };
            for (int u = 0; u < 2 && u < items && ok; ++u) ok = qk(u);
            for (int u = 0; u < items && ok; ++u) {
                const int kt = tile0 + (shared ? u >> 1 : u), st = kt % STAGES, s = u & 1, step = u >> 1;
                ok = mbar_wait_bounded_warp(B(sh->p_full[s]), (uint32_t)(steps[s] + step) & 1u, abort) &&
                     mbar_wait_bounded_warp(B(sh->v_full[st]), (uint32_t)(kt / STAGES) & 1u, abort);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t vd = smem_desc_mn(base + L::V + st * L::TILE_BYTES, L::HALF);
                    #pragma unroll
                    for (int k = 0; k < TILE / 16; ++k)
                        mma_f16_ts(tmem + TM_O + s * TILE, tmem + TM_S + s * TILE + 8 * k, vd + (uint64_t)(k * 2048 >> 4),
                                   IDESC_PV, step > 0 || k > 0);
                    if (!shared || s == 1) tc_commit(B(sh->v_empty[st]));
                    tc_commit(B(sh->pv_done[s]));
                }
                __syncwarp();
                if (u + 2 < items) ok = qk(u + 2);
            }
            steps[0] += (items + 1) / 2;
            steps[1] += items / 2;
            tile0 += n;
            left -= n;
            ++seg;
            cur.kt += n;
            if (left > 0) cur.next_unit(a, G);
        }
        if (!ok && lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
    } else {
        // --- softmax: one thread a row ----------------------------------------------
        const int s = warp >> 2, row = threadIdx.x & (TILE - 1);
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;                      // TMEM lane quarter
        const uint32_t t_s = tmem + lanes + TM_S + s * TILE, t_o = tmem + lanes + TM_O + s * TILE;
        int left = count, tile0 = 0, steps = 0, meets = 0;
        // all softmax warps (bounded: a warp that gave up elsewhere ends the others' waits)
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->meet));
            const bool met = mbar_wait_bounded_warp(B(sh->meet), (uint32_t)meets & 1u, abort);
            ++meets;
            return met;
        };
        while (left > 0 && ok) {
            const int n = segment(cur, left), rows = unit_rows(cur);
            const int shared = rows > TILE;
            const int mine = shared ? n : (n - s + 1) / 2;                      // this stream's steps
            const int r = cur.rt * ROWS + (shared ? s * TILE : 0) + row;        // row of the unit's list
            const int i = r / G, head = cur.h * G + (r - i * G);
            const bool valid = (shared ? s * TILE : 0) + row < rows;
            const bool active = __any_sync(0xffffffffu, valid);
            const int lim = !valid ? 0 : a.causal ? max(0, cur.s.len - cur.s.n + i + 1) : cur.s.len;
            // the unit's query rows, as the A operand (with few rows both streams use the first tile)
            float down = 1.f;
            if (shared || s == 0 || !std::is_same<T, __half>::value) {
                uint4 raw4[D / 8];
                const T* src = static_cast<const T*>(a.Q) + (size_t)(cur.s.row0 + (valid ? i : 0)) * a.ldq +
                               (size_t)(valid ? head : 0) * D;
                #pragma unroll
                for (int k = 0; k < D / 8; ++k)
                    raw4[k] = valid ? *reinterpret_cast<const uint4*>(src + 8 * k) : make_uint4(0, 0, 0, 0);
                float up = 1.f;
                if (std::is_same<T, __nv_bfloat16>::value) {
                    float top = 0.f;
                    #pragma unroll
                    for (int k = 0; k < D / 8; ++k) {
                        float f[8];
                        Eight<T>::load(reinterpret_cast<const T*>(&raw4[k]), f);
                        #pragma unroll
                        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
                    }
                    row_power(top, up, down);
                }
                if (shared || s == 0) {
                    #pragma unroll
                    for (int k = 0; k < D / 8; ++k) {
                        uint4 v = raw4[k];
                        if (std::is_same<T, __nv_bfloat16>::value) {
                            float f[8];
                            Eight<T>::load(reinterpret_cast<const T*>(&raw4[k]), f);
                            #pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] *= up;
                            Eight<__half>::store(reinterpret_cast<__half*>(&v), f);
                        }
                        st_shared_v4(base + L::Q + s * L::TILE_BYTES + (k >> 3) * L::HALF + sw128_offset(row, k & 7), v.x,
                                     v.y, v.z, v.w);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->q_full));

            float m = NEG_INF, l = 0.f;
            for (int step = 0; step < mine && ok; ++step) {
                const int kt = tile0 + (shared ? step : 2 * step + s), st = kt % STAGES;
                ok = mbar_wait_bounded_warp(B(sh->s_full[s]), (uint32_t)(steps + step) & 1u, abort) &&
                     mbar_wait_bounded_warp(B(sh->info[st]), (uint32_t)(kt / STAGES) & 1u, abort);
                if (!ok) break;
                if (active) {
                    tc_fence_after();
                    const TileInfo& ti = sh->tile[st];
                    const bool edge = ti.edge != 0, masked = a.key_mask != nullptr;
                    const int see = lim - ti.key0;                              // keys [0, see) of the tile
                    float top = NEG_INF;
                    #pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t x[32];
                        tmem_ld_32x32b_x32(t_s + 32 * c, x);
                        tmem_ld_wait();
                        if (edge) {
                            #pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                const float bias = masked ? ti.bias[32 * c + k] : 0.f;
                                if (32 * c + k >= see || bias != 0.f) x[k] = 0xff800000u;
                            }
                        }
                        #pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            float t = __uint_as_float(x[16 * q]);
                            #pragma unroll
                            for (int k = 1; k < 15; k += 2)
                                t = max3(t, __uint_as_float(x[16 * q + k]), __uint_as_float(x[16 * q + k + 1]));
                            t = fmaxf(t, __uint_as_float(x[16 * q + 15]));
                            const float4 b = ti.blk[2 * c + q];
                            // a maximum of -inf: no key of the block is seen (its scale may be anything)
                            if (t != NEG_INF) top = fmaxf(top, fmaf(t, b.x * down, b.y));
                        }
                    }
                    if (__any_sync(0xffffffffu, top > m + LAZY)) {
                        const float to = fmaxf(m, top), f = m == to ? 1.f : ex2(m - to);
                        m = to;
                        l *= f;
                        if (step > 0) {
                            ok = mbar_wait_bounded_warp(B(sh->pv_done[s]), (uint32_t)(steps + step - 1) & 1u, abort);
                            if (!ok) break;
                            tc_fence_after();
                            #pragma unroll
                            for (int c = 0; c < D / 16; ++c) {
                                uint32_t o[16];
                                tmem_ld_32x32b_x16(t_o + 16 * c, o);
                                tmem_ld_wait();
                                #pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                                tmem_st_32x32b_x16(t_o + 16 * c, o);
                            }
                            tmem_st_wait();
                        }
                    }
                    const float sub = m == NEG_INF ? 0.f : m - HEAD;
                    float2 sum = make_float2(0.f, 0.f);
                    #pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t x[32], p[16];
                        tmem_ld_32x32b_x32(t_s + 32 * c, x);
                        tmem_ld_wait();
                        #pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float4 b = ti.blk[2 * c + q];
                            const float ax = b.x * down, cx = b.y - sub;
                            #pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const int e = 16 * q + 2 * k;
                                float2 v = fma2(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])),
                                                make_float2(ax, ax), make_float2(cx, cx));
                                v.x = ex2(v.x);
                                v.y = ex2(v.y);
                                float2 add = make_float2(b.z, b.z);
                                if (edge) {
                                    // a weight that does not count is 0 whatever its block's scale is
                                    const int key = 32 * c + e;
                                    if (key >= see || (masked && ti.bias[key] != 0.f)) v.x = add.x = 0.f;
                                    if (key + 1 >= see || (masked && ti.bias[key + 1] != 0.f)) v.y = add.y = 0.f;
                                }
                                sum = fma2(v, add, sum);
                                const __half2 h = __floats2half2_rn(v.x, v.y);
                                p[8 * q + k] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                        }
                        tmem_st_32x32b_x16(t_s + 16 * c, p);
                    }
                    l += sum.x + sum.y;
                    tmem_st_wait();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(B(sh->p_full[s]));
            }
            steps += mine;
            if (ok && mine > 0) ok = mbar_wait_bounded_warp(B(sh->pv_done[s]), (uint32_t)(steps - 1) & 1u, abort);
            if (!ok) break;
            tc_fence_after();
            // --- the segment's rows: the streams' join, then the output or a partial run ---
            const bool whole = cur.kt == 0 && n == cur.s.nt;
            float* join = reinterpret_cast<float*>(smem + L::Q);
            auto join_at = [&](int c) { return join + row * D + ((c ^ (row & (D / 4 - 1))) << 2); };    // float4 c
            if (!shared) {
                // both streams' products with Q are done, so its memory is free
                if (!(ok = meet())) break;
                if (s == 1 && active) {
                    #pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        if (mine > 0) {
                            tmem_ld_32x32b_x16(t_o + 16 * c, o);
                            tmem_ld_wait();
                        } else {
                            #pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = 0;
                        }
                        #pragma unroll
                        for (int k = 0; k < 4; ++k)
                            *reinterpret_cast<uint4*>(join_at(4 * c + k)) =
                                make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    }
                    sh->ml[row] = make_float2(m, l);
                }
                if (!(ok = meet())) break;
            }
            if (active && (shared || s == 0)) {
                float f0 = 1.f, f1 = 0.f;
                if (!shared) {
                    const float2 o = sh->ml[row];
                    const float top = fmaxf(m, o.x);
                    f0 = m == top ? 1.f : ex2(m - top);
                    f1 = o.x == top ? 1.f : ex2(o.x - top);
                    l = l * f0 + o.y * f1;
                    m = top;
                }
                const float inv = whole ? (l == 0.f ? 0.f : __fdiv_rn(1.f, l)) : 1.f;
                float* slot = slots + ((size_t)blockIdx.x * 2 + (tile0 == 0 ? 0 : 1)) * slot_floats(slot_rows, D);
                const int srow = (shared ? s * TILE : 0) + row;
                T* out = static_cast<T*>(a.Out) + (size_t)(cur.s.row0 + i) * a.ldo + (size_t)head * D;
                #pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t o[16];
                    tmem_ld_32x32b_x16(t_o + 16 * c, o);
                    tmem_ld_wait();
                    float f[16];
                    #pragma unroll
                    for (int k = 0; k < 16; ++k) f[k] = __uint_as_float(o[k]);
                    if (!shared) {
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float4 v = *reinterpret_cast<const float4*>(join_at(4 * c + k));
                            f[4 * k] = f[4 * k] * f0 + v.x * f1;
                            f[4 * k + 1] = f[4 * k + 1] * f0 + v.y * f1;
                            f[4 * k + 2] = f[4 * k + 2] * f0 + v.z * f1;
                            f[4 * k + 3] = f[4 * k + 3] * f0 + v.w * f1;
                        }
                    }
                    if (!valid) continue;
                    if (whole) {
                        float e[2][8];
                        #pragma unroll
                        for (int k = 0; k < 16; ++k) e[k >> 3][k & 7] = l == 0.f ? 0.f : f[k] * inv;
                        Eight<T>::store(out + 16 * c, e[0]);
                        Eight<T>::store(out + 16 * c + 8, e[1]);
                    } else {
                        #pragma unroll
                        for (int k = 0; k < 4; ++k)
                            *reinterpret_cast<float4*>(slot + (size_t)srow * D + 16 * c + 4 * k) =
                                make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
                    }
                }
                if (valid) {
                    if (!whole)
                        reinterpret_cast<float2*>(slot + (size_t)slot_rows * D)[srow] = make_float2(m, l);
                    else if (a.lse != nullptr)
                        a.lse[(size_t)(cur.s.row0 + i) * a.H + head] =
                            l == 0.f ? NEG_INF : (log2f(l) + (m - HEAD)) * 0.6931471805599453f;
                }
            }
            tc_fence_before();
            // the join area is Q's memory: read before the next unit's rows come in
            if (!shared && !(ok = meet())) break;
            tile0 += n;
            left -= n;
            cur.kt += n;
            if (left > 0) cur.next_unit(a, G);
        }
        if (!ok && lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) tmem_dealloc(tmem, 512);
}

template <typename T, int D>
cudaError_t launch_typed(const KvAttnArgs& a, cudaStream_t s) {
    const int G = a.H / a.c.Hkv;
    static DeviceCache<int> ready;
    int dummy = 0;
    cudaError_t e = ready.get(&dummy, [](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(kv_attention_tc_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    Layout<D>::SMEM);
    });
    if (e != cudaSuccess) return e;
    const int ctas = num_sms();
    const long long most = (long long)a.max_new * G;
    const int slot_rows = (int)std::min<long long>(ROWS, most);
    long long* prefix = static_cast<long long*>(a.workspace);
    float* slots = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + prefix_bytes(a.B));
    kv_attention_tc_kernel<T, D><<<ctas, THREADS, Layout<D>::SMEM, s>>>(a, G, slot_rows, prefix, slots);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return launch_join<T, D, ROWS, TILE>(a, G, ctas, slot_rows, prefix, slots, s);
}

}  // namespace

size_t kv_attention_tc_slot_bytes(int max_rows, int D) {
    return (size_t)num_sms() * 2 * slot_floats(max_rows, D) * 4;
}

cudaError_t launch_kv_attention_tc(const KvAttnArgs& a, cudaStream_t s) {
    if (a.dtype == STARQ_BF16)
        return a.c.D == 64 ? launch_typed<__nv_bfloat16, 64>(a, s) : launch_typed<__nv_bfloat16, 128>(a, s);
    return a.c.D == 64 ? launch_typed<__half, 64>(a, s) : launch_typed<__half, 128>(a, s);
}

}  // namespace starq
