// Attention over the paged 8-bit cache for many query rows of a key/value
// head (blocks of positions under denoising, drafted runs with grouped heads;
// the rule stands at the end of kvattn.cu): both products on tcgen05. The
// mathematics is kvattn.cu's.
//
// With R rows a cached key costs 4 R D operations for 2 D bytes, so from
// about 100 rows on the tensor cores' work outweighs the cache's bytes; the
// warp-level MMA would be the bound from 24 rows on. What has to be fed is
// fp16 tiles: one warp brings a tile's codes (128 keys) from their pages by
// bulk copies, three warps for the keys and three for the values turn them
// into fp16 and store them as 128-byte-swizzled tiles; the value product
// takes its tile as an MN-major operand, so no transposition is needed.
// (Loads into the converting warps' registers had to wait for the proxy fence
// of the last hand-over, and it for them.)
//
// A unit is up to 256 rows. Two streams, each with 128 TMEM lanes of rows,
// its own scores, weights and accumulators, and four softmax warps (one
// thread a row), run half a step apart, so that one stream's products hide
// behind the other's exponentials. With more than 128 rows the streams are
// the unit's two row tiles and share every key tile; otherwise they take the
// key tiles in turn, with the same rows, and their results are joined in
// shared memory at the end. Weights replace the scores they came from in
// TMEM (A operand from tensor memory). Warps without rows skip the softmax.
//
// A key that no row sees (masked out, or past the length) costs the softmax
// nothing: its place in the tile takes the codes of another key of its
// 16-key block that is seen (so no score is above those that count), values
// of 0, and a factor of 0 in the sum. A block without such a key has scores
// of -inf. Only the causal boundary is tested score by score.
//
// Measured (bf16, 28 heads on 4 of 128, 32 positions for each of 8 sequences
// of 16384 and fewer tokens, a key mask; 39 GFLOP, 92 MB): 68.1 us, 577
// TFLOP/s, 7.6 us of it the join; the warp-level MMA took 444 us. In clocks of a
// CTA: cutting 4.5 thousand, the queries' rows 10 (beside the first codes), a
// tile's step 4.5 (a stream waits 1.8 for weights - values - next scores,
// takes the maximum in 0.7 and the weights in 1.9; the products need 2.0 of
// the tensor cores), the rows' way out 7.5. Loads from TMEM one at a time made
// the step 5.3 (75.5 us); leaving out the conversion or the codes' copies
// changes it by a few percent.
#include <algorithm>

#include "kvattn.cuh"

namespace starq {
namespace {

constexpr unsigned STATUS_TIMEOUT_KVATTN = 1u << 5;
constexpr int ROWS = 256;                          // rows of a unit
constexpr int TILE = 128;                          // keys of a tile, rows of a stream
constexpr int SOFT_WARPS = 8, CONV_WARPS = 3;      // CONV_WARPS for the keys, as many for the values
constexpr int INFO_WARP = SOFT_WARPS + 2 * CONV_WARPS, MMA_WARP = INFO_WARP + 1;
constexpr int THREADS = (MMA_WARP + 1) * 32;
constexpr int CONV_THREADS = CONV_WARPS * 32;
// fp16 tiles (the keys' scores are taken soon after a tile is there, the
// values wait for the softmax), and tiles of codes
constexpr int K_STAGES = 1, V_STAGES = 1, CK_STAGES = 3, CV_STAGES = 2;
constexpr int INFOS = 4;                           // descriptions of tiles
constexpr uint32_t TM_S = 0, TM_O = 256;           // TMEM columns: two score tiles, two accumulators
constexpr int BLOCKS = TILE / 16;                  // 16-key blocks of a tile (each inside one page)
constexpr float SMALLEST = 1.17549435e-38f;        // 2^-126

struct TileInfo {                                  // what the other warps need of a key tile
    float4 blk[BLOCKS];                            // log2(e) scale s_k, log2 s_v, 1 / s_v
    float inv[TILE];                               // 1 / s_v for each key, 0 for one that is not seen
    uint32_t seen[4];                              // bit b of word j: key 4 b + j is seen
    uint32_t met;                                  // bit b: some key of block b is seen
    int key0, edge;                                // first key; whether the causal boundary is inside
};

struct Shared {
    uint64_t k_full[K_STAGES], k_empty[K_STAGES], v_full[V_STAGES], v_empty[V_STAGES], info[INFOS], info_empty[INFOS];
    uint64_t ck_full[CK_STAGES], ck_empty[CK_STAGES], cv_full[CV_STAGES], cv_empty[CV_STAGES];
    uint64_t q_full, meet, s_full[2], p_full[2], pv_done[2];
    uint32_t tmem_base;
    int abort, never;
    alignas(16) TileInfo tile[INFOS];
    float2 ml[TILE];                               // the odd stream's (m, l) for the join of the two
};

template <int D> struct Layout {
    static constexpr int TILE_BYTES = TILE * D * 2;                  // fp16, 64-channel halves of 16 KB
    static constexpr int HALF = TILE * 128;
    static constexpr int CODES = TILE * D;                           // bytes of a tile's codes (keys or values)
    static constexpr int Q = 0, K = 2 * TILE_BYTES, V = K + K_STAGES * TILE_BYTES, CK = V + V_STAGES * TILE_BYTES;
    static constexpr int CV = CK + CK_STAGES * CODES, END = CV + CV_STAGES * CODES;
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

// Whole-warp wait of the roles that run ahead: polls 40 ns apart, so that they
// leave the issue slots to the softmax.
__device__ __forceinline__ bool wait_idle(uint32_t bar, uint32_t parity, volatile int* abort) {
    const bool ok = mbar_try_wait(bar, parity) || mbar_wait_bounded_sleepy(bar, parity, abort, 40);
    return __all_sync(0xffffffffu, ok);
}

// Whether the phase is complete, without waiting (try_wait may suspend the thread).
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// max(a, b), NaN if a is.
__device__ __forceinline__ float fmaxf_nan(float a, float b) { return a < b ? b : a; }

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

// Waits for the loads from TMEM; x comes from one of them.
__device__ __forceinline__ void tmem_arrived(uint32_t (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
                   "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]),
                   "+r"(x[16]), "+r"(x[17]), "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]),
                   "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]), "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31])
                 :: "memory");
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
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
    volatile int *abort = &sh->abort, *never = &sh->never;       // `never` stays 0: what is in flight lands
    auto B = [](const uint64_t& bar) { return smem_addr(&bar); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < K_STAGES; ++i) {
            mbar_init(B(sh->k_full[i]), CONV_WARPS);
            mbar_init(B(sh->k_empty[i]), 1);
        }
        for (int i = 0; i < V_STAGES; ++i) {
            mbar_init(B(sh->v_full[i]), CONV_WARPS);
            mbar_init(B(sh->v_empty[i]), 1);
        }
        for (int i = 0; i < CK_STAGES; ++i) {
            mbar_init(B(sh->ck_full[i]), 1);
            mbar_init(B(sh->ck_empty[i]), CONV_WARPS);
        }
        for (int i = 0; i < CV_STAGES; ++i) {
            mbar_init(B(sh->cv_full[i]), 1);
            mbar_init(B(sh->cv_empty[i]), CONV_WARPS);
        }
        for (int i = 0; i < INFOS; ++i) {
            mbar_init(B(sh->info[i]), 1);
            mbar_init(B(sh->info_empty[i]), 1);
        }
        mbar_init(B(sh->q_full), SOFT_WARPS);
        mbar_init(B(sh->meet), SOFT_WARPS);
        for (int s = 0; s < 2; ++s) {
            mbar_init(B(sh->s_full[s]), 1);
            mbar_init(B(sh->p_full[s]), 4);
            mbar_init(B(sh->pv_done[s]), 1);
        }
        sh->abort = sh->never = 0;
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
    grid_dependency_wait();
    const Run run = find_run<ROWS, TILE, THREADS>(a, G, prefix);

    // Every role walks the run segment by segment (a segment is the run's
    // part of one unit). In a segment of n key tiles the streams' steps are
    // items: shared = 1 (more than 128 rows): item u is key tile u / 2 for
    // stream u & 1; shared = 0: key tile u for stream u & 1. Either way it is
    // the stream's step u / 2 of the segment.
    Cur cur;
    int count = 0;
    if (run.tau0 < run.tau1) {
        cur.start(a, G, run);
        count = cur.tiles(a, G, run);
    }
    bool ok = count > 0;
    auto unit_rows = [&](const Cur& c) { return min(ROWS, c.s.n * G - c.rt * ROWS); };
    auto segment = [&](const Cur& c, int left) { return min(left, c.s.nt - c.kt); };

    if (count <= 0) {
        // nothing but the release of TMEM
    } else if (warp == INFO_WARP) {
        // --- the tiles' descriptions and codes; lane b < 8 looks after block b -----------
        // A tile's page numbers are loaded two tiles ahead, its scales and mask
        // bytes one ahead (in a row they were 3 of 5 thousand cycles a tile).
        const int shift = __ffs(a.c.page) - 1, b = lane & (BLOCKS - 1);
        auto advance = [&](Cur& q, int& left) {
            if (--left > 0 && ++q.kt == q.s.nt) q.next_unit(a, G);
        };
        auto page_of = [&](const Cur& q) {
            const int key = q.kt * TILE + 16 * b, i = key >> shift;
            int p = -1;
            if (key < q.s.len && i < a.table_ld) p = __ldg(a.page_table + (size_t)q.b * a.table_ld + i);
            return p;
        };
        struct Raw { int page; float sk, sv; uint8_t mask[4]; };
        auto raw_of = [&](const Cur& q, int page) {
            Raw r;
            r.page = page < a.c.pages ? page : -1;
            r.sk = r.sv = 0.f;
            if (r.page >= 0) {
                const size_t blk = (size_t)r.page * a.c.Hkv + q.h;
                r.sk = __ldg(a.c.k_scale + blk);
                r.sv = __ldg(a.c.v_scale + blk);
            }
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = q.kt * TILE + 4 * lane + j;
                r.mask[j] = key < q.s.len;
                if (r.mask[j] && a.key_mask != nullptr) r.mask[j] = __ldg(a.key_mask + (size_t)q.b * a.mask_ld + key);
            }
            return r;
        };
        Cur ahead = cur;                                     // two tiles ahead of `cur`, then one
        int left_ahead = count;
        Raw raw = raw_of(cur, page_of(cur));
        advance(ahead, left_ahead);
        Cur nxt = ahead;
        int next_page = left_ahead > 0 ? page_of(nxt) : -1;
        int k_sent = 0, v_sent = 0;                          // tiles whose codes were asked for
        for (int it = 0; it < count; ++it) {
            const int key0 = cur.kt * TILE, slot = it % INFOS;
            Raw raw_next = raw;
            if (left_ahead > 0) raw_next = raw_of(nxt, next_page);
            advance(ahead, left_ahead);
            if (left_ahead > 0) next_page = page_of(ahead);
            // which keys are seen: bit lane of word j is key 4 lane + j
            uint32_t seen[4];
            #pragma unroll
            for (int j = 0; j < 4; ++j) seen[j] = __ballot_sync(0xffffffffu, raw.mask[j] != 0);
            const int page = raw.page;
            const bool any = ((seen[0] | seen[1] | seen[2] | seen[3]) >> (4 * b) & 0xf) != 0;
            const size_t blk = (size_t)(page < 0 ? 0 : page) * a.c.Hkv + cur.h;
            const unsigned met = __ballot_sync(0xffffffffu, any) & 0xff;
            const bool fetch = any && page >= 0 && lane < BLOCKS;
            const unsigned fetched = __popc(__ballot_sync(0xffffffffu, fetch));
            const size_t at = blk * ((size_t)a.c.page * D) + (size_t)((key0 + 16 * b) & (a.c.page - 1)) * D;
            float4 d = make_float4(0.f, NEG_INF, 0.f, 0.f);
            if (any && page >= 0) {
                const float vs = raw.sv < KV_SCALE_FLOOR ? KV_SCALE_FLOOR : raw.sv;
                d = make_float4(raw.sk * (a.scale * 1.4426950408889634f), __log2f(vs), __fdividef(1.f, vs), 0.f);
            } else if (any) {
                if (lane < BLOCKS) atomicOr(a.status, STATUS_RANGE);
                d = make_float4(__uint_as_float(0x7fffffffu), 0.f, 1.f, 0.f);      // the rows that see it become NaN
            }
            const int edge = a.causal && key0 + TILE > cur.s.len - cur.s.n + 1;
            cur = nxt;
            nxt = ahead;
            raw = raw_next;
            ok = wait_idle(B(sh->info_empty[slot]), ((uint32_t)(it / INFOS) & 1u) ^ 1u, abort);
            if (!ok) break;
            TileInfo& ti = sh->tile[slot];
            if (lane < BLOCKS) ti.blk[lane] = d;
            const float iv = __shfl_sync(0xffffffffu, d.z, lane >> 2);
            *reinterpret_cast<float4*>(ti.inv + 4 * lane) =
                make_float4(seen[0] >> lane & 1 ? iv : 0.f, seen[1] >> lane & 1 ? iv : 0.f,
                            seen[2] >> lane & 1 ? iv : 0.f, seen[3] >> lane & 1 ? iv : 0.f);
            if (lane == 0) {
                ti.met = met;
                ti.seen[0] = seen[0]; ti.seen[1] = seen[1]; ti.seen[2] = seen[2]; ti.seen[3] = seen[3];
                ti.key0 = key0;
                ti.edge = edge;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->info[slot]));
            // the codes: one bulk copy a block
            auto bring = [&](int st, int stages, uint64_t* full, uint64_t* empty, uint32_t area, const uint8_t* codes) {
                if (!wait_idle(B(empty[st]), ((uint32_t)(it / stages) & 1u) ^ 1u, abort)) return false;
                const uint32_t bar = B(full[st]);
                if (lane == 0) mbar_arrive_expect_tx(bar, fetched * (16 * D));
                __syncwarp();
                if (fetch) bulk_load(base + area + st * L::CODES + b * (16 * D), codes + at, 16 * D, bar);
                return true;
            };
            ok = bring(it % CK_STAGES, CK_STAGES, sh->ck_full, sh->ck_empty, L::CK, a.c.K);
            if (!ok) break;
            ++k_sent;
            ok = bring(it % CV_STAGES, CV_STAGES, sh->cv_full, sh->cv_empty, L::CV, a.c.V);
            if (!ok) break;
            ++v_sent;
        }
        // no commit lands after this CTA has exited
        for (int st = 0; st < INFOS && ok; ++st) {
            const int uses = (count - st + INFOS - 1) / INFOS;
            if (uses > 0) ok = wait_idle(B(sh->info_empty[st]), (uint32_t)(uses - 1) & 1u, abort);
        }
        if (!ok) {
            if (lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
            for (int it = max(0, k_sent - CK_STAGES); it < k_sent; ++it)
                wait_idle(B(sh->ck_full[it % CK_STAGES]), (uint32_t)(it / CK_STAGES) & 1u, never);
            for (int it = max(0, v_sent - CV_STAGES); it < v_sent; ++it)
                wait_idle(B(sh->cv_full[it % CV_STAGES]), (uint32_t)(it / CV_STAGES) & 1u, never);
        }
    } else if (warp >= SOFT_WARPS && warp < INFO_WARP) {
        // --- codes to fp16 tiles: keys or values ------------------------------------
        const bool keys = warp < SOFT_WARPS + CONV_WARPS;
        const int ct = threadIdx.x - SOFT_WARPS * 32 - (keys ? 0 : CONV_THREADS);
        constexpr int CPR = D / 16;                          // 16-code chunks of a row
        constexpr int RSTEP = CONV_THREADS / CPR;            // 12 or 24 rows
        constexpr int PER = (TILE + RSTEP - 1) / RSTEP;      // chunks of a thread
        const int c = ct % CPR, r0 = ct / CPR;               // its channels, its rows r0 + RSTEP i
        const int stages = keys ? K_STAGES : V_STAGES, cstages = keys ? CK_STAGES : CV_STAGES;
        const uint32_t tiles = base + (keys ? L::K : L::V);
        const uint8_t* const codes = smem + (keys ? L::CK : L::CV) + 16 * c;
        uint64_t* const full_bar = keys ? sh->k_full : sh->v_full;
        uint64_t* const empty_bar = keys ? sh->k_empty : sh->v_empty;
        uint64_t* const cfull_bar = keys ? sh->ck_full : sh->cv_full;
        uint64_t* const cempty_bar = keys ? sh->ck_empty : sh->cv_empty;
        for (int it = 0; it < count && ok; ++it) {
            const int st = it % stages, cs = it % cstages;
            ok = wait_idle(B(sh->info[it % INFOS]), (uint32_t)(it / INFOS) & 1u, abort) &&
                 wait_idle(B(cfull_bar[cs]), (uint32_t)(it / cstages) & 1u, abort);
            if (!ok) break;
            const TileInfo& ti = sh->tile[it % INFOS];
            const uint32_t w0 = ti.seen[0], w1 = ti.seen[1], w2 = ti.seen[2], w3 = ti.seen[3];
            const bool full = (w0 & w1 & w2 & w3) == 0xffffffffu;
            // this thread's rows are r0 modulo 4
            const uint32_t mine = (r0 & 2) ? ((r0 & 1) ? w3 : w2) : ((r0 & 1) ? w1 : w0);
            uint4 v[PER];                                    // all loads before the first store
            #pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int r = min(r0 + RSTEP * i, TILE - 1);
                int from = r;                                // the row whose codes stand here, -1: zeros
                if (!full && !(mine >> (r >> 2) & 1)) {
                    from = -1;
                    if (keys) {                              // some key of the block that is seen
                        const int q = 4 * (r >> 4);
                        const unsigned n0 = w0 >> q & 0xf, n1 = w1 >> q & 0xf, n2 = w2 >> q & 0xf, n3 = w3 >> q & 0xf;
                        if (n0 | n1 | n2 | n3) {
                            const unsigned n = n0 ? n0 : n1 ? n1 : n2 ? n2 : n3;
                            from = (r & ~15) + 4 * (__ffs(n) - 1) + (n0 ? 0 : n1 ? 1 : n2 ? 2 : 3);
                        }
                    }
                }
                v[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);      // codes 0
                if (from >= 0) v[i] = *reinterpret_cast<const uint4*>(codes + cs * L::CODES + from * D);
            }
            ok = wait_idle(B(empty_bar[st]), ((uint32_t)(it / stages) & 1u) ^ 1u, abort);
            if (!ok) break;
            #pragma unroll
            for (int i = 0; i < PER; ++i)
                if (r0 + RSTEP * i < TILE) store_codes<D>(tiles + st * L::TILE_BYTES, r0 + RSTEP * i, c, v[i]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(B(cempty_bar[cs]));
                mbar_arrive(B(full_bar[st]));
            }
        }
        // the last use of every stage has been given back, so no commit lands after this CTA has exited
        for (int st = 0; st < stages && ok; ++st) {
            const int uses = (count - st + stages - 1) / stages;
            if (uses > 0) ok = wait_idle(B(empty_bar[st]), (uint32_t)(uses - 1) & 1u, abort);
        }
        if (!ok && lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
    } else if (warp == MMA_WARP) {
        // --- the products ---------------------------------------------------------
        constexpr uint32_t IDESC_QK = (1u << 4) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
        constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
        int left = count, tile0 = 0, steps[2] = {0, 0};      // key tiles and stream steps before the segment
        int qks[2] = {0, 0}, pvs[2] = {0, 0};                // products issued, a stream
        int seg = 0;
        while (left > 0 && ok) {
            const int n = segment(cur, left);
            const int shared = unit_rows(cur) > TILE;
            const int items = shared ? 2 * n : n;
            ok = mbar_wait_bounded_warp(B(sh->q_full), (uint32_t)seg & 1u, abort);
            auto qk = [&](int u, bool seen_k) {
                const int kt = tile0 + (shared ? u >> 1 : u), st = kt % K_STAGES, s = u & 1;
                if (!seen_k && !mbar_wait_bounded_warp(B(sh->k_full[st]), (uint32_t)(kt / K_STAGES) & 1u, abort))
                    return false;
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
                ++qks[s];
                return true;
            };
            for (int u = 0; u < 2 && u < items && ok; ++u) ok = qk(u, false);
            for (int u = 0; u < items && ok; ++u) {
                const int kt = tile0 + (shared ? u >> 1 : u), st = kt % V_STAGES, s = u & 1, step = u >> 1;
                const int kn = tile0 + (shared ? (u + 2) >> 1 : u + 2);
                ok = mbar_wait_bounded_warp(B(sh->v_full[st]), (uint32_t)(kt / V_STAGES) & 1u, abort) &&
                     mbar_wait_bounded_warp(B(sh->p_full[s]), (uint32_t)(steps[s] + step) & 1u, abort);
                if (!ok) break;
                const bool k_there = u + 2 < items &&
                                     mbar_test_wait(B(sh->k_full[kn % K_STAGES]), (uint32_t)(kn / K_STAGES) & 1u);
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t vd = smem_desc_mn(base + L::V + st * L::TILE_BYTES, L::HALF);
                    #pragma unroll
                    for (int k = 0; k < TILE / 16; ++k)
                        mma_f16_ts(tmem + TM_O + s * TILE, tmem + TM_S + s * TILE + 8 * k,
                                   vd + (uint64_t)(k * 2048 >> 4), IDESC_PV, step > 0 || k > 0);
                    if (!shared || s == 1) {
                        tc_commit(B(sh->v_empty[st]));
                        tc_commit(B(sh->info_empty[kt % INFOS]));
                    }
                    tc_commit(B(sh->pv_done[s]));
                }
                __syncwarp();
                ++pvs[s];
                if (u + 2 < items) ok = qk(u + 2, __all_sync(0xffffffffu, k_there));
            }
            steps[0] += (items + 1) / 2;
            steps[1] += items / 2;
            tile0 += n;
            left -= n;
            ++seg;
            cur.kt += n;
            if (left > 0) cur.next_unit(a, G);
        }
        if (!ok) {
            if (lane == 0) { sh->abort = 1; atomicOr(a.status, STATUS_TIMEOUT_KVATTN); }
            for (int s = 0; s < 2; ++s) {
                if (qks[s] > 0) mbar_wait_bounded_warp(B(sh->s_full[s]), (uint32_t)(qks[s] - 1) & 1u, never);
                if (pvs[s] > 0) mbar_wait_bounded_warp(B(sh->pv_done[s]), (uint32_t)(pvs[s] - 1) & 1u, never);
            }
        }
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
            // The unit's query rows, as the A operand (with few rows both streams use the first tile): asynchronous
            // copies along the rows, and bf16 rows become fp16 in place, a thread a row. In rolled loops: the same
            // work unrolled ran from cold instruction lines (7 us of a call, now 2).
            float down = 1.f;
            constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
            if (shared || s == 0 || BF16) {
                constexpr int CH = D / 8, RPC = 32 / CH;                        // 16-byte chunks of a row, rows a copy
                const uint32_t tile = base + L::Q + s * L::TILE_BYTES;
                const long long from = valid ? (long long)(cur.s.row0 + i) * a.ldq + (long long)head * D : 0;
                #pragma unroll 4
                for (int r0 = 0; r0 < 32; r0 += RPC) {
                    const int rr = r0 + lane / CH, k = lane % CH;
                    const long long off = __shfl_sync(0xffffffffu, from, rr);
                    const bool real = __shfl_sync(0xffffffffu, (int)valid, rr) != 0;
                    cp_async16_or_zero(tile + (k >> 3) * L::HALF + sw128_offset((warp & 3) * 32 + rr, k & 7),
                                       static_cast<const T*>(a.Q) + off + 8 * k, real);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
                if (BF16) {
                    // the largest magnitude: bf16 numbers without their sign are ordered as integers
                    auto chunk = [&](int k) {
                        return reinterpret_cast<uint4*>(smem + L::Q + s * L::TILE_BYTES + (k >> 3) * L::HALF +
                                                        sw128_offset(row, k & 7));
                    };
                    uint32_t top = 0;
                    #pragma unroll 4
                    for (int k = 0; k < CH; ++k) {
                        const uint4 v = *chunk(k);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                        #pragma unroll
                        for (int e = 0; e < 4; ++e) top = max(top, max(w[e] << 16 & 0x7fff0000u, w[e] & 0x7fff0000u));
                    }
                    float up;
                    row_power(__uint_as_float(top), up, down);
                    if (shared || s == 0) {
                        #pragma unroll 2
                        for (int k = 0; k < CH; ++k) {
                            uint4 v = *chunk(k);
                            uint32_t w[4] = {v.x, v.y, v.z, v.w};
                            #pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __half2 p = __floats2half2_rn(__uint_as_float(w[e] << 16) * up,
                                                                    __uint_as_float(w[e] & 0xffff0000u) * up);
                                w[e] = *reinterpret_cast<const uint32_t*>(&p);
                            }
                            *chunk(k) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(B(sh->q_full));

            float m = NEG_INF, l = 0.f;
            for (int step = 0; step < mine && ok; ++step) {
                const int kt = tile0 + (shared ? step : 2 * step + s), st = kt % INFOS;
                ok = mbar_wait_bounded_warp(B(sh->s_full[s]), (uint32_t)(steps + step) & 1u, abort) &&
                     mbar_wait_bounded_warp(B(sh->info[st]), (uint32_t)(kt / INFOS) & 1u, abort);
                if (!ok) break;
                if (active) {
                    tc_fence_after();
                    const TileInfo& ti = sh->tile[st];
                    const bool edge = ti.edge != 0;  // the causal boundary is in the tile
                    float top = NEG_INF;
                    unsigned met = edge ? 0u : ti.met;                          // blocks of which the row sees a key
                    // Two chunks of 32 keys at a time, the second on its way from TMEM while the first is worked on.
                    auto chunks = [&](auto&& work) {
                        #pragma unroll 1
                        for (int c = 0; c < 4; c += 2) {
                            uint32_t x[32], y[32];
                            tmem_ld_32x32b_x32(t_s + 32 * c, x);
                            tmem_arrived(x);
                            tmem_ld_32x32b_x32(t_s + 32 * c + 32, y);
                            work(c, x);
                            tmem_arrived(y);
                            work(c + 1, y);
                        }
                    };
                    auto largest = [&](const uint32_t* y) {
                        float t = __uint_as_float(y[0]);
                        #pragma unroll
                        for (int k = 1; k < 15; k += 2) t = max3(t, __uint_as_float(y[k]), __uint_as_float(y[k + 1]));
                        return fmaxf(t, __uint_as_float(y[15]));
                    };
                    if (!edge) {
                        chunks([&](int c, const uint32_t (&x)[32]) {
                            #pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const float4 b = ti.blk[2 * c + q];
                                top = fmaxf(top, fmaf(largest(&x[16 * q]), b.x * down, b.y));
                            }
                        });
                    } else {
                        #pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t x[32];
                            tmem_ld_32x32b_x32(t_s + 32 * c, x);
                            tmem_arrived(x);
                            const int see = lim - ti.key0 - 32 * c;
                            uint32_t live[4];                                   // bit k / 4 of word k % 4: key 32 c + k
                            #pragma unroll
                            for (int j = 0; j < 4; ++j) live[j] = ti.seen[j] >> (8 * c);
                            #pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (k >= see || !(live[k & 3] >> (k >> 2) & 1)) x[k] = 0xff800000u;
                            #pragma unroll
                            for (int q = 0; q < 2; ++q) {                       // for the second pass
                                uint32_t y[16];
                                #pragma unroll
                                for (int k = 0; k < 16; ++k) y[k] = x[16 * q + k];
                                tmem_st_32x32b_x16(t_s + 32 * c + 16 * q, y);
                                const float t = largest(y);
                                const float4 b = ti.blk[2 * c + q];
                                if (b.y != NEG_INF && t != NEG_INF) {
                                    met |= 1u << (2 * c + q);
                                    top = fmaxf(top, fmaf(t, b.x * down, b.y));
                                }
                            }
                        }
                    }
                    if (edge) tmem_st_wait();
                    if (__any_sync(0xffffffffu, top > m + LAZY)) {
                        const float to = fmaxf(m, top), f = m == to ? 1.f : ex2(m - to);
                        m = to;
                        l *= f;
                        if (step > 0) {
                            ok = mbar_wait_bounded_warp(B(sh->pv_done[s]), (uint32_t)(steps + step - 1) & 1u, abort);
                            if (!ok) break;
                            tc_fence_after();
                            #pragma unroll 1
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
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    // `all`: every row sees a key of every block. Else a block without one weighs nothing,
                    // whatever its scales are.
                    auto weights = [&](auto all) {
                        chunks([&](int c, const uint32_t (&x)[32]) {
                            uint32_t p[16];
                            #pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const float4 b = ti.blk[2 * c + q];
                                // a factor that underflows (a zero row, a zero block, a tiny scale) times
                                // the -inf of an unseen key would be NaN; at this floor no score counts
                                const float ax = fmaxf_nan(b.x * down, SMALLEST), cx = b.y - sub;
                                const bool any = decltype(all)::value || (met >> (2 * c + q) & 1);
                                #pragma unroll
                                for (int k = 0; k < 16; k += 4) {
                                    const float4 f = *reinterpret_cast<const float4*>(ti.inv + 32 * c + 16 * q + k);
                                    float2 v[2];
                                    #pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        v[h] = fma2(make_float2(__uint_as_float(x[16 * q + k + 2 * h]),
                                                                __uint_as_float(x[16 * q + k + 2 * h + 1])),
                                                    make_float2(ax, ax), make_float2(cx, cx));
                                        v[h].x = ex2(v[h].x);
                                        v[h].y = ex2(v[h].y);
                                        const __half2 w = __floats2half2_rn(v[h].x, v[h].y);
                                        p[8 * q + k / 2 + h] = any ? *reinterpret_cast<const uint32_t*>(&w) : 0u;
                                    }
                                    if (any) {
                                        sum[0] = fma2(v[0], make_float2(f.x, f.y), sum[0]);
                                        sum[1] = fma2(v[1], make_float2(f.z, f.w), sum[1]);
                                    }
                                }
                            }
                            tmem_st_32x32b_x16(t_s + 16 * c, p);                // over scores of chunks up to c / 2
                        });
                    };
                    if (__all_sync(0xffffffffu, met == 0xffu)) weights(std::true_type{});
                    else weights(std::false_type{});
                    l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
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
                // Half of the columns at a time through this warp's part of the Q area (its rows of the join
                // area, or its quarter of the stream's Q tile), so that the stores run along the rows.
                constexpr int C4 = D / 8, RPW = 32 / C4;                        // float4s of half a row, rows a warp store
                const float inv = whole ? (l == 0.f ? 0.f : __fdiv_rn(1.f, l)) : 1.f;
                float* slot = slots + ((size_t)blockIdx.x * 2 + (tile0 == 0 ? 0 : 1)) * slot_floats(slot_rows, D);
                const int srow = (shared ? s * TILE : 0) + row;
                const long long at = whole ? (long long)(cur.s.row0 + i) * a.ldo + (long long)head * D
                                           : (long long)srow * D;
                float* stage = reinterpret_cast<float*>(smem + L::Q + s * L::TILE_BYTES + (warp & 3) * (64 * D));
                auto stage_at = [&](int r, int c) { return stage + r * (D / 2) + ((c ^ (r & (C4 - 1))) << 2); };
                #pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    #pragma unroll 2
                    for (int c = half * (D / 32); c < (half + 1) * (D / 32); ++c) {
                        uint32_t o[16];
                        tmem_ld_32x32b_x16(t_o + 16 * c, o);
                        tmem_ld_wait();
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float4 v = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                                         __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
                            if (!shared) {
                                float4* other = reinterpret_cast<float4*>(join_at(4 * c + k));
                                const float4 w = *other;
                                *other = make_float4(v.x * f0 + w.x * f1, v.y * f0 + w.y * f1, v.z * f0 + w.z * f1,
                                                     v.w * f0 + w.w * f1);
                            } else {
                                *reinterpret_cast<float4*>(stage_at(lane, 4 * c + k - half * C4)) = v;
                            }
                        }
                    }
                    __syncwarp();
                    #pragma unroll 4
                    for (int r0 = 0; r0 < 32; r0 += RPW) {
                        const int r = r0 + lane / C4, c = lane % C4, c4 = half * C4 + c;
                        const long long to = __shfl_sync(0xffffffffu, at, r);
                        const float scale = __shfl_sync(0xffffffffu, inv, r);
                        const bool put = __shfl_sync(0xffffffffu, (int)valid, r) != 0;
                        const int jr = row - lane + r;                          // the row in the join area
                        const float4 v = *reinterpret_cast<const float4*>(
                            shared ? stage_at(r, c) : join + jr * D + ((c4 ^ (jr & (D / 4 - 1))) << 2));
                        if (put && whole) {
                            // (no key seen: accumulators and scale are 0)
                            const T e[4] = {(T)(v.x * scale), (T)(v.y * scale), (T)(v.z * scale), (T)(v.w * scale)};
                            *reinterpret_cast<uint2*>(static_cast<T*>(a.Out) + to + 4 * c4) =
                                *reinterpret_cast<const uint2*>(e);
                        } else if (put) {
                            *reinterpret_cast<float4*>(slot + to + 4 * c4) = v;
                        }
                    }
                    __syncwarp();
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
            // the join and staging areas are Q's memory: read before the next unit's rows come in
            if (!(ok = meet())) break;
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
    if ((e = launch_overlapped(kv_attention_tc_kernel<T, D>, dim3(ctas), THREADS, Layout<D>::SMEM, s, a, G, slot_rows,
                               prefix, slots)) != cudaSuccess || a.whole)
        return e;
    return launch_join<T, D, ROWS, TILE>(a, G, ctas, slot_rows, prefix, slots, s);
}

}  // namespace

size_t kv_attention_tc_slot_bytes(int max_rows, int D) {
    return (size_t)num_sms() * 2 * slot_floats(max_rows, D) * 4;
}

cudaError_t launch_kv_attention_tc(const KvAttnArgs& args, cudaStream_t s) {
    KvAttnArgs a = args;
    a.whole = whole_units(a, ROWS, TILE, num_sms());
    if (a.dtype == STARQ_BF16)
        return a.c.D == 64 ? launch_typed<__nv_bfloat16, 64>(a, s) : launch_typed<__nv_bfloat16, 128>(a, s);
    return a.c.D == 64 ? launch_typed<__half, 64>(a, s) : launch_typed<__half, 128>(a, s);
}

}  // namespace starq
