// Attention of new query tokens over the paged 8-bit key/value cache.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j),
//   k_j = s_k(j) c_j,  v_j = s_v(j) e_j     (one scale per block and head)
// over the keys j that row i sees; a row that sees none gives 0 and a
// log-sum-exp of -inf.
//
// Arithmetic. The codes c, e are integers of magnitude <= 127, exact in
// fp16, so both products run on the 16-bit MMA with float32 accumulators.
// (Keys as their bytes c + 128, with the offset taken off the score by
// linearity, save a subtraction for every two codes: 75.0 us for 75.6 over
// four sequences of 131072 tokens, 56.5 for 58.2 with heads of 64. But where
// a few loud channels set a block's scale the other codes are a few units,
// and the offset's rounding is up to 2^-14 of the score. Of the values, a
// channel in which the heavy keys' codes are 0 would show it.)
// A bf16 query row is scaled by a power of two into fp16's range: its eight
// significand bits fit, so only values below 2^-28 of the row's largest
// lose bits. s_k and the softmax scale multiply the float32 score. s_v
// enters through the exponent: with
//   x_ij = log2(e) scale q_i . k_j + log2 s_v(j),  P_ij = 2^(x_ij - m_i + 7)
// the weights P_ij already carry the value's scale and are at most 2^15, so
// rounding them to fp16 (2^-11 relative, as a 16-bit attention does) loses
// only weights 2^-32 below the row's largest, which is at least 2^7; the sum
// of the plain weights is sum_j P_ij / s_v(j) in float32 from the unrounded
// P. m_i is a running maximum that moves only when a score passes it by 8
// (2^8 of headroom), so most tiles do not rescale the accumulators. Below
// 2^-126 of that scale, i.e. p_ij s_v(j) some 2^-125 below the row's largest,
// a key drops out of the sum too: in blocks of values that are all 0 (s_v at
// its floor) weights of 2^-24 of the largest still count beside blocks of
// values up to 6 10^4, fp16's range.
//
// Work. For one query token the cache is read once and the rest is small:
// bound by memory. The G query heads of a key/value head and the new tokens
// share a unit's rows (16 of an MMA tile), so a key is loaded once for all
// of them (with more than 16 rows a unit is 16 of them, and the later units
// find the keys in the L2 cache). The 128-key tiles of all units are cut into
// equal runs, one per CTA: a long sequence is spread over the whole GPU and
// short ones are packed, whatever the lengths are. A run that covers a unit writes its
// rows; partial runs leave (sum, maximum, accumulators) in the workspace and
// a second kernel joins them in run order (results do not depend on timing).
//
// In a CTA each of four warps owns 32 keys of a tile (two blocks) and a
// private ring of cp.async stages (three with up to 8 rows, else two), so
// warps meet only at the ends of a unit; the query fragments, alike for all,
// are in shared memory (with up to 8 rows in registers). 16-byte chunks
// are XOR-swizzled by row so that both fragments read without bank
// conflicts. The MMA's k order is free: a key's fragment takes 4 consecutive
// channels per thread, and value columns are taken in the order that makes a
// thread's 16 bytes one row's 16 columns, so no transposition is needed.
//
// Measured (bf16, 28 heads on 4 of 128): one token for each of four sequences
// of 131072 and fewer tokens (407 MB): 76.2 us, 5.3 TB/s, 3.6 us of it the
// join. Most instructions turn bytes into fragments. One sequence of 777
// tokens takes 8.5 us, a chain of two launches and their loads.
#include <algorithm>
#include <type_traits>

#include "kvattn.cuh"

namespace starq {
namespace {

constexpr int WARPS = 4;
constexpr int THREADS = WARPS * 32;
constexpr int ROWS = 16;               // query rows of a unit
constexpr int WKEYS = 32;              // keys of a warp in a tile: two 16-key blocks
constexpr int TILE = WARPS * WKEYS;    // 128 keys
// Tiles of a warp that are there or on their way, and CTAs an SM. Up to 8 rows
// need fewer instructions a tile and wait for memory sooner: 74.3 us with 3
// tiles and 2 CTAs for 77.3 with 2 and 3 (four sequences of 131072 tokens);
// 40 rows over 4001 tokens the other way round, 19.2 for 20.3. (Both with
// the keys' offset taken off the scores.)
constexpr int MOST_CTAS = 3;
template <bool NARROW> constexpr int STAGES = NARROW ? 3 : 2;
template <bool NARROW> constexpr int CTAS_PER_SM = NARROW ? 2 : MOST_CTAS;
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory");
}

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                 "{%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Transposes an 8 x 8 matrix of 16-bit numbers (a row in four threads).
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The codes of bytes 0 and 1 (2 and 3) of a word.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return codes_half2(prmt(w, 0x64646464u, 0x4140u)); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return codes_half2(prmt(w, 0x64646464u, 0x4342u)); }

// Byte offset of 16-byte chunk c of row r (of 16) in a warp's stage.
template <int D> __device__ __forceinline__ uint32_t stage_offset(int r, int c) {
    if (D == 128) return r * 128 + ((c ^ (r & 7) ^ ((r & 1) << 2)) << 4);
    return (r >> 1) * 128 + (((r & 1) ^ ((r >> 2) & 1)) << 6) + ((c ^ (((r >> 1) & 1) << 1)) << 4);
}

// Fragments of one query row (half of the A operand's registers): channels
// 64 h + 16 t + 4 s + {0, 1} in q[h][s][0], {2, 3} in q[h][s][1]; returns the
// power of two that undoes the row's scaling.
template <typename T, int D>
__device__ __forceinline__ float load_row(const T* row, int t, uint32_t (&q)[D / 64][4][2]) {
    float v[D / 64][16], top = 0.f;
    #pragma unroll
    for (int h = 0; h < D / 64; ++h) {
        float x[8];
        #pragma unroll
        for (int k = 0; k < 2; ++k) {
            #pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
            if (row != nullptr) Eight<T>::load(row + 64 * h + 16 * t + 8 * k, x);
            #pragma unroll
            for (int i = 0; i < 8; ++i) { v[h][8 * k + i] = x[i]; top = fmaxf(top, fabsf(x[i])); }
        }
    }
    float up = 1.f, down = 1.f;
    if (std::is_same<T, __nv_bfloat16>::value) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        row_power(top, up, down);
    }
    #pragma unroll
    for (int h = 0; h < D / 64; ++h)
        #pragma unroll
        for (int s = 0; s < 4; ++s)
            #pragma unroll
            for (int k = 0; k < 2; ++k) {
                const __half2 p = __floats2half2_rn(v[h][4 * s + 2 * k] * up, v[h][4 * s + 2 * k + 1] * up);
                q[h][s][k] = *reinterpret_cast<const uint32_t*>(&p);
            }
    return down;
}

template <typename T, int D, bool NARROW>
struct AttnSmem {
    static constexpr int STAGE = 2 * WKEYS * D + 16;            // bytes of a warp's stage: keys, values, the blocks' scales
    static constexpr int RING = WARPS * STAGES<NARROW> * STAGE;
    static constexpr int MERGE = ROWS * D * 4 + WARPS * ROWS * 8;
    static constexpr int QUERY = RING;                          // fragments [D / 16][32 lanes][4], until the merge
    static constexpr int BYTES = RING + MERGE;
};

// NARROW: at most 8 rows. Then the keys are the MMA's 16-row operand and the
// query rows its 8 columns (scores^T = K Q^T, out^T = V^T P^T): half the MMAs
// and half the exponentials, none of them for rows that do not exist. A
// thread has the columns (rows of the unit) 2t and 2t + 1. Measured (7 rows, as
// above, both forms with the keys' offset and two stages): four long sequences
// 77.7 us for 86.0, one of 777 tokens 8.5 for 12.2, 64 of up to 1000 tokens
// 19.7 for 28.
template <typename T, int D, bool NARROW>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM<NARROW>) kv_attention_kernel(const KvAttnArgs a, int G, long long* prefix_out,
                                                                 float* slots) {
    using SM = AttnSmem<T, D, NARROW>;
    constexpr int KH = D / 64;               // 64-channel halves of a key
    constexpr int DN = D / 8;                // value columns per thread, and column tiles
    constexpr int HELD = NARROW ? 8 : ROWS;  // rows that can be there
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

    grid_dependency_wait();
    const Run run = find_run<ROWS, TILE, THREADS>(a, G, prefix_out);
    if (run.tau0 >= run.tau1) return;
    Cursor<ROWS, TILE> cur;
    cur.start(a, G, run);
    Cursor<ROWS, TILE> pre = cur;
    int left = cur.tiles(a, G, run);         // tiles of the run
    int pre_left = left;                     // tiles still to be fetched

    const uint32_t ring = smem_addr(smem) + warp * (STAGES<NARROW> * SM::STAGE);
    const int shift = __ffs(a.c.page) - 1;
    const size_t block_bytes = (size_t)a.c.page * D;
    // where this lane's 16-byte chunks of a 16-key block go
    uint32_t dst_at[D / 32];
    #pragma unroll
    for (int i = 0; i < D / 32; ++i) dst_at[i] = stage_offset<D>((lane + 32 * i) / (D / 16), (lane + 32 * i) % (D / 16));

    // One warp's keys of the next tile, block by block (a page holds whole blocks).
    auto fetch = [&](int slot) {
        if (pre_left > 0) {
            #pragma unroll
            for (int blk16 = 0; blk16 < WKEYS / 16; ++blk16) {
                const int key0 = pre.kt * TILE + warp * WKEYS + 16 * blk16;
                if (key0 < pre.s.len) {
                    const int page_i = key0 >> shift;
                    int page = -1;
                    if (page_i < a.table_ld) page = __ldg(a.page_table + (size_t)pre.b * a.table_ld + page_i);
                    const uint32_t dst = ring + slot * SM::STAGE, dst_s = dst + 2 * WKEYS * D + 8 * blk16;
                    if (page < 0 || page >= a.c.pages) {
                        if (lane == 0) {
                            atomicOr(a.status, STATUS_RANGE);
                            // the rows that see these keys become NaN
                            asm volatile("st.shared.v2.b32 [%0], {%1, %2};"
                                         :: "r"(dst_s), "r"(0x7fffffffu), "r"(0x3f800000u) : "memory");
                        }
                    } else {
                        const size_t blk = (size_t)page * a.c.Hkv + pre.h;
                        const size_t off = blk * block_bytes + (size_t)(key0 & (a.c.page - 1)) * D + lane * 16;
                        const uint8_t* k = a.c.K + off;
                        const uint8_t* v = a.c.V + off;
                        #pragma unroll
                        for (int i = 0; i < D / 32; ++i) cp_async16(dst + 16 * blk16 * D + dst_at[i], k + 512 * i);
                        #pragma unroll
                        for (int i = 0; i < D / 32; ++i)
                            cp_async16(dst + (WKEYS + 16 * blk16) * D + dst_at[i], v + 512 * i);
                        if (lane < 2) cp_async4(dst_s + 4 * lane, (lane ? a.c.v_scale : a.c.k_scale) + blk);
                    }
                }
            }
            --pre_left;
            if (++pre.kt == pre.s.nt && pre_left > 0) pre.next_unit(a, G);
        }
        cp_async_commit();
    };
    #pragma unroll
    for (int i = 0; i < STAGES<NARROW> - 1; ++i) fetch(i);

    uint4* const query = reinterpret_cast<uint4*>(smem + SM::QUERY) + lane;      // this lane's fragment of k step 0
    constexpr int OT = NARROW ? DN / 2 : DN; // tiles of the accumulators
    uint32_t qb[NARROW ? KH : 1][4][2];      // NARROW: the query fragments
    float o[OT][4], m[2], l[2], rs[2];
    int lim[2];                              // keys [0, lim) are visible to the rows (causal limit and length)
    const float unit_scale = a.scale * 1.4426950408889634f;
    bool fresh = true;
    int seg_kt0 = cur.kt;
    int tau = 0;                             // tiles done

    int st = 0;
    #pragma unroll 1
    while (left > 0) {
        {
            if (fresh) {                     // a new unit: its query rows
                uint32_t q2[2][KH][4][2];
                #pragma unroll
                for (int k = 0; k < (NARROW ? 1 : 2); ++k) {
                    const int r = cur.rt * ROWS + g + 8 * k, i = r / G, j = r - i * G;
                    const T* row = nullptr;
                    lim[k] = 0;
                    if (i < cur.s.n) {
                        row = static_cast<const T*>(a.Q) + (size_t)(cur.s.row0 + i) * a.ldq +
                              (size_t)(cur.h * G + j) * D;
                        lim[k] = a.causal ? max(0, cur.s.len - cur.s.n + i + 1) : cur.s.len;
                    }
                    rs[k] = load_row<T, D>(row, t, q2[k]);
                }
                m[0] = m[1] = NEG_INF;
                l[0] = l[1] = 0.f;
                if constexpr (NARROW) {
                    #pragma unroll
                    for (int h = 0; h < KH; ++h)
                        #pragma unroll
                        for (int s = 0; s < 4; ++s) { qb[h][s][0] = q2[0][h][s][0]; qb[h][s][1] = q2[0][h][s][1]; }
                    const float r = rs[0];
                    const int v = lim[0];
                    #pragma unroll
                    for (int k = 0; k < 2; ++k) {           // from the threads of row g = 2t + k
                        rs[k] = __shfl_sync(0xffffffffu, r, 4 * (2 * t + k));
                        lim[k] = __shfl_sync(0xffffffffu, v, 4 * (2 * t + k));
                    }
                } else {
                // every warp has the fragments; each stores its part of them for all
                #pragma unroll
                for (int h = 0; h < KH; ++h)
                    #pragma unroll
                    for (int s = 0; s < 4; ++s)
                        if ((4 * h + s) % WARPS == warp)
                            query[(4 * h + s) * 32] = make_uint4(q2[0][h][s][0], q2[1][h][s][0], q2[0][h][s][1],
                                                                 q2[1][h][s][1]);
                __syncthreads();             // (the unit before ended with a barrier: its fragments are done with)
                }
                #pragma unroll
                for (int j = 0; j < OT; ++j)
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) o[j][k] = 0.f;
                fresh = false;
                seg_kt0 = cur.kt;
            }
            fetch((st + STAGES<NARROW> - 1) % STAGES<NARROW>);
            cp_async_wait<STAGES<NARROW> - 1>();
            __syncwarp();
            const int key0 = cur.kt * TILE + warp * WKEYS;
            if (key0 < cur.s.len) {
                // one byte a lane, on its way beside the scores (a byte for each score took 59 us for 42 where 55
                // sequences of 8 heads and up to 575 tokens have 64 rows)
                uint8_t mask_byte = 1;
                if (a.key_mask != nullptr && key0 + lane < cur.s.len)
                    mask_byte = __ldg(a.key_mask + (size_t)cur.b * a.mask_ld + key0 + lane);
                const uint8_t* stage = smem + warp * (STAGES<NARROW> * SM::STAGE) + st * SM::STAGE;
                // --- scores of 32 keys: four column tiles, a k step for all of them ---
                constexpr int XT = NARROW ? 2 : 4;           // tiles: NARROW 16 keys x 8 rows, else 16 rows x 8 keys
                float x[XT][4];
                #pragma unroll
                for (int nt = 0; nt < XT; ++nt)
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) x[nt][k] = 0.f;
                #pragma unroll
                for (int h = 0; h < KH; ++h) {
                    uint4 w[4];
                    #pragma unroll
                    for (int nt = 0; nt < 4; ++nt)
                        w[nt] = *reinterpret_cast<const uint4*>(stage + stage_offset<D>(nt * 8 + g, 4 * h + t));
                    #pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        auto word = [&](int nt) { return s == 0 ? w[nt].x : s == 1 ? w[nt].y : s == 2 ? w[nt].z : w[nt].w; };
                        if constexpr (NARROW) {
                            #pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                const uint32_t u = word(2 * b), v = word(2 * b + 1);
                                const uint32_t ka[4] = {codes_lo(u), codes_lo(v), codes_hi(u), codes_hi(v)};
                                mma_16816(x[b], ka, qb[h][s][0], qb[h][s][1]);
                            }
                        } else {
                            const uint4 q = query[(4 * h + s) * 32];
                            const uint32_t qa[4] = {q.x, q.y, q.z, q.w};
                            #pragma unroll
                            for (int nt = 0; nt < 4; ++nt) mma_16816(x[nt], qa, codes_lo(word(nt)), codes_hi(word(nt)));
                        }
                    }
                }
                // element k of a tile: which of the thread's two rows, and which key of the warp's 32
                auto row_of = [](int k) { return NARROW ? k & 1 : k >> 1; };
                auto key_of = [&](int nt, int k) {
                    return NARROW ? 16 * nt + g + 8 * (k >> 1) : 8 * nt + 2 * t + (k & 1);
                };
                auto block_of = [](int nt) { return NARROW ? nt : nt >> 1; };
                const float4 scales = *reinterpret_cast<const float4*>(stage + 2 * WKEYS * D);
                float iv[2];
                #pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float ks = (b ? scales.z : scales.x) * unit_scale, sv = b ? scales.w : scales.y;
                    // a value scale below the floor counts as the floor (an empty block's codes are 0)
                    const float vs = sv < KV_SCALE_FLOOR ? KV_SCALE_FLOOR : sv;
                    const float lv = __log2f(vs);
                    iv[b] = __fdividef(1.f, vs);
                    const float k0 = ks * rs[0], k1 = ks * rs[1];
                    #pragma unroll
                    for (int nt = b * (XT / 2); nt < (b + 1) * (XT / 2); ++nt)
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) x[nt][k] = fmaf(x[nt][k], row_of(k) ? k1 : k0, lv);
                }
                const bool edge = key0 + WKEYS > cur.s.len || a.key_mask != nullptr ||
                                  (a.causal && key0 + WKEYS > cur.s.len - cur.s.n + 1);
                unsigned seen = 0xffff;      // bit 4 nt + k: x[nt][k] counts
                if (edge) {
                    const unsigned live = __ballot_sync(0xffffffffu, mask_byte != 0);       // bit i: key key0 + i
                    seen = 0;
                    #pragma unroll
                    for (int nt = 0; nt < XT; ++nt)
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int key = key0 + key_of(nt, k);
                            const bool ok = key < lim[row_of(k)] && (live >> key_of(nt, k) & 1);
                            if (ok) seen |= 1u << (4 * nt + k);
                            else x[nt][k] = NEG_INF;
                        }
                }
                // --- running maximum, moved only when it is passed by LAZY ---
                float top0 = NEG_INF, top1 = NEG_INF;
                #pragma unroll
                for (int nt = 0; nt < XT; ++nt) {
                    top0 = fmaxf(top0, fmaxf(x[nt][0], x[nt][NARROW ? 2 : 1]));
                    top1 = fmaxf(top1, fmaxf(x[nt][NARROW ? 1 : 2], x[nt][3]));
                }
                if (__any_sync(0xffffffffu, top0 > m[0] + LAZY || top1 > m[1] + LAZY)) {
                    #pragma unroll
                    for (int d = NARROW ? 4 : 1; d < (NARROW ? 32 : 4); d <<= 1) {
                        top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, d));
                        top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, d));
                    }
                    const float n0 = fmaxf(m[0], top0), n1 = fmaxf(m[1], top1);
                    const float f0 = m[0] == n0 ? 1.f : ex2(m[0] - n0), f1 = m[1] == n1 ? 1.f : ex2(m[1] - n1);
                    m[0] = n0; m[1] = n1;
                    l[0] *= f0; l[1] *= f1;
                    #pragma unroll
                    for (int j = 0; j < OT; ++j)
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) o[j][k] *= row_of(k) ? f1 : f0;
                }
                const float s0 = m[0] == NEG_INF ? 0.f : m[0] - HEAD, s1 = m[1] == NEG_INF ? 0.f : m[1] - HEAD;
                #pragma unroll
                for (int nt = 0; nt < XT; ++nt)
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) x[nt][k] = ex2(x[nt][k] - (row_of(k) ? s1 : s0));
                if (!edge) {
                    #pragma unroll
                    for (int nt = 0; nt < XT; ++nt)
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) l[row_of(k)] = fmaf(x[nt][k], iv[block_of(nt)], l[row_of(k)]);
                } else {
                    // a masked weight is 0 whatever its block's scale is
                    #pragma unroll
                    for (int nt = 0; nt < XT; ++nt)
                        #pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (seen >> (4 * nt + k) & 1) l[row_of(k)] = fmaf(x[nt][k], iv[block_of(nt)], l[row_of(k)]);
                }
                #pragma unroll
                for (int b = 0; b < 2; ++b) {
                    uint32_t p[4];                           // NARROW: two registers, keys along a thread
                    #pragma unroll
                    for (int nt = 0; nt < XT / 2; ++nt) {
                        const int xt = b * (XT / 2) + nt;
                        const __half2 pa = __floats2half2_rn(x[xt][0], x[xt][1]);
                        const __half2 pb = __floats2half2_rn(x[xt][2], x[xt][3]);
                        p[2 * nt] = *reinterpret_cast<const uint32_t*>(&pa);
                        p[2 * nt + 1] = *reinterpret_cast<const uint32_t*>(&pb);
                    }
                    if constexpr (NARROW) {
                        p[0] = transposed(p[0]);
                        p[1] = transposed(p[1]);
                    }
                    // --- values: keys 2t, 2t+1, 2t+8, 2t+9 of the block, columns DN g .. ---
                    const uint8_t* vst = stage + (WKEYS + 16 * b) * D;
                    #pragma unroll
                    for (int c = 0; c < D / 64; ++c) {       // 8 columns at a time
                        uint2 r[4];
                        #pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int key = 2 * t + (k & 1) + 8 * (k >> 1);
                            if (D == 128)
                                r[k] = *reinterpret_cast<const uint2*>(vst + stage_offset<D>(key, g) + 8 * c);
                            else
                                r[k] = *reinterpret_cast<const uint2*>(vst + stage_offset<D>(key, g >> 1) + 8 * (g & 1));
                        }
                        #pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t k0w = w ? r[0].y : r[0].x, k1w = w ? r[1].y : r[1].x;
                            const uint32_t k8w = w ? r[2].y : r[2].x, k9w = w ? r[3].y : r[3].x;
                            const uint32_t lo01 = prmt(k0w, k1w, 0x5140u), hi01 = prmt(k0w, k1w, 0x7362u);
                            const uint32_t lo89 = prmt(k8w, k9w, 0x5140u), hi89 = prmt(k8w, k9w, 0x7362u);
                            // two keys' codes of channels 4w .. 4w + 3 of the eight
                            const uint32_t e[4] = {codes_half2(prmt(lo01, 0x64646464u, 0x4140u)),
                                                   codes_half2(prmt(lo01, 0x64646464u, 0x4342u)),
                                                   codes_half2(prmt(hi01, 0x64646464u, 0x4140u)),
                                                   codes_half2(prmt(hi01, 0x64646464u, 0x4342u))};
                            const uint32_t f[4] = {codes_half2(prmt(lo89, 0x64646464u, 0x4140u)),
                                                   codes_half2(prmt(lo89, 0x64646464u, 0x4342u)),
                                                   codes_half2(prmt(hi89, 0x64646464u, 0x4140u)),
                                                   codes_half2(prmt(hi89, 0x64646464u, 0x4342u))};
                            if constexpr (NARROW) {
                                #pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const uint32_t va[4] = {e[2 * k], e[2 * k + 1], f[2 * k], f[2 * k + 1]};
                                    mma_16816(o[4 * c + 2 * w + k], va, p[0], p[1]);
                                }
                            } else {
                                #pragma unroll
                                for (int k = 0; k < 4; ++k) mma_16816(o[8 * c + 4 * w + k], p, e[k], f[k]);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            st = (st + 1) % STAGES<NARROW>;
            --left;
            ++tau;
            if (++cur.kt == cur.s.nt || left == 0) {
                // --- end of the unit in this CTA: join the four warps --------
                float* buf = reinterpret_cast<float*>(smem + SM::RING);            // [16][D]
                float2* ml = reinterpret_cast<float2*>(smem + SM::RING + ROWS * D * 4);   // [warp][16]
                #pragma unroll
                for (int k = 0; k < 2; ++k)
                    #pragma unroll
                    for (int d = NARROW ? 4 : 1; d < (NARROW ? 32 : 4); d <<= 1) l[k] += __shfl_xor_sync(0xffffffffu, l[k], d);
                const int own[2] = {NARROW ? 2 * t : g, NARROW ? 2 * t + 1 : g + 8};       // this thread's rows
                const bool first_of_row = (NARROW ? g : t) == 0;
                if (first_of_row) {
                    ml[warp * ROWS + own[0]] = make_float2(m[0], l[0]);
                    ml[warp * ROWS + own[1]] = make_float2(m[1], l[1]);
                }
                __syncthreads();
                float mm[2], ll[2];
                #pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float top = NEG_INF;
                    #pragma unroll
                    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, ml[w * ROWS + own[k]].x);
                    float sum = 0.f;
                    #pragma unroll
                    for (int w = 0; w < WARPS; ++w) {
                        const float2 v = ml[w * ROWS + own[k]];
                        if (v.x != NEG_INF || v.y != 0.f) sum += v.y * (v.x == top ? 1.f : ex2(v.x - top));
                    }
                    mm[k] = top; ll[k] = sum;
                    const float f = m[k] == top ? 1.f : ex2(m[k] - top);           // 0 for a warp that saw nothing
                    #pragma unroll
                    for (int j = 0; j < OT; ++j) {
                        o[j][NARROW ? k : 2 * k] *= f;
                        o[j][NARROW ? 2 + k : 2 * k + 1] *= f;
                    }
                }
                for (int w = 0; w < WARPS; ++w) {
                    if (warp == w) {
                        #pragma unroll
                        for (int k = 0; k < (NARROW ? 2 : 4); ++k) {
                            float4* dst = reinterpret_cast<float4*>(
                                buf + (NARROW ? own[k & 1] * D + DN * g : own[k >> 1] * D + DN * (2 * t + (k & 1))));
                            #pragma unroll
                            for (int j = 0; j < DN; j += 4) {
                                float4 v;
                                if constexpr (NARROW)
                                    v = make_float4(o[j / 2][k], o[j / 2][2 + k], o[j / 2 + 1][k], o[j / 2 + 1][2 + k]);
                                else v = make_float4(o[j][k], o[j + 1][k], o[j + 2][k], o[j + 3][k]);
                                if (w > 0) {
                                    const float4 u = dst[j / 4];
                                    v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                                }
                                dst[j / 4] = v;
                            }
                        }
                    }
                    __syncthreads();
                }
                if (warp == 0 && first_of_row) {
                    ml[own[0]] = make_float2(mm[0], ll[0]);
                    ml[own[1]] = make_float2(mm[1], ll[1]);
                }
                __syncthreads();
                const bool whole = seg_kt0 == 0 && cur.kt == cur.s.nt;
                if (whole) {
                    for (int e = tid; e < HELD * (D / 8); e += THREADS) {
                        const int r = e / (D / 8), c = e % (D / 8);
                        const int rr = cur.rt * ROWS + r, i = rr / G, j = rr - i * G;
                        if (i >= cur.s.n) continue;
                        const float2 v = ml[r];
                        const float inv = v.y == 0.f ? 0.f : __fdiv_rn(1.f, v.y);
                        float f[8];
                        #pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] = v.y == 0.f ? 0.f : buf[r * D + 8 * c + k] * inv;
                        const size_t row = (size_t)(cur.s.row0 + i);
                        Eight<T>::store(static_cast<T*>(a.Out) + row * a.ldo + (size_t)(cur.h * G + j) * D + 8 * c, f);
                        if (c == 0 && a.lse != nullptr)
                            a.lse[row * a.H + cur.h * G + j] =
                                v.y == 0.f ? NEG_INF : (log2f(v.y) + (v.x - HEAD)) * 0.6931471805599453f;
                    }
                } else {
                    // slot 0: the run begins with (or inside) this unit; slot 1: it ends in it
                    const bool first = tau == cur.kt - seg_kt0;
                    float* dst = slots + ((size_t)blockIdx.x * 2 + (first ? 0 : 1)) * slot_floats(ROWS, D);
                    for (int e = tid; e < HELD * D / 4; e += THREADS)
                        reinterpret_cast<float4*>(dst)[e] = reinterpret_cast<const float4*>(buf)[e];
                    if (tid < HELD) reinterpret_cast<float2*>(dst + ROWS * D)[tid] = ml[tid];
                }
                __syncthreads();
                if (left > 0) cur.next_unit(a, G);
                fresh = true;
            }
        }
    }
    cp_async_wait<0>();
}

template <typename T, int D, bool NARROW>
cudaError_t launch_rows(const KvAttnArgs& args, cudaStream_t s) {
    const int ctas = num_sms() * CTAS_PER_SM<NARROW>;
    KvAttnArgs a = args;
    a.whole = whole_units(a, ROWS, TILE, ctas);
    const int G = a.H / a.c.Hkv;
    static DeviceCache<int> ready;
    int dummy = 0;
    cudaError_t e = ready.get(&dummy, [](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(kv_attention_kernel<T, D, NARROW>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    AttnSmem<T, D, NARROW>::BYTES);
    });
    if (e != cudaSuccess) return e;
    long long* prefix = static_cast<long long*>(a.workspace);
    float* slots = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + prefix_bytes(a.B));
    if ((e = launch_overlapped(kv_attention_kernel<T, D, NARROW>, dim3(ctas), THREADS, AttnSmem<T, D, NARROW>::BYTES, s,
                               a, G, prefix, slots)) != cudaSuccess || a.whole)
        return e;
    return launch_join<T, D, ROWS, TILE>(a, G, ctas, ROWS, prefix, slots, s);
}

template <typename T, int D>
cudaError_t launch_typed(const KvAttnArgs& a, cudaStream_t s) {
    return a.max_new * (a.H / a.c.Hkv) <= 8 ? launch_rows<T, D, true>(a, s) : launch_rows<T, D, false>(a, s);
}

}  // namespace

// Which kernel. This one reads a unit's keys once for every 16 rows; the
// tcgen05 kernel reads them once, at up to three times the speed with many
// rows, but begins and ends slower. Up to 64 rows and a bounded number of
// (16 rows) x (cached tokens) come here, half as many with four times 16 rows,
// whose keys are converted most often. max_len is the bound that the host
// knows: a generous one leads to the other kernel. Measured, this kernel / that
// one, us (bf16, 8 query heads on a key/value head, causal; units = sequences x
// key/value heads; a key mask changes either by less than a tenth):
//   heads of 64, 24 rows: 64 units of 4000 tokens 20 / 27, 16000 tokens 50 / 58;
//     40 rows: 32 units of 8000 tokens 25 / 27, 64 of 16000 66 / 59; 64 rows:
//     32 units of 4000 tokens 21 / 23, 8000 tokens 30 / 27, 440 of 300 32 / 31
//   heads of 128, 24 rows: 32 units of 4000 tokens 28 / 31, 64 of 16000 79 / 77;
//     40 rows: 32 units of 2000 tokens 26 / 28, 4000 tokens 32 / 31, 64 of 2000
//     35 / 32; 64 rows: 32 units of 1000 tokens 24 / 27, 2000 tokens 29 / 28,
//     64 of 600 22 / 20, 2 of 8000 (this one) 21 / 17
// Where it errs: up to 32 rows of hundreds of units (440 of 2000 tokens, 24
// rows: 53 / 84 with heads of 64, 92 / 119 with heads of 128) go to the slower
// kernel, and 64 rows of 64 units of 1000 tokens with heads of 128 (27 / 29).
static bool warp_kernel(const KvAttnArgs& a) {
    const long long rows = (long long)a.max_new * (a.H / a.c.Hkv), tiles = (rows + ROWS - 1) / ROWS;
    if (tiles <= 1) return true;
    return tiles <= 4 && tiles * a.B * a.c.Hkv * (long long)a.max_len <= (a.c.D == 64 ? 1 << 20 : 1 << 18) >> (tiles == 4);
}

// Enough for either kernel, since max_len may change from call to call.
size_t kv_attention_workspace_bytes(int B, int max_new, int H, int Hkv, int D) {
    const long long rows = (long long)max_new * (H / Hkv);
    size_t slots = rows <= 4 * ROWS ? (size_t)num_sms() * MOST_CTAS * 2 * slot_floats(ROWS, D) * 4 : 0;
    if (rows > ROWS) slots = std::max(slots, kv_attention_tc_slot_bytes((int)(rows < 256 ? rows : 256), D));
    return prefix_bytes(B) + slots;
}

cudaError_t launch_kv_attention(const KvAttnArgs& a, cudaStream_t s) {
    if (!warp_kernel(a)) return launch_kv_attention_tc(a, s);
    if (a.dtype == STARQ_BF16)
        return a.c.D == 64 ? launch_typed<__nv_bfloat16, 64>(a, s) : launch_typed<__nv_bfloat16, 128>(a, s);
    return a.c.D == 64 ? launch_typed<__half, 64>(a, s) : launch_typed<__half, 128>(a, s);
}

}  // namespace starq
