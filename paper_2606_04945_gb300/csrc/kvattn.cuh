// What the two attention kernels over the 8-bit cache share (kvattn.cu: few
// query rows of a key/value head; kvattn_tc.cu: many): the cutting of
// all units' key tiles into one run per CTA, and the kernel that joins the
// partial runs of a unit.
//
// A unit is a sequence, a key/value head and up to ROWS query rows (new
// tokens x query heads of the group); its work is a list of key tiles of
// TILE keys. The tiles of all units, in order, are cut into gridDim.x runs
// of equal length. A unit inside one run is written at once; otherwise each
// of its runs leaves, in slot 2 c (the run of CTA c begins with or inside the
// unit) or 2 c + 1 (it ends in it), the rows' accumulators, maxima and sums.
// Where the sequences are short by their bound, the units themselves are
// dealt out instead (`whole`), and there is nothing to join.
#pragma once

#include <algorithm>
#include <type_traits>

#include "decode.cuh"

namespace starq {
namespace {

constexpr float HEAD = 7.f;            // weights are 2^(x - m + HEAD)
constexpr float LAZY = 8.f;            // m moves when x > m + LAZY
constexpr float NEG_INF = -__builtin_huge_valf();

// Workspace: prefix [B + 1] (tiles before each sequence), then the slots:
// [rows][D] accumulators, then (m, l) for each row; an odd number of rows
// takes the room of one more, so that every slot begins on 16 bytes.
constexpr size_t prefix_bytes(int B) { return ((size_t)(B + 1) * 8 + 255) / 256 * 256; }
constexpr size_t slot_floats(int rows, int D) { return (size_t)(rows + (rows & 1)) * (D + 2); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two bytes u (code + 128) in the low bytes of 0x64uu halves (1024 + u) to
// the two codes in fp16, exactly.
__device__ __forceinline__ uint32_t codes_half2(uint32_t biased) {
    const __half2 k = __half2half2(__ushort_as_half((unsigned short)0x6480));       // 1152
    __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&biased), k);
    return *reinterpret_cast<uint32_t*>(&v);
}

// The power of two that brings a bf16 row with largest magnitude `top` into
// fp16's range (its largest value to [2^14, 2^15)), and the one that undoes it.
__device__ __forceinline__ void row_power(float top, float& up, float& down) {
    const int e = max((int)(__float_as_uint(top) >> 23) - 127, -112);
    up = __uint_as_float((uint32_t)(14 - e + 127) << 23);
    down = __uint_as_float((uint32_t)(e - 14 + 127) << 23);
}

// a / b, a >= 0 (64-bit divisions take a hundred instructions each; few lists
// of tiles need them).
__device__ __forceinline__ long long quotient(long long a, int b) {
    return a < (1ll << 31) ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

struct SeqShape { int len, n, row0, nt, rt; };       // cached tokens, new tokens, first row, key tiles, row tiles

// The lengths of sequence b; a sequence whose numbers do not fit their
// bounds counts as having no rows.
template <int ROWS, int TILE>
__device__ __forceinline__ SeqShape seq_shape(const KvAttnArgs& a, int G, int b, bool report) {
    SeqShape s;
    s.row0 = __ldg(a.seq_start + b);
    s.n = __ldg(a.seq_start + b + 1) - s.row0;
    s.len = __ldg(a.kv_len + b);
    const bool bad = s.n < 0 || s.n > a.max_new || s.row0 < 0 || s.row0 > a.T - s.n || s.len < 0 || s.len > a.max_len;
    if (bad) {
        if (report) atomicOr(a.status, STATUS_RANGE);
        s.n = 0; s.len = 0; s.row0 = 0;
    }
    // (a whole unit without keys has a tile all the same: its CTA writes its rows)
    s.nt = s.n > 0 ? max((s.len + TILE - 1) / TILE, a.whole) : 0;
    s.rt = (s.n * G + ROWS - 1) / ROWS;
    return s;
}

// This CTA's run [tau0, tau1) of the flat list of tiles (whole: of units), the
// sequence that tau0 falls into and the tiles (units) before that sequence.
// CTA 0 writes `prefix`.
struct Run { long long tau0, tau1, before; int b; };
template <int ROWS, int TILE, int THREADS>
__device__ __forceinline__ Run find_run(const KvAttnArgs& a, int G, long long* prefix) {
    constexpr int WARPS = THREADS / 32;
    __shared__ long long s_part[WARPS], s_before;
    __shared__ int s_b;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto tiles_of = [&](int b, bool report) {
        if (b >= a.B) return 0ll;
        const SeqShape s = seq_shape<ROWS, TILE>(a, G, b, report);
        return (long long)(a.whole ? s.nt > 0 : s.nt) * s.rt * a.c.Hkv;
    };
    if (a.B <= 32) {                                          // every warp by itself, without barriers
        const long long cnt = tiles_of(lane, blockIdx.x == 0 && warp == 0);
        long long sum = cnt;
        #pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += u;
        }
        const long long total = __shfl_sync(0xffffffffu, sum, 31);
        const long long share = quotient(total + gridDim.x - 1, (int)gridDim.x);
        Run r;
        r.tau0 = share * blockIdx.x;
        r.tau1 = min(total, r.tau0 + share);
        r.b = __ffs(__ballot_sync(0xffffffffu, r.tau0 >= sum - cnt && r.tau0 < sum)) - 1;
        r.before = __shfl_sync(0xffffffffu, sum - cnt, max(r.b, 0));
        if (blockIdx.x == 0 && warp == 0) {
            if (lane < a.B) prefix[lane] = sum - cnt;
            if (lane == 0) prefix[a.B] = total;
        }
        return r;
    }
    // inclusive sums over the CTA's threads; part sums of the warps in s_part
    auto scan = [&](long long v) {
        #pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, m);
            if (lane >= m) v += u;
        }
        __syncthreads();
        if (lane == 31) s_part[warp] = v;
        __syncthreads();
        for (int w = 0; w < warp; ++w) v += s_part[w];
        return v;
    };
    if (tid == 0) { s_b = -1; s_before = 0; }
    const long long first = tiles_of(tid, blockIdx.x == 0);   // the first THREADS sequences: read once
    const long long first_sum = scan(first);
    long long total = 0;
    for (int w = 0; w < WARPS; ++w) total += s_part[w];
    long long rest = 0;
    for (int b = tid + THREADS; b < a.B; b += THREADS) rest += tiles_of(b, blockIdx.x == 0);
    if (a.B > THREADS) {
        scan(rest);
        for (int w = 0; w < WARPS; ++w) total += s_part[w];
    }
    const long long share = quotient(total + gridDim.x - 1, (int)gridDim.x);
    Run r;
    r.tau0 = share * blockIdx.x;
    r.tau1 = min(total, r.tau0 + share);
    r.b = -1;
    r.before = 0;
    long long done = 0;                                       // tiles before the current chunk of sequences
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + tid;
        const long long cnt = b0 == 0 ? first : tiles_of(b, false);
        const long long at = done + (b0 == 0 ? first_sum : scan(cnt)) - cnt;
        if (b < a.B) {
            if (blockIdx.x == 0) prefix[b] = at;
            if (cnt > 0 && r.tau0 >= at && r.tau0 < at + cnt) { s_b = b; s_before = at; }
        }
        if (b0 + THREADS < a.B) {                             // the chunk's sum: its last thread's
            __shared__ long long s_done;
            if (tid == THREADS - 1) s_done = at + cnt;
            __syncthreads();
            done = s_done;
        }
    }
    if (tid == 0 && blockIdx.x == 0) prefix[a.B] = total;
    __syncthreads();
    r.b = s_b;
    r.before = s_before;
    return r;
}

// Position in the flat list of tiles: sequence, head, row tile, key tile.
template <int ROWS, int TILE>
struct Cursor {
    int b, h, rt, kt;
    SeqShape s;
    __device__ __forceinline__ void start(const KvAttnArgs& a, int G, const Run& r) {
        b = r.b;
        s = seq_shape<ROWS, TILE>(a, G, b, false);
        const long long off = r.tau0 - r.before, unit = a.whole ? off : quotient(off, s.nt);
        kt = a.whole ? 0 : (int)(off - unit * s.nt);
        h = (int)quotient(unit, s.rt);
        rt = (int)(unit - (long long)h * s.rt);
    }
    __device__ __forceinline__ void next_unit(const KvAttnArgs& a, int G) {
        kt = 0;
        if (++rt < s.rt) return;
        rt = 0;
        if (++h < a.c.Hkv) return;
        h = 0;
        do {
            if (++b >= a.B) return;
            s = seq_shape<ROWS, TILE>(a, G, b, false);
        } while (s.nt == 0);
    }
    // Tiles of the run that begins here.
    __device__ __forceinline__ int tiles(const KvAttnArgs& a, int G, const Run& r) const {
        if (!a.whole) return (int)(r.tau1 - r.tau0);
        Cursor q = *this;
        int n = q.s.nt;
        for (long long u = r.tau0 + 1; u < r.tau1; ++u) {
            q.next_unit(a, G);
            n += q.s.nt;
        }
        return n;
    }
};

// Whether units are dealt out whole, from the bounds that the host knows.
// Counted in key tiles of the busiest CTA, cutting and joining cost 2 and, as
// the joins are many, 4 for each unit a CTA; beyond 8 tiles the spread of the
// lengths under their bound would weigh more. Measured, cut / whole, us: one
// row of 28 heads on 4, 100 tokens 7.8 / 6.2, 256 tokens 8.2 / 7.4, 500 tokens
// 8.5 / 9.9 (cut); 64 such sequences, up to 300 tokens 14.8 / 11.1, 1000
// tokens 21.5 / 19.7; 32 rows of them, 8 sequences, 250 tokens 20.9 / 18.6,
// 500 tokens 21.9 / 23.4 (cut); 32 sequences, 500 tokens 48 / 24.8.
inline bool whole_units(const KvAttnArgs& a, int rows, int tile, int ctas) {
    const long long t = std::max(1, (a.max_len + tile - 1) / tile);
    const long long n = ((long long)a.max_new * (a.H / a.c.Hkv) + rows - 1) / rows * a.B * a.c.Hkv;      // units
    return t <= 8 && t * ((n + ctas - 1) / ctas) * ctas <= std::max<long long>(ctas, n * t) + 2 * ctas + 4 * n;
}

// Joins the partial runs of a row's unit, and writes the rows that no key
// reaches. SHARE warps take a row: one where there are many rows (their units
// have few runs each), all eight of a CTA where there are few (a long
// sequence's unit has up to a run per CTA). Every warp takes its runs in run
// order, AT_ONCE of them on their way together, and the warps' sums are added
// in warp order.
constexpr int JOIN_WARPS = 8;
template <typename T, int D, int ROWS, int TILE, int SHARE>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
kv_attention_join_kernel(const KvAttnArgs a, int G, int ctas, int slot_rows, const long long* prefix,
                         const float* slots) {
    constexpr int PER = D / 32, AT_ONCE = 8;
    __shared__ float s_acc[SHARE > 1 ? SHARE : 1][D];
    __shared__ float2 s_ml[SHARE > 1 ? SHARE : 1];
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % SHARE;
    const int b = blockIdx.y;
    const SeqShape s = seq_shape<ROWS, TILE>(a, G, b, false);
    const long long total = prefix[a.B], before = prefix[b];
    const int idx = blockIdx.x * (JOIN_WARPS / SHARE) + warp / SHARE;      // token * H + head
    const int i = idx / a.H, head = idx - i * a.H;
    if (i >= s.n) return;
    const size_t row = (size_t)(s.row0 + i);
    T* out = static_cast<T*>(a.Out) + row * a.ldo + (size_t)head * D + lane * PER;
    const int h = head / G, r = i * G + (head - h * G);
    const int rt = r / ROWS, rr = r - rt * ROWS;
    int c0 = 0, c1 = -1;
    long long u0 = 0, share = 1;
    if (s.nt > 0) {
        u0 = before + ((long long)h * s.rt + rt) * s.nt;
        // (64-bit divisions take a hundred instructions each; few lists need them)
        if (total < (1ll << 31)) {
            const unsigned sh = ((unsigned)total + ctas - 1) / (unsigned)ctas;
            share = sh;
            c0 = (int)((unsigned)u0 / sh);
            c1 = (int)((unsigned)(u0 + s.nt - 1) / sh);
        } else {
            share = (total + ctas - 1) / ctas;
            c0 = (int)(u0 / share);
            c1 = (int)((u0 + s.nt - 1) / share);
        }
        if (c0 == c1) return;                             // one run covered the unit
    }
    float top = NEG_INF, l = 0.f, acc[PER];
    #pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] = 0.f;
    for (int c = c0 + part; c <= c1; c += AT_ONCE * SHARE) {
        float2 ml[AT_ONCE];
        float v[AT_ONCE][PER];
        #pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
            const int cq = c + q * SHARE;
            ml[q] = make_float2(NEG_INF, 0.f);
            #pragma unroll
            for (int k = 0; k < PER; ++k) v[q][k] = 0.f;
            if (cq <= c1) {
                // the run's first slot, or its second when the unit begins inside the run
                const float* p = slots + ((size_t)cq * 2 + (cq == c0 && u0 > (long long)c0 * share ? 1 : 0)) *
                                             slot_floats(slot_rows, D);
                ml[q] = *reinterpret_cast<const float2*>(p + (size_t)slot_rows * D + 2 * rr);
                #pragma unroll
                for (int k = 0; k < PER; k += 2) {
                    const float2 w = *reinterpret_cast<const float2*>(p + (size_t)rr * D + lane * PER + k);
                    v[q][k] = w.x; v[q][k + 1] = w.y;
                }
            }
        }
        float to = top;
        #pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) to = fmaxf(to, ml[q].x);
        const float f0 = top == to ? 1.f : ex2(top - to);
        top = to;
        l *= f0;
        #pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] *= f0;
        #pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
            const float f = ml[q].x == top ? 1.f : ex2(ml[q].x - top);
            l = fmaf(ml[q].y, f, l);
            #pragma unroll
            for (int k = 0; k < PER; ++k) acc[k] = fmaf(v[q][k], f, acc[k]);
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
    #pragma unroll
    for (int k = 0; k < PER; ++k) out[k] = (T)(l == 0.f ? 0.f : acc[k] * inv);
    if (lane == 0 && a.lse != nullptr)
        a.lse[row * a.H + head] = l == 0.f ? NEG_INF : (log2f(l) + (top - HEAD)) * 0.6931471805599453f;
}

template <typename T, int D, int ROWS, int TILE>
cudaError_t launch_join(const KvAttnArgs& a, int G, int ctas, int slot_rows, const long long* prefix,
                        const float* slots, cudaStream_t s) {
    const size_t rows = (size_t)a.max_new * a.H;
    if (rows * a.B <= 4 * (size_t)num_sms())              // up to four CTAs an SM
        return launch_overlapped(kv_attention_join_kernel<T, D, ROWS, TILE, JOIN_WARPS>,
                                 dim3((unsigned)rows, (unsigned)a.B), JOIN_WARPS * 32, 0, s, a, G, ctas, slot_rows,
                                 prefix, slots);
    return launch_overlapped(kv_attention_join_kernel<T, D, ROWS, TILE, 1>,
                             dim3((unsigned)((rows + JOIN_WARPS - 1) / JOIN_WARPS), (unsigned)a.B), JOIN_WARPS * 32, 0,
                             s, a, G, ctas, slot_rows, prefix, slots);
}

}  // namespace

// kvattn_tc.cu
size_t kv_attention_tc_slot_bytes(int max_rows, int D);
cudaError_t launch_kv_attention_tc(const KvAttnArgs& a, cudaStream_t s);

}  // namespace starq
