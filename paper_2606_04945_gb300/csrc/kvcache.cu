// The paged 8-bit key/value cache: appending rows (keys rotated on the way)
// and reading rows back.
//
// A block is the tokens of one page and one key/value head: codes
// [page][D], one float32 scale for keys and one for values. A value is
// s (byte - 128) with byte - 128 in [-127, 127].
//
// Appending rows x to a block that keeps n rows (its first n):
//   top = max |x| over the new rows' channels (rotated keys in float32)
//   s'  = max(s if n > 0, top / 127, 2^-100)
//   kept codes c -> rne(c s / s')           (only when s' > s)
//   new codes    -> clamp(rne(x (1 / s')), -127, 127)
// The scale of a block that keeps rows never shrinks, so appending the same
// rows behind the same prefix again gives the same block. A value that is
// not finite makes the block's scale NaN and its codes 0: every read of the
// block shows it, and it stays so until the block is begun anew.
//
// Memory-bound: the new rows are read once into registers (rotated there),
// the maximum is taken over the CTA, and the codes are written once; a
// block's kept codes move only when its scale grows. One CTA per (sequence,
// touched block, head, keys or values) owns the block, so nothing is shared
// between CTAs and no atomics are needed. The queries' rotation rides in the
// same launch, in CTAs after the blocks'. The rows are on their way, as they
// lie in memory, before the page is known and the table is read. Measured
// (bfloat16, 4 sequences of 2048 rows behind 37, 28 heads on 4 of 128
// channels, then read back; 131 MB): 28.8 us, 4.5 TB/s; 42 us with floats
// held while loads are on their way and CTAs of 256 threads (64: 34 us).
// One token for each of 64 sequences, appended and read back (7.8 MB), takes
// 7.1 us, which is two launches and their chains of five dependent loads.
#include <limits.h>

#include "decode.cuh"

namespace starq {
namespace {

constexpr int Q_HEADS = 4;          // heads that share a thread's table entries (queries)

__device__ __forceinline__ uint32_t code_byte(float x, float r) {
    const float q = fminf(fmaxf(rintf(__fmul_rn(x, r)), -127.f), 127.f);
    return (uint32_t)((int)q + 128);
}

template <typename T, int D, int PAGE>
struct AppendShape {
    static constexpr int UNITS = PAGE * D / 16;                          // 16-channel units of a block
    static constexpr int THREADS = UNITS < 128 ? UNITS : 128;            // at least two warps (16 x 64)
    static constexpr int PER = UNITS / THREADS;
};

template <typename T, int D, int PAGE>
__global__ void __launch_bounds__(AppendShape<T, D, PAGE>::THREADS)
kv_append_kernel(const KvAppendArgs a, int blocks_per_seq, unsigned kv_ctas, int q_groups, unsigned q_items) {
    using S = AppendShape<T, D, PAGE>;
    constexpr int U = D / 16;                // units per row
    grid_dependency_wait();
    if (blockIdx.x >= kv_ctas) {             // the queries' rotation
        const unsigned t = (blockIdx.x - kv_ctas) * S::THREADS + threadIdx.x;
        if (t >= q_items) return;
        const int u = (int)(t % U);
        const unsigned tg = t / U;
        const int g = (int)(tg % (unsigned)q_groups);
        const int tok = (int)(tg / (unsigned)q_groups);
        const bool turn = u < a.rot / 16;
        const int lo = turn ? rope_unit_lo(u, a.interleaved) : 16 * u;
        const int hi = turn ? rope_unit_hi(u, a.rot, a.interleaved) : 16 * u + 8;
        const T* x = static_cast<const T*>(a.Q) + (size_t)tok * a.ldq;
        T* y = static_cast<T*>(a.Qo) + (size_t)tok * a.ldqo;
        Packed8<T> l[Q_HEADS], h[Q_HEADS];
        #pragma unroll
        for (int k = 0; k < Q_HEADS; ++k) {
            const int head = g + k * q_groups;
            if (head < a.H) {
                l[k].load(x + head * D + lo);
                h[k].load(x + head * D + hi);
            }
        }
        float2 cs[8];
        if (turn) rope_load(cs, a.table, a.positions, a.rot, __ldg(a.pos + tok), u, 0, a.status);
        #pragma unroll
        for (int k = 0; k < Q_HEADS; ++k) {
            const int head = g + k * q_groups;
            if (head < a.H) {
                float p[8], q[8];
                l[k].open(p);
                h[k].open(q);
                if (turn) rope_unit(p, q, cs, a.interleaved);
                Eight<T>::store(y + head * D + lo, p);
                Eight<T>::store(y + head * D + hi, q);
            }
        }
        return;
    }

    __shared__ unsigned part[S::THREADS / 32];
    // CTA -> (sequence, touched block, head, keys / values)
    unsigned id = blockIdx.x;
    const bool values = id & 1;
    id >>= 1;
    const int head = (int)(id % (unsigned)a.c.Hkv);
    id /= (unsigned)a.c.Hkv;
    const int blk = (int)(id % (unsigned)blocks_per_seq);
    const int b = (int)(id / (unsigned)blocks_per_seq);
    const int row0 = __ldg(a.seq_start + b), n = __ldg(a.seq_start + b + 1) - row0;
    const int past = __ldg(a.past + b);
    if (n == 0) return;
    // a range that does not fit its bounds: nothing is written
    if (n < 0 || n > a.max_new || row0 < 0 || row0 > a.T - n || past < 0 || past > INT_MAX - 256 - a.max_new) {
        if (threadIdx.x == 0) atomicOr(a.status, STATUS_RANGE);
        return;
    }
    const int page_i = past / PAGE + blk;
    const int slot0 = page_i * PAGE;                     // first slot of the block
    if (slot0 >= past + n) return;
    int page = -1;
    if (page_i < a.table_ld) page = __ldg(a.page_table + (size_t)b * a.table_ld + page_i);
    const int kept = max(0, past - slot0);               // rows of the block that stay
    const int end = min(PAGE, past + n - slot0);         // rows [kept, end) are new
    const T* src = static_cast<const T*>(values ? a.V : a.K);
    const int ld = values ? a.ldv : a.ldk;
    const int rot = values ? 0 : a.rot;

    // The new rows' units, dense over the threads: unit j covers row
    // kept + j / U. At most PER units a thread, all on their way before the
    // page is known.
    const int todo = (end - kept) * U;
    Packed8<T> pl[S::PER], ph[S::PER];
    int pos[S::PER];
    #pragma unroll
    for (int k = 0; k < S::PER; ++k) {
        const int j = threadIdx.x + k * S::THREADS;
        if (j < todo) {
            const int u = j % U, row = row0 + (slot0 + kept + j / U - past);
            const bool turn = u < rot / 16;
            const T* x = src + (size_t)row * ld + head * D;
            pl[k].load(x + (turn ? rope_unit_lo(u, a.interleaved) : 16 * u));
            ph[k].load(x + (turn ? rope_unit_hi(u, rot, a.interleaved) : 16 * u + 8));
            if (turn) pos[k] = __ldg(a.pos + row);
        }
    }
    if (page < 0 || page >= a.c.pages) {
        if (threadIdx.x == 0) atomicOr(a.status, STATUS_RANGE);
        return;
    }
    const size_t blk_id = (size_t)page * a.c.Hkv + head;
    uint8_t* codes = (values ? a.c.V : a.c.K) + blk_id * (PAGE * D);
    float* scale = (values ? a.c.v_scale : a.c.k_scale) + blk_id;
    const float old = kept > 0 ? *scale : 0.f;
    float lo[S::PER][8], hi[S::PER][8];
    unsigned top = 0;                                    // max of |x| as bits: NaN above infinity above the rest
    #pragma unroll
    for (int k = 0; k < S::PER; ++k) {
        const int j = threadIdx.x + k * S::THREADS;
        if (j < todo) {
            const int u = j % U;
            pl[k].open(lo[k]);
            ph[k].open(hi[k]);
            if (u < rot / 16) {
                float2 cs[8];
                rope_load(cs, a.table, a.positions, rot, pos[k], u, 0, a.status);
                rope_unit(lo[k], hi[k], cs, a.interleaved);
            }
            #pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = max(top, __float_as_uint(lo[k][i]) & 0x7fffffffu);
                top = max(top, __float_as_uint(hi[k][i]) & 0x7fffffffu);
            }
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
    #pragma unroll
    for (int w = 0; w < S::THREADS / 32; ++w) top = max(top, part[w]);
    const bool bad = top >= 0x7f800000u || old != old;   // not finite, or poisoned before
    const float s = bad ? __uint_as_float(0x7fffffffu)
                        : fmaxf(fmaxf(old, __fdiv_rn(__uint_as_float(top), 127.f)), KV_SCALE_FLOOR);
    const float r = bad ? 0.f : __fdiv_rn(1.f, s);
    if (kept > 0 && (bad || s > old)) {                  // the kept rows' codes on the grown scale
        const float ratio = bad ? 0.f : __fdiv_rn(old, s);
        uint4* c4 = reinterpret_cast<uint4*>(codes);
        for (int j = threadIdx.x; j < kept * U; j += S::THREADS) {
            uint4 v = c4[j];
            uint32_t* w = reinterpret_cast<uint32_t*>(&v);
            #pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t o = 0;
                #pragma unroll
                for (int k = 0; k < 4; ++k)
                    o |= code_byte((float)((int)((w[i] >> (8 * k)) & 0xff) - 128), ratio) << (8 * k);
                w[i] = o;
            }
            c4[j] = v;
        }
    }
    #pragma unroll
    for (int k = 0; k < S::PER; ++k) {
        const int j = threadIdx.x + k * S::THREADS;
        if (j < todo) {
            const int u = j % U, row = kept + j / U;
            const bool turn = u < rot / 16;
            const int cl = turn ? rope_unit_lo(u, a.interleaved) : 16 * u;
            const int ch = turn ? rope_unit_hi(u, rot, a.interleaved) : 16 * u + 8;
            uint2 l = make_uint2(0x80808080u, 0x80808080u), h = l;
            if (!bad) {
                l = h = make_uint2(0, 0);
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    l.x |= code_byte(lo[k][i], r) << (8 * i);
                    l.y |= code_byte(lo[k][4 + i], r) << (8 * i);
                    h.x |= code_byte(hi[k][i], r) << (8 * i);
                    h.y |= code_byte(hi[k][4 + i], r) << (8 * i);
                }
            }
            *reinterpret_cast<uint2*>(codes + row * D + cl) = l;
            *reinterpret_cast<uint2*>(codes + row * D + ch) = h;
        }
    }
    if (threadIdx.x == 0) *scale = s;
}

// One thread per 16 channels of a key and of a value row: grid.y sequences.
template <typename T, int D>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvReadArgs a) {
    constexpr int U = D / 16;
    grid_dependency_wait();
    const int b = blockIdx.y;
    const int row0 = __ldg(a.out_start + b), n = __ldg(a.out_start + b + 1) - row0;
    const int first = __ldg(a.first + b);
    if (n == 0) return;
    if (n < 0 || n > a.max_rows || row0 < 0 || row0 > a.T - n || first < 0 || first > INT_MAX - n) {
        if (threadIdx.x == 0) atomicOr(a.status, STATUS_RANGE);
        return;
    }
    const size_t items = (size_t)n * a.c.Hkv * U;
    for (size_t t = (size_t)blockIdx.x * 256 + threadIdx.x; t < items; t += (size_t)gridDim.x * 256) {
        const int u = (int)(t % U);
        const size_t th = t / U;
        const int head = (int)(th % a.c.Hkv);
        const int i = (int)(th / a.c.Hkv);
        const int slot = first + i, page_i = slot / a.c.page;
        int page = -1;
        if (page_i < a.table_ld) page = __ldg(a.page_table + (size_t)b * a.table_ld + page_i);
        if (page < 0 || page >= a.c.pages) { atomicOr(a.status, STATUS_RANGE); continue; }
        const size_t blk = (size_t)page * a.c.Hkv + head;
        const size_t at = (blk * a.c.page + slot % a.c.page) * D + 16 * u;
        const size_t to = (size_t)(row0 + i) * a.ld + (size_t)head * D + 16 * u;
        #pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            T* out = static_cast<T*>(kv ? a.V : a.K);
            if (out == nullptr) continue;
            const uint4 c = *reinterpret_cast<const uint4*>((kv ? a.c.V : a.c.K) + at);
            const float s = (kv ? a.c.v_scale : a.c.k_scale)[blk];
            const uint32_t w[4] = {c.x, c.y, c.z, c.w};
            float f[2][8];
            #pragma unroll
            for (int k = 0; k < 16; ++k)
                f[k >> 3][k & 7] = __fmul_rn((float)((int)((w[k >> 2] >> (8 * (k & 3))) & 0xff) - 128), s);
            Eight<T>::store(out + to, f[0]);
            Eight<T>::store(out + to + 8, f[1]);
        }
    }
}

template <typename T, int D, int PAGE>
cudaError_t launch_append_shape(const KvAppendArgs& a, cudaStream_t s) {
    using S = AppendShape<T, D, PAGE>;
    // blocks that max_new rows can touch from any offset
    const size_t per_seq = ((size_t)a.max_new + PAGE - 2) / PAGE + 1;
    const size_t kv = (size_t)a.B * per_seq * a.c.Hkv * 2;
    const int groups = (a.H + Q_HEADS - 1) / Q_HEADS;
    const size_t items = a.Q != nullptr ? (size_t)a.T * groups * (D / 16) : 0;
    const size_t grid = kv + (items + S::THREADS - 1) / S::THREADS;
    if (grid > 0x7fffffffull || items > 0x7fffffffull) return cudaErrorInvalidValue;
    return launch_overlapped(kv_append_kernel<T, D, PAGE>, dim3((unsigned)grid), S::THREADS, 0, s, a, (int)per_seq,
                             (unsigned)kv, groups, (unsigned)items);
}

template <typename T, int D>
cudaError_t launch_append_page(const KvAppendArgs& a, cudaStream_t s) {
    switch (a.c.page) {
        case 16: return launch_append_shape<T, D, 16>(a, s);
        case 32: return launch_append_shape<T, D, 32>(a, s);
        case 64: return launch_append_shape<T, D, 64>(a, s);
        default: return launch_append_shape<T, D, 128>(a, s);
    }
}

template <typename T>
cudaError_t launch_read_typed(const KvReadArgs& a, cudaStream_t s) {
    const size_t items = (size_t)a.max_rows * a.c.Hkv * (a.c.D / 16);
    size_t x = (items + 255) / 256;
    const size_t cap = ((size_t)num_sms() * 32 + a.B - 1) / a.B;       // about 32 CTAs per SM in all
    if (x > cap) x = cap;
    const dim3 grid((unsigned)x, (unsigned)a.B);
    if (a.c.D == 64) return launch_overlapped(kv_read_kernel<T, 64>, grid, 256, 0, s, a);
    return launch_overlapped(kv_read_kernel<T, 128>, grid, 256, 0, s, a);
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs& a, cudaStream_t s) {
    if (a.dtype == STARQ_BF16)
        return a.c.D == 64 ? launch_append_page<__nv_bfloat16, 64>(a, s) : launch_append_page<__nv_bfloat16, 128>(a, s);
    return a.c.D == 64 ? launch_append_page<__half, 64>(a, s) : launch_append_page<__half, 128>(a, s);
}

cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s) {
    switch (a.dtype) {
        case STARQ_F16: return launch_read_typed<__half>(a, s);
        case STARQ_BF16: return launch_read_typed<__nv_bfloat16>(a, s);
        default: return launch_read_typed<float>(a, s);
    }
}

}  // namespace starq
