// Rotary position embedding from a table: a table of cosines and sines
// (plain, or scaled for contexts longer than the trained one), and its
// application to the heads of a row in the half or the interleaved layout,
// on all or the first `rot` channels of a head, forward or transposed (the
// gradient: the rotation is orthogonal up to the table's factor, so the
// gradient of y = R x is R^T g, the same pass with the sine negated).
//
// Table: entry (p, i) = m (cos(p f_i), sin(p f_i)), angles, cosines and
// sines in float64, one rounding to float32. A float32 angle would be off by
// up to p 2^-24 radians, which a long context shows.
//
// rope_apply is bound by memory: every channel is read and written once
// (2 + 2 bytes), three float32 operations for each. A thread takes the same
// eight pairs of HEADS heads of a token, so that a table entry is loaded once
// for HEADS heads and 2 * HEADS 16-byte loads are in flight; they wait in
// registers as they lie in memory. Measured (bfloat16, 8192 rows of 32 heads
// of 128, 138 MB): 24.0 us, 5.8 TB/s; 35 us with floats instead (128
// registers), 25 us with CTAs of 256, 31 us with a head a thread.
#include <math.h>

#include "decode.cuh"

namespace starq {
namespace {

constexpr int THREADS = 128;
constexpr int HEADS = 4;

__global__ void rope_table_kernel(float2* __restrict__ table, int positions, int rot, double theta, int scaling,
                                  double factor, double low, double high, double m) {
    const int half = rot / 2;
    const size_t n = (size_t)positions * half;
    for (size_t t = (size_t)blockIdx.x * blockDim.x + threadIdx.x; t < n; t += (size_t)gridDim.x * blockDim.x) {
        const int i = (int)(t % half);
        const size_t p = t / half;
        double f = pow(theta, -(double)(2 * i) / (double)rot);
        if (scaling == STARQ_ROPE_LINEAR) f /= factor;
        if (scaling == STARQ_ROPE_PARTS) {
            const double ramp = fmin(fmax(((double)i - low) / (high - low), 0.0), 1.0);
            f = f / factor * ramp + f * (1.0 - ramp);
        }
        double s, c;
        sincos((double)p * f, &s, &c);
        table[t] = make_float2((float)(c * m), (float)(s * m));
    }
}

// Thread -> (token, group of HEADS heads, unit of 16 channels). Units below
// rot / 16 rotate; the others copy their 16 channels (not in place).
template <typename T>
__global__ void __launch_bounds__(THREADS) rope_apply_kernel(const RopeArgs a, int groups, int units, unsigned n) {
    grid_dependency_wait();
    const unsigned t = blockIdx.x * THREADS + threadIdx.x;
    if (t >= n) return;
    const int u = (int)(t % (unsigned)units);
    const unsigned tg = t / (unsigned)units;
    const int g = (int)(tg % (unsigned)groups);
    const int tok = (int)(tg / (unsigned)groups);
    const bool turn = u < a.rot / 16;
    const int lo = turn ? rope_unit_lo(u, a.interleaved) : 16 * u;
    const int hi = turn ? rope_unit_hi(u, a.rot, a.interleaved) : 16 * u + 8;
    const T* x = static_cast<const T*>(a.X) + (size_t)tok * a.ldx;
    T* y = static_cast<T*>(a.Y) + (size_t)tok * a.ldy;
    Packed8<T> l[HEADS], h[HEADS];
    #pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int head = g + k * groups;
        if (head < a.heads) {
            l[k].load(x + (size_t)head * a.D + lo);
            h[k].load(x + (size_t)head * a.D + hi);
        }
    }
    float2 cs[8];
    if (turn) rope_load(cs, a.table, a.positions, a.rot, __ldg(a.pos + tok), u, a.inverse, a.status);
    #pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int head = g + k * groups;
        if (head < a.heads) {
            float p[8], q[8];
            l[k].open(p);
            h[k].open(q);
            if (turn) rope_unit(p, q, cs, a.interleaved);
            Eight<T>::store(y + (size_t)head * a.D + lo, p);
            Eight<T>::store(y + (size_t)head * a.D + hi, q);
        }
    }
}

// Any even rot, any D and any alignment: one thread for each rotation pair
// or copied channel.
template <typename T>
__global__ void __launch_bounds__(THREADS) rope_apply_scalar_kernel(const RopeArgs a, size_t n) {
    grid_dependency_wait();
    const int half = a.rot / 2, per = half + (a.D - a.rot);
    for (size_t t = (size_t)blockIdx.x * THREADS + threadIdx.x; t < n; t += (size_t)gridDim.x * THREADS) {
        const int i = (int)(t % per);
        const size_t th = t / per;
        const int head = (int)(th % a.heads);
        const size_t tok = th / a.heads;
        const T* x = static_cast<const T*>(a.X) + tok * a.ldx + (size_t)head * a.D;
        T* y = static_cast<T*>(a.Y) + tok * a.ldy + (size_t)head * a.D;
        if (i >= half) { y[a.rot + i - half] = x[a.rot + i - half]; continue; }
        const int lo = a.interleaved ? 2 * i : i, hi = a.interleaved ? 2 * i + 1 : i + half;
        const int p = a.pos[tok];
        float2 cs = make_float2(1.f, 0.f);
        if (p < 0 || p >= a.positions) atomicOr(a.status, STATUS_RANGE);
        else cs = a.table[(size_t)p * half + i];
        float u = (float)x[lo], v = (float)x[hi];
        rope_pair(u, v, cs.x, a.inverse ? -cs.y : cs.y);
        y[lo] = (T)u;
        y[hi] = (T)v;
    }
}

template <typename T>
cudaError_t launch_typed(const RopeArgs& a, cudaStream_t s) {
    const size_t e = sizeof(T);
    const bool wide = a.D % 16 == 0 && a.rot % 16 == 0 && (a.ldx * e) % 16 == 0 && (a.ldy * e) % 16 == 0 &&
                      reinterpret_cast<uintptr_t>(a.X) % 16 == 0 && reinterpret_cast<uintptr_t>(a.Y) % 16 == 0 &&
                      reinterpret_cast<uintptr_t>(a.table) % 16 == 0;
    const int groups = (a.heads + HEADS - 1) / HEADS;
    // in place, the channels that do not rotate stay where they are
    const int units = (a.X == a.Y && a.ldx == a.ldy ? a.rot : a.D) / 16;
    const size_t n = (size_t)a.L * groups * units;
    if (wide && n == 0) return cudaSuccess;
    if (wide && n < (1ull << 31)) {
        return launch_overlapped(rope_apply_kernel<T>, dim3((unsigned)((n + THREADS - 1) / THREADS)), THREADS, 0, s, a, groups,
                                 units, (unsigned)n);
    } else {
        const size_t m = (size_t)a.L * a.heads * (a.rot / 2 + (a.D - a.rot));
        size_t blocks = (m + THREADS - 1) / THREADS;
        const size_t cap = (size_t)num_sms() * 32;
        if (blocks > cap) blocks = cap;
        return launch_overlapped(rope_apply_scalar_kernel<T>, dim3((unsigned)blocks), THREADS, 0, s, a, m);
    }
}

}  // namespace

cudaError_t launch_rope_table(float2* table, int positions, int rot, double theta, int scaling, double factor,
                              double original, double beta_fast, double beta_slow, double mscale, cudaStream_t s) {
    double low = 0.0, high = 1.0;
    if (scaling == STARQ_ROPE_NTK) theta *= rot > 2 ? pow(factor, (double)rot / (double)(rot - 2)) : 1.0;
    if (scaling == STARQ_ROPE_PARTS) {
        // the pair whose wave turns r times within the original length:
        // original f_i = 2 pi r  =>  i = rot ln(original / (2 pi r)) / (2 ln theta)
        const double pi = 3.14159265358979323846;
        auto pair = [&](double r) { return rot * log(original / (2.0 * pi * r)) / (2.0 * log(theta)); };
        low = fmax(floor(pair(beta_fast)), 0.0);
        high = fmin(ceil(pair(beta_slow)), (double)(rot - 1));
        if (high <= low) high = low + 1e-3;
    }
    const size_t n = (size_t)positions * (rot / 2);
    size_t blocks = (n + THREADS - 1) / THREADS;
    const size_t cap = (size_t)num_sms() * 32;
    if (blocks > cap) blocks = cap;
    rope_table_kernel<<<(unsigned)blocks, THREADS, 0, s>>>(table, positions, rot, theta, scaling, factor, low, high,
                                                           mscale);
    return cudaGetLastError();
}

double rope_parts_mscale(double factor) { return 0.1 * log(factor) + 1.0; }

cudaError_t launch_rope_apply(const RopeArgs& a, cudaStream_t s) {
    switch (a.dtype) {
        case STARQ_F16: return launch_typed<__half>(a, s);
        case STARQ_BF16: return launch_typed<__nv_bfloat16>(a, s);
        default: return launch_typed<float>(a, s);
    }
}

}  // namespace starq
