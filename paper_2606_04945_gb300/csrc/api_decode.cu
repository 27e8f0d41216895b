// C ABI of the cached-decoding operators (declared in include/starq.h):
// argument validation and error reporting. Nothing is launched by a call
// that returns an error.
#include <cstdarg>
#include <cstdio>

#include "decode.cuh"

namespace starq {
namespace {

int fail(int code, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return report_error(code, msg);
}

int launched(cudaError_t e, const char* who) {
    return e == cudaSuccess ? STARQ_OK : fail(STARQ_ERR_CUDA, "%s launch: %s", who, cudaGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool half_type(int t) { return t == STARQ_F16 || t == STARQ_BF16; }
bool any_type(int t) { return half_type(t) || t == STARQ_F32; }

constexpr int MAX_ROWS = 1 << 28;      // rows, sequences' tokens: index sums stay inside int32

int check_cache(const char* who, const starq_kv_cache* c) {
    if (!c) return fail(STARQ_ERR_ARG, "%s: NULL cache", who);
    if (c->D != 64 && c->D != 128) return fail(STARQ_ERR_SHAPE, "%s: head size %d: 64 or 128", who, c->D);
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128)
        return fail(STARQ_ERR_SHAPE, "%s: page of %d tokens: 16, 32, 64 or 128", who, c->page);
    if (c->Hkv < 1 || c->Hkv > 65535 || c->pages < 0)
        return fail(STARQ_ERR_SHAPE, "%s: Hkv=%d, pages=%d: need 1 <= Hkv <= 65535, pages >= 0", who, c->Hkv, c->pages);
    return STARQ_OK;
}

int check_cache_pointers(const char* who, const starq_kv_cache* c) {
    if (!c->K || !c->V || !c->k_scale || !c->v_scale) return fail(STARQ_ERR_ARG, "%s: NULL array in the cache", who);
    if (!aligned(c->K, 16) || !aligned(c->V, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
        return fail(STARQ_ERR_ALIGN, "%s: cache codes must be 16-byte aligned, scales 4", who);
    return STARQ_OK;
}

int check_sequences(const char* who, int T, int B, int max_new, int table_ld) {
    if (T < 0 || T > MAX_ROWS || B < 0 || B > 65535 || max_new < 0 || max_new > MAX_ROWS || table_ld < 0)
        return fail(STARQ_ERR_SHAPE, "%s: T=%d, B=%d, max_new=%d, table_ld=%d: need 0 <= T, max_new <= 2^28, "
                    "0 <= B <= 65535, table_ld >= 0", who, T, B, max_new, table_ld);
    return STARQ_OK;
}

int check_rows(const char* who, const char* name, const void* p, int ld, int width, int elem) {
    if (!p) return fail(STARQ_ERR_ARG, "%s: NULL %s", who, name);
    if (ld < width) return fail(STARQ_ERR_SHAPE, "%s: row stride %d of %s is less than its %d channels", who, ld, name, width);
    if (!aligned(p, 16) || ((size_t)ld * elem) % 16 != 0)
        return fail(STARQ_ERR_ALIGN, "%s: %s and its rows must be 16-byte aligned", who, name);
    return STARQ_OK;
}

}  // namespace
}  // namespace starq

using namespace starq;

extern "C" {

int glue_rope_table(float* table, int positions, int rot, double theta, int scaling, double factor, double original,
                    double beta_fast, double beta_slow, double mscale, void* stream) {
    if (scaling < STARQ_ROPE_NONE || scaling > STARQ_ROPE_PARTS)
        return fail(STARQ_ERR_ARG, "glue_rope_table: unknown scaling %d", scaling);
    if (positions < 0 || positions > MAX_ROWS || rot < 2 || rot > 1024 || rot % 2 != 0)
        return fail(STARQ_ERR_SHAPE, "glue_rope_table: positions=%d, rot=%d: need 0 <= positions <= 2^28, "
                    "an even rot in [2, 1024]", positions, rot);
    if (!(theta > 1.0) || !(theta < 1e300)) return fail(STARQ_ERR_ARG, "glue_rope_table: theta must be > 1");
    if (scaling != STARQ_ROPE_NONE && (!(factor >= 1.0) || !(factor < 1e9)))
        return fail(STARQ_ERR_ARG, "glue_rope_table: factor must be >= 1");
    if (scaling == STARQ_ROPE_PARTS && (!(original > 0.0) || !(beta_slow > 0.0) || !(beta_fast > beta_slow)))
        return fail(STARQ_ERR_ARG, "glue_rope_table: need original > 0 and beta_fast > beta_slow > 0");
    if (!(mscale >= 0.0) || !(mscale < 1e9)) return fail(STARQ_ERR_ARG, "glue_rope_table: mscale must be >= 0");
    if (positions == 0) return STARQ_OK;
    if (!table) return fail(STARQ_ERR_ARG, "glue_rope_table: NULL table");
    if (!aligned(table, 16)) return fail(STARQ_ERR_ALIGN, "glue_rope_table: table must be 16-byte aligned");
    if (mscale == 0.0) mscale = scaling == STARQ_ROPE_PARTS ? rope_parts_mscale(factor) : 1.0;
    return launched(launch_rope_table(reinterpret_cast<float2*>(table), positions, rot, theta, scaling, factor,
                                      original, beta_fast, beta_slow, mscale, static_cast<cudaStream_t>(stream)),
                    "glue_rope_table");
}

int glue_rope_apply(const void* X, int ldx, int dtype, int L, int heads, int D, int rot, int interleaved, int inverse,
                    const int32_t* pos, const float* table, int positions, void* Y, int ldy, void* stream) {
    if (!any_type(dtype)) return fail(STARQ_ERR_ARG, "glue_rope_apply: unknown dtype %d", dtype);
    if (L < 0 || L > MAX_ROWS || heads < 1 || heads > 65535 || D < 1 || D > 4096)
        return fail(STARQ_ERR_SHAPE, "glue_rope_apply: L=%d, heads=%d, D=%d: need 0 <= L <= 2^28, "
                    "1 <= heads <= 65535, 1 <= D <= 4096", L, heads, D);
    if (rot < 0 || rot > D || rot % 2 != 0)
        return fail(STARQ_ERR_SHAPE, "glue_rope_apply: rot=%d: need an even number of the head's %d channels", rot, D);
    if ((long long)ldx < (long long)heads * D || (long long)ldy < (long long)heads * D)
        return fail(STARQ_ERR_SHAPE, "glue_rope_apply: ldx=%d, ldy=%d: need at least heads * D = %lld", ldx, ldy,
                    (long long)heads * D);
    if (positions < 0) return fail(STARQ_ERR_SHAPE, "glue_rope_apply: positions=%d < 0", positions);
    if (X == Y && ldx != ldy) return fail(STARQ_ERR_ARG, "glue_rope_apply: in place needs ldy = ldx");
    if (L == 0) return STARQ_OK;
    if (!X || !Y || (rot > 0 && (!pos || !table)))
        return fail(STARQ_ERR_ARG, "glue_rope_apply: NULL X, Y, pos or table");
    const size_t e = dtype == STARQ_F32 ? 4 : 2;
    if (!aligned(X, e) || !aligned(Y, e) || !aligned(pos, 4) || !aligned(table, 8))
        return fail(STARQ_ERR_ALIGN, "glue_rope_apply: X, Y, pos and table (8 B) must be aligned to their elements");
    int rc = STARQ_OK;
    RopeArgs a{X, Y, dtype, L, ldx, ldy, heads, D, rot, interleaved != 0, inverse != 0, pos,
               reinterpret_cast<const float2*>(table), positions, device_status(&rc)};
    if (!a.status) return rc;
    return launched(launch_rope_apply(a, static_cast<cudaStream_t>(stream)), "glue_rope_apply");
}

int kv_cache_append(const starq_kv_cache* cache, const void* K, int ldk, const void* V, int ldv, const void* Q,
                    int ldq, void* Qo, int ldqo, int H, int dtype, int T, const int32_t* seq_start,
                    const int32_t* past, int B, int max_new, const int32_t* page_table, int table_ld,
                    const int32_t* pos, const float* table, int positions, int rot, int interleaved, void* stream) {
    const char* who = "kv_cache_append";
    int rc = check_cache(who, cache);
    if (rc) return rc;
    if (!half_type(dtype)) return fail(STARQ_ERR_ARG, "%s: dtype must be F16 or BF16", who);
    if ((rc = check_sequences(who, T, B, max_new, table_ld))) return rc;
    if (rot < 0 || rot > cache->D || rot % 16 != 0)
        return fail(STARQ_ERR_SHAPE, "%s: rot=%d: need a multiple of 16, at most the head size %d", who, rot, cache->D);
    if (positions < 0) return fail(STARQ_ERR_SHAPE, "%s: positions=%d < 0", who, positions);
    if ((Q != nullptr) != (Qo != nullptr)) return fail(STARQ_ERR_ARG, "%s: Q and Qo go together", who);
    if (Q && (H < 1 || H > 65535)) return fail(STARQ_ERR_SHAPE, "%s: H=%d: need 1 <= H <= 65535", who, H);
    if (Q && Q == Qo && ldq != ldqo) return fail(STARQ_ERR_ARG, "%s: in place needs ldqo = ldq", who);
    if (T == 0 || B == 0 || max_new == 0) return STARQ_OK;
    if ((rc = check_cache_pointers(who, cache))) return rc;
    const int w = cache->Hkv * cache->D;
    if ((rc = check_rows(who, "K", K, ldk, w, 2)) || (rc = check_rows(who, "V", V, ldv, w, 2))) return rc;
    if (Q && ((rc = check_rows(who, "Q", Q, ldq, H * cache->D, 2)) ||
              (rc = check_rows(who, "Qo", Qo, ldqo, H * cache->D, 2))))
        return rc;
    if (!seq_start || !past || (!page_table && table_ld > 0) || (rot > 0 && (!pos || !table)))
        return fail(STARQ_ERR_ARG, "%s: NULL seq_start, past, page_table, pos or table", who);
    if (!aligned(seq_start, 4) || !aligned(past, 4) || !aligned(page_table, 4) || !aligned(pos, 4) ||
        !aligned(table, 16))
        return fail(STARQ_ERR_ALIGN, "%s: index arrays must be 4-byte aligned, table 16", who);
    KvAppendArgs a{*cache, K, ldk, V, ldv, Q, ldq, Qo, ldqo, Q ? H : 1, dtype, T, seq_start, past, B, max_new,
                   page_table, table_ld, pos, reinterpret_cast<const float2*>(table), positions, rot,
                   interleaved != 0, device_status(&rc)};
    if (!a.status) return rc;
    const cudaError_t e = launch_kv_append(a, static_cast<cudaStream_t>(stream));
    if (e == cudaErrorInvalidValue)
        return fail(STARQ_ERR_SHAPE, "%s: B=%d sequences of up to %d rows need more than 2^31 CTAs", who, B, max_new);
    return launched(e, who);
}

int kv_cache_read(const starq_kv_cache* cache, const int32_t* page_table, int table_ld, const int32_t* first,
                  const int32_t* out_start, int B, int max_rows, int T, void* K, void* V, int ld, int dtype,
                  void* stream) {
    const char* who = "kv_cache_read";
    int rc = check_cache(who, cache);
    if (rc) return rc;
    if (!any_type(dtype)) return fail(STARQ_ERR_ARG, "%s: unknown dtype %d", who, dtype);
    if ((rc = check_sequences(who, T, B, max_rows, table_ld))) return rc;
    if (T == 0 || B == 0 || max_rows == 0 || (!K && !V)) return STARQ_OK;
    if ((rc = check_cache_pointers(who, cache))) return rc;
    const int w = cache->Hkv * cache->D, e = dtype == STARQ_F32 ? 4 : 2;
    if (K && (rc = check_rows(who, "K", K, ld, w, e))) return rc;
    if (V && (rc = check_rows(who, "V", V, ld, w, e))) return rc;
    if ((!page_table && table_ld > 0) || !first || !out_start) return fail(STARQ_ERR_ARG, "%s: NULL page_table, first or out_start", who);
    if (!aligned(page_table, 4) || !aligned(first, 4) || !aligned(out_start, 4))
        return fail(STARQ_ERR_ALIGN, "%s: index arrays must be 4-byte aligned", who);
    KvReadArgs a{*cache, page_table, table_ld, first, out_start, B, max_rows, T, K, V, ld, dtype, device_status(&rc)};
    if (!a.status) return rc;
    return launched(launch_kv_read(a, static_cast<cudaStream_t>(stream)), who);
}

size_t kv_cache_attention_workspace_size(int B, int max_new, int H, int Hkv, int D) {
    if (B < 0 || B > 65535 || max_new < 0 || max_new > MAX_ROWS || H < 1 || Hkv < 1 || H % Hkv != 0 ||
        (D != 64 && D != 128))
        return 0;
    return kv_attention_workspace_bytes(B, max_new, H, Hkv, D);
}

int kv_cache_attention(const void* Q, int ldq, int dtype, int T, const int32_t* seq_start, int B, int max_new, int H,
                       const starq_kv_cache* cache, const int32_t* page_table, int table_ld, const int32_t* kv_len,
                       int max_len, int causal, const uint8_t* key_mask, int mask_ld, float scale, void* Out, int ldo,
                       float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "kv_cache_attention";
    int rc = check_cache(who, cache);
    if (rc) return rc;
    if (!half_type(dtype)) return fail(STARQ_ERR_ARG, "%s: dtype must be F16 or BF16", who);
    if ((rc = check_sequences(who, T, B, max_new, table_ld))) return rc;
    if (H < 1 || H > 65535 || H % cache->Hkv != 0)
        return fail(STARQ_ERR_SHAPE, "%s: H=%d: need a multiple of Hkv=%d, at most 65535", who, H, cache->Hkv);
    if ((long long)max_new * H > MAX_ROWS)
        return fail(STARQ_ERR_SHAPE, "%s: max_new * H = %lld: at most 2^28", who, (long long)max_new * H);
    if (max_len < 0 || max_len > MAX_ROWS) return fail(STARQ_ERR_SHAPE, "%s: max_len=%d: need 0 .. 2^28", who, max_len);
    if (key_mask && mask_ld < max_len)
        return fail(STARQ_ERR_SHAPE, "%s: mask_ld=%d is less than max_len=%d", who, mask_ld, max_len);
    if (!(scale > 0.f) || !(scale < 1e30f)) return fail(STARQ_ERR_ARG, "%s: scale must be positive and finite", who);
    if (T == 0 || B == 0 || max_new == 0) return STARQ_OK;
    if ((rc = check_cache_pointers(who, cache))) return rc;
    const int w = H * cache->D;
    if ((rc = check_rows(who, "Q", Q, ldq, w, 2)) || (rc = check_rows(who, "Out", Out, ldo, w, 2))) return rc;
    if (!seq_start || !kv_len || (!page_table && table_ld > 0) || !workspace)
        return fail(STARQ_ERR_ARG, "%s: NULL seq_start, kv_len, page_table or workspace", who);
    if (!aligned(seq_start, 4) || !aligned(kv_len, 4) || !aligned(page_table, 4) || !aligned(lse, 4) ||
        !aligned(workspace, 256))
        return fail(STARQ_ERR_ALIGN, "%s: index arrays and lse must be 4-byte aligned, workspace 256", who);
    const size_t need = kv_attention_workspace_bytes(B, max_new, H, cache->Hkv, cache->D);
    if (workspace_bytes < need)
        return fail(STARQ_ERR_ARG, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
    KvAttnArgs a{*cache, Q, ldq, dtype, T, seq_start, B, max_new, H, page_table, table_ld, kv_len, max_len,
                 causal != 0, key_mask, mask_ld, scale, Out, ldo, lse, workspace, device_status(&rc)};
    if (!a.status) return rc;
    return launched(launch_kv_attention(a, static_cast<cudaStream_t>(stream)), who);
}

int w4g_linear(const void* X, int ldx, int dtype, int L, int K, const uint8_t* Wq, const float* scales, int group,
               int N, const float* bias, void* Y, int ldy, int y_dtype, void* stream) {
    const char* who = "w4g_linear";
    if (!half_type(dtype)) return fail(STARQ_ERR_ARG, "%s: dtype must be F16 or BF16", who);
    if (!any_type(y_dtype)) return fail(STARQ_ERR_ARG, "%s: unknown output dtype %d", who, y_dtype);
    if (L < 0 || L > 32) return fail(STARQ_ERR_SHAPE, "%s: L=%d: need 0 <= L <= 32", who, L);
    if (group != 32 && group != 64 && group != 128)
        return fail(STARQ_ERR_SHAPE, "%s: group=%d: 32, 64 or 128", who, group);
    if (K < group || K % group != 0 || K > (1 << 24))
        return fail(STARQ_ERR_SHAPE, "%s: K=%d: need a multiple of group=%d, at most 2^24", who, K, group);
    if (N < 1 || N > (1 << 28)) return fail(STARQ_ERR_SHAPE, "%s: N=%d: need 1 <= N <= 2^28", who, N);
    if (ldx < K || ldy < N) return fail(STARQ_ERR_SHAPE, "%s: ldx=%d, ldy=%d: need ldx >= K=%d, ldy >= N=%d", who, ldx, ldy, K, N);
    if (L == 0) return STARQ_OK;
    if (!X || !Wq || !scales || !Y) return fail(STARQ_ERR_ARG, "%s: NULL X, Wq, scales or Y", who);
    if (!aligned(X, 16) || ((size_t)ldx * 2) % 16 != 0 || !aligned(Wq, 16) || !aligned(scales, 4) ||
        !aligned(bias, 4) || !aligned(Y, y_dtype == STARQ_F32 ? 4 : 2))
        return fail(STARQ_ERR_ALIGN, "%s: X, its rows and Wq must be 16-byte aligned, the others to their elements", who);
    const W4gArgs a{X, ldx, dtype, L, K, Wq, scales, group, N, bias, Y, ldy, y_dtype};
    return launched(launch_w4g_linear(a, static_cast<cudaStream_t>(stream)), who);
}

}  // extern "C"
