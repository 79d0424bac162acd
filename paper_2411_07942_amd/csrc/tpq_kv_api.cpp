// Host side of the C ABI's part on the 4-bit cache of keys and values: layout, argument validation, dispatch.
// Every check here runs before anything is enqueued.
#include <math.h>
#include <string.h>

#include <memory>
#include <new>

#include "tpq_kv.h"

namespace tpq {

static int log2_of(int v)
{
    int lg = 0;
    while ((1 << lg) < v) ++lg;
    return lg;
}

static bool one_of(int v, int lo, int hi)  // a power of two in lo .. hi
{
    return v >= lo && v <= hi && (v & (v - 1)) == 0;
}

int kv_check_layout(const tpq_kv_layout *L)
{
    if (!L) return TPQ_ERR_NULL;
    if (!one_of(L->D, 64, 256) || !one_of(L->G, 32, L->D) || !one_of(L->page, 16, 256)) return TPQ_ERR_UNSUPPORTED;
    if (L->heads < 1 || L->heads > TPQ_KV_MAX_HEADS) return TPQ_ERR_SHAPE;
    if (L->ng != L->D / L->G || L->cell_bytes != static_cast<int64_t>(L->page) * (L->D + 8 * L->ng) ||
        L->page_bytes != L->heads * L->cell_bytes)
        return TPQ_ERR_SHAPE;
    return TPQ_OK;
}

int kv_check_batch(const tpq_kv_layout *L, const tpq_kv_batch *b)
{
    const int rc = kv_check_layout(L);
    if (rc) return rc;
    if (!b || !b->table || !b->lens) return TPQ_ERR_NULL;
    if (b->n_seqs < 1 || b->n_seqs > 65535 || b->ld_table < 1 || static_cast<int64_t>(b->ld_table) * L->page > 1 << 28 ||
        b->max_new < 1 || b->max_new > 1 << 20 || b->max_len < 1 || b->max_len > static_cast<int64_t>(b->ld_table) * L->page ||
        b->rows < 0 || b->rows > 0x7FFFFFFF || b->n_pages < 1 || b->n_pages > 0x7FFFFFFF)
        return TPQ_ERR_SHAPE;
    if (!b->starts && (b->max_new != 1 || b->rows < b->n_seqs)) return TPQ_ERR_SHAPE;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(b->table) | reinterpret_cast<uintptr_t>(b->lens) | reinterpret_cast<uintptr_t>(b->starts);
    return (bits & 3u) ? TPQ_ERR_ALIGN : TPQ_OK;
}

KvArgs kv_args(const tpq_kv_layout *L, const void *cache, const tpq_kv_batch *b)
{
    KvArgs a;
    memset(&a, 0, sizeof a);
    a.cache = static_cast<uint8_t *>(const_cast<void *>(cache));
    a.table = b->table; a.lens = b->lens; a.starts = b->starts;
    a.rows = b->rows; a.n_pages = b->n_pages; a.page_bytes = L->page_bytes;
    a.n_seqs = b->n_seqs; a.ld_table = b->ld_table; a.max_new = b->max_new;
    a.heads = L->heads; a.lg_page = log2_of(L->page); a.ng = L->ng; a.lg_group = log2_of(L->G);
    a.cell_bytes = static_cast<uint32_t>(L->cell_bytes);
    return a;
}

}  // namespace tpq

using namespace tpq;

static bool bad_query_heads(const tpq_kv_layout *L, int q_heads)
{
    return q_heads < L->heads || q_heads > 4 * TPQ_KV_MAX_HEADS || q_heads % L->heads != 0;
}

extern "C" {

int tpq_kv_layout_init(tpq_kv_layout *L, int heads, int D, int G, int page)
{
    if (!L) return TPQ_ERR_NULL;
    if (!one_of(D, 64, 256) || !one_of(G, 32, D) || !one_of(page, 16, 256)) return TPQ_ERR_UNSUPPORTED;
    if (heads < 1 || heads > TPQ_KV_MAX_HEADS) return TPQ_ERR_SHAPE;
    memset(L, 0, sizeof *L);
    L->heads = heads;
    L->D = D;
    L->G = G;
    L->page = page;
    L->ng = D / G;
    L->cell_bytes = static_cast<int64_t>(page) * (D + 8 * L->ng);
    L->page_bytes = heads * L->cell_bytes;
    return TPQ_OK;
}

int tpq_kv_check(const tpq_kv_layout *L, const tpq_kv_batch *batch, void *stream)
{
    int rc = kv_check_batch(L, batch);
    if (rc) return rc;
    const size_t B = static_cast<size_t>(batch->n_seqs), W = static_cast<size_t>(batch->ld_table);
    const std::unique_ptr<int32_t[]> host(new (std::nothrow) int32_t[B * W + B + B + 1]);
    if (!host) return TPQ_ERR_WORKSPACE;
    int32_t *const table = host.get(), *const lens = table + B * W, *const starts = lens + B;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    rc = hip_result(hipMemcpyAsync(table, batch->table, B * W * sizeof(int32_t), hipMemcpyDeviceToHost, s));
    if (!rc) rc = hip_result(hipMemcpyAsync(lens, batch->lens, B * sizeof(int32_t), hipMemcpyDeviceToHost, s));
    if (!rc && batch->starts) rc = hip_result(hipMemcpyAsync(starts, batch->starts, (B + 1) * sizeof(int32_t), hipMemcpyDeviceToHost, s));
    const int waited = hip_result(hipStreamSynchronize(s));  // (also behind an error: the copies' target goes away)
    if (rc || waited) return rc ? rc : waited;
    for (size_t b = 0; b < B; ++b) {
        int64_t n = 1;
        if (batch->starts) {
            n = static_cast<int64_t>(starts[b + 1]) - starts[b];
            if (starts[b] < 0 || n < 0 || starts[b + 1] > batch->rows || n > batch->max_new) return TPQ_ERR_INDEX;
        }
        if (lens[b] < n || lens[b] > static_cast<int64_t>(batch->ld_table) * L->page) return TPQ_ERR_INDEX;
        for (int64_t e = 0; e * L->page < lens[b]; ++e)
            if (table[b * W + e] < 0 || table[b * W + e] >= batch->n_pages) return TPQ_ERR_INDEX;
    }
    return TPQ_OK;
}

int tpq_kv_append(const tpq_kv_layout *L, void *cache, const tpq_kv_batch *batch, const uint16_t *K, int64_t ldK,
                  const uint16_t *V, int64_t ldV, const float *rot_cos, const float *rot_sin, int rot, int rot_rows,
                  int rot_mode, const uint16_t *Q, int64_t ldQ, int q_heads, uint16_t *Q_out, int64_t ldQo, void *stream)
{
    const int rc = kv_check_batch(L, batch);
    if (rc) return rc;
    if (rot_mode != TPQ_ROT_HALVES && rot_mode != TPQ_ROT_PAIRS) return TPQ_ERR_UNSUPPORTED;
    const int64_t E = static_cast<int64_t>(L->heads) * L->D, Eq = static_cast<int64_t>(q_heads) * L->D;
    if (rot < 0 || rot > L->D || (rot % 16) != 0 || (rot > 0 && rot_rows < 1)) return TPQ_ERR_SHAPE;
    if (ldK < E || ldV < E) return TPQ_ERR_SHAPE;
    if (Q && (bad_query_heads(L, q_heads) || ldQ < Eq || ldQo < Eq)) return TPQ_ERR_SHAPE;
    if ((ldK % 8) != 0 || (ldV % 8) != 0 || (Q && ((ldQ % 8) != 0 || (ldQo % 8) != 0))) return TPQ_ERR_ALIGN;
    if (batch->rows == 0) return TPQ_OK;
    if (!cache || !K || !V || (rot > 0 && (!rot_cos || !rot_sin)) || (Q && !Q_out)) return TPQ_ERR_NULL;
    if (!aligned16(cache) || !aligned16(K) || !aligned16(V) || (rot > 0 && (!aligned16(rot_cos) || !aligned16(rot_sin))) ||
        (Q && (!aligned16(Q) || !aligned16(Q_out))))
        return TPQ_ERR_ALIGN;
    KvAppendArgs p;
    memset(&p, 0, sizeof p);
    p.K = reinterpret_cast<const uint8_t *>(K); p.V = reinterpret_cast<const uint8_t *>(V);
    p.ldK = 2 * ldK; p.ldV = 2 * ldV;
    if (Q) {
        p.Q = reinterpret_cast<const uint8_t *>(Q); p.Q_out = reinterpret_cast<uint8_t *>(Q_out);
        p.ldQ = 2 * ldQ; p.ldQo = 2 * ldQo;
    }
    p.cosines = rot_cos; p.sines = rot_sin;
    p.rot = rot; p.rot_rows = rot_rows; p.pairs = rot_mode == TPQ_ROT_PAIRS;
    p.units = 2 * L->heads + (Q ? q_heads : 0);
    return launch_kv_append(kv_args(L, cache, batch), p, L->D, static_cast<hipStream_t>(stream));
}

int tpq_kv_read(const tpq_kv_layout *L, const void *cache, const tpq_kv_batch *batch, int out_dtype, void *K_out,
                int64_t ldK, void *V_out, int64_t ldV, void *stream)
{
    const int rc = kv_check_batch(L, batch);
    if (rc) return rc;
    if (out_dtype != TPQ_OUT_BF16 && out_dtype != TPQ_OUT_FP32) return TPQ_ERR_UNSUPPORTED;
    const int64_t E = static_cast<int64_t>(L->heads) * L->D, step = out_dtype == TPQ_OUT_FP32 ? 4 : 8;
    if ((K_out && ldK < E) || (V_out && ldV < E)) return TPQ_ERR_SHAPE;
    if ((K_out && ldK % step) || (V_out && ldV % step)) return TPQ_ERR_ALIGN;
    if (batch->rows == 0 || (!K_out && !V_out)) return TPQ_OK;
    if (!cache) return TPQ_ERR_NULL;
    if (!aligned16(cache) || !aligned16(K_out) || !aligned16(V_out)) return TPQ_ERR_ALIGN;
    KvReadArgs p;
    memset(&p, 0, sizeof p);
    const int bytes = out_dtype == TPQ_OUT_FP32 ? 4 : 2;
    p.K = static_cast<uint8_t *>(K_out); p.V = static_cast<uint8_t *>(V_out);
    p.ldK = bytes * ldK; p.ldV = bytes * ldV;
    p.fp32 = out_dtype == TPQ_OUT_FP32;
    p.first = K_out ? 0 : L->heads;
    p.units = (K_out ? L->heads : 0) + (V_out ? L->heads : 0);
    return launch_kv_read(kv_args(L, cache, batch), p, L->D, static_cast<hipStream_t>(stream));
}

size_t tpq_kv_attention_workspace_bytes(const tpq_kv_layout *L, const tpq_kv_batch *batch, int q_heads)
{
    if (kv_check_batch(L, batch) != TPQ_OK || bad_query_heads(L, q_heads)) return 0;
    return kv_attend_workspace_bytes(kv_args(L, nullptr, batch), L->D, q_heads / L->heads, batch->max_len);
}

int tpq_kv_attention(const tpq_kv_layout *L, const void *cache, const tpq_kv_batch *batch, const uint16_t *Q, int64_t ldQ,
                     int q_heads, float scale, int window, int sinks, float softcap, uint16_t *out, int64_t ldOut,
                     void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = kv_check_batch(L, batch);
    if (rc) return rc;
    if (bad_query_heads(L, q_heads)) return TPQ_ERR_SHAPE;
    const int64_t Eq = static_cast<int64_t>(q_heads) * L->D;
    if (ldQ < Eq || ldOut < Eq || window < 0 || window > 1 << 28 || sinks < 0 || sinks > 1 << 28) return TPQ_ERR_SHAPE;
    if (!isfinite(scale) || !isfinite(softcap)) return TPQ_ERR_SHAPE;
    // (a bounded score is off by 2^-22 of the bound, whatever its size; 1 / softcap times a score stays finite)
    if (softcap != 0.0f && !(softcap >= 0x1p-20f && softcap <= TPQ_KV_MAX_SOFTCAP)) return TPQ_ERR_SHAPE;
    if ((ldQ % 8) != 0 || (ldOut % 8) != 0) return TPQ_ERR_ALIGN;
    if (batch->rows == 0) return TPQ_OK;
    if (!cache || !Q || !out || !workspace) return TPQ_ERR_NULL;
    if (!aligned16(cache) || !aligned16(Q) || !aligned16(out) || !aligned16(workspace)) return TPQ_ERR_ALIGN;
    const size_t need = tpq_kv_attention_workspace_bytes(L, batch, q_heads);
    if (need == 0) return TPQ_ERR_HIP;
    if (ws_bytes < need) return TPQ_ERR_WORKSPACE;
    KvAttendArgs p;
    memset(&p, 0, sizeof p);
    p.Q = reinterpret_cast<const uint8_t *>(Q);
    p.out = reinterpret_cast<uint8_t *>(out);
    p.ldQ = 2 * ldQ; p.ldOut = 2 * ldOut;
    p.R = q_heads / L->heads;
    p.window = window; p.sinks = sinks;
    p.scale = scale; p.softcap = softcap;
    return launch_kv_attend(kv_args(L, cache, batch), p, L->D, batch->max_len, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
