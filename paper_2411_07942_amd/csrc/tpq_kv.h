// Declarations shared by the kernels of the 4-bit cache of keys and values (host + device).
#pragma once

#include "tpq_internal.h"

namespace tpq {

// The cache and the batch, as every kernel takes them.
struct KvArgs {
    uint8_t *cache;
    const int32_t *table, *lens, *starts;
    int64_t rows, n_pages, page_bytes;
    int32_t n_seqs, ld_table, max_new;
    int32_t heads, lg_page, ng, lg_group;  // lg_page, lg_group: logarithms of page and G
    uint32_t cell_bytes;
};

// Division by a number that the host knows: two multiplications' worth of scalar instructions instead of the 40 of an
// integer division (eight of them took 0.4 us in front of a kernel's first load).
struct KvDivisor {
    uint32_t d, mul, shift;  // n / d = (t + ((n - t) >> 1)) >> shift with t = mulhi(n, mul), for d > 1
    KvDivisor() = default;
    explicit KvDivisor(uint32_t by) : d(by), mul(0), shift(0)
    {
        if (by < 2) return;
        uint32_t lg = 0;
        while ((1ull << lg) < by) ++lg;
        mul = static_cast<uint32_t>(((((1ull << lg) - by) << 32) / by) + 1);
        shift = lg - 1;
    }
    __host__ __device__ __forceinline__ int of(int n) const  // n >= 0
    {
        if (d == 1) return n;
        const uint32_t u = static_cast<uint32_t>(n), t = static_cast<uint32_t>((static_cast<uint64_t>(u) * mul) >> 32);
        return static_cast<int>((t + ((u - t) >> 1)) >> shift);
    }
};

struct KvAppendArgs {
    const uint8_t *K, *V, *Q;
    uint8_t *Q_out;
    int64_t ldK, ldV, ldQ, ldQo;  // bytes
    const float *cosines, *sines;
    int32_t rot, rot_rows, pairs;
    int32_t units;    // head rows of a token: 2 heads + q_heads
    int32_t columns;  // workgroups side by side that they take
    KvDivisor by_columns;
};

struct KvReadArgs {
    uint8_t *K, *V;
    int64_t ldK, ldV;  // bytes
    int32_t fp32;
    int32_t first, units;  // head rows of a token: [first, first + units) of the keys' and the values' heads
    int32_t columns;
    KvDivisor by_columns;
};

// (In this order: with window and scale in front of the numbers that a workgroup finds its item by, a call took 0.2 us longer: one token of 5 heads over 641 9.3, so 9.15.)
struct KvAttendArgs {
    const uint8_t *Q;
    uint8_t *out;
    int64_t ldQ, ldOut;  // bytes
    int32_t *plan;       // the list of items, of more than 64 sequences
    float *part;         // partial results: accumulators, then their maxima and sums
    float *part_ml;
    int32_t R;                          // query heads per key/value head
    KvDivisor by_R, by_rows, by_heads;  // (rows: of a tile)
    int32_t splits;      // 1: no tile of rows is cut; with one sequence: shares of a tile's steps
    int32_t odd;         // 1: shares of an odd number of steps
    int32_t items, row_tiles, min_tiles;  // items of a head, most tiles of rows of a sequence, least steps of a share
    int32_t window, sinks;
    float scale, softcap;
};

// A sequence's new rows and its length; false: its starts are no range of rows.
__host__ __device__ __forceinline__ bool kv_sequence(const KvArgs &a, int b, int64_t &row0, int &n, int &len)
{
    len = min(max(a.lens[b], 0), 1 << 30);
    row0 = b;
    n = 1;
    if (!a.starts) return true;
    const int s0 = a.starts[b], s1 = a.starts[b + 1];
    row0 = s0;
    n = s1 - s0;
    return s0 >= 0 && s1 >= s0 && s1 <= a.rows;
}

// The cell of a position's token in head 0, and its slot there; null: absent.
__device__ __forceinline__ uint8_t *kv_cell(const KvArgs &a, int b, int pos, int &slot)
{
    slot = pos & ((1 << a.lg_page) - 1);
    if (pos < 0 || pos >> a.lg_page >= a.ld_table) return nullptr;
    const int id = a.table[static_cast<int64_t>(b) * a.ld_table + (pos >> a.lg_page)];
    if (static_cast<uint32_t>(id) >= static_cast<uint64_t>(a.n_pages)) return nullptr;
    return a.cache + id * a.page_bytes;
}

// ---- host side ------------------------------------------------------------------------------
int kv_check_layout(const tpq_kv_layout *L);
int kv_check_batch(const tpq_kv_layout *L, const tpq_kv_batch *batch);
KvArgs kv_args(const tpq_kv_layout *L, const void *cache, const tpq_kv_batch *batch);
int launch_kv_append(const KvArgs &a, const KvAppendArgs &p, int D, hipStream_t s);
int launch_kv_read(const KvArgs &a, const KvReadArgs &p, int D, hipStream_t s);
size_t kv_attend_workspace_bytes(const KvArgs &a, int D, int R, int max_len);
int launch_kv_attend(const KvArgs &a, KvAttendArgs p, int D, int max_len, void *workspace, hipStream_t s);

}  // namespace tpq
