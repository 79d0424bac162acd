// The work list of the attention over the 4-bit cache (host + device): the steps that a tile of rows goes through, the shares they
// are cut into, and what the host chooses for a batch.
#pragma once

#include <algorithm>

#include "tpq_kv.h"

namespace tpq {

constexpr int kKvTile = 32;            // tokens of a step of a wave (few rows)
constexpr int64_t kKvMaxItems = (1ll << 32) / 512 - 1;  // (a launch has fewer than 2^32 threads)

// The steps that rows at positions lo .. hi go through: the tiles that hold visible first tokens, then those from the first
// row's window to the last row's position.
struct KvSpan {
    int first, start, tiles;  // tiles of first tokens, first tile of the rest, all tiles
    __host__ __device__ __forceinline__ int tile(int v) const { return v < first ? v : start + (v - first); }
};
template <int TOK>
__host__ __device__ __forceinline__ KvSpan kv_span(const KvArgs &a, const KvAttendArgs &p, int lo, int hi, int len)
{
    const int end = min(min(hi + 1, len), a.ld_table << a.lg_page);
    KvSpan s = {0, 0, 0};
    if (end <= 0) return s;
    const int last = (end + TOK - 1) / TOK;
    if (p.window > 0) {
        s.start = max(lo - p.window + 1, 0) / TOK;
        s.first = min((min(p.sinks, end) + TOK - 1) / TOK, s.start);
    }
    s.tiles = s.first + max(last - s.start, 0);
    return s;
}

// A sequence's rows of a key/value head in tiles of `rows` (row i R + r: query head r of new token i).
struct KvSeq {
    int row0, n, base, len;  // first row of the tensors, new tokens (at most max_new), position of the first, tokens
    int row_tiles, most;     // tiles of rows (0: none), steps of the last of them (with a window no bound of the others')
};
template <int TOK>
__host__ __device__ __forceinline__ KvSeq kv_seq(const KvArgs &a, const KvAttendArgs &p, int rows, int b)
{
    KvSeq q = {0, 0, 0, 0, 0, 0};
    int64_t row0;
    if (b >= a.n_seqs || !kv_sequence(a, b, row0, q.n, q.len)) return q;
    q.row0 = static_cast<int>(row0);
    q.base = q.len - q.n;
    q.n = min(q.n, a.max_new);
    if (q.n == 0) return q;
    const int last = p.by_rows.of(q.n * p.R - 1);
    q.row_tiles = last + 1;
    q.most = kv_span<TOK>(a, p, q.base + p.by_R.of(last * rows), q.base + q.n - 1, q.len).tiles;
    return q;
}

// As many items for each tile: nothing to look up.
__host__ __device__ __forceinline__ bool kv_even(const KvArgs &a, const KvAttendArgs &p) { return a.n_seqs == 1 || (p.splits == 1 && p.row_tiles == 1); }
// Items of a sequence whose tiles are cut into shares of `step` steps.
__host__ __device__ __forceinline__ uint32_t kv_items(const KvSeq &q, uint32_t step) { return q.row_tiles * max((q.most + step - 1) / step, 1u); }
__host__ __device__ __forceinline__ uint64_t kv_work(const KvSeq &q) { return static_cast<uint64_t>(q.most) * q.row_tiles; }

// The least steps of a share with which all sequences' items fit p.items, to a sixteenth.  work, tiles: the thread's sequences'
// steps and tiles, `threads` + 1 threads; total(n): the sum over all of them; items_of(step): the thread's.
template <typename Total, typename Items>
__host__ __device__ __forceinline__ uint32_t kv_step(const KvAttendArgs &p, uint64_t work, uint32_t tiles, uint32_t threads, Total &&total, Items &&items_of)
{
    const uint32_t uncut = 1u << 30;
    if (p.splits == 1) return uncut;
    const uint32_t most = 0x7FFFFFFFu / (threads + 1);
    if (total(work > most ? 1u : 0u) != 0) return uncut;  // (more steps than can be counted)
    const uint32_t all = total(static_cast<uint32_t>(work)), items = p.items;
    tiles = total(tiles);
    // nearly all / items, at most all / (items - tiles)
    const uint32_t least = p.min_tiles;
    uint32_t low = max((all + items - 1) / items, least), good = max(all / (items > tiles ? items - tiles : 1u) + 1, low);
    if (total(items_of(low)) <= items) good = low;
    while (good - low > low >> 4) {
        const uint32_t mid = low + ((good - low) >> 1);
        if (mid == low) break;
        if (total(items_of(mid)) <= items) good = mid;
        else low = mid;
    }
    return good;
}

// A workgroup's item: a tile of a sequence's rows and a share of the steps that they go through.  A head's items lie in one
// list, sequence by sequence and tile by tile, so that no workgroup is without work: one that finds none still costs 11 ns of
// the launch.  With several sequences the list's length is given and the largest share sought that fits it: long sequences are
// cut into more shares than short ones (16 drafts of 5 over 300 to 9000 tokens, 8 heads: 64 us with as many shares for each, 41 with this).
// Every tile of a sequence owns `cuts` items, as many as its last one needs, and has shares of that one's size; but with a window
// an earlier tile may go through more steps than the last (it has more rows, or lies across one more tile of tokens), and then its
// shares are as long as its own steps ask for, so that there are never more of them than items.
struct KvShare {
    int b, rt, split;
    int64_t row0, item0;    // the tensors' row of the sequence's first, the tile's first item
    int n_rows, base, len;  // rows of the sequence and head, position of row 0, tokens
    int lo, hi;             // first and last position among the tile's rows
    KvSpan span;
    int live, share;        // shares that have steps (1 .. the tile's items), steps of a share
};
// Of tile s.rt of a sequence whose tiles have `cuts` items each, from item `first` on (the last tile's: its rows have the most keys).
template <int TOK>
__host__ __device__ __forceinline__ void kv_tile_share(const KvArgs &a, const KvAttendArgs &p, int rows, const KvSeq &q, int cuts, int first, KvShare &s)
{
    s.row0 = q.row0;
    s.base = q.base;
    s.len = q.len;
    s.n_rows = q.n * p.R;
    s.item0 = first + static_cast<int64_t>(q.row_tiles - 1 - s.rt) * cuts;
    s.lo = q.base + p.by_R.of(s.rt * rows);
    s.hi = q.base + p.by_R.of(min((s.rt + 1) * rows, s.n_rows) - 1);
    s.span = kv_span<TOK>(a, p, s.lo, s.hi, q.len);
    s.share = s.span.tiles;
    s.live = 1;
    if (cuts > 1) {
        s.share = max(static_cast<int>(static_cast<uint32_t>(max(q.most, s.span.tiles) + cuts - 1) / static_cast<uint32_t>(cuts)), p.min_tiles);
        s.share |= p.odd;
        s.live = max(static_cast<int>(static_cast<uint32_t>(s.span.tiles + s.share - 1) / static_cast<uint32_t>(s.share)), 1);
    }
}

struct KvChoice {
    bool many, cols;
    int rows, row_tiles, splits, min_tiles;
    int64_t items;
    size_t partial_rows;  // of the workspace, whatever number of rows the tensors have
};

inline KvChoice choose(const KvArgs &a, int D, int R, int reach, int compute_units)
{
    KvChoice c;
    const int most = a.max_new * R;  // rows of a head and sequence
    // The few rows' kernel reads the cache once for 16 of them, the other one dequantises every tile, for 128 or 256 (16 sequences of
    // 4096 tokens, 8 heads of 128: 64 rows 46 us to 61, with two groups 55 to 64, with four 98 to 64; 96 rows 78 to 64; 64 tokens alone,
    // 40 heads: 5.8 to 10.2).  Four groups: 32 rows 52 us to 63.  Of 8 groups it takes two rows at once (heads of 256: 4 rows 72 us to
    // 135, 8 rows 118 to 136, 16 rows 214 to 136).
    c.many = most > (a.ng <= 2 ? 64 : a.ng == 4 ? 32 : 8);
    // A column for each row and group: one accumulation for all groups, but only 16 / ng rows a tile.  Two tiles of it are still
    // faster than one of 16 rows whose groups come one after the other if those are 4 (8 rows of heads of 128: 35 us to 40, 16 rows 62
    // to 42), not if they are 2 (16 rows 35 to 28); with heads of 256 and 4 groups the latter lacks registers (16 rows 91 to 151).
    c.cols = a.ng > 1 && !c.many && (a.ng == 8 || (D == 256 && a.ng == 4) || most * a.ng <= (a.ng == 4 ? 32 : 16));
    c.rows = c.many ? 128 : c.cols ? 16 / a.ng : 16;
    // 256 rows a workgroup dequantise a tile half as often as 128, if they fill the device and are most of a tile (4096 tokens over
    // 16384, 32 heads: 1060 us and 1110; 2048 over 2048, 5 heads, which do not: 38 and 36).
    if (c.many && D <= 128) {
        const int64_t big = std::min<int64_t>(static_cast<int64_t>(a.n_seqs) * ((most + 255) / 256), a.rows * R / 256 + a.n_seqs);
        if (a.heads * big >= compute_units && a.rows * R >= 512ll * a.n_seqs) c.rows = 256;
    }
    const int tok = !c.many ? kKvTile : D == 256 ? 32 : 64;
    // at least 128 tokens a share, a step for each wave, or 256 ones that many rows take together
    c.min_tiles = (c.many ? 256 : 128) / tok;
    const int64_t slots = std::max<int64_t>((c.many ? 1 : 3) * compute_units / a.heads, 1);
    const int64_t cuts = std::min<int64_t>(((reach + tok - 1) / tok + 1) / c.min_tiles, 256);
    // Where tiles of rows fill the device uncut, a long sequence among short ones is cut all the same, if there may be one (one
    // of 100 000 tokens among 99 of 200 to 1000, 8 heads: 69 us, uncut 953; 64 equal ones of 8192, 40 heads: 344 and 346).
    const bool always = !c.many && reach >= 8192;
    const auto tiles_of = [&](int rows) { return static_cast<int64_t>((most + rows - 1) / rows); };
    // One sequence: as many shares as fit; two where its first tiles of rows are so much shorter than its last that they fit anyway
    // (4096 tokens over themselves, 5 heads: 96 us to 67; 2048, which three shares fit, with six of them 33 to 36).
    const auto wanted = [&](int64_t groups) {
        const int64_t seen = static_cast<int64_t>(reach) * 2 - std::min(a.max_new, reach);  // of 2 reach, by an average row
        return std::max(slots / groups, std::min<int64_t>(c.many ? slots * 2 * reach / (groups * seen) : 0, 2));
    };
    const auto listed = [&](int64_t groups) { return std::min(std::max(slots, groups + std::max<int64_t>(groups / 2, 1)), groups * cuts); };
    c.row_tiles = tiles_of(c.rows);
    // tiles of rows: no more than the rows there are and one more of each sequence
    const int64_t all = a.n_seqs * tiles_of(c.rows), groups = std::min(all, a.rows * R / c.rows + a.n_seqs);
    c.splits = 1;
    c.items = groups;
    if (cuts > 1 && (slots > groups || (always && a.n_seqs > 1))) {
        c.splits = a.n_seqs > 1 ? 2 : std::max<int64_t>(std::min(wanted(groups), cuts), 1);
        c.items = a.n_seqs > 1 ? listed(groups) : groups * c.splits;
    }
    // (fewer rows than sequences times max_new may leave room for shares; tiles of 256 rows fill the device uncut)
    c.partial_rows = 0;
    if (cuts > 1) {
        const int rows = c.many ? 128 : c.rows;
        const int64_t top = std::min(a.n_seqs * tiles_of(rows), always ? INT64_MAX : slots - 1);
        if (top > 0) c.partial_rows = static_cast<size_t>(a.heads) * rows * std::max(listed(top), std::min(c.many ? 2 * slots : slots, top * cuts));
    }
    return c;
}

// Tokens that a tile of rows may go through: no more than the workspace was sized for.
inline int reach_of(const KvArgs &a, const KvAttendArgs &p, int max_len)
{
    return p.window == 0 ? max_len : static_cast<int>(std::min<int64_t>(max_len, static_cast<int64_t>(p.window) + p.sinks + a.max_new));
}

inline void take_choice(const KvArgs &a, const KvChoice &c, KvAttendArgs &p)
{
    p.splits = c.splits;
    p.by_R = KvDivisor(p.R);
    p.by_heads = KvDivisor(a.heads);
    p.by_rows = KvDivisor(c.rows);
    p.items = c.items;
    p.row_tiles = c.row_tiles;
    p.min_tiles = c.min_tiles;
    p.odd = c.many;
}

}  // namespace tpq
