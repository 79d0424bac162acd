// Attention over the 4-bit cache of keys and values.
//
//   s_j = scale * q . k_j,  out = sum_j exp(s_j) v_j / sum_j exp(s_j),  k_j, v_j = code * scale_j + zero_j per group
//
// in one pass over the keys with a running maximum and sum.  Two kernels read the cache and a third joins shares of long sequences.
//
// Few rows (single tokens, drafts, short prompts) are bound by reading the cache, D + 8 ng bytes a token and head, so codes are
// never dequantised.  Per group, with code c of a key and of a value,
//   q . k_j = scale_j * sum(q c) + zero_j * sum(q),  sum_j w_j v_j = sum_j (w_j scale_j) c + sum_j w_j zero_j:
// the products' operands are the codes themselves.  128 + c is a bf16 number whose lowest bits are c's (one and-or for two codes), and
// -128 * sum(q) is where an accumulator starts; for the values a row of ones gives 128 * (sum of the weights as the products see
// them), which comes off at the end.  Weights are two bf16 numbers each, 17 bits: at the price of a second product, which has
// nothing to wait for.  (64 sequences of 1024 to 4096 tokens, 40 heads of 128: 908 MB in 193 us, 4.7 TB/s of the 5.0 that a copy reaches.)
//
// Many rows are bound by products, and every key meets 128 or 256 of them: tiles of 64 tokens are dequantised once, to fp16, into
// LDS for 4 or 8 waves of 32 rows, products are 32 x 32 x 16.  (4096 tokens over 16384, 32 heads: 0.98 ms, 980 TFLOP/s; matrix
// cores busy 48 % and the vector unit 55 % of the time, at 1.9 GHz.)
#include <atomic>
#include <type_traits>
#include <utility>

#include "tpq_device.h"
#include "tpq_kv_items.h"

namespace tpq {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kKvLowest = -3.0e38f;  // the running maximum before the first score

__device__ __forceinline__ uint32_t wave_total(uint32_t v) { return __builtin_amdgcn_readlane(wave_inclusive_sum(v), 63); }

// Of more than 64 sequences the list is drawn up once, ahead of the workgroups that look theirs up (each by itself: 300 sequences of 200
// to 1000 tokens and one of 20000 57 us, so 36; of 100 69 to 67): plan[0] the steps of a share,
// plan[1 + b] sequence b's first item, plan[1 + n_seqs] their number.
template <int TOK>
__global__ __launch_bounds__(1024) void k_kv_plan(KvArgs a, KvAttendArgs p, int rows)
{
    __shared__ uint32_t part[2][16];
    int turn = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto sums = [&](uint32_t mine, uint32_t &before) {  // over the workgroup, and over the waves in front
        turn ^= 1;  // (the last sum's parts may still be read)
        if (lane == 0) part[turn][wave] = mine;
        __syncthreads();
        uint32_t sum = 0;
        before = 0;
        for (int w = 0; w < 16; ++w) {
            before += w < wave ? part[turn][w] : 0u;
            sum += part[turn][w];
        }
        return sum;
    };
    uint64_t work = 0;
    uint32_t tiles = 0, unused;
    for (int b = threadIdx.x; b < a.n_seqs; b += 1024) {
        const KvSeq q = kv_seq<TOK>(a, p, rows, b);
        work += kv_work(q);
        tiles += q.row_tiles;
    }
    const uint32_t step = kv_step(p, work, tiles, 1023, [&](uint32_t n) { return sums(wave_total(n), unused); }, [&](uint32_t by) {
        uint32_t n = 0;
        for (int b = threadIdx.x; b < a.n_seqs; b += 1024) n += kv_items(kv_seq<TOK>(a, p, rows, b), by);
        return n;
    });
    uint32_t first = 0;
    for (int c = 0; c < a.n_seqs; c += 1024) {
        const int b = c + static_cast<int>(threadIdx.x);
        const uint32_t n = kv_items(kv_seq<TOK>(a, p, rows, b), step), sum = wave_inclusive_sum(n);
        uint32_t before;
        const uint32_t all = sums(__builtin_amdgcn_readlane(sum, 63), before);
        if (b < a.n_seqs) p.plan[1 + b] = static_cast<int32_t>(first + before + sum - n);
        first += all;
    }
    if (threadIdx.x == 0) {
        p.plan[0] = static_cast<int32_t>(step);
        p.plan[1 + a.n_seqs] = static_cast<int32_t>(first);
    }
}

// item >= 0: that item's.  item < 0: of tile s.rt of sequence s.b.  All lanes of the wave take part; the answer is the same in all.
template <int TOK>
__device__ __forceinline__ bool kv_share(const KvArgs &a, const KvAttendArgs &p, int rows, int item, KvShare &s)
{
    const int lane = threadIdx.x & 63;
    KvSeq q;
    int cuts = 1, first = 0;
    if (kv_even(a, p)) {  // as many items for each tile
        cuts = p.splits;
        if (item >= 0) s.b = a.n_seqs == 1 ? 0 : item;
        q = kv_seq<TOK>(a, p, rows, s.b);
        first = a.n_seqs == 1 ? 0 : s.b;
    } else {
        uint32_t step;
        if (a.n_seqs <= 64) {  // a lane has a sequence
            const KvSeq mine = kv_seq<TOK>(a, p, rows, lane);
            step = kv_step(p, kv_work(mine), mine.row_tiles, 63, [](uint32_t n) { return wave_total(n); }, [&](uint32_t by) { return kv_items(mine, by); });
            const uint32_t n = kv_items(mine, step), sum = wave_inclusive_sum(n);
            if (item >= 0) {
                const uint64_t past = __builtin_amdgcn_ballot_w64(static_cast<uint32_t>(item) < sum);
                if (!past) return false;
                s.b = __builtin_ctzll(past);
            }
            q.row0 = __builtin_amdgcn_readlane(mine.row0, s.b);
            q.n = __builtin_amdgcn_readlane(mine.n, s.b);
            q.base = __builtin_amdgcn_readlane(mine.base, s.b);
            q.len = __builtin_amdgcn_readlane(mine.len, s.b);
            q.row_tiles = __builtin_amdgcn_readlane(mine.row_tiles, s.b);
            q.most = __builtin_amdgcn_readlane(mine.most, s.b);
            first = __builtin_amdgcn_readlane(sum - n, s.b);
        } else {  // k_kv_plan has been at it: the sequence looked for 64 at a time
            if (item >= 0) {
                if (item >= p.plan[1 + a.n_seqs]) return false;
                s.b = 0;
                for (int count = a.n_seqs; count > 1;) {
                    const int by = (count + 63) / 64, at = lane * by;
                    const uint64_t before = __builtin_amdgcn_ballot_w64(at < count && p.plan[1 + s.b + min(at, count - 1)] <= item);
                    const int nth = max(__builtin_popcountll(before), 1) - 1;
                    s.b += nth * by;
                    count = min(by, count - nth * by);
                }
            }
            step = p.plan[0];
            first = p.plan[1 + s.b];
            q = kv_seq<TOK>(a, p, rows, s.b);
        }
        cuts = max((q.most + step - 1) / step, 1u);
    }
    s.split = 0;
    if (item >= 0) {  // (the last rows have the most keys: first)
        const int nth = cuts == 1 ? item - first : static_cast<int>(static_cast<uint32_t>(item - first) / static_cast<uint32_t>(cuts));
        s.rt = q.row_tiles - 1 - nth;
        s.split = item - first - nth * cuts;
    }
    if (s.rt < 0 || s.rt >= q.row_tiles) return false;
    kv_tile_share<TOK>(a, p, rows, q, cuts, first, s);
    return s.split < s.live && s.item0 + s.split < p.items;
}

// Over lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them (the swaps leave the rows of 16 and the halves beside each other).
__device__ __forceinline__ float group4_max(float v)
{
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const uint32_t y = __float_as_uint(v);
    const auto t = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float group4_sum(float v)
{
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const uint32_t y = __float_as_uint(v);
    const auto t = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// The value that lane N of the caller's row of 16 holds.
template <int N>
__device__ __forceinline__ float of_row(float v)
{
    return dpp_f32<0x150 + N>(v);
}
template <int N, typename F, int... I>
__device__ __forceinline__ void for_each_of(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void for_each(F &&f)
{
    for_each_of<N>(f, std::make_integer_sequence<int, N>{});
}

// codes of a dword -> 128 + code in bf16 (8 bits of significand: exact), nibbles t and 4 + t a pair
// (one instruction with both constants in registers, one of them scalar: neither may be a literal)
struct CodePair {
    uint32_t mask = 0x000F000Fu, base = 0x43004300u;
    __device__ __forceinline__ CodePair() { asm volatile("" : "+s"(mask), "+v"(base)); }
    __device__ __forceinline__ uint32_t operator()(uint32_t w) const { return (w & mask) | base; }
};

// The value that lane N of the caller's group of RW lanes holds (RW = 2: lane N % 2).
template <int RW, int N>
__device__ __forceinline__ float of_group(float v)
{
    constexpr int s = RW == 2 ? (N & 1) * 0x55 + 0xA0 : N * 0x55;
    return dpp_f32<s>(v);
}

// What a wave reads of a step's 32 tokens: lane (m, g) = (l % 16, l / 16).
template <int D, int NG, bool COLS>
struct KvRaw {
    static constexpr int KW = D / 32, VW = D == 256 ? 2 : 1;  // words: of a token's quarter of K codes; of a token's chunk of V codes
    uint32_t k[2][KW];       // tokens 16 j + m
    uint32_t v[2][4][VW];    // tokens 16 j + 4 g + i
    static constexpr int X = NG == 8 ? 2 : 1, META = COLS ? 4 * X : NG;
    uint32_t meta[META];     // COLS: 4 kv + 2 j ... of the lane's group; else lane 8 kv + 4 j + i of a row of 16: keys' (kv = 0) or values' scale and zero of token 16 j + 4 g + i
    bool bad[2];             // (uniform) a page that is none
};

// Few rows: 4 waves, each with its own tiles of 32 tokens and a copy of the accumulators, put together at the end.  A tile's 32
// tokens are its products' rows and the queries its columns, so that a score's lane holds what the second product's operand wants: no
// exchange between them.  COLS: a column for each row and group (the row's features of that group, zeros beside them); otherwise groups
// one after the other.  Bound by memory at one and two groups and by columns (4.2 to 4.7 TB/s over long contexts), by the
// vector unit at four groups in turn; short contexts by the chain arguments, lengths, pages, codes, 6 us.
template <int D, int GROUPS, bool COLS>
__global__ __launch_bounds__(256, D <= 128 && (COLS || GROUPS <= 2) ? 3 : 2) void k_kv_attend_few(KvArgs a, KvAttendArgs p)
{
    constexpr int NG = COLS ? 1 : GROUPS;  // groups one after the other
    constexpr int KK = D / 32, NT = D / 16, KPG = KK / NG, TPG = NT / NG, ROWS = COLS ? 16 / GROUPS : 16;
    constexpr int RW = COLS ? 16 / GROUPS : 16;  // columns of a group
    typedef KvRaw<D, GROUPS, COLS> Raw;
    __shared__ float sO[2][ROWS][D + 4];
    __shared__ float sM[2][ROWS], sL[2][ROWS];
    const CodePair code_pair;
    const uint32_t ln = threadIdx.x & 63u, m = ln & 15u, g = ln >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    KvShare w;
    const int item = p.by_heads.of(blockIdx.x), h = blockIdx.x - item * a.heads;
    if (!kv_share<kKvTile>(a, p, ROWS, item, w)) return;
    const int rt = w.rt, split = w.split, b = w.b;
    const int64_t row0 = w.row0;
    const int n_rows = w.n_rows, base = w.base, len = w.len, hi = w.hi, live = w.live, share = w.share;
    const KvSpan span = w.span;
    const int v1 = min((split + 1) * share, span.tiles);

    // queries: column m of the products' right operand; COLS: column RW gr + r has row r's features of group gr
    const uint32_t mr = m % RW, mg = m / RW;
    bf16x8_t q[KK];
    float qs[NG];
    const int row = rt * ROWS + static_cast<int>(mr), rc = min(row, n_rows - 1), i = p.by_R.of(rc), pos = base + i;
    const uint8_t *src = p.Q + (row0 + i) * p.ldQ + (h * p.R + rc - i * p.R) * (2 * D) + 16 * g;
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
        float sum = 0.0f;
#pragma unroll
        for (int kk = gr * KPG; kk < (gr + 1) * KPG; ++kk) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(src + 64 * kk);
            if (p.scale < 0.0f) w ^= 0x80008000u;  // (scores are then multiplied by |scale|: their order is the products')
            if (COLS && static_cast<uint32_t>(kk * GROUPS / KK) != mg) w = u32x4{0, 0, 0, 0};
            q[kk] = __builtin_bit_cast(bf16x8_t, w);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += bf16_lo_to_f32(ws[e]) + bf16_hi_to_f32(ws[e]);
        }
        qs[gr] = group4_sum(sum);
    }

    const int n_blocks = (min(len, a.ld_table << a.lg_page) + 15) / 16;  // blocks of 16 tokens that exist
    const int all_to = min(w.lo, 16 * n_blocks - 1);                     // last token that every row may see (rows may lie past the table)
    const uint32_t page_len = 1u << a.lg_page, page_mask = page_len - 1u;
    const int32_t *table = a.table + static_cast<int64_t>(b) * a.ld_table;
    // The page numbers of the wave's next 32 steps, two a step, one a lane: one load's latency for all of them.
    auto pages_of = [&](int v) {
        const int tile = span.tile(min(v + 4 * static_cast<int>(ln >> 1), v1 - 1));
        const int block = min(2 * tile + static_cast<int>(ln & 1u), n_blocks - 1);
        return table[(16 * block) >> a.lg_page];
    };
    auto load = [&](Raw &raw, int v, int pages, int nth) {
        const int tile = span.tile(v);
        const uint8_t *metas[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int block = min(2 * tile + j, n_blocks - 1);
            const uint32_t slot = (16u * block) & page_mask;
            const int id = __builtin_amdgcn_readlane(pages, 2 * nth + j);
            raw.bad[j] = static_cast<uint32_t>(id) >= static_cast<uint64_t>(a.n_pages);
            const uint8_t *cell = a.cache + (raw.bad[j] ? 0 : id) * a.page_bytes + static_cast<int64_t>(h) * a.cell_bytes;
            const uint8_t *k = cell + slot * (D / 2);
            const uint32_t ko = m * (D / 2) + g * (D / 8);
#pragma unroll
            for (int w = 0; w < Raw::KW; ++w) raw.k[j][w] = reinterpret_cast<const uint32_t *>(k + ko)[w];
            const uint8_t *vc = cell + (page_len + slot) * (D / 2);
            const uint32_t vo = g * (2 * D) + (D == 64 ? m / 2 * 4 : m * (D / 32));
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < Raw::VW; ++w) raw.v[j][i][w] = reinterpret_cast<const uint32_t *>(vc + vo + i * (D / 2))[w];
            metas[j] = cell + page_len * D + 4 * slot;
        }
        if constexpr (COLS) {
            // a lane's own group's, token 4 g + m % 4 (RW = 2: 4 g + 2 x + m % 2)
            const uint32_t at = mg * page_len + 4 * g + (m & (RW == 2 ? 1u : 3u));
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int x = 0; x < Raw::X; ++x)
                        raw.meta[(2 * kv + j) * Raw::X + x] = *reinterpret_cast<const uint32_t *>(metas[j] + 4 * (at + kv * GROUPS * page_len + 2 * x));
        } else {
            const uint8_t *meta = (m & 4u ? metas[1] : metas[0]) + (m & 8u ? 4 * NG * page_len : 0u) + 16 * g + 4 * (m & 3u);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) raw.meta[gr] = *reinterpret_cast<const uint32_t *>(meta + 4 * (gr * page_len));
        }
    };

    f32x4 o[NT], oc;  // accumulators; row gr of oc: 128 * (sum of group gr's weights as the products see them)
    float zs[NG], mx = kKvLowest, l = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = f32x4{0, 0, 0, 0};
    oc = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) zs[gr] = 0.0f;
    const float log2e = 1.44269504f;

    // scores in powers of two: exp(s) = 2^(s log2 e)
    const int window = p.window > 0 ? p.window : 1 << 30;
    const float k_score = p.softcap > 0.0f ? 1.0f : fabsf(p.scale) * log2e;
    const float cap_in = p.softcap > 0.0f ? fabsf(p.scale) / p.softcap * 2.0f * log2e : 0.0f, cap_out = p.softcap * log2e;

    // scale or zero of key (kv = 0) or value 16 J + 4 g + I, for the caller's group
    auto meta_of = [&](auto kv, auto jj, auto ii, const float (&from)[Raw::META], int gr) __attribute__((always_inline)) {
        constexpr int KV = decltype(kv)::value, J = decltype(jj)::value, I = decltype(ii)::value;
        if constexpr (COLS) return of_group<RW, I>(from[(2 * KV + J) * Raw::X + (Raw::X == 2 ? I / 2 : 0)]);
        else return of_row<8 * KV + 4 * J + I>(from[gr]);
    };
    constexpr std::integral_constant<int, 0> of_keys{};
    constexpr std::integral_constant<int, 1> of_values{};

    auto metas_of = [&](const Raw &raw, int gr, float (&sc)[Raw::META], float (&ze)[Raw::META]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < Raw::META; ++x)
            if (COLS || x == gr) {
                sc[x] = bf16_lo_to_f32(raw.meta[x]);
                ze[x] = bf16_hi_to_f32(raw.meta[x]);
            }
    };

    auto step = [&](const Raw &raw, int v) {
        const int t0 = span.tile(v) * kKvTile;
        const bool whole = t0 + kKvTile - 1 <= all_to && (p.window == 0 || t0 > hi - p.window || t0 + kKvTile <= p.sinks) && !raw.bad[0] && !raw.bad[1];
        float s[2][4];
        bool vis[2][4];
        for_each<2>([&](auto jj) {
            constexpr int J = decltype(jj)::value;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float c0 = -128.0f * qs[gr];
                asm volatile("" : "+v"(c0));  // (anew in every step: kept outside the loop it would take four registers)
                f32x4 acc = {c0, c0, c0, c0};
#pragma unroll
                for (int kk = gr * KPG; kk < (gr + 1) * KPG; ++kk) {
                    const uint32_t w = raw.k[J][kk];
                    const u32x4 c = {code_pair(w), code_pair(w >> 4), code_pair(w >> 8), code_pair(w >> 12)};
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, c), q[kk], acc, 0, 0, 0);
                }
                float sc[Raw::META], ze[Raw::META];
                metas_of(raw, gr, sc, ze);
                for_each<4>([&](auto i) {
                    constexpr int I = decltype(i)::value;
                    // (products, whose operand the exchange goes into; multiply-adds would take a move for each)
                    const float x = meta_of(of_keys, jj, i, sc, gr) * acc[I], z = meta_of(of_keys, jj, i, ze, gr) * qs[gr];
                    s[J][I] = gr == 0 ? x + z : (s[J][I] + x) + z;
                    // the groups' parts (in an order that leaves the same sum in all of them)
                    if (COLS && RW <= 8) s[J][I] += dpp_f32<0x128>(s[J][I]);
                    if (COLS && RW <= 4) s[J][I] += dpp_f32<0x124>(s[J][I]);
                    if (COLS && RW <= 2) s[J][I] += dpp_f32<0x122>(s[J][I]);
                });
            }
        });
        if (p.softcap > 0.0f) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                // cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1)
                const float e = __builtin_amdgcn_exp2f(s[x >> 2][x & 3] * cap_in) + 1.0f;
                s[x >> 2][x & 3] = __builtin_fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(e), cap_out);
            }
        }
        if (!whole) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const int j = x >> 2, i = x & 3, key = t0 + 16 * j + 4 * static_cast<int>(g) + i;
                vis[j][i] = (key <= pos) & ((key > pos - window) | (key < p.sinks)) & !raw.bad[j] & (key < 16 * n_blocks);
                s[j][i] = vis[j][i] ? s[j][i] : kKvLowest;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int x = 1; x < 8; ++x) top = fmaxf(top, s[x >> 2][x & 3]);
        top *= k_score;
        // The maximum only follows where a weight would pass 2^8: weights are relative anyway, and a step without it saves
        // the accumulators' rescaling.
        if (__builtin_amdgcn_ballot_w64(top > mx + 8.0f)) {
            const float now = fmaxf(mx, group4_max(top)), alpha = __builtin_amdgcn_exp2f(mx - now);
            mx = now;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t] *= alpha;
            oc *= alpha;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) zs[gr] *= alpha;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            float &e = s[x >> 2][x & 3];  // the weight, in the score's place
            e = __builtin_amdgcn_exp2f(__builtin_fmaf(e, k_score, -mx));
            if (!whole) e = vis[x >> 2][x & 3] ? e : 0.0f;
            l += e;
        }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            float sc[Raw::META], ze[Raw::META];
            metas_of(raw, gr, sc, ze);
            u32x4 ph, pl;
            for_each<2>([&](auto jj) {
                constexpr int J = decltype(jj)::value;
                float w[4];
                for_each<4>([&](auto i) {
                    constexpr int I = decltype(i)::value;
                    w[I] = meta_of(of_values, jj, i, sc, gr) * s[J][I];
                });
                if (whole) {
                    for_each<4>([&](auto i) {
                        constexpr int I = decltype(i)::value;
                        zs[gr] += meta_of(of_values, jj, i, ze, gr) * s[J][I];
                    });
                } else {  // (what lies behind a hidden key may be anything)
                    for_each<4>([&](auto i) {
                        constexpr int I = decltype(i)::value;
                        const float z = meta_of(of_values, jj, i, ze, gr) * s[J][I];
                        zs[gr] += vis[J][I] ? z : 0.0f;
                        w[I] = vis[J][I] ? w[I] : 0.0f;
                    });
                }
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const uint32_t hi2 = pack_bf16x2(w[i], w[i + 1]);
                    ph[2 * J + i / 2] = hi2;
                    pl[2 * J + i / 2] = pack_bf16x2(w[i] - bf16_lo_to_f32(hi2), w[i + 1] - bf16_hi_to_f32(hi2));
                }
            });
            const bf16x8_t bh = __builtin_bit_cast(bf16x8_t, ph), bl = __builtin_bit_cast(bf16x8_t, pl);
            uint32_t one = NG == 1 || m == static_cast<uint32_t>(gr) ? code_pair.base : 0u;
            if (NG > 1) asm volatile("" : "+v"(one));
            const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, (u32x4{one, one, one, one}));
            oc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, bh, oc, 0, 0, 0);
            oc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, bl, oc, 0, 0, 0);
#pragma unroll
            for (int t = gr * TPG; t < (gr + 1) * TPG; ++t) {
                const int word = t / 8, byte = (t % 8) / 2;
                const uint32_t at = D == 64 ? byte + 2 * (m & 1u) : byte;
                const uint32_t sel = 0x0C000C00u | ((4u + at) << 16) | at;
                u32x4 c;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int j = x >> 1, i = 2 * (x & 1);
                    const uint32_t y = __builtin_amdgcn_perm(raw.v[j][i + 1][word], raw.v[j][i][word], sel);
                    c[x] = code_pair(t & 1 ? y >> 4 : y);
                }
                const bf16x8_t av = __builtin_bit_cast(bf16x8_t, c);
                o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bh, o[t], 0, 0, 0);
                o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bl, o[t], 0, 0, 0);
            }
            if (NG > 1) __builtin_amdgcn_sched_barrier(0);  // (one group's codes and weights in registers at a time)
        }
    };

    // A step's loads are issued before the step in front of it is worked on.
    const int v0 = split * share + wave;
    Raw even, odd;
    int pages = 0;
    if (v0 < v1) {
        pages = pages_of(v0);
        load(even, v0, pages, 0);
    }
    for (int v = v0, nth = 0; v < v1; v += 8) {
        if (v + 4 < v1) load(odd, v + 4, pages, nth + 1);
        __builtin_amdgcn_sched_barrier(0);
        step(even, v);
        if (v + 4 >= v1) break;
        nth += 2;
        if (nth == 32) {
            nth = 0;
            pages = pages_of(v + 8);
        }
        if (v + 8 < v1) load(even, v + 8, pages, nth);
        __builtin_amdgcn_sched_barrier(0);
        step(odd, v + 4);
    }

    // 128 * (sum of the weights) off the codes, the zeros' share on
    l = group4_sum(l);
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
        const float z = group4_sum(zs[gr]), c = NG == 1 ? oc[0] : __shfl(oc[gr & 3], 16 * (gr >> 2) + m, 64);
#pragma unroll
        for (int t = gr * TPG; t < (gr + 1) * TPG; ++t) o[t] = o[t] - c + z;
    }
    // (COLS: a lane's accumulators are its column's, of which those of its own group count)
    const auto mine = [&](int t) { return !COLS || static_cast<uint32_t>(t * GROUPS / NT) == mg; };
    // the four waves' results into wave 0's: 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (int from = 2; from >= 1; from >>= 1) {
        if (wave >= from && wave < 2 * from) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (mine(t)) *reinterpret_cast<f32x4 *>(&sO[wave - from][mr][16 * t + 4 * g]) = o[t];
            if (g == 0 && mg == 0) {
                sM[wave - from][mr] = mx;
                sL[wave - from][mr] = l;
            }
        }
        __syncthreads();
        if (wave < from) {
            const float m2 = sM[wave][mr], now = fmaxf(mx, m2);
            const float f1 = __builtin_amdgcn_exp2f(mx - now), f2 = __builtin_amdgcn_exp2f(m2 - now);
            mx = now;
            l = l * f1 + sL[wave][mr] * f2;
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (mine(t)) o[t] = o[t] * f1 + *reinterpret_cast<const f32x4 *>(&sO[wave][mr][16 * t + 4 * g]) * f2;
        }
        __syncthreads();
    }
    if (wave != 0 || row >= n_rows) return;
    if (live == 1) {
        const int i = p.by_R.of(row);
        uint8_t *dst = p.out + (row0 + i) * p.ldOut + (h * p.R + row - i * p.R) * (2 * D) + 8 * g;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (mine(t)) *reinterpret_cast<uint2 *>(dst + 32 * t) = make_uint2(pack_bf16x2(o[t][0] * inv, o[t][1] * inv), pack_bf16x2(o[t][2] * inv, o[t][3] * inv));
    } else {
        const int64_t at = (h * static_cast<int64_t>(p.items) + w.item0 + split) * ROWS + mr;
        float *dst = p.part + at * D + 4 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (mine(t)) *reinterpret_cast<f32x4 *>(dst + 16 * t) = o[t];
        if (g == 0 && mg == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(mx, l);
    }
}

// ---- many rows ----------------------------------------------------------------------------------

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}
// c * scale + zero of two codes that sit in bits 4 .. 7 of the halves of w: there a code is the fp16 number c 2^-20
// (below fp16's normal range its patterns count in equal steps), which the scale makes good.
__device__ __forceinline__ uint32_t dequant2(uint32_t w, uint32_t scale, uint32_t zero)
{
    const f16x2_t c = __builtin_bit_cast(f16x2_t, w & 0x00F000F0u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, __builtin_bit_cast(f16x2_t, scale), __builtin_bit_cast(f16x2_t, zero)));
}

// W waves of 32 rows; the keys and values of TOK tokens at a time, dequantised into LDS by all of them.  A step is bound by issue:
// 32 products (1024 cycles at a row of 128), about 64 exponentials' worth of vector work and 64 codes a lane; hence the rounds
// below, in which products run while the vector unit makes weights and dequantises (a tile of 64 tokens, 128 rows: 1.4 us; one
// step after the other, as where keys are hidden, 2.8).  Heads of 256 take all registers, so one wave a SIMD, and tiles of 32 tokens
// (1.7 us).  Where nothing fills the device, what is left is the way to the first product, 6 us: arguments, lengths, page numbers,
// then scales and zeros of the whole share.
template <int D, int NG, int W, int TOK>
__global__ __launch_bounds__(64 * W, D == 256 ? 1 : 2) void k_kv_attend_many(KvArgs a, KvAttendArgs p)
{
    constexpr int KS = D / 16, DT = D / 32, TB = TOK / 32, ROWS = 32 * W, BLOCKS = TOK / 16;
    // a wave dequantises one of PARTS parts of a block of 16 tokens: PIECES times 8 features of a key, or 2 of 4 values, a lane
    constexpr int PARTS = W / BLOCKS, PIECES = D / 32 / PARTS, GROUPS = NG > PARTS ? NG / PARTS : 1;  // groups of a part
    constexpr int KROW = 2 * D, VROW = 2 * TOK, KBYTES = TOK * KROW, VBYTES = D * VROW;
    constexpr int WINDOW = 64 / BLOCKS;  // tiles whose page numbers a wave holds at a time
    static_assert(W % BLOCKS == 0 && PIECES >= 1 && GROUPS <= 4, "parts");
    extern __shared__ u32x4 smem_kv[];
    uint8_t *const lds = reinterpret_cast<uint8_t *>(smem_kv);
    __shared__ uint32_t reduced[3];
    const uint32_t ln = threadIdx.x & 63u, c32 = ln & 31u, hh = ln >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    KvShare w;
    const int item = p.by_heads.of(blockIdx.x), h = blockIdx.x - item * a.heads;
    if (!kv_share<TOK>(a, p, ROWS, item, w)) return;
    const int rt = w.rt, split = w.split, b = w.b;
    const int v0 = split * w.share, v1 = min(v0 + w.share, w.span.tiles);
    const int wrow = rt * ROWS + 32 * wave;
    const int wlo = w.base + p.by_R.of(wrow);  // the wave's first and last position
    const int whi = w.base + p.by_R.of(min(wrow + 32, w.n_rows) - 1);
    const bool idle = wrow >= w.n_rows;

    // queries in fp16, exactly (but for elements below 2^-27 of a row's largest): each row at a power of two of its own
    const int row = wrow + static_cast<int>(c32), rc = min(row, w.n_rows - 1), qi = p.by_R.of(rc);
    const int pos = w.base + qi;
    // Rows of both operands are cut into slots of 16 bytes, which lie permuted by their row's number: 16 lanes are served at once
    // if they touch every one of 64 banks once, in reads (16 rows, one slot) and in writes (4 keys' 4 slots; 16 features' halves of
    // one or two) alike.
    auto key_slot = [](uint32_t t) { return D == 64 ? (((t >> 1) & 1u) << 2) | ((t >> 2) & 3u) : ((t & 3u) << 2) | ((t >> 2) & 3u); };
    auto value_slot = [](uint32_t d) { return TOK == 64 ? (d >> 1) & 7u : (d >> 2) & 3u; };
    u32x4 raw[KS];
    {
        const uint8_t *src = p.Q + (w.row0 + qi) * p.ldQ + (h * p.R + rc - qi * p.R) * (2 * D) + 16 * hh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) raw[ks] = *reinterpret_cast<const u32x4 *>(src + 32 * ks);
    }

    const int n_blocks = (min(w.len, a.ld_table << a.lg_page) + 15) / 16;
    const uint32_t page_len = 1u << a.lg_page, page_mask = page_len - 1u;
    const int32_t *table = a.table + static_cast<int64_t>(b) * a.ld_table;
    const uint8_t *const cache_h = a.cache + static_cast<int64_t>(h) * a.cell_bytes;
    // page numbers of the WINDOW steps from v on: lane BLOCKS * step + block (-1: no page)
    auto pages_of = [&](int v) __attribute__((always_inline)) {
        const int block = w.span.tile(min(v + static_cast<int>(ln) / BLOCKS, v1 - 1)) * BLOCKS + static_cast<int>(ln) % BLOCKS;
        const int id = table[(16 * min(block, n_blocks - 1)) >> a.lg_page];
        return block < n_blocks && static_cast<uint32_t>(id) < static_cast<uint64_t>(a.n_pages) ? id : -1;
    };

    // What a lane loads of its wave's part of a tile: codes of one key and of four values, and one of the scales and zeros
    // of each that its neighbours and it need.  Keys: lane l has quarter l % 4 of token l / 4 and group l % 4 of the part.
    // Values: chunk m = l % 16 of the 4 tokens from 8 (l / 16 % 2) + 4 (l / 32) on, and group m / 4 of token m % 4.
    // (No branches: the loads' order is known, and so is how many are younger than the ones waited for.)
    struct Codes {
        uint32_t k[PIECES], v[4], km, vm;
    };
    const int block = wave % BLOCKS, part = wave / BLOCKS;
    const uint32_t m16 = ln & 15u, quad = ln & 3u, vt = 8u * ((ln >> 4) & 1u) + 4u * hh;
    const uint32_t group0 = part * NG / PARTS, k_at = ln * (D / 8) + 4u * PIECES * part, v_at = vt * (D / 2) + (D == 64 ? m16 / 2 * 4 : D == 256 ? m16 * 8 + 4 * part : m16 * 4);
    const uint32_t km_at = 4u * ((group0 + min(quad, GROUPS - 1u)) * page_len + (ln >> 2)), vm_at = 4u * ((NG + group0 + min(m16 >> 2, GROUPS - 1u)) * page_len + vt + (m16 & 3u));
    // (keys of step vk, values of step vv; of steps past the last: the last's)
    auto load_codes = [&](Codes &c, int vk, int vv, int base, int pages) __attribute__((always_inline)) {
        const int k = min(vk, v1 - 1), v = min(vv, v1 - 1);
        const int idk = max(__builtin_amdgcn_readlane(pages, (k - base) * BLOCKS + block), 0), idv = max(__builtin_amdgcn_readlane(pages, (v - base) * BLOCKS + block), 0);
        const uint32_t sk = (16u * (w.span.tile(k) * BLOCKS + block)) & page_mask, sv = (16u * (w.span.tile(v) * BLOCKS + block)) & page_mask;
        const uint8_t *ck = cache_h + idk * a.page_bytes, *cv = cache_h + idv * a.page_bytes;
        const uint8_t *ks = ck + sk * (D / 2), *vs = cv + (page_len + sv) * (D / 2);
        c.km = *reinterpret_cast<const uint32_t *>(ck + page_len * D + 4 * sk + km_at);
#pragma unroll
        for (int e = 0; e < PIECES; ++e) c.k[e] = reinterpret_cast<const uint32_t *>(ks + k_at)[e];
        c.vm = *reinterpret_cast<const uint32_t *>(cv + page_len * D + 4 * sv + vm_at);
#pragma unroll
        for (int i = 0; i < 4; ++i) c.v[i] = *reinterpret_cast<const uint32_t *>(vs + v_at + i * (D / 2));
    };
    // (the first pages' numbers of the scan below too: one latency)
    constexpr int U = NG <= 2 ? 4 : 2, PER = 64 / TOK;  // loads of a lane in flight together, tiles that a wave's lanes cover
    int base = v0, pages = 0, key[U], id[U];
    auto scanned = [&](int v) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            key[u] = w.span.tile(min(v + PER * (wave + u * W) + static_cast<int>(ln) / TOK, v1 - 1)) * TOK + static_cast<int>(ln) % TOK;
            id[u] = table[min(key[u], 16 * n_blocks - 1) >> a.lg_page];
        }
    };
    Codes ca = {}, cb = {};
    if (v0 < v1) {
        pages = pages_of(v0);
        scanned(v0);
        load_codes(ca, v0, v0, base, pages);
        load_codes(cb, v0 + 1, v0 + 1, base, pages);
    }

    // The normalisation of keys and of values: a power of two that brings the largest among those that some row sees into
    // 2^-3 .. 2^-2, so that scales fit fp16 times the codes' 2^20 (what is 2^12 times smaller than the largest still has
    // fp16's 11 bits, and then one less for every halving).  From scales and zeros alone, 8 ng bytes a token and head.
    float k_norm, v_norm, k_undo, v_undo;
    bool absent;  // a block of 16 tokens at or before some row has no page, or lies past the table
    {
        if (threadIdx.x < 3) reduced[threadIdx.x] = 0;
        uint32_t top[2] = {0, 0}, missing = 0;
        for (int v = v0; v < v1; v += PER * U * W) {
            if (v > v0) scanned(v);
            uint32_t x[U][2 * NG];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool exists = key[u] < 16 * n_blocks, good = static_cast<uint32_t>(id[u]) < static_cast<uint64_t>(a.n_pages);
                missing |= (!(exists & good) & (key[u] <= w.hi)) ? 1u : 0u;
                const bool seen = exists & good & (key[u] <= w.hi) & ((p.window == 0) | (key[u] > w.lo - p.window) | (key[u] < p.sinks));
                const uint32_t *src = reinterpret_cast<const uint32_t *>(cache_h + (good ? id[u] : 0) * a.page_bytes + page_len * D) + (static_cast<uint32_t>(key[u]) & page_mask);
#pragma unroll
                for (int g = 0; g < 2 * NG; ++g) x[u][g] = seen ? src[g * page_len] : 0u;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int g = 0; g < 2 * NG; ++g) {
                    const float z = bf16_hi_to_f32(x[u][g]), z1 = __builtin_fmaf(15.0f, bf16_lo_to_f32(x[u][g]), z);
                    const uint32_t big = max(__float_as_uint(z) & 0x7FFFFFFFu, __float_as_uint(z1) & 0x7FFFFFFFu);
                    top[g / NG] = max(top[g / NG], big < 0x7F800000u ? big : 0u);  // (what is not finite has no part in it)
                }
        }
        __syncthreads();
        const uint32_t kt = wave_max(top[0]), vt = wave_max(top[1]);
        if (ln == 0) {
            atomicMax(&reduced[0], kt);
            atomicMax(&reduced[1], vt);
        }
        if (__builtin_amdgcn_ballot_w64(missing != 0) && ln == 0) atomicOr(&reduced[2], 1u);
        __syncthreads();
        const int ku = min(max(251 - static_cast<int>(reduced[0] >> 23), 1), 254), vu = min(max(251 - static_cast<int>(reduced[1] >> 23), 1), 254);
        k_norm = __uint_as_float(static_cast<uint32_t>(ku) << 23);
        v_norm = __uint_as_float(static_cast<uint32_t>(vu) << 23);
        k_undo = __builtin_amdgcn_ldexpf(1.0f, 127 - ku);
        v_undo = __builtin_amdgcn_ldexpf(1.0f, 127 - vu);
        absent = reduced[2] != 0;
    }

    // (heads of 256: in LDS, laid out as the keys are; beside 128 accumulators 64 registers are too many)
    constexpr bool q_in_lds = D == 256;
    uint8_t *const q_row = lds + 2 * KBYTES + 2 * VBYTES + (32 * wave + c32) * KROW;
    const uint32_t kf = key_slot(c32), vf = value_slot(c32);
    f16x8_t q[q_in_lds ? 1 : KS];
    float row_scale;
    {
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max(top, max((raw[ks][e] << 16) & 0x7FFFFFFFu, raw[ks][e] & 0x7FFF0000u));
        const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
        const uint32_t x = both[0], y = both[1];
        const int up = min(max(267 - static_cast<int>(max(x, y) >> 23), 1), 254);  // times 2^(up - 127): the largest in 2^13 .. 2^14
        const float f = __uint_as_float(static_cast<uint32_t>(up) << 23) * (p.scale < 0.0f ? -1.0f : 1.0f);
        row_scale = fabsf(p.scale) * __builtin_amdgcn_ldexpf(1.0f, 127 - up);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = pack_f16x2(bf16_lo_to_f32(raw[ks][e]) * f, bf16_hi_to_f32(raw[ks][e]) * f);
            if (q_in_lds) *reinterpret_cast<u32x4 *>(q_row + 16 * ((2 * ks + hh) ^ kf)) = o;  // (read by this wave alone)
            else q[ks] = __builtin_bit_cast(f16x8_t, o);
        }
        if (q_in_lds) wave_lds_fence();
    }

    // Scale (times the codes' 2^20) and zero in fp16, normalised.  What is larger than the normalisation knows, or not a
    // number, is no row's: zeros, so that it stays finite next to weights of 0.
    auto converted = [&](uint32_t x, float f) __attribute__((always_inline)) {
        const float sc = bf16_lo_to_f32(x) * f, ze = bf16_hi_to_f32(x) * f, z1 = __builtin_fmaf(15.0f, sc, ze);
        const bool ok = max(__float_as_uint(ze) & 0x7FFFFFFFu, __float_as_uint(z1) & 0x7FFFFFFFu) <= 0x3E800000u;
        const uint32_t y = pack_f16x2(sc * 0x1p20f, ze);
        return ok ? y : 0u;
    };
    auto store_keys = [&](const Codes &c, auto piece, int pk) __attribute__((always_inline)) {
        constexpr int i = decltype(piece)::value, gr = NG >= PARTS ? i / (D / 32 / NG) : 0;
        const uint32_t t = 16u * block + (ln >> 2), kk = part * PIECES + i;
        const uint32_t mt = __builtin_amdgcn_update_dpp(0u, c.km, 0x55 * gr, 0xF, 0xF, true);  // lane gr of each four
        const uint32_t sc = __builtin_amdgcn_perm(mt, mt, 0x01000100u), ze = __builtin_amdgcn_perm(mt, mt, 0x03020302u);
        const uint32_t y = c.k[i];
        const u32x4 o = {dequant2(y << 4, sc, ze), dequant2(y, sc, ze), dequant2(y >> 4, sc, ze), dequant2(y >> 8, sc, ze)};
        *reinterpret_cast<u32x4 *>(lds + pk * KBYTES + t * KROW + 16 * ((4 * kk + quad) ^ key_slot(t))) = o;
    };
    const uint32_t byte0 = (D == 256 ? 0u : static_cast<uint32_t>(part * PIECES)) + (D == 64 ? 2u * (m16 & 1u) : 0u), sel0 = 0x0C000C00u | ((4u + byte0) << 16) | byte0;
    auto store_values = [&](const Codes &c, auto piece, int pv) __attribute__((always_inline)) {
        constexpr int i = decltype(piece)::value, lane = NG >= PARTS ? 4 * (i / (D / 32 / NG)) : 0;  // lanes 4 gr .. 4 gr + 3 of the row have the group's four tokens
        const uint32_t chunk = 2u * block + hh, half = (ln >> 4) & 1u, sel = sel0 + i * 0x00010001u;
        const uint32_t m0 = __builtin_amdgcn_update_dpp(0u, c.vm, 0x150 + lane, 0xF, 0xF, true), m1 = __builtin_amdgcn_update_dpp(0u, c.vm, 0x151 + lane, 0xF, 0xF, true);
        const uint32_t m2 = __builtin_amdgcn_update_dpp(0u, c.vm, 0x152 + lane, 0xF, 0xF, true), m3 = __builtin_amdgcn_update_dpp(0u, c.vm, 0x153 + lane, 0xF, 0xF, true);
        const uint32_t sc[2] = {__builtin_amdgcn_perm(m1, m0, 0x05040100u), __builtin_amdgcn_perm(m3, m2, 0x05040100u)};
        const uint32_t ze[2] = {__builtin_amdgcn_perm(m1, m0, 0x07060302u), __builtin_amdgcn_perm(m3, m2, 0x07060302u)};
        const uint32_t y0 = __builtin_amdgcn_perm(c.v[1], c.v[0], sel), y1 = __builtin_amdgcn_perm(c.v[3], c.v[2], sel);
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const uint32_t d = 16 * (2 * (part * PIECES + i) + odd) + m16;
            const uint2 o = make_uint2(dequant2(odd ? y0 : y0 << 4, sc[0], ze[0]), dequant2(odd ? y1 : y1 << 4, sc[1], ze[1]));
            *reinterpret_cast<uint2 *>(lds + 2 * KBYTES + pv * VBYTES + d * VROW + 16 * (chunk ^ value_slot(m16)) + 8 * half) = o;
        }
    };
    auto store_codes = [&](Codes &c, int pk, int pv) __attribute__((always_inline)) {
        c.km = converted(c.km, k_norm);
        c.vm = converted(c.vm, v_norm);
        for_each<PIECES>([&](auto piece) __attribute__((always_inline)) {
            store_keys(c, piece, pk);
            store_values(c, piece, pv);
        });
    };

    f32x16 o[DT];
    float mx = kKvLowest, l = 0.0f, k_exp = 0.0f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    const float log2e = 1.44269504f;
    const float cap_in = p.softcap > 0.0f ? 2.0f * log2e / p.softcap : 0.0f, cap_out = p.softcap * log2e;

    // where a lane reads its rows of the two operands (par: which of the two buffers)
    auto key_at = [&](int par, int i) __attribute__((always_inline)) {  // i = tb * KS + k
        return __builtin_bit_cast(f16x8_t, *reinterpret_cast<const u32x4 *>(lds + par * KBYTES + (32 * (i / KS) + c32) * KROW + 16 * ((2 * (i % KS) + hh) ^ kf)));
    };
    auto value_at = [&](int par, int j) __attribute__((always_inline)) {  // j = step of 16 tokens * DT + t
        return __builtin_bit_cast(f16x8_t, *reinterpret_cast<const u32x4 *>(lds + 2 * KBYTES + par * VBYTES + (32 * (j % DT) + c32) * VROW + 16 * ((2 * (j / DT) + hh) ^ vf)));
    };
    constexpr int NQ = TB * KS, NP = 2 * TB * DT, NS = 16 * TB;  // products with keys, with values; scores of a lane
    uint32_t pw[NS / 2];                                         // weights, in the order in which the products take them

    auto query_at = [&](int i) __attribute__((always_inline)) {
        if constexpr (q_in_lds) return __builtin_bit_cast(f16x8_t, *reinterpret_cast<const u32x4 *>(q_row + 16 * ((2 * (i % KS) + hh) ^ kf)));
        else return q[i % KS];
    };
    auto score = [&](f32x16 (&acc)[TB], const f16x8_t &key, const f16x8_t &query, int i) __attribute__((always_inline)) {
        const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        acc[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key, query, i % KS ? acc[i / KS] : zero, 0, 0, 0);
    };
    auto value = [&](const f16x8_t &val, int j) __attribute__((always_inline)) {
        const int first = 4 * (j / DT);
        const f16x8_t pb = __builtin_bit_cast(f16x8_t, (u32x4{pw[first], pw[first + 1], pw[first + 2], pw[first + 3]}));
        o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(val, pb, o[j % DT], 0, 0, 0);
    };
    // all of a tile's scores: operands read ahead
    auto all_scores = [&](f32x16 (&acc)[TB], int par) __attribute__((always_inline)) {
        constexpr int A = q_in_lds ? 2 : 4;
        f16x8_t fr[A + 1], fq[A + 1];
#pragma unroll
        for (int i = 0; i < A; ++i) {
            fr[i] = key_at(par, i);
            fq[i] = query_at(i);
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (i + A < NQ) {
                fr[(i + A) % (A + 1)] = key_at(par, i + A);
                fq[(i + A) % (A + 1)] = query_at(i + A);
            }
            score(acc, fr[i % (A + 1)], fq[i % (A + 1)], i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto take = [&](float (&s)[NS], const f32x16 (&acc)[TB]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NS; ++i) s[i] = acc[i / 16][i % 16];
    };
    auto exp_pair = [&](float (&s)[NS], int i) __attribute__((always_inline)) {  // in the scores' place
        s[2 * i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i], k_exp, -mx));
        s[2 * i + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i + 1], k_exp, -mx));
        asm volatile("" : "+v"(s[2 * i]), "+v"(s[2 * i + 1]));  // (here, not where they are needed)
    };
    auto pack_pair = [&](const float (&s)[NS], int i) __attribute__((always_inline)) {  // (the sum takes the weights as the products do)
        pw[i] = pack_f16x2(s[2 * i], s[2 * i + 1]);
        l = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, pw[i]), __builtin_bit_cast(f16x2_t, 0x3C003C00u), l, false);
        asm volatile("" : "+v"(pw[i]), "+v"(l));
    };
    // The running maximum brought up to a tile's.  Weights reach 2^14: 2^6 where the maximum has just been taken, and a maximum
    // follows past 2^8 of that only.
    auto settle = [&](float top) __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(top > kKvLowest && top * k_exp > mx + 14.0f) == 0) return;
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        const float both = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        const float now = both > kKvLowest ? fmaxf(mx, both * k_exp - 6.0f) : mx, alpha = __builtin_amdgcn_exp2f(mx - now);
        mx = now;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= alpha;
    };

    // Step by step: the keys of tile i + 2 and the values of i + 1 are dequantised while tile i is worked on, from codes that
    // were loaded two steps before (two sets in turn).
    if (v0 < v1) {
        store_codes(ca, 0, 0);
        cb.km = converted(cb.km, k_norm);
        for_each<PIECES>([&](auto piece) __attribute__((always_inline)) { store_keys(cb, piece, 1); });  // of the second tile
        load_codes(ca, v0 + 2, v0 + 1, base, pages);
        load_codes(cb, v0 + 3, v0 + 2, base, pages);
        __syncthreads();

        auto begin = [&](int v) __attribute__((always_inline)) {
            if (v + 4 - base >= WINDOW) {
                base = v;
                pages = pages_of(v);
            }
        };
        // a tile's values, and in the products' time the codes of the tiles to come
        auto values_and_codes = [&](auto parity, Codes &codes, int v) __attribute__((always_inline)) {
            constexpr int P = decltype(parity)::value, Q = P ^ 1, A = q_in_lds ? 2 : 4;
            f16x8_t fr[A + 1];
#pragma unroll
            for (int j = 0; j < A; ++j) fr[j] = value_at(P, j);
            codes.km = converted(codes.km, k_norm);
            codes.vm = converted(codes.vm, v_norm);
            for_each<NP>([&](auto jj) __attribute__((always_inline)) {
                constexpr int j = decltype(jj)::value;
                if constexpr (j + A < NP) fr[(j + A) % (A + 1)] = value_at(P, j + A);
                value(fr[j % (A + 1)], j);
                for_each<PIECES>([&](auto piece) __attribute__((always_inline)) {
                    constexpr int x = decltype(piece)::value;
                    if constexpr (2 * x * NP / (2 * PIECES) == j) store_keys(codes, piece, P);
                    if constexpr ((2 * x + 1) * NP / (2 * PIECES) == j) store_values(codes, piece, Q);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
            load_codes(codes, v + 4, v + 3, base, pages);
        };
        // tiles that every row of the workgroup sees whole: steps f0 .. f1 - 1 (but for absent blocks, and for bounded scores)
        const int tile0 = p.window > 0 && w.hi - p.window >= 0 ? (w.hi - p.window) / TOK + 1 : 0, tile1 = w.lo < 0 ? 0 : (w.lo + 1) / TOK;
        const int f0 = max(max(v0, w.span.first), w.span.first + tile0 - w.span.start);
        const int f1 = p.softcap > 0.0f || absent ? 0 : min(v1, w.span.first + tile1 - w.span.start);
        const float scale2 = row_scale * k_undo;

        for (int v = v0; v < v1;) {
            if (((v - v0) & 1) == 0 && v >= f0 && v + 2 < f1) {
                // Two tiles a round.  While the weights of a tile are made of its scores, the products that give the next tile's
                // run in the matrix cores; while its values are multiplied, the next maximum is looked for and codes
                // are dequantised.  A slice is one product and the vector instructions of about its time (the order is
                // pinned); operands are read slices ahead.
                float sa[NS], sb[NS], top;
                k_exp = scale2 * log2e;
                {
                    f32x16 acc[TB];
                    all_scores(acc, 0);
                    take(sa, acc);
                    top = sa[0];
#pragma unroll
                    for (int i = 1; i < NS; ++i) top = fmaxf(top, sa[i]);
                    __syncthreads();
                }
                auto fused = [&](auto parity, float (&s)[NS], float (&next)[NS], Codes &codes, int v) __attribute__((always_inline)) {
                    constexpr int P = decltype(parity)::value, Q = P ^ 1, QP = NS / 2 * 3 / 4, R = NS / 2 - QP, H = TB == 1 ? NP / 4 : NP / 2, M = NP / 2;
                    static_assert(H < NP - DT, "the last weights are packed before the slices that take them");
                    constexpr int A = q_in_lds ? 2 : 3;  // slices that operands are read ahead
                    begin(v);
                    settle(top);
                    __builtin_amdgcn_sched_barrier(0);
                    f32x16 acc[TB];
                    f16x8_t fr[A + 1], fq[A + 1];
#pragma unroll
                    for (int i = 0; i < A; ++i) {
                        fr[i] = key_at(Q, i);
                        fq[i] = query_at(i);
                    }
                    for_each<NQ>([&](auto ii) __attribute__((always_inline)) {
                        constexpr int i = decltype(ii)::value;
                        fr[(i + A) % (A + 1)] = i + A < NQ ? key_at(Q, i + A) : value_at(P, i + A - NQ);
                        if constexpr (i + A < NQ) fq[(i + A) % (A + 1)] = query_at(i + A);
                        score(acc, fr[i % (A + 1)], fq[i % (A + 1)], i);
#pragma unroll
                        for (int x = i * QP / NQ; x < (i + 1) * QP / NQ; ++x) exp_pair(s, x);
#pragma unroll
                        for (int x = i == 0 ? 0 : (i - 1) * QP / NQ; x < i * QP / NQ; ++x) pack_pair(s, x);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    take(next, acc);
                    for_each<NP>([&](auto jj) __attribute__((always_inline)) {
                        constexpr int j = decltype(jj)::value;
                        if constexpr (j == 0) {
#pragma unroll
                            for (int x = (NQ - 1) * QP / NQ; x < QP; ++x) pack_pair(s, x);
                        }
                        if constexpr (j + A < NP) fr[(NQ + j + A) % (A + 1)] = value_at(P, j + A);
                        value(fr[(NQ + j) % (A + 1)], j);
                        if constexpr (j < H) {
#pragma unroll
                            for (int x = QP + j * R / H; x < QP + (j + 1) * R / H; ++x) exp_pair(s, x);
                        }
                        if constexpr (j > 0 && j <= H) {
#pragma unroll
                            for (int x = QP + (j - 1) * R / H; x < QP + j * R / H; ++x) pack_pair(s, x);
                        }
                        if constexpr (j >= M) {
#pragma unroll
                            for (int x = (j - M) * NS / (NP - M); x < (j - M + 1) * NS / (NP - M); ++x) top = x == 0 ? next[0] : fmaxf(top, next[x]);
                            asm volatile("" : "+v"(top));
                        }
                        constexpr int S = NP / 4;  // (the first quarter is left to the codes' last delay)
                        if constexpr (j == S - 1) {
                            codes.km = converted(codes.km, k_norm);
                            codes.vm = converted(codes.vm, v_norm);
                        }
                        for_each<PIECES>([&](auto piece) __attribute__((always_inline)) {
                            constexpr int x = decltype(piece)::value;
                            if constexpr (S + 2 * x * (NP - S) / (2 * PIECES) == j) store_keys(codes, piece, P);
                            if constexpr (S + (2 * x + 1) * (NP - S) / (2 * PIECES) == j) store_values(codes, piece, Q);
                        });
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    load_codes(codes, v + 4, v + 3, base, pages);
                    __syncthreads();
                };
                do {
                    fused(std::integral_constant<int, 0>{}, sa, sb, ca, v);
                    fused(std::integral_constant<int, 1>{}, sb, sa, cb, v + 1);
                    v += 2;
                } while (v + 2 < f1);
                // the last one, whose scores are there
                begin(v);
                settle(top);
#pragma unroll
                for (int i = 0; i < NS / 2; ++i) exp_pair(sa, i);
#pragma unroll
                for (int i = 0; i < NS / 2; ++i) pack_pair(sa, i);
            } else {
                // any tile: bounded scores, hidden keys
                begin(v);
                const int t0 = w.span.tile(v) * TOK, par = (v - v0) & 1;
                const bool active = !idle && t0 <= whi && (p.window == 0 || t0 + TOK > wlo - p.window + 1 || t0 < p.sinks);
                if (active) {
                    f32x16 acc[TB];
                    all_scores(acc, par);
                    k_exp = scale2 * (p.softcap > 0.0f ? 1.0f : log2e);
                    float s[NS], top = kKvLowest;
                    take(s, acc);
                    if (p.softcap > 0.0f) {
#pragma unroll
                        for (int i = 0; i < NS; ++i) {
                            const float y = __builtin_amdgcn_exp2f(s[i] * (k_exp * cap_in)) + 1.0f;
                            s[i] = __builtin_fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(y), cap_out);
                        }
                        k_exp = 1.0f;
                    }
                    const int from = t0 + 4 * static_cast<int>(hh), below = pos - from, low = p.window > 0 ? below - p.window : -(1 << 30), first = p.sinks - from;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const int key = 8 * (i >> 2) + (i & 3);  // (after the lane's first)
                        s[i] = (key <= below) & ((key > low) | (key < first)) ? s[i] : kKvLowest;
                    }
                    if (absent) {
                        const uint32_t bad = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(pages < 0) >> ((v - base) * BLOCKS));
#pragma unroll
                        for (int i = 0; i < NS; ++i) s[i] = (bad >> (i >> 3)) & 1u ? kKvLowest : s[i];
                    }
#pragma unroll
                    for (int i = 0; i < NS; ++i) top = fmaxf(top, s[i]);
                    settle(top);
#pragma unroll
                    for (int i = 0; i < NS; ++i) s[i] = s[i] > kKvLowest ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], k_exp, -mx)) : 0.0f;
#pragma unroll
                    for (int i = 0; i < NS / 2; ++i) pack_pair(s, i);
                } else {
#pragma unroll
                    for (int i = 0; i < NS / 2; ++i) pw[i] = 0;
                }
                __syncthreads();  // (the keys' buffer is the next one's)
            }
            if ((v - v0) & 1) values_and_codes(std::integral_constant<int, 1>{}, cb, v);
            else values_and_codes(std::integral_constant<int, 0>{}, ca, v);
            __syncthreads();
            ++v;
        }
    }

    {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (row >= w.n_rows) return;
    if (w.live == 1) {
        uint8_t *dst = p.out + (w.row0 + qi) * p.ldOut + (h * p.R + row - qi * p.R) * (2 * D) + 8 * hh;
        const float inv = l > 0.0f ? v_undo / l : 0.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<uint2 *>(dst + 64 * t + 4 * e) =
                    make_uint2(pack_bf16x2(o[t][e] * inv, o[t][e + 1] * inv), pack_bf16x2(o[t][e + 2] * inv, o[t][e + 3] * inv));
    } else {
        const int64_t at = (h * static_cast<int64_t>(p.items) + w.item0 + split) * ROWS + (row - rt * ROWS);
        float *dst = p.part + at * D + 4 * hh;
        const float f = v_undo;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(dst + 32 * t + 2 * e) = f32x4{o[t][e] * f, o[t][e + 1] * f, o[t][e + 2] * f, o[t][e + 3] * f};
        if (hh == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(mx, l);
    }
}

// The shares of a row put together: D / 4 lanes a row, 8 shares' maxima, sums and accumulators in flight at a time (32 shares of
// 24 rows of 128: 7 us, most of it the way to the first load).  The grid has every row that the batch may have; those that were not cut
// return once their share is known.
template <int D, int TOK>
__global__ __launch_bounds__(256) void k_kv_join(KvArgs a, KvAttendArgs p, int rows)
{
    constexpr int LPR = D / 4, RPW = 256 / LPR;
    const int h = blockIdx.y, c = threadIdx.x % LPR, row = blockIdx.x * RPW + threadIdx.x / LPR;
    KvShare w;
    w.b = blockIdx.z;
    w.rt = p.by_rows.of(row);
    if (!kv_share<TOK>(a, p, rows, -1, w) || row >= w.n_rows || w.live == 1 || w.item0 + w.live > p.items) return;
    const int64_t at = (h * static_cast<int64_t>(p.items) + w.item0) * rows + (row - w.rt * rows);
    const float *part = p.part + at * D + 4 * c;
    const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml) + at;
    float mx = kKvLowest, l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int s = 0; s < w.live; s += 8) {
        float2 x[8];
        f32x4 y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t r = static_cast<int64_t>(min(s + u, w.live - 1)) * rows;
            x[u] = ml[r];
            y[u] = *reinterpret_cast<const f32x4 *>(part + r * D);
        }
        float now = mx;
#pragma unroll
        for (int u = 0; u < 8; ++u) now = fmaxf(now, x[u].x);
        const float f = __builtin_amdgcn_exp2f(mx - now);
        mx = now;
        l *= f;
        o *= f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float g = s + u < w.live ? __builtin_amdgcn_exp2f(x[u].x - now) : 0.0f;
            l += x[u].y * g;
            o += y[u] * g;
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const int i = p.by_R.of(row);
    uint8_t *dst = p.out + (w.row0 + i) * p.ldOut + (h * p.R + row - i * p.R) * (2 * D) + 8 * c;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

// ---- host -----------------------------------------------------------------------------------

static size_t plan_bytes(const KvArgs &a) { return a.n_seqs > 64 ? (4 * (static_cast<size_t>(a.n_seqs) + 2) + 15) / 16 * 16 : 0; }

size_t kv_attend_workspace_bytes(const KvArgs &a, int D, int R, int max_len)
{
    int cu;
    if (compute_units_of_current_device(&cu) != hipSuccess) return 0;
    return plan_bytes(a) + std::max<size_t>(choose(a, D, R, max_len, cu).partial_rows * (D + 2) * sizeof(float), 16);
}

template <int D>
static auto few_kernel(int ng, bool cols)
{
    if constexpr (D == 256) {
        if (ng == 8) return k_kv_attend_few<D, 8, true>;
        if (ng == 4) return k_kv_attend_few<D, 4, true>;
    }
    if constexpr (D == 128)
        if (ng == 4) return cols ? k_kv_attend_few<D, 4, true> : k_kv_attend_few<D, 4, false>;
    return ng == 1 ? k_kv_attend_few<D, 1, false> : cols ? k_kv_attend_few<D, 2, true> : k_kv_attend_few<D, 2, false>;
}

// Two tiles of keys and of values, heads of 256 their queries too: more than the default limit of LDS, allowed once per device.
template <int D, int NG, int W, int TOK>
static hipError_t launch_many(const KvArgs &a, const KvAttendArgs &p, dim3 grid, hipStream_t s)
{
    constexpr int bytes = 2 * 2 * TOK * 2 * D + (D == 256 ? 32 * W * 2 * D : 0);
    static std::atomic<uint64_t> allowed;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(k_kv_attend_many<D, NG, W, TOK>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    launch_kernel(k_kv_attend_many<D, NG, W, TOK>, grid, dim3(64 * W), bytes, s, a, p);
    return hipSuccess;
}

template <int D, int W, int TOK>
static hipError_t launch_many_of(const KvArgs &a, const KvAttendArgs &p, dim3 grid, hipStream_t s)
{
    switch (a.ng) {
    case 1: return launch_many<D, 1, W, TOK>(a, p, grid, s);
    case 2: return launch_many<D, 2, W, TOK>(a, p, grid, s);
    case 4: return launch_many<D, D >= 128 ? 4 : 2, W, TOK>(a, p, grid, s);
    default: return launch_many<D, D >= 256 ? 8 : 2, W, TOK>(a, p, grid, s);
    }
}

template <int D, int TOK>
static void launch_join(const KvArgs &a, const KvAttendArgs &p, const KvChoice &c, hipStream_t s)
{
    constexpr int per = 256 / (D / 4);
    const dim3 grid((std::min<int64_t>(a.max_new, a.rows) * p.R + per - 1) / per, a.heads, a.n_seqs);
    if (c.many) hipLaunchKernelGGL((k_kv_join<D, TOK>), grid, dim3(256), 0, s, a, p, c.rows);
    else hipLaunchKernelGGL((k_kv_join<D, kKvTile>), grid, dim3(256), 0, s, a, p, c.rows);
}

int launch_kv_attend(const KvArgs &a, KvAttendArgs p, int D, int max_len, void *workspace, hipStream_t s)
{
    int cu;
    hipError_t e = compute_units_of_current_device(&cu);
    if (e != hipSuccess) return hip_result(e);
    const KvChoice c = choose(a, D, p.R, reach_of(a, p, max_len), cu);
    take_choice(a, c, p);
    p.plan = static_cast<int32_t *>(workspace);
    p.part = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + plan_bytes(a));
    p.part_ml = p.part + static_cast<size_t>(a.heads) * c.items * c.rows * D;
    if (c.items * a.heads > kKvMaxItems) return TPQ_ERR_SHAPE;
    if (c.splits > 1 && static_cast<uint64_t>(c.items) * a.heads * c.rows > choose(a, D, p.R, max_len, cu).partial_rows) return TPQ_ERR_WORKSPACE;
    if (a.n_seqs > 64 && !kv_even(a, p)) {
        const auto plan = c.many && D <= 128 ? k_kv_plan<64> : k_kv_plan<32>;
        hipLaunchKernelGGL(plan, dim3(1), dim3(1024), 0, s, a, p, c.rows);
    }
    const dim3 grid(static_cast<uint32_t>(c.items) * a.heads);
    if (c.many) {
        e = D == 256 ? launch_many_of<256, 4, 32>(a, p, grid, s)
            : c.rows == 256 ? (D == 64 ? launch_many_of<64, 8, 64>(a, p, grid, s) : launch_many_of<128, 8, 64>(a, p, grid, s))
                            : (D == 64 ? launch_many_of<64, 4, 64>(a, p, grid, s) : launch_many_of<128, 4, 64>(a, p, grid, s));
        if (e != hipSuccess) return hip_result(e);
    } else {
        const auto kernel = D == 256 ? few_kernel<256>(a.ng, c.cols)
                            : (D == 64 ? few_kernel<64>(a.ng, c.cols) : few_kernel<128>(a.ng, c.cols));
        launch_kernel(kernel, grid, dim3(256), 0, s, a, p);
    }
    if (c.splits > 1) {
        if (D == 64) launch_join<64, 64>(a, p, c, s);
        else if (D == 128) launch_join<128, 64>(a, p, c, s);
        else launch_join<256, 32>(a, p, c, s);
    }
    return hip_result(hipGetLastError());
}

}  // namespace tpq
