// Attention over the 4-bit cache of keys and values.
//
//   s_j = scale * q . k_j,  out = sum_j exp(s_j) v_j / sum_j exp(s_j),  k_j, v_j = code * scale_j + zero_j per group
#include <algorithm>
#include <type_traits>
#include <utility>

#include "tpq_device.h"
#include "tpq_kv.h"

namespace tpq {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kKvTile = 32;            // tokens of a step of a wave
constexpr float kKvLowest = -3.0e38f;  // the running maximum before the first score

// The steps that rows at positions lo .. hi go through: the tiles that hold visible first tokens, then those from the first
// row's window to the last row's position.
struct KvSpan {
    int first, start, tiles;  // tiles of first tokens, first tile of the rest, all tiles
    __device__ __forceinline__ int tile(int v) const { return v < first ? v : start + (v - first); }
};
__device__ __forceinline__ KvSpan kv_span(const KvArgs &a, int window, int sinks, int lo, int hi, int len)
{
    const int end = min(min(hi + 1, len), a.ld_table << a.lg_page);
    KvSpan s = {0, 0, 0};
    if (end <= 0) return s;
    const int last = (end + kKvTile - 1) / kKvTile;
    if (window > 0) {
        s.start = max(lo - window + 1, 0) / kKvTile;
        s.first = min((min(sinks, end) + kKvTile - 1) / kKvTile, s.start);
    }
    s.tiles = s.first + max(last - s.start, 0);
    return s;
}
// Steps of one split of `splits`, and how many splits have any (at least one).
constexpr int kKvMinTiles = 4;
__device__ __forceinline__ int kv_share(int tiles, int splits) { return max((tiles + splits - 1) / splits, kKvMinTiles); }
__device__ __forceinline__ int kv_live(int tiles, int share) { return max((tiles + share - 1) / share, 1); }

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

// What a wave reads of a step's 32 tokens: lane (m, g) = (l % 16, l / 16).
template <int D, int NG>
struct KvRaw {
    static constexpr int KW = D / 32, VW = D == 256 ? 2 : 1;  // words: of a token's quarter of K codes; of a token's chunk of V codes
    uint32_t k[2][KW];       // tokens 16 j + m
    uint32_t v[2][4][VW];    // tokens 16 j + 4 g + i
    uint32_t meta[NG];       // lane 8 kv + 4 j + i of a row of 16: keys' (kv = 0) or values' scale and zero of token 16 j + 4 g + i
    bool bad[2];             // (uniform) a page that is none
};

template <int D, int NG, int NR>
__global__ __launch_bounds__(256, D * NR <= 128 && NG <= 2 ? 3 : 2) void k_kv_attend_few(KvArgs a, KvAttendArgs p)
{
    constexpr int KK = D / 32, NT = D / 16, KPG = KK / NG, TPG = NT / NG, ROWS = 16 * NR;
    typedef KvRaw<D, NG> Raw;
    __shared__ float sO[2][ROWS][D + 4];
    __shared__ float sM[2][ROWS], sL[2][ROWS];
    const CodePair code_pair;
    const uint32_t ln = threadIdx.x & 63u, m = ln & 15u, g = ln >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int split = blockIdx.x % p.splits, rt = blockIdx.x / p.splits, h = blockIdx.y, b = blockIdx.z;
    int64_t row0;
    int n, len;
    if (!kv_sequence(a, b, row0, n, len)) return;
    const int n_rows = min(n, a.max_new) * p.R;
    if (rt * ROWS >= n_rows) return;
    const int base = len - n;  // position of row 0's token
    const int lo = base + rt * ROWS / p.R, hi = base + (min((rt + 1) * ROWS, n_rows) - 1) / p.R;
    const KvSpan span = kv_span(a, p.window, p.sinks, lo, hi, len);
    const int share = kv_share(span.tiles, p.splits), live = kv_live(span.tiles, share);
    if (split >= live) return;
    const int v1 = min((split + 1) * share, span.tiles);

    // queries: column m of the products' right operand
    bf16x8_t q[NR][KK];
    float qs[NR][NG];
    int pos[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = rt * ROWS + 16 * r + static_cast<int>(m);
        const int rc = min(row, n_rows - 1), i = rc / p.R;
        pos[r] = base + i;
        const uint8_t *src = p.Q + (row0 + i) * p.ldQ + (h * p.R + rc - i * p.R) * (2 * D) + 16 * g;
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            float sum = 0.0f;
#pragma unroll
            for (int kk = gr * KPG; kk < (gr + 1) * KPG; ++kk) {
                u32x4 w = *reinterpret_cast<const u32x4 *>(src + 64 * kk);
                if (p.scale < 0.0f) w ^= 0x80008000u;  // (scores are then multiplied by |scale|: their order is the products')
                q[r][kk] = __builtin_bit_cast(bf16x8_t, w);
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += bf16_lo_to_f32(ws[e]) + bf16_hi_to_f32(ws[e]);
            }
            qs[r][gr] = group4_sum(sum);
        }
    }

    const int n_blocks = (min(len, a.ld_table << a.lg_page) + 15) / 16;  // blocks of 16 tokens that exist
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
        const uint8_t *meta = (m & 4u ? metas[1] : metas[0]) + (m & 8u ? 4 * NG * page_len : 0u) + 16 * g + 4 * (m & 3u);
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) raw.meta[gr] = *reinterpret_cast<const uint32_t *>(meta + 4 * (gr * page_len));
    };

    f32x4 o[NR][NT], oc[NR];  // accumulators; row gr of oc: 128 * (sum of group gr's weights as the products see them)
    float zs[NR][NG], mx[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        mx[r] = kKvLowest;
        l[r] = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[r][t] = f32x4{0, 0, 0, 0};
        oc[r] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) zs[r][gr] = 0.0f;
    }
    const float log2e = 1.44269504f;

    // scores in powers of two: exp(s) = 2^(s log2 e)
    const float k_score = p.softcap > 0.0f ? 1.0f : fabsf(p.scale) * log2e;
    const float cap_in = p.softcap > 0.0f ? fabsf(p.scale) / p.softcap * 2.0f * log2e : 0.0f, cap_out = p.softcap * log2e;

    auto step = [&](const Raw &raw, int v) {
        const int t0 = span.tile(v) * kKvTile;
        const bool whole = t0 + kKvTile - 1 <= lo && (p.window == 0 || t0 > hi - p.window || t0 + kKvTile <= p.sinks) && !raw.bad[0] && !raw.bad[1];
        float s[NR][2][4];
        bool vis[NR][2][4];
        for_each<2>([&](auto jj) {
            constexpr int J = decltype(jj)::value;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                f32x4 acc[NR];
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    float c0 = -128.0f * qs[r][gr];
                    asm volatile("" : "+v"(c0));  // (anew in every step: kept outside the loop it would take four registers)
                    acc[r] = f32x4{c0, c0, c0, c0};
                }
#pragma unroll
                for (int kk = gr * KPG; kk < (gr + 1) * KPG; ++kk) {
                    const uint32_t w = raw.k[J][kk];
                    const u32x4 c = {code_pair(w), code_pair(w >> 4), code_pair(w >> 8), code_pair(w >> 12)};
#pragma unroll
                    for (int r = 0; r < NR; ++r)
                        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, c), q[r][kk], acc[r], 0, 0, 0);
                }
                const float sc = bf16_lo_to_f32(raw.meta[gr]), ze = bf16_hi_to_f32(raw.meta[gr]);
                for_each<4>([&](auto i) {
                    constexpr int I = decltype(i)::value;
                    // (products, whose operand the exchange goes into; multiply-adds would take a move for each)
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        const float x = of_row<4 * J + I>(sc) * acc[r][I], z = of_row<4 * J + I>(ze) * qs[r][gr];
                        s[r][J][I] = gr == 0 ? x + z : (s[r][J][I] + x) + z;
                    }
                });
            }
        });
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if (p.softcap > 0.0f) {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    // cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1)
                    const float e = __builtin_amdgcn_exp2f(s[r][x >> 2][x & 3] * cap_in) + 1.0f;
                    s[r][x >> 2][x & 3] = __builtin_fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(e), cap_out);
                }
            }
            if (!whole) {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int j = x >> 2, i = x & 3, key = t0 + 16 * j + 4 * static_cast<int>(g) + i;
                    vis[r][j][i] = key <= pos[r] && (p.window == 0 || key > pos[r] - p.window || key < p.sinks) && !raw.bad[j] && key < 16 * n_blocks;
                    s[r][j][i] = vis[r][j][i] ? s[r][j][i] : kKvLowest;
                }
            }
            float top = s[r][0][0];
#pragma unroll
            for (int x = 1; x < 8; ++x) top = fmaxf(top, s[r][x >> 2][x & 3]);
            top *= k_score;
            // The maximum only follows where a weight would pass 2^8: weights are relative anyway, and a step without it saves
            // the accumulators' rescaling.
            if (__builtin_amdgcn_ballot_w64(top > mx[r] + 8.0f)) {
                const float now = fmaxf(mx[r], group4_max(top)), alpha = __builtin_amdgcn_exp2f(mx[r] - now);
                mx[r] = now;
                l[r] *= alpha;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[r][t] *= alpha;
                oc[r] *= alpha;
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) zs[r][gr] *= alpha;
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                float &e = s[r][x >> 2][x & 3];  // the weight, in the score's place
                e = __builtin_amdgcn_exp2f(__builtin_fmaf(e, k_score, -mx[r]));
                if (!whole) e = vis[r][x >> 2][x & 3] ? e : 0.0f;
                l[r] += e;
            }
        }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            bf16x8_t bh[NR], bl[NR];
            const float sc = bf16_lo_to_f32(raw.meta[gr]), ze = bf16_hi_to_f32(raw.meta[gr]);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                u32x4 ph, pl;
                for_each<2>([&](auto jj) {
                    constexpr int J = decltype(jj)::value;
                    float w[4];
                    for_each<4>([&](auto i) {
                        constexpr int I = decltype(i)::value;
                        w[I] = of_row<8 + 4 * J + I>(sc) * s[r][J][I];
                    });
                    if (whole) {
                        for_each<4>([&](auto i) {
                            constexpr int I = decltype(i)::value;
                            zs[r][gr] += of_row<8 + 4 * J + I>(ze) * s[r][J][I];
                        });
                    } else {  // (what lies behind a hidden key may be anything)
                        for_each<4>([&](auto i) {
                            constexpr int I = decltype(i)::value;
                            const float z = of_row<8 + 4 * J + I>(ze) * s[r][J][I];
                            zs[r][gr] += vis[r][J][I] ? z : 0.0f;
                            w[I] = vis[r][J][I] ? w[I] : 0.0f;
                        });
                    }
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const uint32_t hi2 = pack_bf16x2(w[i], w[i + 1]);
                        ph[2 * J + i / 2] = hi2;
                        pl[2 * J + i / 2] = pack_bf16x2(w[i] - bf16_lo_to_f32(hi2), w[i + 1] - bf16_hi_to_f32(hi2));
                    }
                });
                bh[r] = __builtin_bit_cast(bf16x8_t, ph);
                bl[r] = __builtin_bit_cast(bf16x8_t, pl);
            }
            uint32_t one = NG == 1 || m == static_cast<uint32_t>(gr) ? code_pair.base : 0u;
            if (NG > 1) asm volatile("" : "+v"(one));
            const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, (u32x4{one, one, one, one}));
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                oc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, bh[r], oc[r], 0, 0, 0);
                oc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, bl[r], oc[r], 0, 0, 0);
            }
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
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bh[r], o[r][t], 0, 0, 0);
                    o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bl[r], o[r][t], 0, 0, 0);
                }
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
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] = group4_sum(l[r]);
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            const float z = group4_sum(zs[r][gr]), c = NG == 1 ? oc[r][0] : __shfl(oc[r][gr & 3], 16 * (gr >> 2) + m, 64);
#pragma unroll
            for (int t = gr * TPG; t < (gr + 1) * TPG; ++t) o[r][t] = o[r][t] - c + z;
        }
    }
    // the four waves' results into wave 0's: 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (int from = 2; from >= 1; from >>= 1) {
        if (wave >= from && wave < 2 * from) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
#pragma unroll
                for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(&sO[wave - from][16 * r + m][16 * t + 4 * g]) = o[r][t];
                if (g == 0) {
                    sM[wave - from][16 * r + m] = mx[r];
                    sL[wave - from][16 * r + m] = l[r];
                }
            }
        }
        __syncthreads();
        if (wave < from) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const float m2 = sM[wave][16 * r + m], now = fmaxf(mx[r], m2);
                const float f1 = __builtin_amdgcn_exp2f(mx[r] - now), f2 = __builtin_amdgcn_exp2f(m2 - now);
                mx[r] = now;
                l[r] = l[r] * f1 + sL[wave][16 * r + m] * f2;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[r][t] = o[r][t] * f1 + *reinterpret_cast<const f32x4 *>(&sO[wave][16 * r + m][16 * t + 4 * g]) * f2;
            }
        }
        __syncthreads();
    }
    if (wave != 0) return;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = rt * ROWS + 16 * r + static_cast<int>(m);
        if (row >= n_rows) continue;
        if (live == 1) {
            const int i = row / p.R;
            uint8_t *dst = p.out + (row0 + i) * p.ldOut + (h * p.R + row - i * p.R) * (2 * D) + 8 * g;
            const float inv = l[r] > 0.0f ? 1.0f / l[r] : 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
                *reinterpret_cast<uint2 *>(dst + 32 * t) = make_uint2(pack_bf16x2(o[r][t][0] * inv, o[r][t][1] * inv), pack_bf16x2(o[r][t][2] * inv, o[r][t][3] * inv));
        } else {
            const int64_t at = (((static_cast<int64_t>(b) * a.heads + h) * p.row_tiles + rt) * p.splits + split) * ROWS + 16 * r + m;
            float *dst = p.part + at * D + 4 * g;
#pragma unroll
            for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(dst + 16 * t) = o[r][t];
            if (g == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(mx[r], l[r]);
        }
    }
}

// The splits' results into the output: a row of a head by D / 4 lanes.
template <int D>
__global__ __launch_bounds__(256) void k_kv_join(KvArgs a, KvAttendArgs p, int rows_per_tile)
{
    constexpr int LPR = D / 4, RPW = 256 / LPR;
    const int h = blockIdx.y, b = blockIdx.z, c = threadIdx.x % LPR;
    const int row = blockIdx.x * RPW + threadIdx.x / LPR;
    int64_t row0;
    int n, len;
    if (!kv_sequence(a, b, row0, n, len)) return;
    const int n_rows = min(n, a.max_new) * p.R;
    if (row >= n_rows) return;
    const int rt = row / rows_per_tile, base = len - n;
    const int lo = base + rt * rows_per_tile / p.R, hi = base + (min((rt + 1) * rows_per_tile, n_rows) - 1) / p.R;
    const KvSpan span = kv_span(a, p.window, p.sinks, lo, hi, len);
    const int live = kv_live(span.tiles, kv_share(span.tiles, p.splits));
    if (live == 1) return;
    const int64_t at = (((static_cast<int64_t>(b) * a.heads + h) * p.row_tiles + rt) * p.splits) * rows_per_tile + (row - rt * rows_per_tile);
    float mx = kKvLowest, l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int s = 0; s < live; ++s) {
        const int64_t r = at + static_cast<int64_t>(s) * rows_per_tile;
        const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * r);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(p.part + r * D + 4 * c);
        const float now = fmaxf(mx, ml.x), f1 = __builtin_amdgcn_exp2f(mx - now), f2 = __builtin_amdgcn_exp2f(ml.x - now);
        mx = now;
        l = l * f1 + ml.y * f2;
        o = o * f1 + x * f2;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const int i = row / p.R;
    uint8_t *dst = p.out + (row0 + i) * p.ldOut + (h * p.R + row - i * p.R) * (2 * D) + 8 * c;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

// ---- host -----------------------------------------------------------------------------------

struct KvChoice {
    int rows, row_tiles, splits;
};

static KvChoice choose(const KvArgs &a, int D, int R, int max_len, int compute_units)
{
    KvChoice c;
    c.rows = D <= 128 && a.ng == 1 && a.max_new * R > 16 ? 32 : 16;
    c.row_tiles = (a.max_new * R + c.rows - 1) / c.rows;
    const int64_t tiles = (max_len + kKvTile - 1) / kKvTile + 1, groups = static_cast<int64_t>(a.n_seqs) * a.heads * c.row_tiles;
    const int64_t want = (4ll * compute_units + groups - 1) / groups;
    c.splits = static_cast<int>(std::min<int64_t>(std::max<int64_t>(std::min(want, tiles / kKvMinTiles), 1), 256));
    return c;
}

size_t kv_attend_workspace_bytes(const KvArgs &a, int D, int R, int max_len)
{
    int cu;
    if (compute_units_of_current_device(&cu) != hipSuccess) return 0;
    const KvChoice c = choose(a, D, R, max_len, cu);
    if (c.splits == 1) return 16;
    return static_cast<size_t>(a.n_seqs) * a.heads * c.row_tiles * c.splits * c.rows * (D + 2) * sizeof(float);
}

template <int D>
static auto few_kernel(int ng)
{
    switch (ng) {
    case 1: return k_kv_attend_few<D, 1, 1>;
    case 2: return k_kv_attend_few<D, 2, 1>;
    case 4: return k_kv_attend_few<D, D >= 128 ? 4 : 2, 1>;
    default: return k_kv_attend_few<D, D >= 256 ? 8 : 2, 1>;
    }
}

int launch_kv_attend(const KvArgs &a, KvAttendArgs p, int D, int max_len, void *workspace, hipStream_t s)
{
    int cu;
    const hipError_t e = compute_units_of_current_device(&cu);
    if (e != hipSuccess) return hip_result(e);
    const KvChoice c = choose(a, D, p.R, max_len, cu);
    p.splits = c.splits;
    p.row_tiles = c.row_tiles;
    p.part = static_cast<float *>(workspace);
    p.part_ml = p.part + static_cast<size_t>(a.n_seqs) * a.heads * c.row_tiles * c.splits * c.rows * D;
    const auto kernel = D == 256 ? few_kernel<256>(a.ng)
                        : c.rows == 32 ? (D == 64 ? k_kv_attend_few<64, 1, 2> : k_kv_attend_few<128, 1, 2>)
                                       : (D == 64 ? few_kernel<64>(a.ng) : few_kernel<128>(a.ng));
    launch_kernel(kernel, dim3(static_cast<uint32_t>(c.splits) * c.row_tiles, a.heads, a.n_seqs), dim3(256), 0, s, a, p);
    if (c.splits > 1) {
        const int per = 256 / (D / 4);
        const auto join = D == 64 ? k_kv_join<64> : D == 128 ? k_kv_join<128> : k_kv_join<256>;
        hipLaunchKernelGGL(join, dim3((a.max_new * p.R + per - 1) / per, a.heads, a.n_seqs), dim3(256), 0, s, a, p, c.rows);
    }
    return hip_result(hipGetLastError());
}

}  // namespace tpq
