// Attention over the 4-bit cache of keys and values.
//
//   s_j = scale * q . k_j,  out = sum_j exp(s_j) v_j / sum_j exp(s_j),  k_j, v_j = code * scale_j + zero_j per group
#include <algorithm>

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

__device__ __forceinline__ float group4_max(float v)  // over lanes l, l ^ 16, l ^ 32, l ^ 48
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float group4_sum(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// codes of a dword -> 128 + code in bf16 (8 bits of significand: exact), nibbles t and 4 + t a pair
__device__ __forceinline__ uint32_t code_pair(uint32_t w) { return (w & 0x000F000Fu) | 0x43004300u; }

// What a wave reads of a step's 32 tokens: lane (m, g) = (l % 16, l / 16).
template <int D, int NG>
struct KvRaw {
    static constexpr int KW = D / 32, VW = D == 256 ? 2 : 1;  // words: of a token's quarter of K codes; of a token's chunk of V codes
    uint32_t k[2][KW];       // tokens 16 j + m
    uint32_t v[2][4][VW];    // tokens 16 j + 4 g + i
    u32x4 km[2][NG], vm[2][NG];
    bool bad[2];             // (uniform) a page that is none
};

template <int D, int NG, int NR>
__global__ __launch_bounds__(256) void k_kv_attend_few(KvArgs a, KvAttendArgs p)
{
    constexpr int KK = D / 32, NT = D / 16, KPG = KK / NG, TPG = NT / NG, ROWS = 16 * NR;
    typedef KvRaw<D, NG> Raw;
    __shared__ float sO[2][ROWS][D + 4];
    __shared__ float sM[2][ROWS], sL[2][ROWS];
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
                const u32x4 w = *reinterpret_cast<const u32x4 *>(src + 64 * kk);
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
    auto load = [&](Raw &raw, int tile) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int block = min(2 * tile + j, n_blocks - 1);
            const uint32_t slot = (16u * block) & page_mask;
            const int id = table[(16 * block) >> a.lg_page];
            raw.bad[j] = static_cast<uint32_t>(id) >= static_cast<uint64_t>(a.n_pages);
            const uint8_t *cell = a.cache + (raw.bad[j] ? 0 : id) * a.page_bytes + static_cast<int64_t>(h) * a.cell_bytes;
            const uint8_t *k = cell + (slot + m) * (D / 2) + g * (D / 8);
#pragma unroll
            for (int w = 0; w < Raw::KW; ++w) raw.k[j][w] = reinterpret_cast<const uint32_t *>(k)[w];
            const uint8_t *v = cell + page_len * (D / 2) + (slot + 4 * g) * (D / 2) + (D == 64 ? m / 2 * 4 : m * (D / 32));
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < Raw::VW; ++w) raw.v[j][i][w] = reinterpret_cast<const uint32_t *>(v + i * (D / 2))[w];
            const uint8_t *meta = cell + page_len * D + 4 * (slot + 4 * g);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                raw.km[j][gr] = *reinterpret_cast<const u32x4 *>(meta + 4 * (gr * page_len));
                raw.vm[j][gr] = *reinterpret_cast<const u32x4 *>(meta + 4 * ((NG + gr) * page_len));
            }
        }
    };

    f32x4 o[NR][NT], oc[NR][NG];
    float zs[NR][NG], mx[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        mx[r] = kKvLowest;
        l[r] = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[r][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            oc[r][gr] = f32x4{0, 0, 0, 0};
            zs[r][gr] = 0.0f;
        }
    }
    const float log2e = 1.44269504f;
    const u32x4 c128 = {0x43004300u, 0x43004300u, 0x43004300u, 0x43004300u};

    for (int v = split * share + wave; v < v1; v += 4) {
        Raw raw;
        const int tile = span.tile(v), t0 = tile * kKvTile;
        load(raw, tile);
        const bool whole = t0 + kKvTile - 1 <= lo && (p.window == 0 || t0 > hi - p.window || t0 + kKvTile <= p.sinks) && !raw.bad[0] && !raw.bad[1];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float s[2][4];
            bool vis[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][i] = 0.0f;
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    const float c0 = -128.0f * qs[r][gr];
                    f32x4 acc = {c0, c0, c0, c0};
#pragma unroll
                    for (int kk = gr * KPG; kk < (gr + 1) * KPG; ++kk) {
                        const uint32_t w = raw.k[j][kk];
                        const u32x4 c = {code_pair(w), code_pair(w >> 4), code_pair(w >> 8), code_pair(w >> 12)};
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, c), q[r][kk], acc, 0, 0, 0);
                    }
                    const uint32_t meta[4] = {raw.km[j][gr].x, raw.km[j][gr].y, raw.km[j][gr].z, raw.km[j][gr].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[j][i] = __builtin_fmaf(bf16_lo_to_f32(meta[i]), acc[i], __builtin_fmaf(bf16_hi_to_f32(meta[i]), qs[r][gr], s[j][i]));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (p.softcap > 0.0f) {
                        // cap * tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1)
                        const float e = __builtin_amdgcn_exp2f(s[j][i] * (p.scale / p.softcap * 2.0f * log2e));
                        s[j][i] = (p.softcap - 2.0f * p.softcap / (e + 1.0f)) * log2e;
                    } else {
                        s[j][i] *= p.scale * log2e;
                    }
                    vis[j][i] = true;
                    if (!whole) {
                        const int key = t0 + 16 * j + 4 * static_cast<int>(g) + i;
                        vis[j][i] = key <= pos[r] && (p.window == 0 || key > pos[r] - p.window || key < p.sinks) && !raw.bad[j] &&
                                    key < 16 * n_blocks;
                        s[j][i] = vis[j][i] ? s[j][i] : kKvLowest;
                    }
                }
            }
            float top = s[0][0];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[j][i]);
            const float now = fmaxf(mx[r], group4_max(top)), alpha = __builtin_amdgcn_exp2f(mx[r] - now);
            mx[r] = now;
            l[r] *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[r][t] *= alpha;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                oc[r][gr] *= alpha;
                zs[r][gr] *= alpha;
            }
            float e[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[j][i] = __builtin_amdgcn_exp2f(s[j][i] - now);
                    e[j][i] = vis[j][i] ? e[j][i] : 0.0f;
                    l[r] += e[j][i];
                }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                u32x4 ph, pl;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t meta[4] = {raw.vm[j][gr].x, raw.vm[j][gr].y, raw.vm[j][gr].z, raw.vm[j][gr].w};
                    float w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t mt = vis[j][i] ? meta[i] : 0u;  // (what lies behind a hidden key may be anything)
                        w[i] = e[j][i] * bf16_lo_to_f32(mt);
                        zs[r][gr] = __builtin_fmaf(e[j][i], bf16_hi_to_f32(mt), zs[r][gr]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const uint32_t hi2 = pack_bf16x2(w[i], w[i + 1]);
                        ph[2 * j + i / 2] = hi2;
                        pl[2 * j + i / 2] = pack_bf16x2(w[i] - bf16_lo_to_f32(hi2), w[i + 1] - bf16_hi_to_f32(hi2));
                    }
                }
                const bf16x8_t bh = __builtin_bit_cast(bf16x8_t, ph), bl = __builtin_bit_cast(bf16x8_t, pl);
                const bf16x8_t ac = __builtin_bit_cast(bf16x8_t, c128);
                oc[r][gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ac, bh, oc[r][gr], 0, 0, 0);
                oc[r][gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ac, bl, oc[r][gr], 0, 0, 0);
#pragma unroll
                for (int t = gr * TPG; t < (gr + 1) * TPG; ++t) {
                    const int word = t / 8, byte = (t % 8) / 2;
                    const uint32_t at = D == 64 ? byte + 2 * (m & 1u) : byte;
                    const uint32_t sel = 0x0C000C00u | ((4u + at) << 16) | at;
                    u32x4 c;
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const uint32_t x = __builtin_amdgcn_perm(raw.v[j][i + 1][word], raw.v[j][i][word], sel);
                            c[2 * j + i / 2] = code_pair(t & 1 ? x >> 4 : x);
                        }
                    const bf16x8_t av = __builtin_bit_cast(bf16x8_t, c);
                    o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bh, o[r][t], 0, 0, 0);
                    o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bl, o[r][t], 0, 0, 0);
                }
            }
        }
    }

    // 128 * (sum of the weights) off the codes, the zeros' share on
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] = group4_sum(l[r]);
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            const float z = group4_sum(zs[r][gr]);
#pragma unroll
            for (int t = gr * TPG; t < (gr + 1) * TPG; ++t) o[r][t] = o[r][t] - oc[r][gr] + z;
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

static KvChoice choose(const KvArgs &a, int R, int max_len, int compute_units)
{
    KvChoice c;
    c.rows = 16;
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
    const KvChoice c = choose(a, R, max_len, cu);
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
    const KvChoice c = choose(a, p.R, max_len, cu);
    p.splits = c.splits;
    p.row_tiles = c.row_tiles;
    p.part = static_cast<float *>(workspace);
    p.part_ml = p.part + static_cast<size_t>(a.n_seqs) * a.heads * c.row_tiles * c.splits * c.rows * D;
    const auto kernel = D == 64 ? few_kernel<64>(a.ng) : D == 128 ? few_kernel<128>(a.ng) : few_kernel<256>(a.ng);
    launch_kernel(kernel, dim3(static_cast<uint32_t>(c.splits) * c.row_tiles, a.heads, a.n_seqs), dim3(256), 0, s, a, p);
    if (c.splits > 1) {
        const int per = 256 / (D / 4);
        const auto join = D == 64 ? k_kv_join<64> : D == 128 ? k_kv_join<128> : k_kv_join<256>;
        hipLaunchKernelGGL(join, dim3((a.max_new * p.R + per - 1) / per, a.heads, a.n_seqs), dim3(256), 0, s, a, p, c.rows);
    }
    return hip_result(hipGetLastError());
}

}  // namespace tpq
