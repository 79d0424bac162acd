// Into the 4-bit cache of keys and values and out of it: the quantiser of tpq_encode (per row of a
// head and group of G features: zero = minimum, scale = bf16(range / 15), code = rint((x - zero) / scale)) behind
// the rotation by position, and its inverse.
//
// A unit is one head's row of one token: D / 8 lanes with 8 features (16 bytes) each, so that a group's range is a
// reduction over G / 8 lanes of the vector unit.  A token's keys, values and queries are its units side by side, whatever matrices they
// come from: one launch serves a step.  A workgroup takes 16 tokens (8 with heads of 256) of one or four columns of units: side by
// side in a page, their scales, 4 bytes a token, fill a line of one XCD's cache, where tokens of different XCDs would each write back
// theirs (a batch of 37 ragged prompts, 16 900 tokens, heads of 64: append and read 79 us by sequence and token, 66 so).
// Bound by memory: 295 MB there, 4.5 TB/s; small calls by the chain of loads arguments, starts, table, codes.
#include "tpq_device.h"
#include "tpq_kv.h"

namespace tpq {

// Range of each aligned run of 2^lg lanes (lg = 2 .. 5), in all of its lanes.
__device__ __forceinline__ void run_minmax(int lg, float &mn, float &mx)
{
    switch (lg) {
    case 2: group_minmax<4>(mn, mx); break;
    case 3: group_minmax<8>(mn, mx); break;
    case 4: group_minmax<16>(mn, mx); break;
    default: group_minmax<32>(mn, mx); break;
    }
}

// 4 bytes of 0..15 -> 4 nibbles
__device__ __forceinline__ uint32_t nibbles_of_bytes(uint32_t w)
{
    w = (w | (w >> 4)) & 0x00FF00FFu;
    return (w | (w >> 8)) & 0xFFFFu;
}

// The tokens of a wave's rows.  Lane l looks at sequence lo + l, lo found 64 sequences at a time: all of their starts and
// lengths are one load's latency, whatever the batch.
struct KvWindow {
    int lo, s0, s1, len;
};
__device__ __forceinline__ KvWindow kv_window(const KvArgs &a, int64_t first)
{
    const int lane = threadIdx.x & 63;
    KvWindow w = {0, 0, 0, 0};
    for (int count = a.n_seqs; count > 64;) {
        const int step = (count + 63) / 64, at = lane * step;
        const uint64_t before = __builtin_amdgcn_ballot_w64(at < count && a.starts[w.lo + min(at, count - 1)] <= first);
        const int nth = max(__builtin_popcountll(before), 1) - 1;
        w.lo += nth * step;
        count = min(step, count - nth * step);
    }
    const int at = min(w.lo + lane, a.n_seqs - 1);
    w.s0 = a.starts[at];
    w.s1 = a.starts[at + 1];
    w.len = a.lens[at];
    return w;
}

// A row's token: its sequence and its position; pos < 0: it is no sequence's.
struct KvToken {
    int b, pos;
};
// Of rows first .. first + N - 1 (first uniform): row first + r in the lanes with that r.
template <int N>
__device__ __forceinline__ KvToken kv_token(const KvArgs &a, KvWindow w, int64_t first, int r)
{
    KvToken t = {0, -1};
    const int lane = threadIdx.x & 63;
    for (;;) {
        const bool good = w.lo + lane < a.n_seqs && w.s0 >= 0 && w.s1 <= a.rows;
        const int base = min(max(w.len, 0), 1 << 30) - w.s1;  // a row's position less its number
        for (int k = 0; k < N;) {
            const uint64_t has = __builtin_amdgcn_ballot_w64(good & (w.s0 <= first + k) & (first + k < w.s1));
            if (!has) {
                ++k;
                continue;
            }
            const int l = __builtin_ctzll(has), s0 = __builtin_amdgcn_readlane(w.s0, l), to = __builtin_amdgcn_readlane(base, l);
            const int end = static_cast<int>(min(__builtin_amdgcn_readlane(w.s1, l) - first, static_cast<int64_t>(N)));
            const int row = static_cast<int>(first) + r;
            if (r >= k && r < end) {
                t.b = w.lo + l;
                t.pos = row - s0 < a.max_new ? to + row : -1;
            }
            k = end;
        }
        w.lo += 64;
        if (w.lo >= a.n_seqs || __builtin_amdgcn_readlane(w.s1, 63) >= first + N) return t;
        const int at = min(w.lo + lane, a.n_seqs - 1);
        w.s0 = a.starts[at];
        w.s1 = a.starts[at + 1];
        w.len = a.lens[at];
    }
}

// Cosines and sines of 8 features from f0 on at a position, halves: of the features f0 and f0 + rot / 2 are a pair of.
struct KvTurn {
    float c[8], s[8];
};
__device__ __forceinline__ KvTurn turn_of(const KvAppendArgs &p, int f0, int pos)
{
    KvTurn t = {};
    const int half = p.rot >> 1;
    if (p.pairs) {
        const int64_t at = static_cast<int64_t>(pos) * half + (f0 >> 1);
        const float4 c = *reinterpret_cast<const float4 *>(p.cosines + at), n = *reinterpret_cast<const float4 *>(p.sines + at);
        t.c[0] = c.x; t.c[1] = c.y; t.c[2] = c.z; t.c[3] = c.w;
        t.s[0] = n.x; t.s[1] = n.y; t.s[2] = n.z; t.s[3] = n.w;
        return t;
    }
    const int64_t at = static_cast<int64_t>(pos) * half + (f0 < half ? f0 : f0 - half);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const float4 c = reinterpret_cast<const float4 *>(p.cosines + at)[v], n = reinterpret_cast<const float4 *>(p.sines + at)[v];
        t.c[4 * v] = c.x; t.c[4 * v + 1] = c.y; t.c[4 * v + 2] = c.z; t.c[4 * v + 3] = c.w;
        t.s[4 * v] = n.x; t.s[4 * v + 1] = n.y; t.s[4 * v + 2] = n.z; t.s[4 * v + 3] = n.w;
    }
    return t;
}

// 8 features turned.  other: in halves mode, the 8 features rot / 2 away.
__device__ __forceinline__ void rotate8(const KvAppendArgs &p, const KvTurn &t, bool lower, u32x4 other, float (&x)[8])
{
    if (p.pairs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = x[2 * e] * t.c[e] - x[2 * e + 1] * t.s[e], z = x[2 * e + 1] * t.c[e] + x[2 * e] * t.s[e];
            x[2 * e] = round_via_bf16(y);
            x[2 * e + 1] = round_via_bf16(z);
        }
        return;
    }
    const uint32_t ws[4] = {other.x, other.y, other.z, other.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float o = e & 1 ? bf16_hi_to_f32(ws[e >> 1]) : bf16_lo_to_f32(ws[e >> 1]);
        const float y = o * t.s[e];
        x[e] = round_via_bf16(x[e] * t.c[e] + (lower ? -y : y));
    }
}

// A workgroup's units: T rows of tokens by P columns at a time, PASSES times the next P columns.
template <int D>
struct KvTile {
    static constexpr int LPU = D / 8, UPW = 256 / LPU, T = UPW < 16 ? UPW : 16, P = UPW / T, N = 64 / LPU;  // N: rows of a wave
};

template <int D, int PASSES>
__global__ __launch_bounds__(256) void k_kv_append(KvArgs a, KvAppendArgs p)
{
    typedef KvTile<D> Tile;
    constexpr int LPU = Tile::LPU;
    __shared__ uint32_t turned[256];  // a unit's row of value codes
    const int l = threadIdx.x % LPU, r = threadIdx.x / LPU % Tile::T;
    const int block = p.by_columns.of(blockIdx.x), column = (blockIdx.x - block * p.columns) * (Tile::P * PASSES) + threadIdx.x / (LPU * Tile::T);
    const int wave_row = __builtin_amdgcn_readfirstlane(r);
    const int64_t first = static_cast<int64_t>(block) * Tile::T + wave_row, t = min(static_cast<int64_t>(block) * Tile::T + r, a.rows - 1);
    // all loads that need no other's answer (first those that others wait for: answers come in order)
    KvWindow window = {};
    if (a.starts) window = kv_window(a, first);
    else window.len = a.lens[min(block * Tile::T + r, a.n_seqs - 1)];
    u32x4 w[PASSES];
#pragma unroll
    for (int x = 0; x < PASSES; ++x) {
        const int hh = min(column + x * Tile::P, p.units - 1);
        const bool is_q = hh >= 2 * a.heads, is_v = !is_q && hh >= a.heads;
        const int head = is_q ? hh - 2 * a.heads : is_v ? hh - a.heads : hh;
        const uint8_t *row = (is_q ? p.Q + t * p.ldQ : is_v ? p.V + t * p.ldV : p.K + t * p.ldK) + head * (2 * D);
        w[x] = *reinterpret_cast<const u32x4 *>(row + 16 * l);
    }
    KvToken token;
    if (a.starts) token = kv_token<Tile::N>(a, window, first, r - wave_row);
    else token = {min(block * Tile::T + r, a.n_seqs - 1), block * Tile::T + r < a.n_seqs ? min(window.len, 1 << 30) - 1 : -1};
    const int pos = token.pos;
    int slot;
    uint8_t *page = kv_cell(a, token.b, pos, slot);
    const bool turns = 8 * l < p.rot, there = page && !(p.rot > 0 && pos >= p.rot_rows);
    KvTurn turn = {};
    if (turns && there) turn = turn_of(p, 8 * l, pos);
    const int half = p.rot >> 1;
    const bool lower = 8 * l < half;
    const int partner = (threadIdx.x & 63) + (turns ? (lower ? half : -half) / 8 : 0);
#pragma unroll
    for (int x = 0; x < PASSES; ++x) {
        const int hh = column + x * Tile::P;
        const bool is_q = hh >= 2 * a.heads, is_v = !is_q && hh >= a.heads;
        const int head = is_q ? hh - 2 * a.heads : is_v ? hh - a.heads : hh;
        u32x4 other = w[x];
        if (p.rot > 0 && !p.pairs) {  // (every lane of the wave)
            other.x = __shfl(w[x].x, partner, 64);
            other.y = __shfl(w[x].y, partner, 64);
            other.z = __shfl(w[x].z, partner, 64);
            other.w = __shfl(w[x].w, partner, 64);
        }
        if (!there || hh >= p.units) continue;
        float x8[8] = {bf16_lo_to_f32(w[x].x), bf16_hi_to_f32(w[x].x), bf16_lo_to_f32(w[x].y), bf16_hi_to_f32(w[x].y),
                       bf16_lo_to_f32(w[x].z), bf16_hi_to_f32(w[x].z), bf16_lo_to_f32(w[x].w), bf16_hi_to_f32(w[x].w)};
        if (!is_v && turns) rotate8(p, turn, lower, other, x8);
        if (is_q) {
            const u32x4 o = {pack_bf16x2(x8[0], x8[1]), pack_bf16x2(x8[2], x8[3]), pack_bf16x2(x8[4], x8[5]), pack_bf16x2(x8[6], x8[7])};
            *reinterpret_cast<u32x4 *>(p.Q_out + t * p.ldQo + head * (2 * D) + 16 * l) = o;
            continue;
        }

        float mn = x8[0], mx = x8[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            mn = fminf(mn, x8[e]);
            mx = fmaxf(mx, x8[e]);
        }
        const int lg_run = a.lg_group - 3;
        run_minmax(lg_run, mn, mx);
        mn = mn + 0.0f;
        const float s32 = div_by_15(mx - mn);
        const uint32_t sb = pack_bf16x2(s32, s32) & 0xFFFFu;
        const float s = bf16_bits_to_f32(sb);
        const bool constant = s < 1e-30f;
        const float inv = constant ? 0.0f : reciprocal_of_scale(s);
        uint32_t even = 0, odd = 0;  // features 0, 2, 4, 6 and 1, 3, 5, 7, a byte each
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float df = x8[e] - mn;
            const float q = df * inv;
            if (e & 1) odd = __builtin_amdgcn_cvt_pk_u8_f32(q, e >> 1, odd);
            else even = __builtin_amdgcn_cvt_pk_u8_f32(q, e >> 1, even);
        }
        uint8_t *cell = page + static_cast<int64_t>(head) * a.cell_bytes;
        const uint32_t page_len = 1u << a.lg_page;
        uint8_t *codes = cell + (is_v ? page_len * (D / 2) : 0u) + slot * (D / 2);
        if (!is_v) {
            *reinterpret_cast<uint32_t *>(codes + 4 * ((l & 3) * (D / 32) + (l >> 2))) = nibbles_of_bytes(even) | (nibbles_of_bytes(odd) << 16);
        } else {
            // feature 16 n + m in nibble n of chunk m: lane l has m = 8 (l & 1) + 0..7 of n = l / 2, lane l ^ 2 the
            // other nibble of the same bytes; the lane of even n puts together features 0, 2, 4, 6, the other one 1, 3, 5, 7
            const uint32_t oe = __float_as_uint(dpp_f32<0x4E>(__uint_as_float(even))), oo = __float_as_uint(dpp_f32<0x4E>(__uint_as_float(odd)));
            const bool second = l & 2;
            const uint32_t both = second ? oo | (odd << 4) : even | (oe << 4);
            uint8_t *mine = reinterpret_cast<uint8_t *>(turned + threadIdx.x - l);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                mine[(8 * (l & 1) + 2 * t + (second ? 1 : 0)) * (D / 32) + (l >> 2)] = static_cast<uint8_t>(both >> (8 * t));
            wave_lds_fence();
            *reinterpret_cast<uint32_t *>(codes + 4 * l) = turned[threadIdx.x];
            wave_lds_fence();  // (before the next pass's)
        }
        if ((l & ((1 << lg_run) - 1)) == 0) {
            uint32_t *meta = reinterpret_cast<uint32_t *>(cell + page_len * D) + (is_v ? a.ng << a.lg_page : 0);
            meta[((l >> lg_run) << a.lg_page) + slot] = (constant ? 0u : sb) | (__float_as_uint(mn) & 0xFFFF0000u);
        }
    }
}

template <int D, int PASSES>
__global__ __launch_bounds__(256) void k_kv_read(KvArgs a, KvReadArgs p)
{
    typedef KvTile<D> Tile;
    constexpr int LPU = Tile::LPU;
    __shared__ uint32_t turned[256];
    const int l = threadIdx.x % LPU, r = threadIdx.x / LPU % Tile::T;
    const int block = p.by_columns.of(blockIdx.x), column = (blockIdx.x - block * p.columns) * (Tile::P * PASSES) + threadIdx.x / (LPU * Tile::T);
    const int wave_row = __builtin_amdgcn_readfirstlane(r);
    const int64_t t = static_cast<int64_t>(block) * Tile::T + r;
    const int64_t first = static_cast<int64_t>(block) * Tile::T + wave_row;
    KvWindow window = {};
    if (a.starts) window = kv_window(a, first);
    else window.len = a.lens[min(block * Tile::T + r, a.n_seqs - 1)];
    KvToken token;
    if (a.starts) token = kv_token<Tile::N>(a, window, first, r - wave_row);
    else token = {min(block * Tile::T + r, a.n_seqs - 1), block * Tile::T + r < a.n_seqs ? min(window.len, 1 << 30) - 1 : -1};
    int slot;
    const uint8_t *page = kv_cell(a, token.b, token.pos, slot);
    if (!page) return;
    const uint32_t page_len = 1u << a.lg_page;
    const uint32_t meta_at = (((8 * l) >> a.lg_group) << a.lg_page) + slot;
    uint32_t w[PASSES], meta[PASSES];
#pragma unroll
    for (int x = 0; x < PASSES; ++x) {
        const int hh = p.first + min(column + x * Tile::P, p.units - 1);
        const bool is_v = hh >= a.heads;
        const uint8_t *cell = page + static_cast<int64_t>(is_v ? hh - a.heads : hh) * a.cell_bytes;
        const uint8_t *codes = cell + (is_v ? page_len * (D / 2) : 0u) + slot * (D / 2);
        w[x] = *reinterpret_cast<const uint32_t *>(codes + 4 * (is_v ? l : (l & 3) * (D / 32) + (l >> 2)));
        meta[x] = reinterpret_cast<const uint32_t *>(cell + page_len * D)[(is_v ? a.ng << a.lg_page : 0) + meta_at];
    }
#pragma unroll
    for (int x = 0; x < PASSES; ++x) {
        if (column + x * Tile::P >= p.units) break;
        const int hh = p.first + column + x * Tile::P;
        const bool is_v = hh >= a.heads;
        const int head = is_v ? hh - a.heads : hh;
        const float scale = bf16_lo_to_f32(meta[x]), zero = bf16_hi_to_f32(meta[x]);
        float v[8];
        if (!is_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = static_cast<float>((w[x] >> (4 * e)) & 15u) * scale + zero;
                v[2 * e + 1] = static_cast<float>((w[x] >> (16 + 4 * e)) & 15u) * scale + zero;
            }
        } else {
            turned[threadIdx.x] = w[x];
            wave_lds_fence();
            const uint8_t *mine = reinterpret_cast<const uint8_t *>(turned + threadIdx.x - l);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = static_cast<float>((mine[(8 * (l & 1) + e) * (D / 32) + (l >> 2)] >> (2 * (l & 2))) & 15u) * scale + zero;
            wave_lds_fence();  // (before the next pass's)
        }
        uint8_t *out = (is_v ? p.V + t * p.ldV : p.K + t * p.ldK) + (head * D + 8 * l) * (p.fp32 ? 4 : 2);
        if (p.fp32) {
            reinterpret_cast<float4 *>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            const u32x4 o = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
            *reinterpret_cast<u32x4 *>(out) = o;
        }
    }
}

// Blocks of T rows, each with its columns of units side by side; 0: too many for a launch.
template <int D>
static uint32_t tile_grid(const KvArgs &a, int columns)
{
    const int64_t blocks = (a.rows + KvTile<D>::T - 1) / KvTile<D>::T * columns;
    return blocks < (1ll << 32) / 256 ? static_cast<uint32_t>(blocks) : 0u;
}

template <int D, int PASSES>
static int append_in(const KvArgs &a, KvAppendArgs p, hipStream_t s)
{
    p.columns = (p.units + KvTile<D>::P * PASSES - 1) / (KvTile<D>::P * PASSES);
    p.by_columns = KvDivisor(p.columns);
    const uint32_t grid = tile_grid<D>(a, p.columns);
    if (grid == 0) return TPQ_ERR_SHAPE;
    launch_kernel(k_kv_append<D, PASSES>, dim3(grid), dim3(256), 0, s, a, p);
    return hip_result(hipGetLastError());
}

template <int D, int PASSES>
static int read_in(const KvArgs &a, KvReadArgs p, hipStream_t s)
{
    p.columns = (p.units + KvTile<D>::P * PASSES - 1) / (KvTile<D>::P * PASSES);
    p.by_columns = KvDivisor(p.columns);
    const uint32_t grid = tile_grid<D>(a, p.columns);
    if (grid == 0) return TPQ_ERR_SHAPE;
    launch_kernel(k_kv_read<D, PASSES>, dim3(grid), dim3(256), 0, s, a, p);
    return hip_result(hipGetLastError());
}

// Four units a lane, where that leaves four workgroups for each compute unit: their loads wait together, and a row's sequence is
// looked up once (4 x 4096 tokens, 32 + 16 heads of 128, append and read: 93 us, with one unit 123; 2048 tokens, 5 + 10 heads: 13.3 and 12.3).
template <int D>
static bool in_passes(const KvArgs &a, int units)
{
    int cu;
    if (compute_units_of_current_device(&cu) != hipSuccess) return false;
    return (a.rows + KvTile<D>::T - 1) / KvTile<D>::T * ((units + KvTile<D>::P * 4 - 1) / (KvTile<D>::P * 4)) >= 4ll * cu;
}

int launch_kv_append(const KvArgs &a, const KvAppendArgs &p, int D, hipStream_t s)
{
    if (D == 64) return in_passes<64>(a, p.units) ? append_in<64, 4>(a, p, s) : append_in<64, 1>(a, p, s);
    if (D == 128) return in_passes<128>(a, p.units) ? append_in<128, 4>(a, p, s) : append_in<128, 1>(a, p, s);
    return in_passes<256>(a, p.units) ? append_in<256, 4>(a, p, s) : append_in<256, 1>(a, p, s);
}

int launch_kv_read(const KvArgs &a, const KvReadArgs &p, int D, hipStream_t s)
{
    if (D == 64) return in_passes<64>(a, p.units) ? read_in<64, 4>(a, p, s) : read_in<64, 1>(a, p, s);
    if (D == 128) return in_passes<128>(a, p.units) ? read_in<128, 4>(a, p, s) : read_in<128, 1>(a, p, s);
    return in_passes<256>(a, p.units) ? read_in<256, 4>(a, p, s) : read_in<256, 1>(a, p, s);
}

}  // namespace tpq
