// Into the 4-bit cache of keys and values and out of it: the quantiser of tpq_encode (per row of a
// head and group of G features: zero = minimum, scale = bf16(range / 15), code = rint((x - zero) / scale)) behind
// the rotation by position, and its inverse.
//
// A unit is one head's row of one token: D / 8 lanes with 8 features (16 bytes) each, so that a group's range is a
// reduction over G / 8 lanes of the vector unit.  A token's keys, values and queries are its units side by side, whatever matrices they
// come from: one launch serves a step.
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

// 8 features turned by their position.  x: the lane's features from f0 on, bf16 bits in pairs; partner in halves
// mode: the 8 features rot / 2 away.
__device__ __forceinline__ void rotate8(const KvAppendArgs &p, const uint8_t *row, int f0, int pos, float (&x)[8])
{
    const int half = p.rot >> 1;
    if (p.pairs) {
        const int64_t at = static_cast<int64_t>(pos) * half + (f0 >> 1);
        const float4 c = *reinterpret_cast<const float4 *>(p.cosines + at), n = *reinterpret_cast<const float4 *>(p.sines + at);
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float y = x[2 * t] * cs[t] - x[2 * t + 1] * sn[t], z = x[2 * t + 1] * cs[t] + x[2 * t] * sn[t];
            x[2 * t] = round_via_bf16(y);
            x[2 * t + 1] = round_via_bf16(z);
        }
        return;
    }
    const bool lower = f0 < half;
    const int p0 = lower ? f0 : f0 - half;
    const u32x4 w = *reinterpret_cast<const u32x4 *>(row + 2 * (lower ? f0 + half : p0));
    const int64_t at = static_cast<int64_t>(pos) * half + p0;
    float cs[8], sn[8];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const float4 c = reinterpret_cast<const float4 *>(p.cosines + at)[v], n = reinterpret_cast<const float4 *>(p.sines + at)[v];
        cs[4 * v] = c.x; cs[4 * v + 1] = c.y; cs[4 * v + 2] = c.z; cs[4 * v + 3] = c.w;
        sn[4 * v] = n.x; sn[4 * v + 1] = n.y; sn[4 * v + 2] = n.z; sn[4 * v + 3] = n.w;
    }
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float o = e & 1 ? bf16_hi_to_f32(ws[e >> 1]) : bf16_lo_to_f32(ws[e >> 1]);
        const float t = o * sn[e];
        x[e] = round_via_bf16(x[e] * cs[e] + (lower ? -t : t));
    }
}

template <int D>
__global__ __launch_bounds__(256) void k_kv_append(KvArgs a, KvAppendArgs p)
{
    constexpr int LPU = D / 8, UPW = 256 / LPU;  // lanes of a unit, units of a workgroup
    __shared__ uint32_t turned[256];             // a unit's row of value codes
    const int b = blockIdx.y, l = threadIdx.x % LPU;
    const uint32_t u = blockIdx.x * UPW + threadIdx.x / LPU;
    const int i = u / p.units, hh = u - i * p.units;
    int64_t row0;
    int n, len, slot;
    if (!kv_sequence(a, b, row0, n, len) || i >= min(n, a.max_new)) return;
    const int pos = len - n + i;
    uint8_t *page = kv_cell(a, b, pos, slot);
    if (!page || (p.rot > 0 && pos >= p.rot_rows)) return;

    const bool is_q = hh >= 2 * a.heads, is_v = !is_q && hh >= a.heads;
    const int head = is_q ? hh - 2 * a.heads : is_v ? hh - a.heads : hh;
    const uint8_t *row = (is_q ? p.Q + (row0 + i) * p.ldQ : is_v ? p.V + (row0 + i) * p.ldV : p.K + (row0 + i) * p.ldK) + head * (2 * D);
    const u32x4 w = *reinterpret_cast<const u32x4 *>(row + 16 * l);
    float x[8] = {bf16_lo_to_f32(w.x), bf16_hi_to_f32(w.x), bf16_lo_to_f32(w.y), bf16_hi_to_f32(w.y),
                  bf16_lo_to_f32(w.z), bf16_hi_to_f32(w.z), bf16_lo_to_f32(w.w), bf16_hi_to_f32(w.w)};
    if (!is_v && 8 * l < p.rot) rotate8(p, row, 8 * l, pos, x);
    if (is_q) {
        const u32x4 o = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        *reinterpret_cast<u32x4 *>(p.Q_out + (row0 + i) * p.ldQo + head * (2 * D) + 16 * l) = o;
        return;
    }

    float mn = x[0], mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        mn = fminf(mn, x[e]);
        mx = fmaxf(mx, x[e]);
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
        const float df = x[e] - mn;
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
    }
    if ((l & ((1 << lg_run) - 1)) == 0) {
        uint32_t *meta = reinterpret_cast<uint32_t *>(cell + page_len * D) + (is_v ? a.ng << a.lg_page : 0);
        meta[((l >> lg_run) << a.lg_page) + slot] = (constant ? 0u : sb) | (__float_as_uint(mn) & 0xFFFF0000u);
    }
}

template <int D>
__global__ __launch_bounds__(256) void k_kv_read(KvArgs a, KvReadArgs p)
{
    constexpr int LPU = D / 8, UPW = 256 / LPU;
    __shared__ uint32_t turned[256];
    const int b = blockIdx.y, l = threadIdx.x % LPU;
    const uint32_t u = blockIdx.x * UPW + threadIdx.x / LPU;
    const int i = u / p.units, hh = p.first + (u - i * p.units);
    int64_t row0;
    int n, len, slot;
    if (!kv_sequence(a, b, row0, n, len) || i >= min(n, a.max_new)) return;
    const uint8_t *page = kv_cell(a, b, len - n + i, slot);
    if (!page) return;
    const bool is_v = hh >= a.heads;
    const int head = is_v ? hh - a.heads : hh;
    const uint32_t page_len = 1u << a.lg_page;
    const uint8_t *cell = page + static_cast<int64_t>(head) * a.cell_bytes;
    const uint8_t *codes = cell + (is_v ? page_len * (D / 2) : 0u) + slot * (D / 2);
    const uint32_t meta = reinterpret_cast<const uint32_t *>(cell + page_len * D)[(is_v ? a.ng << a.lg_page : 0) + (((8 * l) >> a.lg_group) << a.lg_page) + slot];
    const float scale = bf16_lo_to_f32(meta), zero = bf16_hi_to_f32(meta);
    float x[8];
    if (!is_v) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + 4 * ((l & 3) * (D / 32) + (l >> 2)));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[2 * t] = static_cast<float>((w >> (4 * t)) & 15u) * scale + zero;
            x[2 * t + 1] = static_cast<float>((w >> (16 + 4 * t)) & 15u) * scale + zero;
        }
    } else {
        turned[threadIdx.x] = *reinterpret_cast<const uint32_t *>(codes + 4 * l);
        wave_lds_fence();
        const uint8_t *mine = reinterpret_cast<const uint8_t *>(turned + threadIdx.x - l);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = static_cast<float>((mine[(8 * (l & 1) + e) * (D / 32) + (l >> 2)] >> (2 * (l & 2))) & 15u) * scale + zero;
    }
    uint8_t *out = (is_v ? p.V + (row0 + i) * p.ldV : p.K + (row0 + i) * p.ldK) + (head * D + 8 * l) * (p.fp32 ? 4 : 2);
    if (p.fp32) {
        reinterpret_cast<float4 *>(out)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(out)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        const u32x4 o = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        *reinterpret_cast<u32x4 *>(out) = o;
    }
}

static dim3 unit_grid(const KvArgs &a, int units, int D)
{
    const int per = 256 / (D / 8);
    return dim3(static_cast<uint32_t>((std::min<int64_t>(a.max_new, a.rows) * units + per - 1) / per), a.n_seqs);
}

int launch_kv_append(const KvArgs &a, const KvAppendArgs &p, int D, hipStream_t s)
{
    const auto kernel = D == 64 ? k_kv_append<64> : D == 128 ? k_kv_append<128> : k_kv_append<256>;
    launch_kernel(kernel, unit_grid(a, p.units, D), dim3(256), 0, s, a, p);
    return hip_result(hipGetLastError());
}

int launch_kv_read(const KvArgs &a, const KvReadArgs &p, int D, hipStream_t s)
{
    const auto kernel = D == 64 ? k_kv_read<64> : D == 128 ? k_kv_read<128> : k_kv_read<256>;
    launch_kernel(kernel, unit_grid(a, p.units, D), dim3(256), 0, s, a, p);
    return hip_result(hipGetLastError());
}

}  // namespace tpq
