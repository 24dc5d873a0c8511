// kv_write, kv_read: keys and values of tokens into the pages of a cache, quantised on the way, and out of them again.
//
// Bound by HBM where there are many tokens, 8192 tokens of 8 heads of 128, bf16 to fp8: 10.4 .. 10.7 us (33.9 MB read, 17.3 written, 4.8 .. 4.9 TB/s) and back 10.2 us, and by three
// waits one after the other (slots, rows, stores; 2.8 us) where there are few.  Values by single elements throughout took 17 us: a store of one byte for each channel
// of a token.
#include "kv_common.h"
#include "quant_common.h"

namespace ss {

constexpr int KW_WAVES = 4;                          // wavefronts of a workgroup

// 16 or 8 bytes at the alignment of an element
typedef uint32_t kv16_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t kv16f_t __attribute__((ext_vector_type(4), aligned(4)));

// Piece c of a row of D values, 8 c .. 8 c + 7, as it lies in memory; zeros behind the row.  Whole pieces are asked for first, all of them, and what is left of a row
// afterwards: a branch between two loads makes the second wait for the first.
template <typename T> struct KvPiece { uint32_t w[2 * sizeof(T)]; };
__device__ inline void kv_get_whole(const uint16_t* p, int c, int D, KvPiece<uint16_t>& x)
{
    kv16_t v = {0, 0, 0, 0};
    if (8 * c + 8 <= D) v = *reinterpret_cast<const kv16_t*>(p + 8 * c);
#pragma unroll
    for (int j = 0; j < 4; ++j) x.w[j] = v[j];
}
__device__ inline void kv_get_whole(const float* p, int c, int D, KvPiece<float>& x)
{
    kv16f_t a = {0, 0, 0, 0}, b = a;
    if (8 * c + 8 <= D) { a = *reinterpret_cast<const kv16f_t*>(p + 8 * c); b = *reinterpret_cast<const kv16f_t*>(p + 8 * c + 4); }
#pragma unroll
    for (int j = 0; j < 4; ++j) { x.w[j] = a[j]; x.w[4 + j] = b[j]; }
}
__device__ inline void kv_get_rest(const uint16_t* p, int c, int D, KvPiece<uint16_t>& x)
{
    if (8 * c >= D || 8 * c + 8 <= D) return;
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (8 * c + j < D) x.w[j >> 1] |= (uint32_t)p[8 * c + j] << (16 * (j & 1));
}
__device__ inline void kv_get_rest(const float* p, int c, int D, KvPiece<float>& x)
{
    if (8 * c >= D || 8 * c + 8 <= D) return;
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (8 * c + j < D) x.w[j] = __float_as_uint(p[8 * c + j]);
}
// the largest magnitude's bits of a piece, and of m
__device__ inline uint32_t kv_largest(const KvPiece<uint16_t>& x, uint32_t m)      // two to a word
{
    typedef uint16_t two_t __attribute__((ext_vector_type(2)));
    two_t a = __builtin_bit_cast(two_t, m);
#pragma unroll
    for (int j = 0; j < 4; ++j) a = __builtin_elementwise_max(a, __builtin_bit_cast(two_t, x.w[j] & 0x7FFF7FFFu));
    return __builtin_bit_cast(uint32_t, a);
}
__device__ inline uint32_t kv_largest(const KvPiece<float>& x, uint32_t m)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, x.w[j] & 0x7FFFFFFFu);
    return m;
}
template <typename T> __device__ inline uint32_t kv_row_largest(uint32_t m)      // of the eight lanes of a row, as fp32
{
    if constexpr (sizeof(T) == 2) m = max(m << 16, m & 0xFFFF0000u);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
    return m;
}
__device__ inline void kv_floats(const KvPiece<uint16_t>& x, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(x.w[j] << 16); f[2 * j + 1] = __uint_as_float(x.w[j] & 0xFFFF0000u); }
}
__device__ inline void kv_floats(const KvPiece<float>& x, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(x.w[j]);
}
__device__ inline void kv_put8(uint16_t* p, int c, int D, const float (&f)[8])
{
    const int have = D - 8 * c;
    p += 8 * c;
    const uint32_t w[4] = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    if (have >= 8) *reinterpret_cast<kv16_t*>(p) = kv16_t{w[0], w[1], w[2], w[3]};
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < have) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}
__device__ inline void kv_put8(float* p, int c, int D, const float (&f)[8])
{
    const int have = D - 8 * c;
    p += 8 * c;
    if (have >= 8) {
        *reinterpret_cast<kv16f_t*>(p) = kv16f_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
        *reinterpret_cast<kv16f_t*>(p + 4) = kv16f_t{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < have) p[j] = f[j];
    }
}

// Eight codes of a piece, 16 or 8 bytes (in the first two words).  Values of 8 bits need no clamp: |x r| <= Qmax (1 + 2^-22), which is nearest to Qmax.
template <int DT> __device__ inline uint32_t kv_codes4(float x0, float x1, float x2, float x3, float r)
{
    if constexpr (DT == SS_FP8_E4M3) return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2 * r, x3 * r, __builtin_amdgcn_cvt_pk_fp8_f32(x0 * r, x1 * r, 0, false), true);
    else {
        constexpr float ROUND = 12582912.0f;         // 1.5 2^23: the sum's low byte is the nearest integer, ties to even, in two's complement
        return pack_bytes(__float_as_uint(x0 * r + ROUND), __float_as_uint(x1 * r + ROUND), __float_as_uint(x2 * r + ROUND), __float_as_uint(x3 * r + ROUND));
    }
}
template <int DT> __device__ inline uint4 kv_codes8(const float (&f)[8], float r)
{
    if constexpr (DT == SS_BF16) return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    else if constexpr (DT == SS_FP16) {
        auto two = [](float a, float b) { return f32_to_f16_bits(a) | (uint32_t)f32_to_f16_bits(b) << 16; };
        return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
    } else return make_uint4(kv_codes4<DT>(f[0], f[1], f[2], f[3], r), kv_codes4<DT>(f[4], f[5], f[6], f[7], r), 0, 0);
}
// and back
template <int DT> __device__ inline void kv_values8(uint4 v, float s, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (DT == SS_BF16) f[j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
        else if constexpr (DT == SS_FP16) f[j] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j >> 1] >> (16 * (j & 1))));
        else if constexpr (DT == SS_I8) f[j] = (float)(int8_t)(w[j >> 2] >> (8 * (j & 3))) * s;
    }
    if constexpr (DT == SS_FP8_E4M3) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f[4 * h] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 0) * s;
            f[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 1) * s;
            f[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 2) * s;
            f[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 3) * s;
        }
    }
}

// Scale and its inverse from the largest magnitude's bits.  Magnitudes below 2^-100 count as zero, so that the inverse is finite; an infinity or a NaN makes the scale
// a NaN, and with it every product.
__device__ inline void kv_scale(uint32_t largest, float qmax, float& scale, float& inverse)
{
    const float a = __uint_as_float(largest);
    const bool bad = largest >= 0x7F800000u, none = a < 0x1p-100f;
    scale = bad ? __uint_as_float(0x7FC00000u) : none ? 1.0f : a / qmax;
    inverse = bad || none ? 0.0f : qmax * (1.0f / a);
}

// Where a slot's block and head lie, and its token of the block.
__device__ inline int64_t kv_block_of(int slot, int h, int H, int page, Div by_page, int64_t page_bytes, int block_bytes, int& tau)
{
    const int id = quot(slot, by_page), row = slot - id * page;
    tau = row & (KV_BLOCK - 1);
    return id * page_bytes + (int64_t)(h * (page / KV_BLOCK) + row / KV_BLOCK) * block_bytes;
}

// Which of a wavefront's eight tokens base .. base + 7 lie in a whole group: eight tokens side by side whose slots are consecutive from a multiple of 8 on, so that
// they are all that the cache holds of these eight slots.  Lane l holds the slot of token base - 8 + l, l < 24; the group's first token may lie before or behind base.
struct KwGroups {
    int slot;                                        // of token base + (lane >> 3); -1: none
    bool grouped;                                    // whether that one lies in a whole group
    int leader;                                      // the token of base .. base + 7 that a whole group begins with, or -1: there is one at most
    int first_slot;                                  // its slot
};
__device__ inline KwGroups kw_groups(const int32_t* __restrict__ slots, int base, int N, int slots_end)
{
    const int lane = threadIdx.x & 63, n = base - 8 + lane;
    int slot = lane < 24 && n >= 0 && n < N ? slots[n] : -1;
    slot = slot >= 0 && slot < slots_end ? slot : -1;
    const int previous = __shfl_up(slot, 1, 64);     // by all lanes, ahead of any condition
    const uint64_t follows = __ballot(lane > 0 && slot >= 0 && (slot & 7) != 0 && previous == slot - 1);
    uint64_t run = follows >> 1;                     // bit l: l + 1 follows l
    run &= run >> 1;
    run &= run >> 2;
    run &= follows >> 5 & follows >> 6 & follows >> 7;      // l + 1 .. l + 7 do
    run &= __ballot(slot >= 0 && (slot & 7) == 0);
    uint64_t all = run | run << 1;
    all |= all << 2;
    all |= all << 4;
    KwGroups g;
    const int i = lane >> 3;
    g.slot = __shfl(slot, 8 + i, 64);
    g.grouped = all >> (8 + i) & 1;
    const uint64_t here = run >> 8 & 0xFF;
    g.leader = here ? base + __ffsll((unsigned long long)here) - 1 : -1;
    g.first_slot = __builtin_amdgcn_readlane(slot, here ? 7 + __ffsll((unsigned long long)here) : 0);
    return g;
}

__device__ inline void kw_wave_sync()                // what the wavefront's lanes put into LDS is there for all of them
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wavefront takes eight tokens of one head: lane (i, c) = (l >> 3, l & 7) the pieces of 8 values c, c + 8, .. of token i.  First the whole group that begins among
// its tokens, if any, then those that lie in none.  Keys are stored by pieces.  Of values a whole group's eight tokens are turned in LDS, so that a lane stores the
// eight tokens of a channel at once; others are stored by single elements.  CH: pieces of a lane.
template <typename T, int DT, int CH>
__global__ __launch_bounds__(64 * KW_WAVES) void k_kv_write(const T* __restrict__ K, const T* __restrict__ V, int64_t ldk, int64_t hk, int64_t ldv, int64_t hv, const int32_t* __restrict__ slots,
                                                            int N, int H, int D, int steps, uint8_t* __restrict__ pages, int slots_end, int page, Div by_page, int64_t page_bytes, Div by_heads)
{
    constexpr int ES = kv_es(DT);
    __shared__ uint4 turn[KW_WAVES][8 * 64 * CH * ES / 16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane >> 3, c0 = lane & 7;
    const int group = quot(blockIdx.x, by_heads), h = blockIdx.x - group * H;
    const int base = (group * KW_WAVES + wave) * 8, pieces = 4 * steps, half = kv_half_bytes(ES, steps), block_bytes = kv_block_bytes(ES, steps);
    if (base >= N) return;
    const KwGroups g = kw_groups(slots, base, N, slots_end);
    unroll<2>([&](auto pass) {
        constexpr bool whole = decltype(pass)::value == 0;
        const bool there = whole ? true : g.slot >= 0 && !g.grouped;
        if (whole ? g.leader < 0 : __ballot(there) == 0) return;
        const int64_t row = whole ? g.leader + i : there ? base + i : base;
        const T *const k = K + row * ldk + h * hk, *const v = V + row * ldv + h * hv;
        KvPiece<T> kp[CH], vp[CH];
#pragma unroll
        for (int q = 0; q < CH; ++q) { kv_get_whole(k, c0 + 8 * q, D, kp[q]); kv_get_whole(v, c0 + 8 * q, D, vp[q]); }
        if (D & 7) {
#pragma unroll
            for (int q = 0; q < CH; ++q) { kv_get_rest(k, c0 + 8 * q, D, kp[q]); kv_get_rest(v, c0 + 8 * q, D, vp[q]); }
        }
        float kf[CH][8], vf[CH][8];
#pragma unroll
        for (int q = 0; q < CH; ++q) { kv_floats(kp[q], kf[q]); kv_floats(vp[q], vf[q]); }
        float rk = 0.0f, rv = 0.0f, sk = 0.0f, sv = 0.0f;
        if constexpr (ES == 1) {
            uint32_t mk = 0, mv = 0;
#pragma unroll
            for (int q = 0; q < CH; ++q) { mk = kv_largest(kp[q], mk); mv = kv_largest(vp[q], mv); }
            constexpr float qmax = DT == SS_I8 ? 127.0f : 448.0f;
            kv_scale(kv_row_largest<T>(mk), qmax, sk, rk);
            kv_scale(kv_row_largest<T>(mv), qmax, sv, rv);
            // codes of a row whose scale is not a number are zeros
            if (rk == 0.0f || rv == 0.0f) {
#pragma unroll
                for (int q = 0; q < CH; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e) { kf[q][e] = rk == 0.0f ? 0.0f : kf[q][e]; vf[q][e] = rv == 0.0f ? 0.0f : vf[q][e]; }
            }
        }
        int tau;
        uint8_t* const block = pages + kv_block_of(whole ? g.first_slot : there ? g.slot : 0, h, H, page, by_page, page_bytes, block_bytes, tau);      // of a group the same for all lanes
        const int group8 = tau >> 3;
        if constexpr (whole) tau += i;
        if (ES == 1 && there && c0 == 0) {
            float* const scales = reinterpret_cast<float*>(block + 2 * half);
            scales[tau] = sk;
            scales[KV_BLOCK + tau] = sv;
        }
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = c0 + 8 * q;
            if (c >= pieces || !there) continue;
            const uint4 kc = kv_codes8<DT>(kf[q], rk), vc = kv_codes8<DT>(vf[q], rv);
            uint8_t* const to = block + kv_key_at(ES, tau, c);
            if constexpr (ES == 2) *reinterpret_cast<uint4*>(to) = kc;
            else *reinterpret_cast<uint2*>(to) = make_uint2(kc.x, kc.y);
            if constexpr (whole) {                   // [channel][8 tokens]
                const uint32_t w[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(turn[wave])[(8 * c + e) * 8 + i] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                    else reinterpret_cast<uint8_t*>(turn[wave])[(8 * c + e) * 8 + i] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            } else {
                const uint32_t w[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    uint8_t* const one = block + half + kv_value_at(ES, group8, 8 * c + e);
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(one)[tau & 7] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                    else one[tau & 7] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        }
        if constexpr (whole) {
            kw_wave_sync();
            // 16 bytes to a lane as they lie side by side in the block: a channel, or two of 8 bits
            for (int x = lane; x < 32 * steps / (3 - ES); x += 64) {
                if constexpr (ES == 2) *reinterpret_cast<uint4*>(block + half + kv_value_at(2, group8, x)) = turn[wave][x];
                else {
                    const int d = (x >> 4) * 32 + (x & 15);
                    const uint2* const two = reinterpret_cast<const uint2*>(turn[wave]);
                    *reinterpret_cast<uint4*>(block + half + kv_value_at(1, group8, d)) = make_uint4(two[d].x, two[d].y, two[d + 16].x, two[d + 16].y);
                }
            }
        }
    });
}

// A wavefront takes eight tokens of one head, lanes and groups as above; a whole group's values are turned in LDS the other way round.  A slot outside the cache gives zeros.
template <typename T, int DT, int CH>
__global__ __launch_bounds__(64 * KW_WAVES) void k_kv_read(const uint8_t* __restrict__ pages, const int32_t* __restrict__ slots, int N, int H, int D, int steps, int slots_end, int page,
                                                           Div by_page, int64_t page_bytes, T* __restrict__ K, int64_t ldk, int64_t hk, T* __restrict__ V, int64_t ldv, int64_t hv,
                                                           Div by_heads)
{
    constexpr int ES = kv_es(DT), PITCH = 64 * CH + 8;            // elements of a token in LDS; the eight tokens of a channel on different banks
    __shared__ uint4 turn[KW_WAVES][8 * PITCH * ES / 16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane >> 3, c0 = lane & 7;
    const int group = quot(blockIdx.x, by_heads), h = blockIdx.x - group * H;
    const int base = (group * KW_WAVES + wave) * 8, half = kv_half_bytes(ES, steps);
    if (base >= N) return;
    const KwGroups g = kw_groups(slots, base, N, slots_end);
    unroll<2>([&](auto pass) {
        constexpr bool whole = decltype(pass)::value == 0;
        const bool there = whole ? true : base + i < N && !g.grouped;
        if (whole ? g.leader < 0 : __ballot(there) == 0) return;
        const bool valid = whole || g.slot >= 0;
        const int64_t n = whole ? g.leader + i : base + i;
        int tau;
        const uint8_t* const block = pages + kv_block_of(whole ? g.first_slot : valid ? g.slot : 0, h, H, page, by_page, page_bytes, kv_block_bytes(ES, steps), tau);
        const int group8 = tau >> 3;
        if constexpr (whole) tau += i;
        float sk = 1.0f, sv = 1.0f;
        if constexpr (ES == 1) {
            const float* const scales = reinterpret_cast<const float*>(block + 2 * half);
            sk = scales[tau];
            sv = scales[KV_BLOCK + tau];
        }
        if constexpr (whole) {
#pragma unroll
            for (int q = 0; q < CH; ++q) {
                const int d = 64 * q + lane;
                if (d >= 32 * steps) continue;
                const uint8_t* const from = block + half + kv_value_at(ES, group8, d);
                if constexpr (ES == 2) {
                    const uint4 x = *reinterpret_cast<const uint4*>(from);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(turn[wave])[e * PITCH + d] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(from);
#pragma unroll
                    for (int e = 0; e < 8; ++e) reinterpret_cast<uint8_t*>(turn[wave])[e * PITCH + d] = (uint8_t)((e & 4 ? x.y : x.x) >> (8 * (e & 3)));
                }
            }
            kw_wave_sync();
        }
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = c0 + 8 * q;
            if (8 * c >= D || !there) continue;
            uint4 kc = make_uint4(0, 0, 0, 0), vc = kc;
            const uint8_t* const from = block + kv_key_at(ES, tau, c);
            if constexpr (ES == 2) kc = *reinterpret_cast<const uint4*>(from);
            else { const uint2 two = *reinterpret_cast<const uint2*>(from); kc.x = two.x; kc.y = two.y; }
            if constexpr (whole) {
                if constexpr (ES == 2) vc = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(turn[wave]) + i * PITCH + 8 * c);
                else { const uint2 two = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(turn[wave]) + i * PITCH + 8 * c); vc.x = two.x; vc.y = two.y; }
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint8_t* const v = block + half + kv_value_at(ES, group8, 8 * c + e);
                    if constexpr (ES == 2) w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(v)[tau & 7] << (16 * (e & 1));
                    else w[e >> 2] |= (uint32_t)v[tau & 7] << (8 * (e & 3));
                }
                vc = make_uint4(w[0], w[1], w[2], w[3]);
            }
            float kf[8], vf[8];
            kv_values8<DT>(kc, sk, kf);
            kv_values8<DT>(vc, sv, vf);
#pragma unroll
            for (int e = 0; e < 8; ++e) { kf[e] = valid ? kf[e] : 0.0f; vf[e] = valid ? vf[e] : 0.0f; }
            kv_put8(K + n * ldk + h * hk, c, D, kf);
            kv_put8(V + n * ldv + h * hv, c, D, vf);
        }
    });
}

}  // namespace ss

using namespace ss;

extern "C" int64_t kv_page_bytes(int64_t H, int64_t page, int64_t D, ss_dtype dtype) { return kv_valid_page(H, page, D, dtype) ? kv_bytes_of_page(H, page, D, dtype) : -1; }

// rows of keys or values may lie at any distance from each other; in one call no offset passes 2^62
static bool valid_strides(int64_t ld, int64_t h) { return ld >= 0 && h >= 0 && ld <= (int64_t)1 << 40 && h <= (int64_t)1 << 40; }

extern "C" ss_status kv_write(const void* K, int64_t ldk, int64_t hk, const void* V, int64_t ldv, int64_t hv, ss_act_dtype in_dtype, int64_t N, int64_t H, int64_t D, const int32_t* slots,
                              void* pages, int64_t P, int64_t page, ss_dtype dtype, void* stream)
{
    if ((in_dtype != SS_IN_F32 && in_dtype != SS_IN_BF16) || !valid_dtype(dtype)) return SS_ERR_DTYPE;
    if (N < 0 || N > KV_MAX_TOKENS || !kv_valid_page(H, page, D, dtype) || !kv_valid_slots(P, page) || !valid_strides(ldk, hk) || !valid_strides(ldv, hv)) return SS_ERR_SHAPE;
    if (N == 0) return SS_OK;
    if (!K || !V || !slots || !pages) return SS_ERR_NULL;
    if ((((uintptr_t)K | (uintptr_t)V) & (in_dtype == SS_IN_F32 ? 3 : 1)) || ((uintptr_t)slots & 3) || ((uintptr_t)pages & 15)) return SS_ERR_SHAPE;
    const int64_t groups = (N + KW_WAVES * 8 - 1) / (KW_WAVES * 8) * H;
    if (!mx4_grid_fits(groups, 64 * KW_WAVES)) return SS_ERR_SHAPE;
    auto launch = [&](auto kernel, auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(64 * KW_WAVES), 0, static_cast<hipStream_t>(stream), static_cast<const T*>(K), static_cast<const T*>(V), ldk, hk, ldv, hv, slots, (int)N,
                           (int)H, (int)D, kv_steps(D), static_cast<uint8_t*>(pages), (int)(P * page), (int)page, make_div(page), kv_bytes_of_page(H, page, D, dtype), make_div(H));
        return launch_status();
    };
#define SS_KC(T, DT) (kv_steps(D) <= 2 ? launch(k_kv_write<T, DT, 1>, T()) : kv_steps(D) <= 4 ? launch(k_kv_write<T, DT, 2>, T()) : launch(k_kv_write<T, DT, 4>, T()))
#define SS_KW(T) (dtype == SS_I8 ? SS_KC(T, SS_I8) : dtype == SS_FP8_E4M3 ? SS_KC(T, SS_FP8_E4M3) : dtype == SS_BF16 ? SS_KC(T, SS_BF16) : SS_KC(T, SS_FP16))
    return in_dtype == SS_IN_F32 ? SS_KW(float) : SS_KW(uint16_t);
#undef SS_KW
#undef SS_KC
}

extern "C" ss_status kv_read(const void* pages, int64_t P, int64_t page, ss_dtype dtype, const int32_t* slots, int64_t N, int64_t H, int64_t D, ss_act_dtype out_dtype, void* K, int64_t ldk,
                             int64_t hk, void* V, int64_t ldv, int64_t hv, void* stream)
{
    if ((out_dtype != SS_IN_F32 && out_dtype != SS_IN_BF16) || !valid_dtype(dtype)) return SS_ERR_DTYPE;
    if (N < 0 || N > KV_MAX_TOKENS || !kv_valid_page(H, page, D, dtype) || !kv_valid_slots(P, page) || !valid_strides(ldk, hk) || !valid_strides(ldv, hv)) return SS_ERR_SHAPE;
    if (N == 0) return SS_OK;
    if (!K || !V || !slots || !pages) return SS_ERR_NULL;
    if (K == V || !kv_rows_apart(N, ldk, H, hk, D) || !kv_rows_apart(N, ldv, H, hv, D)) return SS_ERR_SHAPE;
    if ((((uintptr_t)K | (uintptr_t)V) & (out_dtype == SS_IN_F32 ? 3 : 1)) || ((uintptr_t)slots & 3) || ((uintptr_t)pages & 15)) return SS_ERR_SHAPE;
    const int64_t groups = (N + KW_WAVES * 8 - 1) / (KW_WAVES * 8) * H;
    if (!mx4_grid_fits(groups, 64 * KW_WAVES)) return SS_ERR_SHAPE;
    auto launch = [&](auto kernel, auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(64 * KW_WAVES), 0, static_cast<hipStream_t>(stream), static_cast<const uint8_t*>(pages), slots, (int)N, (int)H, (int)D, kv_steps(D),
                           (int)(P * page), (int)page, make_div(page), kv_bytes_of_page(H, page, D, dtype), static_cast<T*>(K), ldk, hk, static_cast<T*>(V), ldv, hv, make_div(H));
        return launch_status();
    };
#define SS_KC(T, DT) (kv_steps(D) <= 2 ? launch(k_kv_read<T, DT, 1>, T()) : kv_steps(D) <= 4 ? launch(k_kv_read<T, DT, 2>, T()) : launch(k_kv_read<T, DT, 4>, T()))
#define SS_KR(T) (dtype == SS_I8 ? SS_KC(T, SS_I8) : dtype == SS_FP8_E4M3 ? SS_KC(T, SS_FP8_E4M3) : dtype == SS_BF16 ? SS_KC(T, SS_BF16) : SS_KC(T, SS_FP16))
    return out_dtype == SS_IN_F32 ? SS_KR(float) : SS_KR(uint16_t);
#undef SS_KR
#undef SS_KC
}
