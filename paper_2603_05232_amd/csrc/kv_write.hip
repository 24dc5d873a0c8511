// kv_write, kv_read: keys and values of tokens into the pages of a cache, quantised on the way, and out of them again.
#include "kv_common.h"
#include "quant_common.h"

namespace ss {

constexpr int KW_WAVES = 4;                          // wavefronts of a workgroup
constexpr int KW_SPREAD = 2048;                      // tokens up to which each gets a wavefront of its own

// 16 or 8 bytes at the alignment of an element
typedef uint32_t kv16_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t kv16f_t __attribute__((ext_vector_type(4), aligned(4)));

// values 8 c .. 8 c + 7 of a row of D; zeros behind it
__device__ inline void kv_get8(const uint16_t* p, int c, int D, float (&f)[8])
{
    const int have = D - 8 * c;
    p += 8 * c;
    if (have >= 8) {
        const kv16_t v = *reinterpret_cast<const kv16_t*>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(v[j] << 16); f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < have ? bf16_bits_to_f32(p[j]) : 0.0f;
    }
}
__device__ inline void kv_get8(const float* p, int c, int D, float (&f)[8])
{
    const int have = D - 8 * c;
    p += 8 * c;
    if (have >= 8) {
        const kv16f_t a = *reinterpret_cast<const kv16f_t*>(p), b = *reinterpret_cast<const kv16f_t*>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { f[j] = __uint_as_float(a[j]); f[4 + j] = __uint_as_float(b[j]); }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < have ? p[j] : 0.0f;
    }
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

// Eight codes of a piece, 16 or 8 bytes (in the first two words).
template <int DT> __device__ inline uint4 kv_codes8(const float (&f)[8], float r)
{
    if constexpr (DT == SS_BF16) return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    else if constexpr (DT == SS_FP16) {
        auto two = [](float a, float b) { return f32_to_f16_bits(a) | (uint32_t)f32_to_f16_bits(b) << 16; };
        return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
    } else return make_uint4(quant4<DT>(f[0], f[1], f[2], f[3], r), quant4<DT>(f[4], f[5], f[6], f[7], r), 0, 0);
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

// Scale and its inverse from the largest magnitude's bits.  Magnitudes below 2^-100 count as zero, so that the inverse is finite; an infinity or a NaN makes the scale a NaN, and
// with it every product.
__device__ inline void kv_scale(uint32_t largest, float qmax, float& scale, float& inverse)
{
    const float a = __uint_as_float(largest);
    const bool bad = largest >= 0x7F800000u, none = a < 0x1p-100f;
    scale = bad ? __uint_as_float(0x7FC00000u) : none ? 1.0f : a / qmax;
    inverse = bad || none ? 0.0f : qmax * (1.0f / a);
}

__device__ inline uint32_t kv_row_max(uint32_t v)    // over eight lanes side by side
{
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d, 64));
    return v;
}

// Where a slot's block and head lie, and its token of the block.
__device__ inline int64_t kv_block_of(int slot, int h, int H, int page, Div by_page, int64_t page_bytes, int block_bytes, int& tau)
{
    const int id = quot(slot, by_page), row = slot - id * page;
    tau = row & (KV_BLOCK - 1);
    return id * page_bytes + (int64_t)(h * (page / KV_BLOCK) + row / KV_BLOCK) * block_bytes;
}

// A wavefront takes up to eight tokens of one head at a time whose slots are consecutive and share a group of eight: lane (i, c) = (l >> 3, l & 7) the pieces of 8 values c, c + 8, ..
// of token i.  `span` tokens to a wavefront, which looks for the runs that begin among them.  Keys are stored by pieces.  Of values a whole group of eight tokens is
// turned in LDS, so that a lane stores the eight tokens of a channel at once; a group that is not whole is stored by single elements.
template <typename T, int DT>
__global__ __launch_bounds__(64 * KW_WAVES) void k_kv_write(const T* __restrict__ K, const T* __restrict__ V, int64_t ldk, int64_t hk, int64_t ldv, int64_t hv, const int32_t* __restrict__ slots,
                                                            int N, int H, int D, int steps, uint8_t* __restrict__ pages, int slots_end, int page, Div by_page, int64_t page_bytes,
                                                            int span, Div by_heads)
{
    constexpr int ES = kv_es(DT), CH = KV_MAX_D / 64;
    __shared__ uint4 turn[KW_WAVES][8 * KV_MAX_D * ES / 16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane >> 3, c0 = lane & 7;
    const int group = quot(blockIdx.x, by_heads), h = blockIdx.x - group * H;
    const int base = (group * KW_WAVES + wave) * span, pieces = 4 * steps, half = kv_half_bytes(ES, steps), block_bytes = kv_block_bytes(ES, steps);
    if (base >= N) return;
    // slots of tokens base - 1 + lane
    const int n = base - 1 + lane;
    const int slot = lane < 17 && n >= 0 && n < N ? slots[n] : -1;
    const bool valid = slot >= 0 && slot < slots_end;
    const int before = __shfl_up(slot, 1, 64);
    const bool follows = lane > 0 && valid && before == slot - 1 && (slot & 7) != 0;
    const uint64_t more = __ballot(follows);
    for (uint64_t first = __ballot(valid && !follows && lane >= 1 && lane <= span); first; first &= first - 1) {
        const int at = __ffsll((unsigned long long)first) - 1, r = __ffsll((unsigned long long)~(more >> (at + 1)));      // 1 .. 8 tokens
        const int s0 = __builtin_amdgcn_readlane(slot, at), t0 = base - 1 + at;
        const bool there = i < r;
        const int64_t row = t0 + (there ? i : 0);
        const T *const k = K + row * ldk + h * hk, *const v = V + row * ldv + h * hv;
        float kf[CH][8], vf[CH][8];
#pragma unroll
        for (int q = 0; q < CH; ++q)
            if (c0 + 8 * q < pieces) { kv_get8(k, c0 + 8 * q, D, kf[q]); kv_get8(v, c0 + 8 * q, D, vf[q]); }
        float rk = 0.0f, rv = 0.0f, sk = 0.0f, sv = 0.0f;
        if constexpr (ES == 1) {
            uint32_t mk = 0, mv = 0;
#pragma unroll
            for (int q = 0; q < CH; ++q)
                if (c0 + 8 * q < pieces)
#pragma unroll
                    for (int e = 0; e < 8; ++e) { mk = max(mk, __float_as_uint(kf[q][e]) & 0x7FFFFFFFu); mv = max(mv, __float_as_uint(vf[q][e]) & 0x7FFFFFFFu); }
            constexpr float qmax = DT == SS_I8 ? 127.0f : 448.0f;
            kv_scale(kv_row_max(mk), qmax, sk, rk);
            kv_scale(kv_row_max(mv), qmax, sv, rv);
            // codes of a row whose scale is not a number are zeros
            if (rk == 0.0f || rv == 0.0f) {
#pragma unroll
                for (int q = 0; q < CH; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e) { kf[q][e] = rk == 0.0f ? 0.0f : kf[q][e]; vf[q][e] = rv == 0.0f ? 0.0f : vf[q][e]; }
            }
        }
        int tau;
        uint8_t* const block = pages + kv_block_of(s0, h, H, page, by_page, page_bytes, block_bytes, tau);      // of the whole run
        const int group8 = tau >> 3;
        tau += i;
        if (ES == 1 && there && c0 == 0) {
            float* const scales = reinterpret_cast<float*>(block + 2 * half);
            scales[tau] = sk;
            scales[KV_BLOCK + tau] = sv;
        }
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = c0 + 8 * q;
            if (c >= pieces) continue;
            const uint4 kc = kv_codes8<DT>(kf[q], rk), vc = kv_codes8<DT>(vf[q], rv);
            if (there) {
                uint8_t* const to = block + kv_key_at(ES, tau, c);
                if constexpr (ES == 2) *reinterpret_cast<uint4*>(to) = kc;
                else *reinterpret_cast<uint2*>(to) = make_uint2(kc.x, kc.y);
            }
            if (r == 8) {
                if constexpr (ES == 2) turn[wave][i * pieces + c] = vc;
                else reinterpret_cast<uint2*>(turn[wave])[i * pieces + c] = make_uint2(vc.x, vc.y);
            } else if (there) {
                const uint32_t w[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    uint8_t* const to = block + half + kv_value_at(ES, group8, 8 * c + e);
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(to)[tau & 7] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                    else to[tau & 7] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        }
        if (r == 8) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            const uint32_t* const words = reinterpret_cast<const uint32_t*>(turn[wave]);
            constexpr int PER = 4 / ES;              // channels of a word
            const int pitch = 8 * pieces / PER;      // words of a token
            for (int x = lane; x < pitch; x += 64) {
                uint32_t w[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) w[t] = words[t * pitch + x];
                if constexpr (ES == 2) {
                    uint4 lo, hi;
                    lo.x = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u); hi.x = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
                    lo.y = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u); hi.y = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
                    lo.z = __builtin_amdgcn_perm(w[5], w[4], 0x05040100u); hi.z = __builtin_amdgcn_perm(w[5], w[4], 0x07060302u);
                    lo.w = __builtin_amdgcn_perm(w[7], w[6], 0x05040100u); hi.w = __builtin_amdgcn_perm(w[7], w[6], 0x07060302u);
                    *reinterpret_cast<uint4*>(block + half + kv_value_at(2, group8, 2 * x)) = lo;
                    *reinterpret_cast<uint4*>(block + half + kv_value_at(2, group8, 2 * x + 1)) = hi;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // byte e of four words side by side
                        const uint32_t pick = 0x0C0C0000u | (uint32_t)(4 + e) << 8 | e;
                        const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], pick), b = __builtin_amdgcn_perm(w[3], w[2], pick), c = __builtin_amdgcn_perm(w[5], w[4], pick),
                                       d = __builtin_amdgcn_perm(w[7], w[6], pick);
                        *reinterpret_cast<uint2*>(block + half + kv_value_at(1, group8, 4 * x + e)) = make_uint2(a | b << 16, c | d << 16);
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");      // before the next run's values
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
}

// A wavefront takes eight tokens of one head, lanes as above.  A slot outside the cache gives zeros.
template <typename T, int DT>
__global__ __launch_bounds__(64 * KW_WAVES) void k_kv_read(const uint8_t* __restrict__ pages, const int32_t* __restrict__ slots, int N, int H, int D, int steps, int slots_end, int page,
                                                           Div by_page, int64_t page_bytes, T* __restrict__ K, int64_t ldk, int64_t hk, T* __restrict__ V, int64_t ldv, int64_t hv,
                                                           Div by_heads)
{
    constexpr int ES = kv_es(DT);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c0 = lane & 7;
    const int group = quot(blockIdx.x, by_heads), h = blockIdx.x - group * H;
    const int n = (group * KW_WAVES + wave) * 8 + (lane >> 3);
    if (n >= N) return;
    const int half = kv_half_bytes(ES, steps), slot = slots[n];
    const bool valid = slot >= 0 && slot < slots_end;
    int tau;
    const uint8_t* const block = pages + kv_block_of(valid ? slot : 0, h, H, page, by_page, page_bytes, kv_block_bytes(ES, steps), tau);
    float sk = 1.0f, sv = 1.0f;
    if constexpr (ES == 1) {
        const float* const scales = reinterpret_cast<const float*>(block + 2 * half);
        sk = scales[tau];
        sv = scales[KV_BLOCK + tau];
    }
    for (int c = c0; 8 * c < D; c += 8) {
        uint4 kc = make_uint4(0, 0, 0, 0), vc = kc;
        const uint8_t* const from = block + kv_key_at(ES, tau, c);
        if constexpr (ES == 2) kc = *reinterpret_cast<const uint4*>(from);
        else { const uint2 two = *reinterpret_cast<const uint2*>(from); kc.x = two.x; kc.y = two.y; }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t* const v = block + half + kv_value_at(ES, tau >> 3, 8 * c + e);
            if constexpr (ES == 2) w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(v)[tau & 7] << (16 * (e & 1));
            else w[e >> 2] |= (uint32_t)v[tau & 7] << (8 * (e & 3));
        }
        vc = make_uint4(w[0], w[1], w[2], w[3]);
        float kf[8], vf[8];
        kv_values8<DT>(kc, sk, kf);
        kv_values8<DT>(vc, sv, vf);
#pragma unroll
        for (int e = 0; e < 8; ++e) { kf[e] = valid ? kf[e] : 0.0f; vf[e] = valid ? vf[e] : 0.0f; }
        kv_put8(K + (int64_t)n * ldk + h * hk, c, D, kf);
        kv_put8(V + (int64_t)n * ldv + h * hv, c, D, vf);
    }
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
    const int span = N <= KW_SPREAD ? 1 : 8;
    const int64_t groups = (N + KW_WAVES * span - 1) / (KW_WAVES * span) * H;
    if (!mx4_grid_fits(groups, 64 * KW_WAVES)) return SS_ERR_SHAPE;
    auto launch = [&](auto kernel, auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(64 * KW_WAVES), 0, static_cast<hipStream_t>(stream), static_cast<const T*>(K), static_cast<const T*>(V), ldk, hk, ldv, hv, slots, (int)N,
                           (int)H, (int)D, kv_steps(D), static_cast<uint8_t*>(pages), (int)(P * page), (int)page, make_div(page), kv_bytes_of_page(H, page, D, dtype), span, make_div(H));
        return launch_status();
    };
#define SS_KW(T) (dtype == SS_I8 ? launch(k_kv_write<T, SS_I8>, T()) : dtype == SS_FP8_E4M3 ? launch(k_kv_write<T, SS_FP8_E4M3>, T()) : dtype == SS_BF16 ? launch(k_kv_write<T, SS_BF16>, T()) : launch(k_kv_write<T, SS_FP16>, T()))
    return in_dtype == SS_IN_F32 ? SS_KW(float) : SS_KW(uint16_t);
#undef SS_KW
}

extern "C" ss_status kv_read(const void* pages, int64_t P, int64_t page, ss_dtype dtype, const int32_t* slots, int64_t N, int64_t H, int64_t D, ss_act_dtype out_dtype, void* K, int64_t ldk,
                             int64_t hk, void* V, int64_t ldv, int64_t hv, void* stream)
{
    if ((out_dtype != SS_IN_F32 && out_dtype != SS_IN_BF16) || !valid_dtype(dtype)) return SS_ERR_DTYPE;
    if (N < 0 || N > KV_MAX_TOKENS || !kv_valid_page(H, page, D, dtype) || !kv_valid_slots(P, page) || !valid_strides(ldk, hk) || !valid_strides(ldv, hv)) return SS_ERR_SHAPE;
    if (N == 0) return SS_OK;
    if (!K || !V || !slots || !pages) return SS_ERR_NULL;
    if ((((uintptr_t)K | (uintptr_t)V) & (out_dtype == SS_IN_F32 ? 3 : 1)) || ((uintptr_t)slots & 3) || ((uintptr_t)pages & 15)) return SS_ERR_SHAPE;
    const int64_t groups = (N + KW_WAVES * 8 - 1) / (KW_WAVES * 8) * H;
    if (!mx4_grid_fits(groups, 64 * KW_WAVES)) return SS_ERR_SHAPE;
    auto launch = [&](auto kernel, auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(64 * KW_WAVES), 0, static_cast<hipStream_t>(stream), static_cast<const uint8_t*>(pages), slots, (int)N, (int)H, (int)D, kv_steps(D),
                           (int)(P * page), (int)page, make_div(page), kv_bytes_of_page(H, page, D, dtype), static_cast<T*>(K), ldk, hk, static_cast<T*>(V), ldv, hv, make_div(H));
        return launch_status();
    };
#define SS_KR(T) (dtype == SS_I8 ? launch(k_kv_read<T, SS_I8>, T()) : dtype == SS_FP8_E4M3 ? launch(k_kv_read<T, SS_FP8_E4M3>, T()) : dtype == SS_BF16 ? launch(k_kv_read<T, SS_BF16>, T()) : launch(k_kv_read<T, SS_FP16>, T()))
    return out_dtype == SS_IN_F32 ? SS_KR(float) : SS_KR(uint16_t);
#undef SS_KR
}
