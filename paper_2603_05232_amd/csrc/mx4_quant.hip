// mx4_quant, mx4_dequant, mx4_pack: microscaled 4-bit codes of activations and weights, their values, and the operand order of the products.
#include "mx4_common.h"
#include "quant_common.h"

namespace ss {

// loads and stores of 16 bytes at the alignment of an element
template <typename T> struct Piece;
template <> struct Piece<float> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Piece<uint16_t> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2))); };

// Eight consecutive values of a row from element k on, as they lie in memory; those at or beyond K zero.
template <typename T> struct Eight { uint32_t w[2 * sizeof(T)]; };
template <typename T> __device__ inline Eight<T> load8(const T* row, int64_t k, int64_t K)
{
    typedef typename Piece<T>::V V;
    Eight<T> e;
    if (k + 8 <= K) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const V v = reinterpret_cast<const V*>(row + k)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) e.w[4 * i + j] = v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) e.w[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + j < K) {
                if constexpr (sizeof(T) == 4) e.w[j] = __float_as_uint(row[k + j]);
                else e.w[j >> 1] |= (uint32_t)row[k + j] << (16 * (j & 1));
            }
    }
    return e;
}
__device__ inline float value_of(const Eight<float>& e, int j) { return __uint_as_float(e.w[j]); }
__device__ inline float value_of(const Eight<uint16_t>& e, int j) { return __uint_as_float(j & 1 ? e.w[j >> 1] & 0xFFFF0000u : e.w[j >> 1] << 16); }

// the magnitudes' largest bits, as of an fp32; a NaN's are above infinity's
__device__ inline uint32_t largest8(const Eight<float>& e)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, e.w[j] & 0x7FFFFFFFu);
    return m;
}
__device__ inline uint32_t largest8(const Eight<uint16_t>& e)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, e.w[j] & 0x7FFF7FFFu));
    return (uint32_t)max(m[0], m[1]) << 16;
}

__device__ inline uint32_t scale_byte(uint32_t largest) { return largest >= 0x7F800000u ? 255u : max(largest >> 23, 2u) - 2u; }

// code of x r, r the inverse of the scale: nearest, ties to even, at most 6
__device__ inline uint32_t code_of(float x, float r)
{
    const float v = fabsf(x * r);
    const uint32_t c = (v > 0.25f) + (v >= 0.75f) + (v > 1.25f) + (v >= 1.75f) + (v > 2.5f) + (v >= 3.5f) + (v > 5.0f);
    return c | (__float_as_uint(x) >> 31 << 3);
}
// The eight codes by the conversion instruction, which agrees with code_of where neither the scale nor a value that counts is subnormal.
constexpr uint32_t MX_HW_SCALE = 9;                      // from this scale byte on: a subnormal value is less than 2^-8 of the scale then, code 0
__device__ inline uint32_t codes8(const Eight<float>& e, float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value_of(e, 0), value_of(e, 1), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value_of(e, 2), value_of(e, 3), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value_of(e, 4), value_of(e, 5), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value_of(e, 6), value_of(e, 7), scale, 3);
}
__device__ inline uint32_t codes8(const Eight<uint16_t>& e, float scale)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, e.w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, e.w[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, e.w[2]), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, e.w[3]), scale, 3);
}

// b = max(floor(log2 max|x|) - 2 + 127, 0) of a block, codes round(x 2^(127 - b)).  A thread takes eight values at a time, four threads a block, a
// wavefront two units of a row, CHUNKS times; the largest magnitude goes round by lane permutes, nothing through LDS.  Bound by HBM: 8192 x 4096 bf16
// rows, gathered twice, 29.6 us, 132.5 MB read and 42 written at 5.9 TB/s (codes by compares instead of the conversion instruction: 60 us).
template <typename T, int CHUNKS>
__global__ __launch_bounds__(256) void k_mx4_quant(const T* __restrict__ X, int64_t M, int64_t K, int64_t ldx, const int32_t* __restrict__ rows, int64_t R,
                                                   int U, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int per_row, Div by_row)
{
    const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = quot(item, by_row);
    const int lane = threadIdx.x & 63;
    if (r >= R) return;
    const int u0 = (item - r * per_row) * (2 * CHUNKS) + (lane >> 5);
    const int64_t src = rows ? rows[r] : r;
    const bool there = src >= 0 && src < M;
    const T* const row = X + (there ? src : 0) * ldx;
    Eight<T> e[CHUNKS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) e[i] = load8(row, (int64_t)(u0 + 2 * i) * MX_UNIT + (lane & 31) * 8, there ? K : 0);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int u = u0 + 2 * i;
        uint32_t m = largest8(e[i]);
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));      // quad_perm [1,0,3,2]
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));      // quad_perm [2,3,0,1]
        const uint32_t b = scale_byte(m);
        uint32_t w = codes8(e[i], __uint_as_float(min(b, 254u) << 23));
        if (__ballot(b < MX_HW_SCALE && m != 0)) {
            const float inv = __uint_as_float((254u - min(b, 253u)) << 23);
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) v |= code_of(value_of(e[i], j), inv) << (4 * j);
            if (b < MX_HW_SCALE) w = v;
        }
        if (b == 255) w = 0;
        if (m == 0) {                                     // zeros keep their signs, whatever a scale of 0 makes of them
            w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) w |= (__float_as_uint(value_of(e[i], j)) >> 31) << (4 * j + 3);
        }
        // the bytes of four neighbouring blocks in every sixteenth lane
        uint32_t s = b | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x104, 0xF, 0xF, true) << 8;      // row_shl:4
        s |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x108, 0xF, 0xF, true) << 16;                  // row_shl:8
        if (u < U) {
            *reinterpret_cast<uint32_t*>(codes + ((int64_t)r * U + u) * MX_UNITB + (lane & 31) * 4) = w;
            if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(scales + ((int64_t)u * R + r) * MX_UNITS + ((lane >> 2) & 4)) = s;
        }
    }
}

__device__ inline float code_value(uint32_t c)
{
    const uint32_t e = (c >> 1) & 3, m = c & 1;
    const float v = e ? __uint_as_float(((126 + e) << 23) | (m << 22)) : 0.5f * (float)m;
    return c & 8 ? -v : v;
}

// code times scale, eight codes to a thread, a wavefront two units of a row.  Bound by HBM: 16384 x 4096 to bf16 32.4 us, 42 MB read and 134 written at 5.4 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_dequant(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t R, int64_t K, int U,
                                                     T* __restrict__ Y, int64_t ldy, int per_row, Div by_row)
{
    const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r = quot(item, by_row);
    const int lane = threadIdx.x & 63;
    if (r >= R) return;
    const int u = (item - (int)r * per_row) * 2 + (lane >> 5);
    if (u >= U) return;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + r * U * MX_UNITB + (int64_t)u * MX_UNITB + (lane & 31) * 4);
    const uint32_t b = scales[((int64_t)u * R + r) * MX_UNITS + ((lane & 31) >> 2)];
    const float s = b == 255 ? __uint_as_float(0x7FC00000u) : b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23);
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = code_value(w >> (4 * j)) * s;
    const int64_t k = (int64_t)u * MX_UNIT + (lane & 31) * 8;
    T* const dst = Y + r * ldy + k;
    typedef typename Piece<T>::V V;
    if constexpr (sizeof(T) == 4) {
        if (k + 8 <= K) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                reinterpret_cast<V*>(dst)[i] = V{__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3])};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < K) dst[j] = f[j];
        }
    } else {
        const uint32_t o[4] = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
        if (k + 8 <= K) *reinterpret_cast<V*>(dst) = V{o[0], o[1], o[2], o[3]};
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < K) dst[j] = (T)(o[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// One workgroup per fragment and unit: thread (step, half, lane) moves one lane's 16 bytes, the first 64 threads the scale words.  Bound by HBM: 8 x 28672 x
// 4096 184 us, 499 MB read and as many written at 5.4 TB/s.
__global__ __launch_bounds__(256) void k_mx4_pack(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int64_t all_rows, int U,
                                                  bool gated, int64_t frags, uint8_t* __restrict__ w_vals, uint8_t* __restrict__ w_meta)
{
    const int u = blockIdx.x % U;
    const int64_t f = blockIdx.x / U, expert = f / frags, c0 = (f - expert * frags) * MX_FRAG;
    const int t = threadIdx.x >> 7, half = (threadIdx.x >> 6) & 1, n = threadIdx.x & 15, q = (threadIdx.x >> 4) & 3;
    auto row_of = [&](int64_t c) { return expert * rows + (gated ? (c & 1) * (rows >> 1) + (c >> 1) : c); };
    const int64_t c = c0 + mx4_channel(half, n);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (c < rows) v = *reinterpret_cast<const uint4*>(codes + (row_of(c) * U + u) * MX_UNITB + (2 * q + t) * 16);
    reinterpret_cast<uint4*>(w_vals + (f * U + u) * MX_FRAGB)[threadIdx.x] = v;
    if (threadIdx.x < 64) {
        uint32_t w = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t ch = c0 + mx4_channel(h, n);
            if (ch < rows) w |= (uint32_t)*reinterpret_cast<const uint16_t*>(scales + ((int64_t)u * all_rows + row_of(ch)) * MX_UNITS + 2 * q) << (16 * h);
        }
        reinterpret_cast<uint32_t*>(w_meta + (f * U + u) * MX_FRAGS)[threadIdx.x] = w;
    }
}

}  // namespace ss

using namespace ss;

static bool valid_in(ss_act_dtype t) { return t == SS_IN_F32 || t == SS_IN_BF16; }
static int in_size(ss_act_dtype t) { return t == SS_IN_F32 ? 4 : 2; }

template <typename T, int CHUNKS>
static ss_status launch_quant(const void* X, int64_t M, int64_t K, int64_t ldx, const int32_t* rows, int64_t R, void* codes, void* scales, hipStream_t hs)
{
    const int U = (int)mx4_units(K), per_row = (U + 2 * CHUNKS - 1) / (2 * CHUNKS);
    const int64_t blocks = (R * per_row + 3) / 4;
    if (!mx4_grid_fits(blocks, 256)) return SS_ERR_SHAPE;
    hipLaunchKernelGGL((k_mx4_quant<T, CHUNKS>), dim3((uint32_t)blocks), dim3(256), 0, hs, static_cast<const T*>(X), M, K, ldx, rows, R, U, static_cast<uint8_t*>(codes),
                       static_cast<uint8_t*>(scales), per_row, make_div(per_row));
    return launch_status();
}

extern "C" int64_t mx4_row_bytes(int64_t K) { return K < 1 || K > MX_MAX_K ? -1 : mx4_units(K) * MX_UNITB; }
extern "C" int64_t mx4_row_scales(int64_t K) { return K < 1 || K > MX_MAX_K ? -1 : mx4_units(K) * MX_UNITS; }

extern "C" ss_status mx4_quant(const void* X, ss_act_dtype in_dtype, int64_t M, int64_t K, int64_t ldx, const int32_t* rows, int64_t R, void* codes,
                               void* scales, void* stream)
{
    if (!valid_in(in_dtype)) return SS_ERR_DTYPE;
    if (M < 0 || R < 0 || M > MX_MAX_ROWS || R > MX_MAX_ROWS || K < 1 || K > MX_MAX_K || ldx < K || (!rows && R != M)) return SS_ERR_SHAPE;
    if (R == 0) return SS_OK;
    if ((!X && M > 0) || !codes || !scales) return SS_ERR_NULL;
    if (((uintptr_t)X & (in_size(in_dtype) - 1)) || ((uintptr_t)rows & 3) || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 15)) return SS_ERR_SHAPE;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    return in_dtype == SS_IN_F32 ? launch_quant<float, 1>(X, M, K, ldx, rows, R, codes, scales, hs) : launch_quant<uint16_t, 2>(X, M, K, ldx, rows, R, codes, scales, hs);
}

extern "C" ss_status mx4_dequant(const void* codes, const void* scales, int64_t R, int64_t K, ss_act_dtype out_dtype, void* Y, int64_t ldy, void* stream)
{
    if (!valid_in(out_dtype)) return SS_ERR_DTYPE;
    if (R < 0 || R > MX_MAX_ROWS || K < 1 || K > MX_MAX_K || ldy < K) return SS_ERR_SHAPE;
    if (R == 0) return SS_OK;
    if (!codes || !scales || !Y) return SS_ERR_NULL;
    if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 15) || ((uintptr_t)Y & (in_size(out_dtype) - 1))) return SS_ERR_SHAPE;
    const int U = (int)mx4_units(K), per_row = (U + 1) / 2;
    const int64_t blocks = (R * per_row + 3) / 4;
    if (!mx4_grid_fits(blocks, 256)) return SS_ERR_SHAPE;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (out_dtype == SS_IN_F32)
        hipLaunchKernelGGL(k_mx4_dequant<float>, dim3((uint32_t)blocks), dim3(256), 0, hs, static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), R, K, U,
                           static_cast<float*>(Y), ldy, per_row, make_div(per_row));
    else
        hipLaunchKernelGGL(k_mx4_dequant<uint16_t>, dim3((uint32_t)blocks), dim3(256), 0, hs, static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), R, K, U,
                           static_cast<uint16_t*>(Y), ldy, per_row, make_div(per_row));
    return launch_status();
}

static bool valid_weights(int64_t E, int64_t O, int64_t K, int gated)
{
    return E >= 1 && E <= MX_MAX_EXPERTS && O >= 0 && O < (1 << 22) && K >= 1 && K <= MX_MAX_K && (gated == 0 || gated == 1);
}

extern "C" ss_status mx4_packed_sizes(int64_t E, int64_t O, int64_t K, int gated, size_t* vals_bytes, size_t* meta_bytes)
{
    if (!valid_weights(E, O, K, gated)) return SS_ERR_SHAPE;
    if (!vals_bytes || !meta_bytes) return SS_ERR_NULL;
    const size_t n = (size_t)(E * mx4_frags(O << gated) * mx4_units(K));
    *vals_bytes = n * MX_FRAGB;
    *meta_bytes = n * MX_FRAGS;
    return SS_OK;
}

extern "C" ss_status mx4_pack(const void* codes, const void* scales, int64_t E, int64_t O, int64_t K, int gated, void* w_vals, void* w_meta, void* stream)
{
    if (!valid_weights(E, O, K, gated)) return SS_ERR_SHAPE;
    if (O == 0) return SS_OK;
    if (!codes || !scales || !w_vals || !w_meta) return SS_ERR_NULL;
    if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 15) || ((uintptr_t)w_vals & 15) || ((uintptr_t)w_meta & 15)) return SS_ERR_SHAPE;
    const int64_t rows = O << gated, U = mx4_units(K), frags = mx4_frags(rows);
    if (E * rows > MX_MAX_ROWS * 64 || !mx4_grid_fits(E * frags * U, 256)) return SS_ERR_SHAPE;
    hipLaunchKernelGGL(k_mx4_pack, dim3((uint32_t)(E * frags * U)), dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint8_t*>(codes),
                       static_cast<const uint8_t*>(scales), rows, E * rows, (int)U, gated != 0, frags, static_cast<uint8_t*>(w_vals), static_cast<uint8_t*>(w_meta));
    return launch_status();
}
