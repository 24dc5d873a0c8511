// mx4_gemm, mx4_grouped_gemm: products of microscaled 4-bit operands.  Entry points and the kernel for few tokens.
#include "mx4_common.h"
#include "device_info.h"

namespace ss {

// A workgroup of four wavefronts takes FW fragments of 32 channels and a tile of 16 TB token rows.  The wavefronts share out the units of
// the row; operands go from global memory straight into registers, DEPTH units ahead.
template <int FW, int TB, int DEPTH, bool GROUPED>
__global__ __launch_bounds__(256) void k_mx4_stream(mx4_call c)
{
    constexpr int ACC = FW * TB * 2;                     // blocks of 16 x 16
    __shared__ __attribute__((aligned(16))) float part[4][ACC][4][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    mx4_rows t = {0, (int)blockIdx.y * 16 * TB, min(16 * TB, c.R - (int)blockIdx.y * 16 * TB)};
    if constexpr (GROUPED) t = mx4_find(c.offsets, c.E, c.R, 16 * TB, blockIdx.y);
    if (t.count <= 0) return;
    const bool none = GROUPED && t.expert == c.E;
    const int f0 = blockIdx.x * FW;
    const uint8_t *wv[FW], *wm[FW], *xv[TB], *xm[TB];
#pragma unroll
    for (int f = 0; f < FW; ++f) {
        const int64_t at = ((int64_t)(none ? 0 : t.expert) * c.frags + min(f0 + f, c.frags - 1)) * c.U;
        wv[f] = c.w_vals + at * MX_FRAGB + lane * 16;
        wm[f] = c.w_meta + at * MX_FRAGS + lane * 4;
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int64_t row = t.first + min(16 * b + n, t.count - 1);
        xv[b] = c.codes + row * c.U * MX_UNITB + q * 32;
        xm[b] = c.scales + row * MX_UNITS + q * 2;
    }
    struct Unit { v4i w[FW][4], x[TB][2]; int sw[FW], sx[TB]; };
    Unit ring[DEPTH];
    v4f acc[FW][2][TB];
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < TB; ++b) acc[f][h][b] = v4f{0, 0, 0, 0};
    auto load = [&](Unit& r, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < FW; ++f) {
#pragma unroll
            for (int s = 0; s < 4; ++s) r.w[f][s] = *reinterpret_cast<const v4i*>(wv[f] + (int64_t)u * MX_FRAGB + s * 1024);
            r.sw[f] = *reinterpret_cast<const int*>(wm[f] + (int64_t)u * MX_FRAGS);
        }
#pragma unroll
        for (int b = 0; b < TB; ++b) {
#pragma unroll
            for (int s = 0; s < 2; ++s) r.x[b][s] = *reinterpret_cast<const v4i*>(xv[b] + (int64_t)u * MX_UNITB + s * 16);
            r.sx[b] = *reinterpret_cast<const uint16_t*>(xm[b] + (int64_t)u * c.R * MX_UNITS);
        }
    };
    auto multiply = [&](const Unit& r) __attribute__((always_inline)) {
        unroll<4>([&](auto s) __attribute__((always_inline)) {
            constexpr int T = decltype(s)::value >> 1, H = decltype(s)::value & 1;
#pragma unroll
            for (int f = 0; f < FW; ++f)
#pragma unroll
                for (int b = 0; b < TB; ++b) acc[f][H][b] = mx4_mma<2 * H + T, T>(r.w[f][2 * T + H], r.x[b][T], acc[f][H][b], r.sw[f], r.sx[b]);
        });
    };
    const int mine = none ? 0 : (c.U - wave + 3) / 4;           // units wave, wave + 4, ...
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < mine) load(ring[d], wave + 4 * d);
    for (int i = 0; i < mine; i += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (i + d < mine) multiply(ring[d]);
            if (i + d + DEPTH < mine) load(ring[d], wave + 4 * (i + d + DEPTH));
        }
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[wave][(f * TB + b) * 2 + h][i][lane] = acc[f][h][b][i];
    __syncthreads();
    // A thread adds two neighbouring channels of a row, in the order of the wavefronts.
    for (int i = threadIdx.x; i < FW * TB * 256; i += 256) {
        const int row = (i >> 4) & 15, pair = i & 15, f = i / (256 * TB), b = (i >> 8) % TB, ch = (f0 + f) * MX_FRAG + 2 * pair;
        if (16 * b + row >= t.count) continue;
        const int a = (f * TB + b) * 2 + ((pair >> 1) & 1), e = 2 * (pair & 1), l = 16 * (pair >> 2) + row;
        float v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j] = ((part[0][a][e + j][l] + part[1][a][e + j][l]) + part[2][a][e + j][l]) + part[3][a][e + j][l];
        uint16_t* const y = c.Y + (int64_t)(t.first + 16 * b + row) * c.ldy;
        if (c.gated) {
            if ((ch >> 1) < c.O) y[ch >> 1] = (uint16_t)pack_bf16x2(mx4_gate(v[0], v[1]), 0.0f);
        } else {
            const uint32_t w = pack_bf16x2(v[0], v[1]);
            if (ch + 2 <= c.O) *reinterpret_cast<piece4_t*>(y + ch) = w;
            else if (ch < c.O) y[ch] = (uint16_t)w;
        }
    }
}

template <bool GROUPED> static ss_status launch_mx4_stream(const mx4_call& c, int64_t tiles, hipStream_t stream)
{
    hipLaunchKernelGGL((k_mx4_stream<1, 2, 4, GROUPED>), dim3((uint32_t)c.frags, (uint32_t)tiles), dim3(256), 0, stream, c);
    return launch_status();
}

}  // namespace ss

using namespace ss;

extern "C" size_t mx4_gemm_workspace_bytes(int64_t R, int64_t E, int64_t O, int64_t K, int gated)
{
    (void)R; (void)E; (void)O; (void)K; (void)gated;
    return 0;
}

static ss_status mx4_product(bool grouped, const void* codes, const void* scales, const int32_t* offsets, const void* w_vals, const void* w_meta, int64_t R,
                             int64_t E, int64_t O, int64_t K, int gated, void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream)
{
    if (R < 0 || R > MX_MAX_ROWS || E < 1 || E > MX_MAX_EXPERTS || O < 0 || K < 1 || K > MX_MAX_K || (gated != 0 && gated != 1) || ldy < O || ldy >= (1 << 22))
        return SS_ERR_SHAPE;
    if (workspace_bytes > 0 && !workspace) return SS_ERR_NULL;
    if ((uintptr_t)workspace & 15) return SS_ERR_WORKSPACE;
    if (R == 0 || O == 0) return SS_OK;
    if (!codes || !scales || (grouped && !offsets) || !w_vals || !w_meta || !Y) return SS_ERR_NULL;
    if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 15) || ((uintptr_t)offsets & 3) || ((uintptr_t)w_vals & 15) || ((uintptr_t)w_meta & 15) || ((uintptr_t)Y & 1))
        return SS_ERR_SHAPE;
    mx4_call c = {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), offsets, static_cast<const uint8_t*>(w_vals),
                  static_cast<const uint8_t*>(w_meta), (int)R, (int)E, (int)O, (int)mx4_units(K), (int)mx4_frags(O << gated),
                  static_cast<uint16_t*>(Y), ldy, gated != 0};
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (c.U >= MX_TILE_UNITS && R >= 192 * E) return launch_mx4_tile(c, hs);
    return grouped ? launch_mx4_stream<true>(c, mx4_max_tiles(R, E, 32), hs) : launch_mx4_stream<false>(c, (R + 31) / 32, hs);
}

extern "C" ss_status mx4_gemm(const void* codes, const void* scales, const void* w_vals, const void* w_meta, int64_t M, int64_t O, int64_t K, int gated,
                              void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream)
{
    return mx4_product(false, codes, scales, nullptr, w_vals, w_meta, M, 1, O, K, gated, Y, ldy, workspace, workspace_bytes, stream);
}

extern "C" ss_status mx4_grouped_gemm(const void* codes, const void* scales, const int32_t* offsets, const void* w_vals, const void* w_meta, int64_t R,
                                      int64_t E, int64_t O, int64_t K, int gated, void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream)
{
    return mx4_product(true, codes, scales, offsets, w_vals, w_meta, R, E, O, K, gated, Y, ldy, workspace, workspace_bytes, stream);
}
