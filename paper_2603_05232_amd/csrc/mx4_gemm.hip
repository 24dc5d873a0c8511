// mx4_gemm, mx4_grouped_gemm: products of microscaled 4-bit operands.  Entry points and the kernel for few tokens.
#include "mx4_choice.h"
#include "device_info.h"

namespace ss {

// Y = X W^T of few token rows.  A workgroup of W wavefronts takes a fragment of 32 channels and a tile of 16 TB token rows.  The wavefronts share out the
// units of the row; operands go from global memory straight into registers, DEPTH units ahead (a weight is used once: LDS would only
// add a copy), and the wavefronts' sums meet in LDS.  Bound by the stream of weights; one fragment makes the most workgroups, which is what keeps it going.
//   1 x 3584 -> 37888: 11.6 us, 72.2 MB fetched at 6.2 TB/s, part of it from the memory-side cache (13.5 from HBM);  16 tokens x 2 experts, gated, 8 experts
//   4096 -> 14336: 81 .. 84 us, 499.7 MB at 6.0 TB/s
template <int W, int TB, int DEPTH, bool GROUPED>
__global__ __launch_bounds__(64 * W) void k_mx4_stream(mx4_call c)
{
    constexpr int ACC = TB * 2;                          // blocks of 16 x 16
    __shared__ __attribute__((aligned(16))) float part[W][ACC][4][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int slot = blockIdx.z * gridDim.y + blockIdx.y;
    mx4_rows t = {0, slot * 16 * TB, min(16 * TB, c.R - slot * 16 * TB)};
    if constexpr (GROUPED) t = mx4_find(c.offsets, c.E, c.R, 16 * TB, slot);
    if (t.count <= 0) return;
    const bool none = GROUPED && t.expert == c.E;
    const int f = blockIdx.x;
    const int64_t at = ((int64_t)(none ? 0 : t.expert) * c.frags + f) * c.U;
    const uint8_t *const wv = c.w_vals + at * MX_FRAGB + lane * 16, *const wm = c.w_meta + at * MX_FRAGS + lane * 4;
    const uint8_t *xv[TB], *xm[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int64_t row = t.first + min(16 * b + n, t.count - 1);
        xv[b] = c.codes + row * c.U * MX_UNITB + q * 32;
        xm[b] = c.scales + row * MX_UNITS + q * 2;
    }
    struct Unit { v4i w[4], x[TB][2]; int sw, sx[TB]; };
    Unit ring[DEPTH];
    v4f acc[2][TB];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[h][b] = v4f{0, 0, 0, 0};
    auto load = [&](Unit& r, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 4; ++s) r.w[s] = *reinterpret_cast<const v4i*>(wv + (int64_t)u * MX_FRAGB + s * 1024);
        r.sw = *reinterpret_cast<const int*>(wm + (int64_t)u * MX_FRAGS);
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
            for (int b = 0; b < TB; ++b) acc[H][b] = mx4_mma<2 * H + T, T>(r.w[2 * T + H], r.x[b][T], acc[H][b], r.sw, r.sx[b]);
        });
    };
    const int mine = none ? 0 : (c.U - wave + W - 1) / W;       // units wave, wave + W, ...
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < mine) load(ring[d], wave + W * d);
    for (int i = 0; i < mine; i += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (i + d < mine) multiply(ring[d]);
            if (i + d + DEPTH < mine) load(ring[d], wave + W * (i + d + DEPTH));
        }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][b * 2 + h][i][lane] = acc[h][b][i];
    __syncthreads();
    // A thread adds two neighbouring channels of a row, in the order of the wavefronts.
    for (int i = threadIdx.x; i < TB * 256; i += 64 * W) {
        const int row = (i >> 4) & 15, pair = i & 15, b = i >> 8, ch = f * MX_FRAG + 2 * pair;
        if (16 * b + row >= t.count) continue;
        const int a = b * 2 + ((pair >> 1) & 1), e = 2 * (pair & 1), l = 16 * (pair >> 2) + row;
        float v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v[j] = part[0][a][e + j][l];
#pragma unroll
            for (int w = 1; w < W; ++w) v[j] += part[w][a][e + j][l];
        }
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

template <int W, int TB, int DEPTH> static ss_status launch_stream(const mx4_call& c, hipStream_t stream)
{
    const int64_t tiles = c.offsets ? mx4_max_tiles(c.R, c.E, 16 * TB) : ((int64_t)c.R + 16 * TB - 1) / (16 * TB);
    const int64_t layers = (tiles + 65534) / 65535;      // of the grid's third dimension
    const dim3 grid((uint32_t)c.frags, (uint32_t)((tiles + layers - 1) / layers), (uint32_t)layers);
    if (c.offsets) hipLaunchKernelGGL((k_mx4_stream<W, TB, DEPTH, true>), grid, dim3(64 * W), 0, stream, c);
    else hipLaunchKernelGGL((k_mx4_stream<W, TB, DEPTH, false>), grid, dim3(64 * W), 0, stream, c);
    return launch_status();
}

}  // namespace ss

using namespace ss;

extern "C" size_t mx4_gemm_workspace_bytes(int64_t R, int64_t E, int64_t O, int64_t K, int gated)
{
    if (R < 1 || R > MX_MAX_ROWS || E < 1 || E > MX_MAX_EXPERTS || O < 1 || O >= (1 << 22) || K < 1 || K > MX_MAX_K || (gated != 0 && gated != 1)) return 0;
    const int64_t frags = mx4_frags(O << gated);
    const mx4_plan p = mx4_choose(R, E, mx4_units(K), frags, cu_count(), SIZE_MAX);
    return p.ranges > 1 ? mx4_mid_bytes(R, E, frags, p.kernel - MX_MID, p.ranges) : 0;
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
    const mx4_plan p = mx4_choose(R, E, c.U, c.frags, cu_count(), workspace_bytes);
    switch (p.kernel) {
    case 16: return c.U >= 16 ? launch_stream<8, 1, 2>(c, hs) : launch_stream<4, 1, 4>(c, hs);
    case 32: return launch_stream<4, 2, 4>(c, hs);
    case 256: return launch_mx4_tile(c, hs);
    case MX_SHORT + 16:
    case MX_SHORT + 32: return launch_mx4_short(c, p.kernel - MX_SHORT, hs);
    }
    return launch_mx4_mid(c, p.kernel - MX_MID, p.ranges, workspace, hs);
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
