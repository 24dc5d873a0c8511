// Products of microscaled 4-bit operands on tiles of 128 channels x 16 or 32 token rows whose rows are short (mx4_gemm, mx4_grouped_gemm).
//
// Y = X W^T over rows of one to four units.  What bounds them is the start and the end of a workgroup, a chain of waits (offsets, operands, sums, stores)
// around a few instructions.  So a wavefront takes a fragment and its rows alone: it requests all operands at once into registers, shares nothing and
// waits for nobody, and five to eight such wavefronts on a SIMD hide each other's waits.  (The kernel for few tokens gives two wavefronts of four
// nothing to do with rows of two units and joins sums in LDS; mx4_mid.hip has one or two workgroups on a compute unit, whose ring starts and ends with the tile.)
// Two fragments' worth of rows, 64, measured 42.3 us where 32 measure 23.9: a third as many wavefronts fit.  A loop over a tile's rows with the weights
// kept takes 20.8 to 21.5 there, but 12.6 to 16.5 for 8000 rows, 64 experts, 256 -> 1024 in place of 12.0.
//   500 rows of 64 experts, 512 -> 2048: 10.2 us, 35.7 MB of weights at 3.5 TB/s;  2032 gated rows of 69 experts, 278 -> 1408: 21.1 us (52 MB of weights);
//   8000 rows of 64 experts, 256 -> 1024: 12.6 us (the best other kernel 14.1).
#include "mx4_common.h"
#include "device_info.h"

namespace ss {

// A wavefront takes a fragment of 32 channels and a tile of 16 TB token rows over the whole row of NU units; the four of a workgroup have neighbouring
// fragments of the same tile.  All operands go from global memory straight into registers at once.
template <int NU, int TB, bool GROUPED>
__global__ __launch_bounds__(256) void k_mx4_short(mx4_call c, int panels, int tiles, Div by)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    // Neighbouring workgroups of an XCD share a panel's weights (dense) or a tile's rows (grouped).
    const int id = xcd_run(blockIdx.x, panels * tiles), at = quot(id, by);
    const int panel = GROUPED ? id - at * panels : at, slot = GROUPED ? at : id - at * tiles;
    const int f = panel * 4 + wave;
    if (f >= c.frags) return;
    mx4_rows t = {0, slot * 16 * TB, min(16 * TB, c.R - slot * 16 * TB)};
    if constexpr (GROUPED) t = mx4_find(c.offsets, c.E, c.R, 16 * TB, slot);
    if (t.count <= 0) return;
    const bool none = GROUPED && t.expert == c.E;
    const int64_t first = ((int64_t)(none ? 0 : t.expert) * c.frags + f) * NU, xm_next = (int64_t)c.R * MX_UNITS;
    const uint8_t *const wv = c.w_vals + first * MX_FRAGB, *const wm = c.w_meta + first * MX_FRAGS;
    const uint8_t *const xv = c.codes + (int64_t)t.first * (NU * MX_UNITB), *const xm = c.scales + (int64_t)t.first * MX_UNITS;
    v4i w[NU][4], x[NU][TB][2];
    int sw[NU], sx[NU][TB];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
#pragma unroll
        for (int s = 0; s < 4; ++s) w[u][s] = *reinterpret_cast<const v4i*>(wv + u * MX_FRAGB + s * 1024 + (uint32_t)(lane * 16));
        sw[u] = *reinterpret_cast<const int*>(wm + u * MX_FRAGS + (uint32_t)(lane * 4));
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            const uint32_t row = min(16 * b + n, t.count - 1);
#pragma unroll
            for (int s = 0; s < 2; ++s) x[u][b][s] = *reinterpret_cast<const v4i*>(xv + u * MX_UNITB + s * 16 + (row * (NU * MX_UNITB) + q * 32));
            sx[u][b] = *reinterpret_cast<const uint16_t*>(xm + u * xm_next + (row * MX_UNITS + q * 2));
        }
    }
    v4f acc[2][TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[0][b] = acc[1][b] = v4f{0, 0, 0, 0};
    __builtin_amdgcn_sched_barrier(0);                    // all loads first
    unroll<NU>([&](auto u_c) __attribute__((always_inline)) {
        constexpr int u = decltype(u_c)::value;
        unroll<4>([&](auto s) __attribute__((always_inline)) {
            constexpr int T = decltype(s)::value >> 1, H = decltype(s)::value & 1;
#pragma unroll
            for (int b = 0; b < TB; ++b) acc[H][b] = mx4_mma<2 * H + T, T>(w[u][2 * T + H], x[u][b][T], acc[H][b], sw[u], sx[u][b]);
        });
    });
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        if (16 * b + n >= t.count) continue;
        const v4f zero = {0, 0, 0, 0};
        mx4_store8(none ? zero : acc[0][b], none ? zero : acc[1][b], c.Y + (int64_t)(t.first + 16 * b + n) * c.ldy, f * MX_FRAG + 8 * q, c.O, c.gated);
    }
}

template <int NU, int TB> static ss_status launch(const mx4_call& c, hipStream_t stream)
{
    const int64_t panels = (c.frags + 3) / 4, tiles = c.offsets ? mx4_max_tiles(c.R, c.E, 16 * TB) : ((int64_t)c.R + 16 * TB - 1) / (16 * TB);
    if (!mx4_grid_fits(panels * tiles, 256)) return SS_ERR_SHAPE;
    const Div by = make_div(c.offsets ? panels : tiles);
    const dim3 grid((uint32_t)(panels * tiles));
    if (c.offsets) hipLaunchKernelGGL((k_mx4_short<NU, TB, true>), grid, dim3(256), 0, stream, c, (int)panels, (int)tiles, by);
    else hipLaunchKernelGGL((k_mx4_short<NU, TB, false>), grid, dim3(256), 0, stream, c, (int)panels, (int)tiles, by);
    return launch_status();
}
template <int TB> static ss_status launch(const mx4_call& c, hipStream_t stream)
{
    static_assert(MX_SHORT_UNITS == 4, "the cases");
    switch (c.U) {
    case 1: return launch<1, TB>(c, stream);
    case 2: return launch<2, TB>(c, stream);
    case 3: return launch<3, TB>(c, stream);
    case 4: return launch<4, TB>(c, stream);
    }
    return SS_ERR_SHAPE;
}

ss_status launch_mx4_short(const mx4_call& c, int rows, hipStream_t stream) { return rows == 16 ? launch<1>(c, stream) : launch<2>(c, stream); }

}  // namespace ss
