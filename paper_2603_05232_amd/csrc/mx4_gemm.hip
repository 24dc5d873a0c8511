// mx4_gemm, mx4_grouped_gemm: products of microscaled 4-bit operands.  Entry points and the kernel for few tokens.
#include "mx4_common.h"
#include "device_info.h"
#include <math.h>

namespace ss {

// Y = X W^T of few token rows.  A workgroup of W wavefronts takes a fragment of 32 channels and a tile of 16 TB token rows.  The wavefronts share out the
// units of the row; operands go from global memory straight into registers, DEPTH units ahead (a weight is used once: LDS would only
// add a copy), and the wavefronts' sums meet in LDS.  Bound by the stream of weights; one fragment makes the most workgroups, which is what keeps it going.
//   1 x 3584 -> 37888: 11.5 us, 72.2 MB fetched at 6.3 TB/s;  16 tokens x 2 experts, gated, 8 experts 4096 -> 14336: 83.8 us, 499.7 MB at 6.0 TB/s
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

// The kernel of a product: tiles of 16 or 32 rows of the kernel for few tokens, MX_SHORT + 16 or 32 of mx4_short.hip (rows of MX_SHORT_UNITS and fewer), MX_MID + 32,
// 64 or 128 of mx4_mid.hip, 256 of mx4_tile.hip.  Which is the fastest goes by an estimate of every kernel's time in us: its launch, then the longest of what its workgroups take one after the other (time of a
// unit and of a workgroup's start and end, times workgroups for each compute unit), what the weights take that are read once for every tile of
// rows (MB over MB per us, L2 and memory-side cache), and the weights from HBM.  The group sizes lie on the device: E experts are taken to have R / E rows
// each, and half a tile more.  Constants fitted to the times of all on 137 shapes (R = 1 .. 54000, 1 .. 79 units, 64 .. 37888 channels, 1 to 128
// experts): the choice is 1.02 of the fastest on average, 1.3 at most.  Times of 16 | 32 | MID + 32 | 64 | 128 | 256, us:
//   1 x 3584 -> 37888          14.0 |  15.3 |  18.4 |  19.1 |   -   |   -       200 x 4096 -> 14336       49.3 |  36.8 |  24.3 | 17.8 | 14.9 | 27.3
//   32 x 3584 -> 37888         24.2 |  19.7 |  20.0 |  19.9 | 26.9 | 25.9       777 x 5003 -> 4099        77.7 |  50.9 |  30.0 | 20.7 | 18.1 | 33.6
//   64 x 3584 -> 4608           7.2 |   7.9 |   7.3 |   7.8 |   9.6 | 22.0       3200 x 4096 -> 4096        183 |   136 |  76.2 | 51.9 | 51.5 | 33.4
//   8192 x 256 -> 512          17.9 |  18.2 |   8.2 |   5.8 |   5.8 | 10.1       4000 x 256 -> 4096        56.9 |  59.7 |  23.4 | 15.3 | 15.2 | 13.7
//   500 rows, 8 experts, 4096 -> 4096   43.8 | 33.6 | 30.4 | 22.5 | 27.4 | 29.7      4000 rows, 64 experts, 2048 -> 1408   61.9 | 62.0 | 36.3 | 32.6 | 39.5 | 39.5
// and of rows of one to four units 16 | 32 | SHORT + 16 | 32 | the best of MID | 256:
//   3 x 436 -> 8870             3.1 |   3.4 |   3.1 |   3.1 |   3.8 |   8.9       1 x 1024 -> 4096          3.0 |   3.2 |   3.5 |  3.6 |  4.3 |  9.7
//   476 x 303 -> 1000           4.4 |   4.3 |   3.4 |   4.0 |   4.0 |  12.6       200 x 512 -> 16384       15.1 |  16.5 |   8.7 |  8.4 |  5.9 | 10.0
//   500 rows, 64 experts, 512 -> 2048   17.4 | 23.4 | 10.6 | 10.0 | 13.7 | 21.4      8000 rows, 64 experts, 256 -> 1024   44.9 | 44.1 | 13.9 | 12.6 | 14.1 | 19.1
//   300 gated rows, 60 experts, 1024 -> 1408   24.0 | 33.2 | 21.2 | 21.9 | 23.8 | 52.4      8000 rows, 16 experts, 512 -> 2048   85 | 82 | 33 | 28 | 24.6 | 21.8
// Ranges of units (the second kernel, its launch and MB of sums: 3.5 us + 0.36 a MB), split over unsplit: 256 x 18944 -> 3584 23.5 | 33.8, 777 x 18944 -> 512 17.8 | 28.0,
// 100 x 14336 -> 4096 15.4 | 22.3; 64 x 4096 -> 4096, whose estimate is against it, 8.7 | 6.1.
// The kernel of 16 rows takes eight wavefronts, two units each ahead, where rows have 16 units and more, otherwise four (1 x 18944 -> 3584 10.3 against 12.4, 32 gated
// rows of 8 experts 4096 -> 14336 83.7 against 88.6; 512 rows of 64 experts, 8 units, 26.4 against 22.2).
constexpr int MX_MID = 1000, MX_SHORT = 2000;
struct mx4_plan { int kernel, ranges; };
static mx4_plan mx4_choose(int64_t R, int64_t E, int64_t U, int64_t frags, int64_t cus, size_t ws_bytes)
{
    const bool many = E > 1;
    const double used = many ? (double)E * (1.0 - pow(1.0 - 1.0 / (double)E, (double)R)) : 1.0, MB = (double)(frags * U * (MX_FRAGB + MX_FRAGS)) / 1e6;
    const double hbm = used * MB / 5.2, panels = (double)((frags + 3) / 4), wide = (double)((frags + 7) / 8), u = (double)U;
    auto fits = [&](int64_t T, int64_t threads) { return mx4_grid_fits((frags + 3) / 4 * mx4_max_tiles(R, E, T), threads); };
    auto tiles = [&](int64_t T) { return many ? fmax(used, (double)R / (double)T + 0.5 * used) : (double)((R + T - 1) / T); };
    // workgroups of a compute unit one after the other; a last round that only some have counts as much more than its share as the others wait
    auto rounds = [](double x, double more) { const double part = x - floor(x); return x <= 1.0 ? 1.0 : floor(x) + (part > 0.0 ? fmin(1.0, more + part) : 0.0); };
    mx4_plan best = {};
    double time = INFINITY;
    auto offer = [&](mx4_plan p, double us) {
        if (us < time) { best = p; time = us; }
    };
    const struct { int rows; double launch, rate, row, start, unit; } few[] = {{16, 2.52, 8.5, 0.0, 0.39, 0.056}, {32, 2.67, 5.85, 0.18, 0.73, 0.086}};
    for (const auto& f : few) {
        const double t = tiles(f.rows), shares = (double)frags * t / (double)cus;
        offer({f.rows, 1}, f.launch + fmax(fmax(MB * t / f.rate * (many ? 0.94 : 1.0), f.row * u), fmax((f.start + f.unit * u) * (many ? 1.6 : 1.0) * shares, hbm)));
    }
    if (U <= MX_SHORT_UNITS) {
        const struct { int rows; double launch, start, unit, row; } whole[] = {{16, 2.6, 0.07, 0.41, 0.27}, {32, 2.65, 0.07, 0.70, 0.40}};
        for (const auto& s : whole)
            if (fits(s.rows, 256)) offer({MX_SHORT + s.rows, 1}, s.launch + fmax(fmax((s.start + s.unit * u) * (many ? 1.2 : 1.0) * panels * tiles(s.rows) / (double)cus, s.row * u), 1.13 * hbm));
    }
    const struct { int rows; double launch, unit, ends, hbm, more; } mid[] = {{32, 2.29, 0.39, 0.85, 1.13, 0.0}, {64, 1.92, 0.40, 1.27, 1.13, 0.33}, {128, 1.67, 0.56, 2.76, 1.67, 0.39}};
    for (const auto& m : mid) {
        const double w = panels * tiles(m.rows);
        if (!fits(m.rows, 512)) continue;
        for (int r = 1; r <= 16 && r <= U; ++r) {
            if (r > 1 && (mx4_mid_bytes(R, E, frags, m.rows, r) > ws_bytes || w * r > 2.0 * (double)cus)) break;
            const double add = r > 1 ? 3.5 + 0.36 * w * r * (double)m.rows * 512.0 / 1e6 : 0.0;
            offer({MX_MID + m.rows, r}, m.launch + fmax((m.unit * ceil(u / r) + m.ends) * (many ? 1.46 : 1.0) * rounds(w * r / (double)cus, m.more), m.hbm * hbm + 1.0) + add);
        }
    }
    const double all = wide * tiles(256) / (double)cus, full = fmin(1.0, all);
    offer({256, 1}, 3.94 + fmax(rounds(all, 0.31) * (fmax(u, 3.0) * (1.02 + 0.69 * full) + (0.8 + 3.43 * full) * (many ? 1.83 : 1.0)), hbm));
    return best;
}

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
