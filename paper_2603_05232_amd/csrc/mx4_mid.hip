// Products of microscaled 4-bit operands on tiles of 128 channels x 32, 64 or 128 token rows (mx4_gemm, mx4_grouped_gemm).
//
// A workgroup of eight wavefronts takes one tile.  Operands go through a ring of D units in LDS, filled by direct loads.  The wavefronts meet once a unit,
// when each of them holds its operands: the unit's slot is then free for unit u + D, and unit u + 1 has landed, whose operands are read while
// unit u multiplies.
//
// Y = X W^T between a stream of weights and large tiles.  A unit of a 128 x 128 tile has 512 cycles of products, 470 of reads in LDS and 34 KB of direct loads,
// and takes some 1150 cycles; without the loads 0.8 of that, without the reads 0.75, without both 0.65.  So no one of them bounds it but the meeting, once
// for every 16 products of a wavefront, up to which all three have to be done.  Wider tiles would leave compute units without one.
// 777 x 5003 -> 4099, one tile of 128 rows for a compute unit: 17.1 us in a trace, 1.86 PFLOP/s, a third of it the start (first loads) and the end;
// 2000 rows of 64 experts, 2048 -> 1408, tiles of 64 rows: 27.3 us, 100.5 MB fetched at 3.7 TB/s, the rest start and end.
//
// With few tiles and long rows the units of a row are split into ranges, a workgroup each; their sums go through the workspace and a second kernel
// adds them in the order of the ranges.
#include "mx4_common.h"
#include "mx4_loads.h"
#include "device_info.h"

namespace ss {

// WO x WT wavefronts of FW fragments of 32 channels x TW blocks of 16 rows
template <int FW, int TW, int WO, int WT, int D> struct MidShape {
    static constexpr int ROWS = 16 * TW * WT, A = 4 * MX_FRAGB, B = ROWS * MX_UNITB, MA = 4 * MX_FRAGS, MB = ROWS * MX_UNITS;
    static constexpr int B_OFF = A, MA_OFF = A + B, MB_OFF = MA_OFF + MA, UNIT = MB_OFF + MB, LDS = D * UNIT;
    static constexpr int NB = ROWS >= 64 ? ROWS / 64 : 1;         // loads of token rows of a wavefront for a unit
    static constexpr int LOADS = 3 + NB;                          // all its loads: half a fragment, rows, scales
    static constexpr int NV = 2 * FW * TW;                        // a wavefront's vectors of four sums
    static_assert(FW * WO == 4 && WO * WT == 8 && LDS <= 160 * 1024, "whole shares");
};

template <int FW, int TW, int WO, int WT, int D, bool GROUPED>
__global__ __launch_bounds__(512) void k_mx4_mid(mx4_call c, int panels, int tiles, Div by, Div by_items, KRanges ranges, int S_ranges, v4f* __restrict__ ws)
{
    typedef MidShape<FW, TW, WO, WT, D> S;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int wo = wave % WO, wt = wave / WO, U = c.U;
    const uint32_t lds0 = lds_address(smem);
    // Neighbouring workgroups of an XCD share a panel's weights (dense) or a tile's rows (grouped).
    const int id = xcd_run(blockIdx.x, panels * tiles * S_ranges), range = quot(id, by_items), item = id - range * panels * tiles, at = quot(item, by);
    const int panel = GROUPED ? item - at * panels : at, slot = GROUPED ? at : item - at * tiles;
    mx4_rows t = {0, slot * S::ROWS, min(S::ROWS, c.R - slot * S::ROWS)};
    if constexpr (GROUPED) t = mx4_find(c.offsets, c.E, c.R, S::ROWS, slot);
    if (t.count <= 0) return;
    const bool none = GROUPED && t.expert == c.E;

    // Sources of a unit: half of fragment wave / 2, token rows 8 (8 i + wave) .. + 7 (32 rows: of wavefronts 0 .. 3), and scales: fragment `wave`'s of wavefronts
    // 0 .. 3, those of 32 rows of the others, as far as there are rows in the tile's shape.
    const int64_t first_frag = (int64_t)(none ? 0 : t.expert) * c.frags + panel * 4, begin = range_first(ranges, range);
    const int frags_here = c.frags - panel * 4;
    const bool weights = wave < 4;
    const uint8_t* av = c.w_vals + ((first_frag + min(wave / 2, frags_here - 1)) * U + begin) * MX_FRAGB + (wave & 1) * 2048;
    const uint8_t* bv = c.codes + ((int64_t)t.first * U + begin) * MX_UNITB;
    const uint8_t* mv = weights ? c.w_meta + ((first_frag + min(wave, frags_here - 1)) * U + begin) * MX_FRAGS : c.scales + (begin * c.R + t.first) * MX_UNITS;
    const int64_t m_next = weights ? MX_FRAGS : (int64_t)c.R * MX_UNITS;
    uint32_t boff[S::NB];
#pragma unroll
    for (int i = 0; i < S::NB; ++i) {
        const int row = 8 * (8 * i + wave) + (lane >> 3);
        boff[i] = (uint32_t)min(row, t.count - 1) * (uint32_t)(U * MX_UNITB) + mx4_place((lane & 7) ^ swz(row)) * 16;
    }
    const uint32_t moff = weights ? (uint32_t)lane * 4 : (uint32_t)min((wave & 3) * 32 + (lane >> 1), t.count - 1) * MX_UNITS + (lane & 1) * 4;
    const uint32_t lane16 = lane * 16;
    const int low = wave - 4, b_mask = S::ROWS >= 64 ? -1 : low, m_mask = low | ((wave & 3) * 32 - S::ROWS);      // negative where there is something to load
    const uint32_t a_dst = lds0 + wave * 2048, b_dst = lds0 + S::B_OFF + wave * 1024, m_dst = lds0 + (weights ? S::MA_OFF : S::MB_OFF) + (wave & 3) * 256;
    // Load number `piece` of the next unit, into `slot_off`; without `more` by no lane, so that every wavefront and unit counts the same.  No branch: products
    // that stand before one would be moved behind it, and nothing would run beside the reads any more (777 x 20012 -> 4099: 55 us).
    auto load = [&](auto piece_c, uint32_t slot_off, int more) __attribute__((always_inline)) {
        constexpr int P = decltype(piece_c)::value;
        if constexpr (P < 2) mx4_load16(av + P * 1024, lane16, a_dst + slot_off + P * 1024, more);
        else if constexpr (P < S::LOADS - 1) mx4_load16(bv, boff[P - 2], b_dst + slot_off + (P - 2) * 8192, more & b_mask);
        else {
            mx4_load4(mv, moff, m_dst + slot_off, more & m_mask);
            av += MX_FRAGB;
            bv += MX_UNITB;
            mv += m_next;
        }
    };
    // this wavefront's operands
    const uint32_t ra = wo * FW * MX_FRAGB + lane * 16, rma = S::MA_OFF + wo * FW * MX_FRAGS + lane * 4;
    const uint32_t rb = S::B_OFF + (wt * TW * 16 + n) * ROWB + ((mx4_place(2 * q) ^ swz(n)) << 4), rmb = S::MB_OFF + (wt * TW * 16 + n) * MX_UNITS + 2 * q;

    const int units = __builtin_amdgcn_readfirstlane(none ? 0 : range_units(ranges, range));
#pragma unroll
    for (int d = 0; d < D; ++d) unroll<S::LOADS>([&](auto p) __attribute__((always_inline)) { load(p, d * S::UNIT, d - units); });
    v4f acc[FW][2][TW];
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < TW; ++b) acc[f][h][b] = v4f{0, 0, 0, 0};
    struct Operands { v4i a[2][FW][2], b[2][TW]; int sa[FW], sb[TW]; };
    // operand read number `piece` of READS: a step's rows and weights, the next step's, the scales
    constexpr int SR = 2 * FW + TW, READS = 2 * SR + FW + TW, SN = FW * TW * 2, N = 2 * SN;
    auto read = [&](auto piece_c, Operands& r, uint32_t slot_off) __attribute__((always_inline)) {
        constexpr int P = decltype(piece_c)::value, T = P / SR, Q = P % SR, Z = P - 2 * SR;
        if constexpr (Z >= FW) r.sb[Z - FW] = *reinterpret_cast<const uint16_t*>(smem + rmb + slot_off + (Z - FW) * 128);
        else if constexpr (Z >= 0) r.sa[Z] = *reinterpret_cast<const int*>(smem + rma + slot_off + Z * MX_FRAGS);
        else if constexpr (Q < TW) r.b[T][Q] = *reinterpret_cast<const v4i*>(smem + ((rb + slot_off) ^ (T * 32)) + Q * 2048);
        else r.a[T][(Q - TW) >> 1][(Q - TW) & 1] = *reinterpret_cast<const v4i*>(smem + ra + slot_off + T * 2048 + ((Q - TW) >> 1) * MX_FRAGB + ((Q - TW) & 1) * 1024);
    };
    uint32_t here = 0;
    // One by one between the products: a wavefront issues in order, and a read or a load that has to wait for room in its queue keeps the
    // products behind it from issuing.
    auto unit = [&](Operands& now, Operands& next, int u) __attribute__((always_inline)) {
        wait_vmcnt<(D - 2) * S::LOADS>();                  // unit u + 1 has landed, and this one's operands have arrived
        wait_lgkm0();
        wg_barrier();
        const uint32_t freed = here;
        const int more = u + D - units;                    // a unit to load: negative
        here = here + S::UNIT == D * S::UNIT ? 0 : here + S::UNIT;       // behind the last unit what an older one left is read, for nothing
        __builtin_amdgcn_sched_barrier(0);
        unroll<N>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value, T = i / SN, j = i % SN, b = j / (2 * FW), f = (j >> 1) % FW, h = j & 1;
            constexpr int r0 = i * READS / N, r1 = (i + 1) * READS / N, l0 = i * S::LOADS / N, l1 = (i + 1) * S::LOADS / N;
            acc[f][h][b] = mx4_mma<2 * h + T, T>(now.a[T][f][h], now.b[T][b], acc[f][h][b], now.sa[f], now.sb[b]);
            __builtin_amdgcn_sched_barrier(0);
            unroll<r1 - r0>([&](auto p) __attribute__((always_inline)) { read(std::integral_constant<int, r0 + decltype(p)::value>{}, next, here); });
            unroll<l1 - l0>([&](auto p) __attribute__((always_inline)) { load(std::integral_constant<int, l0 + decltype(p)::value>{}, freed, more); });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    wait_vmcnt<(D - 1) * S::LOADS>();
    wg_barrier();
    Operands r0, r1;
    unroll<READS>([&](auto p) __attribute__((always_inline)) { read(p, r0, 0); });
    int u = 0;
    for (; u + 2 <= units; u += 2) {
        unit(r0, r1, u);
        unit(r1, r0, u + 1);
    }
    if (u < units) unit(r0, r1, u);
    if (S_ranges > 1) {
        v4f* const partial = ws + ((((int64_t)range * panels * tiles + item) * 8 + wave) * S::NV) * 64 + lane;
#pragma unroll
        for (int b = 0; b < TW; ++b)
#pragma unroll
            for (int f = 0; f < FW; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h) partial[((b * FW + f) * 2 + h) * 64] = acc[f][h][b];
        return;
    }
#pragma unroll
    for (int b = 0; b < TW; ++b) {
        const int row = 16 * (wt * TW + b) + n;
        if (row >= t.count) continue;
        uint16_t* const y = c.Y + (int64_t)(t.first + row) * c.ldy;
#pragma unroll
        for (int f = 0; f < FW; ++f) mx4_store8(acc[f][0][b], acc[f][1][b], y, (panel * 4 + wo * FW + f) * MX_FRAG + 8 * q, c.O, c.gated);
    }
}

// adds the sums of the ranges, a thread what one lane of the workgroups before had
template <int FW, int TW, int WO, int WT, int D, bool GROUPED>
__global__ __launch_bounds__(512) void k_mx4_mid_add(mx4_call c, int panels, int tiles, Div by, int S_ranges, const v4f* __restrict__ ws)
{
    typedef MidShape<FW, TW, WO, WT, D> S;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int wo = wave % WO, wt = wave / WO;
    const int item = blockIdx.x, at = quot(item, by);
    const int panel = GROUPED ? item - at * panels : at, slot = GROUPED ? at : item - at * tiles;
    mx4_rows t = {0, slot * S::ROWS, min(S::ROWS, c.R - slot * S::ROWS)};
    if constexpr (GROUPED) t = mx4_find(c.offsets, c.E, c.R, S::ROWS, slot);
    if (t.count <= 0) return;
    const v4f* from = ws + (((int64_t)item * 8 + wave) * S::NV) * 64 + lane;
    const int64_t next = (int64_t)panels * tiles * 8 * S::NV * 64;
    v4f sum[S::NV];
#pragma unroll
    for (int i = 0; i < S::NV; ++i) sum[i] = from[i * 64];
    for (int r = 1; r < S_ranges; ++r) {
        from += next;
#pragma unroll
        for (int i = 0; i < S::NV; ++i) sum[i] += from[i * 64];
    }
#pragma unroll
    for (int b = 0; b < TW; ++b) {
        const int row = 16 * (wt * TW + b) + n;
        if (row >= t.count) continue;
        uint16_t* const y = c.Y + (int64_t)(t.first + row) * c.ldy;
#pragma unroll
        for (int f = 0; f < FW; ++f) mx4_store8(sum[(b * FW + f) * 2], sum[(b * FW + f) * 2 + 1], y, (panel * 4 + wo * FW + f) * MX_FRAG + 8 * q, c.O, c.gated);
    }
}

template <int FW, int TW, int WO, int WT, int D, bool GROUPED> static ss_status launch_kind(const mx4_call& c, int ranges, void* ws, hipStream_t stream)
{
    typedef MidShape<FW, TW, WO, WT, D> S;
    const int64_t panels = (c.frags + 3) / 4, tiles = GROUPED ? mx4_max_tiles(c.R, c.E, S::ROWS) : ((int64_t)c.R + S::ROWS - 1) / S::ROWS, items = panels * tiles;
    if (!mx4_grid_fits(items * ranges, 512)) return SS_ERR_SHAPE;
    if (allow_dynamic_lds<k_mx4_mid<FW, TW, WO, WT, D, GROUPED>>(S::LDS) != SS_OK) return SS_ERR_HIP;
    const Div by = make_div(GROUPED ? panels : tiles);
    hipLaunchKernelGGL((k_mx4_mid<FW, TW, WO, WT, D, GROUPED>), dim3((uint32_t)(items * ranges)), dim3(512), S::LDS, stream, c, (int)panels, (int)tiles, by, make_div(items),
                       k_ranges(c.U, ranges), ranges, static_cast<v4f*>(ws));
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    if (ranges == 1) return SS_OK;
    hipLaunchKernelGGL((k_mx4_mid_add<FW, TW, WO, WT, D, GROUPED>), dim3((uint32_t)items), dim3(512), 0, stream, c, (int)panels, (int)tiles, by, ranges, static_cast<const v4f*>(ws));
    return launch_status();
}
template <int FW, int TW, int WO, int WT, int D> static ss_status launch(const mx4_call& c, int ranges, void* ws, hipStream_t stream)
{
    return c.offsets ? launch_kind<FW, TW, WO, WT, D, true>(c, ranges, ws, stream) : launch_kind<FW, TW, WO, WT, D, false>(c, ranges, ws, stream);
}

ss_status launch_mx4_mid(const mx4_call& c, int rows, int ranges, void* ws, hipStream_t stream)
{
    // The wavefronts' shares by the fewest LDS reads among those that measured alike; 64 rows as <1, 2, 4, 2, 3>: 29.5 against 28.8 us (2000 rows of 64 experts, 2048 ->
    // 1408); 128 as <1, 4, 4, 2, 4>: 14.4 against 12.7 (200 x 4096 -> 14336).  Two groups that multiply one step of a unit each and join their sums at the
    // end read a third less and took 30.5 and 13.0.  Four units in flight in place of three: 36.8 where 64 rows take 30.5 (one workgroup a
    // compute unit instead of two), no difference at 128.
    return rows == 32 ? launch<1, 1, 4, 2, 3>(c, ranges, ws, stream) : rows == 64 ? launch<2, 1, 2, 4, 3>(c, ranges, ws, stream) : launch<2, 2, 2, 4, 3>(c, ranges, ws, stream);
}

}  // namespace ss
