// Products of microscaled 4-bit operands on tiles of 256 channels x 256 token rows (mx4_gemm, mx4_grouped_gemm: many rows).
//
// Y = X W^T of many rows.  Bound by power: at 8192 x 16384 -> 8192 the products alone take 60 % of the time at the clock they leave, LDS reads of operands
// 19 %, direct loads 10 %.  So the tile is as large as the registers and LDS allow, which makes the fewest reads of both a product.
//   8192 x 3584 -> 37888: 510 .. 526 us on one card and another, 4.2 .. 4.4 PFLOP/s;  8192 rows of 8 experts, 14336 -> 4096: 268 us, 3.59 (a third round a
//   quarter full; even groups 218);  8192 x 16384 -> 8192: 453 us, 4.86 PFLOP/s;  4000 x 256 -> 4096, one unit a row: 13.7 us
//
// Persistent workgroups of eight wavefronts, two per SIMD, of 128 channels x 64 rows = 8 x 4 blocks of the 16x16x128 instruction; a unit of 256
// values is two steps.
//
// LDS: weights in three slots of a step (16 KB), token rows in three slots of a unit (32 KB), scales of two units.  Direct loads fill
// them; those of a step are spread from one meeting of the workgroup to the next.  The workgroup meets once a step, behind
// instruction 14: the reads of this step's operands have returned then, so the slots they came from are free, and what the reads
// behind the meeting need was requested two steps before or earlier.  The requests run on across tiles; between two there is only
// the epilogue, which stages in the token slot that is free then.
#include "mx4_common.h"
#include "mx4_loads.h"
#include "tile_common.h"
#include "device_info.h"

namespace ss {

constexpr int XT_A = 16 * 1024, XT_B = 32 * 1024, XT_M = 2048;
constexpr int XT_B_OFF = 3 * XT_A, XT_MA_OFF = XT_B_OFF + 3 * XT_B, XT_MB_OFF = XT_MA_OFF + 2 * XT_M, XT_LDS = XT_MB_OFF + 2 * XT_M;      // 152 KB
constexpr int XT_ENDS = 2 * MX_MAX_EXPERTS * 4;          // last tile and last row of every expert
static_assert(XT_LDS + XT_ENDS <= 160 * 1024, "LDS budget");

// acc[2 f + hh][b][i] of lane (n, q): packed channel 32 f + 8 q + 4 hh + i, row 16 b + n of a sub-tile of 128 x 64 of which rows_left rows and cols_left
// columns of Y exist.  Staged 16 rows at a time through the wavefront's own 4 KB, so that every store writes whole pieces of Y's rows.
// All loads in flight are waited for before the first store (the wait counter counts both).
template <bool GATED>
__device__ inline void xt_store(const v4f (&acc)[8][4], bool zeros, uint16_t* __restrict__ Y_sub, uint32_t ldy, int rows_left, int cols_left, uint8_t* stage)
{
    constexpr int ROW = GATED ? 128 : 256, LANES = ROW / 16, ROWS = 64 / LANES;      // bytes of a staged row, lanes that store one, rows of a store
    const int lane = fresh_lane(), n = lane & 15, q = lane >> 4, sr = lane / LANES, sc = lane % LANES;
    const bool vec_ok = (ldy & 7) == 0 && ((uintptr_t)Y_sub & 15) == 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            const v4f v = zeros ? v4f{0, 0, 0, 0} : acc[2 * f][b], w = zeros ? v4f{0, 0, 0, 0} : acc[2 * f + 1][b];
            if constexpr (GATED)
                *reinterpret_cast<uint2*>(stage + n * ROW + (((2 * f + (q >> 1)) ^ (n & 7)) << 4) + 8 * (q & 1)) =
                    make_uint2(pack_bf16x2(mx4_gate(v[0], v[1]), mx4_gate(v[2], v[3])), pack_bf16x2(mx4_gate(w[0], w[1]), mx4_gate(w[2], w[3])));
            else
                *reinterpret_cast<uint4*>(stage + n * ROW + (((4 * f + q) ^ n) << 4)) =
                    make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]));
        }
        if (b == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < 16 / ROWS; ++i) {
            const int r = i * ROWS + sr;
            const uint4 v = *reinterpret_cast<const uint4*>(stage + r * ROW + ((sc ^ (r & (LANES - 1))) << 4));
            if (16 * b + r < rows_left) {
                uint16_t* const dst = Y_sub + ((uint32_t)(16 * b + r) * ldy + 8 * sc);
                if (8 * sc + 8 <= cols_left) {
                    if (vec_ok) store_once(reinterpret_cast<uint4*>(dst), v);
                    else *reinterpret_cast<piece16_t*>(dst) = piece16_t{v.x, v.y, v.z, v.w};
                } else {
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (8 * sc + e < cols_left) dst[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read out before the next block is staged
    }
}

__device__ const uint4 mx4_zeros[256] = {};            // a fragment's codes of a unit that rows lack, and the scales of anything

// The requests run up to three units ahead and into the next tile only, so a tile has at least three.  SHORT: rows have fewer; the units that they lack are
// zeros times what lies in the first unit, with zeros as scale bytes on both sides.
template <bool GROUPED, bool SHORT>
__global__ __launch_bounds__(512) void k_mx4_tile(mx4_call c, int tiles_o)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wo = wave & 1, wt = wave >> 1, n = lane & 15, q = lane >> 4;
    const uint32_t lds0 = lds_address(smem);
    const int U = SHORT ? 3 : c.U;
    int32_t* const tile_end = reinterpret_cast<int32_t*>(smem + XT_LDS);
    int32_t* const row_end = tile_end + MX_MAX_EXPERTS;

    // The tiles: of every expert its rows by channels, then the rows of no expert.
    int total = tiles_o * ((c.R + BT - 1) / BT);
    if constexpr (GROUPED) {
        if (wave == 0) {
            int tiles = 0, end = 0;
            for (int e0 = 0; e0 < c.E; e0 += 64) {
                const mx4_span r = mx4_spans(c.offsets, c.E, c.R, e0, lane, end);
                const int sum = wave_scan_add((r.last - r.first + BT - 1) / BT * tiles_o);
                if (e0 + lane < c.E) { tile_end[e0 + lane] = tiles + sum; row_end[e0 + lane] = r.last; }
                tiles += __builtin_amdgcn_readlane(sum, 63);
                end = __builtin_amdgcn_readlane(r.last, 63);
            }
        }
        __syncthreads();
        total = __builtin_amdgcn_readfirstlane(tile_end[c.E - 1] + (c.R - row_end[c.E - 1] + BT - 1) / BT * tiles_o);
    }
    struct Tile { int expert, first, rows, o; };          // rows from `first` on, channels 256 o on
    auto tile_of = [&](int round, Tile& t) -> bool {
        const int nb = gridDim.x, base = round * nb;
        if (base + (int)blockIdx.x >= total) return false;
        int id = base + (base + nb <= total || tiles_o <= RUNS_MAX_TILES_O ? xcd_run(blockIdx.x, min(nb, total - base)) : (int)blockIdx.x);
        int first = 0, last = c.R;
        t.expert = 0;
        if constexpr (GROUPED) {
            int begin = 0;
            t.expert = c.E;
            for (int e0 = 0; e0 < c.E; e0 += 64) {
                const int l = fresh_lane();
                const uint64_t has = __ballot(e0 + l < c.E && tile_end[min(e0 + l, c.E - 1)] > id);
                if (has) { t.expert = e0 + __ffsll((unsigned long long)has) - 1; break; }
            }
            if (t.expert > 0) { begin = tile_end[t.expert - 1]; first = row_end[t.expert - 1]; }
            if (t.expert < c.E) last = row_end[t.expert];
            begin = __builtin_amdgcn_readfirstlane(begin);
            first = __builtin_amdgcn_readfirstlane(first);
            last = __builtin_amdgcn_readfirstlane(last);
            id -= begin;
        }
        const int tiles_t = (last - first + BT - 1) / BT;
        constexpr int BAND = 8;                           // as tile_of_round
        const int band = id / (BAND * tiles_o), within = id - band * (BAND * tiles_o), bw = min(BAND, tiles_t - band * BAND);
        t.o = within / bw;
        const int tt = band * BAND + (within - t.o * bw);
        t.first = first + tt * BT;
        t.rows = min(BT, last - t.first);
        return true;
    };

    // Sources of the direct loads, at the unit that is requested next: weights and scales of fragment `wave`, token rows 8 (8 i + wave) .. + 7, scales of
    // rows 64 (wave / 2) + 16 b + 8 (wave % 2) .. + 7, as [row & 15][half of a unit][b 4] words.
    struct Weights { const uint8_t *v, *m; } pa;
    struct Rows { const uint8_t *v, *m; } pb;
    int ua = 0, ub = 0;                                  // SHORT: the units that the requests are at
    uint32_t boff[4], bmoff = 0;
    auto weights_of = [&](const Tile& t) -> Weights {
        const int64_t at = ((int64_t)(GROUPED && t.expert == c.E ? 0 : t.expert) * c.frags + min(t.o * 8 + wave, c.frags - 1)) * c.U;
        return {c.w_vals + at * MX_FRAGB, c.w_meta + at * MX_FRAGS};
    };
    auto set_rows = [&](const Tile& t) {
        const int ln = fresh_lane();
        pb = {c.codes + (int64_t)t.first * c.U * MX_UNITB, c.scales + (int64_t)t.first * MX_UNITS};
        ub = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * (8 * i + wave) + (ln >> 3);
            boff[i] = (uint32_t)min(row, t.rows - 1) * (uint32_t)(c.U * MX_UNITB) + mx4_place((ln & 7) ^ swz(row)) * 16;
        }
        bmoff = (uint32_t)min((wave >> 1) * 64 + 16 * (ln & 3) + (wave & 1) * 8 + (ln >> 3), t.rows - 1) * MX_UNITS + (ln & 4);
    };
    const int64_t mb_next = (int64_t)c.R * MX_UNITS;
    const uint32_t lane16 = lane * 16, lane4 = lane * 4;
    const uint32_t a_wave = lds0 + wave * 2048, b_wave = lds0 + XT_B_OFF + wave * 1024, ma_wave = lds0 + XT_MA_OFF + wave * 256, mb_wave = lds0 + XT_MB_OFF + wave * 256;
    auto load_a = [&](int t, int j, uint32_t slot, int more) __attribute__((always_inline)) {
        mx4_load16(pa.v + (2 * t + j) * 1024, lane16, a_wave + slot + j * 1024, more);
    };
    auto load_ma = [&](uint32_t slot, int more) __attribute__((always_inline)) { mx4_load4(pa.m, lane4, ma_wave + slot, more); };
    auto load_b = [&](int i, uint32_t slot, int more) __attribute__((always_inline)) { mx4_load16(pb.v, boff[i], b_wave + slot + i * 8192, more); };
    auto load_mb = [&](uint32_t slot, int more) __attribute__((always_inline)) { mx4_load4(pb.m, bmoff, mb_wave + slot, more); };
    const uint8_t* const zeros_at = reinterpret_cast<const uint8_t*>(mx4_zeros);
    auto next_a = [&]() __attribute__((always_inline)) {
        const bool none = SHORT && ++ua >= c.U;
        pa.v = none ? zeros_at : pa.v + MX_FRAGB;
        pa.m = none ? zeros_at : pa.m + MX_FRAGS;
    };
    auto next_b = [&]() __attribute__((always_inline)) {
        const bool none = SHORT && ++ub >= c.U;
        pb.v += none ? 0 : MX_UNITB;                     // anything that is there
        pb.m = none ? zeros_at : pb.m + mb_next;
    };

    // LDS offsets of this lane's operand reads
    const uint32_t ra = wo * 8192 + lane * 16;
    const uint32_t rma = XT_MA_OFF + wo * 1024 + lane * 4;
    const uint32_t rb = XT_B_OFF + (wt * 64 + n) * ROWB + ((mx4_place(2 * q) ^ swz(n)) << 4);
    const uint32_t rmb = XT_MB_OFF + wt * 512 + n * 32 + (q >> 1) * 16;
    const uint32_t mb_shift = 16 * (q & 1);               // this lane's two bytes of a word of four scales

    uint32_t a0 = 0, a1 = XT_A, a2 = 2 * XT_A;            // slots of this step's weights and the next two's
    uint32_t b0 = 0, b1 = XT_B, b2 = 2 * XT_B;            // of this unit's token rows and the next two's
    uint32_t m0 = 0, m1 = XT_M;                           // of this unit's scales and the next one's
    Tile now, next;
    if (!tile_of(0, now)) return;
    pa = weights_of(now);
    set_rows(now);
    constexpr int ALL = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(i, b0, ALL);
    load_ma(m0, ALL);
    load_mb(m0, ALL);
    load_a(0, 0, a0, ALL);
    load_a(0, 1, a0, ALL);
    load_a(1, 0, a1, ALL);
    load_a(1, 1, a1, ALL);
    next_a();
    next_b();
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(i, b1, ALL);
    load_ma(m1, ALL);
    load_mb(m1, ALL);
    load_a(0, 0, a2, ALL);
    load_a(0, 1, a2, ALL);
    next_b();
    wait_vmcnt<10>();
    wg_barrier();

    int more_a = ALL, more_b = ALL;                  // none where there is no next tile
    Weights then = pa;                                    // of the next tile
    int have = 1;
    v4f acc[8][4];
    v4i va[8], vb[4];
    int sa[4], sb[4];
    v4i wb;                                               // the next unit's token scales as they were read
    auto rd = [&](uint32_t off) __attribute__((always_inline)) -> v4i { return *reinterpret_cast<const v4i*>(smem + off); };
    auto read_a = [&](int a, uint32_t slot) __attribute__((always_inline)) { va[a] = rd(ra + slot + a * 1024); };
    auto read_sa = [&](int f, uint32_t slot) __attribute__((always_inline)) { sa[f] = *reinterpret_cast<const int*>(smem + rma + slot + f * 256); };
    auto read_b = [&](int b, int t, uint32_t slot) __attribute__((always_inline)) { vb[b] = rd(((rb + slot) ^ (t * 32)) + b * 2048); };
    auto read_sb = [&](uint32_t slot) __attribute__((always_inline)) { wb = rd(rmb + slot); };
    auto set_sb = [&](int b) __attribute__((always_inline)) { sb[b] = (int)((uint32_t)wb[b] >> mb_shift); };
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[a][b] = v4f{0, 0, 0, 0};
    };
    // Step t of a unit.  Instruction i: rows in two halves of 16 instructions, weight fragments 0 .. 7 within each, so that everything has
    // fourteen or more instructions between its last use and its next.
    auto step = [&](auto t_c, int waits) __attribute__((always_inline)) {
        constexpr int T = decltype(t_c)::value;
        __builtin_amdgcn_sched_barrier(0);
        unroll<32>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            constexpr int a = (i >> 1) & 7, b = 2 * (i >> 4) + (i & 1);
            acc[a][b] = mx4_mma<2 * (a & 1) + T, T>(va[a], vb[b], acc[a][b], sa[a >> 1], sb[b]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0 || i == 2) {                       // these registers were in use until the end of the last step
                read_b(2 + i / 2, T, b0);
                if (T == 0) set_sb(2 + i / 2);
            }
            if (i == 1) __builtin_amdgcn_s_setprio(0);
            if (i == 16) __builtin_amdgcn_s_setprio(1);
            if (i == 14) {
                wait_vm_mode<(T == 0 ? 8 : 7)>(waits);
                wait_lgkm0();
                wg_barrier();
            }
            if constexpr (T == 1) {
                if (i == 4) load_b(2, b2, more_b);
                if (i == 9) load_b(3, b2, more_b);
            }
            if (i == 15) load_a(1 - T, 0, a0, more_a);
            if (i == (T == 0 ? 18 : 20)) load_a(1 - T, 1, a0, more_a);
            if (i == (T == 0 ? 21 : 25)) {
                if (T == 0) load_mb(m0, more_b);
                else load_ma(m0, more_a);
            }
            if constexpr (T == 0) {
                if (i == 24) load_b(0, b2, more_b);
                if (i == 27) load_b(1, b2, more_b);
            }
            if (i >= 17 && (i & 1)) {
                read_a((i - 17) >> 1, a1);
                if (T == 1 && (i & 2)) read_sa((i - 19) >> 2, m1);
            }
            if (i == 18 || i == 22) {
                read_b((i - 18) >> 2, 1 - T, T == 0 ? b0 : b1);
                if (T == 1 && i == 18) read_sb(m1);
            }
            if (T == 1 && i == 31) { set_sb(0); set_sb(1); }
            __builtin_amdgcn_sched_barrier(0);
        });
        const uint32_t w = a0;
        a0 = a1; a1 = a2; a2 = w;
        if (T == 1) {
            const uint32_t x = b0, y = m0;
            b0 = b1; b1 = b2; b2 = x;
            m0 = m1; m1 = y;
        }
    };
#pragma unroll
    for (int a = 0; a < 8; ++a) read_a(a, a0);
#pragma unroll
    for (int f = 0; f < 4; ++f) read_sa(f, m0);
#pragma unroll
    for (int b = 0; b < 2; ++b) read_b(b, 0, b0);
    read_sb(m0);
    set_sb(0);
    set_sb(1);
    clear();
    int round = 0, u = 0, waits = 1;
    for (;;) {
        if (u == U - 2) {                                 // the token rows' requests go on to the next tile, the weights' in the second step
            have = __builtin_amdgcn_readfirstlane(tile_of(++round, next) ? 1 : 0);
            if (have) { set_rows(next); then = weights_of(next); }
            more_b = -have;
        }
        step(std::integral_constant<int, 0>{}, waits);
        next_a();                                         // without a branch: the products of a step would sink below it
        const bool wrap = u == U - 2;
        pa.v = wrap ? then.v : pa.v;
        pa.m = wrap ? then.m : pa.m;
        if (SHORT) ua = wrap ? 0 : ua;
        more_a = wrap ? -have : more_a;
        step(std::integral_constant<int, 1>{}, waits);
        next_b();
        waits = 1;
        if (++u < U) continue;
        // The tile's results.  b2 is free, nothing is requested into it before the next meeting.
        const int o_sub = (now.o * BO + wo * 128) >> (c.gated ? 1 : 0), t_sub = wt * 64;
        const int rows_left = min(now.rows - t_sub, 64), cols_left = min(c.O - o_sub, c.gated ? 64 : 128);
        const bool any = rows_left > 0 && cols_left > 0;
        uint16_t* const Y_sub = any ? c.Y + (int64_t)(now.first + t_sub) * c.ldy + o_sub : c.Y;
        uint8_t* const stage = smem + XT_B_OFF + b2 + wave * 4096;
        const bool zeros = GROUPED && now.expert == c.E;
        if (c.gated) xt_store<true>(acc, zeros, Y_sub, (uint32_t)c.ldy, any ? rows_left : 0, any ? cols_left : 0, stage);
        else xt_store<false>(acc, zeros, Y_sub, (uint32_t)c.ldy, any ? rows_left : 0, any ? cols_left : 0, stage);
        if (!have) break;
        now = next;
        u = 0;
        waits = 0;                                        // its first steps' operands landed ahead of the stores
        clear();
    }
}

ss_status launch_mx4_tile(const mx4_call& c, hipStream_t stream)
{
    const int64_t tiles_o = (c.frags + 7) / 8, most = tiles_o * (c.offsets ? mx4_max_tiles(c.R, c.E, BT) : ((int64_t)c.R + BT - 1) / BT);
    if (most > INT32_MAX / 2) return SS_ERR_SHAPE;
    const int cus = cu_count(), grid = (int)(most < cus ? most : cus), lds = XT_LDS + (c.offsets ? XT_ENDS : 0);
    auto launch = [&](auto allow, auto kernel) {
        if (allow != SS_OK) return SS_ERR_HIP;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(512), lds, stream, c, (int)tiles_o);
        return launch_status();
    };
#define SS_XT(G, S) launch(allow_dynamic_lds<k_mx4_tile<G, S>>(lds), k_mx4_tile<G, S>)
    if (c.offsets) return c.U < 3 ? SS_XT(true, true) : SS_XT(true, false);
    return c.U < 3 ? SS_XT(false, true) : SS_XT(false, false);
#undef SS_XT
}

}  // namespace ss
