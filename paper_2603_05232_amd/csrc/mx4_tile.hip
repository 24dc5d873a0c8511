// Products of microscaled 4-bit operands on tiles of 256 channels x 256 token rows (mx4_gemm, mx4_grouped_gemm: many rows).
//
// Persistent workgroups of eight wavefronts, two per SIMD, of 128 channels x 64 rows = 8 x 4 blocks of the 16x16x128 instruction.  A unit of 256
// values is two steps; lane (n, q) = (l & 15, l >> 4) takes block 2 q + t of its row in step t, so that its two scales lie side by side
// in one 16-bit read, whose byte the instruction selects.
//
// LDS: weights in three slots of a step (16 KB), token rows in three slots of a unit (32 KB), scales of two units.  Direct loads fill
// them; those of a step are spread from one meeting of the workgroup to the next.  The workgroup meets once a step, behind
// instruction 14: the reads of this step's operands have returned then, so the slots they came from are free, and what the reads
// behind the meeting need was requested two steps before or earlier.  The requests run on across tiles; between two there is only
// the epilogue, which stages in the token slot that is free then.
#include "mx4_common.h"
#include "lds_pipe.h"
#include "tile_common.h"
#include "device_info.h"

namespace ss {

constexpr int XT_A = 16 * 1024, XT_B = 32 * 1024, XT_M = 2048;
constexpr int XT_B_OFF = 3 * XT_A, XT_MA_OFF = XT_B_OFF + 3 * XT_B, XT_MB_OFF = XT_MA_OFF + 2 * XT_M, XT_LDS = XT_MB_OFF + 2 * XT_M;      // 152 KB
constexpr int XT_ENDS = 2 * MX_MAX_EXPERTS * 4;          // last tile and last row of every expert
static_assert(XT_LDS + XT_ENDS <= 160 * 1024, "LDS budget");

// direct loads by all lanes (more = ~0) or none (0), in a wavefront whose lanes are all active
__device__ inline void xt_load16(const uint8_t* base, uint32_t lane_off, uint32_t lds, uint32_t more)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(more) : "memory", "m0");
}
__device__ inline void xt_load4(const uint8_t* base, uint32_t lane_off, uint32_t lds, uint32_t more)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(more) : "memory", "m0");
}

// 16-byte chunk c of a token row lies at chunk xt_place(c) ^ swz(row): a 16-byte LDS read is served to eight lanes of one q and eight of q ^ 1 at a
// time (rows 0 .. 3, 12 .. 15 of the one, 4 .. 11 of the other), whose chunks 2 apart would meet on the same banks
__device__ inline int xt_place(int c) { return (c & 4) | ((c & 1) << 1) | ((c >> 1) & 1); }      // its own inverse

template <int T> __device__ __forceinline__ v4f mx4_mma16(v4i a, v4i b, v4f c, int sa, int sb)
{
    const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, T, sa, T, sb);
}

// acc[a][b][i] of lane (n, q), a = 4 hh + f: packed channel 32 f + 16 (q & 1) + 8 hh + 4 (q >> 1) + i, row 16 b + n of a sub-tile of 128 x 64 of which
// rows_left rows and cols_left columns of Y exist.  Staged 16 rows at a time through the wavefront's own 4 KB, so that every store
// writes whole pieces of Y's rows.  All loads in flight are waited for before the first store (the wait counter counts both).
template <bool GATED>
__device__ inline void xt_store(const v4f (&acc)[8][4], bool zeros, uint16_t* __restrict__ Y_sub, uint32_t ldy, int rows_left, int cols_left, uint8_t* stage)
{
    constexpr int ROW = GATED ? 128 : 256, LANES = ROW / 16, ROWS = 64 / LANES;      // bytes of a staged row, lanes that store one, rows of a store
    const int lane = fresh_lane(), n = lane & 15, q = lane >> 4, sr = lane / LANES, sc = lane % LANES;
    const bool vec_ok = (ldy & 7) == 0 && ((uintptr_t)Y_sub & 15) == 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            const int f = a & 3, hh = a >> 2;
            const v4f v = zeros ? v4f{0, 0, 0, 0} : acc[a][b];
            if constexpr (GATED) {
                const int chunk = 2 * f + (q & 1);
                *reinterpret_cast<uint32_t*>(stage + n * ROW + ((chunk ^ (n & 7)) << 4) + 8 * hh + 4 * (q >> 1)) = pack_bf16x2(mx4_gate(v[0], v[1]), mx4_gate(v[2], v[3]));
            } else {
                const int chunk = 4 * f + 2 * (q & 1) + hh;
                *reinterpret_cast<uint2*>(stage + n * ROW + ((chunk ^ n) << 4) + 8 * (q >> 1)) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            }
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

// Rows of at least three units.
template <bool GROUPED>
__global__ __launch_bounds__(512) void k_mx4_tile(mx4_call c, int tiles_o)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wo = wave & 1, wt = wave >> 1, n = lane & 15, q = lane >> 4;
    const uint32_t lds0 = lds_address(smem);
    const int U = c.U;
    int32_t* const tile_end = reinterpret_cast<int32_t*>(smem + XT_LDS);
    int32_t* const row_end = tile_end + MX_MAX_EXPERTS;

    // The tiles: of every expert its rows by channels, then the rows of no expert.
    int total = tiles_o * ((c.R + BT - 1) / BT);
    if constexpr (GROUPED) {
        if (wave == 0) {
            int tiles = 0, end = 0;
            for (int e0 = 0; e0 < c.E; e0 += 64) {
                const int e = e0 + lane;
                int last = e < c.E ? min(max(c.offsets[e + 1], 0), c.R) : 0;
                last = max(last, end);
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(last, d, 64);
                    if (lane >= d) last = max(last, o);
                }
                int first = __shfl_up(last, 1, 64);
                if (lane == 0) first = end;
                int sum = (last - first + BT - 1) / BT * tiles_o;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(sum, d, 64);
                    if (lane >= d) sum += o;
                }
                if (e < c.E) { tile_end[e] = tiles + sum; row_end[e] = last; }
                tiles += __shfl(sum, 63, 64);
                end = __shfl(last, 63, 64);
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

    // Sources of the direct loads: weights of fragment `wave`, token rows 8 (8 i + wave) .. + 7, scales of fragment `wave` and of rows 32 wave .. + 31.
    const uint8_t *av = nullptr, *am = nullptr, *bv = nullptr, *bm = nullptr;
    uint32_t boff[4], bmoff = 0;
    auto set_weights = [&](const Tile& t) {
        const int64_t at = ((int64_t)(GROUPED && t.expert == c.E ? 0 : t.expert) * c.frags + min(t.o * 8 + wave, c.frags - 1)) * U;
        av = c.w_vals + at * MX_FRAGB;
        am = c.w_meta + at * MX_FRAGS;
    };
    auto set_rows = [&](const Tile& t) {
        const int ln = fresh_lane();
        bv = c.codes + (int64_t)t.first * U * MX_UNITB;
        bm = c.scales + (int64_t)t.first * MX_UNITS;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * (8 * i + wave) + (ln >> 3);
            boff[i] = (uint32_t)min(row, t.rows - 1) * (uint32_t)(U * MX_UNITB) + xt_place((ln & 7) ^ swz(row)) * 16;
        }
        bmoff = (uint32_t)min(32 * wave + (ln >> 1), t.rows - 1) * MX_UNITS + (ln & 1) * 4;
    };
    const uint32_t lane16 = lane * 16, lane4 = lane * 4;
    const uint32_t a_wave = lds0 + wave * 2048, b_wave = lds0 + XT_B_OFF + wave * 1024, ma_wave = lds0 + XT_MA_OFF + wave * 256, mb_wave = lds0 + XT_MB_OFF + wave * 256;
    auto load_a = [&](int u, int t, int j, uint32_t slot, uint32_t more) __attribute__((always_inline)) {
        xt_load16(av + ((uint32_t)u * MX_FRAGB + (2 * j + t) * 1024), lane16, a_wave + slot + j * 1024, more);
    };
    auto load_ma = [&](int u, uint32_t slot, uint32_t more) __attribute__((always_inline)) { xt_load4(am + (uint32_t)u * MX_FRAGS, lane4, ma_wave + slot, more); };
    auto load_b = [&](int u, int i, uint32_t slot, uint32_t more) __attribute__((always_inline)) {
        xt_load16(bv + (uint32_t)u * MX_UNITB, boff[i], b_wave + slot + i * 8192, more);
    };
    auto load_mb = [&](int u, uint32_t slot, uint32_t more) __attribute__((always_inline)) {
        xt_load4(bm + (int64_t)u * c.R * MX_UNITS, bmoff, mb_wave + slot, more);
    };

    // LDS offsets of this lane's operand reads
    const uint32_t ra = wo * 8192 + (q & 1) * 1024 + ((q >> 1) * 32 + n) * 16;
    const uint32_t rma = XT_MA_OFF + wo * 1024 + ((q >> 1) * 32 + n) * 4 + 2 * (q & 1);
    const uint32_t rb = XT_B_OFF + (wt * 64 + n) * ROWB + ((xt_place(2 * q) ^ swz(n)) << 4);
    const uint32_t rmb = XT_MB_OFF + (wt * 64 + n) * MX_UNITS + 2 * q;

    uint32_t a0 = 0, a1 = XT_A, a2 = 2 * XT_A;            // slots of this step's weights and the next two's
    uint32_t b0 = 0, b1 = XT_B, b2 = 2 * XT_B;            // of this unit's token rows and the next two's
    uint32_t m0 = 0, m1 = XT_M;                           // of this unit's scales and the next one's
    Tile now, next;
    if (!tile_of(0, now)) return;
    set_weights(now);
    set_rows(now);
    constexpr uint32_t ALL = ~0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(0, i, b0, ALL);
    load_ma(0, m0, ALL);
    load_mb(0, m0, ALL);
    load_a(0, 0, 0, a0, ALL);
    load_a(0, 0, 1, a0, ALL);
    load_a(0, 1, 0, a1, ALL);
    load_a(0, 1, 1, a1, ALL);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(1, i, b1, ALL);
    load_ma(1, m1, ALL);
    load_mb(1, m1, ALL);
    load_a(1, 0, 0, a2, ALL);
    load_a(1, 0, 1, a2, ALL);
    wait_vmcnt<10>();
    wg_barrier();

    int ua = 1, ub = 2;                                   // units that the next requests of weights and of token rows are for
    uint32_t more_a = ALL, more_b = ALL;                // none where there is no next tile
    int have = 1;
    v4f acc[8][4];
    v4i va[8], vb[4];
    int sa[8], sb[4];
    auto rd = [&](uint32_t off) __attribute__((always_inline)) -> v4i { return *reinterpret_cast<const v4i*>(smem + off); };
    auto rd2 = [&](uint32_t off) __attribute__((always_inline)) -> int { return *reinterpret_cast<const uint16_t*>(smem + off); };
    auto read_a = [&](int a, uint32_t slot) __attribute__((always_inline)) { va[a] = rd(ra + slot + (a & 3) * 2048 + (a >> 2) * 256); };
    auto read_sa = [&](int a, uint32_t slot) __attribute__((always_inline)) { sa[a] = rd2(rma + slot + (a & 3) * 256 + (a >> 2) * 64); };
    auto read_b = [&](int b, int t, uint32_t slot) __attribute__((always_inline)) { vb[b] = rd(((rb + slot) ^ (t * 32)) + b * 2048); };
    auto read_sb = [&](int b, uint32_t slot) __attribute__((always_inline)) { sb[b] = rd2(rmb + slot + b * 128); };
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
            acc[a][b] = mx4_mma16<T>(va[a], vb[b], acc[a][b], sa[a], sb[b]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0 || i == 2) {                       // these registers were in use until the end of the last step
                read_b(2 + i / 2, T, b0);
                if (T == 0) read_sb(2 + i / 2, m0);
            }
            if (i == 1) __builtin_amdgcn_s_setprio(0);
            if (i == 16) __builtin_amdgcn_s_setprio(1);
            if (i == 14) {
                wait_vm_mode<(T == 0 ? 8 : 7)>(waits);
                wait_lgkm0();
                wg_barrier();
            }
            if constexpr (T == 1) {
                if (i == 4) load_b(ub, 2, b2, more_b);
                if (i == 9) load_b(ub, 3, b2, more_b);
            }
            if (i == 15) load_a(ua, 1 - T, 0, a0, more_a);
            if (i == (T == 0 ? 18 : 20)) load_a(ua, 1 - T, 1, a0, more_a);
            if (i == (T == 0 ? 21 : 25)) {
                if (T == 0) load_mb(ub, m0, more_b);
                else load_ma(ua, m0, more_a);
            }
            if constexpr (T == 0) {
                if (i == 24) load_b(ub, 0, b2, more_b);
                if (i == 27) load_b(ub, 1, b2, more_b);
            }
            if (i >= 17 && (i & 1)) {
                read_a((i - 17) >> 1, a1);
                if (T == 1) read_sa((i - 17) >> 1, m1);
            }
            if (i == 18 || i == 22) {
                read_b((i - 18) >> 2, 1 - T, T == 0 ? b0 : b1);
                if (T == 1) read_sb((i - 18) >> 2, m1);
            }
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
    for (int a = 0; a < 8; ++a) { read_a(a, a0); read_sa(a, m0); }
#pragma unroll
    for (int b = 0; b < 2; ++b) { read_b(b, 0, b0); read_sb(b, m0); }
    clear();
    int round = 0, u = 0, waits = 1;
    for (;;) {
        if (u == U - 2) {                                 // the token rows' requests go on to the next tile
            have = __builtin_amdgcn_readfirstlane(tile_of(++round, next) ? 1 : 0);
            ub = 0;
            if (have) set_rows(next);
            more_b = -have;
        }
        step(std::integral_constant<int, 0>{}, waits);
        if (++ua == U) {                                  // and the weights'
            ua = 0;
            if (have) set_weights(next);
            more_a = -have;
        }
        step(std::integral_constant<int, 1>{}, waits);
        ++ub;
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
    const int cus = cu_count(), grid = (int)(most < cus ? most : cus);
    if (c.offsets) {
        if (allow_dynamic_lds<k_mx4_tile<true>>(XT_LDS + XT_ENDS) != SS_OK) return SS_ERR_HIP;
        hipLaunchKernelGGL(k_mx4_tile<true>, dim3(grid), dim3(512), XT_LDS + XT_ENDS, stream, c, (int)tiles_o);
    } else {
        if (allow_dynamic_lds<k_mx4_tile<false>>(XT_LDS) != SS_OK) return SS_ERR_HIP;
        hipLaunchKernelGGL(k_mx4_tile<false>, dim3(grid), dim3(512), XT_LDS, stream, c, (int)tiles_o);
    }
    return launch_status();
}

}  // namespace ss
