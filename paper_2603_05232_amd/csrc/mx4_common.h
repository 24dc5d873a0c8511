// Microscaled 4-bit operands (mx4): layouts of code rows, scales and packed weights, and what the kernels on them share.
//
// Values.  A code is sign, two exponent bits, one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6); 32 consecutive values of a row share a scale
// byte b = 2^(b - 127), 255 = not a number.  A row is counted in units of 256 values = 128 bytes of codes + 8 scale bytes, its last unit
// completed with zeros.
//   codes[row][unit][128]     two codes to a byte, the even value in the low half; block j of the unit is bytes 16 j .. 16 j + 15
//   scales[unit][row][8]      byte j: block j of the unit.  The units lie outermost so that a tile's rows of one unit are one run.
//
// Operands.  Lane (n, q) = (l & 15, l >> 4) of the 16x16x128 instruction holds 32 values, one block, of row n.  Step t = 0, 1 of a unit takes block
// 2 q + t, so a lane's two blocks are 32 consecutive bytes and their scales lie side by side; the instruction selects the byte.
//   w_vals[expert][fragment of 32 channels][unit][step 2][half 2][lane 64][16 B]      lane (n, q): block 2 q + t of fragment row (half, n)
//   w_meta[expert][fragment][unit][lane 64][4 B]                                      byte 2 half + t: its scale
// Fragment row (half, r) holds channel mx4_channel(half, r), so that a lane's eight sums (4 half + i) are eight consecutive channels.
// Gated layers alternate the channels of gate and up: packed channel 2 c is gate's channel c, 2 c + 1 is up's.
#pragma once
#include "ss_common.h"
#include "mma_types.h"

namespace ss {

constexpr int MX_UNIT = 256;             // values of a row in a unit
constexpr int MX_UNITB = 128;            // their bytes of codes
constexpr int MX_UNITS = 8;              // their scale bytes
constexpr int MX_FRAG = 32;              // channels of a fragment
constexpr int MX_FRAGB = 4096;           // bytes of a fragment's codes of one unit
constexpr int MX_FRAGS = 256;            // bytes of its scales
constexpr int MX_MAX_EXPERTS = 1024;
constexpr int64_t MX_MAX_K = 1 << 24;
constexpr int64_t MX_MAX_ROWS = 1 << 24;

__host__ __device__ inline int64_t mx4_units(int64_t K) { return (K + MX_UNIT - 1) / MX_UNIT; }
__host__ __device__ inline int64_t mx4_frags(int64_t rows) { return (rows + MX_FRAG - 1) / MX_FRAG; }
// channel of a fragment's row: sums i of lane group q belong to rows 4 q + i
__host__ __device__ inline int mx4_channel(int half, int r) { return (r >> 2) * 8 + half * 4 + (r & 3); }

// One 16x16x128 product of 4-bit operands; SA, SB select the bytes of the scale words.
template <int SA, int SB> __device__ __forceinline__ v4f mx4_mma(v4i a, v4i b, v4f c, int sa, int sb)
{
    const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, SA, sa, SB, sb);
}

// 16-byte chunk c of a token row lies at chunk mx4_place(c) ^ swz(row): a 16-byte LDS read is served to eight lanes of one q and eight of q ^ 1 at a
// time (rows 0 .. 3, 12 .. 15 of the one, 4 .. 11 of the other), whose chunks 2 apart would meet on the same banks
__device__ inline int mx4_place(int c) { return (c & 4) | ((c & 1) << 1) | ((c >> 1) & 1); }      // its own inverse

typedef uint32_t piece4_t __attribute__((aligned(2)));

// silu(g) u, in 32 bits
__device__ inline float mx4_gate(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// Eight consecutive packed channels from `ch` on of one row of Y: sums v (half 0) and w (half 1) of one lane.
__device__ inline void mx4_store8(v4f v, v4f w, uint16_t* __restrict__ y, int ch, int O, bool gated)
{
    uint32_t p[4];
    int n = 8;
    if (gated) {
        p[0] = pack_bf16x2(mx4_gate(v[0], v[1]), mx4_gate(v[2], v[3]));
        p[1] = pack_bf16x2(mx4_gate(w[0], w[1]), mx4_gate(w[2], w[3]));
        p[2] = p[3] = 0;
        ch >>= 1;
        n = 4;
    } else {
        p[0] = pack_bf16x2(v[0], v[1]);
        p[1] = pack_bf16x2(v[2], v[3]);
        p[2] = pack_bf16x2(w[0], w[1]);
        p[3] = pack_bf16x2(w[2], w[3]);
    }
    y += ch;
    if (ch + n <= O) {
        if (gated) *reinterpret_cast<piece8_t*>(y) = piece8_t{p[0], p[1]};
        else *reinterpret_cast<piece16_t*>(y) = piece16_t{p[0], p[1], p[2], p[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n && ch + e < O) y[e] = (uint16_t)(p[e >> 1] >> (16 * (e & 1)));
    }
}

// running sum and maximum over the lanes of a wavefront
template <typename F> __device__ inline int wave_scan(int v, int none, F f)
{
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xF, 0xF, false));      // row_shr:1
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xF, 0xF, false));      // 2
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xF, 0xF, false));      // 4
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xF, 0xF, false));      // 8
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xA, 0xF, false));      // row_bcast:15
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xC, 0xF, false));      // row_bcast:31
    return v;
}
__device__ inline int wave_scan_add(int v) { return wave_scan(v, 0, [](int a, int b) { return a + b; }); }
__device__ inline int wave_scan_max(int v) { return wave_scan(v, 0, [](int a, int b) { return a > b ? a : b; }); }      // of values >= 0

// The rows of experts e0 .. e0 + 63, one to a lane (lanes beyond the last expert: those behind its rows).  Offsets outside [0, R] or below one before
// them are moved to the nearest that is not, so that every row belongs to one expert or to none, whatever they hold.
struct mx4_span { int first, last; };
__device__ inline mx4_span mx4_spans(const int32_t* __restrict__ offsets, int E, int R, int e0, int lane, int end)
{
    const int e = e0 + lane, last = max(wave_scan_max(e < E ? min(max(offsets[e + 1], 0), R) : R), end);
    const int before = __builtin_amdgcn_update_dpp(end, last, 0x138, 0xF, 0xF, false);      // wave_shr:1
    return {before, last};
}

// A tile of token rows of one expert.
struct mx4_rows {
    int expert;          // the number of experts: rows of no expert, whose results are zeros
    int first, count;    // count = 0: there is no such tile
};

// Tile number `slot` of the tiles of T rows that the experts' rows and the rows behind the last expert's make, in order.  Called by whole wavefronts.
__device__ inline mx4_rows mx4_find(const int32_t* __restrict__ offsets, int E, int R, int T, int slot)
{
    const int lane = threadIdx.x & 63;
    int before = 0, end = 0;                              // tiles and last row of the experts so far
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const mx4_span s = mx4_spans(offsets, E, R, e0, lane, end);
        const int tiles = (s.last - s.first + T - 1) / T, sum = wave_scan_add(tiles);
        const uint64_t has = __ballot(before + sum > slot);
        if (has) {
            const int at = __ffsll((unsigned long long)has) - 1;
            const int f = __builtin_amdgcn_readlane(s.first, at), l = __builtin_amdgcn_readlane(s.last, at);
            const int start = f + (slot - (before + __builtin_amdgcn_readlane(sum - tiles, at))) * T;
            return {e0 + at, start, min(l - start, T)};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
        end = __builtin_amdgcn_readlane(s.last, 63);
    }
    return {0, 0, 0};
}
// tiles of T rows there can be at most
inline int64_t mx4_max_tiles(int64_t R, int64_t E, int64_t T) { return R < R / T + E + 1 ? R : R / T + E + 1; }

// A product of mx4 operands: dense (offsets = NULL, E = 1, all rows of expert 0) or grouped by expert.
struct mx4_call {
    const uint8_t* codes;
    const uint8_t* scales;
    const int32_t* offsets;
    const uint8_t* w_vals;
    const uint8_t* w_meta;
    int R, E, O;             // token rows, experts, columns of Y
    int U, frags;            // units of a row, fragments of packed channels of an expert
    uint16_t* Y;
    int64_t ldy;
    bool gated;
};

// a launch counts the threads of a grid's dimension in 32 bits
inline bool mx4_grid_fits(int64_t workgroups, int64_t threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

// Tiles of 256 channels x 256 rows (mx4_tile.hip).
ss_status launch_mx4_tile(const mx4_call& c, hipStream_t stream);
// Tiles of 128 channels x 16 or 32 rows (mx4_short.hip); rows of at most MX_SHORT_UNITS units.
constexpr int MX_SHORT_UNITS = 4;
ss_status launch_mx4_short(const mx4_call& c, int rows, hipStream_t stream);
// Tiles of 128 channels x 32, 64 or 128 rows (mx4_mid.hip); more than one range of units: with a workspace of mx4_mid_bytes.
ss_status launch_mx4_mid(const mx4_call& c, int rows, int ranges, void* ws, hipStream_t stream);
inline size_t mx4_mid_bytes(int64_t R, int64_t E, int64_t frags, int rows, int ranges)
{
    return ranges > 1 ? (size_t)((frags + 3) / 4 * mx4_max_tiles(R, E, rows) * ranges) * 512 * rows : 0;      // a grouped call of one expert has more tiles than a dense one
}

}  // namespace ss
