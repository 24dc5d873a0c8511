// Microscaled 4-bit operands (mx4): layouts of code rows, scales and packed weights, and what the kernels on them share.
//
// Values.  A code is sign, two exponent bits, one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6); 32 consecutive values of a row share a scale
// byte b = 2^(b - 127), 255 = not a number.  A row is counted in units of 256 values = 128 bytes of codes + 8 scale bytes, its last unit
// completed with zeros.
//   codes[row][unit][128]     two codes to a byte, the even value in the low half; block j of the unit is bytes 16 j .. 16 j + 15
//   scales[unit][row][8]      byte j: block j of the unit.  The units lie outermost so that a tile's rows of one unit are one run.
//
// Operands.  Lane (n, h) = (l & 31, l >> 5) of the 32x32x64 instruction holds 32 values, one block, of row n.  Step s = 0 .. 3 of a unit
// takes block 4 h + s, so a lane's four blocks are 64 consecutive bytes and their scales one word, whose byte s the instruction selects.
//   w_vals[expert][fragment of 32 channels][unit][step 4][lane 64][16 B]
//   w_meta[expert][fragment][unit][lane 64][4 B]
// Fragment row r holds channel mx4_channel(r), so that a lane's sixteen sums are sixteen consecutive channels.  Gated layers alternate
// the channels of gate and up: packed channel 2 c is gate's channel c, 2 c + 1 is up's.
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
// channel of a fragment's row r: sums i of lane half h belong to rows 8 (i >> 2) + 4 h + (i & 3)
__host__ __device__ inline int mx4_channel(int r) { return ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }

// One 32x32x64 product of 4-bit operands; `S` selects the byte of the scale words.
template <int S> __device__ __forceinline__ v16f mx4_mma(v4i a, v4i b, v16f c, int sa, int sb)
{
    const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, S, sa, S, sb);
}

// silu(g) u, in 32 bits
__device__ inline float mx4_gate(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// A tile of token rows of one expert.
struct mx4_rows {
    int expert;          // the number of experts: rows of no expert, whose results are zeros
    int first, count;    // count = 0: there is no such tile
};

// Tile number `slot` of the tiles of T rows that the experts' rows and the rows behind the last expert's make, in order.  Offsets outside
// [0, R] or below one before them are moved to the nearest that is not, so that every row belongs to one tile whatever they hold.
// Called by whole wavefronts.
__device__ inline mx4_rows mx4_find(const int32_t* __restrict__ offsets, int E, int R, int T, int slot)
{
    const int lane = threadIdx.x & 63;
    int before = 0, end = 0;                              // tiles and last row of the experts so far
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int e = e0 + lane;
        int last = e < E ? min(max(offsets[e + 1], 0), R) : R;
        if (e > E) last = 0;
        last = max(last, end);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {                // running maximum
            const int o = __shfl_up(last, d, 64);
            if (lane >= d) last = max(last, o);
        }
        int first = __shfl_up(last, 1, 64);
        if (lane == 0) first = end;
        const int tiles = e <= E ? (last - first + T - 1) / T : 0;
        int sum = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d, 64);
            if (lane >= d) sum += o;
        }
        const uint64_t has = __ballot(before + sum > slot);
        if (has) {
            const int at = __ffsll((unsigned long long)has) - 1;
            const int f = __shfl(first, at, 64), l = __shfl(last, at, 64), in = slot - (before + __shfl(sum - tiles, at, 64));
            const int start = __builtin_amdgcn_readfirstlane(f + in * T), rest = __builtin_amdgcn_readfirstlane(l) - start;
            return {__builtin_amdgcn_readfirstlane(e0 + at), start, rest < T ? rest : T};
        }
        before += __builtin_amdgcn_readfirstlane(__shfl(sum, 63, 64));
        end = __builtin_amdgcn_readfirstlane(__shfl(last, 63, 64));
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

// Tiles of 256 channels x 256 rows (mx4_tile.hip); rows of MX_TILE_UNITS units and more.
constexpr int MX_TILE_UNITS = 3;
ss_status launch_mx4_tile(const mx4_call& c, hipStream_t stream);

}  // namespace ss
