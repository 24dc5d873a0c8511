// A paged cache of keys and values: its layout, and what its kernels share.
//
// A page holds `page` tokens (a multiple of 32) of every head, head by head, in blocks of 32 tokens.  A block is what one step of the attention reads: the keys and the
// values of 32 tokens as operands of the 16x16x32 instruction, so that every load of a wavefront is one run of 1024 bytes, 16 to a lane.  D is completed to kv_steps(D)
// 32 values.
//
// Scores are K Q^T, 16 tokens x 16 heads in two products t = 0, 1: lane (r, j) = (l & 15, l >> 4) holds 8 values 32 s + 8 j .. + 7 of token row r, and gets the scores of rows
// 4 j .. 4 j + 3 of head r.  Row r of product t is token 8 (r >> 2) + 4 t + (r & 3), so a lane's eight scores are those of tokens 8 j .. 8 j + 7: just what it has to
// hold of the probabilities for the product with the values, V^T P, 32 tokens deep.  Nothing moves between lanes in between.
//   16 bits   keys    [step s][product t][lane][8 values]         values  [16 channels n][lane (r = channel, j)][tokens 8 j .. 8 j + 7]
//    8 bits   keys    [step s][lane][product t][8 values]         values  [32 channels][lane (r, j)][channel 16 h + r][8 tokens], h = 0, 1;      then 32 fp32 scales of keys, 32 of values
#pragma once
#include "mx4_common.h"
#include "device_info.h"

namespace ss {

constexpr int KV_BLOCK = 32;                         // tokens of a block
constexpr int KV_MAX_D = 256;
constexpr int KV_MAX_HEADS = 1024;
constexpr int64_t KV_MAX_REQUESTS = 4096;
constexpr int64_t KV_MAX_TOKENS = 1 << 20;           // rows of one call

// Steps of 32 values of a head; 5 and 7 have no kernel of their own.
__host__ __device__ constexpr int kv_steps(int64_t D) { const int n = (int)((D + 31) / 32); return n == 5 || n == 7 ? n + 1 : n; }
__host__ __device__ constexpr int kv_es(int dt) { return dt == SS_BF16 || dt == SS_FP16 ? 2 : 1; }
// bytes of a block's keys (and of its values), and of a block
__host__ __device__ constexpr int kv_half_bytes(int es, int ns) { return KV_BLOCK * 32 * ns * es; }
__host__ __device__ constexpr int kv_block_bytes(int es, int ns) { return 2 * kv_half_bytes(es, ns) + (es == 1 ? 2 * KV_BLOCK * 4 : 0); }

inline bool kv_valid_page(int64_t H, int64_t page, int64_t D, int dtype)
{
    return H >= 1 && H <= KV_MAX_HEADS && page >= KV_BLOCK && page <= 4096 && page % KV_BLOCK == 0 && D >= 1 && D <= KV_MAX_D && valid_dtype((ss_dtype)dtype);
}
inline int64_t kv_bytes_of_page(int64_t H, int64_t page, int64_t D, int dtype) { return H * (page / KV_BLOCK) * kv_block_bytes(kv_es(dtype), kv_steps(D)); }
// slots and positions are counted in 32 bits
inline bool kv_valid_slots(int64_t pages, int64_t page) { return pages >= 1 && pages <= INT32_MAX / page; }

// Whether N x H rows of D elements, ld and hs elements apart, have none in common: results that do are refused.
inline bool kv_rows_apart(int64_t N, int64_t ld, int64_t H, int64_t hs, int64_t D)
{
    if (N < 2 || H < 2) return (N < 2 || ld >= D) && (H < 2 || hs >= D);
    if (ld < D || hs < D) return false;
    if (ld >= (H - 1) * hs + D || hs >= (N - 1) * ld + D) return true;      // heads within tokens, or tokens within heads
    for (int64_t h = 1; h < H; ++h)                  // h heads on and n tokens back
        for (int64_t n = h * hs / ld, last = n + 1; n <= last; ++n)
            if (n >= 1 && n < N && h * hs - n * ld < D && n * ld - h * hs < D) return false;
    return true;
}

// ---- kv_tables: by how many launches ----
constexpr int KT_THREADS = 1024;
// New tokens up to which the plan's workgroup fills in the slots too.  One workgroup | every one plans | two launches, us a call: 64 requests, 1024 tokens 5.6 | 6.0 |
// 8.4, 2048 6.5 | 6.1 | 8.7, 4096 8.2 | 6.1 | 8.8, 32768 32 | 6.3 | 8.8; one request, 4096 5.4 | 5.5 | 8.6, 32768 17 | 5.5 | 8.6; 512 requests, 4096 9.1 | 6.3 | 9.5.
constexpr int64_t KT_ONE_LAUNCH = 2048;
constexpr int KT_WHOLE = 0, KT_EVERY = 1, KT_PLAN = 2;      // one workgroup; every workgroup plans; the plan goes through memory to a second launch

// whether lists of n and m numbers of 32 bits have memory in common
inline bool kv_overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) { return n > 0 && m > 0 && (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n); }

// Where every workgroup plans, the first one writes new_lens and new_left while others may still read lens, want and left: only if no memory is both.
inline int kt_route(const int32_t* lens, const int32_t* want, int64_t B, const int32_t* left, int64_t N, const int32_t* new_lens, const int32_t* new_left)
{
    if (N <= KT_ONE_LAUNCH) return KT_WHOLE;
    const bool apart = !kv_overlap(new_lens, B, lens, B) && !kv_overlap(new_lens, B, want, B) && !kv_overlap(new_lens, B, left, 1) && !kv_overlap(new_left, 1, lens, B) &&
                       !kv_overlap(new_left, 1, want, B) && !kv_overlap(new_left, 1, left, 1);
    return B <= KT_THREADS && apart ? KT_EVERY : KT_PLAN;
}

// where 8-value piece c (values 8 c .. 8 c + 7) of a token's key lies in its block, for token tau of the block
__device__ inline int kv_key_at(int es, int tau, int c)
{
    const int t = (tau >> 2) & 1, lane = (c & 3) * 16 + 4 * (tau >> 3) + (tau & 3), s = c >> 2;
    return es == 2 ? ((2 * s + t) * 64 + lane) * 16 : ((s * 64 + lane) * 2 + t) * 8;
}
// where the values of channel d of tokens 8 j .. 8 j + 7 lie among a block's values
__device__ inline int kv_value_at(int es, int j, int d)
{
    const int lane = j * 16 + (d & 15);
    return es == 2 ? ((d >> 4) * 64 + lane) * 16 : (((d >> 5) * 64 + lane) * 2 + ((d >> 4) & 1)) * 8;
}

}  // namespace ss
