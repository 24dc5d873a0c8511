// expert_route, expert_combine: which experts a token's row goes to and in what order the rows lie for them, and the weighted sum of what
// the experts answer.
#include "mx4_common.h"
#include "quant_common.h"
#include "device_info.h"

namespace ss {

constexpr int RT_TOKENS = 64;            // tokens of a workgroup: one bit each in the experts' masks
constexpr int RT_WAVES = 16;
constexpr int RT_THREADS = 64 * RT_WAVES;
constexpr int RT_MAX_K = 64;

// Scores as unsigned keys in their order; a NaN lies below every number, 0 is none at all.
__device__ inline uint32_t score_key(float x)
{
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x + 0.0f);                 // -0 equals 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float key_score(uint32_t k) { return k == 1 ? __uint_as_float(0x7FC00000u) : __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k); }

// largest key of a wavefront, in every lane
__device__ inline uint32_t wave_max(uint32_t v)
{
    auto step = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x111, 0xF, 0xF, false));      // row_shr:1
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x112, 0xF, 0xF, false));      // 2
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x114, 0xF, 0xF, false));      // 4
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x118, 0xF, 0xF, false));      // 8
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x142, 0xA, 0xF, false));      // row_bcast:15
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x143, 0xC, 0xF, false));      // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// The experts of 64 tokens: a wavefront per token, EL scores to a lane (expert 64 j + lane).  Which tokens of the workgroup take an expert
// is a mask of 64 bits in LDS; the place of a row among the workgroup's rows for its expert is the number of bits below its own,
// whatever the order in which they were set.
// ONE: the only workgroup, which then knows the order; otherwise slots gets the places and counts[expert][workgroup] the numbers of rows.
template <typename T, int EL, bool ONE>
__global__ __launch_bounds__(RT_THREADS) void k_route_choose(const T* __restrict__ logits, int64_t M, int E, int64_t ld, int k, bool renormalise,
                                                             int32_t* __restrict__ ids, float* __restrict__ weights, int32_t* __restrict__ slots,
                                                             int32_t* __restrict__ rows, int32_t* __restrict__ offsets, int32_t* __restrict__ counts)
{
    __shared__ unsigned long long mask[64 * EL];
    __shared__ int32_t start[ONE ? 64 * EL + 1 : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int e = threadIdx.x; e < 64 * EL; e += RT_THREADS) mask[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * RT_TOKENS;
    const int tokens = (int)min((int64_t)RT_TOKENS, M - first);
    constexpr int PER = RT_TOKENS / RT_WAVES;
    int mine[PER];                                       // lane j < k: the j-th expert of the wavefront's tokens
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = wave + RT_WAVES * p;
        mine[p] = 0;
        if (t >= tokens) continue;
        const T* const row = logits + (first + t) * ld;
        uint32_t key[EL];
#pragma unroll
        for (int j = 0; j < EL; ++j) key[j] = 64 * j + lane < E ? score_key(load_scalar(row + 64 * j + lane)) : 0;
        uint32_t chosen = 0;
        float top = 0.0f, total = 0.0f;
        for (int i = 0; i < k; ++i) {
            uint32_t best = key[0];
#pragma unroll
            for (int j = 1; j < EL; ++j) best = max(best, key[j]);
            best = wave_max(best);
            if (i == 0) {
                top = key_score(best);
                if (!renormalise) {                      // the sum over all experts, before any is taken out
                    float part = 0.0f;
#pragma unroll
                    for (int j = 0; j < EL; ++j)
                        if (key[j]) part += expf(key_score(key[j]) - top);
                    total = wave_sum(part);
                }
            }
            int at = -1;
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                const uint64_t has = __ballot(key[j] == best);
                if (at < 0 && has) {
                    at = 64 * j + __ffsll((unsigned long long)has) - 1;
                    if (lane == (at & 63)) key[j] = 0;
                }
            }
            if (lane == i) { chosen = best; mine[p] = at; }
        }
        float w = lane < k ? expf(key_score(chosen) - top) : 0.0f;
        if (renormalise) total = wave_sum(w);
        w = top == -INFINITY ? 0.0f : w / total;         // all scores of a row at minus infinity: no expert has a weight
        if (lane < k) {
            ids[(first + t) * k + lane] = mine[p];
            weights[(first + t) * k + lane] = w;
            atomicOr(&mask[mine[p]], 1ull << t);
        }
    }
    __syncthreads();
    if constexpr (ONE) {
        if (wave == 0) {                                 // first place of each expert
            int before = 0;
            for (int e0 = 0; e0 < E; e0 += 64) {
                const int c = __popcll(mask[e0 + lane]);
                int sum = c;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(sum, d, 64);
                    if (lane >= d) sum += o;
                }
                start[e0 + lane] = before + sum - c;
                if (e0 + lane < E) offsets[e0 + lane] = before + sum - c;
                before += __shfl(sum, 63, 64);
            }
            if (lane == 0) offsets[E] = before;
        }
        __syncthreads();
    } else {
        for (int e = threadIdx.x; e < E; e += RT_THREADS) counts[(int64_t)e * gridDim.x + blockIdx.x] = __popcll(mask[e]);
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = wave + RT_WAVES * p;
        if (t >= tokens || lane >= k) continue;
        const int place = __popcll(mask[mine[p]] & ((1ull << t) - 1));
        if constexpr (ONE) {
            slots[t * k + lane] = start[mine[p]] + place;
            rows[start[mine[p]] + place] = t;
        } else slots[(first + t) * k + lane] = place;
    }
}

// counts[expert][workgroup] -> rows of the expert before the workgroup's; totals[expert].  A workgroup per expert.
__global__ __launch_bounds__(256) void k_route_scan(int32_t* __restrict__ counts, int B, int32_t* __restrict__ totals)
{
    __shared__ int part[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int32_t* const c = counts + (int64_t)blockIdx.x * B;
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += 256) {
        const int b = b0 + threadIdx.x, v = b < B ? c[b] : 0;
        int sum = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d, 64);
            if (lane >= d) sum += o;
        }
        if (lane == 63) part[wave] = sum;
        __syncthreads();
        int add = before, all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) add += part[w];
            all += part[w];
        }
        if (b < B) c[b] = add + sum - v;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// places within the workgroups -> places in the order of the experts
__global__ __launch_bounds__(256) void k_route_place(const int32_t* __restrict__ ids, const int32_t* __restrict__ counts, const int32_t* __restrict__ totals,
                                                     int64_t M, int E, int k, int B, int32_t* __restrict__ slots, int32_t* __restrict__ rows,
                                                     int32_t* __restrict__ offsets)
{
    __shared__ int32_t start[MX_MAX_EXPERTS + 64];
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        int before = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int c = e0 + lane < E ? totals[e0 + lane] : 0;
            int sum = c;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(sum, d, 64);
                if (lane >= d) sum += o;
            }
            start[e0 + lane] = before + sum - c;
            if (blockIdx.x == 0 && e0 + lane < E) offsets[e0 + lane] = before + sum - c;
            before += __shfl(sum, 63, 64);
        }
        if (blockIdx.x == 0 && lane == 0) offsets[E] = before;
    }
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * RT_TOKENS * k, end = min(first + (int64_t)RT_TOKENS * k, M * k);
    for (int64_t i = first + threadIdx.x; i < end; i += 256) {
        const int e = ids[i], s = start[e] + counts[(int64_t)e * B + blockIdx.x] + slots[i];
        slots[i] = s;
        rows[s] = (int32_t)(i / k);
    }
}

typedef uint32_t row16_t __attribute__((ext_vector_type(4), aligned(2)));

// A thread takes eight columns of a token.
__global__ __launch_bounds__(256) void k_combine(const uint16_t* __restrict__ Y, int64_t R, int64_t O, int64_t ldy, const int32_t* __restrict__ slots,
                                                 const float* __restrict__ weights, int64_t M, int k, const uint16_t* __restrict__ base, int64_t ldb,
                                                 uint16_t* __restrict__ out, int64_t ldo, int64_t per_row)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / per_row, o = (i - m * per_row) * 8;
    if (m >= M) return;
    const int have = (int)min((int64_t)8, O - o);
    float a[8];
    auto get = [&](const uint16_t* p, float (&f)[8]) {
        if (have == 8) {
            const row16_t v = *reinterpret_cast<const row16_t*>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(v[j] << 16); f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u); }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = j < have ? bf16_bits_to_f32(p[j]) : 0.0f;
        }
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = 0.0f;
    for (int q = 0; q < k; ++q) {
        const int64_t s = slots[m * k + q];
        if (s < 0 || s >= R) continue;
        const float w = weights[m * k + q];
        float f[8];
        get(Y + s * ldy + o, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = fmaf(w, f[j], a[j]);
    }
    if (base) {
        float f[8];
        get(base + m * ldb + o, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] += f[j];
    }
    uint16_t* const dst = out + m * ldo + o;
    const uint32_t w[4] = {pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(a[4], a[5]), pack_bf16x2(a[6], a[7])};
    if (have == 8) *reinterpret_cast<row16_t*>(dst) = row16_t{w[0], w[1], w[2], w[3]};
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < have) dst[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}

template <typename T, int EL>
static ss_status launch_route(const void* logits, int64_t M, int64_t E, int64_t ld, int k, bool renormalise, int32_t* ids, float* weights, int32_t* slots,
                              int32_t* rows, int32_t* offsets, int32_t* counts, hipStream_t hs)
{
    const int64_t B = M == 0 ? 1 : (M + RT_TOKENS - 1) / RT_TOKENS;       // without tokens the offsets are written all the same
    const T* const x = static_cast<const T*>(logits);
    if (B == 1) {
        hipLaunchKernelGGL((k_route_choose<T, EL, true>), dim3(1), dim3(RT_THREADS), 0, hs, x, M, (int)E, ld, k, renormalise, ids, weights, slots, rows, offsets, counts);
        return launch_status();
    }
    hipLaunchKernelGGL((k_route_choose<T, EL, false>), dim3((uint32_t)B), dim3(RT_THREADS), 0, hs, x, M, (int)E, ld, k, renormalise, ids, weights, slots, rows, offsets, counts);
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    int32_t* const totals = counts + E * B;
    hipLaunchKernelGGL(k_route_scan, dim3((uint32_t)E), dim3(256), 0, hs, counts, (int)B, totals);
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    hipLaunchKernelGGL(k_route_place, dim3((uint32_t)B), dim3(256), 0, hs, ids, counts, totals, M, (int)E, k, (int)B, slots, rows, offsets);
    return launch_status();
}

}  // namespace ss

using namespace ss;

static bool valid_route(int64_t M, int64_t E, int64_t k) { return M >= 0 && M <= MX_MAX_ROWS && E >= 1 && E <= MX_MAX_EXPERTS && k >= 1 && k <= RT_MAX_K && k <= E && M * k <= INT32_MAX; }

extern "C" size_t expert_route_workspace_bytes(int64_t M, int64_t E, int64_t k)
{
    if (!valid_route(M, E, k) || M <= RT_TOKENS) return 0;
    return (size_t)(E * ((M + RT_TOKENS - 1) / RT_TOKENS + 1)) * 4;
}

extern "C" ss_status expert_route(const void* logits, ss_act_dtype in_dtype, int64_t M, int64_t E, int64_t ld, int k, int renormalise, int32_t* ids,
                                  float* weights, int32_t* slots, int32_t* rows, int32_t* offsets, void* workspace, size_t workspace_bytes, void* stream)
{
    if (in_dtype != SS_IN_F32 && in_dtype != SS_IN_BF16) return SS_ERR_DTYPE;
    if (!valid_route(M, E, k) || ld < E || (renormalise != 0 && renormalise != 1)) return SS_ERR_SHAPE;
    if (!offsets || (M > 0 && (!logits || !ids || !weights || !slots || !rows))) return SS_ERR_NULL;
    const size_t need = expert_route_workspace_bytes(M, E, k);
    if (need > 0 && !workspace) return SS_ERR_NULL;
    if (((uintptr_t)workspace & 15) || workspace_bytes < need) return SS_ERR_WORKSPACE;
    if (((uintptr_t)logits & (in_dtype == SS_IN_F32 ? 3 : 1)) || (((uintptr_t)ids | (uintptr_t)weights | (uintptr_t)slots | (uintptr_t)rows | (uintptr_t)offsets) & 3))
        return SS_ERR_SHAPE;
    hipStream_t hs = static_cast<hipStream_t>(stream);
#define SS_RT(T, EL) launch_route<T, EL>(logits, M, E, ld, k, renormalise != 0, ids, weights, slots, rows, offsets, static_cast<int32_t*>(workspace), hs)
#define SS_RE(T) (E <= 64 ? SS_RT(T, 1) : E <= 128 ? SS_RT(T, 2) : E <= 256 ? SS_RT(T, 4) : E <= 512 ? SS_RT(T, 8) : SS_RT(T, 16))
    return in_dtype == SS_IN_F32 ? SS_RE(float) : SS_RE(uint16_t);
#undef SS_RE
#undef SS_RT
}

extern "C" ss_status expert_combine(const void* Y, int64_t R, int64_t O, int64_t ldy, const int32_t* slots, const float* weights, int64_t M, int k,
                                    const void* base, int64_t ldb, void* out, int64_t ldo, void* stream)
{
    if (R < 0 || R > INT32_MAX || M < 0 || M > MX_MAX_ROWS || O < 0 || O > MX_MAX_K || k < 1 || k > RT_MAX_K || ldy < O || ldo < O || (base && ldb < O)) return SS_ERR_SHAPE;
    if (M == 0 || O == 0) return SS_OK;
    if ((!Y && R > 0) || !slots || !weights || !out) return SS_ERR_NULL;
    if ((((uintptr_t)Y | (uintptr_t)base | (uintptr_t)out) & 1) || (((uintptr_t)slots | (uintptr_t)weights) & 3)) return SS_ERR_SHAPE;
    const int64_t per_row = (O + 7) / 8, blocks = (M * per_row + 255) / 256;
    if (blocks > INT32_MAX) return SS_ERR_SHAPE;
    hipLaunchKernelGGL(k_combine, dim3((uint32_t)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(Y), R, O, ldy, slots, weights, M, k,
                       static_cast<const uint16_t*>(base), ldb, static_cast<uint16_t*>(out), ldo, per_row);
    return launch_status();
}
