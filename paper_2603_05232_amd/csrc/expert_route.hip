// expert_route, expert_combine: which experts a token's row goes to and in what order the rows lie for them, and the weighted sum of what
// the experts answer.
#include "mx4_common.h"
#include "quant_common.h"
#include "device_info.h"

namespace ss {

constexpr int RT_TOKENS = 64;            // tokens of a workgroup: one bit each in the experts' masks
constexpr int RT_THREADS = 16 * RT_TOKENS;
constexpr int RT_MAX_K = 64;

// Scores as unsigned keys in their order; a NaN lies below every number, 0 is none at all.
__device__ inline uint32_t score_key(float x)
{
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x + 0.0f);                 // -0 equals 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float key_score(uint32_t k) { return k == 1 ? __uint_as_float(0x7FC00000u) : __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k); }

// over a row of sixteen lanes, in every lane: rotations by 8, 4, 2 and 1
template <typename F> __device__ inline int row_all(int v, F f)
{
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, true));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, true));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, true));
    return f(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, true));
}
__device__ inline uint32_t row_max(uint32_t v) { return (uint32_t)row_all((int)v, [](int a, int b) { return (int)max((uint32_t)a, (uint32_t)b); }); }
__device__ inline int row_min(int v) { return row_all(v, [](int a, int b) { return min(a, b); }); }
__device__ inline float row_sum(float v) { return __int_as_float(row_all(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); })); }

// The experts of 64 tokens: sixteen lanes to a token, four tokens to a wavefront, EL scores to a lane (expert 16 j + lane).  Which tokens of the
// workgroup take an expert is a mask of 64 bits in LDS; the place of a row among the workgroup's rows for its expert is the number of bits
// below its own, whatever the order in which they were set.
// A lane keeps KL choices, number 16 c + l.
// ONE: the only workgroup, which then knows the order; otherwise slots gets the places and counts[workgroup][expert] the numbers of rows.
// Bound by instructions on the compute units that have a workgroup (8192 x 128 bf16, k = 8: 7.0 us for 2 MB, 128 workgroups on 256): a choice is about 8 EL + 30 of
// them, for four tokens at once (a wavefront for each token, 8192 x 128 bf16, k = 8: 14.4 us).
template <typename T, int EL, int KL, bool ONE>
__global__ __launch_bounds__(RT_THREADS) void k_route_choose(const T* __restrict__ logits, int64_t M, int E, int64_t ld, int k, bool renormalise,
                                                             int32_t* __restrict__ ids, float* __restrict__ weights, int32_t* __restrict__ slots,
                                                             int32_t* __restrict__ rows, int32_t* __restrict__ offsets, int32_t* __restrict__ counts)
{
    constexpr int ALL = 16 * EL;
    __shared__ unsigned long long mask[ALL];
    __shared__ int32_t start[ONE ? ALL : 1];
    const int lane = threadIdx.x & 63, l = lane & 15;
    for (int e = threadIdx.x; e < ALL; e += RT_THREADS) mask[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * RT_TOKENS;
    const int t = threadIdx.x >> 4;                      // this lane's token of the workgroup's
    const bool there = first + t < M;
    const T* const row = logits + (there ? first + t : 0) * ld;
    uint32_t key[EL];
#pragma unroll
    for (int j = 0; j < EL; ++j) key[j] = there && 16 * j + l < E ? score_key(load_scalar(row + 16 * j + l)) : 0;
    uint32_t chosen[KL];
    int mine[KL];
#pragma unroll
    for (int c = 0; c < KL; ++c) { chosen[c] = 0; mine[c] = 0; }
    float top = 0.0f, total = 0.0f;
    for (int i = 0; i < k; ++i) {
        uint32_t best = key[0];
        int at = l;
#pragma unroll
        for (int j = 1; j < EL; ++j) {
            at = key[j] > best ? 16 * j + l : at;        // of equal ones the first
            best = max(best, key[j]);
        }
        const uint32_t most = row_max(best);
        at = row_min(best == most ? at : INT32_MAX);
        if (i == 0) {
            top = key_score(most);
            if (!renormalise) {                          // the sum over all experts, before any is taken out
                float part = 0.0f;
#pragma unroll
                for (int j = 0; j < EL; ++j) part += key[j] ? expf(key_score(key[j]) - top) : 0.0f;
                total = row_sum(part);
            }
        }
#pragma unroll
        for (int j = 0; j < EL; ++j) key[j] = 16 * j + l == at ? 0 : key[j];
#pragma unroll
        for (int c = 0; c < KL; ++c)
            if (i == 16 * c + l) { chosen[c] = most; mine[c] = at; }
    }
    float w[KL];
#pragma unroll
    for (int c = 0; c < KL; ++c) w[c] = there && 16 * c + l < k ? expf(key_score(chosen[c]) - top) : 0.0f;
    if (renormalise) {
        total = w[0];
#pragma unroll
        for (int c = 1; c < KL; ++c) total += w[c];
        total = row_sum(total);
    }
#pragma unroll
    for (int c = 0; c < KL; ++c)
        if (there && 16 * c + l < k) {
            ids[(first + t) * k + 16 * c + l] = mine[c];
            weights[(first + t) * k + 16 * c + l] = top == -INFINITY ? 0.0f : w[c] / total;      // all scores of a row at minus infinity: no expert has a weight
            atomicOr(&mask[mine[c]], 1ull << t);
        }
    __syncthreads();
    if constexpr (ONE) {
        if (threadIdx.x < 64) {                          // first place of each expert
            int before = 0;
            for (int e0 = 0; e0 < E; e0 += 64) {
                const int c = __popcll(mask[e0 + lane]), sum = wave_scan_add(c), at = before + sum - c;
                start[e0 + lane] = at;
                if (e0 + lane < E) offsets[e0 + lane] = at;
                before += __builtin_amdgcn_readlane(sum, 63);
            }
            if (lane == 0) offsets[E] = before;
        }
        __syncthreads();
    } else {
        for (int e = threadIdx.x; e < E; e += RT_THREADS) counts[(int64_t)blockIdx.x * E + e] = __popcll(mask[e]);
    }
#pragma unroll
    for (int c = 0; c < KL; ++c)
        if (there && 16 * c + l < k) {
            const int place = __popcll(mask[mine[c]] & ((1ull << t) - 1));
            if constexpr (ONE) {
                slots[t * k + 16 * c + l] = start[mine[c]] + place;
                rows[start[mine[c]] + place] = t;
            } else slots[(first + t) * k + 16 * c + l] = place;
        }
}

// counts[workgroup][expert] -> rows of the expert in the workgroups before; totals[expert].  A workgroup per expert; bound by the launch and a few waits.
__global__ __launch_bounds__(256) void k_route_scan(int32_t* __restrict__ counts, int E, int B, int32_t* __restrict__ totals)
{
    __shared__ int part[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int32_t* const c = counts + blockIdx.x;
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += 256) {
        const int b = b0 + threadIdx.x, v = b < B ? c[(int64_t)b * E] : 0, sum = wave_scan_add(v);
        if (lane == 63) part[wave] = sum;
        __syncthreads();
        int add = before, all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) add += part[w];
            all += part[w];
        }
        if (b < B) c[(int64_t)b * E] = add + sum - v;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// Places within the workgroups -> places in the order of the experts.  SCANNED: k_route_scan has added the counts up; otherwise every workgroup adds
// up all of them itself, which with few workgroups costs less than the launch in between.  Bound by those waits: 4.0 us for 8192 x 8 places.
// The whole call, own sums | scan, us, at 128 | 256 | 320 | 512 workgroups:
//     8 experts, k = 2    6.3 |  7.5      7.1 |  8.0      9.6 |  9.4     11.0 |  9.8
//    64, k = 4            7.2 |  8.6      8.2 |  9.1     11.2 | 10.9     12.7 | 11.8
//   128, k = 8           10.7 | 11.6     12.3 | 12.5     17.8 | 16.1     22.2 | 17.8
//   256, k = 8           14.8 | 14.9     18.0 | 16.7     27.5 | 22.0     34.7 | 24.7
//  1024, k = 8           55.5 | 51.0     65.1 | 54.8      122 | 96.0      144 |  101
// so beyond 128 experts the line comes late.
constexpr int RT_OWN_SUMS = 256;         // workgroups up to which they do
template <bool SCANNED>
__global__ __launch_bounds__(RT_THREADS) void k_route_place(const int32_t* __restrict__ ids, const int32_t* __restrict__ counts, const int32_t* __restrict__ totals,
                                                            int64_t M, int E, int k, int B, int32_t* __restrict__ slots, int32_t* __restrict__ rows,
                                                            int32_t* __restrict__ offsets)
{
    __shared__ int32_t before[MX_MAX_EXPERTS + 64], total[MX_MAX_EXPERTS + 64];
    const int lane = threadIdx.x & 63;
    for (int e = threadIdx.x; e < MX_MAX_EXPERTS + 64; e += RT_THREADS) {
        before[e] = SCANNED && e < E ? counts[(int64_t)blockIdx.x * E + e] : 0;
        total[e] = SCANNED && e < E ? totals[e] : 0;
    }
    __syncthreads();
    if constexpr (!SCANNED) {
        // a thread for each expert and part of the workgroups
        const int width = E <= 64 ? 64 : E <= 128 ? 128 : E <= 256 ? 256 : E <= 512 ? 512 : 1024, parts = RT_THREADS / width;
        const int e = threadIdx.x & (width - 1), per = (B + parts - 1) / parts, b0 = threadIdx.x / width * per, b1 = min(B, b0 + per);
        if (e < E) {
            int n = 0, all = 0;
#pragma unroll 8
            for (int b = b0; b < b1; ++b) {
                const int v = counts[(int64_t)b * E + e];
                all += v;
                n += b < (int)blockIdx.x ? v : 0;
            }
            if (n) atomicAdd(&before[e], n);              // whole numbers: the order does not matter
            if (all) atomicAdd(&total[e], all);
        }
        __syncthreads();
    }
    if (threadIdx.x < 64) {
        int start = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int c = total[e0 + lane], sum = wave_scan_add(c), at = start + sum - c;
            before[e0 + lane] += at;
            if (blockIdx.x == 0 && e0 + lane < E) offsets[e0 + lane] = at;
            start += __builtin_amdgcn_readlane(sum, 63);
        }
        if (blockIdx.x == 0 && lane == 0) offsets[E] = start;
    }
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * RT_TOKENS * k, end = min(first + (int64_t)RT_TOKENS * k, M * k);
    for (int64_t i = first + threadIdx.x; i < end; i += RT_THREADS) {
        const int s = before[ids[i]] + slots[i];
        slots[i] = s;
        rows[s] = (int32_t)(blockIdx.x * RT_TOKENS + (int)(i - first) / k);
    }
}

// sixteen bytes at the alignment of an element
typedef uint32_t row16_t __attribute__((ext_vector_type(4), aligned(2)));

// eight columns of a row, `have` of which exist
__device__ inline void get8(const uint16_t* p, int have, float (&f)[8])
{
    if (have == 8) {
        const row16_t v = __builtin_nontemporal_load(reinterpret_cast<const row16_t*>(p));      // read once
#pragma unroll
        for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(v[j] << 16); f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < have ? bf16_bits_to_f32(p[j]) : 0.0f;
    }
}

// out = sum of weights Y[slots] + base, in the order of the choices.  A thread takes eight columns of a token; with a known number of rows (K > 0) it asks for
// all of them before it adds the first.  Bound by HBM: 8192 tokens of 8 rows of 2048 57.5 us in a trace, 270.5 MB read and 33.6 written at 5.3 TB/s.
template <int K>
__global__ __launch_bounds__(256) void k_combine(const uint16_t* __restrict__ Y, int64_t R, int64_t O, int64_t ldy, const int32_t* __restrict__ slots,
                                                 const float* __restrict__ weights, int64_t M, int k, const uint16_t* __restrict__ base, int64_t ldb,
                                                 uint16_t* __restrict__ out, int64_t ldo, int64_t per_row)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = per_row == 1 ? i : i / per_row, o = (i - m * per_row) * 8;
    if (m >= M) return;
    const int have = (int)min((int64_t)8, O - o);
    float a[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = 0.0f;
    if constexpr (K > 0) {
        int s[K];
        float w[K], f[K][8];
#pragma unroll
        for (int q = 0; q < K; ++q) { s[q] = slots[m * K + q]; w[q] = weights[m * K + q]; }
#pragma unroll
        for (int q = 0; q < K; ++q) get8(Y + (s[q] >= 0 && s[q] < R ? s[q] : 0) * ldy + o, R > 0 ? have : 0, f[q]);
#pragma unroll
        for (int q = 0; q < K; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = s[q] >= 0 && s[q] < R ? fmaf(w[q], f[q][j], a[j]) : a[j];
    } else {
        for (int q = 0; q < k; ++q) {
            const int64_t s = slots[m * k + q];
            if (s < 0 || s >= R) continue;
            float f[8];
            get8(Y + s * ldy + o, have, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = fmaf(weights[m * k + q], f[j], a[j]);
        }
    }
    if (base) {
        float f[8];
        get8(base + m * ldb + o, have, f);
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

template <typename T, int EL, int KL>
static ss_status launch_route(const void* logits, int64_t M, int64_t E, int64_t ld, int k, bool renormalise, int32_t* ids, float* weights, int32_t* slots,
                              int32_t* rows, int32_t* offsets, int32_t* counts, hipStream_t hs)
{
    const int64_t B = M == 0 ? 1 : (M + RT_TOKENS - 1) / RT_TOKENS;       // without tokens the offsets are written all the same
    const T* const x = static_cast<const T*>(logits);
    if (B == 1) {
        hipLaunchKernelGGL((k_route_choose<T, EL, KL, true>), dim3(1), dim3(RT_THREADS), 0, hs, x, M, (int)E, ld, k, renormalise, ids, weights, slots, rows, offsets, counts);
        return launch_status();
    }
    hipLaunchKernelGGL((k_route_choose<T, EL, KL, false>), dim3((uint32_t)B), dim3(RT_THREADS), 0, hs, x, M, (int)E, ld, k, renormalise, ids, weights, slots, rows, offsets, counts);
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    int32_t* const totals = counts + E * B;
    if (B <= RT_OWN_SUMS) {
        hipLaunchKernelGGL(k_route_place<false>, dim3((uint32_t)B), dim3(RT_THREADS), 0, hs, ids, counts, totals, M, (int)E, k, (int)B, slots, rows, offsets);
        return launch_status();
    }
    hipLaunchKernelGGL(k_route_scan, dim3((uint32_t)E), dim3(256), 0, hs, counts, (int)E, (int)B, totals);
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    hipLaunchKernelGGL(k_route_place<true>, dim3((uint32_t)B), dim3(RT_THREADS), 0, hs, ids, counts, totals, M, (int)E, k, (int)B, slots, rows, offsets);
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
#define SS_RT(T, EL) (k <= 16 ? launch_route<T, EL, 1> : launch_route<T, EL, RT_MAX_K / 16>)(logits, M, E, ld, k, renormalise != 0, ids, weights, slots, rows, offsets, static_cast<int32_t*>(workspace), hs)
#define SS_RE(T) (E <= 64 ? SS_RT(T, 4) : E <= 128 ? SS_RT(T, 8) : E <= 256 ? SS_RT(T, 16) : SS_RT(T, 64))
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
    if (!mx4_grid_fits(blocks, 256)) return SS_ERR_SHAPE;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(Y), R, O, ldy, slots, weights, M, k,
                           static_cast<const uint16_t*>(base), ldb, static_cast<uint16_t*>(out), ldo, per_row);
        return launch_status();
    };
    switch (k) {
    case 1: return launch(k_combine<1>);
    case 2: return launch(k_combine<2>);
    case 4: return launch(k_combine<4>);
    case 8: return launch(k_combine<8>);
    }
    return launch(k_combine<0>);
}
