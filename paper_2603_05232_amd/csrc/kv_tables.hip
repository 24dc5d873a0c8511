// kv_tables: the pages of requests whose lengths change, and the slots of their new tokens, without a trip to the host.
#include "kv_common.h"

namespace ss {

constexpr int KT_CAP = (1 << 30) - 1;                // sums stop here, above any number that means something; two of them are still a number of 32 bits

__device__ inline int cap_add(int a, int b) { return min(a + b, KT_CAP); }

// Inclusive sums over the workgroup's threads (values >= 0), of as many numbers as `part` has rows; total: that of all.  part is used anew in every call.
template <int NUM> __device__ inline void block_scan(int (&v)[NUM], int (*part)[KT_THREADS / 64], int (&total)[NUM])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < NUM; ++q) {
        v[q] = wave_scan(min(v[q], KT_CAP), 0, [](int a, int b) { return cap_add(a, b); });
        if (lane == 63) part[q][wave] = v[q];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NUM; ++q) {
        const int all = wave_scan(lane < KT_THREADS / 64 ? part[q][lane] : 0, 0, [](int a, int b) { return cap_add(a, b); });      // lane w: of wavefronts 0 .. w
        const int before = wave == 0 ? 0 : __builtin_amdgcn_readlane(all, wave - 1);
        v[q] = cap_add(before, v[q]);
        total[q] = __builtin_amdgcn_readlane(all, 63);
    }
}

// What filling in needs of each of up to MAX requests.
template <int MAX> struct KtPlan {
    int32_t start[MAX + 1];                          // its first new token's row
    int32_t len[MAX];                                // its length before
    int32_t first[MAX];                              // pages taken by requests before it; -1: it gets no slots
    int32_t pages;                                   // free pages, those that were given back among them
};
constexpr int KT_MAX = (int)KV_MAX_REQUESTS;

// the last of 0 .. n - 1 at which a list that does not fall is at most x; 0 if there is none
__device__ inline int kt_search(const int32_t* list, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Row i: the request that it belongs to, its position there, its page.  A new page is entered in the table by the row that begins it.  page_at(k): entry k of the stack.
template <int MAX, typename F>
__device__ inline void kt_fill(const int32_t* start, const KtPlan<MAX>& plan, int i, int B, int32_t* __restrict__ table, int64_t ldt, int page, Div by_page, F page_at, int P,
                               int32_t* __restrict__ slots)
{
    if (i >= start[B]) { slots[i] = -1; return; }
    const int b = kt_search(start, B, i), first = plan.first[b];
    if (first < 0) { slots[i] = -1; return; }
    const int len = plan.len[b], at = len + (i - start[b]), column = quot(at, by_page), row = at - column * page, have = quot(len + page - 1, by_page);
    int32_t* const cell = table + b * ldt + column;
    int id;
    if (column >= have) {
        const int k = plan.pages - 1 - (first + column - have);      // from the top of the stack
        id = k >= 0 && k < P ? page_at(k) : -1;
        if (row == 0) *cell = id;
    } else id = *cell;
    slots[i] = id >= 0 && id < P ? id * page + row : -1;
}

// The requests' numbers are few: one workgroup.  Bound by the launch and its waits, lengths and sums and slots: 64 requests of one token more 3.5 us in a trace (4.8 with
// sums by shuffles through LDS).  Every input is read before the barrier behind which outputs are written, so new_lens and new_left may lie in the memory of lens, want
// and left.  With many rows, either
//   KT_EVERY   every workgroup works the plan out, the first one writes it, each fills in its rows; pages that this call gives back are taken from the table, not from
//              the stack that another workgroup is writing.  Where new_lens and new_left are memory of their own (kt_route), for up to 1024 requests.
//   KT_PLAN    the plan goes through memory to a second launch.
template <int MODE>
__global__ __launch_bounds__(KT_THREADS) void k_kv_plan(const int32_t* lens, const int32_t* want, int B, int32_t* table, int64_t ldt, int W, int page, Div by_page, int32_t* pool, int P,
                                                        const int32_t* left, int N, int32_t* new_lens, int32_t* new_left, int32_t* __restrict__ slots,
                                                        int32_t* __restrict__ offsets, KtPlan<KT_MAX>* __restrict__ out)
{
    constexpr int MAX = MODE == KT_EVERY ? KT_THREADS : KT_MAX, PER = MAX / KT_THREADS;
    __shared__ KtPlan<MAX> plan;
    __shared__ int part[2 * PER][2][KT_THREADS / 64];
    __shared__ int taken;
    __shared__ int32_t back_from[MODE == KT_EVERY ? MAX : 1], needs[MODE == KT_EVERY ? MAX : 1];      // pages given back by requests before; pages that are kept
    const bool writes = MODE != KT_EVERY || blockIdx.x == 0;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, most = W * page;
    const int free_before = min(max(*left, 0), P);
    if (threadIdx.x == 0) taken = 0;
    int rows = 0, pages = 0, back = 0;               // sums of the requests before
    int wanted[PER], upto[PER];                      // the thread's requests: length wanted (-1: not possible); pages that are taken up to this one, if it takes any
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const int b0 = q * KT_THREADS, b = b0 + threadIdx.x;
        wanted[q] = upto[q] = 0;
        if (b0 >= B) continue;                       // the same for all threads
        const int l = b < B ? min(max(lens[b], 0), most) : 0, w = b < B ? max(want[b], 0) : 0;
        const int have = quot(l + page - 1, by_page), need = quot(min(w, most) + page - 1, by_page);
        const int grow = max(w - l, 0), fewer = w < l ? have - need : 0;
        int sums[2] = {min(grow, N + 1), fewer}, all[2];
        block_scan(sums, part[2 * q], all);
        const int end = cap_add(rows, sums[0]), given = cap_add(back, sums[1]);
        rows = cap_add(rows, all[0]);
        back = cap_add(back, all[1]);
        const bool possible = w <= most && end <= N;
        const int more = possible ? max(need - have, 0) : 0;
        int taken_to[1] = {more}, all_taken[1];
        block_scan(taken_to, part[2 * q + 1], all_taken);
        const int up = cap_add(pages, taken_to[0]);
        pages = cap_add(pages, all_taken[0]);
        if (b < B) {
            plan.start[b] = min(end - min(grow, N + 1), N);
            plan.len[b] = l;
            plan.first[b] = up - more;
            if constexpr (MODE == KT_EVERY) { back_from[b] = given - fewer; needs[b] = need; }
        }
        upto[q] = more > 0 ? up : 0;
        wanted[q] = possible || w <= l ? w : -1;
        // pages given back: sixteen lanes to a request that has any, four of them at a time
        for (uint64_t has = writes ? __ballot(fewer > 0) : 0; has;) {
            int at = -1;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if (has && lane >> 4 == g) at = __ffsll((unsigned long long)has) - 1;
                has &= has - 1;
            }
            const int from = max(at, 0), n = __shfl(fewer, from, 64), to = free_before + __shfl(given, from, 64) - n, column = __shfl(need, from, 64);
            if (at < 0) continue;
            const int32_t* const ids = table + (int64_t)(b0 + wave * 64 + at) * ldt + column;
            for (int x = lane & 15; x < n; x += 16)
                if (to + x < P) pool[to + x] = ids[x];
        }
    }
    const int all_pages = min(cap_add(free_before, back), P);
    if (threadIdx.x == 0) { plan.start[B] = min(rows, N); plan.pages = all_pages; }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const int b = q * KT_THREADS + threadIdx.x;
        if (b >= B) continue;
        const bool served = wanted[q] >= 0 && upto[q] <= all_pages;
        if (!served) plan.first[b] = -1;
        else if (upto[q] > 0) atomicMax(&taken, upto[q]);            // whole numbers: the order does not matter
        if (writes) {
            new_lens[b] = served ? wanted[q] : plan.len[b];
            offsets[b] = plan.start[b];
        }
    }
    __syncthreads();
    if (writes && threadIdx.x == 0) { offsets[B] = plan.start[B]; *new_left = all_pages - taken; }
    if constexpr (MODE == KT_PLAN) {
        for (int b = threadIdx.x; b <= B; b += KT_THREADS) out->start[b] = plan.start[b];
        for (int b = threadIdx.x; b < B; b += KT_THREADS) { out->len[b] = plan.len[b]; out->first[b] = plan.first[b]; }
        if (threadIdx.x == 0) out->pages = plan.pages;
    } else {
        auto page_at = [&](int k) -> int32_t {
            if constexpr (MODE == KT_EVERY) {
                if (k >= free_before) {
                    const int b = kt_search(back_from, B, k - free_before);
                    return table[b * ldt + needs[b] + (k - free_before - back_from[b])];
                }
            }
            return pool[k];
        };
        for (int i = blockIdx.x * KT_THREADS + threadIdx.x; i < N; i += gridDim.x * KT_THREADS) kt_fill(plan.start, plan, i, B, table, ldt, page, by_page, page_at, P, slots);
    }
}

// Slots by as many workgroups as the rows fill, for which the plan went through memory.
__global__ __launch_bounds__(256) void k_kv_slots(const KtPlan<KT_MAX>* __restrict__ plan, int B, int32_t* table, int64_t ldt, int page, Div by_page, const int32_t* __restrict__ pool, int P, int N,
                                                  int32_t* __restrict__ slots)
{
    __shared__ int32_t start[KT_MAX + 1];
    for (int b = threadIdx.x; b <= B; b += 256) start[b] = plan->start[b];
    __syncthreads();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < N) kt_fill(start, *plan, i, B, table, ldt, page, by_page, [=](int k) { return pool[k]; }, P, slots);
}

}  // namespace ss

using namespace ss;

static bool valid_tables(int64_t B, int64_t N) { return B >= 0 && B <= KV_MAX_REQUESTS && N >= 0 && N <= KV_MAX_TOKENS; }

extern "C" size_t kv_tables_workspace_bytes(int64_t B, int64_t N) { return valid_tables(B, N) && N > KT_ONE_LAUNCH ? sizeof(KtPlan<KT_MAX>) : 0; }

extern "C" ss_status kv_tables(const int32_t* lens, const int32_t* want, int64_t B, int32_t* table, int64_t ldt, int64_t W, int64_t page, int32_t* pool, int64_t P, const int32_t* left,
                               int64_t N, int32_t* new_lens, int32_t* new_left, int32_t* slots, int32_t* offsets, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!valid_tables(B, N) || page < KV_BLOCK || page > 4096 || page % KV_BLOCK || !kv_valid_slots(P, page) || W < 1 || W > INT32_MAX / page - 1 || ldt < W) return SS_ERR_SHAPE;
    if ((B > 0 && (!lens || !want || !table || !new_lens)) || !pool || !left || !new_left || !offsets || (N > 0 && !slots)) return SS_ERR_NULL;
    if (((uintptr_t)lens | (uintptr_t)want | (uintptr_t)table | (uintptr_t)pool | (uintptr_t)left | (uintptr_t)new_lens | (uintptr_t)new_left | (uintptr_t)slots | (uintptr_t)offsets) & 3) return SS_ERR_SHAPE;
    const size_t need = kv_tables_workspace_bytes(B, N);
    if (need > 0 && !workspace) return SS_ERR_NULL;
    if (((uintptr_t)workspace & 15) || workspace_bytes < need) return SS_ERR_WORKSPACE;
    auto meets = [&](const int32_t* list, int64_t n) {
        return kv_overlap(list, n, lens, B) || kv_overlap(list, n, want, B) || kv_overlap(list, n, left, 1) || kv_overlap(list, n, new_lens, B) || kv_overlap(list, n, new_left, 1);
    };
    if (meets(slots, N) || meets(offsets, B + 1) || kv_overlap(slots, N, offsets, B + 1) || kv_overlap(new_lens, B, new_left, 1)) return SS_ERR_SHAPE;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const Div by_page = make_div(page);
    KtPlan<KT_MAX>* const plan = static_cast<KtPlan<KT_MAX>*>(workspace);
    auto launch = [&](auto kernel, int64_t groups) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(KT_THREADS), 0, hs, lens, want, (int)B, table, ldt, (int)W, (int)page, by_page, pool, (int)P, left, (int)N, new_lens, new_left, slots, offsets, plan);
        return launch_status();
    };
    const int route = kt_route(lens, want, B, left, N, new_lens, new_left);
    if (route == KT_WHOLE) return launch(k_kv_plan<KT_WHOLE>, 1);
    if (route == KT_EVERY) return launch(k_kv_plan<KT_EVERY>, (N + KT_THREADS - 1) / KT_THREADS);
    if (launch(k_kv_plan<KT_PLAN>, 1) != SS_OK) return SS_ERR_HIP;
    hipLaunchKernelGGL(k_kv_slots, dim3((uint32_t)((N + 255) / 256)), dim3(256), 0, hs, plan, (int)B, table, ldt, (int)page, by_page, pool, (int)P, (int)N, slots);
    return launch_status();
}
