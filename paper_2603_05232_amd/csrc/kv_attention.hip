// kv_attention: the attention of one new token of each request over its pages of a cache.
//
//   out[b, head] = sum over t of p_t v_t / sum over t of p_t,   p_t = exp(scale q . k_t - m),   t in [max(0, len - window), len)
//
// One pass with a running maximum and sum for each head.  A request's blocks of 32 tokens are divided over workgroups, and a workgroup's over its wavefronts; what
// these hold (maximum, sum, weighted values) is joined in LDS, and what workgroups hold by a second kernel through the caller's workspace.
//
// Bound by HBM: each key and value is read once for all query heads of its head (a product has room for 16), 4 D operations a byte pair on matrix cores that could do
// fifty times that.  A block's products and softmax take some 2500 cycles of a wavefront, so that what counts is bytes under way: a block and a half for each of twelve
// wavefronts of a compute unit, 16 KB a block of 128 channels.  Medians of a trace: 256 requests of 4096 tokens, 4 heads of 128, bf16 319 us, 6.7 TB/s; 64 of 16384
// down to 256 167 (6.3), the same in fp8 92 .. 102 (5.9 .. 5.3); one of 131072 tokens 44.5 (6.0) and 4.6 for the join.  The counters show the cache's bytes read once (2150 MB of
// 2150).  One physical placement of the pages or another makes up to 15 % (the same call 203 and 234 us).  Requests below some 1000 tokens are bound by the waits at
// the start (lengths, table, keys, one after the other: 4.7 us for one token) and by what a compute unit draws by itself, 60 GB/s.
//
// Tried and left: equal shares of all requests' blocks, a workgroup passing from one request to the next (ragged batches the same, few short requests 30 % slower: the
// waits follow one another); eight wavefronts a workgroup; the table's first pages asked for beside the lengths (no gain); up to eight times as many parts (join 4 ->
// 10 us, the stream as it is).
#include "kv_common.h"
#include "quant_common.h"

namespace ss {

constexpr int KA_WAVES = 4;                          // wavefronts of a workgroup
constexpr int KA_COLUMNS = 16;                       // query heads of a product

typedef uint32_t ka16_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t ka8_t __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t ka16f_t __attribute__((ext_vector_type(4), aligned(4)));

// ---- how the blocks are divided ----
// Lengths are known on the device alone, so every workgroup works the division out for itself: a few loads and sums over the requests.  A replayed graph therefore
// follows lengths that grow, and no workgroup is launched for tokens that the table has room for and no request has.
struct KaDivision {
    const int32_t* lens;
    int B, most, window;                             // requests; tokens that a row of the table has room for; 0: no window
    float share;                                     // times the sum of all blocks: one less than what a workgroup takes
};
struct KaSpan { int first, blocks, len, from; };     // blocks of a request that hold tokens to be seen: positions from .. len - 1
__device__ inline KaSpan ka_span(const KaDivision& d, int b)
{
    KaSpan s;
    s.len = b < d.B ? min(max(d.lens[b], 0), d.most) : 0;
    s.from = d.window > 0 ? max(s.len - d.window, 0) : 0;
    s.first = s.from / KV_BLOCK;
    s.blocks = s.len > s.from ? (s.len + KV_BLOCK - 1) / KV_BLOCK - s.first : 0;
    return s;
}
// blocks of a workgroup
__device__ inline int ka_per(const KaDivision& d, const KaSpan& mine)
{
    const int lane = threadIdx.x & 63;
    float sum = (float)mine.blocks;
    for (int b0 = 64; b0 < d.B; b0 += 64) sum += (float)ka_span(d, b0 + lane).blocks;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);      // the same order in every wavefront
    const float n = fminf(sum * d.share, 0x1p30f);       // more than any request has
    return n < 8 * KA_WAVES ? KA_WAVES * max(1, (int)(n * (1.0f / KA_WAVES) + 0.999f)) : (int)n + 1;      // whole rounds of the wavefronts, while these are few
}
__device__ inline int ka_parts(int blocks, int per) { return blocks <= per ? 1 : (blocks + per - 1) / per; }

// ---- types ----
template <int DT> struct Ka;
template <> struct Ka<SS_BF16> {
    typedef v8bf frag;
    __device__ static v4f mma(frag a, frag b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Ka<SS_FP16> {
    typedef v8h frag;
    __device__ static v4f mma(frag a, frag b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Ka<SS_I8> : Ka<SS_BF16> {};       // codes of 8 bits are exact in bf16
template <> struct Ka<SS_FP8_E4M3> : Ka<SS_BF16> {};

__device__ inline uint32_t ka_pack(float a, float b, Ka<SS_BF16>) { return pack_bf16x2(a, b); }
__device__ inline uint32_t ka_pack(float a, float b, Ka<SS_FP16>) { return f32_to_f16_bits(a) | (uint32_t)f32_to_f16_bits(b) << 16; }

// First pieces of two numbers that are taken apart: below each of them and nearer to zero, so that what is left has the number's sign and is zero for zero alone.  Both
// pieces then multiply an infinity to the same one.  What is left is at most a unit u of the first piece's last place; as the second one it is off by 2^-9 u (half
// 2^-12 u), 2^-16 of the number (2^-22).  Above bf16's largest number the first piece is that one.
__device__ inline uint32_t ka_toward_zero(float x) { return __float_as_uint(x) - (x != 0.0f ? 1u : 0u); }
__device__ inline uint32_t ka_pack_below(float a, float b, Ka<SS_BF16>) { return __builtin_amdgcn_perm(ka_toward_zero(b), ka_toward_zero(a), 0x07060302u); }
__device__ inline uint32_t ka_pack_below(float a, float b, Ka<SS_FP16>)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float(ka_toward_zero(a)), __uint_as_float(ka_toward_zero(b))));
}
// and what they leave of a number: in half no less than its smallest, which would be rounded to zero.  PROBABILITY: not below zero, and of a NaN the first piece is one
template <int DT, bool PROBABILITY> __device__ inline void ka_leave(float& a, float& b, uint32_t both)
{
    typedef typename std::conditional<DT == SS_FP16, _Float16, __bf16>::type half_t;
    typedef half_t two_t __attribute__((ext_vector_type(2)));
    const two_t t = __builtin_bit_cast(two_t, both);
    auto rest = [](float x, float piece) {
        const float r = x - piece;
        if constexpr (DT != SS_FP16) return r;
        else if constexpr (PROBABILITY) return fmaxf(r, fminf(x, 0x1p-24f));
        else return r != 0.0f && fabsf(r) < 0x1p-24f ? copysignf(0x1p-24f, r) : r;
    };
    a = rest(a, (float)t[0]);
    b = rest(b, (float)t[1]);
}

// eight codes of 8 bits as bf16, which holds them exactly
template <int DT> __device__ inline v8bf ka_widen(uint32_t lo, uint32_t hi)
{
    if constexpr (DT == SS_FP8_E4M3) {
        typedef __bf16 two __attribute__((ext_vector_type(2)));
        const two a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const two c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        v4i r;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w = h ? hi : lo;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = (float)(int8_t)(w >> (8 * e));
            r[2 * h] = (int)__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
            r[2 * h + 1] = (int)__builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
        }
        return __builtin_bit_cast(v8bf, r);
    }
}

struct KaArgs {
    const void* q; int64_t ldq, hq;
    const uint8_t* pages; int64_t page_bytes;
    const int32_t* table; int64_t ldt;
    int H, G, tiles, D, page, P;                     // heads of keys, query heads to each, products that take
    float scale;                                     // of the scores, times log2(e)
    uint16_t* out; int64_t ldo, ho;
    int2* plan;                                      // of each request: the place of its first part, its parts (if requests are divided)
    float2* sums;                                    // [place][head of keys][tile][column]: maximum, sum
    float* parts;                                    // the same [.. , 32 NS]: weighted values
    int items, places;                               // parts of all requests; those of the requests that are in several
    Div by_heads, by_round, by_blocks;               // H; 8 tiles; blocks of a page
    KaDivision division;
};

// Wavefronts of a SIMD that registers are kept for.  128 channels in fp8 with three of them 92 us for 108 with two (64 requests up to 16384); 256 channels in int8 with
// two 126 for 146 with one.
constexpr int ka_fit(int ns) { return ns <= 4 ? 3 : 2; }
// DT: the cache's type; NS: steps of 32 values of a head; QP: pieces that a query value is taken apart into (1: bf16, 2: fp32); ONCE: up to 16 query heads to a head of
// keys, so that a block is read by one workgroup
template <int DT, int NS, int QP, bool ONCE>
__global__ __launch_bounds__(64 * KA_WAVES, ka_fit(NS)) void k_kv_attend(const KaArgs a)
{
    constexpr int ES = kv_es(DT), HALF = kv_half_bytes(ES, NS), BLOCK = kv_block_bytes(ES, NS), LOADS = HALF / 1024, NT = 2 * NS, CHUNK = NT < 32 / KA_WAVES ? NT : 32 / KA_WAVES;
    typedef typename Ka<DT>::frag frag;
    __shared__ float4 joined[KA_WAVES][CHUNK][64];
    __shared__ float2 wave_sums[KA_WAVES][KA_COLUMNS];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, j = lane >> 4;
    // Workgroups that read the same blocks follow one another on an XCD, 8 apart, so that its L2 has the blocks for all of them.
    int at_head = blockIdx.x, tile = 0;
    if constexpr (!ONCE) {
        const int round = quot(blockIdx.x, a.by_round), within = blockIdx.x - round * 8 * a.tiles;
        tile = within >> 3;
        at_head = round * 8 + (within & 7);
    }
    const int item = quot(at_head, a.by_heads), h = at_head - item * a.H, unit = h * a.tiles + tile;
    if (!ONCE && item >= a.items) return;

    // this workgroup's request and its part of it
    int b = -1, part = 0, parts = 1, place = 0;      // a part's place among those of requests that are divided: the others take none
    KaSpan span = {0, 0, 0, 0};
    if (!a.plan) {
        b = item;
        span = ka_span(a.division, b);
    } else {
        const KaSpan mine = ka_span(a.division, lane);   // of the first 64 requests, which mostly are all
        const int per = ka_per(a.division, mine);
        for (int b0 = 0, before = 0, whole = 0; b0 < a.division.B; b0 += 64) {
            const KaSpan s = b0 == 0 ? mine : ka_span(a.division, b0 + lane);
            const int n = b0 + lane < a.division.B ? ka_parts(s.blocks, per) : 0, upto = before + wave_scan_add(n);
            const uint64_t has = __ballot(upto > item), single = __ballot(n == 1);
            if (has) {
                const int at = __ffsll((unsigned long long)has) - 1;
                b = b0 + at;
                parts = __builtin_amdgcn_readlane(n, at);
                part = item - (__builtin_amdgcn_readlane(upto, at) - parts);
                place = item - whole - __popcll(single & (((uint64_t)1 << at) - 1));
                span = {__builtin_amdgcn_readlane(s.first, at), __builtin_amdgcn_readlane(s.blocks, at), __builtin_amdgcn_readlane(s.len, at), __builtin_amdgcn_readlane(s.from, at)};
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            whole += __popcll(single);
        }
    }
    if (b < 0 || (parts > 1 && place >= a.places)) return;      // (the latter only if lengths are changed while they are read)
    if (a.plan && part == 0 && unit == 0 && threadIdx.x == 0) a.plan[b] = make_int2(place, parts);
    const int each = (span.blocks + parts - 1) / parts, lo = span.first + part * each, end = min(lo + each, span.first + span.blocks);

    // The queries' loads: lane (r, j) gets values 32 s + 8 j .. + 7 of head r, four words of two or eight of one.  Long heads are shared out among the wavefronts,
    // which leave their operands in LDS: all of them would take the registers that a second wavefront of the SIMD needs.
    constexpr bool SHARED = NS > 4;
    constexpr int OWN = SHARED ? (NS + KA_WAVES - 1) / KA_WAVES : NS;
    __shared__ v4i shared_q[SHARED ? QP : 1][SHARED ? NS : 1][64];
    auto own = [&](int u) { return SHARED ? wave + u * KA_WAVES : u; };
    const int column = tile * KA_COLUMNS + r;
    const bool there = column < a.G;
    uint32_t raw[OWN][4 * QP];
    {
        typedef typename std::conditional<QP == 1, uint16_t, float>::type T;
        const T* const p = static_cast<const T*>(a.q) + (b * a.ldq + (int64_t)(h * a.G + (there ? column : 0)) * a.hq);
        // whole pieces first, all of them: a branch between two loads makes the second wait for the first
#pragma unroll
        for (int u = 0; u < OWN; ++u) {
            const int d = 32 * own(u) + 8 * j;
            const bool all = there && d + 8 <= a.D;
            if constexpr (QP == 1) {
                ka16_t x = {0, 0, 0, 0};
                if (all) x = *reinterpret_cast<const ka16_t*>(p + d);
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[u][e] = x[e];
            } else {
                ka16f_t x = {0, 0, 0, 0}, y = x;
                if (all) { x = *reinterpret_cast<const ka16f_t*>(p + d); y = *reinterpret_cast<const ka16f_t*>(p + d + 4); }
#pragma unroll
                for (int e = 0; e < 4; ++e) { raw[u][e] = x[e]; raw[u][4 + e] = y[e]; }
            }
        }
        if (a.D & 7) {
#pragma unroll
            for (int u = 0; u < OWN; ++u) {
                const int d = 32 * own(u) + 8 * j, have = there ? a.D - d : 0;
                if (have <= 0 || have >= 8) continue;
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < have) {
                        if constexpr (QP == 1) raw[u][e >> 1] |= (uint32_t)p[d + e] << (16 * (e & 1));
                        else raw[u][e] = __float_as_uint(p[d + e]);
                    }
            }
        }
    }
    const int per_page = a.page / KV_BLOCK;
    const int32_t* const row = a.table + b * a.ldt;
    // This wavefront's blocks are first, first + KA_WAVES, ..: lane i holds the page of the i-th of 64 of them.  The keys of the next block are asked for when those of
    // this one have been multiplied, the values likewise, into the same registers: a block is always under way.
    const int first = lo + wave, blocks = first < end ? (end - first + KA_WAVES - 1) / KA_WAVES : 0;
    int ids = 0, at_page = 0;                        // at_page: this lane's block of its page
    bool valid = false, next_valid = false;
    const uint8_t* from = a.pages;
    uint4 k[LOADS], v[LOADS];
    float ks[8], vs[8];
    auto go_to = [&](int i) {
        if ((i & 63) == 0) {
            const int block = min(first + (i + lane) * KA_WAVES, end - 1), index = quot(block, a.by_blocks);
            ids = row[index];
            at_page = block - index * per_page;
        }
        const int id = __builtin_amdgcn_readlane(ids, i & 63);
        next_valid = id >= 0 && id < a.P;            // no page: nothing to see, whatever is read instead
        from = a.pages + (next_valid ? id : 0) * a.page_bytes + (int64_t)(h * per_page + __builtin_amdgcn_readlane(at_page, i & 63)) * BLOCK;
    };
    // Blocks that one workgroup reads go past the caches (plain loads: 64 x 16384 ragged 192 us for 171, 256 x 4096 365 for 325); those of more than 16 heads, which
    // several read, do not.
    auto load16 = [&](const uint8_t* p) {
        const uint4* const x = reinterpret_cast<const uint4*>(p) + lane;
        if constexpr (ONCE) return load_once(x);
        else return *x;
    };
    auto load_keys = [&]() {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) k[i] = load16(from + i * 1024);
        if constexpr (ES == 1) {
            const float4* const scales = reinterpret_cast<const float4*>(from + 2 * HALF) + 2 * j;
            const float4 x = scales[0], y = scales[1];
            ks[0] = x.x; ks[1] = x.y; ks[2] = x.z; ks[3] = x.w; ks[4] = y.x; ks[5] = y.y; ks[6] = y.z; ks[7] = y.w;
        }
    };
    auto load_values = [&]() {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) v[i] = load16(from + HALF + i * 1024);
        if constexpr (ES == 1) {
            const float4* const scales = reinterpret_cast<const float4*>(from + 2 * HALF + 4 * KV_BLOCK) + 2 * j;
            const float4 x = scales[0], y = scales[1];
            vs[0] = x.x; vs[1] = x.y; vs[2] = x.z; vs[3] = x.w; vs[4] = y.x; vs[5] = y.y; vs[6] = y.z; vs[7] = y.w;
        }
    };
    if (blocks > 0) {
        go_to(0);
        load_keys();
        load_values();
    }
    // as operands
    frag q[SHARED ? 1 : QP][SHARED ? 1 : NS];
    float back = a.scale, up = 1.0f;                 // of a score; half: what it is multiplied by first, so that 0 times an infinite product never comes up
    {
        float f[OWN][8];
#pragma unroll
        for (int u = 0; u < OWN; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[u][e] = __uint_as_float(QP == 2 ? raw[u][e * (QP - 1)] : e & 1 ? raw[u][e >> 1] & 0xFFFF0000u : raw[u][e >> 1] << 16);
        if constexpr (DT == SS_FP16) {
            // half has 5 bits of exponent: a head's largest value is brought to 2^13 .. 2^14 by a power of two, which its scores get back; the smallest then keep their bits
            float most = 0.0f;
#pragma unroll
            for (int u = 0; u < OWN; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(f[u][e]));
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            if constexpr (SHARED) {
                if (j == 0) wave_sums[wave][r].x = most;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < KA_WAVES; ++w) most = fmaxf(most, wave_sums[w][r].x);
            }
            const int x = most > 0.0f && most < INFINITY ? max((int)(__float_as_uint(most) >> 23) - 140, -126) : 0;      // most < 2^(x + 14)
            const float down = __uint_as_float((uint32_t)(127 - x) << 23);
#pragma unroll
            for (int u = 0; u < OWN; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) f[u][e] *= down;
            (x > 0 ? up : back) *= __uint_as_float((uint32_t)(127 + x) << 23);
        }
#pragma unroll
        for (int u = 0; u < OWN; ++u)
#pragma unroll
            for (int p = 0; p < QP; ++p) {
                v4i w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t both = p + 1 < QP ? ka_pack_below(f[u][2 * e], f[u][2 * e + 1], Ka<DT>()) : ka_pack(f[u][2 * e], f[u][2 * e + 1], Ka<DT>());
                    w[e] = (int)both;
                    if (p + 1 < QP) ka_leave<DT, false>(f[u][2 * e], f[u][2 * e + 1], both);
                }
                if constexpr (!SHARED) q[p][u] = __builtin_bit_cast(frag, w);
                else if (own(u) < NS) shared_q[p][own(u)][lane] = w;
            }
        if constexpr (SHARED) __syncthreads();
    }
    int at_query = lane;
    auto query = [&](int p, int s) -> frag {
        if constexpr (SHARED) return __builtin_bit_cast(frag, shared_q[p][s][at_query]);
        else return q[p][s];
    };

    // The probabilities of half are taken 2^14 times as large, so that the smallest ones keep their bits: all of them, the sum too.
    constexpr float LIFT = DT == SS_FP16 ? 14.0f : 0.0f;
    float top = -INFINITY, sum = 0.0f;               // of head r: its maximum in all j, the sum of this j's tokens
    v4f o[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) o[n] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int step = 0; step < blocks; ++step) {
        const int block = first + step * KA_WAVES;
        valid = next_valid;
        if constexpr (SHARED) asm volatile("" : "+v"(at_query));      // read anew for every block, not kept in registers
        // scores of tokens 8 j + 4 t + i
        v4f s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                frag f;
                if constexpr (ES == 2) f = __builtin_bit_cast(frag, k[2 * i + t]);
                else f = t ? ka_widen<DT>(k[i].z, k[i].w) : ka_widen<DT>(k[i].x, k[i].y);
#pragma unroll
                for (int p = 0; p < QP; ++p) s[t] = Ka<DT>::mma(f, query(p, i), s[t]);
            }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (DT == SS_FP16 ? s[e >> 2][e & 3] * up : s[e >> 2][e & 3]) * (ES == 1 ? back * ks[e] : back);
        if (step + 1 < blocks) {
            go_to(step + 1);
            load_keys();
        }
        const int at = block * KV_BLOCK + 8 * j;
        const bool whole = valid && block * KV_BLOCK >= span.from && block * KV_BLOCK + KV_BLOCK <= span.len;
        uint32_t seen = 0xFF;
        if (!whole) {                                // what nobody wrote may be anything, a NaN too
            seen = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool there = valid && at + e >= span.from && at + e < span.len;
                seen |= there ? 1u << e : 0u;
                x[e] = there ? x[e] : -INFINITY;
            }
        }
        float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        const float top_now = fmaxf(top, most), base = top_now == -INFINITY ? 0.0f : top_now - LIFT, less = top == top_now ? 1.0f : __builtin_amdgcn_exp2f(top - top_now);
        top = top_now;
        float y[8], add = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { y[e] = __builtin_amdgcn_exp2f(x[e] - base); add += y[e]; }
        sum = sum * less + add;
        if constexpr (ES == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = seen >> e & 1 ? y[e] * vs[e] : 0.0f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n] *= less;
        // The probabilities as operands, in two pieces: bf16 alone would cost as much again as the rounding of the result, and half alone an eighth of that.  The second
        // product costs no time in any type (64 requests up to 16384 tokens in half 196 .. 198 us with one and with two); a third would (fp8, 64 channels, 60.9 -> 63.0;
        // bf16 under queries of 32 bits 188 -> 198), and the distance to the exact results stays that of their rounding.  Codes of 8 bits are no infinities: the nearest first
        // piece leaves less.
        constexpr int PP = 2;
        frag p[PP];
#pragma unroll
        for (int i = 0; i < PP; ++i) {
            v4i w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = (int)(ES == 2 && i + 1 < PP ? ka_pack_below(y[2 * e], y[2 * e + 1], Ka<DT>()) : ka_pack(y[2 * e], y[2 * e + 1], Ka<DT>()));
                if (i + 1 < PP) ka_leave<DT, true>(y[2 * e], y[2 * e + 1], (uint32_t)w[e]);
            }
            p[i] = __builtin_bit_cast(frag, w);
        }
        if (!whole) {                                // 0 times a NaN is none
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if constexpr (ES == 2) w[c] &= (seen >> (2 * c) & 1 ? 0xFFFFu : 0u) | (seen >> (2 * c + 1) & 1 ? 0xFFFF0000u : 0u);
                    else {
                        uint32_t m = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) m |= seen >> (4 * (c & 1) + e) & 1 ? 0xFFu << (8 * e) : 0u;
                        w[c] &= m;
                    }
                }
                v[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            frag f;
            if constexpr (ES == 2) f = __builtin_bit_cast(frag, v[n]);
            else f = n & 1 ? ka_widen<DT>(v[n >> 1].z, v[n >> 1].w) : ka_widen<DT>(v[n >> 1].x, v[n >> 1].y);
#pragma unroll
            for (int i = 0; i < PP; ++i) o[n] = Ka<DT>::mma(f, p[i], o[n]);
        }
        if (step + 1 < blocks) load_values();
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);

    // the wavefronts' shares: lane (r, j) holds values 16 n + 4 j + i of head r in o[n][i]
    if (j == 0) wave_sums[wave][r] = make_float2(top, sum);
    __syncthreads();
    float all_top = -INFINITY, all_sum = 0.0f, weight[KA_WAVES];
#pragma unroll
    for (int w = 0; w < KA_WAVES; ++w) all_top = fmaxf(all_top, wave_sums[w][r].x);
#pragma unroll
    for (int w = 0; w < KA_WAVES; ++w) {
        const float2 s = wave_sums[w][r];
        weight[w] = s.x == all_top ? 1.0f : __builtin_amdgcn_exp2f(s.x - all_top);      // both may be minus infinity
        all_sum += s.y * weight[w];
    }
    const int64_t row_at = ((int64_t)place * a.H * a.tiles + unit) * KA_COLUMNS + r;
    if (parts > 1 && wave == 0 && j == 0 && there) a.sums[row_at] = make_float2(all_top, all_sum);
    const bool none = all_sum == 0.0f;               // nothing seen, or scores of minus infinity alone: zeros, though 0 times a value may be no number
    const float inverse = parts > 1 || none ? 1.0f : 1.0f / all_sum;
#pragma unroll
    for (int n0 = 0; n0 < NT; n0 += CHUNK) {
        if (n0 > 0) __syncthreads();
#pragma unroll
        for (int n = 0; n < CHUNK; ++n)
            if (n0 + n < NT) joined[wave][n][lane] = make_float4(o[n0 + n][0], o[n0 + n][1], o[n0 + n][2], o[n0 + n][3]);
        __syncthreads();
        for (int n = wave; n < CHUNK && n0 + n < NT; n += KA_WAVES) {
            v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < KA_WAVES; ++w) {
                const float4 x = joined[w][n][lane];
                v += v4f{x.x, x.y, x.z, x.w} * weight[w];
            }
            const int d = 16 * (n0 + n) + 4 * j;
            if (!there) continue;
            if (parts > 1) *reinterpret_cast<float4*>(a.parts + row_at * (32 * NS) + d) = make_float4(v[0], v[1], v[2], v[3]);
            else if (d < a.D) {
                uint16_t* const to = a.out + b * a.ldo + (int64_t)(h * a.G + column) * a.ho + d;
                const uint32_t w0 = none ? 0 : pack_bf16x2(v[0] * inverse, v[1] * inverse), w1 = none ? 0 : pack_bf16x2(v[2] * inverse, v[3] * inverse);
                if (d + 4 <= a.D) *reinterpret_cast<ka8_t*>(to) = ka8_t{w0, w1};
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (d + i < a.D) to[i] = (uint16_t)((i & 2 ? w1 : w0) >> (16 * (i & 1)));
                }
            }
        }
    }
}

// Joins the parts of a request that was divided: a workgroup for each query head of each request, or for each 32 values of it, which leaves where it was not.  SLICE:
// steps of 32 values of a workgroup, whose rows are 8 lanes wide each.  Bound by the launch and three waits, plan, parts and sums, results: 4.0 .. 4.7 us in a trace
// where nothing is left to join too.  All rows are asked for before their weights are known; one after the other 256 parts of a head took 18 us.  Slices of 32 values
// for few heads of many parts: 512 parts of 16 heads of 256 6 us for 15 by whole rows.
constexpr int KJ_EACH = 8;                           // rows that a thread asks for ahead of their weights
template <int NS, int SLICE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_join(const KaArgs a)
{
    constexpr int WIDTH = 32 * NS, LANES = 8 * SLICE, ROWS = THREADS / LANES, ROUND = ROWS * KJ_EACH;
    __shared__ float4 acc[ROWS][LANES];
    __shared__ float2 sums[ROUND];
    __shared__ float row_sums[ROWS], tops[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slice = blockIdx.x % (NS / SLICE), index = blockIdx.x / (NS / SLICE), heads = a.H * a.G, b = index / heads;
    const int2 plan = a.plan[b];
    const int parts = plan.y;
    if (parts < 2 || plan.x < 0 || parts > a.places - plan.x) return;      // (the last two only if lengths are changed while they are read)
    const int head = index - b * heads, h = head / a.G, column = head - h * a.G;
    const int64_t step = (int64_t)a.H * a.tiles * KA_COLUMNS, first = plan.x * step + (h * a.tiles + column / KA_COLUMNS) * KA_COLUMNS + column % KA_COLUMNS;
    const int at_row = threadIdx.x / LANES, at = threadIdx.x - at_row * LANES, column0 = slice * 32 * SLICE;      // its first value
    float top = -INFINITY, sum = 0.0f;
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = 0; i0 < parts; i0 += ROUND) {      // mostly once
        float4 p[KJ_EACH];
#pragma unroll
        for (int i = 0; i < KJ_EACH; ++i) {
            const int q = i0 + at_row + i * ROWS;
            p[i] = at_row < ROWS && q < parts ? reinterpret_cast<const float4*>(a.parts + (first + q * step) * WIDTH + column0)[at] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        float most = -INFINITY;
        if (i0 > 0) __syncthreads();
        for (int i = threadIdx.x; i < ROUND; i += THREADS) {
            const float2 s = i0 + i < parts ? a.sums[first + (i0 + i) * step] : make_float2(-INFINITY, 0.0f);
            sums[i] = s;
            most = fmaxf(most, s.x);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        if (lane == 0) tops[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) most = fmaxf(most, tops[w]);
        most = fmaxf(most, top);
        const float less = top == most ? 1.0f : __builtin_amdgcn_exp2f(top - most);
        top = most;
        v *= less;
        sum *= less;
#pragma unroll
        for (int i = 0; i < KJ_EACH; ++i) {
            const float2 s = sums[min(at_row, ROWS - 1) + i * ROWS];
            const float weight = s.x == top ? 1.0f : __builtin_amdgcn_exp2f(s.x - top);
            sum += s.y * weight;
            v += v4f{p[i].x, p[i].y, p[i].z, p[i].w} * weight;
        }
    }
    if (at_row < ROWS) {
        acc[at_row][at] = make_float4(v[0], v[1], v[2], v[3]);
        if (at == 0) row_sums[at_row] = sum;
    }
    __syncthreads();
    sum = row_sums[0];
#pragma unroll
    for (int r = 1; r < ROWS; ++r) sum += row_sums[r];
    const bool none = sum == 0.0f;                   // as above
    const float inverse = none ? 1.0f : 1.0f / sum;
    const float* const rows = reinterpret_cast<const float*>(acc);
    for (int d = threadIdx.x; d < 32 * SLICE && column0 + d < a.D; d += THREADS) {
        float x = 0.0f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) x += rows[r * 32 * SLICE + d];
        a.out[b * a.ldo + head * a.ho + column0 + d] = none ? 0 : (uint16_t)pack_bf16x2(x * inverse, 0.0f);
    }
}

template <int DT, int NS> static ss_status launch_attend(const KaArgs& a, bool fp32, bool join, int64_t groups, int64_t rows, hipStream_t hs)
{
    auto attend = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(64 * KA_WAVES), 0, hs, a); };
    if (a.tiles == 1) fp32 ? attend(k_kv_attend<DT, NS, 2, true>) : attend(k_kv_attend<DT, NS, 1, true>);
    else fp32 ? attend(k_kv_attend<DT, NS, 2, false>) : attend(k_kv_attend<DT, NS, 1, false>);
    if (!join) return launch_status();
    if (launch_status() != SS_OK) return SS_ERR_HIP;
    if (rows * NS <= cu_count()) hipLaunchKernelGGL((k_kv_join<NS, 1, 512>), dim3((uint32_t)(rows * NS)), dim3(512), 0, hs, a);
    else if (rows <= 2 * cu_count()) hipLaunchKernelGGL((k_kv_join<NS, NS, 512>), dim3((uint32_t)rows), dim3(512), 0, hs, a);
    else hipLaunchKernelGGL((k_kv_join<NS, NS, 128>), dim3((uint32_t)rows), dim3(128), 0, hs, a);
    return launch_status();
}

// Workgroups that all heads' parts come to, about.  256 channels, where two of a compute unit run at once, 3 | 2 for each: 22 requests of 7079 tokens, 8 heads, 234 |
// 261 us; 14 of 20177, 4 heads, int8 116 | 123.  128 channels: one request of 131072 tokens 50.9 | 48.9, 64 up to 16384 174 | 170.
static int64_t wanted_groups(int64_t D) { return (kv_steps(D) == 8 ? 3 : 2) * (int64_t)cu_count(); }
// Blocks of a row of the table up to which requests are not divided, by the workgroups that they are without.  A division costs the second launch, 4 us; what it saves
// is that a compute unit draws some 60 GB/s at most.  Not divided | divided, us a pass:
//   up to 1 for each compute unit   1 x 512 (8 heads of 128) 7.3, 1 x 576 | 10;   8 x 500 9.1, 8 x 576 | 13.1;   1 x 1024 12.3 | 11.9;   1 x 1536 16.9 | 11.9;   8 x 2048 24.8 | 18.3
//   up to 4                         40 x 1024 33.0 | 34.6;   64 x 1024 44 .. 47 | 49;   64 x 2048 82.8 | 85.5, lengths up to 2048 34.6 | 31.1;   40 x 2048 62.7 | 59.3
//   more                            200 x up to 1024 52.3 | 57.1;   256 x up to 2048 (4 heads) 64.8 | 68.1;   256 x up to 4096 120 | 112
static int64_t undivided_blocks(int64_t groups) { return groups <= cu_count() ? 16 : groups <= 4 * cu_count() ? 32 : 64; }
// bytes of a part of a request: sums and values of all heads
static int64_t part_bytes(int64_t units, int64_t D) { return units * KA_COLUMNS * (8 + 4 * 32 * kv_steps(D)); }
// Parts of requests that are in several, for so many workgroups: such a request has more blocks than one of these takes, so that there are no more such requests than
// workgroups, and one part each beyond what the blocks come to.  The rest covers the roundings of a share.
static int64_t places_for(int64_t wanted, int64_t B) { return wanted + (B < wanted ? B : wanted) + 2; }
// and of the plan that lies before them
static int64_t plan_bytes(int64_t B) { return (8 * B + 15) & ~(int64_t)15; }

}  // namespace ss

using namespace ss;

static bool valid_attention(int64_t B, int64_t Hq, int64_t H, int64_t D)
{
    return B >= 0 && B <= KV_MAX_REQUESTS && H >= 1 && H <= KV_MAX_HEADS && Hq >= H && Hq <= KV_MAX_HEADS && Hq % H == 0 && D >= 1 && D <= KV_MAX_D;
}

extern "C" size_t kv_attention_workspace_bytes(int64_t B, int64_t Hq, int64_t H, int64_t D)
{
    if (!valid_attention(B, Hq, H, D) || B == 0) return 0;
    const int64_t units = H * ((Hq / H + KA_COLUMNS - 1) / KA_COLUMNS);
    const int64_t wanted = wanted_groups(D) / units;
    return wanted > 1 ? (size_t)(plan_bytes(B) + places_for(wanted, B) * part_bytes(units, D)) : 0;
}

extern "C" ss_status kv_attention(const void* Q, ss_act_dtype in_dtype, int64_t ldq, int64_t hq, const void* pages, int64_t P, int64_t page, ss_dtype dtype, const int32_t* table,
                                  int64_t ldt, int64_t W, const int32_t* lens, int64_t B, int64_t Hq, int64_t H, int64_t D, float scale, int64_t window, void* out, int64_t ldo,
                                  int64_t ho, void* workspace, size_t workspace_bytes, void* stream)
{
    if ((in_dtype != SS_IN_F32 && in_dtype != SS_IN_BF16) || !valid_dtype(dtype)) return SS_ERR_DTYPE;
    constexpr int64_t FAR = (int64_t)1 << 40;
    const float scale2 = scale * 1.44269504088896340736f;      // of scores to the base 2
    if (!valid_attention(B, Hq, H, D) || !kv_valid_page(H, page, D, dtype) || !kv_valid_slots(P, page) || W < 1 || W > INT32_MAX / page - 1 || ldt < W || window < 0 || !(scale2 - scale2 == 0.0f) ||
        ldq < 0 || ldq > FAR || hq < 0 || hq > FAR || ldo < 0 || ldo > FAR || ho < 0 || ho > FAR || ldt > FAR)
        return SS_ERR_SHAPE;
    if (B == 0) return SS_OK;
    if (!Q || !pages || !table || !lens || !out || (!workspace && workspace_bytes > 0)) return SS_ERR_NULL;
    if (!kv_rows_apart(B, ldo, Hq, ho, D)) return SS_ERR_SHAPE;
    if (((uintptr_t)Q & (in_dtype == SS_IN_F32 ? 3 : 1)) || ((uintptr_t)out & 1) || (((uintptr_t)table | (uintptr_t)lens) & 3) || ((uintptr_t)pages & 15)) return SS_ERR_SHAPE;
    if ((uintptr_t)workspace & 15) return SS_ERR_WORKSPACE;
    const int ns = kv_steps(D);
    KaArgs a = {};
    a.q = Q; a.ldq = ldq; a.hq = hq;
    a.pages = static_cast<const uint8_t*>(pages);
    a.page_bytes = kv_bytes_of_page(H, page, D, dtype);
    a.table = table; a.ldt = ldt;
    a.H = (int)H; a.G = (int)(Hq / H); a.tiles = (a.G + KA_COLUMNS - 1) / KA_COLUMNS; a.D = (int)D; a.page = (int)page; a.P = (int)P;
    a.scale = scale2;
    a.out = static_cast<uint16_t*>(out); a.ldo = ldo; a.ho = ho;
    const int64_t units = H * a.tiles;
    // Parts of all requests together: sum of blocks / per + one for each request.  None where no request can be long enough, or the workspace has no room.
    const int64_t bytes = (int64_t)(workspace_bytes < (size_t)1 << 50 ? workspace_bytes : (size_t)1 << 50) - plan_bytes(B);
    const int64_t places = bytes / part_bytes(units, D) - 2, room = places - B > places / 2 ? places - B : places / 2, want = wanted_groups(D) / units, wanted = room < want ? room : want;
    const bool join = wanted > 1 && W * page > undivided_blocks(B * units) * KV_BLOCK;
    a.division = {lens, (int)B, (int)(W * page), (int)(window < INT32_MAX ? window : 0), join ? 1.0f / (float)wanted : 0.0f};
    a.items = (int)(join ? wanted + 2 + B : B);
    a.places = (int)(join ? places_for(wanted, B) : 0);
    a.plan = join ? static_cast<int2*>(workspace) : nullptr;
    a.sums = join ? reinterpret_cast<float2*>(static_cast<char*>(workspace) + plan_bytes(B)) : nullptr;
    a.parts = join ? reinterpret_cast<float*>(a.sums + a.places * units * KA_COLUMNS) : nullptr;
    a.by_heads = make_div(H);
    a.by_round = make_div(8 * a.tiles);
    a.by_blocks = make_div(page / KV_BLOCK);
    const int64_t heads = a.items * H, groups = a.tiles == 1 ? heads : (heads + 7) / 8 * 8 * a.tiles, rows = B * Hq;
    if (!mx4_grid_fits(groups, 64 * KA_WAVES) || !mx4_grid_fits(rows, 128)) return SS_ERR_SHAPE;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const bool fp32 = in_dtype == SS_IN_F32;
#define SS_KA(DT)                                                                     \
    switch (ns) {                                                                     \
    case 1: return launch_attend<DT, 1>(a, fp32, join, groups, rows, hs);             \
    case 2: return launch_attend<DT, 2>(a, fp32, join, groups, rows, hs);             \
    case 3: return launch_attend<DT, 3>(a, fp32, join, groups, rows, hs);             \
    case 4: return launch_attend<DT, 4>(a, fp32, join, groups, rows, hs);             \
    case 6: return launch_attend<DT, 6>(a, fp32, join, groups, rows, hs);             \
    default: return launch_attend<DT, 8>(a, fp32, join, groups, rows, hs);            \
    }
    switch (dtype) {
    case SS_I8: SS_KA(SS_I8)
    case SS_FP8_E4M3: SS_KA(SS_FP8_E4M3)
    case SS_BF16: SS_KA(SS_BF16)
    default: SS_KA(SS_FP16)
    }
#undef SS_KA
}
