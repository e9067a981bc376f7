// Attention of drafted trees over the paged cache.
//
// Every node of a tree sees the sequence's prefix and its own ancestors, so all nodes of a sequence share the scan of the
// prefix: row (node, head of the group) is a column of S^T = K Q^T, and a workgroup reads K and V once for all its rows.
//   - Four waves: WR of them side by side over the rows (a wave holds NT blocks of 32 columns), WK = 4 / WR of them taking turns
//     along the keys.  Up to 32 rows: WR = 1, each wave scans its own keys; 256 rows: WR = 4, NT = 2.
//   - Keys come in steps of 32 (two pages) per wave, copied into a ring of LDS slots by the memory system, in the order in which
//     the matrix instructions take them: a wave's operand read is always 1 KB in lane order (no bank conflicts), and copies in
//     flight take no registers.  The WR waves of a key group share the copy.
//   - Both products run on the 32x32x16 instruction.  Row rho of S^T stands for token swap23(rho % 16) of page rho / 16, so that
//     the accumulator registers of lane (h, n) are tokens 8h .. 8h + 7 of the first page, then of the second, for column n:
//     packed to bf16 they are the B operands of O^T += V^T P^T as they stand, and the matching A operand is 16 bytes (e4m3: 8)
//     of a V row.  fp32: the same with the 32x32x2 instruction, one dim of a K piece or one token of a V piece per step.
//   - The masks are looked at on the pages that hold nodes only.
// The running maximum is a reference in log2 units that is raised when a score exceeds it by more than 16.
#include <type_traits>

#include "ts_device.h"
#include "ts_launch.h"

namespace ts {

constexpr int kTrWaves = 4;
constexpr float kRaiseTr = 16.0f;
// Reference maximum of a column that has seen no key: finite, so that differences stay defined.
constexpr float kNoKeyTr = -3.402823466e38f;

// LDS image of 32 keys (two pages), in blocks of 64 pieces of 16 bytes:
//   K block j: piece (h, n) = 16-byte chunk 2j + h of token swap23(n % 16) of page n / 16
//   V, bf16: block (page p, dims 32 d ..): piece (h, n) = tokens 8h .. 8h + 7 of dim 32 d + n;  e4m3: block d: piece (p, n) = the
//   16 tokens of dim 32 d + n of page p;  fp32: block (p, d, i): piece (h, n) = tokens 8h + 4i .. + 3
template <typename KT, int D> struct TrStep {
    static constexpr int ES = (int)sizeof(KT), PB = 16 * D * ES;       // bytes of an element, of a tile
    static constexpr int NK = D * ES / 32, NV = NK, NB = NK + NV;      // blocks
    static constexpr int kBytes = NB * 1024;
};
__device__ __forceinline__ int tr_swap23(int s) { return (s & 3) | ((s & 4) << 1) | ((s & 8) >> 1); }

__device__ __forceinline__ uint32_t tr_lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
// 64 x 16 bytes straight into LDS, lane l's at lds + 16 l; counted by vmcnt.
__device__ __forceinline__ void tr_copy(uint32_t lds, const char* p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n" :: "s"(lds), "v"(p) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void tr_wait_copies()
{
    static_assert(N >= 0 && N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14));    // vmcnt(N); expcnt and lgkmcnt untouched
}

// The blocks wr, wr + WR, ... of two pages on their way into LDS.
template <int WR, typename KT, int D>
__device__ __forceinline__ void tr_copy_step(uint32_t lds, const char* kc, const char* vc, int64_t tile0, int64_t tile1, int wr, int lane)
{
    using S = TrStep<KT, D>;
    const int n = lane & 31, h = lane >> 5;
    const char* k = kc + (n >= 16 ? tile1 : tile0) * S::PB + h * 256 + tr_swap23(n & 15) * 16;
#pragma unroll
    for (int i = 0; i < S::NB / WR; ++i) {
        const int b = wr + WR * i;
        const char* p;
        if (b < S::NK) p = k + b * 512;
        else {
            const int v = b - S::NK;
            if constexpr (S::ES == 1) p = vc + (h ? tile1 : tile0) * S::PB + (32 * v + n) * 16;
            else {
                constexpr int PER = S::NV / 2;                         // blocks of a page
                const int in = v % PER;
                const int d = S::ES == 2 ? in : in / 2, i16 = S::ES == 2 ? 0 : in % 2;
                p = vc + (v >= PER ? tile1 : tile0) * S::PB + (32 * d + n) * (16 * S::ES) + h * (8 * S::ES) + i16 * 16;
            }
        }
        tr_copy(lds + b * 1024, p);
    }
}

__device__ __forceinline__ uint2 tr_widen(uint32_t w)          // four e4m3 -> four bf16 (exact)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
}

// Q^T operand of one column, the dims in the order of the K pieces.
template <typename KT, int D> struct TrQ {
    using T = std::conditional_t<sizeof(KT) == 4, f32x4, bf16x8>;
    static constexpr int N = sizeof(KT) == 4 ? D / 8 : D / 16;
    T q[N];
};
template <typename KT, int D>
__device__ __forceinline__ void tr_load_q(TrQ<KT, D>& t, const void* q, int64_t at, int h, bool negate)
{
#pragma unroll
    for (int b = 0; b < TrQ<KT, D>::N; ++b) {
        if constexpr (sizeof(KT) == 4) {
            t.q[b] = *(const f32x4*)((const float*)q + at + 4 * (2 * b + h));
            if (negate) t.q[b] = -t.q[b];
        } else {
            const int d0 = sizeof(KT) == 2 ? 8 * (2 * b + h) : 16 * (2 * (b >> 1) + h) + 8 * (b & 1);
            uint4 x = *(const uint4*)((const uint16_t*)q + at + d0);
            if (negate) x = make_uint4(x.x ^ 0x80008000u, x.y ^ 0x80008000u, x.z ^ 0x80008000u, x.w ^ 0x80008000u);
            t.q[b] = __builtin_bit_cast(bf16x8, x);
        }
    }
}

// S^T of 32 keys for NT blocks of 32 columns.
template <int NT, typename KT, int D>
__device__ __forceinline__ void tr_scores(f32x16 (&s)[NT], const unsigned char* lk, const TrQ<KT, D> (&q)[NT], int lane)
{
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
    for (int b = 0; b < TrStep<KT, D>::NK; ++b) {
        const uint4 k = *(const uint4*)(lk + b * 1024 + lane * 16);
        if constexpr (sizeof(KT) == 4) {
            const f32x4 kf = __builtin_bit_cast(f32x4, k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q[t].q[b][e], s[t], 0, 0, 0);
        } else if constexpr (sizeof(KT) == 2) {
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), q[t].q[b], s[t], 0, 0, 0);
        } else {
            const uint2 a0 = tr_widen(k.x), a1 = tr_widen(k.y), a2 = tr_widen(k.z), a3 = tr_widen(k.w);
            const bf16x8 lo = __builtin_bit_cast(bf16x8, make_uint4(a0.x, a0.y, a1.x, a1.y)), hi = __builtin_bit_cast(bf16x8, make_uint4(a2.x, a2.y, a3.x, a3.y));
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, q[t].q[2 * b], s[t], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, q[t].q[2 * b + 1], s[t], 0, 0, 0);
        }
    }
}

// A lane's eight tokens (8h ..) of dim 32 d + n of page p, as they lie in LDS: VW words.
template <typename KT, int D> struct TrV { static constexpr int VW = 2 * (int)sizeof(KT); uint32_t w[VW]; };
template <typename KT, int D>
__device__ __forceinline__ TrV<KT, D> tr_load_v(const unsigned char* lv, int p, int d, int lane)
{
    TrV<KT, D> v;
    constexpr int DB = D / 32;
    if constexpr (sizeof(KT) == 1) {
        const uint2 x = *(const uint2*)(lv + d * 1024 + (p * 32 + (lane & 31)) * 16 + (lane >> 5) * 8);
        v.w[0] = x.x; v.w[1] = x.y;
    } else {
        constexpr int I = (int)sizeof(KT) / 2;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const uint4 x = *(const uint4*)(lv + ((p * DB + d) * I + i) * 1024 + lane * 16);
            v.w[4 * i] = x.x; v.w[4 * i + 1] = x.y; v.w[4 * i + 2] = x.z; v.w[4 * i + 3] = x.w;
        }
    }
    return v;
}
template <typename KT, int D>
__device__ __forceinline__ float tr_element(const TrV<KT, D>& v, int e)
{
    if constexpr (sizeof(KT) == 4) return __uint_as_float(v.w[e]);
    else if constexpr (sizeof(KT) == 2) return bf16_bits_to_float(v.w[e / 2] >> (16 * (e & 1)) & 0xffffu);
    else return (v.w[e / 4] >> (8 * (e & 3)) & 0x7fu) == 0x7fu ? __builtin_nanf("") : 0.0f;    // (asked whether it is finite)
}
// Clears what does not exist (tokens from `have` on) and what is not finite; true if there was any of the latter.
template <typename KT, int D>
__device__ __forceinline__ bool tr_clean_v(TrV<KT, D>& v, int have)
{
    constexpr int ES = (int)sizeof(KT), PER = 4 / ES;
    constexpr uint32_t kField = ES == 4 ? 0xffffffffu : (1u << (8 * ES % 32)) - 1, kOdd = ES == 4 ? 0x7f800000u : (ES == 2 ? 0x7f80u : 0x7fu);
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int sh = 8 * ES * (e % PER);
        const bool bad = (v.w[e / PER] >> sh & kOdd) == kOdd;
        if (e >= have || bad) v.w[e / PER] &= ~(kField << sh);
        odd |= bad && e < have;
    }
    return odd;
}

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2)); }

// The keys from node number j0 on (j0 a multiple of 8 below node 0 or anything; negative: the prefix, which everybody sees) that
// a node sees, as bits 0 .. 7; nodes from n_nodes on do not exist.  Without a mask a node sees those up to itself.
// There is no divergent branch here or anywhere else in the steps: the compiler was seen to save a register before the lanes of such
// a branch are back together, so that the others' values (addresses of the next copies) were lost.
__device__ __forceinline__ uint32_t tr_visible(const uint64_t* mask, int words, int n_nodes, int node, int j0)
{
    const int w = j0 >> 6, sh = j0 & 63;                       // (rounded down)
    uint64_t lo = ~0ull, hi = ~0ull;
    if (mask) {                                                // the same for the whole launch
        lo = mask[min(max(w, 0), words - 1)];
        hi = mask[min(max(w + 1, 0), words - 1)];
    }
    lo = w < 0 ? ~0ull : lo;
    hi = w + 1 < 0 ? ~0ull : hi;
    // (sh 0: the high word is shifted by 63 and then by 1, out of sight)
    const uint32_t bits = (uint32_t)(lo >> sh | hi << (63 - sh) << 1) & 0xffu;
    const int exist = (mask ? n_nodes : node + 1) - j0;        // of the eight, those below this count
    return bits & (exist >= 8 ? 0xffu : (1u << max(exist, 0)) - 1u);
}

__device__ __forceinline__ uint32_t tr_seen(const TreeArgs& a, int row0, int n_nodes, int node, int j0)
{
    return tr_visible(a.mask ? a.mask + (int64_t)(row0 + node) * a.mask_words : nullptr, a.mask_words, n_nodes, node, j0);
}

// What a workgroup does, from the launch's list.
struct TrItem { int seq, node_rows, n_nodes, row0, prefix, g, group, part, parts, part_row0; };
__device__ __forceinline__ TrItem tr_item(const TreeArgs& a, const TreeSeqs& s)
{
    const int lane = threadIdx.x & 63, w = blockIdx.x;
    int i = -1;
#pragma unroll
    for (int b = 0; b < kTreeSeqs; b += 64)
        i += __builtin_popcountll(__ballot((b + lane < s.n) & (s.seq[b + lane].first_item <= w)));
    const TreeSeq q = s.seq[i];
    TrItem t;
    t.seq = i; t.row0 = q.row0; t.n_nodes = s.seq[i + 1].row0 - q.row0; t.prefix = q.prefix; t.parts = q.parts; t.part_row0 = q.part_row0;
    t.node_rows = t.n_nodes * a.geo.G;
    // The groups of rows of one scan (KV head, range of pages) read the same pages: they go to the same die, one after the
    // other (workgroup i runs on die i % 8).
    const int groups = (t.node_rows + a.rows - 1) / a.rows, scans = a.geo.Hkv * q.parts, k = w - q.first_item;
    int scan;
    if (groups > 1 && scans % 8 == 0) { t.group = k / 8 % groups; scan = k / (8 * groups) * 8 + k % 8; }
    else { t.group = k % groups; scan = k / groups; }
    t.g = scan % a.geo.Hkv;
    t.part = scan / a.geo.Hkv;
    return t;
}

template <typename KT>
__device__ __forceinline__ void tr_store_out(const TreeArgs& a, int64_t at, f32x4 v)
{
    if constexpr (sizeof(KT) == 4) *(f32x4*)((float*)a.out + at) = v;
    else *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

// One over the weights' sum.  A sum of zero: the row sees nothing (its output is zeros), or only scores of -inf (NaN, 0 / 0).
__device__ __forceinline__ float tr_inverse(const TreeArgs& a, float l, int prefix, int n_nodes, int row0, int node)
{
    float inv = 1.0f / l;
    if (__any(l == 0.0f)) {
        uint32_t any = prefix > 0 ? 1u : 0u;
        for (int j = 0; j < n_nodes; j += 8) any |= tr_seen(a, row0, n_nodes, node, j);
        inv = l != 0.0f ? inv : (any ? __builtin_nanf("") : 0.0f);
    }
    return inv;
}

// LDS slots of the ring: two workgroups per CU where at least two slots fit (80 of 160 KB), four at the most.
template <typename KT, int D, int WR> constexpr int tr_ring()
{
    constexpr int slot = TrStep<KT, D>::kBytes * (kTrWaves / WR), fit = 80 * 1024 / slot;
    return fit < 2 ? 2 : (fit > 4 ? 4 : fit);
}

template <typename KT, int D, int WR, int NT>
__global__ __launch_bounds__(64 * kTrWaves, NT == 1 ? 2 : 1) void tree_kernel(TreeArgs a, TreeSeqs s)
{
    using S = TrStep<KT, D>;
    constexpr int WK = kTrWaves / WR, DB = D / 32, ROWS = 32 * WR * NT, R = tr_ring<KT, D, WR>(), C = S::NB / WR;
    static_assert(S::NB % WR == 0 && C * (R - 2) < 64, "copies per wave");
    __shared__ __align__(16) unsigned char ring[R][WK][S::kBytes];
    static_assert(sizeof ring >= (size_t)(kTrWaves - WR) * (NT * DB * 4096 + NT * 256), "the ring holds the waves' states at the end");
    const TrItem it = tr_item(a, s);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, n = lane & 31;
    const int wr = wave % WR, kg = wave / WR;
    const int Hq = a.geo.Hq, Hkv = a.geo.Hkv, G = a.geo.G;
    const int ctx_len = it.prefix + it.n_nodes, pages = (ctx_len + kPage - 1) / kPage;
    const int page0 = it.part * a.part_pages, page1 = min(page0 + a.part_pages, pages);
    const int n_step = (page1 - page0 + 2 * WK - 1) / (2 * WK);
    const int first_row = it.group * ROWS + wr * (32 * NT);
    const bool works = first_row < it.node_rows;               // (a wave without rows only copies)

    const int32_t TS_CONSTANT* bt = as_constant(a.block_table) + (int64_t)it.seq * a.geo.max_pages;
    const char* kc = (const char*)a.k_cache;
    const char* vc = (const char*)a.v_cache;
    // (past the end of the range: its last page again, whose keys do not count a second time)
    auto page_of = [&](int i) { return page0 + 2 * (WK * i + kg); };
    auto tile_of = [&](int page) { return (int64_t)bt[min(page, page1 - 1)] * Hkv + it.g; };
    int64_t next0 = tile_of(page_of(0)), next1 = tile_of(page_of(0) + 1);
    auto issue = [&](int i) {
        tr_copy_step<WR, KT, D>(tr_lds_address(ring[i % R][kg]), kc, vc, next0, next1, wr, lane);
        next0 = tile_of(page_of(i + 1)); next1 = tile_of(page_of(i + 1) + 1);
    };
#pragma unroll
    for (int i = 0; i < R - 1; ++i)
        if (i < n_step) issue(i);

    // scores are wanted in log2 units: s * c; a negative c (e4m3 scale) is taken into Q, so that the maximum can be taken of s
    // (a scale of zero becomes a very small one: what is masked, -inf, keeps a weight of zero)
    const float c_signed = a.sm_scale * (sizeof(KT) == 1 ? a.k_scale[it.g] : 1.0f) * kLog2e;
    const float c = c_signed == 0.0f ? 1e-37f : __builtin_fabsf(c_signed);
    TrQ<KT, D> q[NT];
    int node[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = min(first_row + 32 * t + n, it.node_rows - 1);
        node[t] = row / G;
        tr_load_q(q[t], a.q, ((int64_t)(it.row0 + node[t]) * Hq + it.g * G + row % G) * D, h, c_signed < 0.0f);
    }
    f32x16 acc[NT][DB];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = kNoKeyTr; l[t] = 0.0f;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][b][i] = 0.0f;
    }

    auto step = [&](const unsigned char* lk, int page, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const unsigned char* lv = lk + S::NK * 1024;
        f32x16 x[NT];
        tr_scores<NT, KT, D>(x, lk, q, lane);
        [[maybe_unused]] uint32_t seen[NT];                    // bits 0 .. 7: tokens 8h .. of the first page, 8 .. 15: of the second
        if constexpr (MASKED) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int j0 = page * kPage + 8 * h - it.prefix;
                seen[t] = tr_seen(a, it.row0, it.n_nodes, node[t], j0) | tr_seen(a, it.row0, it.n_nodes, node[t], j0 + kPage) << 8;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = seen[t] >> i & 1 ? x[t][i] : -INFINITY;
            }
        }
        float top[NT];
        bool higher = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = fmaxf(x[t][i], x[t][i + 8]);
            top[t] = fmaxf(fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3])), fmaxf(fmaxf(u[4], u[5]), fmaxf(u[6], u[7]))) * c;
            higher |= top[t] > m[t] + kRaiseTr;
        }
        if (__any(higher)) {                                   // rare
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float m_new = fmaxf(m[t], pair32_max(top[t]));
                const float alpha = __builtin_amdgcn_exp2f(m[t] - m_new);
#pragma unroll
                for (int b = 0; b < DB; ++b) acc[t][b] *= alpha;
                l[t] *= alpha;
                m[t] = m_new;
            }
        }
        float p[NT][16];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][i], c, -m[t]));
            }
            float sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = (p[t][i] + p[t][i + 4]) + (p[t][i + 8] + p[t][i + 12]);
            l[t] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        [[maybe_unused]] bool odd = false;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            [[maybe_unused]] bf16x8 pb[NT];
            if constexpr (sizeof(KT) != 4) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    pb[t] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(p[t][8 * u], p[t][8 * u + 1]), pack_bf16(p[t][8 * u + 2], p[t][8 * u + 3]),
                                                                  pack_bf16(p[t][8 * u + 4], p[t][8 * u + 5]), pack_bf16(p[t][8 * u + 6], p[t][8 * u + 7])));
            }
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                TrV<KT, D> v = tr_load_v<KT, D>(lv, u, b, lane);
                // (masked) what does not exist does not enter the sums, and what is not finite enters below, in those rows that see it
                if constexpr (MASKED) odd |= tr_clean_v(v, ctx_len - (page + u) * kPage - 8 * h);
                if constexpr (sizeof(KT) == 4) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            acc[t][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v.w[e]), p[t][8 * u + e], acc[t][b], 0, 0, 0);
                } else {
                    uint4 w;
                    if constexpr (sizeof(KT) == 2) w = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
                    else {
                        const uint2 w0 = tr_widen(v.w[0]), w1 = tr_widen(v.w[1]);
                        w = make_uint4(w0.x, w0.y, w1.x, w1.y);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pb[t], acc[t][b], 0, 0, 0);
                }
            }
        }
        if constexpr (MASKED) {
            if (__any(odd)) {
                // How many values of +inf (or NaN) and of -inf (or NaN) a row sees of a dim: products of zeros and ones.
                for (int u = 0; u < 2; ++u) {                  // (not unrolled: rarely taken)
                    const int have = ctx_len - (page + u) * kPage - 8 * h;
                    uint4 on[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint32_t bits = seen[t] >> (8 * u);
                        auto two = [&](int e) { return (bits >> e & 1 ? 0x3f80u : 0u) | (bits >> (e + 1) & 1 ? 0x3f800000u : 0u); };
                        on[t] = make_uint4(two(0), two(2), two(4), two(6));
                    }
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        const TrV<KT, D> v = tr_load_v<KT, D>(lv, u, b, lane);
                        uint32_t plus[4] = {}, minus[4] = {};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = tr_element(v, e);
                            plus[e / 2] |= e < have && !(f < INFINITY) ? 0x3f80u << (16 * (e & 1)) : 0u;
                            minus[e / 2] |= e < have && !(f > -INFINITY) ? 0x3f80u << (16 * (e & 1)) : 0u;
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            f32x16 zero = {};
                            const f32x16 np = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(plus[0], plus[1], plus[2], plus[3])), __builtin_bit_cast(bf16x8, on[t]), zero, 0, 0, 0);
                            const f32x16 nm = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(minus[0], minus[1], minus[2], minus[3])), __builtin_bit_cast(bf16x8, on[t]), zero, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                if (np[r] > 0.0f) acc[t][b][r] += INFINITY;
                                if (nm[r] > 0.0f) acc[t][b][r] -= INFINITY;
                            }
                        }
                    }
                }
            }
        }
    };

    const int plain = it.prefix / kPage;                       // pages whose keys everybody sees
    auto round = [&](int i, auto masked) {
        // the copies of step i have landed (up to R - 2 later ones may be under way), and everybody is done with step i - 1
        const int later = min(R - 2, n_step - 1 - i);
        if (R > 3 && later == 2) tr_wait_copies<(R > 3 ? 2 * C : 0)>();
        else if (R > 2 && later == 1) tr_wait_copies<(R > 2 ? C : 0)>();
        else tr_wait_copies<0>();
        if constexpr (WR > 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + R - 1 < n_step) issue(i + R - 1);
        if (works) step(ring[i % R][kg], page_of(i), masked);
    };
    int i = 0;
    for (; page0 + 2 * WK * (i + 1) <= min(plain, page1); ++i) round(i, std::false_type{});
    for (; i < n_step; ++i) round(i, std::true_type{});

    // the waves of other keys hand over their states through LDS: every lane's registers as they are
#pragma unroll
    for (int t = 0; t < NT; ++t) l[t] = pair32_sum(l[t]);      // (both lanes of a column hold the same reference)
    if constexpr (WK > 1) {
        float* state = (float*)&ring[0][0][0];
        constexpr int kState = NT * DB * 1024 + NT * 64;       // words of a wave
        float* mine = state + (wave - WR) * kState;
        __syncthreads();                                       // (nobody reads or fills the ring any more)
        if (kg > 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        *(f32x4*)(mine + ((t * DB + b) * 4 + r) * 256 + lane * 4) = f32x4{acc[t][b][4 * r], acc[t][b][4 * r + 1], acc[t][b][4 * r + 2], acc[t][b][4 * r + 3]};
                if (h == 0) *(f32x2*)(mine + NT * DB * 1024 + t * 64 + 2 * n) = f32x2{m[t], l[t]};
            }
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            auto ml_of = [&](int k) { return *(const f32x2*)(state + (k * WR + wr - WR) * kState + NT * DB * 1024 + t * 64 + 2 * n); };
            float top = m[t];
#pragma unroll
            for (int k = 1; k < WK; ++k) top = fmaxf(top, ml_of(k).x);
            const float f0 = __builtin_amdgcn_exp2f(m[t] - top);
            l[t] *= f0;
#pragma unroll
            for (int b = 0; b < DB; ++b) acc[t][b] *= f0;
#pragma unroll 1
            for (int k = 1; k < WK; ++k) {                     // (in the order of the waves)
                const f32x2 ml = ml_of(k);
                const float f = __builtin_amdgcn_exp2f(ml.x - top);
                const float* other = state + (k * WR + wr - WR) * kState;
                l[t] += ml.y * f;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 o = *(const f32x4*)(other + ((t * DB + b) * 4 + r) * 256 + lane * 4);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[t][b][4 * r + j] += o[j] * f;
                    }
            }
            m[t] = top;
        }
    }
    if (!works) return;
    const float vscale = sizeof(KT) == 1 ? a.v_scale[it.g] : 1.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = first_row + 32 * t + n;
        if (row >= it.node_rows) continue;
        if (it.parts == 1) {
            const float inv = tr_inverse(a, l[t], it.prefix, it.n_nodes, it.row0, node[t]) * vscale;
            const int64_t at = ((int64_t)(it.row0 + node[t]) * Hq + it.g * G + row % G) * D + 4 * h;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    tr_store_out<KT>(a, at + 32 * b + 8 * r, f32x4{acc[t][b][4 * r], acc[t][b][4 * r + 1], acc[t][b][4 * r + 2], acc[t][b][4 * r + 3]} * inv);
        } else {
            const int64_t at = it.part_row0 + ((int64_t)it.g * it.parts + it.part) * it.node_rows + row;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *(f32x4*)(a.part_o + at * D + 4 * h + 32 * b + 8 * r) = f32x4{acc[t][b][4 * r], acc[t][b][4 * r + 1], acc[t][b][4 * r + 2], acc[t][b][4 * r + 3]};
            if (h == 0) *(f32x2*)(a.part_ml + 2 * at) = f32x2{m[t], l[t]};
        }
    }
}

// Rows whose scan was cut: D / 4 threads per row add up its parts in order.
template <typename KT, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, TreeSeqs s, int n_rows)
{
    constexpr int TPR = D / 4;
    const int w = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, d4 = threadIdx.x % TPR;
    // (the rows of a workgroup may belong to several sequences: every lane looks for its own)
    int i = 0;
    for (int b = 1; b < s.n; ++b) i += s.seq[b].first_merge <= w ? 1 : 0;
    if (w >= n_rows) return;
    const TreeSeq q = s.seq[i];
    const int n_nodes = s.seq[i + 1].row0 - q.row0, rows = n_nodes * a.geo.G, k = w - q.first_merge, g = k / rows, row = k % rows;
    const int64_t at = q.part_row0 + (int64_t)g * q.parts * rows + row;
    // (eight parts at a time: their loads wait together)
    float top = kNoKeyTr, sum = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < q.parts; p0 += 8) {
        f32x2 ml[8];
        f32x4 v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) ml[p] = *(const f32x2*)(a.part_ml + 2 * (at + (int64_t)min(p0 + p, q.parts - 1) * rows));
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = *(const f32x4*)(a.part_o + (at + (int64_t)min(p0 + p, q.parts - 1) * rows) * D + 4 * d4);
        float m = top;
#pragma unroll
        for (int p = 0; p < 8; ++p) m = fmaxf(m, ml[p].x);
        const float f0 = __builtin_amdgcn_exp2f(top - m);
        o *= f0; sum *= f0; top = m;
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            if (p0 + p >= q.parts) continue;
            const float f = __builtin_amdgcn_exp2f(ml[p].x - top);
            o += v[p] * f;
            sum += ml[p].y * f;
        }
    }
    const int nd = row / a.geo.G;
    const float inv = tr_inverse(a, sum, q.prefix, n_nodes, q.row0, nd) * (sizeof(KT) == 1 ? a.v_scale[g] : 1.0f);
    tr_store_out<KT>(a, ((int64_t)(q.row0 + nd) * a.geo.Hq + g * a.geo.G + row % a.geo.G) * D + 4 * d4, o * inv);
}

template <typename KT, int D>
static int launch_tree_d(const TreeArgs& a, const TreeSeqs& s, int64_t items, hipStream_t st, hipEvent_t done)
{
    const dim3 grid((unsigned)items), block(64 * kTrWaves);
    if (a.rows == 64) return launch_kernel(tree_kernel<KT, D, 2, 1>, grid, block, st, done, a, s);
    if (a.rows == 128) return launch_kernel(tree_kernel<KT, D, 4, 1>, grid, block, st, done, a, s);
    if constexpr (sizeof(KT) != 4) {
        if (a.rows == 32) return launch_kernel(tree_kernel<KT, D, 1, 1>, grid, block, st, done, a, s);
    }
    return (int)hipErrorInvalidValue;
}

int launch_tree(const TreeArgs& a, const TreeSeqs& s, int64_t items, void* stream, void* done)
{
    if (items <= 0) return (int)hipSuccess;
    if (items > kMaxWorkgroups || s.n > kTreeSeqs || (a.geo.D != 128 && a.geo.D != 64)) return (int)hipErrorInvalidValue;
    hipStream_t st = (hipStream_t)stream;
    hipEvent_t ev = (hipEvent_t)done;
    const bool d128 = a.geo.D == 128;
    if (a.geo.q_dtype == TS_F32) return d128 ? launch_tree_d<float, 128>(a, s, items, st, ev) : launch_tree_d<float, 64>(a, s, items, st, ev);
    if (a.geo.kv_dtype == TS_BF16) return d128 ? launch_tree_d<uint16_t, 128>(a, s, items, st, ev) : launch_tree_d<uint16_t, 64>(a, s, items, st, ev);
    return d128 ? launch_tree_d<uint8_t, 128>(a, s, items, st, ev) : launch_tree_d<uint8_t, 64>(a, s, items, st, ev);
}

int launch_tree_merge(const TreeArgs& a, const TreeSeqs& s, int32_t rows, void* stream, void* done)
{
    if (rows <= 0) return (int)hipSuccess;
    hipStream_t st = (hipStream_t)stream;
    hipEvent_t ev = (hipEvent_t)done;
    const bool d128 = a.geo.D == 128;
    const int per = 256 / (a.geo.D / 4);
    const dim3 grid((unsigned)((rows + per - 1) / per)), block(256);
    if (a.geo.q_dtype == TS_F32) return d128 ? launch_kernel(tree_merge_kernel<float, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<float, 64>, grid, block, st, ev, a, s, rows);
    if (a.geo.kv_dtype == TS_BF16) return d128 ? launch_kernel(tree_merge_kernel<uint16_t, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<uint16_t, 64>, grid, block, st, ev, a, s, rows);
    return d128 ? launch_kernel(tree_merge_kernel<uint8_t, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<uint8_t, 64>, grid, block, st, ev, a, s, rows);
}

}  // namespace ts
