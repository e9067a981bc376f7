// Attention of drafted trees over the paged cache.
//
// Every node of a tree sees the sequence's prefix and its own ancestors, so all nodes of a sequence share the scan of the
// prefix: row (node, head of the group) is a column of S^T = K Q^T, and a workgroup reads K and V once for all its rows.
//   - Four waves of 32 columns: WR of them side by side over the rows, WK = 4 / WR of them taking turns along the keys.  A workgroup
//     has 32 WR rows; with WR = 1 each wave scans keys of its own.
//   - Keys come in steps of 32 (two pages) per wave, copied into a ring of LDS slots by the memory system, in the order in which
//     the matrix instructions take them: a wave's operand read is always 1 KB in lane order (no bank conflicts), and copies in
//     flight take no registers.  The WR waves of a key group share the copy.
//   - Both products run on the 32x32x16 instruction.  Row rho of S^T stands for token swap23(rho % 16) of page rho / 16, so that
//     the accumulator registers of lane (h, n) are tokens 8h .. 8h + 7 of the first page, then of the second, for column n:
//     packed to bf16 they are the B operands of O^T += V^T P^T as they stand, and the matching A operand is 16 bytes (e4m3: 8)
//     of a V row.  fp32: the same with the 32x32x2 instruction, one dim of a K piece or one token of a V piece per step.
//   - The masks are looked at on the pages that hold nodes only.
// The running maximum is a reference in log2 units that is raised only when a step's weights add up to more than 2^16 in some lane:
// any reference gives the same quotient, and the maximum itself is not needed for as long.
// Weights are rounded to q's type, which the second product's matrix instruction takes (in two parts, so that nothing is lost, it would be run
// twice), and the sum below the quotient is that of the rounded ones: where many keys have one score their weights are all rounded alike, by
// up to 2^-8, and a sum of the unrounded ones would leave that in the result.  32 trees of 64 nodes over 8 Ki tokens, 64/8 heads of 128, take 564 us,
// 543 with the other sum (e4m3 557 and 550; heads of 64 228 and 229, e4m3 193 and 220).
#include <type_traits>

#include "ts_device.h"
#include "ts_launch.h"

namespace ts {

constexpr int kTrWaves = kTreeWaves;
constexpr float kBigTr = 65536.0f;
// Reference maximum of a column that has seen no key: finite, so that differences stay defined.
constexpr float kNoKeyTr = -3.402823466e38f;

// LDS image of 32 keys (two pages), in blocks of 64 pieces of 16 bytes, each of one page, so that a copy takes a scalar base and a lane's
// offset that never changes (with bases per lane, 32 trees of 64 nodes over 8 Ki tokens took 600 us instead of 566, with steps
// one after the other):
//   K block i of a page: piece 16 c + t = 16-byte chunk 4i + c of token swap23(t)
//   V, bf16: block d: piece (h, n) = tokens 8h .. 8h + 7 of dim 32 d + n;  e4m3: block i: piece n = the 16 tokens of dim 64 i + n;
//   fp32: block (d, i): piece (h, n) = tokens 8h + 4i .. + 3 of dim 32 d + n
template <typename KT, int D> struct TrStep {
    static constexpr int ES = (int)sizeof(KT), PB = 16 * D * ES;       // bytes of an element, of a tile
    static constexpr int NK = D * ES / 32, NV = NK, NB = NK + NV;      // blocks of K, of V, of both
    static constexpr int HK = NK / 2;                                  // blocks of a page's K (or V)
    static constexpr int kBytes = NB * 1024;
};
__device__ __forceinline__ int tr_swap23(int s) { return (s & 3) | ((s & 4) << 1) | ((s & 8) >> 1); }

__device__ __forceinline__ uint32_t tr_lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
// 64 x 16 bytes straight into LDS, lane l's from base + offset to lds + 16 l; counted by vmcnt.  (The wait states: m0 is read one
// instruction after it was written at the earliest, a scalar register that a vector instruction wrote -- a spilled one read back -- five.)
__device__ __forceinline__ void tr_copy(uint32_t lds, const char* base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n" :: "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void tr_wait_copies()
{
    static_assert(N >= 0 && N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14));    // vmcnt(N); expcnt and lgkmcnt untouched
}

// At most `later` steps of C copies each, N at the most, are under way behind this.
template <int N, int C>
__device__ __forceinline__ void tr_wait_steps(int later)
{
    if constexpr (N == 0) tr_wait_copies<0>();
    else if (later >= N) tr_wait_copies<N * C>();
    else tr_wait_steps<N - 1, C>(later);
}

// Where a lane's pieces lie in the first block of a page's K and V.
struct TrOffsets { uint32_t k, v; };
template <typename KT, int D>
__device__ __forceinline__ TrOffsets tr_offsets(int lane)
{
    constexpr int ES = (int)sizeof(KT);
    const int n = lane & 31, h = lane >> 5;
    return TrOffsets{(uint32_t)((lane >> 4) * 256 + tr_swap23(lane & 15) * 16), (uint32_t)(ES == 1 ? lane * 16 : n * (16 * ES) + h * (8 * ES))};
}
// The blocks wr, wr + WR, ... of two pages on their way into LDS.
template <int WR, typename KT, int D>
__device__ __forceinline__ void tr_copy_step(uint32_t lds, const char* k0, const char* k1, const char* v0, const char* v1, int wr, TrOffsets at)
{
    using S = TrStep<KT, D>;
#pragma unroll
    for (int i = 0; i < S::NB / WR; ++i) {
        const int b = wr + WR * i;
        const bool is_v = S::NK % WR == 0 ? i >= S::NK / WR : b >= S::NK;
        const int c = is_v ? b - S::NK : b;
        const bool second = S::HK % WR == 0 ? i % (S::NK / WR) >= S::HK / WR : c >= S::HK;
        const int block = second ? c - S::HK : c;
        const int from = S::ES == 4 && is_v ? (block >> 1) * 2048 + (block & 1) * 16 : block * 1024;
        tr_copy(lds + b * 1024, (is_v ? (second ? v1 : v0) : (second ? k1 : k0)) + from, is_v ? at.v : at.k);
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

// S^T of 32 keys.  The K pieces come from registers where they fit (16-bit arithmetic), else from LDS one by one.
template <typename KT, int D> struct TrK {
    static constexpr int N = sizeof(KT) == 4 ? 1 : TrStep<KT, D>::NK;
    uint4 piece[N];
};
// Lane (h, n)'s chunk h of token swap23(n % 16) of page n / 16; its chunks 2b + h lie 512 bytes apart.
template <typename KT, int D>
__device__ __forceinline__ int tr_k_at(int lane)
{
    return (lane >> 4 & 1) * (TrStep<KT, D>::HK * 1024) + (lane >> 5) * 256 + (lane & 15) * 16;
}
template <typename KT, int D>
__device__ __forceinline__ void tr_load_k(TrK<KT, D>& k, const unsigned char* lk, int lane)
{
    if constexpr (sizeof(KT) != 4) {
#pragma unroll
        for (int b = 0; b < TrK<KT, D>::N; ++b) k.piece[b] = *(const uint4*)(lk + tr_k_at<KT, D>(lane) + b * 512);
    }
}
// The A operand of 16 dims (the b-th of Q^T's): a piece, or half of an e4m3 one, widened.
template <typename KT, int D>
__device__ __forceinline__ bf16x8 tr_k_operand(const TrK<KT, D>& k, int b)
{
    if constexpr (sizeof(KT) == 2) return __builtin_bit_cast(bf16x8, k.piece[b]);
    else {
        const uint4 w = k.piece[b / 2];
        const uint2 lo = tr_widen(b % 2 ? w.z : w.x), hi = tr_widen(b % 2 ? w.w : w.y);
        return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
}
template <typename KT, int D>
__device__ __forceinline__ f32x16 tr_scores(const TrK<KT, D>& k, [[maybe_unused]] const unsigned char* lk, const TrQ<KT, D>& q, [[maybe_unused]] int lane)
{
    f32x16 s = {};
    if constexpr (sizeof(KT) == 4) {
#pragma unroll
        for (int b = 0; b < TrStep<KT, D>::NK; ++b) {
            const f32x4 kf = *(const f32x4*)(lk + tr_k_at<KT, D>(lane) + b * 512);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q.q[b][e], s, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_k_operand<KT, D>(k, b), q.q[b], s, 0, 0, 0);
        }
    }
    return s;
}

// A lane's eight tokens (8h ..) of dim 32 d + n of page p, as they lie in LDS: VW words.
template <typename KT, int D> struct TrV { static constexpr int VW = 2 * (int)sizeof(KT); uint32_t w[VW]; };
template <typename KT, int D>
__device__ __forceinline__ TrV<KT, D> tr_load_v(const unsigned char* lv, int p, int d, int lane)
{
    TrV<KT, D> v;
    constexpr int DB = D / 32;
    if constexpr (sizeof(KT) == 1) {
        const uint2 x = *(const uint2*)(lv + (p * TrStep<KT, D>::HK + (d >> 1)) * 1024 + ((d & 1) * 32 + (lane & 31)) * 16 + (lane >> 5) * 8);
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
__device__ __forceinline__ bf16x8 tr_v_operand(const TrV<KT, D>& v)
{
    if constexpr (sizeof(KT) == 2) return __builtin_bit_cast(bf16x8, make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]));
    else {
        const uint2 a = tr_widen(v.w[0]), b = tr_widen(v.w[1]);
        return __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y));
    }
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
// sum + both of a pair of bf16, in single precision (measured over 16 Ki random triples: at most 2.5 x 2^-24 short of the exact sum).
__device__ __forceinline__ float add_pair(uint32_t pair, float sum)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}

// Which of the eight keys from node number j0 on a node sees, as bits 0 .. 7.  Negative numbers are the prefix, which everybody sees;
// nodes from n_nodes on do not exist.  Without a mask a node sees those up to itself.
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
struct TrItem { int seq, node_rows, n_nodes, row0, prefix, g, group, part, parts, part_pages, part_row0; };
__device__ __forceinline__ TrItem tr_item(const TreeArgs& a, const TreeSeqs& s)
{
    const int lane = threadIdx.x & 63, w = blockIdx.x;
    int i = -1;
#pragma unroll
    for (int b = 0; b < kTreeSeqs; b += 64) {
        const int k = min(b + lane, kTreeSeqs - 1);
        i += __builtin_popcountll(__ballot((b + lane < s.n) & (s.seq[k].first_item <= w)));
    }
    const TreeSeq q = s.seq[i];
    TrItem t;
    t.seq = q.seq; t.row0 = q.row0; t.n_nodes = q.n_nodes; t.prefix = q.prefix; t.parts = q.parts; t.part_pages = q.part_pages; t.part_row0 = q.part_row0;
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

template <typename KT, int D, int WR> constexpr int tr_ring() { return tree_ring_slots(TrStep<KT, D>::kBytes * (kTrWaves / WR), sizeof(KT) == 2); }

template <typename KT, int D, int WR>
__global__ __launch_bounds__(64 * kTrWaves) void tree_kernel(TreeArgs a, TreeSeqs s)
{
    using S = TrStep<KT, D>;
    constexpr bool F32 = sizeof(KT) == 4;
    constexpr int WK = kTrWaves / WR, DB = D / 32, ROWS = 32 * WR, R = tr_ring<KT, D, WR>(), C = S::NB / WR;
    static_assert(S::NB % WR == 0 && C * (R - 1) < 64, "copies per wave");
    __shared__ __align__(16) unsigned char ring[R][WK][S::kBytes];
    static_assert(sizeof ring >= (size_t)(kTrWaves - WR) * (DB * 4096 + 256), "the ring holds the waves' states at the end");
    const TrItem it = tr_item(a, s);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, n = lane & 31;
    const int wr = wave % WR, kg = wave / WR;
    const int Hq = a.geo.Hq, Hkv = a.geo.Hkv, G = a.geo.G;
    const int ctx_len = it.prefix + it.n_nodes, pages = (ctx_len + kPage - 1) / kPage;
    const int page0 = it.part * it.part_pages, page1 = min(page0 + it.part_pages, pages);
    const int n_step = (page1 - page0 + 2 * WK - 1) / (2 * WK);
    const int first_row = it.group * ROWS + wr * 32;

    const int32_t TS_CONSTANT* bt = as_constant(a.block_table) + (int64_t)it.seq * a.geo.max_pages;
    const char* kc = (const char*)a.k_cache + (int64_t)it.g * S::PB;
    const char* vc = (const char*)a.v_cache + (int64_t)it.g * S::PB;
    const uint32_t page_bytes = (uint32_t)Hkv * S::PB;         // of all heads: below 2^32 (checked by the call)
    const TrOffsets at = tr_offsets<KT, D>(lane);
    // (past the end of the range: its last page again, whose keys do not count a second time)
    auto page_of = [&](int i) { return page0 + 2 * (WK * i + kg); };
    auto id_of = [&](int page) { return bt[min(page, page1 - 1)]; };
    const bool works = first_row < it.node_rows && page_of(0) < page1;     // (a wave without rows or keys only copies)
    // (page ids are asked for a step ahead; the opaque copies keep the wait for them where they are used)
    int32_t next0 = id_of(page_of(0)), next1 = id_of(page_of(0) + 1);
    auto issue = [&](int i) {
        const uint64_t p0 = (uint64_t)(uint32_t)opaque_uniform(next0) * page_bytes, p1 = (uint64_t)(uint32_t)opaque_uniform(next1) * page_bytes;
        next0 = id_of(page_of(i + 1)); next1 = id_of(page_of(i + 1) + 1);
        tr_copy_step<WR, KT, D>(tr_lds_address(ring[i % R][kg]), kc + p0, kc + p1, vc + p0, vc + p1, wr, at);
    };
    // the copies of a step have landed, those of up to `later` steps behind it may be under way; then everybody's have
    auto wait = [&](int later) {
        tr_wait_steps<R - 1, C>(later);
        if constexpr (WR > 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < n_step) issue(i);

    // scores are wanted in log2 units: s * c; a negative c (e4m3 scale) is taken into Q, so that the maximum can be taken of s
    // (a scale of zero becomes a very small one: what is masked, -inf, keeps a weight of zero)
    const float c_signed = a.sm_scale * (sizeof(KT) == 1 ? a.k_scale[it.g] : 1.0f) * kLog2e;
    const float c = c_signed == 0.0f ? 1e-37f : __builtin_fabsf(c_signed);
    const int row = first_row + n, row_in = min(row, it.node_rows - 1), node = row_in / G;
    TrQ<KT, D> q;
    tr_load_q(q, a.q, ((int64_t)(it.row0 + node) * Hq + it.g * G + row_in % G) * D, h, c_signed < 0.0f);
    f32x16 acc[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
    float m = kNoKeyTr, l = 0.0f;

    constexpr bool PIPE = sizeof(KT) == 2 && R == 5;           // steps overlap (below)
    TrK<KT, D> k;
    wait(min(R - 1, n_step - 1));
    if (works) tr_load_k(k, ring[0][kg], lane);
    // step i is done with its LDS slot: the next one's K, and copies of step i + R into the slot
    auto advance = [&](int i) {
        if (i + 1 >= n_step) return;
        wait(min(R - 2, n_step - 2 - i));
        if (i + R < n_step) issue(i + R);
        if (works) tr_load_k(k, ring[(i + 1) % R][kg], lane);
    };

    auto raise = [&](const f32x16& x) {                        // the reference, to the columns' maxima
        float top = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
        const float m_new = fmaxf(m, pair32_max(top) * c);
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
#pragma unroll
        for (int b = 0; b < DB; ++b) acc[b] *= alpha;
        l *= alpha;
        m = m_new;
    };
    auto step = [&](int i, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const unsigned char* lk = ring[i % R][kg];
        const unsigned char* lv = lk + S::NK * 1024;
        const int page = page_of(i);
        // The matrix products go first where two waves of a SIMD want to issue: the other's softmax then fills the gaps (32 trees of 64 nodes
        // over 8 Ki tokens, 64/8 heads: e4m3 589 -> 556 us when this was put in, 587 with the softmax first).
        __builtin_amdgcn_s_setprio(1);
        f32x16 x = tr_scores(k, lk, q, lane);
        // (16-bit arithmetic: V is read while the scores are being made and turned into weights)
        TrV<KT, D> v[F32 ? 1 : 2][F32 ? 1 : DB];
        if constexpr (!F32) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int b = 0; b < DB; ++b) v[u][b] = tr_load_v<KT, D>(lv, u, b, lane);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        [[maybe_unused]] uint32_t seen = 0;                    // bits 0 .. 7: tokens 8h .. of the first page, 8 .. 15: of the second
        if constexpr (MASKED) {
            const int j0 = page * kPage + 8 * h - it.prefix;
            seen = tr_seen(a, it.row0, it.n_nodes, node, j0) | tr_seen(a, it.row0, it.n_nodes, node, j0 + kPage) << 8;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = seen >> e & 1 ? x[e] : -INFINITY;
        }
        float p[16], sum;
        [[maybe_unused]] uint32_t packed[8];                   // (16-bit arithmetic) the weights as they enter the second product
        auto weigh = [&] {
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -m));
            float t[4];
            if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = (p[e] + p[e + 4]) + (p[e + 8] + p[e + 12]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    packed[e] = pack_bf16(p[2 * e], p[2 * e + 1]);
                    t[e & 3] = add_pair(packed[e], e < 4 ? 0.0f : t[e & 3]);
                }
            }
            sum = (t[0] + t[1]) + (t[2] + t[3]);
        };
        weigh();
        if (__any(sum > kBigTr)) {                             // rare: the reference is raised to the column's maximum
            raise(x);
            weigh();
        }
        l += sum;
        [[maybe_unused]] bool odd = false;
        // (masked) what does not exist does not enter the sums, and what is not finite enters below, in those rows that see it
        if constexpr (MASKED && !F32) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int b = 0; b < DB; ++b) odd |= tr_clean_v(v[u][b], ctx_len - (page + u) * kPage - 8 * h);
        }
        bool late = false;                                     // whether the slot is still needed
        if constexpr (MASKED && !F32) late = __any(odd);
        if constexpr (!F32) {
            if (!MASKED) advance(i);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(packed[4 * u], packed[4 * u + 1], packed[4 * u + 2], packed[4 * u + 3]));
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_v_operand<KT, D>(v[u][b]), pb, acc[b], 0, 0, 0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    TrV<KT, D> w = tr_load_v<KT, D>(lv, u, b, lane);
                    if constexpr (MASKED) odd |= tr_clean_v(w, ctx_len - (page + u) * kPage - 8 * h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w.w[e]), p[8 * u + e], acc[b], 0, 0, 0);
                }
            if constexpr (MASKED) late = __any(odd);
        }
        if constexpr (MASKED) {
            if (late) {
                // How many values of +inf (or NaN) and of -inf (or NaN) a row sees of a dim: products of zeros and ones.
                for (int u = 0; u < 2; ++u) {                  // (not unrolled: rarely taken)
                    const int have = ctx_len - (page + u) * kPage - 8 * h;
                    const uint32_t bits = seen >> (8 * u);
                    auto two = [&](int e) { return (bits >> e & 1 ? 0x3f80u : 0u) | (bits >> (e + 1) & 1 ? 0x3f800000u : 0u); };
                    const bf16x8 on = __builtin_bit_cast(bf16x8, make_uint4(two(0), two(2), two(4), two(6)));
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        const TrV<KT, D> w = tr_load_v<KT, D>(lv, u, b, lane);
                        uint32_t plus[4] = {}, minus[4] = {};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = tr_element(w, e);
                            plus[e / 2] |= e < have && !(f < INFINITY) ? 0x3f80u << (16 * (e & 1)) : 0u;
                            minus[e / 2] |= e < have && !(f > -INFINITY) ? 0x3f80u << (16 * (e & 1)) : 0u;
                        }
                        const f32x16 zero = {};
                        const f32x16 np = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(plus[0], plus[1], plus[2], plus[3])), on, zero, 0, 0, 0);
                        const f32x16 nm = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(minus[0], minus[1], minus[2], minus[3])), on, zero, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            if (np[r] > 0.0f) acc[b][r] += INFINITY;
                            if (nm[r] > 0.0f) acc[b][r] -= INFINITY;
                        }
                    }
                }
            }
        }
        if (F32 || MASKED) advance(i);
    };

    // pages whose keys everybody sees, then those that hold nodes
    const int n_plain = max(min(it.prefix / kPage, page1) - page0, 0) / (2 * WK);
    auto one = [&](int i, auto masked) { if (works) step(i, masked); else advance(i); };
    int i = 0;
    if constexpr (PIPE) {
        // Three steps at once: while the matrix unit works on V^T P^T of step i - 1 and K Q^T of step i + 1 in turn, the scores of step i
        // become weights, a share of them behind each instruction, and the operands of the next turn are read from LDS as theirs
        // are used up.  (Between two matrix instructions there is room for six or so vector ones; left to itself the compiler puts
        // the phases one after the other.)  32 trees of 64 nodes over 8 Ki tokens, 64/8 heads of 128, when this was put in: 558 -> 528 us,
        // 1045 TFLOP/s at 1.67 GHz, 462 without the copies, on what LDS holds; heads of 64 406 -> 399.  With the weights added up as they are
        // rounded 564, with the pair packed and added behind the products of K (behind those of P a batch of 288 us takes 301 to 314, all pairs at the
        // step's end 300).  e4m3 keeps the steps apart: four conversions more per matrix instruction do not
        // fit between two (530 us; 545 this way).  A ring of five slots, for step i + 2 is waited for when step i begins.
        if (n_plain > 0) {
            constexpr int NQ = D / 16, NP = 2 * DB, SLOTS = NQ + NP, PER = 16 / SLOTS;
            f32x16 x = {};
            TrV<KT, D> v[2][DB] = {};
            bf16x8 pb[2] = {};
            if (works) x = tr_scores(k, ring[0][kg], q, lane);
            if (n_step > 1) {
                wait(min(R - 2, n_step - 2));
                if (works) tr_load_k(k, ring[1][kg], lane);
            }
            for (; i < n_plain; ++i) {
                if (i + 2 < n_step) {                          // K of step i + 2 is there; V of step i - 1 has been read by everybody
                    wait(min(R - 4, n_step - 3 - i));
                    if (i > 0 && i - 1 + R < n_step) issue(i - 1 + R);
                }
                if (!works) continue;
                const unsigned char* lv = ring[i % R][kg] + S::NK * 1024;
                const unsigned char* lk = ring[(i + 2) % R][kg] + tr_k_at<KT, D>(lane);    // (behind the last step: whatever is there, to no use)
                f32x16 x_next = {};
                __builtin_amdgcn_s_setprio(1);
                float p[16], t[4] = {};
                uint32_t packed[8];
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) {
                    const int o = j / 2;
                    if (j % 2 == 0) {
                        const int u = o / DB, b = o % DB;
                        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_v_operand<KT, D>(v[u][b]), pb[u], acc[b], 0, 0, 0);
                        v[u][b] = tr_load_v<KT, D>(lv, u, b, lane);
                    } else {
                        x_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_k_operand<KT, D>(k, o), q.q[o], x_next, 0, 0, 0);
                        k.piece[o] = *(const uint4*)(lk + o * 512);
                    }
#pragma unroll
                    for (int e = PER * j; e < PER * (j + 1); ++e) {
                        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -m));
                        if (e % 2 == 1) {
                            packed[e / 2] = pack_bf16(p[e - 1], p[e]);
                            t[e / 2 & 3] = add_pair(packed[e / 2], t[e / 2 & 3]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                float sum = (t[0] + t[1]) + (t[2] + t[3]);
                if (__any(sum > kBigTr)) {
                    raise(x);
                    sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -m));
                        if (e % 2 == 1) {
                            packed[e / 2] = pack_bf16(p[e - 1], p[e]);
                            sum = add_pair(packed[e / 2], sum);
                        }
                    }
                }
                l += sum;
#pragma unroll
                for (int u = 0; u < 2; ++u) pb[u] = __builtin_bit_cast(bf16x8, make_uint4(packed[4 * u], packed[4 * u + 1], packed[4 * u + 2], packed[4 * u + 3]));
                x = x_next;
            }
            if (i < n_step) {                                  // the steps with nodes follow one by one
                wait(min(R - 2, n_step - 1 - i));
                if (i - 1 + R < n_step) issue(i - 1 + R);
                if (works) tr_load_k(k, ring[i % R][kg], lane);
            }
            if (works) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int b = 0; b < DB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_v_operand<KT, D>(v[u][b]), pb[u], acc[b], 0, 0, 0);
            }
        }
    } else {
        for (; i < n_plain; ++i) one(i, std::false_type{});
    }
    for (; i < n_step; ++i) one(i, std::true_type{});

    // the waves of other keys hand over their states through LDS: every lane's registers as they are
    l = pair32_sum(l);                                         // (both lanes of a column hold the same reference)
    if constexpr (WK > 1) {
        float* state = (float*)&ring[0][0][0];
        constexpr int kState = DB * 1024 + 64;                 // words of a wave
        float* mine = state + (wave - WR) * kState;
        __syncthreads();                                       // (nobody reads or fills the ring any more)
        if (kg > 0) {
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *(f32x4*)(mine + (b * 4 + r) * 256 + lane * 4) = f32x4{acc[b][4 * r], acc[b][4 * r + 1], acc[b][4 * r + 2], acc[b][4 * r + 3]};
            if (h == 0) *(f32x2*)(mine + DB * 1024 + 2 * n) = f32x2{m, l};
        }
        __syncthreads();
        if (kg > 0) return;
        auto ml_of = [&](int k) { return *(const f32x2*)(state + (k * WR + wr - WR) * kState + DB * 1024 + 2 * n); };
        float top = m;
#pragma unroll
        for (int w = 1; w < WK; ++w) top = fmaxf(top, ml_of(w).x);
        const float f0 = __builtin_amdgcn_exp2f(m - top);
        l *= f0;
#pragma unroll
        for (int b = 0; b < DB; ++b) acc[b] *= f0;
#pragma unroll 1
        for (int w = 1; w < WK; ++w) {                         // (in the order of the waves)
            const f32x2 ml = ml_of(w);
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            const float* other = state + (w * WR + wr - WR) * kState;
            l += ml.y * f;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 o = *(const f32x4*)(other + (b * 4 + r) * 256 + lane * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b][4 * r + j] += o[j] * f;
                }
        }
        m = top;
    }
    if (!works || row >= it.node_rows) return;
    if (it.parts == 1) {
        const float inv = tr_inverse(a, l, it.prefix, it.n_nodes, it.row0, node) * (sizeof(KT) == 1 ? a.v_scale[it.g] : 1.0f);
        const int64_t at = ((int64_t)(it.row0 + node) * Hq + it.g * G + row % G) * D + 4 * h;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                tr_store_out<KT>(a, at + 32 * b + 8 * r, f32x4{acc[b][4 * r], acc[b][4 * r + 1], acc[b][4 * r + 2], acc[b][4 * r + 3]} * inv);
    } else {
        const int64_t at = it.part_row0 + ((int64_t)it.g * it.parts + it.part) * it.node_rows + row;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(f32x4*)(a.part_o + at * D + 4 * h + 32 * b + 8 * r) = f32x4{acc[b][4 * r], acc[b][4 * r + 1], acc[b][4 * r + 2], acc[b][4 * r + 3]};
        if (h == 0) *(f32x2*)(a.part_ml + 2 * at) = f32x2{m, l};
    }
}

// Rows whose scan was cut: a wave per row, four dims per lane: with 128 dims the two halves of the wave
// take every other part, with 64 dims the four quarters every fourth.  Eight parts of each are read together.
template <typename KT, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, TreeSeqs s, int n_rows)
{
    constexpr int SHARES = 256 / D;                            // parts side by side in a wave
    const int lane = threadIdx.x & 63, share = lane / (D / 4), d4 = lane % (D / 4);
    const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (w >= n_rows) return;
    int i = -1;
#pragma unroll
    for (int b = 0; b < kTreeSeqs; b += 64) {
        const int k = min(b + lane, kTreeSeqs - 1);
        i += __builtin_popcountll(__ballot((b + lane < s.n) & (s.seq[k].first_merge <= w)));
    }
    // (a sequence that was not cut has the number of the next one that was, or, behind the last of them, that of all rows, which w is below:
    // the last match is one that was cut)
    const TreeSeq q = s.seq[i];
    const int rows = q.n_nodes * a.geo.G, k = w - q.first_merge, g = k / rows, row = k % rows;
    const int64_t at = q.part_row0 + (int64_t)g * q.parts * rows + row;
    float top = kNoKeyTr, sum = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = share; p0 - share < q.parts; p0 += 8 * SHARES) {
        f32x2 ml[8];
        f32x4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            ml[j] = f32x2{kNoKeyTr, 0.0f};
            v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (p0 - share + j * SHARES < q.parts) {           // (the same for the wave)
                const int64_t from = at + (int64_t)min(p0 + j * SHARES, q.parts - 1) * rows;
                ml[j] = *(const f32x2*)(a.part_ml + 2 * from);
                v[j] = *(const f32x4*)(a.part_o + from * D + 4 * d4);
            }
        }
        float m = top;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, ml[j].x);     // (a part that is read twice changes nothing here)
        const float f0 = __builtin_amdgcn_exp2f(top - m);
        o *= f0; sum *= f0; top = m;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = p0 + j * SHARES < q.parts;
            const float f = __builtin_amdgcn_exp2f(ml[j].x - top);
            const f32x4 add = v[j] * f;
            o = in ? o + add : o;
            sum = in ? sum + ml[j].y * f : sum;
        }
    }
    // the shares meet: quarters first, then halves
    auto meet = [&](int step) {
        const float m = fmaxf(top, __shfl_xor(top, step, 64));
        const float f = __builtin_amdgcn_exp2f(top - m);
        o *= f; sum *= f; top = m;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], step, 64);
        sum += __shfl_xor(sum, step, 64);
    };
    if constexpr (SHARES == 4) meet(16);
    meet(32);
    const int nd = row / a.geo.G;
    const float inv = tr_inverse(a, sum, q.prefix, q.n_nodes, q.row0, nd) * (sizeof(KT) == 1 ? a.v_scale[g] : 1.0f);
    if (share == 0) tr_store_out<KT>(a, ((int64_t)(q.row0 + nd) * a.geo.Hq + g * a.geo.G + row % a.geo.G) * D + 4 * d4, o * inv);
}

template <typename KT, int D>
static int launch_tree_d(const TreeArgs& a, const TreeSeqs& s, int64_t items, hipStream_t st, hipEvent_t done)
{
    const dim3 grid((unsigned)items), block(64 * kTrWaves);
    if (a.rows == 64) return launch_kernel(tree_kernel<KT, D, 2>, grid, block, st, done, a, s);
    if (a.rows == 128) return launch_kernel(tree_kernel<KT, D, 4>, grid, block, st, done, a, s);
    if constexpr (sizeof(KT) != 4 || D == 64) {
        if (a.rows == 32) return launch_kernel(tree_kernel<KT, D, 1>, grid, block, st, done, a, s);
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
    const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
    if (a.geo.q_dtype == TS_F32) return d128 ? launch_kernel(tree_merge_kernel<float, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<float, 64>, grid, block, st, ev, a, s, rows);
    if (a.geo.kv_dtype == TS_BF16) return d128 ? launch_kernel(tree_merge_kernel<uint16_t, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<uint16_t, 64>, grid, block, st, ev, a, s, rows);
    return d128 ? launch_kernel(tree_merge_kernel<uint8_t, 128>, grid, block, st, ev, a, s, rows) : launch_kernel(tree_merge_kernel<uint8_t, 64>, grid, block, st, ev, a, s, rows);
}

}  // namespace ts
