// Attention of drafted trees over the paged cache.
//
// Every node of a tree sees the sequence's prefix and its own ancestors, so all nodes of a sequence share the scan of the
// prefix: row (node, head of the group) is a column of S^T = K Q^T (columns of 16 per matrix instruction), and K and V are
// read once for all rows of a workgroup.
//   - A workgroup takes up to 16 NT rows of one KV head over a range of pages; its four waves take two pages (32 keys) in
//     turn and meet in LDS at the end.  Keys of a wave's two pages are dealt to the accumulator rows of the two score products
//     so that lane (r, n) holds eight neighbouring tokens of column n, keys 8r .. 8r + 7 of the 32: as bf16 they are the B
//     operand of O^T += V^T P^T (16x16x32) as they stand, and the matching A operand is one 16-byte (e4m3: 8-byte) piece of
//     a V row.
//   - fp32: the same with the 16x16x4 instruction, one dim of a 16-byte K piece or one token of a V piece per step.
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

// Two (page, KV head) tiles in registers.
template <typename KT, int D> struct TrTile {
    static constexpr int X = 16 / (int)sizeof(KT), KB = D / (4 * X), VB = D / 16;
    static constexpr int VW = sizeof(KT) == 4 ? 8 : (sizeof(KT) == 2 ? 4 : 2);     // words of a lane's eight tokens of a dim
    uint4 k[2][KB];
    uint32_t v[VB][VW];
};
template <typename KT, int D> struct TrQ {
    using T = std::conditional_t<sizeof(KT) == 4, f32x4, bf16x8>;
    static constexpr int N = sizeof(KT) == 4 ? D / 16 : D / 32;
    T q[N];
};

// Lane (r, n): rows i = n of the score products stand for page i / 8, slot 8 (i / 4 % 2) + i % 4 + 4 m; V piece: page r / 2,
// slots 8 (r % 2) .. + 7 of dim 16 b + n.
template <typename KT, int D>
__device__ __forceinline__ void tr_load_k(TrTile<KT, D>& t, const char* kc, int64_t tile0, int64_t tile1, int lane)
{
    constexpr int kBytes = 16 * D * (int)sizeof(KT);
    const int n = lane & 15, r = lane >> 4;
    const char* p = kc + (n >= 8 ? tile1 : tile0) * kBytes + (r * 16 + 8 * ((n >> 2) & 1) + (n & 3)) * 16;
#pragma unroll
    for (int b = 0; b < TrTile<KT, D>::KB; ++b) {
        t.k[0][b] = *(const uint4*)(p + b * 1024);
        t.k[1][b] = *(const uint4*)(p + b * 1024 + 64);
    }
}
template <typename KT, int D>
__device__ __forceinline__ void tr_load_v(TrTile<KT, D>& t, const char* vc, int64_t tile0, int64_t tile1, int lane)
{
    constexpr int kBytes = 16 * D * (int)sizeof(KT), ES = (int)sizeof(KT);
    const int n = lane & 15, r = lane >> 4;
    const char* p = vc + (r >= 2 ? tile1 : tile0) * kBytes + n * (16 * ES) + (r & 1) * (8 * ES);
#pragma unroll
    for (int b = 0; b < TrTile<KT, D>::VB; ++b) {
        if constexpr (ES == 1) {
            const uint2 x = *(const uint2*)(p + b * 256);
            t.v[b][0] = x.x; t.v[b][1] = x.y;
        } else {
#pragma unroll
            for (int j = 0; j < TrTile<KT, D>::VW / 4; ++j) {
                const uint4 x = *(const uint4*)(p + b * (256 * ES) + 16 * j);
                t.v[b][4 * j] = x.x; t.v[b][4 * j + 1] = x.y; t.v[b][4 * j + 2] = x.z; t.v[b][4 * j + 3] = x.w;
            }
        }
    }
}

__device__ __forceinline__ uint2 tr_widen(uint32_t w)          // four e4m3 -> four bf16 (exact)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
}

// Q^T operand of one column: the dims in the order of the K pieces.
template <typename KT, int D>
__device__ __forceinline__ void tr_load_q(TrQ<KT, D>& t, const void* q, int64_t at, int r, bool negate)
{
    if constexpr (sizeof(KT) == 4) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            t.q[b] = *(const f32x4*)((const float*)q + at + 4 * (4 * b + r));
            if (negate) t.q[b] = -t.q[b];
        }
    } else {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            const int d0 = sizeof(KT) == 2 ? 8 * (4 * b + r) : 16 * (4 * (b >> 1) + r) + 8 * (b & 1);
            uint4 x = *(const uint4*)((const uint16_t*)q + at + d0);
            if (negate) x = make_uint4(x.x ^ 0x80008000u, x.y ^ 0x80008000u, x.z ^ 0x80008000u, x.w ^ 0x80008000u);
            t.q[b] = __builtin_bit_cast(bf16x8, x);
        }
    }
}

// S^T of 16 keys (half M of the pair) and 16 columns.
template <int M, typename KT, int D>
__device__ __forceinline__ f32x4 tr_scores(const TrTile<KT, D>& t, const TrQ<KT, D>& q)
{
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (sizeof(KT) == 4) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            const f32x4 k = __builtin_bit_cast(f32x4, t.k[M][b]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q.q[b][e], s, 0, 0, 0);
        }
    } else if constexpr (sizeof(KT) == 2) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[M][b]), q.q[b], s, 0, 0, 0);
    } else {
#pragma unroll
        for (int b = 0; b < D / 64; ++b) {
            const uint2 a0 = tr_widen(t.k[M][b].x), a1 = tr_widen(t.k[M][b].y), a2 = tr_widen(t.k[M][b].z), a3 = tr_widen(t.k[M][b].w);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(a0.x, a0.y, a1.x, a1.y)), q.q[2 * b], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(a2.x, a2.y, a3.x, a3.y)), q.q[2 * b + 1], s, 0, 0, 0);
        }
    }
    return s;
}

// A lane's eight tokens of dim 16 b + n in the form of the second product's operand, and as numbers.
template <typename KT, int D>
__device__ __forceinline__ uint4 tr_v_bf16(const TrTile<KT, D>& t, int b)
{
    if constexpr (sizeof(KT) == 1) {
        const uint2 x = tr_widen(t.v[b][0]), y = tr_widen(t.v[b][1]);
        return make_uint4(x.x, x.y, y.x, y.y);
    } else return make_uint4(t.v[b][0], t.v[b][1], t.v[b][2], t.v[b][3]);
}

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2)); }

// Eight bits of a node's row of the mask from node j0 on (j0 may be negative: the prefix, which everybody sees); nodes from
// n_nodes on do not exist.  Without a mask a node sees those up to itself.
__device__ __forceinline__ uint32_t tr_visible(const uint64_t* mask, int words, int n_nodes, int node, int j0)
{
    auto word = [&](int i) -> uint64_t {
        if (i < 0) return ~0ull;
        const int exist = (mask ? n_nodes : node + 1) - 64 * i;
        if (exist <= 0) return 0;
        const uint64_t m = mask && i < words ? mask[i] : ~0ull;
        return exist >= 64 ? m : m & ((1ull << exist) - 1);
    };
    const int w = j0 >> 6, sh = j0 & 63;                       // (rounded down)
    uint64_t bits = word(w) >> sh;
    if (sh > 56) bits |= word(w + 1) << (64 - sh);
    return (uint32_t)bits & 0xffu;
}

// What a workgroup does, from the launch's list.
struct TrItem { int seq, node_rows, n_nodes, row0, prefix, g, group, part, parts, part_row0; };
__device__ __forceinline__ TrItem tr_item(const TreeArgs& a, const TreeSeqs& s)
{
    const int lane = threadIdx.x & 63, w = blockIdx.x;
    int i = -1;
#pragma unroll
    for (int b = 0; b < kTreeSeqs; b += 64)
        i += __builtin_popcountll(__ballot(b + lane < s.n && s.seq[min(b + lane, kTreeSeqs - 1)].first_item <= w));
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
    if (l != 0.0f) return 1.0f / l;
    if (prefix > 0) return __builtin_nanf("");
    uint32_t any = 0;
    for (int j = 0; j < n_nodes; j += 8) any |= tr_visible(a.mask ? a.mask + (int64_t)(row0 + node) * a.mask_words : nullptr, a.mask_words, n_nodes, node, j);
    return any ? __builtin_nanf("") : 0.0f;
}

template <typename KT, int D, int NT>
__global__ __launch_bounds__(64 * kTrWaves) void tree_kernel(TreeArgs a, TreeSeqs s)
{
    constexpr int DB = D / 16, ROWS = 16 * NT;
    __shared__ f32x4 mo[kTrWaves][16][D / 4 + 1];
    __shared__ float mm[kTrWaves][ROWS], ml[kTrWaves][ROWS];
    const TrItem it = tr_item(a, s);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane >> 4, n = lane & 15;
    const int Hq = a.geo.Hq, Hkv = a.geo.Hkv, G = a.geo.G;
    const int ctx_len = it.prefix + it.n_nodes, pages = (ctx_len + kPage - 1) / kPage;
    const int page0 = it.part * a.part_pages, page1 = min(page0 + a.part_pages, pages);
    const int first_row = it.group * ROWS;

    // scores are wanted in log2 units: s * c; a negative c (e4m3 scale) is taken into Q, so that the maximum can be taken of s
    const float c_signed = a.sm_scale * (sizeof(KT) == 1 ? a.k_scale[it.g] : 1.0f) * kLog2e, c = __builtin_fabsf(c_signed);
    TrQ<KT, D> q[NT];
    int node[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = min(first_row + 16 * t + n, it.node_rows - 1);
        node[t] = row / G;
        tr_load_q(q[t], a.q, ((int64_t)(it.row0 + node[t]) * Hq + it.g * G + row % G) * D, r, c_signed < 0.0f);
    }
    f32x4 acc[NT][DB];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = kNoKeyTr; l[t] = 0.0f;
#pragma unroll
        for (int b = 0; b < DB; ++b) acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t TS_CONSTANT* bt = as_constant(a.block_table) + (int64_t)it.seq * a.geo.max_pages;
    const char* kc = (const char*)a.k_cache;
    const char* vc = (const char*)a.v_cache;

    auto step = [&](int page, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const int64_t tile0 = (int64_t)bt[page] * Hkv + it.g, tile1 = (int64_t)bt[min(page + 1, page1 - 1)] * Hkv + it.g;
        TrTile<KT, D> tile;
        tr_load_k(tile, kc, tile0, tile1, lane);
        tr_load_v(tile, vc, tile0, tile1, lane);
        const int key0 = page * kPage + 8 * r;                 // the lane's first key
        // (masked) what no row sees does not enter the sums, and values that are not finite enter those of the rows that see them only
        [[maybe_unused]] bool odd = false;
        if constexpr (MASKED) {
            const int have = ctx_len - key0;                   // keys of the lane that exist
#pragma unroll
            for (int b = 0; b < DB; ++b) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (sizeof(KT) == 4) {
                        if (e >= have) tile.v[b][e] = 0;
                        else if ((tile.v[b][e] & 0x7f800000u) == 0x7f800000u) { odd = true; tile.v[b][e] = 0; }
                    } else if constexpr (sizeof(KT) == 2) {
                        const uint32_t field = 0xffffu << (16 * (e & 1)), inf = 0x7f80u << (16 * (e & 1));
                        if (e >= have) tile.v[b][e / 2] &= ~field;
                        else if ((tile.v[b][e / 2] & inf) == inf) { odd = true; tile.v[b][e / 2] &= ~field; }
                    } else {
                        const uint32_t field = 0xffu << (8 * (e & 3)), nan = 0x7fu << (8 * (e & 3));
                        if (e >= have) tile.v[b][e / 4] &= ~field;
                        else if ((tile.v[b][e / 4] & nan) == nan) { odd = true; tile.v[b][e / 4] &= ~field; }
                    }
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x4 s0 = tr_scores<0>(tile, q[t]), s1 = tr_scores<1>(tile, q[t]);
            float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
            [[maybe_unused]] uint32_t seen = 0xff;
            if constexpr (MASKED) {
                seen = tr_visible(a.mask ? a.mask + (int64_t)(it.row0 + node[t]) * a.mask_words : nullptr, a.mask_words, it.n_nodes, node[t], key0 - it.prefix);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = (seen >> e) & 1 ? x[e] : -INFINITY;
            }
            const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * c;
            if (__any(top > m[t] + kRaiseTr)) {                // rare
                const float m_new = fmaxf(m[t], pair32_max(pair16_max(top)));
                const float alpha = __builtin_amdgcn_exp2f(m[t] - m_new);
#pragma unroll
                for (int b = 0; b < DB; ++b) acc[t][b] *= alpha;
                l[t] *= alpha;
                m[t] = m_new;
            }
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -m[t]));
                if constexpr (MASKED) p[e] = (seen >> e) & 1 ? p[e] : 0.0f;
            }
            l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            if constexpr (sizeof(KT) == 4) {
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tile.v[b][e]), p[e], acc[t][b], 0, 0, 0);
            } else {
                const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])));
#pragma unroll
                for (int b = 0; b < DB; ++b)
                    acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, tr_v_bf16(tile, b)), pb, acc[t][b], 0, 0, 0);
            }
            if constexpr (MASKED) {
                if (__any(odd)) {
                    // lane (r, n) of the accumulator: dims 16 b + 4 r + j of column n; key 8 k + e: weight in lane (k, n).  Only
                    // values that are not finite are added here.
                    for (int k = 0; k < 4; ++k) {
                        const KT* v = (const KT*)vc + (k >= 2 ? tile1 : tile0) * (kPage * D) + 4 * r * kPage + 8 * (k & 1);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float pe = __shfl(p[e], 16 * k + n, 64);
                            const bool on = (__shfl((int)seen, 16 * k + n, 64) >> e) & 1;
                            for (int d = 0; on && d < D; d += 16) {
                                for (int j = 0; j < 4; ++j) {
                                    const KT x = v[(d + j) * kPage + e];
                                    float f;
                                    if constexpr (sizeof(KT) == 4) f = x;
                                    else if constexpr (sizeof(KT) == 2) f = bf16_bits_to_float(x);
                                    else f = (x & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
                                    if ((__float_as_uint(f) & 0x7f800000u) != 0x7f800000u) continue;
#pragma unroll
                                    for (int b = 0; b < DB; ++b)
#pragma unroll
                                        for (int i = 0; i < 4; ++i)
                                            if (16 * b == d && i == j) acc[t][b][i] += pe * f;
                                }
                            }
                        }
                    }
                }
            }
        }
    };

    // pages whose keys everybody sees; then those that hold nodes
    const int plain = min(it.prefix / kPage, page1);
    int page = page0 + 2 * wave;
    for (; page + 2 <= plain; page += 2 * kTrWaves) step(page, std::false_type{});
    for (; page < page1; page += 2 * kTrWaves) step(page, std::true_type{});

    // the waves' states meet, one block of 16 rows after the other
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float sum = pair32_sum(pair16_sum(l[t]));
        // (the four lane groups of a column hold the same reference: it is raised from the column's maximum)
        if (lane < 16) { mm[wave][16 * t + n] = m[t]; ml[wave][16 * t + n] = sum; }
    }
    const float vscale = sizeof(KT) == 1 ? a.v_scale[it.g] : 1.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (first_row + 16 * t >= it.node_rows) break;         // the same for the whole workgroup
        __syncthreads();
#pragma unroll
        for (int b = 0; b < DB; ++b) mo[wave][n][4 * b + r] = acc[t][b];
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += 64 * kTrWaves) {
            const int col = i / (D / 4), d4 = i % (D / 4), row = first_row + 16 * t + col;
            if (row >= it.node_rows) continue;
            float top = mm[0][16 * t + col];
#pragma unroll
            for (int w = 1; w < kTrWaves; ++w) top = fmaxf(top, mm[w][16 * t + col]);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kTrWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(mm[w][16 * t + col] - top);
                if (ml[w][16 * t + col] == 0.0f) continue;     // (a wave without a key of this column)
                o += mo[w][col][d4] * f;
                sum += ml[w][16 * t + col] * f;
            }
            const int nd = row / G;
            if (it.parts == 1) {
                const float inv = tr_inverse(a, sum, it.prefix, it.n_nodes, it.row0, nd) * vscale;
                tr_store_out<KT>(a, ((int64_t)(it.row0 + nd) * Hq + it.g * G + row % G) * D + 4 * d4, o * inv);
            } else {
                const int64_t at = it.part_row0 + ((int64_t)it.g * it.parts + it.part) * it.node_rows + row;
                *(f32x4*)(a.part_o + at * D + 4 * d4) = o;
                if (d4 == 0) *(f32x2*)(a.part_ml + 2 * at) = f32x2{top, sum};
            }
        }
    }
}

// Rows whose scan was cut: D / 4 threads per row add up its parts in order.
template <typename KT, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, TreeSeqs s, int n_rows)
{
    constexpr int TPR = D / 4;
    const int lane = threadIdx.x & 63;
    const int w = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, d4 = threadIdx.x % TPR;
    // (the rows of a workgroup may belong to several sequences: every lane looks for its own)
    int i = 0;
    for (int b = 1; b < s.n; ++b) i += s.seq[b].first_merge <= w ? 1 : 0;
    (void)lane;
    if (w >= n_rows) return;
    const TreeSeq q = s.seq[i];
    const int n_nodes = s.seq[i + 1].row0 - q.row0, rows = n_nodes * a.geo.G, k = w - q.first_merge, g = k / rows, row = k % rows;
    const int64_t at = q.part_row0 + (int64_t)g * q.parts * rows + row;
    float top = kNoKeyTr;
    for (int p = 0; p < q.parts; ++p) top = fmaxf(top, a.part_ml[2 * (at + (int64_t)p * rows)]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.0f;
    for (int p = 0; p < q.parts; ++p) {
        const f32x2 ml = *(const f32x2*)(a.part_ml + 2 * (at + (int64_t)p * rows));
        if (ml.y == 0.0f) continue;
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        o += *(const f32x4*)(a.part_o + (at + (int64_t)p * rows) * D + 4 * d4) * f;
        sum += ml.y * f;
    }
    const int nd = row / a.geo.G;
    const float inv = tr_inverse(a, sum, q.prefix, n_nodes, q.row0, nd) * (sizeof(KT) == 1 ? a.v_scale[g] : 1.0f);
    tr_store_out<KT>(a, ((int64_t)(q.row0 + nd) * a.geo.Hq + g * a.geo.G + row % a.geo.G) * D + 4 * d4, o * inv);
}

template <typename KT, int D>
static int launch_tree_d(const TreeArgs& a, const TreeSeqs& s, int64_t items, hipStream_t st, hipEvent_t done)
{
    const dim3 grid((unsigned)items), block(64 * kTrWaves);
    if (a.rows == 16) return launch_kernel(tree_kernel<KT, D, 1>, grid, block, st, done, a, s);
    if (a.rows == 32) return launch_kernel(tree_kernel<KT, D, 2>, grid, block, st, done, a, s);
    if constexpr (sizeof(KT) != 4)
        if (a.rows == 64) return launch_kernel(tree_kernel<KT, D, 4>, grid, block, st, done, a, s);
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
