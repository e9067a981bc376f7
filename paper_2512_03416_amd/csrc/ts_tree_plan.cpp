// Host side of the rotary append and of the attention of drafted trees: frequencies, masks, how a batch is cut.
#include <algorithm>
#include <cmath>

#include "ts_internal.h"

namespace ts {

namespace {
constexpr double kTwoPi = 6.283185307179586476925;
}

int rope_frequencies(const ts_rope_desc* r, double* freq, double* scale, std::string* err)
{
    auto fail = [&](const char* msg) { if (err) *err = msg; return (int)TS_ERR_INVALID_ARG; };
    if (!r) return fail("rope description is NULL");
    if (r->rot_dim < 2 || r->rot_dim > 2 * kMaxPairs || r->rot_dim % 2) return fail("rot_dim must be even, 2 .. 128");
    if (r->layout != TS_ROPE_HALF && r->layout != TS_ROPE_INTERLEAVED) return fail("unknown rotary layout");
    if (r->scaling < TS_ROPE_NONE || r->scaling > TS_ROPE_TABLE) return fail("unknown rotary scaling");
    if (!(r->attn_scale >= 0.0) || !std::isfinite(r->attn_scale)) return fail("attn_scale must be 0 or positive");
    const int n = r->rot_dim / 2;
    double m = 1.0;
    if (r->scaling == TS_ROPE_TABLE) {
        if (!r->table) return fail("table is NULL");
        for (int i = 0; i < n; ++i)
            if (!std::isfinite(r->table[i])) return fail("table holds a value that is not finite");
        if (freq) std::copy(r->table, r->table + n, freq);
    } else {
        if (!(r->base > 1.0) || !std::isfinite(r->base)) return fail("base must be above 1");
        const bool scaled = r->scaling != TS_ROPE_NONE, ranged = r->scaling == TS_ROPE_YARN || r->scaling == TS_ROPE_WAVELENGTH;
        if (scaled && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return fail("factor must be at least 1");
        if (ranged && r->original_length <= 0) return fail("original_length must be positive");
        double low = r->low, high = r->high;
        if (ranged) {
            if (low == 0.0) low = 1.0;
            if (high == 0.0) high = r->scaling == TS_ROPE_YARN ? 32.0 : 4.0;
            if (!(low > 0.0) || !(high > low) || !std::isfinite(high)) return fail("need 0 < low < high");
        }
        double base = r->base;
        if (r->scaling == TS_ROPE_NTK && n > 1) base *= std::pow(r->factor, (double)r->rot_dim / (r->rot_dim - 2));
        double ramp_lo = 0.0, ramp_hi = 0.0;
        if (r->scaling == TS_ROPE_YARN) {
            auto pair_of = [&](double turns) { return r->rot_dim * std::log(r->original_length / (turns * kTwoPi)) / (2.0 * std::log(base)); };
            ramp_lo = std::max(std::floor(pair_of(high)), 0.0);
            ramp_hi = std::min(std::ceil(pair_of(low)), (double)r->rot_dim - 1.0);
            m = 1.0 + 0.1 * std::log(r->factor);
        }
        for (int i = 0; i < n; ++i) {
            const double b = std::pow(base, -2.0 * i / r->rot_dim);
            double f = b;
            if (r->scaling == TS_ROPE_LINEAR) f = b / r->factor;
            if (r->scaling == TS_ROPE_YARN) {
                const double ramp = std::min(std::max((i - ramp_lo) / std::max(ramp_hi - ramp_lo, 0.001), 0.0), 1.0);
                f = b * (1.0 - ramp) + b / r->factor * ramp;
            }
            if (r->scaling == TS_ROPE_WAVELENGTH) {
                const double keep = std::min(std::max((r->original_length * b / kTwoPi - low) / (high - low), 0.0), 1.0);
                f = b * keep + b / r->factor * (1.0 - keep);
            }
            if (freq) freq[i] = f;
        }
    }
    if (scale) *scale = r->attn_scale > 0.0 ? r->attn_scale : m;
    return TS_OK;
}

// A page's rotations are worked out by every workgroup that takes a share of its heads: as many heads as leave the GPU full.
int32_t rope_heads_per_slice(const ts_attn_desc& d, int64_t units, int n_cu)
{
    int32_t heads = d.num_q_heads;
    while (heads > 8 && units * (d.num_kv_heads + (d.num_q_heads + heads - 1) / heads) < (int64_t)n_cu * 8) heads = (heads + 1) / 2;
    return heads;
}

// A scan with less than a round of workgroups is cut along the keys, into pieces of at least kMinPages pages.
constexpr int32_t kMinPages = 16;

TreePlan plan_tree(const ts_attn_desc& d, const int32_t* q_lens, const int32_t* ctx_lens, int num_seqs, int n_cu)
{
    TreePlan p;
    const int32_t G = d.num_q_heads / d.num_kv_heads, Hkv = d.num_kv_heads;
    int64_t most = 0;
    int32_t longest = 0;
    for (int s = 0; s < num_seqs; ++s)
        if (q_lens[s] > 0) { most = std::max<int64_t>(most, (int64_t)q_lens[s] * G); longest = std::max(longest, ctx_lens[s]); }
    p.rows = most <= 32 && d.q_dtype != TS_F32 ? 32 : (most <= 64 ? 64 : 128);
    int64_t pages = 0;                                     // pages read, over the workgroups' groups of rows
    for (int s = 0; s < num_seqs; ++s)
        if (q_lens[s] > 0) pages += (int64_t)tree_groups(q_lens[s], G, p.rows) * ((ctx_lens[s] + kPage - 1) / kPage) * Hkv;
    const int64_t slots = (int64_t)n_cu * 2;
    int64_t part = std::max<int64_t>(kMinPages, (pages + slots - 1) / slots);
    const int64_t whole = (longest + kPage - 1) / kPage;
    for (;; part *= 2) {
        part = std::min<int64_t>((part + 7) / 8 * 8, (whole + 7) / 8 * 8);     // (whole rounds of the waves)
        p.part_pages = (int32_t)part;
        p.part_rows = p.items = 0;
        for (int s = 0; s < num_seqs; ++s) {
            if (q_lens[s] <= 0) continue;
            const int64_t n = tree_parts(ctx_lens[s], p.part_pages);
            p.items += n * Hkv * tree_groups(q_lens[s], G, p.rows);
            if (n > 1) p.part_rows += n * Hkv * G * q_lens[s];
        }
        if (p.part_rows <= kTreePartRows || part >= whole) return p;
    }
}

}  // namespace ts

extern "C" int ts_rope_frequencies(const ts_rope_desc* rope, double* freq, double* scale)
{
    return ts::rope_frequencies(rope, freq, scale, nullptr);
}

extern "C" int ts_tree_masks(const int32_t* parents, const int32_t* q_lens, int num_seqs, int mask_words, uint64_t* mask, int32_t* depth)
{
    if (num_seqs < 0 || (num_seqs > 0 && !q_lens)) return TS_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int s = 0; s < num_seqs; ++s) {
        if (q_lens[s] < 0) return TS_ERR_INVALID_ARG;
        if (mask && (int64_t)mask_words * 64 < q_lens[s]) return TS_ERR_INVALID_ARG;
        total += q_lens[s];
    }
    if (total > 0 && !parents) return TS_ERR_INVALID_ARG;
    int64_t row = 0;
    for (int s = 0; s < num_seqs; ++s) {                   // (checked as a whole before anything is written)
        for (int32_t i = 0; i < q_lens[s]; ++i)
            if (parents[row + i] < -1 || parents[row + i] >= i) return TS_ERR_INVALID_ARG;
        row += q_lens[s];
    }
    row = 0;
    for (int s = 0; s < num_seqs; ++s) {
        for (int32_t i = 0; i < q_lens[s]; ++i) {
            const int32_t parent = parents[row + i];
            if (depth) depth[row + i] = parent < 0 ? 0 : depth[row + parent] + 1;
            if (mask) {
                uint64_t* m = mask + (row + i) * mask_words;
                for (int w = 0; w < mask_words; ++w) m[w] = parent < 0 ? 0 : mask[(row + parent) * mask_words + w];
                m[i / 64] |= (uint64_t)1 << (i % 64);
            }
        }
        row += q_lens[s];
    }
    return TS_OK;
}
