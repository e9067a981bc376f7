// Host side of the rotary append and of the attention of drafted trees: frequencies, masks, how a batch is cut.
#include <algorithm>
#include <cmath>
#include <functional>
#include <utility>

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

// A page's angles are worked out by every workgroup that takes a share of its heads: as many heads as leave the GPU full.  Decode rows
// are pages of one token, of which a workgroup takes more where there are many: 256 rows (64/8 heads of 128) 15.1 us in 2304 workgroups,
// 7.7 in 512.  Chunks of the same launch go by their own rule (258 rows next to a chunk of 22 tokens, 40/8 heads: 12.6 us; all by the rows' rule 32.6).
RopeSlices rope_slices(const ts_attn_desc& d, bool few, int64_t pages, int n_cu, bool with_q)
{
    const int64_t enough = (int64_t)n_cu * (few ? 2 : 8);
    RopeSlices r;
    r.kv_per_slice = few && pages * d.num_kv_heads > enough ? std::min(8, d.num_kv_heads) : 1;
    r.kv_slices = (d.num_kv_heads + r.kv_per_slice - 1) / r.kv_per_slice;
    int32_t heads = d.num_q_heads;
    while (heads > 8 && pages * (r.kv_slices + (d.num_q_heads + heads - 1) / heads) < enough) heads = (heads + 1) / 2;
    r.heads_per_slice = heads;
    r.q_slices = with_q ? (d.num_q_heads + heads - 1) / heads : 0;
    return r;
}

// Times of the tree kernel in us, measured, from which its rows per workgroup and its cuts are chosen.
struct TreeTimes {
    double page_alone;                 // a page (K and V of one KV head) of a workgroup that has the GPU to itself: bound by latency, in
                                       // proportion to the waves that share it (64-row workgroups take two pages at a time, 32-row ones four)
    double page_full;                  // the same with a workgroup in every place: bound by the matrix products, the softmax and the LDS
    double page_read;                  // a page read from HBM, by whichever of its groups of rows comes first
    int64_t places;                    // workgroups resident at once
    double item;                       // a workgroup's fixed share of its CU: 29 trees of 16 nodes over 10 tokens (64/8 heads) take 10.7 us in 232
                                       // workgroups of 128 rows, 14.9 in 464 of 64, 28 in 928 of 32
    double alone;                      // ... and its least time: 35 trees of 2-6 nodes over 0-5 tokens (40/8 heads, bf16), 280 workgroups, take 14.3 us
                                       // with 32 rows (256 places), 9.3 with 64
    double start, round;               // launch, page ids, queries, first copies, last stores; of a later workgroup in the same place
    double merge, merge_row;           // merge launch, and a partial row written and read again
};
static int tree_round(int rows) { return 2 * kTreeWaves * 32 / rows; }     // pages that a workgroup's waves take in turn
static bool tree_rows_fit(const ts_attn_desc& d, int rows)             // (fp32 with 128 dims: a ring for four waves' own keys exceeds the LDS)
{
    return rows > 32 || d.q_dtype != TS_F32 || d.head_dim == 64;
}
static TreeTimes tree_times(const ts_attn_desc& d, int rows, int n_cu)
{
    const int elem = d.kv_dtype == TS_F32 ? 4 : (d.kv_dtype == TS_BF16 ? 2 : 1);
    const int slot = tree_round(rows) * 2 * kPage * d.head_dim * elem;
    const double dims = d.head_dim / 128.0, math = d.q_dtype == TS_F32 ? 8.0 : 1.0;
    TreeTimes t;
    const int per_cu = std::max(1, std::min(2, 160 * 1024 / (slot * tree_ring_slots(slot, elem == 2))));
    t.places = (int64_t)n_cu * per_cu;
    t.page_alone = 0.36 * rows / 128 * (0.3 + 0.7 * dims) * math;
    // 32 trees of 64 nodes over 8 Ki tokens (64/8 heads of 128): bf16 556 us with 128 rows, 652 with 64, 1007 with 32 (one workgroup per CU, and
    // L2 reads of 17 TB/s), e4m3 546, 572, 642; 8 trees of 100-128 nodes over 2-9 Ki, e4m3: 209, 186, 198
    const bool e4m3 = elem == 1;
    t.page_full = (rows == 32 ? (per_cu == 1 ? 0.118 : (e4m3 ? 0.155 : 0.16)) : (rows == 64 ? (per_cu == 1 ? 0.2 : (e4m3 ? 0.288 : 0.335)) : (per_cu == 1 ? 0.36 : (e4m3 ? 0.525 : 0.49)))) * dims * math;
    t.page_read = 2.0 * kPage * d.head_dim * elem / 6.2e6;     // 6.2 TB/s
    t.item = 4.0;
    t.alone = 4.6;
    t.start = 5.0;
    t.round = 2.5;
    t.merge = 6.0;
    t.merge_row = 8.0 * d.head_dim / 4e6;
    return t;
}

// Rows per workgroup: 128 share every copied page four ways; with 32, each wave copies and scans keys of its own and waits for no other,
// which is faster wherever L2 and HBM keep up (4 trees of 7-26 nodes over 0.5-2.5 Ki tokens, 32/8 heads, 16.9 us with 32 rows, 19.5 with 128).
// Cuts: uncut, a scan writes no partial results, and the longest scans come first, so that a batch with a workgroup or more for every place
// comes out even by itself: 32 trees of 32-64 nodes over 1-8 Ki tokens (64/8 heads) took 287 us uncut, 312 in ranges of at most 384
// pages, 325 in ranges of 192.  Smaller batches are cut until the workgroups fill the places: 8 trees of 30 nodes over 4000 tokens
// (32/8 heads, 128 rows) 92 us uncut, 39 to 41 in ranges of 32 to 64 pages, 53 in ranges of 16 (most of it partial results).  Ranges of a sequence
// are of one length.  Both are taken from the times above.  On 29 of 30 batches of 16-bit queries the number of rows that they choose is within 8 % of the
// best one's time, on one 10 %; on 15 of fp32, whose page times are the 16-bit ones eight times over, within 16 %.
void plan_tree(const ts_attn_desc& d, const int32_t* q_lens, const int32_t* ctx_lens, int num_seqs, int n_cu, TreePlan* plan)
{
    const int32_t G = d.num_q_heads / d.num_kv_heads, Hkv = d.num_kv_heads;
    plan->seqs.clear();
    int64_t most = 0, row = 0;                                 // most rows of a sequence
    int32_t longest = 0;
    const double page_bytes = 2.0 * kPage * d.head_dim * (d.kv_dtype == TS_F32 ? 4 : (d.kv_dtype == TS_BF16 ? 2 : 1));
    double held = 0.0;                                         // bytes of all scans
    auto pages_of = [](const TreeSeq& s) { return (s.prefix + s.n_nodes + kPage - 1) / kPage; };
    for (int s = 0; s < num_seqs; ++s) {
        if (q_lens[s] > 0) {
            most = std::max<int64_t>(most, (int64_t)q_lens[s] * G);
            plan->seqs.push_back(TreeSeq{s, (int32_t)row, q_lens[s], ctx_lens[s] - q_lens[s], 0, 1, 0, 0, 0});
            const int32_t pages = pages_of(plan->seqs.back());
            longest = std::max(longest, pages);
            held += (double)pages * Hkv * page_bytes;
        }
        row += q_lens[s];
    }
    auto cut_to = [&](int32_t L, int round) {                  // ranges of at most L pages, a multiple of round
        for (TreeSeq& s : plan->seqs) {
            const int32_t pages = pages_of(s);
            s.parts = 1;
            s.part_pages = L;
            if (pages > L) {
                const int32_t parts = (pages + L - 1) / L;
                s.part_pages = ((pages + parts - 1) / parts + round - 1) / round * round;
                s.parts = (pages + s.part_pages - 1) / s.part_pages;
            }
        }
    };
    // What a group reads after another one comes from HBM again now and then, unless the batch fits the 256 MB behind the L2 caches
    // (14 trees of 9-25 nodes over 2-27 Ki tokens, 32/8 heads: 188 us with 32 rows, 160 with 128).
    const double again = held > 256e6 ? 0.15 : 0.05;
    std::vector<std::pair<int32_t, int32_t>> ranges;
    plan->rows = 128;
    int32_t best = 0;
    double best_time = 0.0;
    for (int rows_wg = 128; rows_wg >= 32; rows_wg /= 2) {
        if (!tree_rows_fit(d, rows_wg)) break;
        // (half of the rows would be empty everywhere: only where workgroups of half as many need more than one round of places)
        if (rows_wg > 32 && tree_rows_fit(d, rows_wg / 2) && most <= rows_wg / 2 &&
            (int64_t)plan->seqs.size() * Hkv <= tree_times(d, rows_wg / 2, n_cu).places) continue;
        const TreeTimes t = tree_times(d, rows_wg, n_cu);
        const int32_t round = tree_round(rows_wg), whole = (longest + round - 1) / round * round;
        auto groups_of = [&](const TreeSeq& s) { return tree_groups(s.n_nodes, G, rows_wg); };
        int64_t total = 0;                                     // pages of all scans' groups of rows
        double reads = 0.0;                                    // ... that come from HBM
        for (const TreeSeq& s : plan->seqs) {
            total += (int64_t)pages_of(s) * groups_of(s);
            reads += pages_of(s) * (1.0 + again * (groups_of(s) - 1));
        }
        for (int32_t L = whole; L >= round; L = std::min((L / 4 * 3 + round - 1) / round * round, L - round)) {
            int64_t items = 0, rows = 0;
            int32_t len = 0;
            cut_to(L, round);
            for (const TreeSeq& s : plan->seqs) {
                items += (int64_t)s.parts * Hkv * groups_of(s);
                len = std::max(len, std::min(s.part_pages, pages_of(s)));
                if (s.parts > 1) rows += (int64_t)s.parts * s.n_nodes * d.num_q_heads;
            }
            if (rows > kTreePartRows) break;                   // (shorter ranges have more of them)
            const double fill = std::min(1.0, (double)items / t.places), page = std::max(t.page_alone, t.page_full * fill);
            // the longest range, or all of them on the places they have (one behind the other, the shortest last, leaves a little
            // unevenness), or HBM
            double time = std::max(len * t.page_alone, (double)total * Hkv / std::min<int64_t>(items, t.places) * page);
            if (items > n_cu && items <= t.places) {           // the longest ranges share their CUs with those from number n_cu on
                ranges.clear();
                for (const TreeSeq& s : plan->seqs) ranges.push_back({std::min(s.part_pages, pages_of(s)), s.parts * Hkv * groups_of(s)});
                std::sort(ranges.begin(), ranges.end(), std::greater<>());
                int64_t before = 0;
                size_t k = 0;
                while (k + 1 < ranges.size() && before + ranges[k].second <= n_cu) before += ranges[k++].second;
                time = std::max(time, 0.85 * (len * t.page_alone + ranges[k].first * std::max(0.0, t.page_full - t.page_alone)));
            }
            if (items > t.places) time += 0.15 * page * total * Hkv / items + ((double)items / t.places - 1.0) * t.round;
            time = t.start + std::max({time, reads * Hkv * t.page_read, (double)items / n_cu * t.item, (double)((items + t.places - 1) / t.places) * t.alone});
            if (rows > 0) time += t.merge + rows * t.merge_row;
            if (best == 0 || time < best_time) { plan->rows = rows_wg; best = L; best_time = time; }
            if (items > 4 * t.places) break;
        }
    }
    cut_to(std::max(best, 1), tree_round(plan->rows));
    plan->part_rows = 0;
    for (TreeSeq& s : plan->seqs)
        if (s.parts > 1) {
            s.part_row0 = (int32_t)plan->part_rows;
            plan->part_rows += (int64_t)s.parts * s.n_nodes * d.num_q_heads;
        }
    std::stable_sort(plan->seqs.begin(), plan->seqs.end(), [&](const TreeSeq& x, const TreeSeq& y) { return std::min(x.part_pages, pages_of(x)) > std::min(y.part_pages, pages_of(y)); });
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
