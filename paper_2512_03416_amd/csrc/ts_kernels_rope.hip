// Rotary positions and the append in one launch; moving cache entries; reading them back as rows.
//
// All three only move data: what bounds them is memory, or, for a few tokens, the launch.
#include "ts_device.h"
#include "ts_launch.h"

namespace ts {

// (cos, sin) of 2 pi * pos * turns, times the scale.  The quarter of the turn is found in double precision -- a position of
// 10^6 keeps 2^-33 of a turn -- and what is left of it, at most pi / 4 to either side, goes through the functions' power
// series in single precision (up to y^9 and y^10: the next terms are below 2^-28).
__device__ __forceinline__ f32x2 rope_angle(double turns, int pos, float scale)
{
    const double t = turns * (double)pos * 4.0;
    const double whole = __builtin_rint(t);
    const float y = (float)(t - whole) * 1.57079632679489662f;
    // (the quarter modulo 4; a whole number beyond 2^31 keeps its low bits this way)
    const int quarter = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));
    const float z = y * y;
    const float s = __builtin_fmaf(y * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), y);
    const float c = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
    return f32x2{(quarter == 1 || quarter == 2 ? -cs : cs) * scale, (quarter & 2 ? -sn : sn) * scale};
}

// A pair turned; dims behind the rotated ones stay as they are (not times (1, 0): an infinity next door would make a NaN of it).
__device__ __forceinline__ f32x2 rotated(float x, float y, f32x2 c, bool turns)
{
    if (!turns) return f32x2{x, y};
    return f32x2{__builtin_fmaf(x, c.x, -(y * c.y)), __builtin_fmaf(y, c.x, x * c.y)};
}

// The sequence that page number u of the launch belongs to (a sequence without new tokens shares the number of the next one:
// the last match counts).
__device__ __forceinline__ int seq_of_page(const AppendSeqs& s, int u)
{
    const int lane = threadIdx.x & 63;
    int i = -1;
#pragma unroll
    for (int b = 0; b < kAppendSeqs; b += 64)
        i += __builtin_popcountll(__ballot(b + lane < s.n && s.seq[min(b + lane, kAppendSeqs - 1)].first_page <= u));
    return i;
}

// One page's share of a sequence's tokens: slots [lo, hi) hold rows row_slot0 + slot.
struct PageRun { int seq, page_idx, lo, hi, row_slot0; };
__device__ __forceinline__ PageRun page_run(const AppendSeqs& s, int u)
{
    const int i = seq_of_page(s, u);
    const AppendSeq q = s.seq[i];
    const int n = s.seq[i + 1].row0 - q.row0, page = (q.prefix >> 4) + u - q.first_page;
    return PageRun{i, page, max(q.prefix - page * kPage, 0), min(q.prefix + n - page * kPage, kPage), q.row0 + page * kPage - q.prefix};
}

template <typename T> __device__ __forceinline__ float load_float(const T* p)
{
    if constexpr (sizeof(T) == 4) return *(const float*)p;
    else return bf16_bits_to_float(*p);
}
template <typename T> __device__ __forceinline__ void store_float(T* p, float f)
{
    if constexpr (sizeof(T) == 4) *(float*)p = f;
    else *p = (uint16_t)float_to_bf16_bits(f);
}
// An element on its way into the cache.
template <typename CT> __device__ __forceinline__ CT to_cache(float f, float scale)
{
    if constexpr (sizeof(CT) == 4) return f;
    else if constexpr (sizeof(CT) == 2) return (CT)float_to_bf16_bits(f);
    else return (CT)float_to_e4m3_bits(f / scale);
}

// ST: element type of the new tokens (float, or uint16_t for bf16 bits), CT: of the cache.
// A workgroup takes one page's new tokens: of one KV head (K rotated, V, both into the cache), or of some query heads.
template <typename ST, typename CT, int D>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a, AppendSeqs s)
{
    constexpr int P = D / 2;
    __shared__ f32x2 turn[kPage][P];
    __shared__ float rows[kPage][D + 1];
    const int Hkv = a.geo.Hkv, Hq = a.geo.Hq;
    const int per = Hkv + a.q_slices;
    const int u = a.first_unit + (int)blockIdx.x / per, job = blockIdx.x % per;
    const PageRun r = page_run(s, u);
    const int tid = threadIdx.x, n_tok = r.hi - r.lo, row0 = r.row_slot0 + r.lo;
    const int half = a.rope.rot_dim / 2;
    for (int i = tid; i < n_tok * P; i += 256) {
        const int t = i / P, p = i % P;
        const int pos = a.positions ? a.positions[row0 + t] : r.page_idx * kPage + r.lo + t;
        if (p < half) turn[t][p] = rope_angle(a.rope.turns[p], pos, a.rope.scale);
    }
    // pair p of a head: its two dims
    const bool inter = a.rope.interleaved;
    auto dims = [&](int p, int& x, int& y) {
        if (inter || p >= half) { x = 2 * p; y = 2 * p + 1; }
        else { x = p; y = p + half; }
    };
    __syncthreads();
    if (job >= Hkv) {
        const int h0 = (job - Hkv) * a.heads_per_slice, h1 = min(h0 + a.heads_per_slice, Hq), nh = h1 - h0;
        for (int i = tid; i < n_tok * nh * P; i += 256) {
            const int p = i % P, h = h0 + i / P % nh, t = i / P / nh;
            const ST* q = (const ST*)a.q + (row0 + t) * a.q_stride + h * D;
            ST* o = (ST*)a.q_out + ((int64_t)(row0 + t) * Hq + h) * D;
            int x, y;
            dims(p, x, y);
            const f32x2 v = rotated(load_float(q + x), load_float(q + y), turn[t][p], p < half);
            store_float(o + x, v.x);
            store_float(o + y, v.y);
        }
        return;
    }
    const int g = job;
    const int64_t tile = tile_elem_base(a.block_table[(int64_t)r.seq * a.geo.max_pages + r.page_idx], Hkv, g, D);
    constexpr int X = 16 / (int)sizeof(CT);
    CT* kt = (CT*)a.k_cache + tile;
    CT* vt = (CT*)a.v_cache + tile;
    const float ks = sizeof(CT) == 1 ? a.k_scale[g] : 1.f, vs = sizeof(CT) == 1 ? a.v_scale[g] : 1.f;
    for (int i = tid; i < n_tok * P; i += 256) {
        const int p = i % P, t = i / P, slot = r.lo + t;
        const ST* k = (const ST*)a.k + (row0 + t) * a.k_stride + g * D;
        int x, y;
        dims(p, x, y);
        const f32x2 v = rotated(load_float(k + x), load_float(k + y), turn[t][p], p < half);
        kt[(x / X) * (kPage * X) + slot * X + x % X] = to_cache<CT>(v.x, ks);
        kt[(y / X) * (kPage * X) + slot * X + y % X] = to_cache<CT>(v.y, ks);
    }
    for (int i = tid; i < n_tok * D; i += 256) {
        const int t = i / D, d = i % D;
        rows[t][d] = load_float((const ST*)a.v + (row0 + t) * a.v_stride + g * D + d);
    }
    __syncthreads();
    for (int i = tid; i < n_tok * D; i += 256) {
        const int t = i % n_tok, d = i / n_tok;
        vt[d * kPage + r.lo + t] = to_cache<CT>(rows[t][d], vs);
    }
}

template <typename ST, typename CT>
static int launch_rope_d(const RopeArgs& a, const AppendSeqs& s, int64_t blocks, hipStream_t st, hipEvent_t done)
{
    const dim3 grid((unsigned)blocks);
    if (a.geo.D == 128) return launch_kernel(rope_append_kernel<ST, CT, 128>, grid, dim3(256), st, done, a, s);
    return launch_kernel(rope_append_kernel<ST, CT, 64>, grid, dim3(256), st, done, a, s);
}

int launch_rope_append(const RopeArgs& a, const AppendSeqs& s, int32_t units, void* stream, void* done)
{
    if (a.geo.D != 128 && a.geo.D != 64) return (int)hipErrorInvalidValue;
    RopeArgs part = a;
    const int per = a.geo.Hkv + a.q_slices;
    const int64_t most = kMaxWorkgroups / per;
    if (most < 1) return (int)hipErrorInvalidValue;
    for (int64_t u = 0; u < units; u += most) {
        const int64_t n = units - u < most ? units - u : most;
        part.first_unit = (int32_t)u;
        hipStream_t st = (hipStream_t)stream;
        hipEvent_t ev = u + n < units ? nullptr : (hipEvent_t)done;
        int e;
        if (a.geo.q_dtype == TS_F32) e = launch_rope_d<float, float>(part, s, n * per, st, ev);
        else if (a.geo.kv_dtype == TS_BF16) e = launch_rope_d<uint16_t, uint16_t>(part, s, n * per, st, ev);
        else e = launch_rope_d<uint16_t, uint8_t>(part, s, n * per, st, ev);
        if (e != (int)hipSuccess) return e;
    }
    return (int)hipSuccess;
}

// Reading back: a workgroup takes one page of one KV head through LDS.
template <typename CT, typename OT, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a, AppendSeqs s)
{
    const int Hkv = a.geo.Hkv;
    const int u = a.first_unit + (int)blockIdx.x / Hkv, g = blockIdx.x % Hkv;
    const PageRun r = page_run(s, u);
    const int64_t tile = tile_elem_base(a.block_table[(int64_t)r.seq * a.geo.max_pages + r.page_idx], Hkv, g, D);
    constexpr int X = 16 / (int)sizeof(CT);
    const CT* kt = (const CT*)a.k_cache + tile;
    const CT* vt = (const CT*)a.v_cache + tile;
    const int n_tok = r.hi - r.lo;
    auto widen = [](CT c, float scale) {
        if constexpr (sizeof(CT) == 4) return (float)c;
        else if constexpr (sizeof(CT) == 2) return bf16_bits_to_float(c);
        else return e4m3_bits_to_float(c) * scale;
    };
    for (int which = 0; which < 2; ++which) {
        OT* out = (OT*)(which ? a.v_out : a.k_out);
        if (!out) continue;
        const float scale = sizeof(CT) == 1 ? (which ? a.v_scale : a.k_scale)[g] : 1.f;
        for (int i = threadIdx.x; i < n_tok * D; i += 256) {
            const int t = i / D, d = i % D, slot = r.lo + t;
            const CT c = which ? vt[d * kPage + slot] : kt[(d / X) * (kPage * X) + slot * X + d % X];
            store_float(out + ((int64_t)(r.row_slot0 + slot) * Hkv + g) * D + d, widen(c, scale));
        }
    }
}

int launch_kv_read(const ReadArgs& a, const AppendSeqs& s, int32_t units, void* stream, void* done)
{
    if (a.geo.D != 128 && a.geo.D != 64) return (int)hipErrorInvalidValue;
    ReadArgs part = a;
    const int64_t most = kMaxWorkgroups / a.geo.Hkv;
    if (most < 1) return (int)hipErrorInvalidValue;
    const bool d128 = a.geo.D == 128;
    for (int64_t u = 0; u < units; u += most) {
        const int64_t n = units - u < most ? units - u : most;
        part.first_unit = (int32_t)u;
        hipStream_t st = (hipStream_t)stream;
        hipEvent_t ev = u + n < units ? nullptr : (hipEvent_t)done;
        const dim3 grid((unsigned)(n * a.geo.Hkv)), block(256);
        int e;
        if (a.geo.q_dtype == TS_F32)
            e = d128 ? launch_kernel(kv_read_kernel<float, float, 128>, grid, block, st, ev, part, s) : launch_kernel(kv_read_kernel<float, float, 64>, grid, block, st, ev, part, s);
        else if (a.geo.kv_dtype == TS_BF16)
            e = d128 ? launch_kernel(kv_read_kernel<uint16_t, uint16_t, 128>, grid, block, st, ev, part, s) : launch_kernel(kv_read_kernel<uint16_t, uint16_t, 64>, grid, block, st, ev, part, s);
        else
            e = d128 ? launch_kernel(kv_read_kernel<uint8_t, uint16_t, 128>, grid, block, st, ev, part, s) : launch_kernel(kv_read_kernel<uint8_t, uint16_t, 64>, grid, block, st, ev, part, s);
        if (e != (int)hipSuccess) return e;
    }
    return (int)hipSuccess;
}

// Moving entries: a workgroup takes one sequence's pairs for one KV head.  Everything is read into LDS before anything is
// written, so the pairs may overlap and chain in any way.  ET: an integer of the element's size.
template <typename ET, int D>
__global__ __launch_bounds__(256) void kv_move_kernel(MoveArgs a, MoveSeqs s)
{
    __shared__ int from[TS_MAX_MOVES], to[TS_MAX_MOVES];
    __shared__ int64_t src_tile[TS_MAX_MOVES], dst_tile[TS_MAX_MOVES];
    __shared__ ET held[TS_MAX_MOVES][D + 4 / sizeof(ET)];
    const int Hkv = a.geo.Hkv;
    const int i = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
    const int first = s.first[i], n = s.first[i + 1] - first, len = s.ctx_len[i];
    const int tid = threadIdx.x;
    if (tid < n) { from[tid] = a.src[first + tid]; to[tid] = a.dst[first + tid]; }
    __syncthreads();
    if (tid < n) {
        bool keep = from[tid] >= 0 && from[tid] < len && to[tid] >= 0 && to[tid] < len;
        for (int j = tid + 1; keep && j < n; ++j)          // a later pair with the same destination, and a valid source, counts
            if (to[j] == to[tid] && from[j] >= 0 && from[j] < len) keep = false;
        const int32_t* bt = a.block_table + (int64_t)i * a.geo.max_pages;
        src_tile[tid] = keep ? tile_elem_base(bt[from[tid] >> 4], Hkv, g, D) : -1;
        dst_tile[tid] = keep ? tile_elem_base(bt[to[tid] >> 4], Hkv, g, D) : -1;
    }
    constexpr int X = 16 / (int)sizeof(ET);
    for (int which = 0; which < 2; ++which) {
        ET* c = (ET*)(which ? a.v_cache : a.k_cache);
        auto place = [&](int64_t tile, int slot, int d) { return tile + (which ? d * kPage + slot : (d / X) * (kPage * X) + slot * X + d % X); };
        __syncthreads();
        for (int e = tid; e < n * D; e += 256) {
            const int p = e / D, d = e % D;
            if (src_tile[p] >= 0) held[p][d] = c[place(src_tile[p], from[p] & 15, d)];
        }
        __syncthreads();
        for (int e = tid; e < n * D; e += 256) {
            const int p = e / D, d = e % D;
            if (src_tile[p] >= 0) c[place(dst_tile[p], to[p] & 15, d)] = held[p][d];
        }
    }
}

int launch_kv_move(const MoveArgs& a, const MoveSeqs& s, void* stream, void* done)
{
    if (s.n <= 0) return (int)hipSuccess;
    if (s.n > kMoveSeqs || (a.geo.D != 128 && a.geo.D != 64) || (int64_t)s.n * a.geo.Hkv > kMaxWorkgroups) return (int)hipErrorInvalidValue;
    const dim3 grid((unsigned)(s.n * a.geo.Hkv)), block(256);
    hipStream_t st = (hipStream_t)stream;
    hipEvent_t ev = (hipEvent_t)done;
    const bool d128 = a.geo.D == 128;
    if (a.geo.kv_dtype == TS_F32)
        return d128 ? launch_kernel(kv_move_kernel<uint32_t, 128>, grid, block, st, ev, a, s) : launch_kernel(kv_move_kernel<uint32_t, 64>, grid, block, st, ev, a, s);
    if (a.geo.kv_dtype == TS_BF16)
        return d128 ? launch_kernel(kv_move_kernel<uint16_t, 128>, grid, block, st, ev, a, s) : launch_kernel(kv_move_kernel<uint16_t, 64>, grid, block, st, ev, a, s);
    return d128 ? launch_kernel(kv_move_kernel<uint8_t, 128>, grid, block, st, ev, a, s) : launch_kernel(kv_move_kernel<uint8_t, 64>, grid, block, st, ev, a, s);
}

// Debug check of the page tables (option "validate_block_table"), as check_pages_kernel, with the lengths as arguments.
__global__ __launch_bounds__(256) void check_pages_few_kernel(PageCheck c, const int32_t* __restrict__ bt, int max_pages, int64_t num_pages,
                                                              int32_t* result)
{
    const int s = blockIdx.x;
    for (int p = threadIdx.x; p < c.pages[s]; p += blockDim.x) {
        const int32_t id = bt[(int64_t)(c.first + s) * max_pages + p];
        if (id < 0 || id >= num_pages) {
            if (atomicAdd(&result[0], 1) == 0) { result[1] = c.first + s; result[2] = p; }
        }
    }
}

int launch_check_pages(const PageCheck& p, const int32_t* block_table, int max_pages, int64_t num_pages, int32_t* result, void* stream)
{
    if (p.n <= 0) return (int)hipSuccess;
    if (p.n > kPageCheckSeqs) return (int)hipErrorInvalidValue;
    return launch_kernel(check_pages_few_kernel, dim3((unsigned)p.n), dim3(256), (hipStream_t)stream, nullptr, p, block_table, max_pages, num_pages, result);
}

}  // namespace ts
