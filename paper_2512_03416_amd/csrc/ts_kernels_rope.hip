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

// The sum over the lanes up to this one.
__device__ __forceinline__ int sum_up_to_lane(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);     // within rows of 16: from 1, 2, 4, 8 lanes before
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // rows 1 and 3: the last lane of the row before
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);    // rows 2 and 3: lane 31
    return x;
}

// The sequence and the page of it that job number u of the launch belongs to: slots [lo, hi) of the page hold rows row_slot0 + slot.  A page
// has `few` or `chunk` jobs, of which this is number `job`.
struct PageRun { int seq, page_idx, lo, hi, row_slot0, job; bool few; };
__device__ __forceinline__ PageRun page_run(const OpSeqs& s, int u, int chunk, int few)
{
    int b = 0, before = 0;                                 // the last 64 sequences that begin at u or earlier
#pragma unroll
    for (int k = 1; k < kOpSeqs / 64; ++k)
        if (s.first_page[k] <= u) { b = k; before = s.first_page[k]; }
    const int i = b * 64 + (int)(threadIdx.x & 63), at = min(i, s.n - 1);
    struct { int row0, prefix, next; } q;                  // (the next entry's row0: one load of 12 bytes)
    __builtin_memcpy(&q, &s.seq[at], sizeof q);
    const int len = i < s.n ? q.next - q.row0 : 0;
    const int pages = len > 0 ? ((q.prefix + len - 1) >> 4) - (q.prefix >> 4) + 1 : 0;
    const int per = rope_few(len, pages) ? few : chunk, jobs = pages * per;
    const int end = before + sum_up_to_lane(jobs);
    const int lane = __builtin_ctzll(__ballot(pages > 0 && end > u));      // (the first whose jobs reach beyond u)
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
    const int prefix = of(q.prefix), n = of(len), row0 = of(q.row0), j = u - of(end - jobs), of_page = of(per);
    const int page = (prefix >> 4) + j / of_page;
    return PageRun{b * 64 + lane, page, max(prefix - page * kPage, 0), min(prefix + n - page * kPage, kPage), row0 + page * kPage - prefix,
                   j % of_page, rope_few(n, of(pages))};
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
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a, OpSeqs s)
{
    constexpr int P = D / 2;
    __shared__ f32x2 turn[kPage][P];
    __shared__ ST rows[kPage][D + 4 / (int)sizeof(ST)];
    const int Hkv = a.geo.Hkv, Hq = a.geo.Hq;
    const PageRun r = page_run(s, a.first_unit + (int)blockIdx.x, a.chunk.jobs(), a.few.jobs());
    const RopeSlices sl = r.few ? a.few : a.chunk;
    const int job = r.job;
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
    if (job >= sl.kv_slices) {
        const int h0 = (job - sl.kv_slices) * sl.heads_per_slice, h1 = min(h0 + sl.heads_per_slice, Hq), nh = h1 - h0;
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
    const int64_t page = a.block_table[(int64_t)r.seq * a.geo.max_pages + r.page_idx];
    constexpr int X = 16 / (int)sizeof(CT);
    for (int g = job * sl.kv_per_slice; g < min((job + 1) * sl.kv_per_slice, Hkv); ++g) {
        const int64_t tile = tile_elem_base(page, Hkv, g, D);
        CT* kt = (CT*)a.k_cache + tile;
        CT* vt = (CT*)a.v_cache + tile;
        [[maybe_unused]] const float ks = sizeof(CT) == 1 ? a.k_scale[g] : 1.f, vs = sizeof(CT) == 1 ? a.v_scale[g] : 1.f;
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
            rows[t][d] = ((const ST*)a.v)[(row0 + t) * a.v_stride + g * D + d];
        }
        __syncthreads();
        for (int i = tid; i < n_tok * D; i += 256) {
            const int t = i % n_tok, d = i / n_tok;
            if constexpr (sizeof(CT) == 1) vt[d * kPage + r.lo + t] = to_cache<CT>(load_float(&rows[t][d]), vs);
            else vt[d * kPage + r.lo + t] = rows[t][d];                   // same element type: plain copy of the bits
        }
        __syncthreads();
    }
}

// The same in 16-byte pieces (bases and strides that allow it; with TS_ROPE_HALF rot_dim / 2 has to be whole pieces).  A thread takes a
// unit of X pairs (X = elements of a piece) of one token -- two pieces, which hold the pairs' two sides, or X pairs side by side -- and
// keeps their angles in registers while it goes through the heads; the angles are worked out once per workgroup, in LDS.
// What bounds it: memory.  34 188 tokens (64/8 heads of 128, bf16, 1.40 GB read and written): 284 us, 4.9 TB/s where a large copy
// reaches 4.7 to 5.1.  Stores carry the non-temporal hint (in two launches 296 us, 310 without; 2024 tokens of 40/8 heads 14.1 -> 12.8), loads
// do not: with it the large append took 283 us instead of 296, but inputs that the projection has just left in the caches come from memory (2024 tokens 18.4 us).
template <typename ST> struct RopePiece { static constexpr int X = 16 / (int)sizeof(ST); float v[X]; };
template <typename ST>
__device__ __forceinline__ RopePiece<ST> piece_of(uint4 w)
{
    RopePiece<ST> p;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(ST) == 4) p.v[i] = __uint_as_float(u[i]);
        else { p.v[2 * i] = __uint_as_float(u[i] << 16); p.v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
    return p;
}
__device__ __forceinline__ uint32_t pack_pair(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2)); }
template <typename ST>
__device__ __forceinline__ uint4 words_of(const RopePiece<ST>& p)
{
    if constexpr (sizeof(ST) == 4) return make_uint4(__float_as_uint(p.v[0]), __float_as_uint(p.v[1]), __float_as_uint(p.v[2]), __float_as_uint(p.v[3]));
    else return make_uint4(pack_pair(p.v[0], p.v[1]), pack_pair(p.v[2], p.v[3]), pack_pair(p.v[4], p.v[5]), pack_pair(p.v[6], p.v[7]));
}
// Four floats -> four e4m3 bytes, as float_to_e4m3_bits makes them (see encode_e4m3x16 in the append kernels: the hardware conversion
// agrees with it on every input but NaN once the value is clamped).
__device__ __forceinline__ uint32_t e4m3_word(float a, float b, float c, float d)
{
    const bool nan = !(a == a) | !(b == b) | !(c == c) | !(d == d);
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(a, -448.f, 448.f), __builtin_amdgcn_fmed3f(b, -448.f, 448.f), 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(c, -448.f, 448.f), __builtin_amdgcn_fmed3f(d, -448.f, 448.f), v, true);
    if (__any(nan))
        v = nan ? (int)(float_to_e4m3_bits(a) | float_to_e4m3_bits(b) << 8 | float_to_e4m3_bits(c) << 16 | float_to_e4m3_bits(d) << 24) : v;
    return (uint32_t)v;
}

template <typename ST, typename CT, int D>
__global__ __launch_bounds__(256) void rope_append_vec_kernel(RopeArgs a, OpSeqs s)
{
    constexpr int P = D / 2, X = 16 / (int)sizeof(ST), U = P / X;     // pairs of a head, of a unit; units of a head
    constexpr int kPad = D + X;                                       // LDS row of V: other banks for the next slot
    __shared__ __align__(16) f32x2 turn[kPage][P];
    __shared__ __align__(16) ST vrow[kPage][kPad];
    const int Hkv = a.geo.Hkv, Hq = a.geo.Hq;
    const PageRun r = page_run(s, a.first_unit + (int)blockIdx.x, a.chunk.jobs(), a.few.jobs());
    const RopeSlices sl = r.few ? a.few : a.chunk;
    const int job = r.job;
    const int tid = threadIdx.x, n_tok = r.hi - r.lo, row0 = r.row_slot0 + r.lo;
    const int half = a.rope.rot_dim / 2;
    const bool inter = a.rope.interleaved;
    // the thread's unit: token t, dims of its two pieces, its heads
    const int slots = n_tok * U, mine = tid % slots, first = tid / slots, step = 256 / slots;
    const int t = mine / U, u = mine % U;
    const bool paired = !inter && u * X < half;                       // two sides of X pairs; else 2 X dims side by side
    const int d0 = paired || inter ? (inter ? 2 : 1) * u * X : 2 * u * X, d1 = paired ? d0 + half : d0 + X;
    const bool is_q = job >= sl.kv_slices;
    const int h0 = is_q ? (job - sl.kv_slices) * sl.heads_per_slice : job * sl.kv_per_slice;
    const int h1 = is_q ? min(h0 + sl.heads_per_slice, Hq) : min(h0 + sl.kv_per_slice, Hkv);
    const ST* src = is_q ? (const ST*)a.q + (row0 + t) * a.q_stride : (const ST*)a.k + (row0 + t) * a.k_stride;
    const bool active = first < step;
    int h = h0 + first;
    uint4 w0 = {}, w1 = {};
    if (active && h < h1) {                                           // (on its way while the angles are worked out)
        w0 = *(const uint4*)(src + h * D + d0);
        w1 = *(const uint4*)(src + h * D + d1);
    }
    const bool one_head = h1 - h0 == 1;
    if (!is_q && one_head) {
        for (int i = tid; i < n_tok * (D / X); i += 256) {
            const int tv = i / (D / X), c = i % (D / X);
            *(uint4*)&vrow[r.lo + tv][c * X] = *(const uint4*)((const ST*)a.v + (row0 + tv) * a.v_stride + h0 * D + c * X);
        }
    }
    for (int i = tid; i < n_tok * P; i += 256) {
        const int ti = i / P, p = i % P;
        const int pos = a.positions ? a.positions[row0 + ti] : r.page_idx * kPage + r.lo + ti;
        if (p < half) turn[ti][p] = rope_angle(a.rope.turns[p], pos, a.rope.scale);
    }
    __syncthreads();
    f32x2 c[X];
    bool on[X];
#pragma unroll
    for (int e = 0; e < X; ++e) {
        on[e] = u * X + e < half;
        c[e] = turn[t][u * X + e];
    }
    auto rotate = [&](RopePiece<ST>& x, RopePiece<ST>& y) {
        if (!inter) {
#pragma unroll
            for (int e = 0; e < X; ++e) {
                const f32x2 v = rotated(x.v[e], y.v[e], c[e], on[e]);
                x.v[e] = v.x; y.v[e] = v.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < X; ++e) {
                RopePiece<ST>& z = e < X / 2 ? x : y;
                const int i = 2 * (e % (X / 2));
                const f32x2 v = rotated(z.v[i], z.v[i + 1], c[e], on[e]);
                z.v[i] = v.x; z.v[i + 1] = v.y;
            }
        }
    };
    if (is_q) {
        if (!active) return;
        for (; h < h1;) {
            RopePiece<ST> x = piece_of<ST>(w0), y = piece_of<ST>(w1);
            const int at = h;
            h += step;
            if (h < h1) {                                             // the next head's pieces
                w0 = *(const uint4*)(src + h * D + d0);
                w1 = *(const uint4*)(src + h * D + d1);
            }
            rotate(x, y);
            ST* o = (ST*)a.q_out + ((int64_t)(row0 + t) * Hq + at) * D;
            store_nt(o + d0, words_of(x));
            store_nt(o + d1, words_of(y));
        }
        return;
    }
    const int64_t page = a.block_table[(int64_t)r.seq * a.geo.max_pages + r.page_idx];
    if (active) {
        for (; h < h1;) {
            RopePiece<ST> x = piece_of<ST>(w0), y = piece_of<ST>(w1);
            const int g = h, slot = r.lo + t;
            h += step;
            if (h < h1) {
                w0 = *(const uint4*)(src + h * D + d0);
                w1 = *(const uint4*)(src + h * D + d1);
            }
            rotate(x, y);
            CT* kt = (CT*)a.k_cache + tile_elem_base(page, Hkv, g, D);
            auto store = [&](int d, const RopePiece<ST>& p) {
                if constexpr (sizeof(CT) == 1) {
                    const float ks = a.k_scale[g];
                    uint32_t w[X / 4];
#pragma unroll
                    for (int i = 0; i < X / 4; ++i) w[i] = e4m3_word(p.v[4 * i] / ks, p.v[4 * i + 1] / ks, p.v[4 * i + 2] / ks, p.v[4 * i + 3] / ks);
                    *(uint2*)(kt + (d / 16) * 256 + slot * 16 + d % 16) = make_uint2(w[0], w[X / 4 - 1]);
                } else store_nt(kt + (d / X) * (kPage * X) + slot * X, words_of(p));
            };
            store(d0, x);
            store(d1, y);
        }
    }
    if (!one_head) {                                                  // few tokens: V element by element, neighbouring threads neighbouring dims
        for (int i = tid; i < n_tok * (h1 - h0) * D; i += 256) {
            const int d = i % D, g = h0 + i / D % (h1 - h0), tv = i / D / (h1 - h0);
            const ST e = ((const ST*)a.v)[(row0 + tv) * a.v_stride + g * D + d];
            CT* vt = (CT*)a.v_cache + tile_elem_base(page, Hkv, g, D) + d * kPage + r.lo + tv;
            if constexpr (sizeof(CT) == 1) *vt = to_cache<CT>(load_float(&e), a.v_scale[g]);
            else *vt = e;
        }
        return;
    }
    const int g = h0;
    CT* vt = (CT*)a.v_cache + tile_elem_base(page, Hkv, g, D);
    // V: slots fastest in the tile.  A page that is filled whole leaves in 16-byte pieces
    if (n_tok == kPage) {
        constexpr int E = 16 / (int)sizeof(CT), PER = kPage / E;      // slots of a piece, pieces of a dim
        for (int i = tid; i < D * PER; i += 256) {
            const int d = i / PER, s0 = i % PER * E;
            if constexpr (sizeof(CT) == 1) {
                const float vs = a.v_scale[g];
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = e4m3_word(load_float(&vrow[4 * j][d]) / vs, load_float(&vrow[4 * j + 1][d]) / vs, load_float(&vrow[4 * j + 2][d]) / vs, load_float(&vrow[4 * j + 3][d]) / vs);
                store_nt(vt + d * kPage, make_uint4(w[0], w[1], w[2], w[3]));
            } else {
                ST e[E];
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] = vrow[s0 + j][d];
                uint4 w;
                __builtin_memcpy(&w, e, 16);
                store_nt(vt + d * kPage + s0, w);
            }
        }
    } else {
        for (int i = tid; i < n_tok * D; i += 256) {
            const int tv = i % n_tok, d = i / n_tok;
            const ST e = vrow[r.lo + tv][d];
            if constexpr (sizeof(CT) == 1) vt[d * kPage + r.lo + tv] = to_cache<CT>(load_float(&e), a.v_scale[g]);
            else vt[d * kPage + r.lo + tv] = e;
        }
    }
}

template <typename ST, typename CT>
static int launch_rope_d(const RopeArgs& a, const OpSeqs& s, int64_t blocks, hipStream_t st, hipEvent_t done)
{
    const dim3 grid((unsigned)blocks);
    const bool vec = a.vectors && (a.rope.interleaved || (a.rope.rot_dim / 2) % (16 / (int)sizeof(ST)) == 0);
    if (a.geo.D == 128) {
        if (vec) return launch_kernel(rope_append_vec_kernel<ST, CT, 128>, grid, dim3(256), st, done, a, s);
        return launch_kernel(rope_append_kernel<ST, CT, 128>, grid, dim3(256), st, done, a, s);
    }
    if (vec) return launch_kernel(rope_append_vec_kernel<ST, CT, 64>, grid, dim3(256), st, done, a, s);
    return launch_kernel(rope_append_kernel<ST, CT, 64>, grid, dim3(256), st, done, a, s);
}

int launch_rope_append(const RopeArgs& a, const OpSeqs& s, void* stream, void* done)
{
    if (a.geo.D != 128 && a.geo.D != 64) return (int)hipErrorInvalidValue;
    RopeArgs part = a;
    const int64_t units = s.n_jobs, most = kMaxWorkgroups;
    for (int64_t u = 0; u < units; u += most) {
        const int64_t n = units - u < most ? units - u : most;
        part.first_unit = (int32_t)u;
        hipStream_t st = (hipStream_t)stream;
        hipEvent_t ev = u + n < units ? nullptr : (hipEvent_t)done;
        int e;
        if (a.geo.q_dtype == TS_F32) e = launch_rope_d<float, float>(part, s, n, st, ev);
        else if (a.geo.kv_dtype == TS_BF16) e = launch_rope_d<uint16_t, uint16_t>(part, s, n, st, ev);
        else e = launch_rope_d<uint16_t, uint8_t>(part, s, n, st, ev);
        if (e != (int)hipSuccess) return e;
    }
    return (int)hipSuccess;
}

// Reading back: a workgroup takes one page of one KV head.  Element by element, for outputs on any address:
template <typename CT, typename OT, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a, OpSeqs s)
{
    const int Hkv = a.geo.Hkv;
    const int u = a.first_unit + (int)blockIdx.x / Hkv, g = blockIdx.x % Hkv;
    const PageRun r = page_run(s, u, 1, 1);
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

// In 16-byte pieces (16-byte aligned outputs).  K: a thread reads a piece of the tile -- 16 bytes of one token -- and writes it, neighbouring
// threads neighbouring dims, so that rows leave whole.  V: the tile's pieces (16 bytes of consecutive tokens of one dim) turn into rows in
// LDS.  What bounds it: memory.  108 951 tokens of an e4m3 cache (64/8 heads of 128, 0.22 GB read, 0.45 written): 129 us, 5.2 TB/s, 166
// without the non-temporal hint on the stores; loads with it 154.
template <typename CT, typename OT, int D>
__global__ __launch_bounds__(256) void kv_read_vec_kernel(ReadArgs a, OpSeqs s)
{
    constexpr int X = 16 / (int)sizeof(CT), C = D / X, PER = kPage / X;   // elements of a piece; K pieces of a token; V pieces of a dim
    constexpr int W = 16 / (int)sizeof(OT), kPad = D + W;
    constexpr int N = (kPage * C + 255) / 256;                            // pieces of a tile per thread
    __shared__ __align__(16) OT rows[kPage][kPad];
    const int Hkv = a.geo.Hkv, tid = threadIdx.x;
    // (workgroup i runs on die i % 8: a page's heads, whose rows lie next to each other, go to one die; over three caches in turn 156.2 ->
    // 153.4 us when this was put in.  The same for the append changes nothing, 294 us, or costs 2 %, drafted trees)
    const int w = (int)(blockIdx.x / 8), g = w % Hkv, u = a.first_unit + w / Hkv * 8 + (int)blockIdx.x % 8;
    if (u >= s.n_jobs) return;
    const PageRun r = page_run(s, u, 1, 1);
    const int64_t tile = tile_elem_base(a.block_table[(int64_t)r.seq * a.geo.max_pages + r.page_idx], Hkv, g, D);
    const CT* kt = (const CT*)a.k_cache + tile;
    const CT* vt = (const CT*)a.v_cache + tile;
    const int64_t out0 = ((int64_t)r.row_slot0 * Hkv + g) * D;            // (slot 0's row; only slots lo .. hi - 1 are touched)
    uint4 kw[N], vw[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = tid + 256 * j, slot = i / C, c = i % C;
        kw[j] = vw[j] = make_uint4(0, 0, 0, 0);
        if (a.k_out && slot >= r.lo && slot < r.hi) kw[j] = *(const uint4*)(kt + c * (kPage * X) + slot * X);
        if (a.v_out && i < D * PER) vw[j] = *(const uint4*)(vt + i * X);
    }
    auto value = [](uint4 w, int e, float scale) {                        // element e of a piece, e4m3 only
        const uint32_t u4[4] = {w.x, w.y, w.z, w.w};
        return e4m3_bits_to_float(u4[e / 4] >> (8 * (e % 4)) & 0xffu) * scale;
    };
    if (a.k_out) {
        OT* out = (OT*)a.k_out + out0;
        const float scale = sizeof(CT) == 1 ? a.k_scale[g] : 1.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = tid + 256 * j, slot = i / C, c = i % C;
            if (slot < r.lo || slot >= r.hi) continue;
            OT* o = out + (int64_t)slot * Hkv * D + c * X;
            if constexpr (sizeof(CT) == 1) {
                uint4 w[2];
                uint32_t* p = (uint32_t*)w;
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = pack_pair(value(kw[j], 2 * e, scale), value(kw[j], 2 * e + 1, scale));
                store_nt(o, w[0]);
                store_nt(o + 8, w[1]);
            } else store_nt(o, kw[j]);
        }
    }
    if (!a.v_out) return;
    const float scale = sizeof(CT) == 1 ? a.v_scale[g] : 1.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = tid + 256 * j;
        if (i >= D * PER) continue;
        const int d = i / PER, s0 = i % PER * X;
        if constexpr (sizeof(CT) == 1) {
#pragma unroll
            for (int e = 0; e < X; ++e) rows[s0 + e][d] = (OT)pack_pair(value(vw[j], e, scale), 0.f);
        } else {
            CT e[X];
            __builtin_memcpy(e, &vw[j], 16);
#pragma unroll
            for (int k = 0; k < X; ++k) rows[s0 + k][d] = e[k];
        }
    }
    __syncthreads();
    OT* out = (OT*)a.v_out + out0;
    for (int i = tid; i < kPage * (D / W); i += 256) {
        const int slot = i / (D / W), c = i % (D / W);
        if (slot >= r.lo && slot < r.hi) store_nt(out + (int64_t)slot * Hkv * D + c * W, *(const uint4*)&rows[slot][c * W]);
    }
}

template <typename CT, typename OT, int D>
static int launch_read_d(const ReadArgs& a, const OpSeqs& s, dim3 grid, hipStream_t st, hipEvent_t done)
{
    if (a.vectors) return launch_kernel(kv_read_vec_kernel<CT, OT, D>, grid, dim3(256), st, done, a, s);
    return launch_kernel(kv_read_kernel<CT, OT, D>, grid, dim3(256), st, done, a, s);
}

int launch_kv_read(const ReadArgs& a, const OpSeqs& s, void* stream, void* done)
{
    const int64_t units = s.n_jobs;
    if (a.geo.D != 128 && a.geo.D != 64) return (int)hipErrorInvalidValue;
    ReadArgs part = a;
    const int64_t most = kMaxWorkgroups / a.geo.Hkv / 8 * 8;
    if (most < 1) return (int)hipErrorInvalidValue;
    const bool d128 = a.geo.D == 128;
    for (int64_t u = 0; u < units; u += most) {
        int64_t n = units - u < most ? units - u : most;
        part.first_unit = (int32_t)u;
        hipStream_t st = (hipStream_t)stream;
        hipEvent_t ev = u + most < units ? nullptr : (hipEvent_t)done;
        if (a.vectors) n = (n + 7) / 8 * 8;
        const dim3 grid((unsigned)(n * a.geo.Hkv));
        int e;
        if (a.geo.q_dtype == TS_F32) e = d128 ? launch_read_d<float, float, 128>(part, s, grid, st, ev) : launch_read_d<float, float, 64>(part, s, grid, st, ev);
        else if (a.geo.kv_dtype == TS_BF16) e = d128 ? launch_read_d<uint16_t, uint16_t, 128>(part, s, grid, st, ev) : launch_read_d<uint16_t, uint16_t, 64>(part, s, grid, st, ev);
        else e = d128 ? launch_read_d<uint8_t, uint16_t, 128>(part, s, grid, st, ev) : launch_read_d<uint8_t, uint16_t, 64>(part, s, grid, st, ev);
        if (e != (int)hipSuccess) return e;
    }
    return (int)hipSuccess;
}

// Moving entries: a workgroup takes one sequence's pairs for one KV head.  Everything is read before anything is written, so the pairs
// may overlap and chain in any way.  ET: an integer of the element's size.  A path's few entries: what bounds it is the chain of
// dependent reads (pairs, page ids, entries), which K (in 16-byte pieces) and V go through together, and in large batches the lines of
// the V tiles, all of which an entry touches (one element per dim): 256 paths of 1-9 tokens over 8 KV heads of 128 dims, e4m3, 8.0 us (9.9
// with K and V one after the other; 8.7 with the pairs looked at by every wave, without an exchange through LDS).
template <typename ET, int D>
__global__ __launch_bounds__(256) void kv_move_kernel(MoveArgs a, MoveSeqs s)
{
    constexpr int X = 16 / (int)sizeof(ET), C = D / X;
    __shared__ int from[TS_MAX_MOVES], to[TS_MAX_MOVES];
    __shared__ int64_t src_tile[TS_MAX_MOVES], dst_tile[TS_MAX_MOVES];
    __shared__ __align__(16) uint4 held_k[TS_MAX_MOVES][C];
    __shared__ ET held_v[TS_MAX_MOVES][D];
    const int Hkv = a.geo.Hkv;
    const int i = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
    const int first = s.first[i], n = s.first[i + 1] - first, len = s.ctx_len[i];
    if (n == 0) return;
    const int tid = threadIdx.x;
    if (tid < n) {
        from[tid] = a.src[first + tid];
        to[tid] = a.dst[first + tid];
    }
    __syncthreads();
    if (tid < n) {
        const int f = from[tid], t = to[tid];
        bool keep = f >= 0 && f < len && t >= 0 && t < len;
        for (int j = tid + 1; keep && j < n; ++j)          // a later pair with the same destination, and a valid source, counts
            if (to[j] == t && from[j] >= 0 && from[j] < len) keep = false;
        keep = keep && f != t;
        const int32_t* bt = a.block_table + (int64_t)i * a.geo.max_pages;
        src_tile[tid] = keep ? tile_elem_base(bt[f >> 4], Hkv, g, D) : -1;
        dst_tile[tid] = keep ? tile_elem_base(bt[t >> 4], Hkv, g, D) : -1;
    }
    __syncthreads();
    ET* kc = (ET*)a.k_cache;
    ET* vc = (ET*)a.v_cache;
    for (int e = tid; e < n * C; e += 256) {
        const int p = e / C, c = e % C;
        if (src_tile[p] >= 0) held_k[p][c] = *(const uint4*)(kc + src_tile[p] + c * (kPage * X) + (from[p] & 15) * X);
    }
    for (int e = tid; e < n * D; e += 256) {
        const int p = e / D, d = e % D;
        if (src_tile[p] >= 0) held_v[p][d] = vc[src_tile[p] + d * kPage + (from[p] & 15)];
    }
    __syncthreads();
    for (int e = tid; e < n * C; e += 256) {
        const int p = e / C, c = e % C;
        if (src_tile[p] >= 0) *(uint4*)(kc + dst_tile[p] + c * (kPage * X) + (to[p] & 15) * X) = held_k[p][c];
    }
    for (int e = tid; e < n * D; e += 256) {
        const int p = e / D, d = e % D;
        if (src_tile[p] >= 0) vc[dst_tile[p] + d * kPage + (to[p] & 15)] = held_v[p][d];
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
    for (int p = c.from[s] + threadIdx.x; p < c.to[s]; p += blockDim.x) {
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
