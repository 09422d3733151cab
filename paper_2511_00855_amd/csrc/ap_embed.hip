// Dense rows out of token lists, and their gradients.
//
//   out_r = scale sum_{e in list r} w_e T[t_e]
//   dT[v] = scale sum_{e: t_e = v} w_e G[row(e)],   dw_e = scale <T[t_e], G[row(e)]>
//
// All three gather rows and are bound by how fast these come out of the caches and memory.  The gradient of the table is
// summed along the tokens' order: few entries find their equals by reading the list, many are sorted (a stable radix sort,
// so that a token's entries stay in their order) and cut into runs of one length, whatever the tokens' frequencies; a token
// whose entries lie in several runs gets the runs' sums added in their order.  No sum depends on which wave came first.
#include <algorithm>
#include "ap_common.hpp"

template <int DT> struct ApRow16;   // 16 bytes of a row as f32
template <> struct ApRow16<AP_F32> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(uint4 w, float *v) { v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w); }
};
template <> struct ApRow16<AP_BF16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(uint4 w, float *v) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
    }
};
// N consecutive values to a row of f32 or bf16 (rounded to nearest)
template <int OT, int N> __device__ __forceinline__ void put_row(void *row, int64_t col, const float *v) {
    if (OT == AP_F32) {
        float *p = static_cast<float *>(row) + col;
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        __bf16 *p = static_cast<__bf16 *>(row) + col;
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<b4 *>(p + i) = b4{(__bf16)v[i], (__bf16)v[i + 1], (__bf16)v[i + 2], (__bf16)v[i + 3]};
    }
}

struct ApEmbed {
    const char *table;             // or the gradient of the rows
    int64_t ld, vocab;             // ld in bytes
    int32_t dim, lanes;            // lanes: threads a row, a power of two up to 64; each has 16 bytes at a time
    const int32_t *tokens;
    const float *weights;
    const int64_t *indptr;
    int64_t n, rows;
    float scale;
    char *out;
};

#define AP_EMBED_AHEAD 8   // rows of the table that a thread has on their way

// `lanes` threads take one list and 16 bytes a thread of its columns at a time.  WAYS: as many waves share a list, each a run of its entries,
// and the first adds up the sums.
template <int DT, int OT, int WAYS>
__global__ __launch_bounds__(256) void k_embed(ApEmbed p) {
    constexpr int N = ApRow16<DT>::N;
    __shared__ float s_sum[WAYS > 1 ? 256 * N : 1];
    const int groups = p.dim / N, slabs = (groups + p.lanes - 1) / p.lanes;   // of a row
    const int per_wave = 64 / p.lanes, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t unit = WAYS > 1 ? (int64_t)blockIdx.x * per_wave + lane / p.lanes : ((int64_t)blockIdx.x * 4 + wave) * per_wave + lane / p.lanes;
    const int64_t row = unit / slabs;
    const int group = (int)(unit % slabs) * p.lanes + (lane & (p.lanes - 1));
    const bool mine = row < p.rows && group < groups;
    int64_t e = 0, end = 0;
    if (mine) {
        if (!p.indptr) { e = row; end = row + 1; }
        else if (ap_row_ok(p.indptr, row, p.n)) { e = p.indptr[row]; end = p.indptr[row + 1]; }
    }
    if (WAYS > 1) {
        const int64_t each = (end - e + WAYS - 1) / WAYS, b = e + wave * each;
        end = min(end, b + each);
        e = b;
    }
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; i++) sum[i] = 0.f;
    for (; e < end; e += AP_EMBED_AHEAD) {
        uint4 v[AP_EMBED_AHEAD];
        float w[AP_EMBED_AHEAD];
#pragma unroll
        for (int i = 0; i < AP_EMBED_AHEAD; i++) {
            const int64_t at = e + i < end ? e + i : end - 1;
            const int32_t t = p.tokens[at];
            const bool used = e + i < end && t >= 0 && t < p.vocab;
            w[i] = p.scale * (p.weights ? p.weights[at] : 1.f);
            v[i] = make_uint4(0, 0, 0, 0);
            if (used) v[i] = *reinterpret_cast<const uint4 *>(p.table + (int64_t)t * p.ld + group * 16);
            else w[i] = 0.f;   // whatever weight a slot has that names no row
        }
#pragma unroll
        for (int i = 0; i < AP_EMBED_AHEAD; i++) {
            float x[N];
            ApRow16<DT>::get(v[i], x);
#pragma unroll
            for (int j = 0; j < N; j++) sum[j] = fmaf(w[i], x[j], sum[j]);
        }
    }
    if (WAYS > 1) {
#pragma unroll
        for (int i = 0; i < N; i++) s_sum[i * 256 + threadIdx.x] = sum[i];
        __syncthreads();
        if (wave) return;
        for (int k = 1; k < WAYS; k++)
#pragma unroll
            for (int i = 0; i < N; i++) sum[i] += s_sum[i * 256 + k * 64 + lane];
    }
    if (mine) put_row<OT, N>(p.out + row * p.dim * (OT == AP_F32 ? 4 : 2), group * N, sum);
}

// ------------------------------------------------------------------ gradient of the table
__global__ __launch_bounds__(256) void k_embed_zero(uint4 *__restrict__ p, int64_t n) {
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = make_uint4(0, 0, 0, 0);
}

// The list that entry e lies in, -1 for none.
__device__ __forceinline__ int64_t row_of(const int64_t *indptr, int64_t rows, int64_t e) {
    if (!indptr) return e;
    int64_t lo = 0, hi = rows;   // indptr[lo] <= e, or lo = 0
    while (hi - lo > 1) { const int64_t m = (lo + hi) / 2; if (indptr[m] <= e) lo = m; else hi = m; }
    return indptr[lo] <= e && e < indptr[lo + 1] ? lo : -1;
}

// Few entries: a wave takes an entry and a slab of its columns; if no earlier entry names the same token it adds up all that do, in order.
template <int GT, int OT>
__global__ __launch_bounds__(256) void k_embed_grad_few(ApEmbed p) {
    constexpr int N = ApRow16<GT>::N;
    const int groups = p.dim / N, slabs = (groups + 63) / 64, lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t e0 = unit / slabs;
    if (e0 >= p.n) return;
    const int32_t t = p.tokens[e0];
    if (t < 0 || t >= p.vocab) return;
    for (int64_t e = 0; e < e0; e += 64)
        if (__any(e + lane < e0 && p.tokens[e + lane] == t)) return;
    const int group = (int)(unit % slabs) * 64 + lane;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; i++) sum[i] = 0.f;
    for (int64_t e = e0; e < p.n; e += 64) {
        const bool same = e + lane < p.n && p.tokens[e + lane] == t;
        int64_t row = -1;
        float w = 0.f;
        if (same) { row = row_of(p.indptr, p.rows, e + lane); w = p.scale * (p.weights ? p.weights[e + lane] : 1.f); }
        for (uint64_t m = __ballot(row >= 0); m; m &= m - 1) {
            const int k = __ffsll((unsigned long long)m) - 1;
            const int64_t r = (int64_t)__shfl((unsigned long long)row, k, 64);
            const float wk = __shfl(w, k, 64);
            if (group < groups) {
                float x[N];
                ApRow16<GT>::get(*reinterpret_cast<const uint4 *>(p.table + r * p.ld + group * 16), x);
#pragma unroll
                for (int j = 0; j < N; j++) sum[j] = fmaf(wk, x[j], sum[j]);
            }
        }
    }
    if (group < groups) put_row<OT, N>(p.out + (int64_t)t * p.dim * (OT == AP_F32 ? 4 : 2), group * N, sum);
}

// Stable radix sort of the entries by token: 4,096 entries a block, up to 9 bits a pass.  What names no row of the table sorts last.
#define AP_SORT_ITEMS 4096
#define AP_SORT_BINS 512
__device__ __forceinline__ uint32_t sort_key(const int32_t *tokens, int64_t vocab, int64_t i) { const int32_t t = tokens[i]; return t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab; }

// keys: NULL in the first pass, which takes the tokens
__global__ __launch_bounds__(256) void k_sort_count(const int32_t *__restrict__ tokens, int64_t vocab, const uint32_t *__restrict__ keys, int64_t n, int shift, int bits, uint32_t *__restrict__ hist,
                                                    int64_t blocks) {
    __shared__ uint32_t s_cnt[AP_SORT_BINS];
    for (int b = threadIdx.x; b < 1 << bits; b += 256) s_cnt[b] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * AP_SORT_ITEMS;
    for (int i = threadIdx.x; i < AP_SORT_ITEMS && i0 + i < n; i += 256) {
        const uint32_t k = keys ? keys[i0 + i] : sort_key(tokens, vocab, i0 + i);
        atomicAdd(&s_cnt[(k >> shift) & ((1 << bits) - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < 1 << bits; b += 256) hist[b * blocks + blockIdx.x] = s_cnt[b];
}
__global__ __launch_bounds__(1024) void k_sort_scan(uint32_t *__restrict__ h, int64_t count) {   // exclusive sums, by one block
    __shared__ uint32_t s_wave[16];
    uint32_t before = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t i0 = 0; i0 < count; i0 += 4096) {
        const int64_t at = i0 + threadIdx.x * 4;
        uint32_t v[4], own = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) { v[j] = at + j < count ? h[at + j] : 0; own += v[j]; }
        uint32_t sum = own;
        for (int o = 1; o < 64; o <<= 1) { const uint32_t t = __shfl_up(sum, o, 64); if (lane >= o) sum += t; }
        if (lane == 63) s_wave[wave] = sum;
        __syncthreads();
        uint32_t base = before, all = 0;
        for (int w = 0; w < 16; w++) { if (w < wave) base += s_wave[w]; all += s_wave[w]; }
        base += sum - own;
#pragma unroll
        for (int j = 0; j < 4; j++) { if (at + j < count) h[at + j] = base; base += v[j]; }
        before += all;
        __syncthreads();
    }
}
// The last pass also brings along what the sums need of an entry: its row (-1: none) and its weight.
__global__ __launch_bounds__(256) void k_sort_scatter(ApEmbed p, const uint32_t *__restrict__ keys, const int32_t *__restrict__ entries, int shift, int bits, const uint32_t *__restrict__ hist,
                                                      int64_t blocks, uint32_t *__restrict__ keys_out, int32_t *__restrict__ entries_out, int last, int32_t *__restrict__ row_out,
                                                      float *__restrict__ w_out) {
    __shared__ uint32_t s_at[4][AP_SORT_BINS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t mask = (1u << bits) - 1;
    for (int b = threadIdx.x; b < 4 * AP_SORT_BINS; b += 256) (&s_at[0][0])[b] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * AP_SORT_ITEMS + wave * (AP_SORT_ITEMS / 4);   // a wave's entries lie together
    for (int i = lane; i < AP_SORT_ITEMS / 4; i += 64)
        if (i0 + i < p.n) atomicAdd(&s_at[wave][((keys ? keys[i0 + i] : sort_key(p.tokens, p.vocab, i0 + i)) >> shift) & mask], 1u);
    __syncthreads();
    for (uint32_t b = threadIdx.x; b <= mask; b += 256) {
        uint32_t at = hist[b * blocks + blockIdx.x];
#pragma unroll
        for (int w = 0; w < 4; w++) { const uint32_t c = s_at[w][b]; s_at[w][b] = at; at += c; }
    }
    __syncthreads();
    for (int i = 0; i < AP_SORT_ITEMS / 4; i += 64) {
        if (i0 + i >= p.n) break;
        const bool is = i0 + i + lane < p.n;
        const uint32_t k = !is ? 0 : keys ? keys[i0 + i + lane] : sort_key(p.tokens, p.vocab, i0 + i + lane), d = (k >> shift) & mask;
        uint64_t same = __ballot(is);
        for (int b = 0; b < bits; b++) { const uint64_t m = __ballot((d >> b) & 1); same &= (d >> b) & 1 ? m : ~m; }
        uint32_t at = 0;
        if (is) at = s_at[wave][d] + __popcll(same & ((1ull << lane) - 1));
        ap_wave_sync();
        if (is && (same >> lane) == 1) s_at[wave][d] = at + 1;   // the last lane of its digit
        ap_wave_sync();
        if (is) {
            const int64_t e = entries ? entries[i0 + i + lane] : i0 + i + lane;
            keys_out[at] = k;
            if (!last) entries_out[at] = (int32_t)e;
            else { row_out[at] = (int32_t)row_of(p.indptr, p.rows, e); w_out[at] = p.scale * (p.weights ? p.weights[e] : 1.f); }
        }
    }
}

// A run of `run` sorted entries, a slab of 16 bytes a lane.  Tokens whose entries all lie in the run are written; the sum of a token that began
// in an earlier run goes to carry[run][0], that of one that goes on in the next to carry[run][1].
struct ApRuns { const uint32_t *keys; const int32_t *rows; const float *w; float *carry; int32_t run; };
template <int GT, int OT>
__global__ __launch_bounds__(256) void k_embed_grad_runs(ApEmbed p, ApRuns s) {
    constexpr int N = ApRow16<GT>::N;
    const int groups = p.dim / N, slabs = (groups + 63) / 64, lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), run = unit / slabs;
    const int64_t b = run * s.run, end = min(b + s.run, p.n);
    if (b >= p.n || s.keys[b] >= p.vocab) return;
    const int group = (int)(unit % slabs) * 64 + lane;
    const bool mine = group < groups;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; i++) sum[i] = 0.f;
    bool begun = b > 0 && s.keys[b - 1] == s.keys[b];   // the present token began in an earlier run
    for (int64_t e = b; e < end; e += 64) {
        const bool is = e + lane < end;
        const uint32_t key = is ? s.keys[e + lane] : 0xffffffffu;
        const uint32_t next = e + lane + 1 < p.n ? s.keys[min(e + lane + 1, p.n - 1)] : 0xffffffffu;
        const int32_t row = is ? s.rows[e + lane] : -1;
        const float w = is ? s.w[e + lane] : 0.f;
        const int count = (int)min((int64_t)64, end - e);
        for (int k0 = 0; k0 < count; k0 += 8) {
            uint4 v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const int32_t r = __builtin_amdgcn_readlane(row, k0 + k);   // -1 past the end of the run
                v[k] = make_uint4(0, 0, 0, 0);
                if (r >= 0 && mine) v[k] = *reinterpret_cast<const uint4 *>(p.table + r * p.ld + group * 16);
            }
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const uint32_t t = __builtin_amdgcn_readlane(key, k0 + k);
                if (t >= p.vocab) break;   // the end, or what names no row
                const float wk = __builtin_amdgcn_readlane(row, k0 + k) >= 0 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), k0 + k)) : 0.f;
                float x[N];
                ApRow16<GT>::get(v[k], x);
#pragma unroll
                for (int j = 0; j < N; j++) sum[j] = fmaf(wk, x[j], sum[j]);
                const bool ends = (uint32_t)__builtin_amdgcn_readlane(next, k0 + k) != t;
                const bool leaves = !ends && e + k0 + k + 1 == end;
                if (!ends && !leaves) continue;
                if (mine) {
                    if (begun) put_row<AP_F32, N>(s.carry + run * 2 * p.dim, group * N, sum);
                    else if (leaves) put_row<AP_F32, N>(s.carry + (run * 2 + 1) * p.dim, group * N, sum);
                    else put_row<OT, N>(p.out + (int64_t)t * p.dim * (OT == AP_F32 ? 4 : 2), group * N, sum);
                }
#pragma unroll
                for (int j = 0; j < N; j++) sum[j] = 0.f;
                begun = false;
            }
        }
    }
}
// One block for each run whose last token goes on: adds up the sums of the runs that it lies in.  16 waves share them.
template <int OT>
__global__ __launch_bounds__(1024) void k_embed_grad_join(ApEmbed p, ApRuns s, int64_t runs) {
    __shared__ float4 s_sum[16][64];
    const int64_t run = blockIdx.x, last = run * s.run + s.run - 1;   // the run's last entry
    if (last + 1 >= p.n) return;
    const uint32_t t = s.keys[last];
    if (t >= p.vocab || s.keys[last + 1] != t) return;                     // it ends here
    if (run > 0 && s.keys[run * s.run] == t && s.keys[run * s.run - 1] == t) return;   // it began earlier
    int64_t lo = run + 1, hi = runs;   // the runs that begin with t: run + 1 .. lo - 1
    while (lo < hi) { const int64_t m = (lo + hi) / 2; if (s.keys[m * s.run] == t) lo = m + 1; else hi = m; }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t each = (lo - run - 1 + 15) / 16, b = run + 1 + wave * each, end = min(lo, b + each);
    for (int c0 = blockIdx.y * 64; c0 * 4 < p.dim; c0 += gridDim.y * 64) {
        const int c = (c0 + lane) * 4;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < p.dim) {
            if (wave == 0) sum = *reinterpret_cast<const float4 *>(s.carry + (run * 2 + 1) * p.dim + c);
#pragma unroll 8
            for (int64_t r = b; r < end; r++) {
                const float4 v = *reinterpret_cast<const float4 *>(s.carry + r * 2 * p.dim + c);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
        }
        s_sum[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && c < p.dim) {
            for (int w = 1; w < 16; w++) { const float4 v = s_sum[w][lane]; sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w; }
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
            put_row<OT, 4>(p.out + (int64_t)t * p.dim * (OT == AP_F32 ? 4 : 2), c, v);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ gradient of the weights
// A wave takes 8 entries in a row.  g: the gradient of the rows.
template <int DT, int GT>
__global__ __launch_bounds__(256) void k_embed_grad_weights(ApEmbed p, const char *__restrict__ g, int64_t ldg, float *__restrict__ out) {
    const int lane = threadIdx.x & 63;
    const int64_t e0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 8;
    if (e0 >= p.n) return;
    const int64_t e = e0 + (lane & 7);
    int64_t row = -1;
    int32_t tok = -1;
    if (e < p.n) { tok = p.tokens[e]; row = tok >= 0 && tok < p.vocab ? row_of(p.indptr, p.rows, e) : -1; }
    float sum[8];
    const char *a8[8], *b8[8];   // the rows of each entry; NULL: it has none
#pragma unroll
    for (int k = 0; k < 8; k++) {
        const int32_t r = __builtin_amdgcn_readlane((int32_t)row, k), t = __builtin_amdgcn_readlane(tok, k);
        sum[k] = 0.f;
        a8[k] = r < 0 ? nullptr : p.table + (int64_t)t * p.ld;
        b8[k] = r < 0 ? nullptr : g + r * ldg;
    }
    for (int c = lane * 4; c < p.dim; c += 256) {
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const char *a = a8[k], *b = b8[k];
            if (!a) continue;
            float x[4], y[4];
            if (DT == AP_F32) { const float4 v = *reinterpret_cast<const float4 *>(a + c * 4); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
            else { const uint2 v = *reinterpret_cast<const uint2 *>(a + c * 2); x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u); x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u); }
            if (GT == AP_F32) { const float4 v = *reinterpret_cast<const float4 *>(b + c * 4); y[0] = v.x; y[1] = v.y; y[2] = v.z; y[3] = v.w; }
            else { const uint2 v = *reinterpret_cast<const uint2 *>(b + c * 2); y[0] = __uint_as_float(v.x << 16); y[1] = __uint_as_float(v.x & 0xffff0000u); y[2] = __uint_as_float(v.y << 16); y[3] = __uint_as_float(v.y & 0xffff0000u); }
#pragma unroll
            for (int j = 0; j < 4; j++) sum[k] = fmaf(x[j], y[j], sum[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; k++) {
        const float v = ap_wave_sum(sum[k]) * p.scale;
        if (lane == k && e < p.n) out[e] = v;
    }
}

// ------------------------------------------------------------------ host side
static int64_t div_up(int64_t v, int64_t m) { return (v + m - 1) / m; }
static int check_matrix(const char *what, const void *p, int64_t ld, int32_t dim, int32_t dtype) {
    AP_REQUIRE(dtype == AP_F32 || dtype == AP_BF16, "%s: dtype = %d is not AP_F32/AP_BF16", what, dtype);
    AP_REQUIRE(p != nullptr, "%s is NULL", what);
    AP_REQUIRE(((uintptr_t)p & 15) == 0, "%s must be 16-byte aligned", what);
    const int group = dtype == AP_BF16 ? 8 : 4;
    AP_REQUIRE(dim >= group && dim % group == 0 && dim <= 8192, "%s: dim = %d must be a multiple of %d and at most 8192", what, dim, group);
    AP_REQUIRE(ld >= dim && ld % group == 0 && ld <= (1 << 20), "%s: %lld elements from row to row, must be a multiple of %d in [dim, 2^20]", what, (long long)ld, group);
    return AP_OK;
}
static int check_lists(const ap_lists *l, int64_t vocab) {
    AP_REQUIRE(l != nullptr, "lists is NULL");
    AP_REQUIRE(vocab >= 1 && vocab < (1ll << 30), "vocab = %lld must be in [1, 2^30)", (long long)vocab);
    AP_REQUIRE(l->rows >= 0 && l->rows < (1ll << 28) && l->n >= 0 && l->n < (1ll << 28), "rows = %lld and n = %lld must be in [0, 2^28)", (long long)l->rows, (long long)l->n);
    AP_REQUIRE(l->n == 0 || l->tokens, "tokens is NULL");
    AP_REQUIRE(l->indptr || l->rows == l->n, "without indptr every token is a row: rows = %lld, n = %lld", (long long)l->rows, (long long)l->n);
    return AP_OK;
}
static ApEmbed args_of(const void *table, int64_t ld, int32_t dtype, int64_t vocab, int32_t dim, const ap_lists *l, float scale, void *out) {
    return ApEmbed{static_cast<const char *>(table), ld * (dtype == AP_BF16 ? 2 : 4), vocab, dim, 64, l->tokens, l->weights, l->indptr, l->n, l->rows, scale, static_cast<char *>(out)};
}
#define AP_TYPES(a, b, CALL)                                              \
    do {                                                                  \
        if ((a) == AP_F32 && (b) == AP_F32) CALL(AP_F32, AP_F32);         \
        else if ((a) == AP_F32) CALL(AP_F32, AP_BF16);                    \
        else if ((b) == AP_F32) CALL(AP_BF16, AP_F32);                    \
        else CALL(AP_BF16, AP_BF16);                                      \
        AP_CHECK_HIP(hipGetLastError());                                  \
    } while (0)

extern "C" int ap_embed(const void *table, int64_t ld, int32_t dtype, int64_t vocab, int32_t dim, const ap_lists *lists, float scale, void *out, int32_t out_dtype, void *stream) {
    AP_TRY(check_lists(lists, vocab));
    AP_TRY(check_matrix("table", table, ld, dim, dtype));
    if (lists->rows == 0) return AP_OK;
    AP_TRY(check_matrix("out", out, dim, dim, out_dtype));
    hipStream_t st = static_cast<hipStream_t>(stream);
    ApEmbed p = args_of(table, ld, dtype, vocab, dim, lists, scale, out);
    const int groups = dim / (dtype == AP_BF16 ? 8 : 4);
    while (p.lanes / 2 >= groups) p.lanes /= 2;
    const int64_t units = lists->rows * div_up(groups, p.lanes), waves = div_up(units, 64 / p.lanes);
    // few waves with long lists: four share a list
    const bool share = waves < 4096 && lists->n / lists->rows >= 16;
    const int64_t blocks = share ? waves : div_up(waves, 4);
    AP_REQUIRE(blocks < (1ll << 23), "too many rows");
#define AP_EMBED(A, B)                                                                                                   \
    do {                                                                                                                 \
        if (share) hipLaunchKernelGGL((k_embed<A, B, 4>), dim3((unsigned)blocks), dim3(256), 0, st, p);                  \
        else hipLaunchKernelGGL((k_embed<A, B, 1>), dim3((unsigned)blocks), dim3(256), 0, st, p);                        \
    } while (0)
    AP_TYPES(dtype, out_dtype, AP_EMBED);
#undef AP_EMBED
    return AP_OK;
}

#define AP_EMBED_FEW 4096   // entries that find their equals by reading the list

struct GradWs {
    int64_t blocks, runs;
    int32_t run, passes, bits;
    uint32_t *keys[2], *hist;
    int32_t *entries[2], *rows;
    float *w, *carry;
    size_t lay(char *base, int64_t n, int64_t vocab, int32_t dim) {
        size_t at = 0;
        auto take = [&](int64_t count) { char *p = base ? base + at : nullptr; at += (size_t)div_up(count * 4, 256) * 256; return p; };
        int all = 1;
        while ((1ll << all) <= vocab) all++;   // keys 0 .. vocab
        passes = (int32_t)div_up(all, 9);
        bits = (int32_t)div_up(all, passes);
        blocks = div_up(n, AP_SORT_ITEMS);
        run = 64;
        while (run < 256 && n / run > 8192) run *= 2;
        runs = div_up(n, run);
        for (int i = 0; i < 2; i++) { keys[i] = (uint32_t *)take(n); entries[i] = (int32_t *)take(n); }
        hist = (uint32_t *)take(blocks << bits);
        rows = (int32_t *)take(n);
        w = (float *)take(n);
        carry = (float *)take(runs * 2 * dim);
        return at;
    }
};
static bool embed_few(int64_t n) { return n <= (g_ap_debug.embed_few ? g_ap_debug.embed_few - 1 : AP_EMBED_FEW); }

extern "C" int ap_embed_grad_bytes(int64_t n, int64_t vocab, int32_t dim, size_t *out) {
    AP_REQUIRE(out != nullptr, "out is NULL");
    AP_REQUIRE(n >= 0 && n < (1ll << 28) && vocab >= 1 && vocab < (1ll << 30) && dim >= 1 && dim <= 8192, "n, vocab or dim is out of range");
    GradWs ws;
    *out = embed_few(n) ? 0 : ws.lay(nullptr, n, vocab, dim);
    return AP_OK;
}

extern "C" int ap_embed_grad(const void *grad_out, int64_t ld, int32_t dtype, int32_t dim, const ap_lists *lists, int64_t vocab, float scale, void *grad_table, int32_t table_dtype,
                             void *workspace, size_t bytes, void *stream) {
    AP_TRY(check_lists(lists, vocab));
    AP_REQUIRE(dtype == AP_F32 || dtype == AP_BF16, "dtype = %d is not AP_F32/AP_BF16", dtype);
    if (lists->rows) AP_TRY(check_matrix("grad_out", grad_out, ld, dim, dtype));
    AP_TRY(check_matrix("grad_table", grad_table, dim, dim, table_dtype));
    GradWs ws;
    const size_t need = embed_few(lists->n) ? 0 : ws.lay(static_cast<char *>(workspace), lists->n, vocab, dim);
    AP_REQUIRE(bytes >= need && (workspace || need == 0), "workspace of %zu bytes, %zu are needed", bytes, need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t words = vocab * dim / (table_dtype == AP_BF16 ? 8 : 4);
    hipLaunchKernelGGL(k_embed_zero, dim3((unsigned)std::min<int64_t>(div_up(words, 256), 8192)), dim3(256), 0, st, static_cast<uint4 *>(grad_table), words);
    AP_CHECK_HIP(hipGetLastError());
    if (lists->n == 0 || lists->rows == 0) return AP_OK;
    ApEmbed p = args_of(grad_out, ld, dtype, vocab, dim, lists, scale, grad_table);
    const int64_t slabs = div_up(dim / (dtype == AP_BF16 ? 8 : 4), 64);
    if (embed_few(lists->n)) {
        const dim3 grid((unsigned)div_up(lists->n * slabs, 4));
#define AP_FEW(A, B) hipLaunchKernelGGL((k_embed_grad_few<A, B>), grid, dim3(256), 0, st, p)
        AP_TYPES(dtype, table_dtype, AP_FEW);
#undef AP_FEW
        return AP_OK;
    }
    for (int i = 0; i < ws.passes; i++) {
        const uint32_t *keys = i ? ws.keys[(i - 1) & 1] : nullptr;
        const int32_t *entries = i ? ws.entries[(i - 1) & 1] : nullptr;
        hipLaunchKernelGGL(k_sort_count, dim3((unsigned)ws.blocks), dim3(256), 0, st, lists->tokens, vocab, keys, lists->n, i * ws.bits, ws.bits, ws.hist, ws.blocks);
        hipLaunchKernelGGL(k_sort_scan, dim3(1), dim3(1024), 0, st, ws.hist, ws.blocks << ws.bits);
        hipLaunchKernelGGL(k_sort_scatter, dim3((unsigned)ws.blocks), dim3(256), 0, st, p, keys, entries, i * ws.bits, ws.bits, ws.hist, ws.blocks, ws.keys[i & 1], ws.entries[i & 1],
                           i + 1 == ws.passes, ws.rows, ws.w);
        AP_CHECK_HIP(hipGetLastError());
    }
    const ApRuns s{ws.keys[(ws.passes - 1) & 1], ws.rows, ws.w, ws.carry, ws.run};
    const dim3 grid((unsigned)div_up(ws.runs * slabs, 4)), joins((unsigned)ws.runs, (unsigned)std::max<int64_t>(1, std::min<int64_t>(div_up(dim, 256), (1ll << 21) / ws.runs)));   // below 2^31 threads
#define AP_RUNS(A, B) hipLaunchKernelGGL((k_embed_grad_runs<A, B>), grid, dim3(256), 0, st, p, s)
    AP_TYPES(dtype, table_dtype, AP_RUNS);
#undef AP_RUNS
    if (table_dtype == AP_F32) hipLaunchKernelGGL((k_embed_grad_join<AP_F32>), joins, dim3(1024), 0, st, p, s, ws.runs);
    else hipLaunchKernelGGL((k_embed_grad_join<AP_BF16>), joins, dim3(1024), 0, st, p, s, ws.runs);
    AP_CHECK_HIP(hipGetLastError());
    return AP_OK;
}

extern "C" int ap_embed_grad_weights(const void *grad_out, int64_t ldg, int32_t grad_dtype, const void *table, int64_t ld, int32_t dtype, int64_t vocab, int32_t dim, const ap_lists *lists,
                                     float scale, float *grad_weights, void *stream) {
    AP_TRY(check_lists(lists, vocab));
    if (lists->n == 0) return AP_OK;
    AP_TRY(check_matrix("table", table, ld, dim, dtype));
    if (lists->rows) AP_TRY(check_matrix("grad_out", grad_out, ldg, dim, grad_dtype));
    AP_REQUIRE(grad_weights != nullptr, "grad_weights is NULL");
    hipStream_t st = static_cast<hipStream_t>(stream);
    const ApEmbed p = args_of(table, ld, dtype, vocab, dim, lists, scale, nullptr);
    const char *g = static_cast<const char *>(grad_out);
    const int64_t ldb = ldg * (grad_dtype == AP_BF16 ? 2 : 4);
    if (lists->rows == 0) return ap_fill_u32(grad_weights, (size_t)lists->n, 0, st);
    const dim3 grid((unsigned)div_up(lists->n, 32));
#define AP_WEIGHTS(A, B) hipLaunchKernelGGL((k_embed_grad_weights<A, B>), grid, dim3(256), 0, st, p, g, ldb, grad_weights)
    AP_TYPES(dtype, grad_dtype, AP_WEIGHTS);
#undef AP_WEIGHTS
    return AP_OK;
}
