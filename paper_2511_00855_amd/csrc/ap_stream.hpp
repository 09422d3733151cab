// Few queries against many rows: one pass over the rows, 16 of them at a time by each wave, straight from memory into the
// registers that the matrix instructions read; the queries lie in LDS in the order in which the lanes take them.  Bound by
// the bytes of the rows.  A row's 64 bytes from byte 64 s on are step s: lane l holds 16 of them, of row l % 16 from byte
// 64 s + 16 (l / 16) on, and of query l % 16 likewise.
#pragma once
#include "ap_gemm.hpp"

#ifdef __HIPCC__
typedef float ap_s_f32x4 __attribute__((ext_vector_type(4)));

// SUMS partial sums of an element: f32 products are added in as many chains, which are shorter (less rounding) and do not wait for each other.
struct ApStreamF32 {
    typedef ap_s_f32x4 Acc;
    static constexpr int SUMS = 4;
    static __device__ __forceinline__ void mul(ap_g_i32x4 a, ap_g_i32x4 b, Acc (&c)[SUMS]) {   // the four lanes of a row feed k = 4 (l / 16) + i
        const ap_s_f32x4 x = __builtin_bit_cast(ap_s_f32x4, a), y = __builtin_bit_cast(ap_s_f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; i++) c[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c[i], 0, 0, 0);
    }
    static __device__ __forceinline__ Acc sum(const Acc (&c)[SUMS]) { return (c[0] + c[1]) + (c[2] + c[3]); }
};
struct ApStreamBf16 {
    typedef ap_s_f32x4 Acc;
    static constexpr int SUMS = 1;
    static __device__ __forceinline__ void mul(ap_g_i32x4 a, ap_g_i32x4 b, Acc (&c)[SUMS]) {
        c[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ap_g_bf16x8, a), __builtin_bit_cast(ap_g_bf16x8, b), c[0], 0, 0, 0);
    }
    static __device__ __forceinline__ Acc sum(const Acc (&c)[SUMS]) { return c[0]; }
};
struct ApStreamI8 {
    typedef ap_g_i32x4 Acc;
    static constexpr int SUMS = 1;
    static __device__ __forceinline__ void mul(ap_g_i32x4 a, ap_g_i32x4 b, Acc (&c)[SUMS]) { c[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c[0], 0, 0, 0); }
    static __device__ __forceinline__ Acc sum(const Acc (&c)[SUMS]) { return c[0]; }
};

#define AP_STREAM_THREADS 512
#define AP_STREAM_LDS (150 * 1024)   // at most, for the queries: a workgroup has a compute unit to itself
#define AP_STREAM_AHEAD 8            // steps that a wave's loads are ahead

// One workgroup a compute unit at most, and of these as many as give every wave the same number of times 16 rows: 100,000 f32 rows of 768 columns
// take 53 us (5.8 TB/s) with 196 workgroups of 4 times, 62 with 256, of which a twentieth works alone at the end, and 82 with 261.
static inline int64_t ap_stream_blocks(int64_t n) {
    const int64_t tiles = (n + 15) / 16, waves = AP_STREAM_THREADS / 64, each = (tiles + 256 * waves - 1) / (256 * waves);
    return (tiles + each * waves - 1) / (each * waves);
}
static inline int64_t ap_stream_lds(int64_t rows, int64_t row_bytes) { return (rows + 15) / 16 * 16 * ((row_bytes + 63) / 64 * 64); }

// Where byte `at` of query q lies in LDS, of `nq` groups of 16 queries.
__device__ __forceinline__ int ap_stream_place(int q, int at, int nq) { return (((at >> 6) * nq + (q >> 4)) * 64 + ((at >> 4) & 3) * 16 + (q & 15)) * 16 + (at & 15); }

// Calls done(first row, acc, with) for every 16 rows that this wave takes; acc[g][r]: row first + 4 (lane / 16) + r, query 16 g + lane % 16.
// Rows past the last are the last row again.  `with` is what before(first row) has read ahead for them.
template <class OP, int NQ, class B, class F>
__device__ __forceinline__ void ap_stream(const char *rows, int64_t ld, int64_t n, int32_t row_bytes, const char *lds, int64_t wave, int64_t waves, B before, F done) {
    const int lane = threadIdx.x & 63, part = (lane >> 4) * 16, steps = (row_bytes + 63) / 64;
    for (int64_t first = wave * 16; first < n; first += waves * 16) {
        const int64_t row = first + (lane & 15);
        const char *p = rows + (row < n ? row : n - 1) * ld;
        const auto with = before(first);
        typename OP::Acc sums[NQ][OP::SUMS];
#pragma unroll
        for (int g = 0; g < NQ; g++)
#pragma unroll
            for (int i = 0; i < OP::SUMS; i++) sums[g][i] = typename OP::Acc{0, 0, 0, 0};
        for (int s0 = 0; s0 < steps; s0 += AP_STREAM_AHEAD) {
            ap_g_i32x4 a[AP_STREAM_AHEAD];
#pragma unroll
            for (int i = 0; i < AP_STREAM_AHEAD; i++) {
                const int at = (s0 + i) * 64 + part;
                a[i] = *reinterpret_cast<const ap_g_i32x4 *>(p + (at < row_bytes ? at : 0));
            }
            __builtin_amdgcn_sched_barrier(0);   // all of them on their way before the first is waited for
#pragma unroll
            for (int i = 0; i < AP_STREAM_AHEAD; i++) {
                const bool is = (s0 + i) * 64 + part < row_bytes;   // past the end of the row, and of what LDS holds: zeros
                const int s = s0 + i < steps ? s0 + i : 0;
#pragma unroll
                for (int j = 0; j < 4; j++) a[i][j] = is ? a[i][j] : 0;
#pragma unroll
                for (int g = 0; g < NQ; g++) OP::mul(a[i], *reinterpret_cast<const ap_g_i32x4 *>(lds + ((s * NQ + g) * 64 + lane) * 16), sums[g]);
            }
        }
        typename OP::Acc acc[NQ];
#pragma unroll
        for (int g = 0; g < NQ; g++) acc[g] = OP::sum(sums[g]);
        done(first, acc, with);
    }
}
#endif
