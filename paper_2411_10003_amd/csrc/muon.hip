// The update of the experts' parameters: momentum, orthogonalised by Newton-Schulz products (the Muon rule), applied to the
// weights.  Per matrix (short side m, long side n):
//
//   M <- mu M + G,  U = G + mu M (nesterov) or M,  X = U / (|U|_F + eps)
//   steps times, X lying on its long side:  A = X X^T,  X <- a X + (b A + c A A) X
//   W <- (1 - lr wd) W - lr scale X
//
// All matrices of a call, of all its tensors, are one batch: they have the same two sides and lie on the long one here.
//
// Every X is Q X0 with Q a polynomial in A0 = X0 X0^T, so the steps can be taken on the short side: B = a + b A + c A A,  Q <- B Q,
// A <- B A B (all of them polynomials in A0: they commute and are symmetric, half of each product is the other half), and X = Q X0 at
// the end.  Five steps: 6 m^2 n + 14 m^3 operations, halves of symmetric products, where the form above takes 15 m^2 n + 5 m^3; as many at
// n = m, 0.58 of it at n = 4 m.  A carries the squares of the singular values, and what a rounding adds to those near zero grows by a^2 = 11.9 a
// step that goes on with the same A: after three steps (each, where the short side is 64 or less) A is formed again from X.  Off the
// factor that 64 bits give, 11 bits kept, 256 x 1024 of a falling spectrum: the form above 3.4e-3; all five steps on one A 1.2e-1; two, then
// three 1.5e-2; three, then two 3.5e-3.
//
// What X, A and the polynomial are kept in.  The products take 16-bit operands and add in fp32.  fp16, with its 11 bits, at the rate of
// bf16 with 8; its range is made up for by powers of two.  X is stored times S = 2^floor(log2 sqrt(mn)), at most 2^14, which brings the elements of the
// first, of Frobenius norm 1, near 1; its singular values stay below 1.3 with the usual coefficients and have to below 3.  A, whose
// eigenvalues are their squares, times 2^10, B, at most a, times 2^6, Q, at most a^3, times 2^3.  Of the 65504 that fp16 holds an element
// is then, singular values of 3 and a = 16 given, X 49152, A 9216, B 1024 and Q 32768 at most.
// What a rounding leaves outside the range of U, some 2^-12 of |X| in 11 bits, grows by a a step, 485 times in five.  Off the orthogonal factor it is
// 1.5e-3 of it for a dense spectrum, 5e-3 for one of a quarter of the rank with noise below it, and up to 0.15 / sqrt(r) for a rank r without: 0.15,
// 6e-2, 3e-2, 1.5e-2 at ranks 1, 4, 16, 64 (bf16: up to eight times that).  The factor changes a weight by a few per cent of it: short of the lowest
// ranks that is nothing that a bf16 weight resolves, and there it is a step of its rounding.
// fp32 weights do resolve it: for them every operand is two fp16 numbers, the second the rounding error of the first (22 bits), and a
// product is three, hi lo + lo hi + hi hi, segments of one contraction (2e-6 to 4e-6 off the factor, as fp32 throughout is; 3e-5 / sqrt(r) at rank r,
// where fp32 throughout leaves 1e-4).
#include "tile.h"

#include <cmath>
#include <type_traits>

namespace {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef float quad_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned oct_t __attribute__((ext_vector_type(4), aligned(2)));        // 8 numbers of 16 bits that begin anywhere

constexpr int MAX_SEGMENTS = 3;
constexpr int MAX_CUT = 512;                               // tiles of a launch that are cut: fewer than there are places for blocks

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const moe_f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
__device__ __forceinline__ u32x4 pack_f16x8(const float* v)
{
    return u32x4{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]), pack_f16x2(v[4], v[5]), pack_f16x2(v[6], v[7])};
}
__device__ __forceinline__ void unpack_f16x8(const u32x4& w, float* v)
{
    const f16x8 h = __builtin_bit_cast(f16x8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
}
// What the first number leaves of the value.
__device__ __forceinline__ u32x4 pack_rest(const float* v, const u32x4& first)
{
    float f[8], r[8];
    unpack_f16x8(first, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i] - f[i];
    return pack_f16x8(r);
}

// ---- momentum, and the sum of U^2 in parts ----------------------------------------------------------
// Bound by HBM: G read, M read and written.  Squares are added in 64 bits: fp32 ones of a gradient of 1e-25 or 1e25 are none.
struct Tensors {
    const float* grad[MUON_MAX_TENSORS];
    float* momentum[MUON_MAX_TENSORS];
    int transposed[MUON_MAX_TENSORS];                      // lies on its short side
};

__device__ __forceinline__ float direction(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m, g) : m; }

// Past the caches where gradients and momenta are more than they keep until the first X is formed from them (eight matrices of 2048 x 8192, 1.07
// GB of the two: the call 3265 -> 3228 us).
template <bool NT> __device__ __forceinline__ quad_t load_quad(const float* p)
{
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const quad_t*>(p));
    else return *reinterpret_cast<const quad_t*>(p);
}
constexpr size_t CACHE_BYTES = (size_t)256 << 20;

constexpr int MOMENTUM_UNROLL = 4;
template <bool NT>
__global__ __launch_bounds__(256) void momentum_kernel(const Tensors t, int count, size_t elements, int chunks, float mu, int nesterov,
                                                       double* __restrict__ partial, int* __restrict__ arrived)
{
    // the counters of the products' cut tiles, whatever the workspace held; from here on every use leaves them zero
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < MAX_CUT; i += 256) arrived[i] = 0;
    const int matrix = blockIdx.y, tensor = matrix / count;
    const size_t base = (size_t)(matrix % count) * elements;
    const float* __restrict__ G = t.grad[tensor] + base;
    float* __restrict__ M = t.momentum[tensor] + base;
    const size_t quads = elements / 4, step = (size_t)chunks * 256;
    double sum = 0.0;
    auto add = [&](float u) { sum = fma((double)u, (double)u, sum); };
    for (size_t q0 = (size_t)blockIdx.x * 256 + threadIdx.x; q0 < quads; q0 += step * MOMENTUM_UNROLL) {
        quad_t g[MOMENTUM_UNROLL], m[MOMENTUM_UNROLL];
#pragma unroll
        for (int i = 0; i < MOMENTUM_UNROLL; ++i) {
            const size_t q = q0 + i * step < quads ? q0 + i * step : quads - 1;      // past the end: the last ones again
            g[i] = load_quad<NT>(G + 4 * q);
            m[i] = load_quad<NT>(M + 4 * q);
        }
#pragma unroll
        for (int i = 0; i < MOMENTUM_UNROLL; ++i) {
            const size_t q = q0 + i * step;
            if (q >= quads) break;
#pragma unroll
            for (int k = 0; k < 4; ++k) { m[i][k] = fmaf(mu, m[i][k], g[i][k]); add(direction(g[i][k], m[i][k], mu, nesterov)); }
            if constexpr (NT) __builtin_nontemporal_store(m[i], reinterpret_cast<quad_t*>(M + 4 * q));
            else *reinterpret_cast<quad_t*>(M + 4 * q) = m[i];
        }
    }
    if (blockIdx.x == 0 && threadIdx.x < elements % 4) {
        const size_t i = quads * 4 + threadIdx.x;
        const float g = G[i], m = fmaf(mu, M[i], g);
        M[i] = m;
        add(direction(g, m, mu, nesterov));
    }
    __shared__ double words[4];
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) partial[(size_t)matrix * chunks + blockIdx.x] = (words[0] + words[1]) + (words[2] + words[3]);
}

// ---- the first X, in fp16, on its long side, with zeros up to multiples of 64 ---------------------------
// U is formed again from G and M: half of what writing and reading it would move.  64 rows x 256 columns of X per block, by way of LDS
// where the tensor lies on its short side.
constexpr int START_COLS = 256;
template <bool NT>
__global__ __launch_bounds__(256) void start_kernel(const Tensors t, int count, int m, int n, int mp, int np, int chunks, float mu, int nesterov,
                                                    float eps, float S, const double* __restrict__ partial, f16* __restrict__ X, f16* __restrict__ X_rest)
{
    __shared__ double words[4];
    __shared__ float tile[64][65];
    const int matrix = blockIdx.z, tensor = matrix / count, lane = threadIdx.x & 63;
    const size_t base = (size_t)(matrix % count) * ((size_t)m * n);
    const float* __restrict__ G = t.grad[tensor] + base;
    const float* __restrict__ M = t.momentum[tensor] + base;
    double sum = threadIdx.x < chunks ? partial[(size_t)matrix * chunks + threadIdx.x] : 0.0;
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) words[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double factor = (double)S / (sqrt((words[0] + words[1]) + (words[2] + words[3])) + (double)eps);
    const bool tall = t.transposed[tensor] != 0;
    const int r0 = blockIdx.y * 64, src_cols = tall ? m : n, src_rows = tall ? n : m;
    for (int c0 = blockIdx.x * START_COLS; c0 < min(np, (int)(blockIdx.x + 1) * START_COLS); c0 += 64) {
        const int sr0 = tall ? c0 : r0, sc0 = tall ? r0 : c0;
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
            const int r = pass * 16 + threadIdx.x / 16, c = threadIdx.x % 16 * 4;
            float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (sr0 + r < src_rows && sc0 + c < src_cols) {
                const size_t at = (size_t)(sr0 + r) * src_cols + sc0 + c;
                const int there = min(4, src_cols - sc0 - c);
                float gv[4] = {0.0f, 0.0f, 0.0f, 0.0f}, mv[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (there == 4) {
                    const quad_t mq = load_quad<NT>(M + at);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mv[k] = mq[k];
                    if (nesterov) {
                        const quad_t gq = load_quad<NT>(G + at);
#pragma unroll
                        for (int k = 0; k < 4; ++k) gv[k] = gq[k];
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < there) { mv[k] = M[at + k]; gv[k] = nesterov ? G[at + k] : 0.0f; }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k] = (float)((double)direction(gv[k], mv[k], mu, nesterov) * factor);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (tall) tile[c + k][r] = u[k];
                else tile[r][c + k] = u[k];
            }
        }
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            const int r = pass * 32 + threadIdx.x / 8, c = threadIdx.x % 8 * 8;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = tile[r][c + k];
            const size_t at = ((size_t)matrix * mp + r0 + r) * np + c0 + c;
            const u32x4 first = pack_f16x8(v);
            *reinterpret_cast<u32x4*>(X + at) = first;
            if (X_rest) *reinterpret_cast<u32x4*>(X_rest + at) = pack_rest(v, first);
        }
    }
}

// ---- the products --------------------------------------------------------------------------------------
// out = alpha sum_k A[i][k] B[k][j] + beta D + diag I, per matrix of the batch, B symmetric or given by its rows as B^T:
//   ROWS  B is read along its rows' contraction (A B^T: X X^T, and products of symmetric matrices)
//   COLS  B lies with the contraction as its slow index (the polynomial times X)
// Sides and contractions are multiples of 64 (of zeros past the matrix), in tiles of 256 or 128 that may hang over.
enum Operand { ROWS = 0, COLS = 1 };
enum Output { STORE = 0, UPDATE = 1 };

struct Product {
    const f16 *A[MAX_SEGMENTS], *B[MAX_SEGMENTS];          // the contraction's segments, one after the other
    int n_seg, K;                                          // contraction of a segment
    long a_stride, b_stride, o_stride;                     // numbers from a matrix to the next
    int lda, ldb, ldo;
    int M, N;                                              // output
    int symmetric;                                         // the output is: tiles on and above the diagonal, each stored twice
    int row_tiles, col_tiles, tiles;                       // of a matrix
    // Tiles [0, whole) are computed by a block each; the `cut` tiles after them by `parts` blocks, one after the other along the contraction
    int whole, whole_per_xcd, cut, parts, part_per_xcd;
    float* part_ws;                                        // what a part leaves: [cut tile][part][wave][fragment][lane] as float4
    int* arrived;                                          // parts of a cut tile that have been stored; all zero between two launches
    float alpha, beta, diag;
    const f16 *D, *D_rest;                                 // addend, laid out like the output
    f16 *O, *O_rest;                                       // STORE
    // UPDATE: the weights, as the caller has them
    int count, m, n;
    int transposed[MUON_MAX_TENSORS];
    void* W[MUON_MAX_TENSORS];
    uint16_t* copies[MUON_MAX_TENSORS];                    // bf16 copies of fp32 weights, or null
    float keep, rate;                                      // w <- keep w - rate out
    int32_t* version;                                      // a counter per matrix of a tensor, or null
};

// Eight weights in a row, as they lie in memory (raw_t) and as numbers.
template <typename WT> struct WeightOps;
template <> struct WeightOps<bf16_t> {
    typedef oct_t raw_t;
    static __device__ __forceinline__ raw_t load8(const bf16_t* p) { return *reinterpret_cast<const oct_t*>(p); }
    static __device__ __forceinline__ void numbers(const raw_t& v, float* w)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[2 * i] = __uint_as_float(v[i] << 16); w[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store8(bf16_t* p, const float* w)
    {
        *reinterpret_cast<oct_t*>(p) = oct_t{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
    }
    static __device__ __forceinline__ void load4(const bf16_t* p, float* w)
    {
        typedef unsigned two_t __attribute__((ext_vector_type(2), aligned(2)));
        const two_t v = *reinterpret_cast<const two_t*>(p);
#pragma unroll
        for (int i = 0; i < 2; ++i) { w[2 * i] = __uint_as_float(v[i] << 16); w[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store4(bf16_t* p, const float* w)
    {
        typedef unsigned two_t __attribute__((ext_vector_type(2), aligned(2)));
        *reinterpret_cast<two_t*>(p) = two_t{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
    }
    static __device__ __forceinline__ float load(const bf16_t* p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void store(bf16_t* p, float w) { *p = f32_to_bf16(w); }
};
template <> struct WeightOps<float> {
    struct raw_t { quad_t q[2]; };
    static __device__ __forceinline__ raw_t load8(const float* p)
    {
        return raw_t{{*reinterpret_cast<const quad_t*>(p), *reinterpret_cast<const quad_t*>(p + 4)}};
    }
    static __device__ __forceinline__ void numbers(const raw_t& v, float* w)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = v.q[i / 4][i % 4];
    }
    static __device__ __forceinline__ void store8(float* p, const float* w)
    {
        *reinterpret_cast<quad_t*>(p) = quad_t{w[0], w[1], w[2], w[3]};
        *reinterpret_cast<quad_t*>(p + 4) = quad_t{w[4], w[5], w[6], w[7]};
    }
    static __device__ __forceinline__ void load4(const float* p, float* w)
    {
        const quad_t v = *reinterpret_cast<const quad_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
    }
    static __device__ __forceinline__ void store4(float* p, const float* w) { *reinterpret_cast<quad_t*>(p) = quad_t{w[0], w[1], w[2], w[3]}; }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, float w) { *p = w; }
};

// Where a CU gets one tile of 128 x 128 at most it has all of LDS for it, and what the loop waits for is the way of a request: seven slices
// ahead instead of three.
typedef Geometry<2, 2, 2, 2, 9, 1> Deep;
// 64 x 64, four waves of 32 x 32, two blocks on a CU: twice the bytes a product, where there are not tiles enough for the chip.
typedef Geometry<2, 2, 1, 1, 9, 2> Fine;

// ADD: there is an addend (and a diagonal); PLANES: numbers an operand is kept in; CUT: some of the tiles are.  Everything past the loop runs once per tile, from code that is
// not in the instruction cache: what a product does not need is not in its kernel.
// The loop is that of the grouped FFN (ffn_bf16.hip): slices of 32 straight from memory into a ring of LDS buffers, an operand read along its
// rows in whole 128-byte lines, two slices of half of the tile's rows at a time; in the 256 x 256 tile the two rows of waves
// alternate between fetching fragments and multiplying.  One tile per block; consecutive items go to one XCD, so that the tiles in flight
// there share operands of one matrix in its L2.
template <int KIND, int OUT, bool ADD, int PLANES, typename WT, class GEO, bool CUT>
__global__ __launch_bounds__(GEO::THREADS, GEO::BLOCKS * GEO::NWAVES / 4) void product_kernel(const Product p)
{
    constexpr int WGN = GEO::WGN, NWAVES = GEO::NWAVES, WM = GEO::WM, WN = GEO::WN, BM = GEO::BM, BN = GEO::BN, TM = GEO::TM, TN = GEO::TN;
    constexpr int STAGES = GEO::STAGES, PA = GEO::PA, PB = GEO::PB, FM = 2 * TM, FN = 2 * TN, SLICE_OPS = PA + PB;
    constexpr uint32_t A_BYTES = GEO::A_BYTES, STAGE_BYTES = GEO::STAGE_BYTES;
    constexpr bool B_COLS = KIND == COLS;

    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WGN, wn = wave % WGN;

    // what the first requests need, asked for at once: left to where it is used, it is read from memory in two steps, one after the other
    asm volatile("" :: "s"(p.A[0]), "s"(p.B[0]), "s"(p.a_stride), "s"(p.b_stride), "s"(p.lda), "s"(p.ldb), "s"(p.n_seg), "s"(p.K), "s"(p.M), "s"(p.N),
                 "s"(p.tiles), "s"(p.whole), "s"(p.whole_per_xcd), "s"(p.symmetric));
    // ---- which tile, and which part of it
    const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3;
    int item = xcd * p.whole_per_xcd + turn, part = 0, unit = 0;
    int parts = 1;
    if (CUT && turn >= p.whole_per_xcd) {
        const int i = xcd * p.part_per_xcd + turn - p.whole_per_xcd;
        if (i >= p.cut * p.parts) return;
        parts = p.parts;
        part = i / p.cut;                                  // neighbours work on the same stretch of the contraction
        unit = i - part * p.cut;
        item = p.whole + unit;
    } else if (item >= p.whole) {
        return;
    }
    const int matrix = item / p.tiles, t = item - matrix * p.tiles;
    int rt, ct;
    if (p.symmetric) {                                     // columns of the upper triangle, one after the other
        ct = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while ((ct + 1) * (ct + 2) / 2 <= t) ++ct;
        while (ct * (ct + 1) / 2 > t) --ct;
        rt = t - ct * (ct + 1) / 2;
    } else {                                               // bands of 8 row tiles, column by column
        const int band = t / (8 * p.col_tiles), in_band = t - band * 8 * p.col_tiles, band_rows = min(8, p.row_tiles - band * 8);
        rt = band * 8 + in_band % band_rows;
        ct = in_band / band_rows;
    }
    const int m0 = rt * BM, n0 = ct * BN;

    // ---- requests: what lies past the operand's last row reads as zero
    uint32_t voffA[PA], voffB[PB], ldsA[PA], ldsB[PB];
    auto line_source = [&](int blk, long ld) {
        const int row = blk * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
        return (uint32_t)((row * ld + piece * 8) * 2);
    };
#pragma unroll
    for (int i = 0; i < PA; ++i) { ldsA[i] = (wave + NWAVES * i) * 1024; voffA[i] = line_source(wave + NWAVES * i, p.lda); }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
        ldsB[i] = (wave + NWAVES * i) * 1024;
        voffB[i] = B_COLS ? kmajor_source<BN>((wave + NWAVES * i) * 64 + lane, p.ldb) : line_source(wave + NWAVES * i, p.ldb);
    }
    const int k_per_seg = p.K / BK;
    auto part_begin = [&](int i) { return (int)((long)i * (p.n_seg * k_per_seg) / parts) & ~1; };     // parts begin at even slices
    const int k_lo = part_begin(part), k_cnt = (part + 1 == parts ? p.n_seg * k_per_seg : part_begin(part + 1)) - k_lo;    // an even number, at least two
    rsrc_t ra, rb;
    int seg = CUT ? k_lo / k_per_seg : 0;
    auto open_segment = [&]() {
        const f16* a = p.A[seg] + (size_t)matrix * p.a_stride;
        const f16* b = p.B[seg] + (size_t)matrix * p.b_stride;
        ra = make_rsrc(a + (size_t)m0 * p.lda, (long long)(p.M - m0) * p.lda * 2);
        rb = B_COLS ? make_rsrc(b + n0, ((long long)p.K * p.ldb - n0) * 2) : make_rsrc(b + (size_t)n0 * p.ldb, (long long)(p.N - n0) * p.ldb * 2);
    };
    open_segment();
    const rsrc_t rnull = make_rsrc(p.A[0], 0);
    const uint32_t stepA = BK * 2, stepB = B_COLS ? (uint32_t)(BK * p.ldb * 2) : BK * 2;
    const uint32_t halfA = (uint32_t)(BM / 2 * p.lda * 2), halfB = (uint32_t)(BN / 2 * p.ldb * 2);
    int iss_stage = 0, iss_in_seg = k_lo - seg * k_per_seg;
    uint32_t soffA = (uint32_t)iss_in_seg * stepA, soffB = (uint32_t)iss_in_seg * stepB;
    auto request_piece = [&](int n, uint32_t st, const rsrc_t a, const rsrc_t b, uint32_t oa, uint32_t ob) {
        if (n < PA) dma16(a, st + ldsA[n], voffA[n], oa);
        else dma16(b, st + A_BYTES + ldsB[n - PA], voffB[n - PA], ob);
    };
    auto group_offsets = [&](auto PAR, uint32_t& oa, uint32_t& ob) {
        constexpr int par = decltype(PAR)::value;
        oa = par ? soffA + halfA : soffA;
        ob = (!B_COLS && par) ? soffB + halfB : soffB;
    };
    auto group_done = [&](auto PAR) {
        constexpr int par = decltype(PAR)::value;
        iss_stage = iss_stage + 1 == STAGES ? 0 : iss_stage + 1;
        ++iss_in_seg;
        if (par) soffA += 2 * stepA;
        if (B_COLS || par) soffB += B_COLS ? stepB : 2 * stepB;
    };
    auto issue_group = [&](auto PAR, const rsrc_t a, const rsrc_t b) {
        const uint32_t st = lds0 + (uint32_t)iss_stage * STAGE_BYTES;
        uint32_t oa, ob;
        group_offsets(PAR, oa, ob);
#pragma unroll
        for (int n = 0; n < SLICE_OPS; ++n) request_piece(n, st, a, b, oa, ob);
        group_done(PAR);
    };
    auto group_fixups = [&]() {                            // after an odd group: the next segment, if there is one
        if (iss_in_seg != k_per_seg) return;
        iss_in_seg = 0; soffA = 0; soffB = 0;
        if (++seg < p.n_seg) open_segment();
    };

    // ---- fragment addresses inside a ring buffer
    uint32_t fk_addr[FN], fpa[2], fpb[2];                  // chunks of 16 columns: the wave's own of a line of 64
#pragma unroll
    for (int c = 0; c < FN; ++c) fk_addr[c] = kmajor_off<BN>(8 * (lane >> 4) + ((lane & 15) >> 2), wn * WN + c * 16 + 4 * (lane & 3));
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        fpa[v] = halfpair_off(lane & 15, lane >> 4) ^ (uint32_t)(v << 6);
        fpb[v] = A_BYTES + (halfpair_off((wn % (WGN / 2)) * WN + (lane & 15), lane >> 4) ^ (uint32_t)(v << 6));
    }
    f32x4 acc[FM][FN];
    // AHEAD: four waves have the CU to themselves, and nobody's products to fill the time of a slice's fragment reads: they read those of the next
    // slice into a second set of registers while they multiply.
    constexpr bool AHEAD = GEO::BLOCKS == 1 && !GEO::TWO_PHASE;
    f16x8 fa2[AHEAD ? 2 : 1][FM], fb2[AHEAD ? 2 : 1][FN];
    auto goes_out = [](int n) { return (n + 1) % ((FM + FN) / SLICE_OPS) == 0 ? (n + 1) / ((FM + FN) / SLICE_OPS) - 1 : -1; };
    auto load_frags = [&](uint32_t stA, uint32_t stB, auto PAR, auto after) {
        constexpr int par = decltype(PAR)::value;
        f16x8 (&fa)[FM] = fa2[AHEAD ? par : 0];
        f16x8 (&fb)[FN] = fb2[AHEAD ? par : 0];
        const uint32_t a = stA + fpa[par];
        auto frag_a = [&](auto I) { lds_frag_kcontig_at<decltype(I)::value * 2048>(fa[decltype(I)::value], a); after(decltype(I)::value); };
        frag_a(std::integral_constant<int, 0>{}); frag_a(std::integral_constant<int, 1>{});
        if constexpr (FM >= 4) { frag_a(std::integral_constant<int, 2>{}); frag_a(std::integral_constant<int, 3>{}); }
        if constexpr (FM == 8) {
            frag_a(std::integral_constant<int, 4>{}); frag_a(std::integral_constant<int, 5>{});
            frag_a(std::integral_constant<int, 6>{}); frag_a(std::integral_constant<int, 7>{});
        }
        if constexpr (B_COLS) {
#pragma unroll
            for (int j = 0; j < FN; ++j) { lds_frag_kmajor_at<BN * 8, 0>(fb[j], stB + A_BYTES + fk_addr[j]); after(FM + j); }
        } else {
            const uint32_t b = stB + fpb[par];
            auto frag_b = [&](auto J) { lds_frag_kcontig_at<decltype(J)::value * 2048>(fb[decltype(J)::value], b); after(FM + decltype(J)::value); };
            frag_b(std::integral_constant<int, 0>{}); frag_b(std::integral_constant<int, 1>{});
            if constexpr (FN == 4) { frag_b(std::integral_constant<int, 2>{}); frag_b(std::integral_constant<int, 3>{}); }
        }
    };
    auto mma_first = [&](const f16x8 (&fa)[FM], const f16x8 (&fb)[FN]) {       // the first products take zero as their addend
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int jj = 0; jj < FN; ++jj) {
                const int j = (i & 1) ? FN - 1 - jj : jj;
                asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, 0" : "=a"(acc[i][j]) : "v"(fb[j]), "v"(fa[i]));
            }
    };
    auto mma = [&](const f16x8 (&fa)[FM], const f16x8 (&fb)[FN]) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int jj = 0; jj < FN; ++jj) {
                const int j = (i & 1) ? FN - 1 - jj : jj;
                asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(fb[j]), "v"(fa[i]));
            }
    };

    // ---- main loop: slice t reads the groups of its pair and requests group t + L
    constexpr int L = STAGES - 2;                          // into the slot of group t - 2, last read in slice t - 1
    static_assert(L % 2 == 1, "the group a slice requests is of the other parity");
    typedef std::integral_constant<int, 0> even_t;
    typedef std::integral_constant<int, 1> odd_t;
#pragma unroll
    for (int g = 0; g + 1 < L; g += 2) {                   // groups 0 .. L - 1, those that there are
        const bool there = g < k_cnt;
        issue_group(even_t{}, there ? ra : rnull, there ? rb : rnull);
        issue_group(odd_t{}, there ? ra : rnull, there ? rb : rnull);
        if (there) group_fixups();
    }
    issue_group(even_t{}, L - 1 < k_cnt ? ra : rnull, L - 1 < k_cnt ? rb : rnull);
    WAIT_VMCNT((L - 2) * SLICE_OPS);                       // groups 0 and 1 have landed: slices 0 and 1
    BLOCK_BARRIER();
    if (GEO::TWO_PHASE && wm == 1) BLOCK_BARRIER();
    int cur = 0, pair0 = 0;                                // ring slots of the slice's own group, of the even group of its pair
    const int hA = wm, hB = wn / (WGN / 2);                // which group of a pair holds this wave's rows of A and of B
    auto slot_base = [&](int slot) { return lds0 + (uint32_t)(slot >= STAGES ? slot - STAGES : slot) * STAGE_BYTES; };
    auto wait_frags = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);                 // no product moves above the wait
    };
    auto slice = [&](auto PAR, auto FIRST, auto LAST, const rsrc_t a, const rsrc_t b) {
        constexpr int par = decltype(PAR)::value;
        typedef std::integral_constant<int, 1 - par> other_t;
        const uint32_t to = lds0 + (uint32_t)iss_stage * STAGE_BYTES;
        uint32_t oa, ob;
        group_offsets(other_t{}, oa, ob);
        auto request_between = [&](int n) { if (goes_out(n) >= 0) { __builtin_amdgcn_sched_barrier(0); request_piece(goes_out(n), to, a, b, oa, ob); __builtin_amdgcn_sched_barrier(0); } };
        if constexpr (AHEAD) {
            // the next slice's groups, of the L - 1 + t that are on their way
            WAIT_VMCNT((par ? L - 3 : L - 2) * SLICE_OPS);
            BLOCK_BARRIER();
            cur = (cur + 1 == STAGES) ? 0 : cur + 1;
            if (par) pair0 = (pair0 + 2 >= STAGES) ? pair0 + 2 - STAGES : pair0 + 2;
            if constexpr (!decltype(LAST)::value) load_frags(slot_base(pair0 + hA), B_COLS ? slot_base(cur) : slot_base(pair0 + hB), other_t{}, request_between);
            group_done(other_t{});
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(FIRST)::value) mma_first(fa2[par], fb2[par]); else mma(fa2[par], fb2[par]);
            wait_frags();
        } else {
            load_frags(slot_base(pair0 + hA), B_COLS ? slot_base(cur) : slot_base(pair0 + hB), PAR, request_between);
            group_done(other_t{});
            WAIT_VMCNT((par ? L - 2 : L - 1) * SLICE_OPS);                 // next: a pair's two groups, or the second one of a pair that has landed
            wait_frags();
            BLOCK_BARRIER();
            __builtin_amdgcn_s_setprio(1);
            if constexpr (decltype(FIRST)::value) mma_first(fa2[0], fb2[0]); else mma(fa2[0], fb2[0]);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            if (GEO::TWO_PHASE) BLOCK_BARRIER();
            cur = (cur + 1 == STAGES) ? 0 : cur + 1;
            if (par) pair0 = (pair0 + 2 >= STAGES) ? pair0 + 2 - STAGES : pair0 + 2;
        }
    };
    if constexpr (AHEAD) {                                 // the first slice's fragments
        load_frags(slot_base(hA), B_COLS ? slot_base(0) : slot_base(hB), even_t{}, [](int) {});
        wait_frags();
    }
    typedef std::true_type yes_t;
    typedef std::false_type no_t;
    if (L < k_cnt) { slice(even_t{}, yes_t{}, no_t{}, ra, rb); group_fixups(); }
    else slice(even_t{}, yes_t{}, no_t{}, rnull, rnull);
    int s = 1;
    while (s < k_cnt - 1) {
        const bool more = s + L < k_cnt;                   // the pair of slices s + L, s + L + 1 exists
        const int n = more ? min((k_cnt - L - s + 1) / 2, (k_per_seg - iss_in_seg) / 2) : (k_cnt - 1 - s) / 2;
        const rsrc_t a = more ? ra : rnull, b = more ? rb : rnull;
        for (int i = 0; i < n; ++i) {
            slice(odd_t{}, no_t{}, no_t{}, a, b);
            slice(even_t{}, no_t{}, no_t{}, a, b);
        }
        s += 2 * n;
        if (more) group_fixups();
    }
    slice(odd_t{}, no_t{}, yes_t{}, rnull, rnull);         // the last one
    WAIT_VMCNT(0);                                         // the empty requests too: the epilogue reuses the ring
    if (GEO::TWO_PHASE && wm == 0) BLOCK_BARRIER();        // both rows have passed the same number of barriers
    BLOCK_BARRIER();
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");     // the last products have written back before they are read

    // ---- a part of a tile.  All of its parts but the last to be done leave their sums in the workspace; the last adds them, itself among them, in
    // the order of the contraction (the same bits whichever part is last) and goes on with the tile.  Nobody waits for another block.
    // The sums and the count go past the L2 of the XCD (sc1), of which every XCD has its own.
    constexpr int AT_DEVICE = 16, UNIT_FLOATS = GEO::BM * GEO::BN;
    static_assert(NWAVES * FM * FN * 64 * 4 == UNIT_FLOATS, "a part fills its unit");
    auto part_rsrc = [&](int i) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)(p.part_ws + ((size_t)unit * parts + i) * UNIT_FLOATS), 0, UNIT_FLOATS * 4, 0x00020000);
    };
    const int part_ofs = (wave * (FM * FN) * 64 + lane) * 16;
    if (CUT && parts > 1) {
        auto tell = [&](int v) {                           // what thread 0 knows, to all
            int* word = reinterpret_cast<int*>(smem);
            if (tid == 0) *word = v;
            __syncthreads();
            const int r = __builtin_amdgcn_readfirstlane(*word);
            __syncthreads();
            return r;
        };
        int* counter = p.arrived + unit;
        int before = tell(tid == 0 ? __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0);
        if (before != parts - 1) {                         // else all the others are there already
            const buf_rsrc_t to = part_rsrc(part);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), to, part_ofs + (i * FN + j) * 1024, 0, AT_DEVICE);
            WAIT_VMCNT(0);                                 // every wave's stores are complete before the count
            __syncthreads();
            before = tell(tid == 0 ? __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0);
            if (before != parts - 1) return;
        }
        if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }

    // ---- epilogue: 64 x 64 results at a time through a patch of LDS, the wave's own or, of four waves of 32 x 32, the block's, so that memory sees whole lines along the rows
    // and, where the result is wanted the other way round too, along the columns.
    // Its rows are 16 slots of 4 numbers, permuted by the row so that neither the writes (16 rows of a slot), nor the reads along a row, nor
    // those along a column (8 columns of rows 8 apart) meet in a bank.
    // Slot c4 of row r lies at r * 256 + 16 (c4 ^ (r & 15) ^ ((r >> 3) & 6)); below, as a part of the lane's own, combined with a constant.
    constexpr int PATCH = 64 * 256;
    constexpr bool SHARED = WN == 32;
    constexpr int OF64 = SHARED ? 1 : WM / 64, FRAG_ROWS = SHARED ? 2 : 4, PASSES = SHARED ? 2 : 8;    // blocks of 64, rows of fragments in one, passes of the wave
    static_assert((SHARED ? WM == 32 && NWAVES == 4 : WN == 64 && WM % 64 == 0) && NWAVES * PATCH <= (int)GEO::LDS_BYTES, "patches inside the ring");
    unsigned char* patch = smem + (SHARED ? 0 : wave * PATCH);
    const int pass0 = SHARED ? 2 * wave : 0;
    const int r8 = lane >> 3, c8 = (lane & 7) * 8;         // row of eight that a pass takes, first of its eight columns
    const int put_at = (lane & 15) * 256 + (SHARED ? wm * 32 * 256 : 0);
    const int put_slot = (lane >> 4) ^ (lane & 15) ^ (SHARED ? wn * 8 ^ wm * 4 : 0);                                // row i 16 + lane % 16, slot j 4 + lane / 16
    const int row_at = r8 * 256, row_slot = (c8 / 4) ^ r8;                                                     // row pass 8 + r8, from column c8
    const int col_at = c8 * 256 + (r8 & 3) * 4, col_slot = (r8 >> 2) ^ (c8 & 8) ^ ((c8 >> 3) & 6);             // column pass 8 + r8, from row c8
    const int col0 = n0 + (SHARED ? 0 : wn * WN);
    const int tensor = OUT == UPDATE ? matrix / p.count : 0;
    const bool tall = OUT == UPDATE && p.transposed[tensor] != 0;
    WT* W = nullptr;
    uint16_t* copy = nullptr;
    if constexpr (OUT == UPDATE) {
        const size_t base = (size_t)(matrix % p.count) * ((size_t)p.m * p.n);
        W = (WT*)p.W[tensor] + base;
        copy = p.copies[tensor] ? p.copies[tensor] + base : nullptr;
        if (p.version && t == 0 && tensor == 0 && tid == 0) p.version[matrix] += 1;
    }
#pragma unroll
    for (int block = 0; block < OF64; ++block) {
        const int row0 = m0 + (SHARED ? 0 : wm * WM + block * 64);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        // rows of fragments at a time: all loads of a part are on their way before the first is added, as far as there are registers for them
        constexpr int ROWS_AT_ONCE = GEO::NWAVES == 8 || SHARED ? 2 : 4;
#pragma unroll
        for (int i0 = 0; i0 < FRAG_ROWS; i0 += ROWS_AT_ONCE) {
            f32x4 val[ROWS_AT_ONCE][FN];
            if constexpr (!CUT) {
#pragma unroll
                for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) {
                        asm volatile("" : "+a"(acc[block * FRAG_ROWS + i0 + i][j]));
                        val[i][j] = acc[block * FRAG_ROWS + i0 + i][j];
                    }
            } else {
#pragma unroll
            for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) val[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            auto add_parts = [&](int q0, int q1) {
#pragma unroll 1
                for (int q = q0; q < q1; ++q) {
                    f32x4 x[ROWS_AT_ONCE][FN];
                    const buf_rsrc_t from = part_rsrc(q);
#pragma unroll
                    for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j)
                            x[i][j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, part_ofs + ((block * FRAG_ROWS + i0 + i) * FN + j) * 1024, 0, AT_DEVICE));
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) val[i][j] += x[i][j];
                }
            };
            add_parts(0, part);
#pragma unroll
            for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    asm volatile("" : "+a"(acc[block * FRAG_ROWS + i0 + i][j]));   // they stay where they are until here: read earlier, all at once, they would not fit
                    val[i][j] += acc[block * FRAG_ROWS + i0 + i][j];
                }
            add_parts(part + 1, parts);
            }
#pragma unroll
            for (int i = 0; i < ROWS_AT_ONCE; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    *reinterpret_cast<float4*>(patch + put_at + (i0 + i) * 4096 + ((put_slot ^ (j * 4) ^ ((i0 + i) * 2)) << 4)) = make_float4(val[i][j][0], val[i][j][1], val[i][j][2], val[i][j][3]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (SHARED) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
        if (row0 >= p.M || col0 >= p.N) continue;          // sides are multiples of 64: all of it or none
        auto row_of = [&](int pass, float* v) {            // eight columns of a row of the block
            const int k = ((pass & 1) << 3) ^ (pass & 6);
            *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(patch + row_at + pass * 2048 + ((row_slot ^ k) << 4));
            *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(patch + row_at + pass * 2048 + ((row_slot ^ k ^ 1) << 4));
        };
        auto column_of = [&](int pass, float* v) {         // eight rows of a column
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const float*>(patch + col_at + e * 256 + ((col_slot ^ (pass * 2) ^ e) << 4));
        };
        if constexpr (OUT == STORE) {
            // Along the rows, and off the diagonal of a symmetric product along the columns too: the addend is symmetric as well and
            // is read where the result goes.  What memory and LDS give is requested for several passes before the first is used.
            constexpr int BATCH = GEO::NWAVES == 8 || SHARED ? 2 : 8;
            const bool diagonal = row0 == col0;
            auto put = [&](auto COLUMNS) {
                constexpr bool columns = decltype(COLUMNS)::value;
                const size_t o = (size_t)matrix * p.o_stride + (size_t)((columns ? col0 : row0) + r8) * p.ldo + (columns ? row0 : col0) + c8 + (size_t)pass0 * 8 * p.ldo;
                const size_t pass_step = (size_t)8 * p.ldo;
#pragma unroll
                for (int b = 0; b < PASSES; b += BATCH) {
                    if (BATCH < PASSES) __builtin_amdgcn_sched_barrier(0);      // no more than a batch in the registers beside the accumulators
                    u32x4 d[ADD ? PLANES : 1][BATCH];
                    float v[BATCH][8];
                    if constexpr (ADD)
#pragma unroll
                        for (int i = 0; i < BATCH; ++i) {
                            d[0][i] = *reinterpret_cast<const u32x4*>(p.D + o + (b + i) * pass_step);
                            if constexpr (PLANES == 2) d[1][i] = *reinterpret_cast<const u32x4*>(p.D_rest + o + (b + i) * pass_step);
                        }
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        if constexpr (columns) column_of(pass0 + b + i, v[i]);
                        else row_of(pass0 + b + i, v[i]);
                    }
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] *= p.alpha;
                        if constexpr (ADD) {
#pragma unroll
                            for (int k = 0; k < PLANES; ++k) {
                                float x[8];
                                unpack_f16x8(d[k][i], x);
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[i][e] = fmaf(p.beta, x[e], v[i][e]);
                            }
                            if (!columns && diagonal) {
                                const float here = (lane & 7) == pass0 + b + i ? p.diag : 0.0f;
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[i][e] += r8 == e ? here : 0.0f;
                            }
                        }
                        const u32x4 first = pack_f16x8(v[i]);
                        *reinterpret_cast<u32x4*>(p.O + o + (b + i) * pass_step) = first;
                        if constexpr (PLANES == 2) *reinterpret_cast<u32x4*>(p.O_rest + o + (b + i) * pass_step) = pack_rest(v[i], first);
                    }
                }
            };
            put(std::false_type{});
            if (p.symmetric && rt != ct) put(std::true_type{});
        } else {
            // along the rows of the weights, which are columns of the block where they lie on their short side
            typedef WeightOps<WT> Ops;
            const int wr = (tall ? col0 : row0) + r8 + pass0 * 8, wc = (tall ? row0 : col0) + c8, w_rows = tall ? p.n : p.m, w_cols = tall ? p.m : p.n;
            const int there = w_cols - wc;
            typename Ops::raw_t raw[PASSES];
            if (there >= 8)
#pragma unroll
                for (int pass = 0; pass < PASSES; ++pass)
                    if (wr + 8 * pass < w_rows) raw[pass] = Ops::load8(W + (size_t)(wr + 8 * pass) * w_cols + wc);
#pragma unroll
            for (int pass = 0; pass < PASSES; ++pass) {
                float x[8], w[8];
                if (tall) column_of(pass0 + pass, x); else row_of(pass0 + pass, x);
                if (wr + 8 * pass >= w_rows) continue;
                const size_t at = (size_t)(wr + 8 * pass) * w_cols + wc;
                if (there >= 8) {
                    Ops::numbers(raw[pass], w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = fmaf(-p.rate, x[e] * p.alpha, p.keep * w[e]);
                    Ops::store8(W + at, w);
                    if constexpr (PLANES == 2)
                        if (copy) WeightOps<bf16_t>::store8(copy + at, w);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < there) {
                            const float one = fmaf(-p.rate, x[e] * p.alpha, p.keep * Ops::load(W + at + e));
                            Ops::store(W + at + e, one);
                            if constexpr (PLANES == 2)
                                if (copy) WeightOps<bf16_t>::store(copy + at + e, one);
                        }
                }
            }
        }
    }
}

// ---- small matrices: the whole update in one launch -----------------------------------------------------
// A block per matrix, X, A and B in LDS from beginning to end (the form with X on its long side: nothing is gained by the Gram matrix here).
// What bounds the general way here is what a launch costs: 17 of them, 6 us and more each, 133 us for four matrices of 64 x 256 in two numbers,
// where this takes 34: 4 us for the momentum, 3.5 for X, 20 for five steps, 4 for the weights.
// Rows of X, A and B lie in LDS as they are, the 16-byte pieces of 128 bytes permuted by the row (a fragment reads a piece of 16 rows, a transposing
// one 4 columns of 4 rows at a time).
constexpr int FEW_WAVES = 8;
constexpr int FEW_QUADS = 16, FEW_ELEMENTS = FEW_QUADS * 4 * FEW_WAVES * 64;      // of a matrix that a thread, a block has in registers
constexpr size_t FEW_LDS = 159 * 1024;                     // X, A and B; the rest of the 160 KB holds the parts of the norm
struct Few {
    int m, n, np, count, nesterov, steps;
    float mu, eps, S, SA, SB, a, b, c, keep, rate;
    const float* grad[MUON_MAX_TENSORS];
    float* momentum[MUON_MAX_TENSORS];
    void* W[MUON_MAX_TENSORS];
    uint16_t* copies[MUON_MAX_TENSORS];
    int transposed[MUON_MAX_TENSORS];
    int32_t* version;
};
inline size_t few_lds(int mp, int np, int planes) { return (size_t)planes * 2 * ((size_t)mp * np + 2 * (size_t)mp * mp); }

// PLANES numbers an element, MT row tiles of 16
template <int PLANES, int MT, typename WT>
__global__ __launch_bounds__(FEW_WAVES * 64) void few_kernel(const Few p)
{
    constexpr int MP = MT * 16, THREADS = FEW_WAVES * 64, TILES = MT * MT / FEW_WAVES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ double words[FEW_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int matrix = blockIdx.x, tensor = matrix / p.count;
    const bool tall = p.transposed[tensor] != 0;
    const size_t base = (size_t)(matrix % p.count) * ((size_t)p.m * p.n);
    const float* __restrict__ G = p.grad[tensor] + base;
    float* __restrict__ M = p.momentum[tensor] + base;

    const uint32_t x_plane = (uint32_t)MP * p.np * 2;
    constexpr uint32_t A_PLANE = MP * MP * 2;
    unsigned char *const X = smem, *const A = smem + PLANES * x_plane, *const B = A + PLANES * A_PLANE;
    auto at = [](int row, int col, int ld) { return (uint32_t)(row * ld * 2 + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2); };
    // 16 rows from `row`, 32 steps from `col`
    auto frag = [&](const unsigned char* m, int row, int col, int ld) {
        return *reinterpret_cast<const f16x8*>(m + at(row + (lane & 15), col + 8 * (lane >> 4), ld));
    };
    // 16 columns from `col`, 32 steps, which are rows, from `row`
    auto frag_columns = [&](const unsigned char* m, int row, int col, int ld) {
        typedef __attribute__((__vector_size__(8))) __fp16 four_t;
        typedef __attribute__((address_space(3))) four_t lds_four_t;
        f16x8 f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t o = at(row + 8 * (lane >> 4) + 4 * h + ((lane & 15) >> 2), col + 4 * (lane & 3), ld);
            const four_t v = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_four_t*)(m + o));
#pragma unroll
            for (int i = 0; i < 4; ++i) f[4 * h + i] = (f16)v[i];
        }
        return f;
    };
    // four numbers of a row from a result: row l % 16, columns 4 (l / 16) .. + 3 of a tile
    auto put = [&](unsigned char* m, uint32_t plane, int row, int col, int ld, const f32x4& v) {
        const uint32_t o = at(row + (lane & 15), col + 4 * (lane >> 4), ld);
        const uint32_t lo = pack_f16x2(v[0], v[1]), hi = pack_f16x2(v[2], v[3]);
        *reinterpret_cast<uint2*>(m + o) = make_uint2(lo, hi);
        if constexpr (PLANES == 2) {
            const f16x2 f0 = __builtin_bit_cast(f16x2, lo), f1 = __builtin_bit_cast(f16x2, hi);
            *reinterpret_cast<uint2*>(m + plane + o) = make_uint2(pack_f16x2(v[0] - (float)f0[0], v[1] - (float)f0[1]), pack_f16x2(v[2] - (float)f1[0], v[3] - (float)f1[1]));
        }
    };
    // The sum of a product of numbers in two planes: hi lo + lo hi apart from hi hi until the end.
    struct Sum { f32x4 big, small; };
    auto clear = [](Sum& a) { a.big = a.small = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; };
    auto mma = [](Sum& a, const f16x8 (&rows)[PLANES], const f16x8 (&cols)[PLANES]) {
        if constexpr (PLANES == 2) {
            a.small = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols[1], rows[0], a.small, 0, 0, 0);
            a.small = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols[0], rows[1], a.small, 0, 0, 0);
        }
        a.big = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols[0], rows[0], a.big, 0, 0, 0);
    };
    auto total = [](const Sum& a, int e) { return PLANES == 2 ? a.big[e] + a.small[e] : a.big[e]; };

    // ---- momentum and the norm, all of a thread's elements in its registers; then X, with zeros up to the padded sides
    const int elements = p.m * p.n, quads = elements / 4, w_cols = tall ? p.m : p.n;
    float u[FEW_QUADS][4], u_tail = 0.0f;
    {
        quad_t g[FEW_QUADS], v[FEW_QUADS];
#pragma unroll
        for (int k = 0; k < FEW_QUADS; ++k) {
            const int q = tid + k * THREADS;
            if (q < quads) { g[k] = *reinterpret_cast<const quad_t*>(G + 4 * q); v[k] = *reinterpret_cast<const quad_t*>(M + 4 * q); }
        }
        for (uint32_t o = tid * 16; o < PLANES * x_plane; o += THREADS * 16) *reinterpret_cast<u32x4*>(X + o) = u32x4{0, 0, 0, 0};
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < FEW_QUADS; ++k) {
            const int q = tid + k * THREADS;
            if (q < quads) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[k][e] = fmaf(p.mu, v[k][e], g[k][e]);
                    u[k][e] = direction(g[k][e], v[k][e], p.mu, p.nesterov);
                    sum = fma((double)u[k][e], (double)u[k][e], sum);
                }
                *reinterpret_cast<quad_t*>(M + 4 * q) = v[k];
            }
        }
        if (tid < elements % 4) {
            const int e = quads * 4 + tid;
            const float gt = G[e], vt = fmaf(p.mu, M[e], gt);
            M[e] = vt;
            u_tail = direction(gt, vt, p.mu, p.nesterov);
            sum = fma((double)u_tail, (double)u_tail, sum);
        }
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if (lane == 0) words[wave] = sum;
    }
    __syncthreads();
    // row and column of a thread's quads: q grows by THREADS
    auto for_each_quad = [&](auto use) {
        int i = 4 * tid / w_cols, j = 4 * tid - i * w_cols;
        const int di = 4 * THREADS / w_cols, dj = 4 * THREADS - di * w_cols;
#pragma unroll
        for (int k = 0; k < FEW_QUADS; ++k) {
            if (tid + k * THREADS < quads) {
                int r = i, c = j;
                uint32_t o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = tall ? at(c, r, p.np) : at(r, c, p.np);
                    if (++c == w_cols) { c = 0; ++r; }
                }
                use(k, o);
            }
            i += di; j += dj;
            if (j >= w_cols) { j -= w_cols; ++i; }
        }
    };
    const int tail_e = quads * 4 + tid, tail_i = tail_e / w_cols, tail_j = tail_e - tail_i * w_cols;
    const uint32_t tail_o = tall ? at(tail_j, tail_i, p.np) : at(tail_i, tail_j, p.np);        // of the threads that have one
    auto put_one = [&](uint32_t o, float x) {
        const f16 h = (f16)x;
        *reinterpret_cast<f16*>(X + o) = h;
        if constexpr (PLANES == 2) *reinterpret_cast<f16*>(X + x_plane + o) = (f16)(x - (float)h);
    };
    auto get_one = [&](uint32_t o) {
        float x = (float)*reinterpret_cast<const f16*>(X + o);
        if constexpr (PLANES == 2) x += (float)*reinterpret_cast<const f16*>(X + x_plane + o);
        return x;
    };
    {
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) sum += words[w];
        const double factor = (double)p.S / (sqrt(sum) + (double)p.eps);
        for_each_quad([&](int k, const uint32_t (&o)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) put_one(o[e], (float)((double)u[k][e] * factor));
        });
        if (tid < elements % 4) put_one(tail_o, (float)((double)u_tail * factor));
    }
    __syncthreads();

    const int row_tile = wave * TILES / MT, col_tile0 = wave * TILES % MT;         // of A and B: TILES tiles of a row
    for (int step = 0; step < p.steps; ++step) {
        Sum acc[TILES];
        {                                                  // A = X X^T
#pragma unroll
            for (int t = 0; t < TILES; ++t) clear(acc[t]);
#pragma unroll 2
            for (int k = 0; k < p.np; k += 32) {
                f16x8 fa[PLANES], fb[TILES][PLANES];
#pragma unroll
                for (int q = 0; q < PLANES; ++q) {
                    fa[q] = frag(X + q * x_plane, row_tile * 16, k, p.np);
#pragma unroll
                    for (int t = 0; t < TILES; ++t) fb[t][q] = frag(X + q * x_plane, (col_tile0 + t) * 16, k, p.np);
                }
#pragma unroll
                for (int t = 0; t < TILES; ++t) mma(acc[t], fa, fb[t]);
            }
            const float alpha = p.SA / (p.S * p.S);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = total(acc[t], e) * alpha;
                put(A, A_PLANE, row_tile * 16, (col_tile0 + t) * 16, MP, v);
            }
        }
        __syncthreads();
        {                                                  // B = a + b A + c A A
            const float alpha = p.c * p.SB / (p.SA * p.SA), beta = p.b * p.SB / p.SA, diag = p.a * p.SB;
#pragma unroll
            for (int t = 0; t < TILES; ++t) clear(acc[t]);
#pragma unroll
            for (int k = 0; k < MP; k += 32) {
                f16x8 fa[PLANES];
#pragma unroll
                for (int q = 0; q < PLANES; ++q) fa[q] = frag(A + q * A_PLANE, row_tile * 16, k, MP);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    f16x8 fb[PLANES];
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) fb[q] = frag(A + q * A_PLANE, (col_tile0 + t) * 16, k, MP);
                    mma(acc[t], fa, fb);
                }
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const int row = row_tile * 16 + (lane & 15), col = (col_tile0 + t) * 16 + 4 * (lane >> 4);
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = total(acc[t], e) * alpha;
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) x = fmaf(beta, (float)*reinterpret_cast<const f16*>(A + q * A_PLANE + at(row, col + e, MP)), x);
                    v[e] = x + (row == col + e ? diag : 0.0f);
                }
                put(B, A_PLANE, row_tile * 16, (col_tile0 + t) * 16, MP, v);
            }
        }
        __syncthreads();
        // X = B X: a wave takes twice 16 columns at a time, which nobody else reads now
        for (int col0 = wave * 16; col0 < p.np; col0 += 2 * FEW_WAVES * 16) {
            const bool two = col0 + FEW_WAVES * 16 < p.np;
            Sum sum[2][MT];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < MT; ++t) clear(sum[h][t]);
#pragma unroll
            for (int k = 0; k < MP; k += 32) {
                f16x8 fx[2][PLANES];
#pragma unroll
                for (int q = 0; q < PLANES; ++q) {
                    fx[0][q] = frag_columns(X + q * x_plane, k, col0, p.np);
                    fx[1][q] = frag_columns(X + q * x_plane, k, two ? col0 + FEW_WAVES * 16 : col0, p.np);
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    f16x8 fb[PLANES];
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) fb[q] = frag(B + q * A_PLANE, t * 16, k, MP);
                    mma(sum[0][t], fb, fx[0]);
                    mma(sum[1][t], fb, fx[1]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1 && !two) break;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = total(sum[h][t], e) * (1.0f / p.SB);
                    put(X, x_plane, t * 16, col0 + h * FEW_WAVES * 16, p.np, v);
                }
            }
        }
        __syncthreads();
    }

    // ---- the weights, along their rows
    typedef WeightOps<WT> Ops;
    WT* W = (WT*)p.W[tensor] + base;
    uint16_t* copy = PLANES == 2 && p.copies[tensor] ? p.copies[tensor] + base : nullptr;
    auto one = [&](float w, uint32_t o) { return fmaf(-p.rate, get_one(o), p.keep * w); };
    float w[FEW_QUADS][4];
#pragma unroll
    for (int k = 0; k < FEW_QUADS; ++k)
        if (tid + k * THREADS < quads) Ops::load4(W + 4 * (tid + k * THREADS), w[k]);
    for_each_quad([&](int k, const uint32_t (&o)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[k][e] = one(w[k][e], o[e]);
        Ops::store4(W + 4 * (tid + k * THREADS), w[k]);
        if (PLANES == 2 && copy) WeightOps<bf16_t>::store4(copy + 4 * (tid + k * THREADS), w[k]);
    });
    if (tid < elements % 4) {
        const float x = one(Ops::load(W + tail_e), tail_o);
        Ops::store(W + tail_e, x);
        if (PLANES == 2 && copy) WeightOps<bf16_t>::store(copy + tail_e, x);
    }
    if (p.version && tensor == 0 && tid == 0) p.version[matrix] += 1;
}

template <int PLANES, int MT, typename WT> hipError_t launch_few(const Few& f, int matrices, hipStream_t st)
{
    static PerDeviceOnce once;
    const int dev = current_device();
    auto kern = few_kernel<PLANES, MT, WT>;
    if (!once.is_done(dev)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)FEW_LDS);
        if (e != hipSuccess) return e;
        once.mark(dev);
    }
    hipLaunchKernelGGL(kern, dim3(matrices), dim3(FEW_WAVES * 64), few_lds(MT * 16, f.np, PLANES), st, f);
    return hipGetLastError();
}

// How a product is laid out: the geometry, and into how many parts the tiles after the last full round of the chip's places are cut.
// us of a slice (of all the blocks a CU holds), of what a tile costs beside its slices, and of joining two parts (a quarter more for each
// further one).  A slice of 128 x 128 takes as long whether one or two blocks share a CU: what more parts gain is CUs, not overlap.  Of its 560 to 590
// clocks the matrix pipes have 256 and the fragment reads 177, and it fetches 29 bytes a clock, half of what the path from L2 gives: counted on the
// squares of 4 x 1024 x 4096, no one of them bounds it, their order between two barriers does.  Measured, us: squares of m = 4096 (six; 816 tiles of 256, 128 slices) 413 whole, 370 with the last 48 in five parts; X X^T
// of 4 x 1024 x 4096 (144 tiles of 128, 128 slices) 38 whole, 33 in three parts, of 6 x 500 x 1333 in two numbers (60 tiles, 126 slices) 42 and 25
// in four; its squares (48 slices) 17.8 whole, 18.8 in three.  64 x 64 tiles where those of 128 do not fill the CUs, the whole call, us: two numbers, 6 x
// 1333 x 500 374 -> 272, 16 x 200 x 300 233 -> 153; bf16, 8 x 256 x 1024 149 -> 108, 6 x 384 x 768 167 -> 121; 4 x 1024 x 4096, whose squares are 144
// tiles of 128, 387 either way.
struct GeometryTime { float slice, over, join; int least; };           // least: slices of a part
constexpr GeometryTime LARGE_TIME{0.70f, 11.0f, 12.0f, 24}, SMALL_TIME{0.50f, 6.0f, 5.0f, 16}, DEEP_TIME{0.245f, 6.0f, 8.0f, 16}, FINE_TIME{0.20f, 5.0f, 5.0f, 16};
constexpr int MAX_PARTS = 8;
struct Layout { float us; int whole, cut, parts; };
template <class GEO> Layout layout_of(const GeometryTime& g, int tiles, int slices, int cus)
{
    const int places = cus * GEO::BLOCKS;
    const int whole = tiles / places * places, rem = tiles - whole;
    const float rounds = (float)(whole / places) * (slices * g.slice + g.over);
    Layout best{rounds + (rem ? slices * g.slice + g.over : 0.0f), tiles, 0, 1};
    for (int n = 2; n <= MAX_PARTS && rem > 0 && rem * n <= places && rem < MAX_CUT && slices / n >= g.least; ++n) {
        const float us = rounds + (float)((slices + n - 1) / n) * g.slice + g.over + g.join * (1.0f + 0.25f * (n - 2));
        if (us < best.us) best = Layout{us, whole, rem, n};
    }
    return best;
}

template <int KIND, int OUT, bool ADD, int PLANES, typename WT, class GEO>
hipError_t launch_tiles(Product p, const Layout& l, size_t part_bytes, hipStream_t st)
{
    if ((size_t)l.cut * l.parts * GEO::UNIT_BYTES > part_bytes) return hipErrorInvalidValue;   // the plan has room for any layout (parts_bytes)
    p.row_tiles = (p.M + GEO::BM - 1) / GEO::BM;
    p.col_tiles = (p.N + GEO::BN - 1) / GEO::BN;
    p.tiles = p.symmetric ? p.row_tiles * (p.row_tiles + 1) / 2 : p.row_tiles * p.col_tiles;
    p.whole = l.whole;
    p.whole_per_xcd = (l.whole + 7) / 8;                   // with cut tiles after them they are full rounds: a multiple of 8
    p.cut = l.cut;
    p.parts = l.parts;
    p.part_per_xcd = (l.cut * l.parts + 7) / 8;
    static PerDeviceOnce once;
    const int dev = current_device();
    // (256 x 256 always with the code for parts: one of the kernels without it spills 17 registers)
    auto kern = product_kernel<KIND, OUT, ADD, PLANES, WT, GEO, GEO::NWAVES == 8>;
    auto kern_cut = product_kernel<KIND, OUT, ADD, PLANES, WT, GEO, true>;
    if (!once.is_done(dev)) {
        for (auto k : {kern, kern_cut}) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)GEO::LDS_BYTES);
            if (e != hipSuccess) return e;
        }
        once.mark(dev);
    }
    hipLaunchKernelGGL(l.cut ? kern_cut : kern, dim3(8 * (p.whole_per_xcd + p.part_per_xcd)), dim3(GEO::THREADS), GEO::LDS_BYTES, st, p);
    return hipGetLastError();
}

template <class GEO> int tiles_of(const Product& p, int matrices)
{
    const int rt = (p.M + GEO::BM - 1) / GEO::BM, ct = (p.N + GEO::BN - 1) / GEO::BN;
    return (p.symmetric ? rt * (rt + 1) / 2 : rt * ct) * matrices;
}

template <int KIND, int OUT, bool ADD, int PLANES, typename WT> hipError_t launch_product(const Product& p, int matrices, int cus, size_t part_bytes, hipStream_t st)
{
    const int slices = p.n_seg * (p.K / BK), tiles = tiles_of<Small>(p, matrices);
    const Layout l = layout_of<Large>(LARGE_TIME, tiles_of<Large>(p, matrices), slices, cus), m = layout_of<Small>(SMALL_TIME, tiles, slices, cus);
    if (tiles <= cus) {
        const Layout f = layout_of<Fine>(FINE_TIME, tiles_of<Fine>(p, matrices), slices, cus), d = layout_of<Deep>(DEEP_TIME, tiles, slices, cus);
        if (f.us < d.us && f.us < l.us && f.us < m.us) return launch_tiles<KIND, OUT, ADD, PLANES, WT, Fine>(p, f, part_bytes, st);
        if (d.us < l.us && d.us < m.us) return launch_tiles<KIND, OUT, ADD, PLANES, WT, Deep>(p, d, part_bytes, st);
    }
    return l.us < m.us ? launch_tiles<KIND, OUT, ADD, PLANES, WT, Large>(p, l, part_bytes, st) : launch_tiles<KIND, OUT, ADD, PLANES, WT, Small>(p, m, part_bytes, st);
}

// What the parts of a product's cut tiles take at most: no more than MAX_PARTS of each tile, no more than there are places for blocks.
constexpr int MAX_CUS = 256;
template <class GEO> size_t parts_bytes(const GeometryTime& g, const Product& p, int matrices)
{
    const long units = (long)tiles_of<GEO>(p, matrices) * MAX_PARTS, places = (long)MAX_CUS * GEO::BLOCKS;
    return p.n_seg * (p.K / BK) / 2 < g.least ? 0 : (size_t)(units < places ? units : places) * GEO::UNIT_BYTES;
}
size_t parts_bytes(const Product& p, int matrices)
{
    size_t most = 0;
    for (size_t b : {parts_bytes<Large>(LARGE_TIME, p, matrices), parts_bytes<Small>(SMALL_TIME, p, matrices), parts_bytes<Deep>(DEEP_TIME, p, matrices),
                     parts_bytes<Fine>(FINE_TIME, p, matrices)})
        most = b > most ? b : most;
    return most;
}

// Compute units of the current device, a multiple of 8 (blocks are dealt to 8 XCDs); MAX_CUS at most, which the workspace for parts is sized for.
inline int device_cus()
{
    static std::atomic<int> of[64];
    const int dev = current_device();
    int n = (dev >= 0 && dev < 64) ? of[dev].load(std::memory_order_acquire) : 0;
    if (n == 0) {
        if (dev < 0 || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 8) n = MAX_CUS;
        n = n > MAX_CUS ? MAX_CUS : n / 8 * 8;
        if (dev >= 0 && dev < 64) of[dev].store(n, std::memory_order_release);
    }
    return n;
}

// Steps that are taken on one Gram matrix, see the head of this file.  What a rounding of A amounts to in one direction grows with the share of A
// that one element is, and where the short side is one tile a step costs its launches, of which the form above has fewer (15 for five
// steps, 18).  Off the factor with one | three steps, 11 bits, 8 x 8 3.9e-3 | 3.9e-2, 64 x 64 4.4e-3 | 5.2e-3, 1024 x 1024 4.0e-3 | 4.7e-3;
// 22 bits 1.1e-6 | 1.6e-5, 1.7e-6 | 2.4e-6, 3.3e-6 | 3.7e-6 (fp32 throughout: 0.8e-6, 1.5e-6, 3.6e-6).
inline int steps_per_gram(int m) { return m <= 64 ? 1 : 3; }

inline int round_up64(int x) { return (x + 63) / 64 * 64; }
inline size_t align_ws(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr int MAX_CHUNKS = 256;                            // parts of a matrix' sum of squares: one per thread of the block that adds them
struct MuonPlan {
    int matrices, m, n, mp, np, planes, chunks;
    size_t x_numbers, a_numbers;                           // of all matrices
    size_t part_bytes, off_partial, off_arrived, off_parts, off_x[2], off_a[4], bytes;         // a second plane, where there is one, follows the first
};
// Whether a block takes a whole matrix (few_kernel), and the padded short side it is made for.
inline int few_side(const MuonPlan& p) { return p.mp <= 64 ? 64 : 128; }
inline bool takes_few(const MuonPlan& p)
{
    return p.mp <= (p.planes == 1 ? 128 : 64) && p.m * p.n <= FEW_ELEMENTS && few_lds(few_side(p), p.np, p.planes) <= FEW_LDS;
}
MuonPlan plan_of(const moe_muon_t& c)
{
    MuonPlan p{};
    p.matrices = c.n_tensors * c.count;
    p.m = c.rows < c.cols ? c.rows : c.cols;
    p.n = c.rows < c.cols ? c.cols : c.rows;
    p.mp = round_up64(p.m);
    p.np = round_up64(p.n);
    p.planes = c.dtype == MOE_F32 ? 2 : 1;
    const size_t chunks = ((size_t)p.m * p.n + 8191) / 8192;
    p.chunks = (int)(chunks < MAX_CHUNKS ? chunks : MAX_CHUNKS);
    p.x_numbers = (size_t)p.matrices * p.mp * p.np;
    p.a_numbers = (size_t)p.matrices * p.mp * p.mp;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += align_ws(bytes); return at; };
    p.off_partial = take((size_t)p.matrices * p.chunks * sizeof(double));
    p.off_arrived = take(MAX_CUT * sizeof(int));
    if (!takes_few(p)) {
        Product square{}, product{};
        square.n_seg = product.n_seg = p.planes == 1 ? 1 : 3;
        square.M = square.N = product.M = product.K = p.mp;
        square.K = product.N = p.np;                       // X X^T; the others' contraction is shorter
        square.symmetric = 1;
        const size_t a = parts_bytes(square, p.matrices), b = parts_bytes(product, p.matrices);
        p.part_bytes = a > b ? a : b;
    }
    p.off_parts = take(p.part_bytes);
    for (size_t& x : p.off_x) x = take(p.x_numbers * sizeof(f16) * p.planes);
    for (size_t& a : p.off_a) a = take(p.a_numbers * sizeof(f16) * p.planes);
    p.bytes = off;
    return p;
}

// A batch of matrices in the workspace: its numbers and, with two planes, what they leave off.
struct Stored { f16 *first, *rest; };

template <int PLANES, typename WT>
hipError_t muon_step(const moe_muon_t& c, const float* const* grads, float* const* momenta, void* const* weights, uint16_t* const* copies,
                     int32_t* version, void* ws, hipStream_t st)
{
    const MuonPlan P = plan_of(c);
    char* base = (char*)ws;
    double* partial = (double*)(base + P.off_partial);
    int* arrived = (int*)(base + P.off_arrived);
    const int cus = device_cus();
    auto stored = [&](size_t off, size_t numbers) { f16* f = (f16*)(base + off); return Stored{f, P.planes == 2 ? f + numbers : nullptr}; };
    Stored X = stored(P.off_x[0], P.x_numbers), X2 = stored(P.off_x[1], P.x_numbers);
    const float S = exp2f(fminf(14.0f, floorf(log2f(sqrtf((float)P.m * (float)P.n))))), SA = 1024.0f, SB = 64.0f, SQ = 8.0f;

    Tensors t{};
    for (int i = 0; i < c.n_tensors; ++i) {
        t.grad[i] = grads[i];
        t.momentum[i] = momenta[i];
        // what lies on its short side
        t.transposed[i] = (c.rows <= c.cols) == (c.transposed[i] != 0) && c.rows != c.cols ? 1 : 0;
    }
    const float keep = (float)(1.0 - (double)c.lr * c.weight_decay), rate = (float)((double)c.lr * c.scale / S);
    if (takes_few(P)) {
        Few f{};
        f.m = P.m; f.n = P.n; f.np = P.np; f.count = c.count; f.nesterov = c.nesterov; f.steps = c.steps;
        f.mu = c.momentum; f.eps = c.eps; f.S = S; f.SA = SA; f.SB = SB; f.a = c.a; f.b = c.b; f.c = c.c; f.keep = keep; f.rate = rate;
        for (int i = 0; i < c.n_tensors; ++i) {
            f.grad[i] = grads[i]; f.momentum[i] = momenta[i]; f.W[i] = weights[i]; f.copies[i] = copies ? copies[i] : nullptr; f.transposed[i] = t.transposed[i];
        }
        f.version = version;
        if (few_side(P) == 64) return launch_few<PLANES, 4, WT>(f, P.matrices, st);
        if constexpr (PLANES == 1) return launch_few<PLANES, 8, WT>(f, P.matrices, st);    // two numbers of 128 x 128 twice leave no room for X
    }
    const bool nt = (size_t)P.matrices * P.m * P.n * 8 >= CACHE_BYTES;
    hipLaunchKernelGGL(nt ? momentum_kernel<true> : momentum_kernel<false>, dim3(P.chunks, P.matrices), dim3(256), 0, st, t, c.count, (size_t)P.m * P.n, P.chunks, c.momentum, c.nesterov, partial, arrived);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(nt ? start_kernel<true> : start_kernel<false>, dim3((P.np + START_COLS - 1) / START_COLS, P.mp / 64, P.matrices), dim3(256), 0, st, t, c.count, P.m, P.n, P.mp, P.np,
                       P.chunks, c.momentum, c.nesterov, c.eps, S, partial, X.first, X.rest);
    e = hipGetLastError();

    const long xs = (long)P.mp * P.np, as = (long)P.mp * P.mp;
    auto operands = [&](Product& p, const Stored& a, long a_stride, int lda, const Stored& b, long b_stride, int ldb, int K) {
        p.n_seg = a.rest ? 3 : 1;                          // the small ones first: the sum is rounded at its size in the last segment only
        p.A[p.n_seg - 1] = a.first; p.B[p.n_seg - 1] = b.first;
        if (a.rest) {
            p.A[0] = a.first; p.B[0] = b.rest;
            p.A[1] = a.rest; p.B[1] = b.first;
        }
        p.a_stride = a_stride; p.lda = lda;
        p.b_stride = b_stride; p.ldb = ldb;
        p.K = K;
    };
    // out = alpha A B + beta add + diag I, a symmetric matrix of the short side
    auto square = [&](const Stored& out, const Stored& a, const Stored& b, long stride, int ld, float alpha, const Stored* add, float beta, float diag) {
        if (e != hipSuccess) return;
        Product p{};
        operands(p, a, stride, ld, b, stride, ld, ld);
        p.M = p.N = p.ldo = P.mp; p.o_stride = as; p.symmetric = 1;
        p.part_ws = (float*)(base + P.off_parts); p.arrived = arrived;
        p.alpha = alpha; p.beta = beta; p.diag = diag;
        if (add) { p.D = add->first; p.D_rest = add->rest; }
        p.O = out.first; p.O_rest = out.rest;
        e = add ? launch_product<ROWS, STORE, true, PLANES, float>(p, P.matrices, cus, P.part_bytes, st) : launch_product<ROWS, STORE, false, PLANES, float>(p, P.matrices, cus, P.part_bytes, st);
    };
    const Stored A = stored(P.off_a[0], P.a_numbers);
    for (int left = c.steps, of = 0; left > 0 && e == hipSuccess; left -= of) {
        of = left < steps_per_gram(P.m) ? left : steps_per_gram(P.m);
        Stored B = stored(P.off_a[1], P.a_numbers), Q = B, free0 = stored(P.off_a[2], P.a_numbers), free1 = stored(P.off_a[3], P.a_numbers);
        float q_scale = SB;
        square(A, X, X, xs, P.np, SA / (S * S), nullptr, 0.0f, 0.0f);
        square(B, A, A, as, P.mp, c.c * SB / (SA * SA), &A, c.b * SB / SA, c.a * SB);          // B = a + b A + c A A
        for (int step = 1; step < of; ++step) {
            square(free0, B, A, as, P.mp, 1.0f / SB, nullptr, 0.0f, 0.0f);                     // A <- B A B
            square(A, free0, B, as, P.mp, 1.0f / SB, nullptr, 0.0f, 0.0f);
            const Stored last_B = B, last_Q = Q;
            B = free0;
            square(B, A, A, as, P.mp, c.c * SB / (SA * SA), &A, c.b * SB / SA, c.a * SB);
            Q = step == 1 ? free1 : last_B;                // the first Q is B itself: there is one buffer more to spare then
            square(Q, B, last_Q, as, P.mp, SQ / (SB * q_scale), nullptr, 0.0f, 0.0f);          // Q <- B Q
            q_scale = SQ;
            free0 = last_Q;
        }
        if (e != hipSuccess) break;
        Product q{};                                       // X <- Q X
        operands(q, Q, as, P.mp, X, xs, P.np, P.mp);
        q.M = P.mp; q.N = q.ldo = P.np; q.o_stride = xs;
        q.part_ws = (float*)(base + P.off_parts); q.arrived = arrived;
        q.alpha = 1.0f / q_scale;
        if (of < left) {
            q.O = X2.first; q.O_rest = X2.rest;
            e = launch_product<COLS, STORE, false, PLANES, float>(q, P.matrices, cus, P.part_bytes, st);
            const Stored x = X; X = X2; X2 = x;
        } else {
            q.count = c.count; q.m = P.m; q.n = P.n;
            for (int i = 0; i < c.n_tensors; ++i) { q.transposed[i] = t.transposed[i]; q.W[i] = weights[i]; q.copies[i] = copies ? copies[i] : nullptr; }
            q.keep = keep;
            q.rate = rate;
            q.version = version;
            e = launch_product<COLS, UPDATE, false, PLANES, WT>(q, P.matrices, cus, P.part_bytes, st);
        }
    }
    return e;
}

}  // namespace

size_t muon_workspace_bytes(const moe_muon_t& c) { return plan_of(c).bytes; }

hipError_t launch_muon_step(const moe_muon_t& c, const float* const* grads, float* const* momenta, void* const* weights, uint16_t* const* copies,
                            int32_t* version, void* ws, hipStream_t st)
{
    return c.dtype == MOE_F32 ? muon_step<2, float>(c, grads, momenta, weights, copies, version, ws, st)
                              : muon_step<1, bf16_t>(c, grads, momenta, weights, copies, version, ws, st);
}
