// The layer norm of a pre-norm block with the sum of the residual stream, and its gradient.
//
// forward, per row of d elements:  s = x + r (rounded once to the element type),  mean = sum s / d,
//   rstd = 1 / sqrt(sum (s - mean)^2 / d + eps),  y = (s - mean) rstd gamma + beta
// backward, with xh = (s - mean) rstd, g = dy gamma, c1 = sum g / d, c2 = sum g xh / d:
//   dx = ds + rstd (g - c1 - xh c2);  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Bound by HBM: two to four elements move per element of the rows and a dozen vector instructions go with them.  A row
// is read once: it stays in the registers of the TPR threads that share it, U pieces of 16 bytes each, through both of the forward sums
// (the variance is that of the centred row, not a difference of squares).  Sums are fp32 and in a fixed order.
//
// Measured on buffers that change from call to call, bf16 with a residual: 32768 x 4096 forward 184 us, 5.8 TB/s, backward with the parameters'
// gradients 174, 6.2 TB/s (512 partial sums and no row ahead 207; rows through the caches, with stores and loads as usual, 192 and 207);
// 16384 x 2048 47 and 52.  One row of 2048: 3.4 us on the GPU.
#include "internal.h"

#include <type_traits>

namespace {

// 16 bytes of a row.  Rows of odd widths begin at any multiple of an element; the memory path takes such requests whole.
template <typename ET> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    typedef unsigned mem_t __attribute__((ext_vector_type(4), aligned(4)));
    typedef float one_t;
    static __device__ __forceinline__ void unpack(const moe_piece_t& v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ moe_piece_t pack(const float* f) {
        return moe_piece_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    typedef unsigned mem_t __attribute__((ext_vector_type(4), aligned(2)));
    typedef bf16_t one_t;
    static __device__ __forceinline__ void unpack(const moe_piece_t& v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ moe_piece_t pack(const float* f) {
        return moe_piece_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    }
};

// TAIL: a row's last piece is short, `n` of its N elements are inside the row (elsewhere n = N, or 0 and less where a thread has no piece).
//   1  It is requested as the row's last N elements, those of the piece before it among them, and moved down when it is used (settle): nothing is
//      waited for where the request is made, which is a row ahead in the backward pass (the gradient of 20000 x 2500 in bf16 117 us, of 20000 x 2496 91).
//   2  Element by element: rows shorter than a piece, and the forward pass, which waits for its row at once (59811 x 2244 230 us, moved down 250;
//      20000 x 5001 192, 235; the gradient of 20000 x 2500 291).
// NT: past the caches (STREAM_BYTES).
template <typename ET, int TAIL, bool NT> __device__ __forceinline__ moe_piece_t load_row_piece(const ET* row, int col, int n, int d)
{
    typedef typename Piece<ET>::mem_t mem_t;
    constexpr int N = Piece<ET>::N;
    if (TAIL == 2 && n < N) {
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (std::is_same<ET, float>::value) f[i] = i < n ? row[col + i] : 0.0f;
            else f[i] = i < n ? bf16_to_f32(row[col + i]) : 0.0f;
        }
        return Piece<ET>::pack(f);
    }
    const mem_t* p = reinterpret_cast<const mem_t*>(row + (TAIL == 1 && n < N ? d - N : col));
    if constexpr (NT) return __builtin_nontemporal_load(p);
    else return *p;
}
template <typename ET, int TAIL> __device__ __forceinline__ void settle(moe_piece_t& v, int n, int d)
{
    constexpr int N = Piece<ET>::N;
    if (TAIL != 1 || n >= N || n <= 0) return;
    int bits = (N - n) * (int)sizeof(ET) * 8;              // zeros come in at the end
    uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
    if (bits >= 64) { lo = hi; hi = 0; bits -= 64; }
    if (bits > 0) { lo = lo >> bits | hi << (64 - bits); hi >>= bits; }
    v = moe_piece_t{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    // The gradient may be written over dY or dS.  A short piece's request reads columns of the piece before it, which a thread of another wave stores once
    // it is past the barrier of the row's sums: what was requested has arrived here, and this stays ahead of that barrier, also for dS, which
    // nothing uses until after it (20000 x 2500 in bf16 109 -> 117 us, 4000 x 16383 in fp32 417 -> 402, most widths as before).
    asm volatile("" : "+v"(v));
}
template <typename ET, int TAIL, bool NT> __device__ __forceinline__ void store_row_piece(ET* p, const moe_piece_t& v, int n)
{
    typedef typename Piece<ET>::mem_t mem_t;
    constexpr int N = Piece<ET>::N;
    if (!TAIL || n == N) {
        if constexpr (NT) __builtin_nontemporal_store((mem_t)v, reinterpret_cast<mem_t*>(p));
        else *reinterpret_cast<mem_t*>(p) = v;
        return;
    }
    typedef unsigned two_t __attribute__((ext_vector_type(2), aligned(2)));
    typedef unsigned one_t __attribute__((aligned(2)));
    const int words = n * (int)sizeof(ET) / 4;             // whole 32-bit words
    if (words & 2) *reinterpret_cast<two_t*>(p) = two_t{v[0], v[1]};
    if (words & 1) *reinterpret_cast<one_t*>(p + (words & 2) * 4 / sizeof(ET)) = words & 2 ? v[2] : v[0];
    if constexpr (N == 8)
        if (n & 1) p[n - 1] = (bf16_t)(words == 0 ? v[0] : words == 1 ? v[1] : words == 2 ? v[2] : v[3]);
}
// The parameters of a piece's columns; zeros past the row's end.
template <int N, int TAIL> __device__ __forceinline__ void load_columns(const float* all, int col, int n, int d, float* f)
{
    typedef float quad_t __attribute__((ext_vector_type(4), aligned(4)));
    if (TAIL == 2 && n < N) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = i < n ? all[col + i] : 0.0f;
        return;
    }
    const float* p = all + (TAIL == 1 && n < N ? d - N : col);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const quad_t q = *reinterpret_cast<const quad_t*>(p + 4 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[4 * i + k] = q[k];
    }
    if (TAIL == 1 && n < N) {
        const int k = N - n;
#pragma unroll
        for (int step = N / 2; step >= 1; step /= 2)
            if (k & step)
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = i + step < N ? f[i + step] : 0.0f;
    }
}

// Rows of a wave or less share a block of 256; the threads of a wider one are the block.
constexpr int threads_of(int tpr) { return tpr > 64 ? tpr : 256; }

// Sums of M values over the TPR threads of a row, the same bits in each of them.  Rows of more than a wave go through `words`
// (LDS, M x waves floats); two sets of them in turn, so that one barrier a sum is enough.
template <int TPR, int M> __device__ __forceinline__ void row_sums(float (&v)[M], float* words, int& turn)
{
#pragma unroll
    for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] += __shfl_xor(v[i], off, 64);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* w = words + turn * (2 * W);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < M; ++i) w[i * W + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < M; ++i) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) s += w[i * W + k];
            v[i] = s;
        }
    }
}

template <typename ET, int TPR, int U, int TAIL, bool NT>
__global__ __launch_bounds__(threads_of(TPR)) void norm_fwd_kernel(
    const ET* X, const ET* R, const float* __restrict__ gamma, const float* __restrict__ beta, ET* S, ET* Y,
    float* __restrict__ mean_out, float* __restrict__ rstd_out, int rows, int d, float eps)
{
    constexpr int N = Piece<ET>::N, RPB = threads_of(TPR) / TPR;
    __shared__ float words[TPR > 64 ? 4 * (TPR / 64) : 1];
    int turn = 0;
    const int c = threadIdx.x % TPR;
    const float inv_d = 1.0f / (float)d;
    int n[U];                                              // elements of a piece inside the row
#pragma unroll
    for (int u = 0; u < U; ++u) n[u] = min(N, max(0, d - (c + u * TPR) * N));
    // rows of a block are a block apart from the next block's; the threads of a row leave the loop together
    for (long row = (long)blockIdx.x * RPB + threadIdx.x / TPR; row < rows; row += (long)gridDim.x * RPB) {
        const size_t base = (size_t)row * d;
        moe_piece_t x[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = moe_piece_t{0, 0, 0, 0};
            if (n[u] > 0) x[u] = load_row_piece<ET, TAIL, NT>(X + base, (c + u * TPR) * N, n[u], d);
        }
        if (R) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                r[u] = moe_piece_t{0, 0, 0, 0};
                if (n[u] > 0) r[u] = load_row_piece<ET, TAIL, NT>(R + base, (c + u * TPR) * N, n[u], d);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float a[N], b[N];
                settle<ET, TAIL>(x[u], n[u], d);
                settle<ET, TAIL>(r[u], n[u], d);
                Piece<ET>::unpack(x[u], a);
                Piece<ET>::unpack(r[u], b);
#pragma unroll
                for (int i = 0; i < N; ++i) a[i] += b[i];
                x[u] = Piece<ET>::pack(a);
                if (n[u] > 0) store_row_piece<ET, TAIL, NT>(S + base + (c + u * TPR) * N, x[u], n[u]);
            }
        }
        if (!R)
#pragma unroll
            for (int u = 0; u < U; ++u) settle<ET, TAIL>(x[u], n[u], d);
        float sum[1] = {0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float a[N];
            Piece<ET>::unpack(x[u], a);                    // zeros past the row's end
#pragma unroll
            for (int i = 0; i < N; ++i) sum[0] += a[i];
        }
        row_sums<TPR>(sum, words, turn);
        const float mean = sum[0] * inv_d;
        float sq[1] = {0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float a[N];
            Piece<ET>::unpack(x[u], a);
            if (n[u] > 0)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float v = (!TAIL || i < n[u]) ? a[i] - mean : 0.0f;
                    sq[0] = fmaf(v, v, sq[0]);
                }
        }
        row_sums<TPR>(sq, words, turn);
        const float rstd = 1.0f / sqrtf(fmaf(sq[0], inv_d, eps));
        if (mean_out && c == 0) { mean_out[row] = mean; rstd_out[row] = rstd; }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n[u] <= 0) continue;
            float a[N], g[N], b[N];
            Piece<ET>::unpack(x[u], a);
            load_columns<N, TAIL>(gamma, (c + u * TPR) * N, n[u], d, g);
#pragma unroll
            for (int i = 0; i < N; ++i) b[i] = 0.0f;
            if (beta) load_columns<N, TAIL>(beta, (c + u * TPR) * N, n[u], d, b);
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = fmaf((a[i] - mean) * rstd, g[i], b[i]);
            store_row_piece<ET, TAIL, NT>(Y + base + (c + u * TPR) * N, Piece<ET>::pack(a), n[u]);
        }
    }
}

// Columns stay with their thread from row to row, so the parameters' gradients are summed in registers; a block leaves one partial
// sum of each in `partial`, [block][2][d]; a block that is alone (partial null) the gradients themselves.
template <typename ET, int TPR, int U, int TAIL, bool NT>
__global__ __launch_bounds__(threads_of(TPR)) void norm_bwd_kernel(
    const ET* dY, const ET* __restrict__ S, const float* __restrict__ gamma, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
    const ET* dS, ET* dX, float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int rows, int d)
{
    constexpr int N = Piece<ET>::N, RPB = threads_of(TPR) / TPR, COLS = TPR * U * N;
    __shared__ float words[TPR > 64 ? 4 * (TPR / 64) : 1];
    __shared__ float join[RPB > 1 ? RPB * COLS : 1];
    int turn = 0;
    const int c = threadIdx.x % TPR, in_block = threadIdx.x / TPR;
    const float inv_d = 1.0f / (float)d;
    // gamma of more than 16 columns (8 where a wave has 128 registers) is read again for every row: with it the registers would not hold the sums
    constexpr bool KEEP_GAMMA = U * N <= (TPR > 512 ? 8 : 16);
    float g[KEEP_GAMMA ? U : 1][N], sg[U][N], sb[U][N];
    int n[U];
#pragma unroll
    for (int u = 0; u < U; ++u) n[u] = min(N, max(0, d - (c + u * TPR) * N));
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < N; ++i) sg[u][i] = sb[u][i] = 0.0f;
        if constexpr (KEEP_GAMMA) {
#pragma unroll
            for (int i = 0; i < N; ++i) g[u][i] = 0.0f;
            if (n[u] > 0) load_columns<N, TAIL>(gamma, (c + u * TPR) * N, n[u], d, g[u]);
        }
    }
    auto columns = [&](int u) -> float (&)[N] {
        if constexpr (KEEP_GAMMA) {
            return g[u];
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) g[0][i] = 0.0f;
            if (n[u] > 0) load_columns<N, TAIL>(gamma, (c + u * TPR) * N, n[u], d, g[0]);
            return g[0];
        }
    };
    // The next row is on its way while this one is worked on (32768 x 4096: 232 us without).
    moe_piece_t ny[U], ns[U], nr[U];
    float n_mean = 0.0f, n_rstd = 0.0f;
    auto request = [&](long row) {
        const size_t base = (size_t)row * d;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ny[u] = ns[u] = nr[u] = moe_piece_t{0, 0, 0, 0};
            if (n[u] > 0) {
                ny[u] = load_row_piece<ET, TAIL, NT>(dY + base, (c + u * TPR) * N, n[u], d);
                ns[u] = load_row_piece<ET, TAIL, NT>(S + base, (c + u * TPR) * N, n[u], d);
                if (dS) nr[u] = load_row_piece<ET, TAIL, NT>(dS + base, (c + u * TPR) * N, n[u], d);
            }
        }
        n_mean = mean_in[row];
        n_rstd = rstd_in[row];
    };
    const long row0 = (long)blockIdx.x * RPB + in_block, row_step = (long)gridDim.x * RPB;
    constexpr bool AHEAD = U < 4;                          // four pieces and the next four do not fit the registers
    if (AHEAD && row0 < rows) request(row0);
    for (long row = row0; row < rows; row += row_step) {
        const size_t base = (size_t)row * d;
        moe_piece_t py[U], ps[U], pr[U];
        if (!AHEAD) request(row);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            py[u] = ny[u]; ps[u] = ns[u]; pr[u] = nr[u];
            settle<ET, TAIL>(py[u], n[u], d);
            settle<ET, TAIL>(ps[u], n[u], d);
            settle<ET, TAIL>(pr[u], n[u], d);
        }
        const float mean = n_mean, rstd = n_rstd;
        if (AHEAD && row + row_step < rows) request(row + row_step);
        float c12[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float y[N], s[N];
            float (&gm)[N] = columns(u);
            Piece<ET>::unpack(py[u], y);                   // zeros past the row's end, and gamma too
            Piece<ET>::unpack(ps[u], s);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float xh = (s[i] - mean) * rstd, gy = y[i] * gm[i];
                c12[0] += gy;
                c12[1] = fmaf(gy, xh, c12[1]);
                sg[u][i] = fmaf(y[i], xh, sg[u][i]);
                sb[u][i] += y[i];
            }
        }
        row_sums<TPR>(c12, words, turn);
        const float c1 = c12[0] * inv_d, c2 = c12[1] * inv_d;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n[u] <= 0) continue;
            float y[N], s[N], r[N];
            float (&gm)[N] = columns(u);
            Piece<ET>::unpack(py[u], y);
            Piece<ET>::unpack(ps[u], s);
            Piece<ET>::unpack(pr[u], r);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float xh = (s[i] - mean) * rstd;
                r[i] = fmaf(rstd, fmaf(-xh, c2, fmaf(y[i], gm[i], -c1)), r[i]);
            }
            store_row_piece<ET, TAIL, NT>(dX + base + (c + u * TPR) * N, Piece<ET>::pack(r), n[u]);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float* out = partial ? partial + ((size_t)blockIdx.x * 2 + k) * d : (k ? dbeta : dgamma);
        if (!out) continue;                                // no bias
        if constexpr (RPB > 1) {
            __syncthreads();                               // the rows of a block are joined in LDS
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) join[in_block * COLS + i * (TPR * U) + u * TPR + c] = k ? sb[u][i] : sg[u][i];
            __syncthreads();
            for (int j = threadIdx.x; j < COLS; j += threads_of(TPR)) {
                float s = 0.0f;
#pragma unroll
                for (int b = 0; b < RPB; ++b) s += join[b * COLS + j];
                const int col = (j % (TPR * U)) * N + j / (TPR * U);
                if (col < d) out[col] = s;
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n[u]) out[(c + u * TPR) * N + i] = k ? sb[u][i] : sg[u][i];
        }
    }
}

// The partial sums of 32 columns, 32 lines of them at a time; their order is fixed by the number of blocks.
constexpr int JOIN_COLS = 32, JOIN_LINES = 32;
__global__ __launch_bounds__(JOIN_COLS * JOIN_LINES) void norm_join_kernel(const float* __restrict__ partial, int blocks, int d,
                                                                         float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float words[JOIN_LINES][JOIN_COLS + 1];
    const int col = blockIdx.x * JOIN_COLS + threadIdx.x % JOIN_COLS, line = threadIdx.x / JOIN_COLS;
    float s = 0.0f;
    if (col < 2 * d)
#pragma unroll 8
        for (int b = line; b < blocks; b += JOIN_LINES) s += partial[(size_t)b * 2 * d + col];
    words[line][threadIdx.x % JOIN_COLS] = s;
    __syncthreads();
    if (line != 0 || col >= 2 * d) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < JOIN_LINES; ++i) t += words[i][threadIdx.x];
    if (col < d) dgamma[col] = t;
    else if (dbeta) dbeta[col - d] = t;
}

// Threads of a row and pieces of each, by the width.  Forward: a wave up to eight pieces a thread, so that most rows need no barrier and every
// thread has several requests on their way (59811 x 2240 in 5 pieces of 64 threads 178 us, 2 of 256 207; 32768 x 4096 in 8 of 64 184, 4 of 128 192, 2 of
// 256 184).  Backward, with the parameters' gradients in registers beside the row: two pieces where the threads are there (a wave of one piece instead
// of 16 threads of four: 16184 x 467 28 -> 18).
template <typename ET, bool BWD, typename F> hipError_t by_width(int d, bool nt, F f)
{
    const int nv = (d + Piece<ET>::N - 1) / Piece<ET>::N;
    const bool tail = d % Piece<ET>::N != 0;
    typedef std::integral_constant<int, 0> whole_t;
    typedef std::integral_constant<int, 2> short_t;
    typedef std::integral_constant<int, BWD ? 1 : 2> tail_t;
    if (d < Piece<ET>::N) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, short_t{}, std::false_type{});
    auto with = [&](auto TPR, auto U) {
        if (nt) return tail ? f(TPR, U, tail_t{}, std::true_type{}) : f(TPR, U, whole_t{}, std::true_type{});
        return tail ? f(TPR, U, tail_t{}, std::false_type{}) : f(TPR, U, whole_t{}, std::false_type{});
    };
#define MOE_NORM_CASE(T, UU) if (nv <= T * UU) return with(std::integral_constant<int, T>{}, std::integral_constant<int, UU>{});
    MOE_NORM_CASE(16, 1)
    MOE_NORM_CASE(16, 2)
    if constexpr (BWD) { MOE_NORM_CASE(64, 1) } else { MOE_NORM_CASE(16, 4) }
    MOE_NORM_CASE(64, 2)
    if constexpr (BWD) {
        MOE_NORM_CASE(256, 1)
        MOE_NORM_CASE(256, 2)
        MOE_NORM_CASE(256, 3)
        MOE_NORM_CASE(512, 2)
        MOE_NORM_CASE(512, 3)
        MOE_NORM_CASE(512, 4)
    } else {
        MOE_NORM_CASE(64, 3)
        MOE_NORM_CASE(64, 4)
        MOE_NORM_CASE(64, 5)
        MOE_NORM_CASE(64, 6)
        MOE_NORM_CASE(64, 8)
        MOE_NORM_CASE(256, 3)
        MOE_NORM_CASE(256, 4)
        MOE_NORM_CASE(1024, 2)
    }
    if constexpr (Piece<ET>::N == 4) { MOE_NORM_CASE(1024, 4) }
#undef MOE_NORM_CASE
    return hipErrorInvalidValue;                           // wider than NORM_MAX_D: the entry points refuse it
}

// Blocks of the backward pass.  Each leaves a partial sum of the parameters' gradients, 8 d bytes written and read again, and needs rows
// enough to be worth it: four at least for each group of threads (rows x d bf16, us with 1 | 4 | 8: 4096 x 1024 13.9 | 12.0 | 14.6, 512 x 4096
// 16.1 | 15.0 | 17.8), but for the first 64 blocks, which cost next to nothing (512 x 64 in fp32, the kernel: 32 blocks 3.3, 8 blocks 4.8), unless a block
// alone, which needs no second launch, has them all.  Rows of two pieces a thread and more keep enough on their way with one block of 256 on a CU (32768 x 4096: 512 blocks 187, 256
// 175), others do not (16384 x 2048: 52, 64).
constexpr int MIN_ROWS = 4, FREE_BLOCKS = 64;
inline int blocks_for(int rows, int tpr, int most)
{
    const int rpb = threads_of(tpr) / tpr, n = (rows - 1) / rpb + 1;
    return n < most ? n : most;
}

template <typename ET>
hipError_t norm_fwd(const moe_norm_t& c, const void* X, const void* R, const float* gamma, const float* beta, void* S, void* Y,
                    float* mean, float* rstd, hipStream_t st)
{
    return by_width<ET, false>(c.d, streams((size_t)c.rows * c.d * sizeof(ET)), [&](auto TPR, auto U, auto TAIL, auto NT) {
        constexpr int tpr = decltype(TPR)::value;
        hipLaunchKernelGGL((norm_fwd_kernel<ET, tpr, decltype(U)::value, decltype(TAIL)::value, decltype(NT)::value>), dim3(blocks_for(c.rows, tpr, 1 << 20)), dim3(threads_of(tpr)), 0, st,
                           (const ET*)X, (const ET*)R, gamma, beta, (ET*)S, (ET*)Y, mean, rstd, c.rows, c.d, c.eps);
        return hipGetLastError();
    });
}

template <typename ET>
hipError_t norm_bwd(const moe_norm_t& c, const void* dY, const void* S, const float* gamma, const float* mean, const float* rstd, const void* dS,
                    void* dX, float* dgamma, float* dbeta, float* partial, hipStream_t st)
{
    int blocks = 0;
    hipError_t e = c.rows == 0 ? hipSuccess : by_width<ET, true>(c.d, streams((size_t)c.rows * c.d * sizeof(ET)), [&](auto TPR, auto U, auto TAIL, auto NT) {
        constexpr int tpr = decltype(TPR)::value;
        constexpr int wide = tpr >= 256 && decltype(U)::value >= 2;
        blocks = blocks_for((c.rows + MIN_ROWS - 1) / MIN_ROWS, tpr, wide ? NORM_PARTIALS / 2 : NORM_PARTIALS);
        if (blocks > 1 && blocks < FREE_BLOCKS) blocks = blocks_for(c.rows, tpr, FREE_BLOCKS);
        hipLaunchKernelGGL((norm_bwd_kernel<ET, tpr, decltype(U)::value, decltype(TAIL)::value, decltype(NT)::value>), dim3(blocks), dim3(threads_of(tpr)), 0, st,
                           (const ET*)dY, (const ET*)S, gamma, mean, rstd, (const ET*)dS, (ET*)dX, blocks > 1 ? partial : nullptr, dgamma, dbeta, c.rows, c.d);
        return hipGetLastError();
    });
    if (e != hipSuccess || blocks == 1) return e;
    hipLaunchKernelGGL(norm_join_kernel, dim3((2 * c.d + JOIN_COLS - 1) / JOIN_COLS), dim3(JOIN_COLS * JOIN_LINES), 0, st, partial, blocks, c.d, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_fwd(const moe_norm_t& c, const void* X, const void* R, const float* gamma, const float* beta, void* S, void* Y,
                           float* mean, float* rstd, hipStream_t st)
{
    if (c.rows == 0) return hipSuccess;
    return c.dtype == MOE_F32 ? norm_fwd<float>(c, X, R, gamma, beta, S, Y, mean, rstd, st) : norm_fwd<bf16_t>(c, X, R, gamma, beta, S, Y, mean, rstd, st);
}

hipError_t launch_norm_bwd(const moe_norm_t& c, const void* dY, const void* S, const float* gamma, const float* mean, const float* rstd, const void* dS,
                           void* dX, float* dgamma, float* dbeta, float* partial, hipStream_t st)
{
    return c.dtype == MOE_F32 ? norm_bwd<float>(c, dY, S, gamma, mean, rstd, dS, dX, dgamma, dbeta, partial, st)
                              : norm_bwd<bf16_t>(c, dY, S, gamma, mean, rstd, dS, dX, dgamma, dbeta, partial, st);
}
