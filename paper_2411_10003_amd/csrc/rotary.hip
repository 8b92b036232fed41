// Queries and keys on their way from the projection to their products: RMS norm of each head, rotation by the position, and for an answer's tokens the
// way into the cache, in one pass; and its gradient.
//
// forward, per head x of d elements:  x <- x rstd gamma, rstd = 1 / sqrt(sum x^2 / d + eps);  pairs (a, b) of its first `rot` columns
//   (a, b) <- amplitude (a cos t - b sin t, b cos t + a sin t),  t = position * frequency
// backward: dy turned back by the same angle, then with xh = x rstd, g = dy gamma:  dx = rstd (g - xh sum g xh / d),  dgamma = sum dy xh
//
// Bound by HBM: an element comes and goes once.  A head is shared by TPH threads with two pieces of eight elements each, which stay in registers; where
// the halves of a head are pairs and whole pieces, a thread has both pieces of its pairs and no word goes between lanes.  Angles are 64-bit products reduced
// to a turn before they are rounded (a position of 10^6 leaves fp32 two digits of its angle), once per row for all heads, kept in LDS.
//
// 32768 rows of 32 and 8 heads of 128, bf16, norms: forward 671 MB in 131 us (5.1 TB/s), gradient 1006 MB in 205 us (4.9 TB/s); a large copy reaches 5.2 TB/s.
// 16 tokens into a cache 4.7 us, one launch; 512 rows of 2 and 2 heads of 32, fp32, gradient with norms 9.1 us, two launches.
#include "internal.h"

#include <type_traits>

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, PIECE = 8, MAX_ANGLES = 512;   // angles that a block keeps at a time

struct side_t { const char *in, *x; char* out; const float* gamma; int heads; long long in_row, in_head, x_row, x_head, out_row, out_head; };      // strides in bytes
struct rotary_args {
    side_t side[3];                                        // queries, keys, values
    const int32_t *positions, *slots;
    const double* frequencies;
    float* partial;                                        // [blocks][d]
    float *dgamma_q, *dgamma_k;
    int rows, d, rot, sides, out_rows, rows_at_once, rows_at_once_k, blocks_q;
    float eps, amplitude, inv_d;
};

constexpr int LANE = 2 * PIECE + 1;                        // words from one lane's elements in LDS to the next lane's
enum Pairs { NEIGHBOURS, HALVES, HALVES_CUT };             // CUT: a half is no whole number of pieces

// A piece as it lies in memory, and its numbers.
template <typename ET> struct Raw { u32x4 w[sizeof(ET) / 2]; };
template <typename ET, bool NT> __device__ __forceinline__ Raw<ET> load_raw(const char* p)
{
    Raw<ET> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(ET) / 2; ++i) r.w[i] = load_piece_of<NT>((const u32x4*)p + i);
    return r;
}
template <typename ET> __device__ __forceinline__ void unpack(const Raw<ET>& r, float* f)
{
    if constexpr (sizeof(ET) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(r.w[0][i] << 16); f[2 * i + 1] = __uint_as_float(r.w[0][i] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(r.w[i / 4][i % 4]);
    }
}
template <typename ET, bool NT> __device__ __forceinline__ void load8(const char* p, float* f) { unpack<ET>(load_raw<ET, NT>(p), f); }
template <typename ET, bool NT> __device__ __forceinline__ void store8(char* p, const float* f)
{
    if constexpr (sizeof(ET) == 2) {
        store_piece_of<NT>((u32x4*)p, u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])});
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) store_piece_of<NT>((f32x4*)p + i, f32x4{f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]});
    }
}

// The two pieces of thread c of a head, by their index; one at or past d / 8 is not there.
template <Pairs PAIRS> __device__ __forceinline__ void pieces_of(int c, int rot, int (&p)[2])
{
    const int pairs = PAIRS == HALVES ? rot / (2 * PIECE) : 0;
    if (PAIRS == HALVES && c < pairs) { p[0] = c; p[1] = c + pairs; }
    else { p[0] = 2 * c; p[1] = 2 * c + 1; }               // 2 pairs + 2 (c - pairs)
}

// Turns the pairs among a thread's two pieces; angles: cosines and sines of the row.  BACK: the other way.
template <Pairs PAIRS, bool BACK>
__device__ __forceinline__ void turn(float (&v)[2][PIECE], const int (&p)[2], const float2* angles, int rot, float* mine, int c)
{
    auto pair = [](float& a, float& b, float2 t) {
        const float s = BACK ? -t.y : t.y, x = a * t.x - b * s, y = b * t.x + a * s;
        a = x;
        b = y;
    };
    if constexpr (PAIRS == NEIGHBOURS) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < PIECE / 2; ++i) {
                const int at = p[u] * (PIECE / 2) + i;
                if (2 * at < rot) pair(v[u][2 * i], v[u][2 * i + 1], angles[at]);
            }
    } else if constexpr (PAIRS == HALVES) {
        if (p[0] * PIECE * 2 < rot) {
#pragma unroll
            for (int i = 0; i < PIECE; ++i) pair(v[0][i], v[1][i], angles[p[0] * PIECE + i]);
        }
    } else {
        // through LDS: a head's threads are lanes of one wave; a word more between lanes keeps them to banks of their own (2898 rows of 16 and 4 heads of 128, 110 turned: 21.2 -> 12.0 us)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < PIECE; ++i) mine[c * LANE + u * PIECE + i] = v[u][i];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < PIECE; ++i) {
                const int at = p[u] * PIECE + i;
                if (at >= rot) continue;
                const bool low = at < rot / 2;
                const int other = low ? at + rot / 2 : at - rot / 2;
                const float w = mine[other + other / (2 * PIECE)];
                float a = low ? v[u][i] : w, b = low ? w : v[u][i];
                pair(a, b, angles[low ? at : at - rot / 2]);
                v[u][i] = low ? a : b;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

template <int TPH, int M> __device__ __forceinline__ void head_sums(float (&v)[M])
{
#pragma unroll
    for (int off = TPH / 2; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] += __shfl_xor(v[i], off, 64);
}

// Cosines and sines, times the amplitude, of `n` rows from `row` on.
__device__ __forceinline__ void make_angles(const rotary_args& a, int row, int n, float2* angles)
{
    const int half = a.rot / 2;
    for (int i = threadIdx.x; i < n * half; i += THREADS) {
        const int r = i / half;
        double t = (double)a.positions[row + r] * a.frequencies[i - r * half] * 0.15915494309189533577;      // in turns
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        angles[i] = make_float2(c * a.amplitude, s * a.amplitude);
    }
}

template <typename ET, int TPH, Pairs PAIRS, bool NORM, bool NT>
__global__ __launch_bounds__(THREADS) void rotary_kernel(rotary_args a)
{
    constexpr int GROUPS = THREADS / TPH;
    __shared__ float2 angles[MAX_ANGLES];
    __shared__ float patch[PAIRS == HALVES_CUT ? GROUPS * TPH * LANE : 1];
    const int c = threadIdx.x % TPH, group = threadIdx.x / TPH, first = blockIdx.x * a.rows_at_once, n = min(a.rows_at_once, a.rows - first);
    int p[2];
    pieces_of<PAIRS>(c, a.rot, p);
    const bool there[2] = {p[0] * PIECE < a.d, p[1] * PIECE < a.d};
    // a block has all sides of its rows, or one of them where there are few rows
    const int side0 = gridDim.y > 1 ? blockIdx.y : 0, side1 = gridDim.y > 1 ? side0 + 1 : a.sides;
    if (side0 < 2) {
        make_angles(a, first, n, angles);
        __syncthreads();
    }
    for (int k = side0; k < side1; ++k) {
        const side_t& s = a.side[k];
        float gamma[2][PIECE];
        if (NORM && k < 2)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < PIECE; ++i) gamma[u][i] = there[u] ? s.gamma[p[u] * PIECE + i] : 0.0f;
        const int items = n * s.heads;
        for (int i0 = 0; i0 < items; i0 += GROUPS) {
            const int item = i0 + group;
            const bool on = item < items;
            const int r = on ? item / s.heads : 0, h = on ? item - r * s.heads : 0, row = first + r;
            const char* in = s.in + row * s.in_row + h * s.in_head;
            float v[2][PIECE];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (on && there[u]) load8<ET, NT>(in + p[u] * PIECE * (int)sizeof(ET), v[u]);
                else
#pragma unroll
                    for (int i = 0; i < PIECE; ++i) v[u][i] = 0.0f;
            }
            const int to = k > 0 && a.slots ? a.slots[row] : row;
            const bool kept = on && (k == 0 || !a.slots || (unsigned)to < (unsigned)a.out_rows);
            if (k < 2) {
                if constexpr (NORM) {
                    float sq[1] = {0.0f};
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < PIECE; ++i) sq[0] = fmaf(v[u][i], v[u][i], sq[0]);
                    head_sums<TPH>(sq);
                    const float rstd = 1.0f / sqrtf(sq[0] * a.inv_d + a.eps);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < PIECE; ++i) v[u][i] *= rstd * gamma[u][i];
                }
                turn<PAIRS, false>(v, p, angles + r * (a.rot / 2), a.rot, patch + group * TPH * LANE, c);
            }
            char* out = s.out + to * s.out_row + h * s.out_head;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (kept && there[u]) store8<ET, NT>(out + p[u] * PIECE * (int)sizeof(ET), v[u]);
        }
    }
}

// The gradient.  A block works on queries or on keys (the first blocks_q of them), the next head's pieces under way while it works on one.  Columns stay with their
// thread from head to head, so a norm's parameters are summed in registers, then over the block's groups in LDS, then over the blocks by a second launch.
template <typename ET, int TPH, Pairs PAIRS, bool NORM, bool NT>
__global__ __launch_bounds__(THREADS) void rotary_bwd_kernel(rotary_args a)
{
    constexpr int GROUPS = THREADS / TPH;
    __shared__ float2 angles[MAX_ANGLES];
    __shared__ float patch[PAIRS == HALVES_CUT || NORM ? GROUPS * TPH * LANE : 1];
    const int c = threadIdx.x % TPH, group = threadIdx.x / TPH;
    const bool keys = (int)blockIdx.x >= a.blocks_q;
    const side_t s = keys ? a.side[1] : a.side[0];
    const int block = keys ? blockIdx.x - a.blocks_q : blockIdx.x, blocks = keys ? gridDim.x - a.blocks_q : a.blocks_q, at_once = keys ? a.rows_at_once_k : a.rows_at_once;
    int p[2];
    pieces_of<PAIRS>(c, a.rot, p);
    const bool there[2] = {p[0] * PIECE < a.d, p[1] * PIECE < a.d};
    float dg[2][PIECE], gamma[2][PIECE];
    if constexpr (NORM)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < PIECE; ++i) {
                dg[u][i] = 0.0f;
                gamma[u][i] = there[u] ? s.gamma[p[u] * PIECE + i] : 0.0f;
            }
    Raw<ET> next_v[2], next_x[2];
    // head `item` of the rows from `first` on, if there is one
    auto fetch = [&](long long first, int items, int item) __attribute__((always_inline)) {
        const bool on = item < items;
        const int r = on ? item / s.heads : 0, h = on ? item - r * s.heads : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = p[u] * PIECE * (int)sizeof(ET);
            next_v[u] = next_x[u] = Raw<ET>{};
            if (on && there[u]) {
                next_v[u] = load_raw<ET, NT>(s.in + (first + r) * s.in_row + h * s.in_head + at);
                if constexpr (NORM) next_x[u] = load_raw<ET, NT>(s.x + (first + r) * s.x_row + h * s.x_head + at);
            }
        }
    };
    auto items_of = [&](long long first) __attribute__((always_inline)) { return first < a.rows ? (int)min((long long)at_once, a.rows - first) * s.heads : 0; };
    const long long stride = (long long)blocks * at_once;
    long long first = (long long)block * at_once;
    fetch(first, items_of(first), group);
    for (; first < a.rows; first += stride) {
        const int items = items_of(first);
        __syncthreads();                                   // the angles of the rows before are done with
        make_angles(a, (int)first, items / s.heads, angles);
        __syncthreads();
        for (int i0 = 0; i0 < items; i0 += GROUPS) {
            const int item = i0 + group;
            const bool on = item < items;
            const int r = on ? item / s.heads : 0, h = on ? item - r * s.heads : 0;
            float v[2][PIECE], x[2][PIECE];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                unpack<ET>(next_v[u], v[u]);
                if constexpr (NORM) unpack<ET>(next_x[u], x[u]);
            }
            if (i0 + GROUPS < items) fetch(first, items, item + GROUPS);
            else fetch(first + stride, items_of(first + stride), group);
            turn<PAIRS, true>(v, p, angles + r * (a.rot / 2), a.rot, patch + group * TPH * LANE, c);
            if constexpr (NORM) {
                float sums[2] = {0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < PIECE; ++i) {
                        sums[0] = fmaf(x[u][i], x[u][i], sums[0]);
                        sums[1] = fmaf(v[u][i] * gamma[u][i], x[u][i], sums[1]);
                    }
                head_sums<TPH>(sums);
                const float rstd = 1.0f / sqrtf(sums[0] * a.inv_d + a.eps), mid = sums[1] * rstd * a.inv_d;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < PIECE; ++i) {
                        const float xh = x[u][i] * rstd;
                        dg[u][i] = fmaf(v[u][i], xh, dg[u][i]);
                        v[u][i] = rstd * (v[u][i] * gamma[u][i] - xh * mid);
                    }
            }
            char* out = s.out + (first + r) * s.out_row + h * s.out_head;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (on && there[u]) store8<ET, NT>(out + p[u] * PIECE * (int)sizeof(ET), v[u]);
        }
    }
    if constexpr (NORM) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (there[u])
#pragma unroll
                for (int i = 0; i < PIECE; ++i) patch[group * a.d + p[u] * PIECE + i] = dg[u][i];
        __syncthreads();
        float* to = blocks > 1 ? a.partial + (size_t)blockIdx.x * a.d : keys ? a.dgamma_k : a.dgamma_q;
        for (int i = threadIdx.x; i < a.d; i += THREADS) {
            float sum = 0.0f;
            for (int g = 0; g < GROUPS; ++g) sum += patch[g * a.d + i];
            to[i] = sum;
        }
    }
}

// dgamma_q (blockIdx.y 0), dgamma_k: sums over the blocks, LINES lines of them side by side, four blocks of a line under way.
constexpr int LINES = 64;
__global__ __launch_bounds__(16 * LINES) void rotary_join_kernel(const float* __restrict__ partial, int blocks_q, int blocks_k, int d, float* __restrict__ dq, float* __restrict__ dk)
{
    __shared__ float lines[LINES][17];
    const int c = threadIdx.x & 15, line = threadIdx.x >> 4, at = blockIdx.x * 16 + c, blocks = blockIdx.y ? blocks_k : blocks_q;
    if (blocks == 1) return;                               // written already
    const float* from = partial + (blockIdx.y ? (size_t)blocks_q * d : 0) + at;
    float sum = 0.0f;
    if (at < d) {
        int b = line;
        for (; b + 3 * LINES < blocks; b += 4 * LINES) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = from[(size_t)(b + i * LINES) * d];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += v[i];
        }
        for (; b < blocks; b += LINES) sum += from[(size_t)b * d];
    }
    lines[line][c] = sum;
    __syncthreads();
    if (line == 0 && at < d) {
        sum = 0.0f;
#pragma unroll
        for (int l = 0; l < LINES; ++l) sum += lines[l][c];
        (blockIdx.y ? dk : dq)[at] = sum;
    }
}

template <typename F> hipError_t by_head(int d, int rot, int interleaved, F f)
{
    auto with = [&](auto TPH) {
        if (interleaved || rot == 0) return f(TPH, std::integral_constant<Pairs, NEIGHBOURS>{});
        if (rot % (2 * PIECE) == 0) return f(TPH, std::integral_constant<Pairs, HALVES>{});
        return f(TPH, std::integral_constant<Pairs, HALVES_CUT>{});
    };
    if (d <= 16) return with(std::integral_constant<int, 1>{});
    if (d <= 32) return with(std::integral_constant<int, 2>{});
    if (d <= 64) return with(std::integral_constant<int, 4>{});
    if (d <= 128) return with(std::integral_constant<int, 8>{});
    return with(std::integral_constant<int, 16>{});
}

inline side_t make_side(const moe_heads_t* in, const moe_heads_t* x, const moe_heads_t* out, const float* gamma, int heads, int size)
{
    side_t s = {};
    s.in = (const char*)in->p, s.in_row = in->row * size, s.in_head = in->head * size;
    if (x) s.x = (const char*)x->p, s.x_row = x->row * size, s.x_head = x->head * size;
    s.out = (char*)out->p, s.out_row = out->row * size, s.out_head = out->head * size;
    s.gamma = gamma, s.heads = heads;
    return s;
}

inline rotary_args make_args(const moe_rotary_t& c, const int32_t* positions, const double* frequencies)
{
    rotary_args a = {};
    a.positions = positions, a.frequencies = frequencies;
    a.rows = c.rows, a.d = c.d, a.rot = c.rot, a.out_rows = c.out_rows;
    a.eps = c.eps, a.amplitude = c.amplitude, a.inv_d = 1.0f / (float)c.d;
    return a;
}

// Rows that a block takes at a time, whose angles it works out together: ROUNDS heads for each of its groups of threads, as long as there are `least` blocks.
// 32768 rows of 32 and 8 heads of 128 with norms, bf16, us: 2 rows a block 170, 4 rows 130 to 137, 9 rows 145.  7999 rows of 12 and 4 heads of 80: at least 256 blocks
// 13.0, 1024 11.1, 4096 19.6.  The gradient with norms has no such bound on its blocks below ROTARY_PARTIALS: 512 tiny rows need 9.0 us so, 21.3 by few blocks.
constexpr int ROUNDS = 6, LEAST = 1024;
constexpr int MOST_BLOCKS = 1 << 22;                       // of a launch: its threads are counted in 32 bits
inline int rows_at_once(const moe_rotary_t& c, int heads, int least)
{
    int tph = 1;
    while (tph * 16 < c.d) tph *= 2;
    long long n = (long long)ROUNDS * (THREADS / tph) / heads;
    const long long room = c.rot > 0 ? MAX_ANGLES / (c.rot / 2) : n, share = c.rows / least;
    n = n < room ? n : room;
    n = n < share ? n : share;
    return n < 1 ? 1 : (int)n;
}

inline bool streams_rows(const moe_rotary_t& c, int size) { return streams((size_t)c.rows * (c.heads + c.kv_heads) * c.d * size); }

}  // namespace

hipError_t launch_rotary_fwd(const moe_rotary_t& c, const moe_heads_t& Q, const moe_heads_t& K, const moe_heads_t* V, const float* gamma_q, const float* gamma_k,
                             const int32_t* positions, const double* frequencies, const int32_t* slots, const moe_heads_t& Qo, const moe_heads_t& Ko,
                             const moe_heads_t* Vo, hipStream_t st)
{
    if (c.rows == 0) return hipSuccess;
    const int size = c.dtype == MOE_BF16 ? 2 : 4;
    rotary_args a = make_args(c, positions, frequencies);
    a.slots = slots;
    a.side[0] = make_side(&Q, nullptr, &Qo, gamma_q, c.heads, size);
    a.side[1] = make_side(&K, nullptr, &Ko, gamma_k, c.kv_heads, size);
    a.sides = 2;
    if (V) a.side[a.sides++] = make_side(V, nullptr, Vo, nullptr, c.kv_heads, size);
    const bool few = c.rows <= 1024;
    a.rows_at_once = few ? 1 : rows_at_once(c, c.heads + c.kv_heads, LEAST);
    auto launch = [&](int blocks) {
        const dim3 grid(blocks, few ? a.sides : 1);
        return by_head(c.d, c.rot, c.interleaved, [&](auto TPH, auto PAIRS) {
            auto go = [&](auto ET, auto NORM, auto NT) {
                hipLaunchKernelGGL((rotary_kernel<decltype(ET), decltype(TPH)::value, decltype(PAIRS)::value, decltype(NORM)::value, decltype(NT)::value>), grid, dim3(THREADS), 0, st, a);
                return hipGetLastError();
            };
            const bool nt = streams_rows(c, size);
            auto typed = [&](auto ET) {
                if (c.norm) return nt ? go(ET, std::true_type{}, std::true_type{}) : go(ET, std::true_type{}, std::false_type{});
                return nt ? go(ET, std::false_type{}, std::true_type{}) : go(ET, std::false_type{}, std::false_type{});
            };
            return size == 2 ? typed(bf16_t{}) : typed(float{});
        });
    };
    // as many rows a launch as MOST_BLOCKS have; the pointers move on to the next ones, not those of a cache
    const int most = (int)(((long long)MOST_BLOCKS * a.rows_at_once < c.rows) ? (long long)MOST_BLOCKS * a.rows_at_once : c.rows);
    for (int left = c.rows; left > 0; left -= most) {
        a.rows = left < most ? left : most;
        const hipError_t e = launch((a.rows + a.rows_at_once - 1) / a.rows_at_once);
        if (e != hipSuccess) return e;
        a.positions += a.rows;
        for (int k = 0; k < a.sides; ++k) {
            a.side[k].in += a.rows * a.side[k].in_row;
            if (k == 0 || !slots) a.side[k].out += a.rows * a.side[k].out_row;
        }
        if (slots) a.slots += a.rows;
    }
    return hipSuccess;
}

hipError_t launch_rotary_bwd(const moe_rotary_t& c, const moe_heads_t& dQo, const moe_heads_t& dKo, const moe_heads_t* Q, const moe_heads_t* K,
                             const float* gamma_q, const float* gamma_k, const int32_t* positions, const double* frequencies, const moe_heads_t& dQ,
                             const moe_heads_t& dK, float* dgamma_q, float* dgamma_k, float* partial, hipStream_t st)
{
    const int size = c.dtype == MOE_BF16 ? 2 : 4;
    rotary_args a = make_args(c, positions, frequencies);
    a.side[0] = make_side(&dQo, Q, &dQ, gamma_q, c.heads, size);
    a.side[1] = make_side(&dKo, K, &dK, gamma_k, c.kv_heads, size);
    a.sides = 2;
    a.partial = partial, a.dgamma_q = dgamma_q, a.dgamma_k = dgamma_k;
    int blocks = 0;
    hipError_t e = hipSuccess;
    if (c.rows > 0) {
        // blocks of queries and of keys, as many as their heads are; with a norm each leaves a partial sum of its parameters
        a.rows_at_once = rows_at_once(c, c.heads, c.norm ? 64 : LEAST);
        a.rows_at_once_k = rows_at_once(c, c.kv_heads, c.norm ? 16 : LEAST / 4);
        const long long all_q = ((long long)c.rows + a.rows_at_once - 1) / a.rows_at_once, all_k = ((long long)c.rows + a.rows_at_once_k - 1) / a.rows_at_once_k;
        long long most_q = MOST_BLOCKS, most_k = MOST_BLOCKS;
        if (c.norm) {                                      // one at least of either, ROTARY_PARTIALS in all
            most_q = (long long)ROTARY_PARTIALS * c.heads / (c.heads + c.kv_heads);
            most_q = most_q < 1 ? 1 : most_q < ROTARY_PARTIALS ? most_q : ROTARY_PARTIALS - 1;
            most_k = ROTARY_PARTIALS - most_q;
        }
        a.blocks_q = (int)(all_q < most_q ? all_q : most_q);
        blocks = a.blocks_q + (int)(all_k < most_k ? all_k : most_k);
        e = by_head(c.d, c.rot, c.interleaved, [&](auto TPH, auto PAIRS) {
            auto go = [&](auto ET, auto NORM, auto NT) {
                hipLaunchKernelGGL((rotary_bwd_kernel<decltype(ET), decltype(TPH)::value, decltype(PAIRS)::value, decltype(NORM)::value, decltype(NT)::value>), dim3(blocks), dim3(THREADS), 0, st, a);
                return hipGetLastError();
            };
            const bool nt = streams_rows(c, size);
            auto typed = [&](auto ET) {
                if (c.norm) return nt ? go(ET, std::true_type{}, std::true_type{}) : go(ET, std::true_type{}, std::false_type{});
                return nt ? go(ET, std::false_type{}, std::true_type{}) : go(ET, std::false_type{}, std::false_type{});
            };
            return size == 2 ? typed(bf16_t{}) : typed(float{});
        });
    }
    if (e != hipSuccess || !c.norm || blocks == 2) return e;
    const int blocks_k = blocks - a.blocks_q;              // none where there are no rows: both sums are written, as zeros
    hipLaunchKernelGGL(rotary_join_kernel, dim3((c.d + 15) / 16, 2), dim3(16 * LINES), 0, st, partial, a.blocks_q, blocks_k, c.d, dgamma_q, dgamma_k);
    return hipGetLastError();
}
