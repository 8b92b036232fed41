// What the attention kernels have in common: which sequence a block works on, tiles of a sequence's rows in LDS, and the fragments that the matrix
// cores take from them.
//
// All products are 32 x 32 blocks.  A fragment is a lane's eight of 16 contraction steps, and both operands of a product only have to agree on which:
//   by rows   lane l holds row l % 32, columns 8 (l / 32) .. + 7 of 16 neighbouring columns (the contraction runs over the head)
//   by keys   lane l holds column l % 32, rows 8 (e / 4) + 4 (l / 32) + e % 4 for e = 0 .. 7 of 16 neighbouring rows (the contraction runs over rows)
// The second is the order in which a product leaves its results, 16 to a lane: what comes out of one product goes into the next as it is, without a word
// between lanes.  bf16 takes one instruction a fragment, fp32 eight (32 x 32 x 2 each, exact fp32).
#pragma once

#include "tile.h"

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.402823466e38f;

// What two lanes that are 32 apart have, in both of them.
struct Halves { float low, high; };
__device__ __forceinline__ Halves halves_of(float v)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return Halves{__uint_as_float(both[0]), __uint_as_float(both[1])};
}
// The highest of three; a NaN is passed over.  (fmaxf first makes every operand canonical, an instruction each.)
__device__ __forceinline__ float highest_of(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float sum_of_halves(float v) { const Halves h = halves_of(v); return h.low + h.high; }
// A branch that all lanes take together, and rarely: what stands in it is not worked out beside the branch, and lies out of the way (a loop that jumps over it
// waits for instructions each time: 4 % of the forward pass).
#define RARELY(condition) if (__builtin_expect(!!(condition), 0))
#define APART() asm volatile("")
// On the lambdas of a kernel: one that became a function of its own would have the kernel's arguments, and all that it shares, in memory.
#define INLINE __attribute__((always_inline))
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename ET> struct Frag;
template <> struct Frag<bf16_t> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x16 mma(const type& a, const type& b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    // Eight results of a product as a fragment: rounded to bf16, by 2^-8 of itself at most, as every operand of the matrix cores is; sums stay in fp32.
    static __device__ __forceinline__ type pack(const f32x16& s, int h)
    {
        const u32x4 v = {pack_bf16x2(s[8 * h], s[8 * h + 1]), pack_bf16x2(s[8 * h + 2], s[8 * h + 3]), pack_bf16x2(s[8 * h + 4], s[8 * h + 5]), pack_bf16x2(s[8 * h + 6], s[8 * h + 7])};
        return __builtin_bit_cast(type, v);
    }
    static __device__ __forceinline__ type load(const char* p) { return __builtin_bit_cast(type, *(const u32x4*)p); }
    static __device__ __forceinline__ type zero() { return __builtin_bit_cast(type, u32x4{0, 0, 0, 0}); }
    static __device__ __forceinline__ float at(const type& f, int e) { return (float)f[e]; }
};
template <> struct Frag<float> {
    typedef f32x8 type;
    static __device__ __forceinline__ f32x16 mma(const type& a, const type& b, f32x16 c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ type pack(const f32x16& s, int h)
    {
        type v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s[8 * h + e];
        return v;
    }
    static __device__ __forceinline__ type load(const char* p)
    {
        const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 16);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ type zero() { return type{0, 0, 0, 0, 0, 0, 0, 0}; }
    static __device__ __forceinline__ float at(const type& f, int e) { return f[e]; }
};

// A tile of rows of DP elements (a head's width, filled up to 64 or 128 with zeros) in LDS.  The 16-byte pieces of a row are XOR-swizzled by the
// row so that 16 neighbouring rows of one piece cover all banks (by rows), and so do 64 bytes of four neighbouring rows (by keys).
template <typename ET, int DP> struct Tile {
    static constexpr int ROW = DP * (int)sizeof(ET), PPR = ROW / 16;
    static constexpr int T = DP / 16, DB = DP / 32;        // contraction steps, blocks of columns
    typedef typename Frag<ET>::type frag;
    static __device__ __forceinline__ int swizzle(int row) { return PPR == 8 ? ((row >> 1) & 1) << 2 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3); }

    // A lane's addresses, the tile's base and the row block's apart.
    uint32_t rows0, keys0[2];
    __device__ __forceinline__ Tile(int lane)
    {
        const int row = lane & 31, hi = lane >> 5;
        rows0 = row * ROW + (((sizeof(ET) == 2 ? hi : 2 * hi) ^ swizzle(row)) << 4);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (sizeof(ET) == 2) {
                const int s = lane & 15, r = 8 * u + 4 * hi + (s >> 2);
                keys0[u] = r * ROW + (((((lane >> 4) & 1) * 2 + ((s & 3) >> 1)) ^ swizzle(r)) << 4) + (s & 1) * 8;
            } else {
                keys0[u] = (8 * u + 4 * hi) * ROW + ((((lane & 31) >> 2) ^ (2 * u + hi)) << 4) + (lane & 3) * 4;
            }
        }
    }
    // A lane's addresses in the tile at `base`; what follows adds constants to them that fit an instruction (the compiler would rather add them to the base and
    // add the base again for each).
    struct RowsAt { uint32_t at[T]; };
    struct KeysAt { uint32_t at[DB][2]; };
    __device__ __forceinline__ RowsAt rows_at(uint32_t base) const
    {
        RowsAt r;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            r.at[t] = base + (rows0 ^ (t << (sizeof(ET) == 2 ? 5 : 6)));
            asm("" : "+v"(r.at[t]));
        }
        return r;
    }
    __device__ __forceinline__ KeysAt keys_at(uint32_t base) const
    {
        KeysAt k;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                k.at[b][u] = base + (keys0[u] ^ (b << (sizeof(ET) == 2 ? 6 : 7)));
                asm("" : "+v"(k.at[b][u]));
            }
        return k;
    }
    // By rows: rows `row0` .. + 31 (a multiple of 32) of the tile `beyond` bytes on, columns 16 t .. + 15.
    static __device__ __forceinline__ frag by_rows(const RowsAt& r, int row0, int t, int beyond = 0)
    {
        const int more = row0 * ROW + beyond;
        if constexpr (sizeof(ET) == 2) {
            return __builtin_bit_cast(frag, *(const LDS_PTR(s16x8))(uintptr_t)(r.at[t] + more));
        } else {
            const f32x4 x = *(const LDS_PTR(f32x4))(uintptr_t)(r.at[t] + more), y = *(const LDS_PTR(f32x4))(uintptr_t)((r.at[t] ^ 16) + more);
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // By keys: rows `row0` .. + 15 (a multiple of 16), columns 32 db .. + 31.
    static __device__ __forceinline__ frag by_keys(const KeysAt& k, int row0, int db, int beyond = 0)
    {
        const int more = row0 * ROW + beyond;
        if constexpr (sizeof(ET) == 2) {
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(k.at[db][0] + more));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(k.at[db][1] + more));
            return __builtin_bit_cast(frag, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            frag f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = *(const LDS_PTR(float))(uintptr_t)((k.at[db][e >> 2] ^ ((e & 3) << 6)) + more + (e & 3) * ROW);
            return f;
        }
    }
};

__device__ __forceinline__ rsrc_t tile_rsrc(const char* base, uint32_t bytes)
{
    const unsigned long long b = (unsigned long long)base;
    return rsrc_t{(int)(unsigned)b, (int)(unsigned)((b >> 32) & 0xffffull), (int)bytes, 0x00020000};
}
// dma16 that reads of LDS may pass: they are of other tiles of the ring, and the barriers keep them on their sides.
__device__ __forceinline__ void tile_dma(rsrc_t r, uint32_t lds_base, uint32_t voff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds_base), "v"(voff), "s"(r));
}

// Requests of a tile of ROWS rows, straight into LDS, by WAVES waves: P 16-byte pieces of each lane.  Columns from the head's width on and rows past the
// sequence arrive as zeros.
template <typename ET, int DP, int ROWS, int WAVES> struct Request {
    typedef Tile<ET, DP> tile;
    static constexpr int P = ROWS * tile::PPR / 64 / WAVES;
    static constexpr uint32_t BYTES = ROWS * tile::ROW;
    static_assert(P * 64 * WAVES == ROWS * tile::PPR, "whole waves");
    uint32_t off[P];
    __device__ __forceinline__ Request(int lane, int wave, uint32_t row_bytes, int d)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int slot = (i * WAVES + wave) * 64 + lane, row = slot / tile::PPR, piece = (slot % tile::PPR) ^ tile::swizzle(row);
            off[i] = piece * 16 < d * (int)sizeof(ET) ? row * row_bytes + piece * 16 : 0xfffffff0u;
        }
    }
    // rows: how many of the tile's rows, from `first` on, are the sequence's (none and fewer: zeros all over).  ROWS rows of 2^23 bytes at most: 32 bits do.
    __device__ __forceinline__ void operator()(const char* first, int rows, uint32_t row_bytes, int d, uint32_t base, int wave) const
    {
        const rsrc_t r = tile_rsrc(first, rows > 0 ? (uint32_t)(rows < ROWS ? rows - 1 : ROWS - 1) * row_bytes + d * (int)sizeof(ET) : 0);
#pragma unroll
        for (int i = 0; i < P; ++i) tile_dma(r, base + (i * WAVES + wave) * 1024, off[i]);
    }
};

// Everything a wave asked of LDS has arrived; then the block meets.
#define LDS_BARRIER() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")

// What was loaded into registers has arrived: said here once, or the compiler waits for it, and for every request since, each time around a loop that uses it.
template <typename T, int N> __device__ __forceinline__ void arrived(const T (&v)[N])
{
#ifdef __HIP_DEVICE_COMPILE__                              // the host's pass knows no registers of this width
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" :: "v"(v[i]));
#endif
}

// The two halves of a block of eight waves work in turn: while the waves of one feed the matrix cores, those of the other, which share their SIMDs, work on
// scores with the vector units (both at the same time would take the two one after the other).  A phase ends for both at a barrier; what is written before it
// stays before it.
#define PHASE_END() do { __builtin_amdgcn_sched_barrier(0); LDS_BARRIER(); __builtin_amdgcn_sched_barrier(0); } while (0)

// The order of a run of N matrix instructions of bf16, instruction i with READS::of(i) requests of LDS: they are under way AHEAD instructions before it, those of
// the first AHEAD before the run.  Left alone the compiler requests each right before it is needed, and the matrix cores wait for LDS every time.  To be
// called at the end of the run, in the same basic block.
template <typename READS, int N, int AHEAD, int I = 0> __device__ __forceinline__ void pace()
{
    constexpr int MATRIX = 0x8, LDS_READ = 0x100;
    if constexpr (I < N) {
        __builtin_amdgcn_sched_group_barrier(MATRIX, 1, 0);
        if constexpr (I + AHEAD < N)
            if constexpr (READS::of(I + AHEAD) > 0) __builtin_amdgcn_sched_group_barrier(LDS_READ, READS::of(I + AHEAD), 0);
        pace<READS, N, AHEAD, I + 1>();
    }
}
// A fragment by rows is one request, one by keys two.
template <int ROWS> struct RowsThenKeys { static constexpr int of(int i) { return i < ROWS ? 1 : 2; } };
template <int KEYS> struct KeysThenRows { static constexpr int of(int i) { return i < KEYS ? 2 : 1; } };

// Tensors of rows x heads x d: element (r, h, c) lies `row` r + `head` h + c elements from the first; here in bytes.
struct heads_t {
    char* p;
    uint32_t row;
    long long head;
};
struct attn_args {
    heads_t Q, K, V, O, dO, dQ, dK, dV;
    float* lse;                            // [heads][q_rows]
    float2* stats;                         // [heads][q_rows]: lse log2 e, <dO, O>
    const int32_t *offsets, *k_begin, *k_end;
    int q_rows, k_rows, seqs, heads, kv_heads, group, d, causal, splits, chunk;
    float scale, scale2;                   // scale2 = scale log2 e: exponentials are powers of two
    float *partial, *partial_k;
};
inline heads_t in_bytes(const moe_heads_t& t, int size) { return heads_t{(char*)t.p, (uint32_t)(t.row * size), t.head * size}; }
__device__ __forceinline__ const char* row_of(const heads_t& t, int head, long long row) { return t.p + (long long)head * t.head + row * t.row; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A sequence: its queries are rows q0 .. q0 + n - 1, its keys rows k0 .. k0 + m - 1; `tile` is the tile of this block.  Offsets come from device memory and
// are taken into the tensors' rows here, whatever they are.
struct Sequence { int q0, n, k0, m, tile; };
__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : v > most ? most : v; }

// Sequence s owns the slots from offsets[s] * mult / SIDE + s on: never fewer than its tiles, whatever the lengths, and one at least, so that the host needs
// to know none of them.  64 sequences are looked at in a step.  The tile may lie past the sequence's last one.
template <int SIDE>
__device__ __forceinline__ Sequence find_sequence(const attn_args& a, const int32_t* begin, int rows, int mult, int slot, int lane)
{
    int lo = 0, left = a.seqs;
    while (left > 1) {
        const int step = (left + 63) >> 6, at = lane * step;
        const bool before = at < left && (int)((long long)clamped(begin[lo + (at < left ? at : 0)], rows) * mult / SIDE) + lo + at <= slot;
        int k = __popcll(__ballot(before));
        k = k < 1 ? 1 : k;
        lo += (k - 1) * step;
        left = min(step, left - (k - 1) * step);
    }
    lo = uniform(lo);
    Sequence s;
    s.tile = uniform(slot - lo - (int)((long long)clamped(begin[lo], rows) * mult / SIDE));
    s.q0 = uniform(clamped(a.offsets[lo], a.q_rows));
    s.n = uniform(clamped(a.offsets[lo + 1], a.q_rows)) - s.q0;
    s.k0 = uniform(clamped(a.k_begin[lo], a.k_rows));
    s.m = uniform(clamped(a.k_end[lo], a.k_rows)) - s.k0;
    s.n = s.n < 0 ? 0 : s.n;
    s.m = s.m < 0 ? 0 : s.m;
    return s;
}

// Small calls: blocks of 32 rows whose waves share the work along the other axis, each through a ring of its own in LDS, and join at the end.
constexpr int FEW_KEYS = 32, FEW_STAGES = 2;
template <typename ET, int DP> constexpr int few_waves() { return DP * (int)sizeof(ET) <= 256 ? 4 : 2; }
// Where row r of a block's 32 lies: token by token, the heads that share a kv head beside each other.
struct FewRow { int token, head; bool there; };
__device__ __forceinline__ FewRow few_row(const attn_args& a, const Sequence& s, int kv, int r)
{
    const long long i = (long long)s.tile * 32 + r;
    FewRow f;
    f.token = (int)(i / a.group);
    f.head = kv * a.group + (int)(i % a.group);
    f.there = f.token < s.n;
    return f;
}

// Keys that the last of a block's rows sees.
__device__ __forceinline__ int few_keys(const attn_args& a, const Sequence& s)
{
    const int last = min(s.n - 1, (int)(((long long)s.tile * 32 + 31) / a.group));
    return a.causal ? min(s.m, max(0, last + 1 + s.m - s.n)) : s.m;
}
// Blocks of 32 rows, and whether a call of so many larger blocks is one for them: where those leave CUs without one, all wait for the longest.  us, small | large blocks, causal:
//   forward   bf16, 128 columns: 64 blocks (4096, 4 heads) 59 | 77, 80 (4 x 1024) 29 | 29, 128 (16 x 256) 18 | 17, 136 (4096) 99 | 78;  64 columns: 80 13 | 22, 160 23 | 23, 240 32 | 24
//   gradient  bf16, 128 columns: 68 125 | 301, 136 (4096) 229 | 304, 128 (16 x 256) 42 | 50, 160 (4 x 1024) 112 | 98, 204 338 | 307;  64 columns: 160 54 | 67, 240 72 | 69
//   fp32, 64 columns (4096): 68 123 | 495, 544 760 | 546, gradient 327 | 1500 and 2248 | 2026
inline long long few_units(const attn_args& a) { return ((long long)a.q_rows * a.group / 32 + a.seqs) * a.kv_heads; }
template <typename ET, int DP> bool is_small(long long blocks, bool gradient)
{
    return blocks <= (sizeof(ET) == 4 ? 256 : gradient ? (DP == 64 ? 208 : 144) : DP == 64 ? 160 : 96);
}
// How the tiles of 32 along a block's other axis are cut into parts, blocks of their own: `chunk` tiles a part as the launch has it, more where that does not reach the
// end.  Parts past the end have nothing to do; a part that is alone writes its rows itself, others are joined by a later launch.
struct Parts {
    int chunk, used;
    __device__ __forceinline__ Parts(const attn_args& a, int tiles)
    {
        chunk = max(a.chunk, (tiles + a.splits - 1) / a.splits);
        used = max(1, (tiles + chunk - 1) / chunk);
    }
};

// Blocks go to the eight XCDs in turn: where the heads are a multiple of eight, an XCD works on heads / 8 neighbouring ones, whose keys and values are the
// same ones where heads share them, and its L2 holds those only.
__device__ __forceinline__ void head_and_slot(int id, int heads, int& head, int& slot)
{
    if ((heads & 7) == 0) {
        const int per = heads >> 3, i = id >> 3;
        head = (id & 7) * per + i % per;
        slot = i / per;
    } else {
        head = id % heads;
        slot = id / heads;
    }
}

inline attn_args attn_make(const moe_attn_t& c)
{
    attn_args a = {};
    a.q_rows = c.q_rows, a.k_rows = c.k_rows, a.seqs = c.seqs, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
    a.d = c.d, a.causal = c.causal, a.splits = 1;
    a.scale = c.scale, a.scale2 = c.scale * LOG2E;
    return a;
}

template <typename ET> __device__ __forceinline__ void store_four(char* p, float a, float b, float c, float d)
{
    if constexpr (sizeof(ET) == 2) *(u32x2*)p = u32x2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
    else *(f32x4*)p = f32x4{a, b, c, d};
}

// The kernel's dynamic LDS, once per device.
template <typename KERNEL> hipError_t allow_lds(KERNEL kernel, size_t bytes, PerDeviceOnce& once)
{
    const int dev = current_device();
    if (once.is_done(dev)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) once.mark(dev);
    return e;
}

}  // namespace
