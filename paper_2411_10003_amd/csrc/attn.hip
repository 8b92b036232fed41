// Attention of packed sequences, forward: O = softmax(scale Q K^T) V, row by row over the keys that the row sees, and the logarithm of each row's sum.
//
// One pass over the keys with a running maximum and sum.  A wave has 32 queries and all of their results: with S^T = K Q^T a lane holds 16 scores of ONE
// query per 32 keys, so maximum and sum stay in the lane (its other half is 32 lanes on), and the exponentials are the second operand of O^T = V^T P^T
// as they lie.  The maximum in use is let go stale by up to 2^8: rescaling the results is rare after the first tiles and exact either way.
#include "attn.h"

#include <type_traits>

namespace {

constexpr int KEYS = 64;                                   // keys of a tile

// What a wave knows of its 32 queries while it goes over the keys.
template <typename ET, int DP> struct Rows {
    typedef Tile<ET, DP> tile;
    typedef typename Frag<ET>::type frag;
    frag q[tile::T];
    f32x16 o[tile::DB];
    float most, sum;                                       // of this lane's query; sum over this lane's keys only

    __device__ __forceinline__ void clear()
    {
        most = LOWEST;
        sum = 0.0f;
#pragma unroll
        for (int b = 0; b < tile::DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    }
    // Scores of NB x 32 keys from row block 0 of the tile at `base`.
    template <int NB> __device__ __forceinline__ void scores(const tile& t, uint32_t base, f32x16 (&s)[NB]) const
    {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < tile::T; ++k)
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = Frag<ET>::mma(t.by_rows(base, 32 * b, k), q[k], s[b]);
    }
    // Keys past `limit` are hidden from this lane's query; `first` is the key of row 0.
    template <int NB> static __device__ __forceinline__ void hide(f32x16 (&s)[NB], int first, int limit, int hi)
    {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = first + 32 * b + 8 * (i >> 2) + 4 * hi + (i & 3) > limit ? -INFINITY : s[b][i];
    }
    // Scores to exponentials under the running maximum.
    template <int NB> __device__ __forceinline__ void soften(f32x16 (&s)[NB], float scale2)
    {
        float top = LOWEST;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = fmaxf(top, other_half(top)) * scale2;
        if (__any(top > most + 8.0f)) {
            const float next = fmaxf(most, top), down = exp2_fast(most - next);
            most = next;
            sum *= down;
#pragma unroll
            for (int b = 0; b < tile::DB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= down;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = exp2_fast(fmaf(s[b][i], scale2, -most));
                sum += s[b][i];
            }
    }
    template <int NB> __device__ __forceinline__ void add(const tile& t, uint32_t base, const f32x16 (&s)[NB])
    {
#pragma unroll
        for (int k = 0; k < 2 * NB; ++k) {
            const frag p = Frag<ET>::pack(s[k >> 1], k & 1);
#pragma unroll
            for (int b = 0; b < tile::DB; ++b) o[b] = Frag<ET>::mma(t.by_keys(base, 16 * k, b), p, o[b]);
        }
    }
};

constexpr int stages_for(int stage_bytes) { return 4 * stage_bytes <= 144 * 1024 ? 4 : 2; }

// A block has WAVES x 32 queries of one head; keys and values of 64 rows at a time go through a ring in LDS.
template <typename ET, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : 1) void attend_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, KEYS, WAVES> request;
    constexpr int SIDE = WAVES * 32;
    constexpr uint32_t STAGE = 2 * request::BYTES;
    constexpr int STAGES = stages_for(STAGE);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int head, slot;
    head_and_slot(blockIdx.x, a.heads, head, slot);
    const Sequence s = find_sequence<SIDE>(a, a.offsets, a.q_rows, 1, gridDim.x / a.heads - 1 - slot, lane);      // later tiles see more keys and go first
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.n) return;
    const int shift = s.m - s.n, first = s.tile * SIDE + wave * 32, row = first + col;     // of the sequence's queries
    // how many keys the block's, this wave's last query sees; the last key that this lane's sees
    const int block_keys = a.causal ? min(s.m, max(0, min(s.n, (s.tile + 1) * SIDE) + shift)) : s.m;
    const int wave_keys = first >= s.n ? 0 : a.causal ? min(s.m, max(0, min(s.n, first + 32) + shift)) : s.m;
    const int limit = (a.causal ? min(s.m, row + shift + 1) : s.m) - 1, least = (a.causal ? min(s.m, first + shift + 1) : s.m) - 1;
    const int tiles = (block_keys + KEYS - 1) / KEYS, wave_tiles = (wave_keys + KEYS - 1) / KEYS;

    const int kv = head / a.group;
    const char* K = row_of(a.K, kv, s.k0);
    const char* V = row_of(a.V, kv, s.k0);
    const tile t(lane);
    const request ask_k(lane, wave, a.K.row, a.d), ask_v(lane, wave, a.V.row, a.d);
    auto ask = [&](int j) {
        const uint32_t at = ring + (j % STAGES) * STAGE;
        ask_k(K + (long long)j * KEYS * a.K.row, s.m - j * KEYS, a.K.row, a.d, at, wave);
        ask_v(V + (long long)j * KEYS * a.V.row, s.m - j * KEYS, a.V.row, a.d, at + request::BYTES, wave);
    };
    Rows<ET, DP> r;
    r.clear();
    {
        const char* q = row_of(a.Q, head, s.q0 + row);
#pragma unroll
        for (int k = 0; k < tile::T; ++k)
            r.q[k] = row < s.n && 16 * k + 8 * hi < a.d ? Frag<ET>::load(q + (16 * k + 8 * hi) * sizeof(ET)) : Frag<ET>::zero();
    }
    if (tiles > 0) {
#pragma unroll
        for (int j = 0; j < STAGES - 1; ++j) ask(j);
        for (int j = 0; j < tiles; ++j) {
            WAIT_VMCNT((STAGES - 2) * 2 * request::P);     // tile j has arrived
            LDS_BARRIER();                                 // everyone's part of it, and nobody reads tile j - 1 any more
            ask(j + STAGES - 1);                           // past the last tile: zeros that nobody reads
            if (j >= wave_tiles) continue;
            const uint32_t at = ring + (j % STAGES) * STAGE;
            f32x16 x[2];
            r.scores(t, at, x);
            if (j * KEYS + KEYS - 1 > least) r.hide(x, j * KEYS, limit, hi);
            r.soften(x, a.scale2);
            r.add(t, at + request::BYTES, x);
        }
        WAIT_VMCNT(0);
    }
    if (row >= s.n) return;
    const float sum = r.sum + other_half(r.sum), by = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;     // a row that sees nothing is zero; NaN stays
    char* o = a.O.p + (long long)head * a.O.head + (long long)(s.q0 + row) * a.O.row;
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 32 * b + 8 * i + 4 * hi;
            if (c < a.d) store_four<ET>(o + c * sizeof(ET), r.o[b][4 * i] * by, r.o[b][4 * i + 1] * by, r.o[b][4 * i + 2] * by, r.o[b][4 * i + 3] * by);
        }
    if (a.lse && hi == 0) a.lse[(long long)head * a.q_rows + s.q0 + row] = sum == 0.0f ? -INFINITY : (r.most + __log2f(sum)) * LN2;
}


// Few rows (answering a token at a time): a block has 32 rows of one sequence, token by token the heads that share a kv head beside each other, and one
// part of the keys; its waves take tiles of 32 keys in turn, each through a ring of its own, and join at the end.  Bound by the keys and values,
// read once for all heads that share them.  With more than one part the unscaled results go to the workspace and a second launch joins them.
constexpr int FEW_KEYS = 32, FEW_STAGES = 2;
template <typename ET, int DP> constexpr int few_waves() { return DP * (int)sizeof(ET) <= 256 ? 4 : 2; }
constexpr int PARTIAL_MORE = 64;                           // of a part's 32 rows: maximum and sum
template <int DP> constexpr int partial_floats() { return 32 * DP + PARTIAL_MORE; }

// Where row r of a block's 32 lies: token and head.
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

// Keys that the last of a block's rows sees, and how they are cut: `chunk` tiles a part as the launch has it, more where that does not reach the end.
__device__ __forceinline__ int few_keys(const attn_args& a, const Sequence& s)
{
    const int last = min(s.n - 1, (int)(((long long)s.tile * 32 + 31) / a.group));
    return a.causal ? min(s.m, max(0, last + 1 + s.m - s.n)) : s.m;
}
struct Parts {
    int tiles, chunk, used;
    __device__ __forceinline__ Parts(const attn_args& a, int keys)
    {
        tiles = (keys + FEW_KEYS - 1) / FEW_KEYS;
        chunk = max(a.chunk, (tiles + a.splits - 1) / a.splits);
        used = max(1, (tiles + chunk - 1) / chunk);
    }
};

template <typename ET, int DP>
__device__ __forceinline__ void few_store(const attn_args& a, const Sequence& s, const FewRow& f, int c, float v0, float v1, float v2, float v3)
{
    char* o = a.O.p + (long long)f.head * a.O.head + (long long)(s.q0 + f.token) * a.O.row;
    store_four<ET>(o + c * sizeof(ET), v0, v1, v2, v3);
}

template <typename ET, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 1) void attend_few_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, FEW_KEYS, 1> request;
    constexpr int PITCH = DP + 4;
    constexpr uint32_t STAGE = 2 * request::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + wave * FEW_STAGES * STAGE;
    const int part = blockIdx.x % a.splits, unit = blockIdx.x / a.splits;
    const int kv = unit % a.kv_heads;
    const Sequence s = find_sequence<32>(a, a.offsets, a.q_rows, a.group, unit / a.kv_heads, lane);
    if (s.tile < 0 || (long long)s.tile * 32 >= (long long)s.n * a.group) return;
    const FewRow me = few_row(a, s, kv, col);
    const int shift = s.m - s.n, keys = few_keys(a, s);
    const int limit = (a.causal ? min(s.m, me.token + shift + 1) : s.m) - 1;
    const Parts parts(a, keys);
    const int begin = part * parts.chunk, end = min(parts.tiles, begin + parts.chunk);
    if (part >= parts.used) return;

    const char* K = row_of(a.K, kv, s.k0);
    const char* V = row_of(a.V, kv, s.k0);
    const tile t(lane);
    const request ask_k(lane, 0, a.K.row, a.d), ask_v(lane, 0, a.V.row, a.d);
    auto ask = [&](int j, int at) {
        const int rows = j < end ? s.m - j * FEW_KEYS : 0;
        ask_k(K + (long long)j * FEW_KEYS * a.K.row, rows, a.K.row, a.d, ring + at * STAGE, 0);
        ask_v(V + (long long)j * FEW_KEYS * a.V.row, rows, a.V.row, a.d, ring + at * STAGE + request::BYTES, 0);
    };
    Rows<ET, DP> r;
    r.clear();
    {
        const char* q = row_of(a.Q, me.head, s.q0 + me.token);
#pragma unroll
        for (int k = 0; k < tile::T; ++k)
            r.q[k] = me.there && 16 * k + 8 * hi < a.d ? Frag<ET>::load(q + (16 * k + 8 * hi) * sizeof(ET)) : Frag<ET>::zero();
    }
    if (begin + wave < end) {
        ask(begin + wave, 0);
        int at = 0;
        for (int j = begin + wave; j < end; j += WAVES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot asked for next has been read
            ask(j + WAVES, at ^ 1);
            WAIT_VMCNT(2 * request::P);
            f32x16 x[1];
            r.scores(t, ring + at * STAGE, x);
            r.hide(x, j * FEW_KEYS, limit, hi);
            r.soften(x, a.scale2);
            r.add(t, ring + at * STAGE + request::BYTES, x);
            at ^= 1;
        }
        WAIT_VMCNT(0);
    }
    LDS_BARRIER();                                         // the rings are done with: each wave's results take their place, a row of PITCH floats a query
    float* mine = reinterpret_cast<float*>(lds);
    float* sums = mine + WAVES * 32 * PITCH;
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4*)&mine[(wave * 32 + col) * PITCH + 32 * b + 8 * i + 4 * hi] = f32x4{r.o[b][4 * i], r.o[b][4 * i + 1], r.o[b][4 * i + 2], r.o[b][4 * i + 3]};
    const float sum = r.sum + other_half(r.sum);
    if (hi == 0) {
        sums[wave * 64 + col] = r.most;
        sums[wave * 64 + 32 + col] = sum;
    }
    __syncthreads();
    constexpr int QUADS = 32 * DP / 4;
    for (int i = threadIdx.x; i < QUADS; i += WAVES * 64) {
        const int q = i / (DP / 4), c = i % (DP / 4) * 4;
        float most = LOWEST, total = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, sums[w * 64 + q]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float down = exp2_fast(sums[w * 64 + q] - most);
            const f32x4 x = *(const f32x4*)&mine[(w * 32 + q) * PITCH + c];
            total = fmaf(sums[w * 64 + 32 + q], down, total);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], down, v[e]);
        }
        const FewRow f = few_row(a, s, kv, q);
        if (!f.there) continue;
        if (parts.used > 1) {
            float* to = a.partial + (size_t)blockIdx.x * partial_floats<DP>();
            *(f32x4*)&to[q * DP + c] = f32x4{v[0], v[1], v[2], v[3]};
            if (c == 0) { to[32 * DP + q] = most; to[32 * DP + 32 + q] = total; }
            continue;
        }
        const float by = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        if (c < a.d) few_store<ET, DP>(a, s, f, c, v[0] * by, v[1] * by, v[2] * by, v[3] * by);
        if (a.lse && c == 0) a.lse[(long long)f.head * a.q_rows + s.q0 + f.token] = total == 0.0f ? -INFINITY : (most + __log2f(total)) * LN2;
    }
}

// The parts of the rows' keys, joined in their order: a block a unit of 32 rows.
template <typename ET, int DP>
__global__ __launch_bounds__(256) void attend_join_kernel(attn_args a)
{
    const int unit = blockIdx.x, kv = unit % a.kv_heads;
    const Sequence s = find_sequence<32>(a, a.offsets, a.q_rows, a.group, unit / a.kv_heads, threadIdx.x & 63);
    if (s.tile < 0 || (long long)s.tile * 32 >= (long long)s.n * a.group) return;
    const Parts parts(a, few_keys(a, s));
    if (parts.used == 1) return;                           // written already
    for (int i = threadIdx.x; i < 32 * DP / 4; i += 256) {
        const int q = i / (DP / 4), c = i % (DP / 4) * 4;
        const FewRow f = few_row(a, s, kv, q);
        if (!f.there) return;                              // nor are the rows after it
        const float* from = a.partial + (size_t)unit * a.splits * partial_floats<DP>();
        float most = LOWEST, total = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < parts.used; ++p) most = fmaxf(most, from[(size_t)p * partial_floats<DP>() + 32 * DP + q]);
        for (int p = 0; p < parts.used; ++p) {
            const float* one = from + (size_t)p * partial_floats<DP>();
            const float down = exp2_fast(one[32 * DP + q] - most);
            const f32x4 x = *(const f32x4*)&one[q * DP + c];
            total = fmaf(one[32 * DP + 32 + q], down, total);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], down, v[e]);
        }
        const float by = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        if (c < a.d) few_store<ET, DP>(a, s, f, c, v[0] * by, v[1] * by, v[2] * by, v[3] * by);
        if (a.lse && c == 0) a.lse[(long long)f.head * a.q_rows + s.q0 + f.token] = total == 0.0f ? -INFINITY : (most + __log2f(total)) * LN2;
    }
}

template <typename ET, int DP, int WAVES> hipError_t launch_rows(const attn_args& a, hipStream_t st)
{
    constexpr int stage = 2 * Request<ET, DP, KEYS, WAVES>::BYTES;
    constexpr size_t bytes = (size_t)stage * stages_for(stage);
    static PerDeviceOnce once;
    const hipError_t e = allow_lds(attend_kernel<ET, DP, WAVES>, bytes, once);
    if (e != hipSuccess) return e;
    const long long slots = a.q_rows / (WAVES * 32) + a.seqs;
    hipLaunchKernelGGL((attend_kernel<ET, DP, WAVES>), dim3((unsigned)(slots * a.heads)), dim3(WAVES * 64), bytes, st, a);
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t launch_few(attn_args a, hipStream_t st)
{
    constexpr int WAVES = few_waves<ET, DP>();
    constexpr size_t ring = (size_t)WAVES * FEW_STAGES * 2 * Request<ET, DP, FEW_KEYS, 1>::BYTES, join = (size_t)WAVES * (32 * (DP + 4) + 64) * 4;
    constexpr size_t bytes = ring > join ? ring : join;
    static PerDeviceOnce once;
    hipError_t e = allow_lds(attend_few_kernel<ET, DP, WAVES>, bytes, once);
    if (e != hipSuccess) return e;
    // parts of the same number of tiles, whatever a sequence's length, so that blocks take equally long; those past a sequence's end have nothing to do
    const long long units = ((long long)a.q_rows * a.group / 32 + a.seqs) * a.kv_heads;
    const long long tiles = ((long long)a.k_rows / a.seqs + FEW_KEYS - 1) / FEW_KEYS;
    const long long want = ATTN_PARTS / units, most = (tiles + 2 * WAVES - 1) / (2 * WAVES);
    a.splits = (int)(want < most ? want : most);
    if (a.splits < 1) a.splits = 1;
    a.chunk = (int)((tiles / a.splits + WAVES) / WAVES * WAVES);
    hipLaunchKernelGGL((attend_few_kernel<ET, DP, WAVES>), dim3((unsigned)(units * a.splits)), dim3(WAVES * 64), bytes, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((attend_join_kernel<ET, DP>), dim3((unsigned)units), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t attend(const attn_args& a, hipStream_t st)
{
    // few rows: what a kv head has of an average sequence fits one block's 32 twice over
    if ((long long)a.q_rows * a.group <= 64ll * a.seqs) return launch_few<ET, DP>(a, st);
    return launch_rows<ET, DP, 8>(a, st);
}

}  // namespace

// The kept parts of a forward call of few rows, or a row's <dO, O> of a backward call.
size_t attn_workspace_bytes(const moe_attn_t& c)
{
    const int dp = c.d <= 64 ? 64 : 128;
    const long long units = ((long long)c.q_rows * (c.heads / c.kv_heads) / 32 + c.seqs) * c.kv_heads, each = c.k_rows / (FEW_KEYS * 4) + 1;
    const size_t parts = units < ATTN_PARTS && units * each < ATTN_PARTS ? units * each : ATTN_PARTS;
    const size_t fwd = parts * (32 * dp + PARTIAL_MORE) * sizeof(float), bwd = (size_t)c.heads * c.q_rows * sizeof(float);
    return ((fwd > bwd ? fwd : bwd) + 256) / 256 * 256;
}

hipError_t launch_attn_fwd(const moe_attn_t& c, const moe_heads_t& Q, const moe_heads_t& K, const moe_heads_t& V, const moe_heads_t& O, float* lse,
                           const int32_t* offsets, const int32_t* k_begin, const int32_t* k_end, void* ws, hipStream_t st)
{
    if (c.q_rows == 0 || c.seqs == 0) return hipSuccess;
    const int size = c.dtype == MOE_BF16 ? 2 : 4;
    attn_args a = attn_make(c);
    a.Q = in_bytes(Q, size), a.K = in_bytes(K, size), a.V = in_bytes(V, size), a.O = in_bytes(O, size);
    a.lse = lse, a.offsets = offsets, a.k_begin = k_begin, a.k_end = k_end;
    a.partial = (float*)ws;
    if (c.dtype == MOE_BF16) return c.d <= 64 ? attend<bf16_t, 64>(a, st) : attend<bf16_t, 128>(a, st);
    return c.d <= 64 ? attend<float, 64>(a, st) : attend<float, 128>(a, st);
}
