// Gradient of the attention: P is formed again from the scores and the kept logarithms of the rows' sums, never stored.
//
//   dQ_i = scale sum_j ds_ij k_j,   dK_j = scale sum_i ds_ij q_i,   dV_j = sum_i p_ij dO_i,   ds_ij = p_ij (<dO_i, v_j> - D_i),   D_i = <dO_i, O_i>
//
// Two kernels, so that no sum needs atomics and the same bits come out every time: a wave of the first has 32 queries and goes over their keys, a wave of
// the second has 32 keys and goes over the queries of all heads that share them.  Scores and <dO, v> are formed in both, 7 products for the 5 of the formulas.
// Bound by the matrix cores (2 d operations a product and pair) beside the vector units, as the forward pass: both kernels of bf16 run in its two phases.
#include "attn.h"

#include <type_traits>

namespace {

constexpr int STAGES = 5, WAVES = 8, SIDE = WAVES * 32;
constexpr int AHEAD = 4;                                   // matrix instructions whose fragments are under way

// 4 bytes a lane from a buffer into LDS at lds_base + lane * 4.
__device__ __forceinline__ void dma4(rsrc_t r, uint32_t lds_base, uint32_t voff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(lds_base), "v"(voff), "s"(r));
}
__device__ __forceinline__ void clear(f32x16& x)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
}

// Keys of a tile of the first kernel: five tiles of keys and values fit LDS.
template <typename ET, int DP> constexpr int keys_of() { return DP * (int)sizeof(ET) <= 256 ? 64 : 32; }

// A block has 256 queries of one head, 32 a wave.  In its matrix phase j a wave adds tile j - 1's keys to the gradient and forms the scores and <dO, v> of tile j;
// in its vector phase these become ds.  Four sequences of 8192, 32 and 8 heads of 128, bf16, causal: 2.66 ms, 1.2 PFLOP/s of its three products, matrix pipes 68 % busy at
// 1.7 GHz.  In fp32 with 128 columns 28 words a lane do not fit the registers: addresses, read again under products that take 24000 clocks a tile.
template <typename ET, int DP>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_dq_kernel(attn_args a)
{
    constexpr int KEYS = keys_of<ET, DP>(), NB = KEYS / 32;
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, KEYS, WAVES> request;
    typedef typename Frag<ET>::type frag;
    constexpr uint32_t STAGE = 2 * request::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int head, slot;
    head_and_slot(blockIdx.x, a.heads, head, slot);
    const Sequence s = find_sequence<SIDE>(a, a.offsets, a.q_rows, 1, gridDim.x / a.heads - 1 - slot, lane);      // later tiles see more keys and go first
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.n) return;
    const int shift = s.m - s.n, first = s.tile * SIDE + wave * 32, row = first + col;
    const int block_keys = a.causal ? min(s.m, max(0, min(s.n, (s.tile + 1) * SIDE) + shift)) : s.m;
    const int wave_keys = first >= s.n ? 0 : a.causal ? min(s.m, max(0, min(s.n, first + 32) + shift)) : s.m;
    const int limit = (a.causal ? min(s.m, row + shift + 1) : s.m) - 1, least = (a.causal ? min(s.m, first + shift + 1) : s.m) - 1;
    const int tiles = uniform((block_keys + KEYS - 1) / KEYS), wave_tiles = uniform((wave_keys + KEYS - 1) / KEYS);

    const int kv = head / a.group;
    const char* K = row_of(a.K, kv, s.k0);
    const char* V = row_of(a.V, kv, s.k0);
    const tile t(lane);
    const request ask_k(lane, wave, a.K.row, a.d), ask_v(lane, wave, a.V.row, a.d);
    int asked = 0, asked_at = 0;                           // rows asked for, and the place of the next ones in the ring
    auto step = [&](int& place) INLINE { place = place == (STAGES - 1) * (int)STAGE ? 0 : place + STAGE; };
    auto ask = [&]() INLINE {                                     // the next tile; past the last one: zeros that nobody reads
        ask_k(K, s.m - asked, a.K.row, a.d, ring + asked_at, wave);
        ask_v(V, s.m - asked, a.V.row, a.d, ring + asked_at + request::BYTES, wave);
        K += (long long)KEYS * a.K.row;
        V += (long long)KEYS * a.V.row;
        asked += KEYS;
        step(asked_at);
    };
    frag q[tile::T], dO[tile::T];
    float D = 0.0f, lse2 = 0.0f;
    {
        const char *pq = row_of(a.Q, head, s.q0 + row), *pd = row_of(a.dO, head, s.q0 + row), *po = row_of(a.O, head, s.q0 + row);
#pragma unroll
        for (int k = 0; k < tile::T; ++k) {
            const int at = (16 * k + 8 * hi) * (int)sizeof(ET);
            const bool there = row < s.n && 16 * k + 8 * hi < a.d;
            q[k] = there ? Frag<ET>::load(pq + at) : Frag<ET>::zero();
            dO[k] = there ? Frag<ET>::load(pd + at) : Frag<ET>::zero();
            const frag o = there ? Frag<ET>::load(po + at) : Frag<ET>::zero();
#pragma unroll
            for (int e = 0; e < 8; ++e) D = fmaf(Frag<ET>::at(dO[k], e), Frag<ET>::at(o, e), D);
        }
        D = sum_of_halves(D);
        const long long at = (long long)head * a.q_rows + s.q0 + row;
        if (row < s.n) {
            lse2 = a.lse[at] * LOG2E;
            if (hi == 0) a.stats[at] = make_float2(lse2, D);
        }
    }
    f32x16 g[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b) clear(g[b]);
    if (tiles > 0) {
        constexpr int BY_KEYS = 2 * NB * tile::DB, N = BY_KEYS + 2 * NB * tile::T, PRE = sizeof(ET) == 4 ? 1 : AHEAD < BY_KEYS ? AHEAD : BY_KEYS;
        f32x16 x[NB], y[NB];
        frag ds[2 * NB], pre[PRE];
        int at = 0;                                        // the place of the tile in hand
        auto scores = [&](int place) INLINE {
            const auto rows = t.rows_at(ring + place);
#pragma unroll
            for (int h = 0; h < NB; ++h) {
                clear(x[h]);
                clear(y[h]);
            }
#pragma unroll
            for (int k = 0; k < tile::T; ++k)
#pragma unroll
                for (int h = 0; h < NB; ++h) {
                    x[h] = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k), q[k], x[h]);
                    y[h] = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k, request::BYTES), dO[k], y[h]);
                }
        };
        auto add = [&](const typename tile::KeysAt& keys) INLINE {
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k)
#pragma unroll
                for (int b = 0; b < tile::DB; ++b) {
                    const int i = k * tile::DB + b;
                    g[b] = Frag<ET>::mma(i < PRE ? pre[i < PRE ? i : 0] : tile::by_keys(keys, 16 * k, b), ds[k], g[b]);
                }
        };
        auto request_first = [&]() INLINE {                       // of the tile in hand's keys
            const auto keys = t.keys_at(ring + at);
#pragma unroll
            for (int i = 0; i < PRE; ++i) pre[i] = tile::by_keys(keys, 16 * (i / tile::DB), i % tile::DB);
        };
        auto soften = [&](int j) INLINE {
#pragma unroll
            for (int h = 0; h < NB; ++h) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[h][i] = exp2_fast(fmaf(x[h][i], a.scale2, -lse2)) * (y[h][i] - D);
                const int key = j * KEYS + 32 * h;
                RARELY(key + 31 > least) {
                    APART();
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[h][i] = key + 8 * (i >> 2) + 4 * hi + (i & 3) > limit ? 0.0f : x[h][i];
                }
                ds[2 * h] = Frag<ET>::pack(x[h], 0);
                ds[2 * h + 1] = Frag<ET>::pack(x[h], 1);
            }
        };
#pragma unroll
        for (int j = 0; j < STAGES - 2; ++j) ask();
        arrived(q);
        arrived(dO);
        WAIT_VMCNT(2 * 2 * request::P);                    // tile 0 has arrived
        PHASE_END();
        if (wave >= WAVES / 2) PHASE_END();                // the second half is a phase behind
        ask();
        if (wave_tiles > 0) scores(0);
        WAIT_VMCNT(2 * 2 * request::P);                    // tile 1
        PHASE_END();
        int j = 0;
        auto vector_phase = [&](int j) INLINE {
            request_first();
            soften(j);
        };
        if (wave_tiles > 0) vector_phase(0);
        // The loop closes at the end of a vector phase, ahead of its barrier: a jump waits for its instructions, and after the barrier everyone would wait with it.
        for (; j < wave_tiles - 1; ++j) {
            PHASE_END();
            const auto keys = t.keys_at(ring + at);
            step(at);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            add(keys);
            ask();                                         // in the place of tile j - 1, which the second half was done with a phase ago
            scores(at);
            if constexpr (sizeof(ET) == 2) pace<KeysThenRows<BY_KEYS>, N, PRE>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            WAIT_VMCNT(2 * 2 * request::P);                // tile j + 2 has arrived
            PHASE_END();
            vector_phase(j + 1);
        }
        PHASE_END();
        for (; j < tiles; ++j) {                           // this wave's last one, and those that only others see
            ask();
            if (j == wave_tiles - 1) add(t.keys_at(ring + at));
            WAIT_VMCNT(2 * 2 * request::P);
            PHASE_END();
            PHASE_END();
        }
        if (wave < WAVES / 2) PHASE_END();
        WAIT_VMCNT(0);
    }
    if (row >= s.n) return;
    char* out = a.dQ.p + (long long)head * a.dQ.head + (long long)(s.q0 + row) * a.dQ.row;
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 32 * b + 8 * i + 4 * hi;
            if (c < a.d)
                store_four<ET>(out + c * sizeof(ET), g[b][4 * i] * a.scale, g[b][4 * i + 1] * a.scale, g[b][4 * i + 2] * a.scale, g[b][4 * i + 3] * a.scale);
        }
}

template <typename ET> __device__ __forceinline__ void store_one(char* p, float v)
{
    if constexpr (sizeof(ET) == 2) *(bf16_t*)p = f32_to_bf16(v);
    else *(float*)p = v;
}

// Scores and <dO, v> of 32 queries (rows) and keys (columns) to p and ds; the queries' statistics lie at `stats`, a pair each.
__device__ __forceinline__ void weigh(f32x16& x, f32x16& y, uint32_t stats, float scale2, int hi)
{
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const f32x4 of = *(const LDS_PTR(f32x4))(uintptr_t)(stats + (8 * (i >> 2) + 4 * hi + (i & 3)) * 8);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            x[i + e] = exp2_fast(fmaf(x[i + e], scale2, -of[2 * e]));
            y[i + e] = x[i + e] * (y[i + e] - of[2 * e + 1]);
        }
    }
}
// Queries before `mine` do not see this lane's key; `first` is the query of row 0.
__device__ __forceinline__ void hide_queries(f32x16& x, f32x16& y, int first, int mine, int hi)
{
    APART();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const bool hidden = first + 8 * (i >> 2) + 4 * hi + (i & 3) < mine;
        x[i] = hidden ? 0.0f : x[i];
        y[i] = hidden ? 0.0f : y[i];
    }
}

template <typename ET> __device__ __forceinline__ void store_keys(const attn_args& a, const Sequence& s, int kv, int row, int c, float dk, float dv)
{
    store_one<ET>(a.dK.p + (long long)kv * a.dK.head + (long long)(s.k0 + row) * a.dK.row + c * (int)sizeof(ET), dk * a.scale);
    store_one<ET>(a.dV.p + (long long)kv * a.dV.head + (long long)(s.k0 + row) * a.dV.row + c * (int)sizeof(ET), dv);
}

// The queries that a block of keys goes over, head by head of those that share them, ROWS at a time.
template <int ROWS> struct Walk {
    int first_head, heads, start, tiles, steps;            // tiles of a head from `start` on, where the first query sees the block's first key
    int head, tile;                                        // the next one to be asked for
    __device__ __forceinline__ Walk(const attn_args& a, const Sequence& s, int kv, int block)
    {
        first_head = kv * a.group, heads = a.group;
        const int from = a.causal ? max(0, block - (s.m - s.n)) : 0;
        start = from / ROWS;
        tiles = uniform(max(0, (s.n + ROWS - 1) / ROWS - start));
        steps = tiles * heads;
        head = first_head, tile = start;
    }
    __device__ __forceinline__ bool there() const { return head < first_head + heads; }
    __device__ __forceinline__ void next() { if (++tile == start + tiles) { tile = start; ++head; } }
};

// fp32: a block has WAVES x 32 keys, keys and values in registers.  Its matrix instructions take eight times as long as those of bf16: what a wave does beside them counts
// for little.  Only calls past is_small come here: 4096 rows, 32 heads of 64, see the figures there.
template <int DP>
__global__ __launch_bounds__(256, 1) void attend_dkv_f32_kernel(attn_args a)
{
    constexpr int WAVES = 4, SIDE = 128, QUERIES = 64, STAGES = 2;
    typedef float ET;
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, QUERIES, WAVES> request;
    typedef typename Frag<ET>::type frag;
    constexpr uint32_t STATS = QUERIES * 8, STAGE = 2 * request::BYTES + WAVES * STATS;      // each wave has the rows' statistics to itself
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int kv, slot;
    head_and_slot(blockIdx.x, a.kv_heads, kv, slot);
    const Sequence s = find_sequence<SIDE>(a, a.k_begin, a.k_rows, 1, slot, lane);      // earlier tiles are seen by more queries and go first
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.m) return;
    const int shift = s.m - s.n, block = s.tile * SIDE, first = block + wave * 32, key = first + col;
    const int mine = a.causal ? key - shift : 0, last = a.causal ? first + 31 - shift : 0;      // the first query that sees this lane's key, the wave's last

    const tile t(lane);
    const request ask_q(lane, wave, a.Q.row, a.d), ask_o(lane, wave, a.dO.row, a.d);
    Walk<QUERIES> walk(a, s, kv, block);
    int slot_at = 0;
    auto ask = [&]() INLINE {                                     // past the end: zeros that nobody reads
        const bool there = walk.there();
        const uint32_t at = ring + slot_at * STAGE;
        const int h = there ? walk.head : walk.first_head, rows = there ? s.n - walk.tile * QUERIES : 0;
        const long long q = s.q0 + (long long)walk.tile * QUERIES;
        ask_q(row_of(a.Q, h, q), rows, a.Q.row, a.d, at, wave);
        ask_o(row_of(a.dO, h, q), rows, a.dO.row, a.d, at + request::BYTES, wave);
        const rsrc_t r = tile_rsrc((const char*)(a.stats + (long long)h * a.q_rows + q), rows > 0 ? min(rows, QUERIES) * 8 : 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) dma4(r, at + 2 * request::BYTES + wave * STATS + i * 256, lane * 4 + i * 256);
        walk.next();
        slot_at ^= 1;
    };
    frag K[tile::T], V[tile::T];
    {
        const char *pk = row_of(a.K, kv, s.k0 + key), *pv = row_of(a.V, kv, s.k0 + key);
#pragma unroll
        for (int k = 0; k < tile::T; ++k) {
            const int at = (16 * k + 8 * hi) * (int)sizeof(ET);
            const bool there = key < s.m && 16 * k + 8 * hi < a.d;
            K[k] = there ? Frag<ET>::load(pk + at) : Frag<ET>::zero();
            V[k] = there ? Frag<ET>::load(pv + at) : Frag<ET>::zero();
        }
    }
    f32x16 dK[tile::DB], dV[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b) {
        clear(dK[b]);
        clear(dV[b]);
    }
    if (walk.steps > 0) {
        ask();
        arrived(K);
        arrived(V);
        int j = walk.start;
        for (int u = 0; u < walk.steps; ++u) {
            WAIT_VMCNT(0);
            LDS_BARRIER();
            const uint32_t at = ring + (u & 1) * STAGE, stats = at + 2 * request::BYTES + wave * STATS;
            ask();
            const auto rows = t.rows_at(at);
            const auto keys = t.keys_at(at);
            const int tile_first = j * QUERIES;
            if (++j == walk.start + walk.tiles) j = walk.start;
#pragma unroll 1
            for (int h = 0; h < QUERIES / 32; ++h) {
                const int query = tile_first + 32 * h;
                if (query >= s.n || (a.causal && query + 31 < first - shift)) continue;
                f32x16 x, y;
                clear(x);
                clear(y);
#pragma unroll
                for (int k = 0; k < tile::T; ++k) {
                    x = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k), K[k], x);
                    y = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k, request::BYTES), V[k], y);
                }
                weigh(x, y, stats + 32 * h * 8, a.scale2, hi);
                RARELY(query < last) hide_queries(x, y, query, mine, hi);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const frag p = Frag<ET>::pack(x, k), ds = Frag<ET>::pack(y, k);
#pragma unroll
                    for (int b = 0; b < tile::DB; ++b) {
                        dV[b] = Frag<ET>::mma(p, tile::by_keys(keys, 32 * h + 16 * k, b, request::BYTES), dV[b]);
                        dK[b] = Frag<ET>::mma(ds, tile::by_keys(keys, 32 * h + 16 * k, b), dK[b]);
                    }
                }
            }
        }
        WAIT_VMCNT(0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = first + 8 * (i >> 2) + 4 * hi + (i & 3);
#pragma unroll
        for (int b = 0; b < tile::DB; ++b)
            if (row < s.m && 32 * b + col < a.d) store_keys<ET>(a, s, kv, row, 32 * b + col, dK[b][i], dV[b][i]);
    }
}

// bf16: a block has 256 keys, 32 a wave, and goes over 32 queries at a time.  In its matrix phase u a wave adds the products of tile u - 1 to both gradients and forms
// the scores and <dO, v> of tile u; in its vector phase these become p and ds.  Registers: 32 rows of two gradients, of keys and of scores; the values, which
// would be 32 more, lie in LDS (128 columns).  Tiles that causality hides from a wave's keys are worked on with zeros: no wave leaves the common step.
// Four sequences of 8192, 32 and 8 heads of 128, causal: 3.94 ms, 1.12 PFLOP/s of its four products, matrix pipes 58 % busy at 1.7 GHz, LDS 43 %: a tile's queries and their
// gradients are each wanted by rows and by keys, and the values too.
struct DkvReads {
    static constexpr int of(int i, int by_keys, bool v_in_lds) { return i < by_keys ? 2 : v_in_lds && ((i - by_keys) & 1) ? 2 : 1; }
};
template <int BY_KEYS, bool V_IN_LDS> struct DkvOrder { static constexpr int of(int i) { return DkvReads::of(i, BY_KEYS, V_IN_LDS); } };

template <int DP> struct Dkv {
    typedef Tile<bf16_t, DP> tile;
    static constexpr bool V_IN_LDS = DP == 128, HALVES = DP == 64;      // 32 rows of 64 columns are a request each of four waves: half of them ask for Q, half for dO
    typedef Request<bf16_t, DP, 32, HALVES ? WAVES / 2 : WAVES> request;
    static constexpr int REQUESTS = HALVES ? 1 : 2 * request::P;
    static constexpr uint32_t STATS = 1024, STAGE = 2 * request::BYTES + STATS, VALUES = V_IN_LDS ? SIDE * tile::ROW : 0;
    static constexpr size_t LDS = VALUES + (size_t)STAGES * STAGE;
};

template <int DP>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_dkv_kernel(attn_args a)
{
    typedef bf16_t ET;
    typedef Dkv<DP> D;
    typedef typename D::tile tile;
    typedef typename D::request request;
    typedef Frag<ET>::type frag;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t values = (uint32_t)(uintptr_t)(LDS_PTR(char))lds, ring = values + D::VALUES;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int kv, slot;
    head_and_slot(blockIdx.x, a.kv_heads, kv, slot);
    const Sequence s = find_sequence<SIDE>(a, a.k_begin, a.k_rows, 1, slot, lane);      // earlier tiles are seen by more queries and go first
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.m) return;
    const int shift = s.m - s.n, block = s.tile * SIDE, first = block + wave * 32, key = first + col;
    const int mine = a.causal ? key - shift : 0, last = a.causal ? first + 31 - shift : 0;      // the first query that sees this lane's key, the wave's last

    const tile t(lane);
    const bool second = wave >= WAVES / 2;
    const request ask_q(lane, D::HALVES ? wave & 3 : wave, D::HALVES && second ? a.dO.row : a.Q.row, a.d), ask_o(lane, wave, a.dO.row, a.d);
    Walk<32> walk(a, s, kv, block);
    int asked_at = 0;
    auto step = [&](int& place) INLINE { place = place == (STAGES - 1) * (int)D::STAGE ? 0 : place + (int)D::STAGE; };
    auto ask = [&]() INLINE {                                     // past the end: zeros that nobody reads
        const bool there = walk.there();
        const uint32_t at = ring + asked_at;
        const int h = there ? walk.head : walk.first_head, rows = there ? s.n - walk.tile * 32 : 0;
        const long long q = s.q0 + (long long)walk.tile * 32;
        if constexpr (D::HALVES) {
            const heads_t& x = second ? a.dO : a.Q;
            ask_q(row_of(x, h, q), rows, x.row, a.d, second ? at + request::BYTES : at, wave & 3);
        } else {
            ask_q(row_of(a.Q, h, q), rows, a.Q.row, a.d, at, wave);
            ask_o(row_of(a.dO, h, q), rows, a.dO.row, a.d, at + request::BYTES, wave);
        }
        if (wave == 0)                                     // 32 rows' statistics, one request for all waves
            dma4(tile_rsrc((const char*)(a.stats + (long long)h * a.q_rows + q), rows > 0 ? min(rows, 32) * 8 : 0), at + 2 * request::BYTES, lane * 4);
        walk.next();
        step(asked_at);
    };
    // All but the requests of the last `n` tiles have arrived.
    auto wait = [&](auto n) INLINE {
        if (wave == 0) WAIT_VMCNT(decltype(n)::value * (D::REQUESTS + 1));
        else WAIT_VMCNT(decltype(n)::value * D::REQUESTS);
    };
    frag K[tile::T], V[D::V_IN_LDS ? 1 : tile::T];
    {
        const char *pk = row_of(a.K, kv, s.k0 + key), *pv = row_of(a.V, kv, s.k0 + key);
#pragma unroll
        for (int k = 0; k < tile::T; ++k) {
            const int at = (16 * k + 8 * hi) * (int)sizeof(ET);
            const bool there = key < s.m && 16 * k + 8 * hi < a.d;
            K[k] = there ? Frag<ET>::load(pk + at) : Frag<ET>::zero();
            if constexpr (!D::V_IN_LDS) V[k] = there ? Frag<ET>::load(pv + at) : Frag<ET>::zero();
        }
    }
    f32x16 dK[tile::DB], dV[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b) {
        clear(dK[b]);
        clear(dV[b]);
    }
    if (walk.steps > 0) {
        // Requests are made in the shorter phase: 128 columns' is that of the vector units (the whole gradient of the case above 6.76 -> 6.69 ms), 64 columns' that of the matrix cores (855 us, 947 the other way).
        constexpr bool LATE = DP == 128;
        constexpr int BY_KEYS = 4 * tile::DB, N = BY_KEYS + 2 * tile::T, PRE = AHEAD < BY_KEYS ? AHEAD : BY_KEYS;
        f32x16 x, y;
        frag p[2], ds[2], pre[PRE];
        int at = 0, j = walk.start;                        // the place of the tile in hand, and which of a head's it is
        if constexpr (D::V_IN_LDS) {
            const Request<ET, DP, SIDE, WAVES> ask_v(lane, wave, a.V.row, a.d);
            ask_v(row_of(a.V, kv, s.k0 + block), s.m - block, a.V.row, a.d, values, wave);
        }
        auto scores = [&](int place) INLINE {
            const auto rows = t.rows_at(ring + place);
            typename tile::RowsAt mine;                    // the same rows of the wave's values
#pragma unroll
            for (int k = 0; k < tile::T; ++k) mine.at[k] = rows.at[k] + (values + wave * 32 * tile::ROW - ring - place);
            clear(x);
            clear(y);
#pragma unroll
            for (int k = 0; k < tile::T; ++k) {
                x = Frag<ET>::mma(tile::by_rows(rows, 0, k), K[k], x);
                y = Frag<ET>::mma(tile::by_rows(rows, 0, k, request::BYTES), D::V_IN_LDS ? tile::by_rows(mine, 0, k) : V[D::V_IN_LDS ? 0 : k], y);
            }
        };
        // product i of a tile's 4 DB: 16 queries, 32 columns, dV and dK in turn
        auto operand = [&](const typename tile::KeysAt& keys, int i) INLINE { return tile::by_keys(keys, 16 * (i / (2 * tile::DB)), i / 2 % tile::DB, i & 1 ? 0 : request::BYTES); };
        auto add = [&](const typename tile::KeysAt& keys) INLINE {
#pragma unroll
            for (int i = 0; i < BY_KEYS; ++i) {
                const frag f = i < PRE ? pre[i < PRE ? i : 0] : operand(keys, i);
                const int k = i / (2 * tile::DB), b = i / 2 % tile::DB;
                if (i & 1) dK[b] = Frag<ET>::mma(ds[k], f, dK[b]);
                else dV[b] = Frag<ET>::mma(p[k], f, dV[b]);
            }
        };
        auto request_first = [&]() INLINE {                       // of the tile in hand's products
            const auto keys = t.keys_at(ring + at);
#pragma unroll
            for (int i = 0; i < PRE; ++i) pre[i] = operand(keys, i);
        };
        auto soften = [&]() INLINE {
            weigh(x, y, ring + at + 2 * request::BYTES, a.scale2, hi);
            RARELY(j * 32 < last) hide_queries(x, y, j * 32, mine, hi);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                p[k] = Frag<ET>::pack(x, k);
                ds[k] = Frag<ET>::pack(y, k);
            }
            RARELY(++j == walk.start + walk.tiles) j = walk.start;
        };
#pragma unroll
        for (int i = 0; i < STAGES - 2; ++i) ask();
        arrived(K);
        arrived(V);
        wait(std::integral_constant<int, 2>{});            // the values and tile 0
        PHASE_END();
        if (second) PHASE_END();                           // the second half is a phase behind
        if constexpr (!LATE) ask();
        scores(0);
        wait(std::integral_constant<int, LATE ? 1 : 2>{});             // tile 1
        PHASE_END();
        request_first();
        if constexpr (LATE) ask();
        soften();
        for (int u = 1; u < walk.steps; ++u) {             // closes as the one above
            PHASE_END();
            const auto keys = t.keys_at(ring + at);
            step(at);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            add(keys);
            scores(at);
            pace<DkvOrder<BY_KEYS, D::V_IN_LDS>, N, PRE>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            if constexpr (!LATE) ask();                    // in the place of tile u - 2, which the second half was done with a phase ago
            wait(std::integral_constant<int, LATE ? 1 : 2>{});         // tile u + 1 has arrived
            PHASE_END();
            request_first();
            if constexpr (LATE) ask();
            soften();
        }
        PHASE_END();
        add(t.keys_at(ring + at));
        if (!second) PHASE_END();
        WAIT_VMCNT(0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = first + 8 * (i >> 2) + 4 * hi + (i & 3);
#pragma unroll
        for (int b = 0; b < tile::DB; ++b)
            if (row < s.m && 32 * b + col < a.d) store_keys<ET>(a, s, kv, row, 32 * b + col, dK[b][i], dV[b][i]);
    }
}

template <typename ET, int DP> struct FewDkv { static constexpr uint32_t STAGE = 2 * Request<ET, DP, 32, 1>::BYTES + 256; };

// Small calls, dQ: a block has 32 rows of a sequence and kv head, its waves take tiles of 32 keys in turn.
template <typename ET, int DP, int FEW_WAVES>
__global__ __launch_bounds__(FEW_WAVES * 64, 1) void attend_dq_few_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, FEW_KEYS, 1> request;
    typedef typename Frag<ET>::type frag;
    constexpr int PITCH = DP + 4;
    constexpr uint32_t STAGE = 2 * request::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + wave * FEW_STAGES * STAGE;
    const int part = blockIdx.x % a.splits, unit = blockIdx.x / a.splits, kv = unit % a.kv_heads;
    const Sequence s = find_sequence<32>(a, a.offsets, a.q_rows, a.group, unit / a.kv_heads, lane);
    if (s.tile < 0 || (long long)s.tile * 32 >= (long long)s.n * a.group) return;
    const FewRow me = few_row(a, s, kv, col);
    const int shift = s.m - s.n, tiles = uniform((few_keys(a, s) + FEW_KEYS - 1) / FEW_KEYS);
    const Parts parts(a, tiles);
    const int begin = part * parts.chunk + wave, end = uniform(min(tiles, (part + 1) * parts.chunk));
    if (part >= parts.used) return;
    const int limit = (a.causal ? min(s.m, me.token + shift + 1) : s.m) - 1, least = (a.causal ? min(s.m, (int)((long long)s.tile * 32 / a.group) + shift + 1) : s.m) - 1;

    const char* K = row_of(a.K, kv, s.k0);
    const char* V = row_of(a.V, kv, s.k0);
    const tile t(lane);
    const request ask_k(lane, 0, a.K.row, a.d), ask_v(lane, 0, a.V.row, a.d);
    auto ask = [&](int j, int at) INLINE {
        const int rows = j < end ? s.m - j * FEW_KEYS : 0;
        ask_k(K + (long long)j * FEW_KEYS * a.K.row, rows, a.K.row, a.d, ring + at * STAGE, 0);
        ask_v(V + (long long)j * FEW_KEYS * a.V.row, rows, a.V.row, a.d, ring + at * STAGE + request::BYTES, 0);
    };
    if (begin < end) ask(begin, 0);
    frag q[tile::T], dO[tile::T];
    float D = 0.0f, lse2 = 0.0f;
    {
        const long long row = s.q0 + me.token;
        const char *pq = row_of(a.Q, me.head, row), *pd = row_of(a.dO, me.head, row), *po = row_of(a.O, me.head, row);
#pragma unroll
        for (int k = 0; k < tile::T; ++k) {
            const int at = (16 * k + 8 * hi) * (int)sizeof(ET);
            const bool there = me.there && 16 * k + 8 * hi < a.d;
            q[k] = there ? Frag<ET>::load(pq + at) : Frag<ET>::zero();
            dO[k] = there ? Frag<ET>::load(pd + at) : Frag<ET>::zero();
            const frag o = there ? Frag<ET>::load(po + at) : Frag<ET>::zero();
#pragma unroll
            for (int e = 0; e < 8; ++e) D = fmaf(Frag<ET>::at(dO[k], e), Frag<ET>::at(o, e), D);
        }
        D = sum_of_halves(D);
        const long long at = (long long)me.head * a.q_rows + row;
        if (me.there) {
            lse2 = a.lse[at] * LOG2E;
            if (hi == 0 && wave == 0 && part == 0) a.stats[at] = make_float2(lse2, D);
        }
    }
    f32x16 g[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b) clear(g[b]);
    arrived(q);
    arrived(dO);
    if (begin < end) {
        int at = 0;
        for (int j = begin; j < end; j += FEW_WAVES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot asked for next has been read
            ask(j + FEW_WAVES, at ^ 1);
            WAIT_VMCNT(2 * request::P);
            const auto rows = t.rows_at(ring + at * STAGE);
            const auto keys = t.keys_at(ring + at * STAGE);
            f32x16 x, y;
            clear(x);
            clear(y);
#pragma unroll
            for (int k = 0; k < tile::T; ++k) {
                x = Frag<ET>::mma(tile::by_rows(rows, 0, k), q[k], x);
                y = Frag<ET>::mma(tile::by_rows(rows, 0, k, request::BYTES), dO[k], y);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = exp2_fast(fmaf(x[i], a.scale2, -lse2)) * (y[i] - D);
            const int key = j * FEW_KEYS;
            RARELY(key + 31 > least) {
                APART();
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = key + 8 * (i >> 2) + 4 * hi + (i & 3) > limit ? 0.0f : x[i];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const frag ds = Frag<ET>::pack(x, k);
#pragma unroll
                for (int b = 0; b < tile::DB; ++b) g[b] = Frag<ET>::mma(tile::by_keys(keys, 16 * k, b), ds, g[b]);
            }
            at ^= 1;
        }
        WAIT_VMCNT(0);
    }
    LDS_BARRIER();                                         // the rings are done with: each wave's sums take their place
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4*)&sums[(wave * 32 + col) * PITCH + 32 * b + 8 * i + 4 * hi] = f32x4{g[b][4 * i], g[b][4 * i + 1], g[b][4 * i + 2], g[b][4 * i + 3]};
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * DP / 4; i += FEW_WAVES * 64) {
        const int r = i / (DP / 4), c = i % (DP / 4) * 4;
        const FewRow f = few_row(a, s, kv, r);
        if (!f.there || c >= a.d) continue;
        f32x4 v = *(const f32x4*)&sums[r * PITCH + c];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) {
            const f32x4 x = *(const f32x4*)&sums[(w * 32 + r) * PITCH + c];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e];
        }
        if (parts.used > 1) {
            *(f32x4*)&a.partial[((size_t)blockIdx.x * 32 + r) * DP + c] = v;
            continue;
        }
        store_four<ET>(a.dQ.p + (long long)f.head * a.dQ.head + (long long)(s.q0 + f.token) * a.dQ.row + c * (int)sizeof(ET), v[0] * a.scale, v[1] * a.scale, v[2] * a.scale,
                       v[3] * a.scale);
    }
}

// Small calls, dK and dV: a block has 32 keys, its waves take tiles of 32 queries, of all heads that share the keys, in turn.
template <typename ET, int DP, int FEW_WAVES>
__global__ __launch_bounds__(FEW_WAVES * 64, 1) void attend_dkv_few_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, 32, 1> request;
    typedef typename Frag<ET>::type frag;
    constexpr int PITCH = DP + 4, REQUESTS = 2 * request::P + 1;
    constexpr uint32_t STAGE = FewDkv<ET, DP>::STAGE;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + wave * FEW_STAGES * STAGE;
    const int part = blockIdx.x % a.splits, unit = blockIdx.x / a.splits, kv = unit % a.kv_heads;
    const Sequence s = find_sequence<32>(a, a.k_begin, a.k_rows, 1, unit / a.kv_heads, lane);
    if (s.tile < 0 || (long long)s.tile * 32 >= s.m) return;
    const int shift = s.m - s.n, first = s.tile * 32, key = first + col;
    const int mine = a.causal ? key - shift : 0, last = a.causal ? first + 31 - shift : 0;      // the first query that sees this lane's key, the block's last

    const tile t(lane);
    const request ask_q(lane, 0, a.Q.row, a.d), ask_o(lane, 0, a.dO.row, a.d);
    const Walk<32> walk(a, s, kv, first);
    const Parts parts(a, walk.steps);
    const int begin = part * parts.chunk + wave, end = uniform(min(walk.steps, (part + 1) * parts.chunk));
    if (part >= parts.used) return;
    auto ask = [&](int u, int at) INLINE {
        const int h = u < end ? u / walk.tiles : 0, j = u < end ? walk.start + u - h * walk.tiles : 0, rows = u < end ? s.n - j * 32 : 0;
        const long long q = s.q0 + (long long)j * 32;
        const int head = walk.first_head + h;
        ask_q(row_of(a.Q, head, q), rows, a.Q.row, a.d, ring + at * STAGE, 0);
        ask_o(row_of(a.dO, head, q), rows, a.dO.row, a.d, ring + at * STAGE + request::BYTES, 0);
        dma4(tile_rsrc((const char*)(a.stats + (long long)head * a.q_rows + q), rows > 0 ? min(rows, 32) * 8 : 0), ring + at * STAGE + 2 * request::BYTES, lane * 4);
    };
    if (begin < end) ask(begin, 0);
    frag K[tile::T], V[tile::T];
    {
        const char *pk = row_of(a.K, kv, s.k0 + key), *pv = row_of(a.V, kv, s.k0 + key);
#pragma unroll
        for (int k = 0; k < tile::T; ++k) {
            const int at = (16 * k + 8 * hi) * (int)sizeof(ET);
            const bool there = key < s.m && 16 * k + 8 * hi < a.d;
            K[k] = there ? Frag<ET>::load(pk + at) : Frag<ET>::zero();
            V[k] = there ? Frag<ET>::load(pv + at) : Frag<ET>::zero();
        }
    }
    f32x16 dK[tile::DB], dV[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b) {
        clear(dK[b]);
        clear(dV[b]);
    }
    arrived(K);
    arrived(V);
    if (begin < end) {
        int at = 0;
        for (int u = begin; u < end; u += FEW_WAVES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot asked for next has been read
            ask(u + FEW_WAVES, at ^ 1);
            WAIT_VMCNT(REQUESTS);
            const auto rows = t.rows_at(ring + at * STAGE);
            const auto keys = t.keys_at(ring + at * STAGE);
            const int query = (walk.start + u % walk.tiles) * 32;
            f32x16 x, y;
            clear(x);
            clear(y);
#pragma unroll
            for (int k = 0; k < tile::T; ++k) {
                x = Frag<ET>::mma(tile::by_rows(rows, 0, k), K[k], x);
                y = Frag<ET>::mma(tile::by_rows(rows, 0, k, request::BYTES), V[k], y);
            }
            weigh(x, y, ring + at * STAGE + 2 * request::BYTES, a.scale2, hi);
            RARELY(query < last) hide_queries(x, y, query, mine, hi);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const frag p = Frag<ET>::pack(x, k), ds = Frag<ET>::pack(y, k);
#pragma unroll
                for (int b = 0; b < tile::DB; ++b) {
                    dV[b] = Frag<ET>::mma(p, tile::by_keys(keys, 16 * k, b, request::BYTES), dV[b]);
                    dK[b] = Frag<ET>::mma(ds, tile::by_keys(keys, 16 * k, b), dK[b]);
                }
            }
            at ^= 1;
        }
        WAIT_VMCNT(0);
    }
    // one gradient after the other through the place of the rings
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        LDS_BARRIER();
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int b = 0; b < tile::DB; ++b) sums[(wave * 32 + 8 * (i >> 2) + 4 * hi + (i & 3)) * PITCH + 32 * b + col] = which ? dV[b][i] : dK[b][i];
        __syncthreads();
        const heads_t& to = which ? a.dV : a.dK;
        const float by = which ? 1.0f : a.scale;
        for (int i = threadIdx.x; i < 32 * DP / 4; i += FEW_WAVES * 64) {
            const int r = i / (DP / 4), c = i % (DP / 4) * 4;
            if (first + r >= s.m || c >= a.d) continue;
            f32x4 v = *(const f32x4*)&sums[r * PITCH + c];
#pragma unroll
            for (int w = 1; w < FEW_WAVES; ++w) {
                const f32x4 x = *(const f32x4*)&sums[(w * 32 + r) * PITCH + c];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += x[e];
            }
            if (parts.used > 1) *(f32x4*)&a.partial_k[(((size_t)blockIdx.x * 2 + which) * 32 + r) * DP + c] = v;
            else store_four<ET>(to.p + (long long)kv * to.head + (long long)(s.k0 + first + r) * to.row + c * (int)sizeof(ET), v[0] * by, v[1] * by, v[2] * by, v[3] * by);
        }
    }
}

// The parts of small calls' gradients, joined in their order: blockIdx.x is a unit of the one kernel (of_keys 0) or the other.
template <typename ET, int DP>
__global__ __launch_bounds__(256) void attend_bwd_join_kernel(attn_args a, int of_keys)
{
    const int unit = blockIdx.x, kv = unit % a.kv_heads, lane = threadIdx.x & 63;
    const Sequence s = of_keys ? find_sequence<32>(a, a.k_begin, a.k_rows, 1, unit / a.kv_heads, lane) : find_sequence<32>(a, a.offsets, a.q_rows, a.group, unit / a.kv_heads, lane);
    if (s.tile < 0 || (long long)s.tile * 32 >= (of_keys ? (long long)s.m : (long long)s.n * a.group)) return;
    const Parts parts(a, of_keys ? Walk<32>(a, s, kv, s.tile * 32).steps : (few_keys(a, s) + FEW_KEYS - 1) / FEW_KEYS);
    if (parts.used == 1) return;                           // written already
    for (int i = blockIdx.y * 256 + threadIdx.x; i < (of_keys ? 2 : 1) * 32 * DP / 4; i += 256 * gridDim.y) {
        const int which = i / (32 * DP / 4), r = i / (DP / 4) % 32, c = i % (DP / 4) * 4;
        const FewRow f = few_row(a, s, kv, r);
        if ((of_keys ? s.tile * 32 + r >= s.m : !f.there) || c >= a.d) continue;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < parts.used; ++p) {
            const size_t from = (size_t)unit * a.splits + p;
            const f32x4 x = *(const f32x4*)(of_keys ? &a.partial_k[((from * 2 + which) * 32 + r) * DP + c] : &a.partial[(from * 32 + r) * DP + c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e];
        }
        const float by = which ? 1.0f : a.scale;
        char* to = of_keys ? (which ? a.dV.p + (long long)kv * a.dV.head + (long long)(s.k0 + s.tile * 32 + r) * a.dV.row
                                    : a.dK.p + (long long)kv * a.dK.head + (long long)(s.k0 + s.tile * 32 + r) * a.dK.row)
                           : a.dQ.p + (long long)f.head * a.dQ.head + (long long)(s.q0 + f.token) * a.dQ.row;
        store_four<ET>(to + c * (int)sizeof(ET), v[0] * by, v[1] * by, v[2] * by, v[3] * by);
    }
}

// Parts of a small call's blocks where those leave CUs without one: enough for ATTN_BWD_PARTS blocks in all, of ATTN_PART_TILES tiles at least for sequences eight times as
// long as the average (fp32, 2003 rows in six sequences: the keys' gradients 108 -> 63 us with their join).
inline void cut(attn_args& a, long long units, long long tiles_of_all)
{
    const long long longest = a.seqs > 8 ? tiles_of_all * 8 / a.seqs : tiles_of_all;
    const long long want = units < 256 ? ATTN_BWD_PARTS / units : 1, most = longest / ATTN_PART_TILES;
    a.splits = (int)(want < most ? want : most);
    if (a.splits < 1) a.splits = 1;
    a.chunk = ATTN_PART_TILES;
}

template <typename ET, int DP> hipError_t launch_dq(attn_args a, hipStream_t st)
{
    const long long blocks = ((long long)a.q_rows / SIDE + a.seqs) * a.heads;
    static PerDeviceOnce once, once_few;
    hipError_t e;
    if (is_small<ET, DP>(blocks, true)) {
        constexpr int W = few_waves<ET, DP>();
        constexpr size_t join = (size_t)W * 32 * (DP + 4) * 4, ring = (size_t)W * FEW_STAGES * 2 * Request<ET, DP, FEW_KEYS, 1>::BYTES, bytes = ring > join ? ring : join;
        if ((e = allow_lds(attend_dq_few_kernel<ET, DP, W>, bytes, once_few)) != hipSuccess) return e;
        const long long units = few_units(a);
        cut(a, units, a.k_rows / 32);
        hipLaunchKernelGGL((attend_dq_few_kernel<ET, DP, W>), dim3((unsigned)(units * a.splits)), dim3(W * 64), bytes, st, a);
        if ((e = hipGetLastError()) != hipSuccess || a.splits == 1) return e;
        hipLaunchKernelGGL((attend_bwd_join_kernel<ET, DP>), dim3((unsigned)units, 32 * DP / 4 / 256), dim3(256), 0, st, a, 0);
    } else {
        constexpr size_t bytes = (size_t)STAGES * 2 * Request<ET, DP, keys_of<ET, DP>(), WAVES>::BYTES;
        if ((e = allow_lds(attend_dq_kernel<ET, DP>, bytes, once)) != hipSuccess) return e;
        hipLaunchKernelGGL((attend_dq_kernel<ET, DP>), dim3((unsigned)blocks), dim3(WAVES * 64), bytes, st, a);
    }
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t launch_dkv(attn_args a, hipStream_t st)
{
    const long long blocks = ((long long)a.k_rows / SIDE + a.seqs) * a.kv_heads;
    static PerDeviceOnce once, once_few;
    hipError_t e;
    if (is_small<ET, DP>(blocks, true)) {
        constexpr int W = few_waves<ET, DP>();
        constexpr size_t join = (size_t)W * 32 * (DP + 4) * 4, ring = (size_t)W * FEW_STAGES * FewDkv<ET, DP>::STAGE, bytes = ring > join ? ring : join;
        if ((e = allow_lds(attend_dkv_few_kernel<ET, DP, W>, bytes, once_few)) != hipSuccess) return e;
        const long long units = ((long long)a.k_rows / 32 + a.seqs) * a.kv_heads;
        cut(a, units, (long long)a.group * a.q_rows / 32);
        hipLaunchKernelGGL((attend_dkv_few_kernel<ET, DP, W>), dim3((unsigned)(units * a.splits)), dim3(W * 64), bytes, st, a);
        if ((e = hipGetLastError()) != hipSuccess || a.splits == 1) return e;
        hipLaunchKernelGGL((attend_bwd_join_kernel<ET, DP>), dim3((unsigned)units, 2 * 32 * DP / 4 / 256), dim3(256), 0, st, a, 1);
    } else if constexpr (sizeof(ET) == 2) {
        if ((e = allow_lds(attend_dkv_kernel<DP>, Dkv<DP>::LDS, once)) != hipSuccess) return e;
        hipLaunchKernelGGL((attend_dkv_kernel<DP>), dim3((unsigned)blocks), dim3(WAVES * 64), Dkv<DP>::LDS, st, a);
    } else {
        constexpr size_t bytes = 2 * (2 * Request<float, DP, 64, 4>::BYTES + 4 * 64 * 8);
        if ((e = allow_lds(attend_dkv_f32_kernel<DP>, bytes, once)) != hipSuccess) return e;
        hipLaunchKernelGGL((attend_dkv_f32_kernel<DP>), dim3((unsigned)((a.k_rows / 128 + a.seqs) * a.kv_heads)), dim3(256), bytes, st, a);
    }
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t attend_bwd(const attn_args& a, hipStream_t st)
{
    const hipError_t e = a.q_rows > 0 ? launch_dq<ET, DP>(a, st) : hipSuccess;         // leaves the statistics that the other one reads
    return e != hipSuccess || a.k_rows == 0 ? e : launch_dkv<ET, DP>(a, st);
}

}  // namespace

hipError_t launch_attn_bwd(const moe_attn_t& c, const moe_heads_t& dO, const moe_heads_t& Q, const moe_heads_t& K, const moe_heads_t& V, const moe_heads_t& O,
                           const float* lse, const int32_t* offsets, const int32_t* k_begin, const int32_t* k_end, const moe_heads_t& dQ, const moe_heads_t& dK,
                           const moe_heads_t& dV, void* ws, hipStream_t st)
{
    if (c.seqs == 0) return hipSuccess;
    const int size = c.dtype == MOE_BF16 ? 2 : 4;
    attn_args a = attn_make(c);
    a.Q = in_bytes(Q, size), a.K = in_bytes(K, size), a.V = in_bytes(V, size), a.O = in_bytes(O, size), a.dO = in_bytes(dO, size);
    a.dQ = in_bytes(dQ, size), a.dK = in_bytes(dK, size), a.dV = in_bytes(dV, size);
    a.lse = const_cast<float*>(lse), a.stats = (float2*)ws;
    a.partial = (float*)((char*)ws + attn_stats_bytes(c.heads, c.q_rows));
    a.offsets = offsets, a.k_begin = k_begin, a.k_end = k_end;
    a.partial_k = a.partial;                               // the first kernel's parts are joined before the second one runs
    if (c.dtype == MOE_BF16) return c.d <= 64 ? attend_bwd<bf16_t, 64>(a, st) : attend_bwd<bf16_t, 128>(a, st);
    return c.d <= 64 ? attend_bwd<float, 64>(a, st) : attend_bwd<float, 128>(a, st);
}
