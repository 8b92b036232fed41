// Attention of packed sequences, forward: O = softmax(scale Q K^T) V, row by row over the keys that the row sees, and the logarithm of each row's sum.
//
// One pass over the keys with a running maximum and sum.  A wave has 32 queries and all of their results: with S^T = K Q^T a lane holds 16 scores of ONE
// query per 32 keys, so maximum and sum stay in the lane (its other half is 32 lanes on), and the exponentials are the second operand of O^T = V^T P^T
// as they lie.  The maximum in use is let go stale: rescaling the results, a rounding of each, is rare after the first tiles, and
// each row decides on it for itself: its bits do not depend on the rows beside it.
//
// Bound by the matrix cores, 4 d operations a pair of query and key, next to the vector units: a wave's 64 keys of 128 columns take 1220 to 1540 clocks of the ones and 930 to
// 1110 of the others, so one has to run under the other.  Over a cache bound by keys and values, read once for the heads that share them.
#include "attn.h"

#include <type_traits>

namespace {

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
    // Scores of NB x 32 keys from row block 0 of the tile on; the first PRE fragments, in the order of the products, are there already.
    template <int NB, int PRE> static __device__ __forceinline__ void request(const typename tile::RowsAt& at, frag (&pre)[PRE])
    {
#pragma unroll
        for (int i = 0; i < PRE; ++i) pre[i] = tile::by_rows(at, 32 * (i % NB), i / NB);
    }
    template <int NB, int PRE> __device__ __forceinline__ void scores(const typename tile::RowsAt& at, const frag (&pre)[PRE], f32x16 (&s)[NB]) const
    {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < tile::T; ++k)
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = Frag<ET>::mma(k * NB + b < PRE ? pre[k * NB + b < PRE ? k * NB + b : 0] : tile::by_rows(at, 32 * b, k), q[k], s[b]);
    }
    // Keys past `limit` are hidden from this lane's query; `first` is the key of row 0.
    template <int NB> static __device__ __forceinline__ void hide(f32x16 (&s)[NB], int first, int limit, int hi)
    {
        APART();
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = first + 32 * b + 8 * (i >> 2) + 4 * hi + (i & 3) > limit ? -INFINITY : s[b][i];
    }
    // Exponentials of the scores over the maximum in use, as they go into the products, and their sum.  Only where a row's sum of them passes STALE in a lane (one of them
    // does, or none of the row's keys came before) is the highest score looked for, the results so far scaled down to it and the exponentials formed again: a
    // maximum of every tile takes a tenth of the vector instructions.  Scores past fp32's range as exponents end there too.
    static constexpr float STALE = 1024.0f;
    template <int NB> __device__ __forceinline__ void soften(const f32x16 (&s)[NB], float scale2, frag (&p)[2 * NB])
    {
        float now = powers(s, scale2, p);
        RARELY(__any(now > STALE)) {
            APART();
            float top = s[0][0];
#pragma unroll
            for (int i = 1; i < 16 * NB; i += 2) top = highest_of(top, s[i / 16][i % 16], s[(i + 1 < 16 * NB ? i + 1 : i) / 16][(i + 1 < 16 * NB ? i + 1 : i) % 16]);
            const Halves h = halves_of(top);
            // the wave takes the branch, each row decides for itself: the others keep their maximum, and so their exponentials, and are multiplied by one
            const Halves of_row = halves_of(now);
            const bool stale = of_row.low > STALE || of_row.high > STALE;
            const float next = stale ? highest_of(most, h.low * scale2, h.high * scale2) : most, down = stale ? exp2_fast(most - next) : 1.0f;
            most = next;
            sum *= down;
#pragma unroll
            for (int b = 0; b < tile::DB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= down;
            now = powers(s, scale2, p);
        }
        sum += now;
    }
    template <int NB> __device__ __forceinline__ float powers(const f32x16 (&s)[NB], float scale2, frag (&p)[2 * NB]) const
    {
        float part[4];                                     // sums side by side: a wave alone on the vector units waits for each it needs at once
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            f32x16 e;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                e[i] = exp2_fast(fmaf(s[b][i], scale2, -most));
                part[i & 3] = b == 0 && i < 4 ? e[i] : part[i & 3] + e[i];
            }
            p[2 * b] = Frag<ET>::pack(e, 0);
            p[2 * b + 1] = Frag<ET>::pack(e, 1);
        }
        return (part[0] + part[1]) + (part[2] + part[3]);
    }
    // Results of the keys whose exponentials are p.
    template <int N> __device__ __forceinline__ void add(const typename tile::KeysAt& at, const frag (&p)[N])
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int b = 0; b < tile::DB; ++b) o[b] = Frag<ET>::mma(tile::by_keys(at, 16 * k, b), p[k], o[b]);
    }
};

// Keys of a tile: five tiles of keys and values fit LDS.
template <typename ET, int DP> constexpr int keys_of() { return DP * (int)sizeof(ET) <= 256 ? 64 : 32; }
constexpr int STAGES = 5, WAVES = 8, SIDE = WAVES * 32;
constexpr int AHEAD = 6;                                   // fragments under way

// A block has 256 queries of one head, 32 a wave; keys and values go through a ring of five tiles in LDS.  In its matrix phase j a wave forms the scores of
// tile j + 1 and adds tile j's values; in its vector phase the scores become exponentials, and the first fragments of the next matrix phase arrive.
// The two waves of a SIMD are in opposite phases, held there by a barrier at each phase's end.  Why 256 rows: a ring of 160 KB serves eight waves, two a SIMD, and a
// tile's way from the L2 all 256 rows.  One sequence of 16384, 32 and 8 heads of 128, bf16, causal: 1.71 to 1.80 ms by the
// card, 2.2 TFLOP at 1.2 to 1.3 PFLOP/s, matrix pipes 74 % busy at the 1.4 GHz that the power cap leaves (a large library product reaches 1.15 to 1.36 PFLOP/s); with waves
// that run freely 2.23 ms.  16384 rows in eleven sequences, 16 and 4 heads of 128: 204 to 218 us, 304 without phases.
template <typename ET, int DP>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_kernel(attn_args a)
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
    const int shift = s.m - s.n, first = s.tile * SIDE + wave * 32, row = first + col;     // of the sequence's queries
    // how many keys the block's, this wave's last query sees; the last key that this lane's, the wave's first sees
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
    auto ask = [&]() INLINE {                                     // the next tile; past the last one: zeros that nobody reads
        const uint32_t at = ring + asked_at;
        ask_k(K, s.m - asked, a.K.row, a.d, at, wave);
        ask_v(V, s.m - asked, a.V.row, a.d, at + request::BYTES, wave);
        K += (long long)KEYS * a.K.row;
        V += (long long)KEYS * a.V.row;
        asked += KEYS;
        asked_at = asked_at == (STAGES - 1) * (int)STAGE ? 0 : asked_at + STAGE;
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
        constexpr int N = NB * tile::T + 2 * NB * tile::DB, PRE = AHEAD < NB * tile::T ? AHEAD : NB * tile::T;
        f32x16 x[NB];
        frag p[2 * NB], pre[PRE];
        int at = 0, next = STAGE;                          // tile j's place in the ring, and that of the one after it
        auto step = [&](int& place) INLINE { place = place == (STAGES - 1) * (int)STAGE ? 0 : place + STAGE; };
        auto soften = [&](int j) INLINE {
            RARELY(j * KEYS + KEYS - 1 > least) r.hide(x, j * KEYS, limit, hi);
            r.soften(x, a.scale2, p);
        };
#pragma unroll
        for (int j = 0; j < STAGES - 1; ++j) ask();
        arrived(r.q);
        WAIT_VMCNT(2 * 2 * request::P);                    // tiles 0 and 1 have arrived
        PHASE_END();
        if (wave >= WAVES / 2) PHASE_END();                // the second half is a phase behind
        if (wave_tiles > 0) {
            const auto rows = t.rows_at(ring);
            r.template request<NB>(rows, pre);
            r.scores(rows, pre, x);
        }
        PHASE_END();
        int j = 0;
        auto vector_phase = [&](int j) INLINE {
            r.template request<NB>(t.rows_at(ring + next), pre);       // whole tiles, also past the wave's last
            soften(j);
        };
        if (wave_tiles > 0) vector_phase(0);
        // The loop closes at the end of a vector phase, ahead of its barrier: a jump waits for its instructions, and after the barrier everyone would wait with it.
        for (; j < wave_tiles - 1; ++j) {
            WAIT_VMCNT(2 * request::P);                    // tile 2 has arrived, the first time round; later nothing is left to wait for
            PHASE_END();
            const auto rows = t.rows_at(ring + next);
            const auto keys = t.keys_at(ring + at + request::BYTES);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            r.scores(rows, pre, x);
            ask();                                         // in the place of tile j - 1, which the second half was done with a phase ago
            r.add(keys, p);
            if constexpr (sizeof(ET) == 2) pace<RowsThenKeys<NB * tile::T>, N, PRE>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            WAIT_VMCNT(2 * request::P);                    // tile j + 3 has arrived
            PHASE_END();
            step(at);
            step(next);
            vector_phase(j + 1);
        }
        WAIT_VMCNT(2 * request::P);                        // as in the loop, for waves that never went through it: others read tile 2 from the next phase on
        PHASE_END();
        for (; j < tiles; ++j) {                           // this wave's last one, and those that only others see
            ask();
            if (j < wave_tiles) r.add(t.keys_at(ring + at + request::BYTES), p);
            WAIT_VMCNT(2 * request::P);
            PHASE_END();
            step(at);
            PHASE_END();
        }
        if (wave < WAVES / 2) PHASE_END();
        WAIT_VMCNT(0);
    }
    if (row >= s.n) return;
    const float sum = sum_of_halves(r.sum), by = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;     // a row that sees nothing is zero; NaN stays
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
constexpr int PARTIAL_MORE = 64;                           // of a part's 32 rows: maximum and sum
template <int DP> constexpr int partial_floats() { return 32 * DP + PARTIAL_MORE; }

template <typename ET, int DP>
__device__ __forceinline__ void few_store(const attn_args& a, const Sequence& s, const FewRow& f, int c, float v0, float v1, float v2, float v3)
{
    char* o = a.O.p + (long long)f.head * a.O.head + (long long)(s.q0 + f.token) * a.O.row;
    store_four<ET>(o + c * sizeof(ET), v0, v1, v2, v3);
}

template <typename ET, int DP, int FEW_WAVES>
__global__ __launch_bounds__(FEW_WAVES * 64, 1) void attend_few_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, FEW_KEYS, 1> request;
    typedef typename Frag<ET>::type frag;
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
    const int least = (a.causal ? min(s.m, (int)((long long)s.tile * 32 / a.group) + shift + 1) : s.m) - 1;
    const int tiles = (keys + FEW_KEYS - 1) / FEW_KEYS;
    const Parts parts(a, tiles);
    const int begin = part * parts.chunk, end = min(tiles, begin + parts.chunk);
    if (part >= parts.used) return;

    const char* K = row_of(a.K, kv, s.k0);
    const char* V = row_of(a.V, kv, s.k0);
    const tile t(lane);
    const request ask_k(lane, 0, a.K.row, a.d), ask_v(lane, 0, a.V.row, a.d);
    auto ask = [&](int j, int at) INLINE {
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
        for (int j = begin + wave; j < end; j += FEW_WAVES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot asked for next has been read
            ask(j + FEW_WAVES, at ^ 1);
            WAIT_VMCNT(2 * request::P);
            f32x16 x[1];
            frag pre[1];
            const auto rows = t.rows_at(ring + at * STAGE);
            r.template request<1>(rows, pre);
            r.scores(rows, pre, x);
            RARELY(j * FEW_KEYS + FEW_KEYS - 1 > least) r.hide(x, j * FEW_KEYS, limit, hi);
            frag p[2];
            r.soften(x, a.scale2, p);
            r.add(t.keys_at(ring + at * STAGE + request::BYTES), p);
            at ^= 1;
        }
        WAIT_VMCNT(0);
    }
    LDS_BARRIER();                                         // the rings are done with: each wave's results take their place, a row of PITCH floats a query
    float* mine = reinterpret_cast<float*>(lds);
    float* sums = mine + FEW_WAVES * 32 * PITCH;
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4*)&mine[(wave * 32 + col) * PITCH + 32 * b + 8 * i + 4 * hi] = f32x4{r.o[b][4 * i], r.o[b][4 * i + 1], r.o[b][4 * i + 2], r.o[b][4 * i + 3]};
    const float sum = sum_of_halves(r.sum);
    if (hi == 0) {
        sums[wave * 64 + col] = r.most;
        sums[wave * 64 + 32 + col] = sum;
    }
    __syncthreads();
    constexpr int QUADS = 32 * DP / 4;
    for (int i = threadIdx.x; i < QUADS; i += FEW_WAVES * 64) {
        const int q = i / (DP / 4), c = i % (DP / 4) * 4;
        float most = LOWEST, total = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) most = fmaxf(most, sums[w * 64 + q]);
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) {
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
    const Parts parts(a, (few_keys(a, s) + FEW_KEYS - 1) / FEW_KEYS);
    if (parts.used == 1) return;                           // written already
    for (int i = threadIdx.x; i < 32 * DP / 4; i += 256) {
        const int q = i / (DP / 4), c = i % (DP / 4) * 4;
        const FewRow f = few_row(a, s, kv, q);
        if (!f.there) return;                              // nor are the rows after it
        const float* from = a.partial + (size_t)unit * a.splits * partial_floats<DP>();
        float most = LOWEST, total = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < parts.used; p += 4) {          // four parts' loads are under way together
            float high[4], sums[4];
            f32x4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float* one = from + (size_t)min(p + k, parts.used - 1) * partial_floats<DP>();
                high[k] = one[32 * DP + q], sums[k] = one[32 * DP + 32 + q], x[k] = *(const f32x4*)&one[q * DP + c];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (p + k >= parts.used) break;
                const float next = fmaxf(most, high[k]), old = exp2_fast(most - next), down = exp2_fast(high[k] - next);
                most = next;
                total = fmaf(sums[k], down, total * old);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(x[k][e], down, v[e] * old);
            }
        }
        const float by = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        if (c < a.d) few_store<ET, DP>(a, s, f, c, v[0] * by, v[1] * by, v[2] * by, v[3] * by);
        if (a.lse && c == 0) a.lse[(long long)f.head * a.q_rows + s.q0 + f.token] = total == 0.0f ? -INFINITY : (most + __log2f(total)) * LN2;
    }
}

template <typename ET, int DP> hipError_t launch_rows(const attn_args& a, hipStream_t st)
{
    constexpr size_t bytes = (size_t)STAGES * 2 * Request<ET, DP, keys_of<ET, DP>(), WAVES>::BYTES;
    static PerDeviceOnce once;
    const hipError_t e = allow_lds(attend_kernel<ET, DP>, bytes, once);
    if (e != hipSuccess) return e;
    const long long slots = a.q_rows / SIDE + a.seqs;
    hipLaunchKernelGGL((attend_kernel<ET, DP>), dim3((unsigned)(slots * a.heads)), dim3(WAVES * 64), bytes, st, a);
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t launch_few(attn_args a, hipStream_t st)
{
    constexpr int FEW_WAVES = few_waves<ET, DP>();
    constexpr size_t ring = (size_t)FEW_WAVES * FEW_STAGES * 2 * Request<ET, DP, FEW_KEYS, 1>::BYTES, join = (size_t)FEW_WAVES * (32 * (DP + 4) + 64) * 4;
    constexpr size_t bytes = ring > join ? ring : join;
    static PerDeviceOnce once;
    hipError_t e = allow_lds(attend_few_kernel<ET, DP, FEW_WAVES>, bytes, once);
    if (e != hipSuccess) return e;
    // parts of the same number of tiles, whatever a sequence's length, so that blocks take equally long; those past a sequence's end have nothing to do.  Where there are
    // blocks for all CUs without them they only cost: 1024 rows, 8 heads of 128, 264 blocks, causal: 42 us with, 15 without.  A token of each of 16 sequences over 1 to 16384
    // keys, 32 and 8 heads of 128, 144 blocks, us: 2048 parts 120, 1024 111, 512 104 (517 MB, 5.0 TB/s), none 197.  Lengths are known to the device alone, so parts are as
    // long as the cache has room for: one token over 4096 keys 15 us in a cache of 4096 rows, 18 of 16384, 30 of 131072; sixteen of them 53, 49, 49
    const long long units = few_units(a);
    const long long tiles = ((long long)a.k_rows / a.seqs + FEW_KEYS - 1) / FEW_KEYS;
    const long long want = units <= 256 ? ATTN_PARTS / units : 1, most = (tiles + 2 * FEW_WAVES - 1) / (2 * FEW_WAVES);
    a.splits = (int)(want < most ? want : most);
    if (a.splits < 1) a.splits = 1;
    a.chunk = (int)((tiles / a.splits + FEW_WAVES) / FEW_WAVES * FEW_WAVES);
    hipLaunchKernelGGL((attend_few_kernel<ET, DP, FEW_WAVES>), dim3((unsigned)(units * a.splits)), dim3(FEW_WAVES * 64), bytes, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((attend_join_kernel<ET, DP>), dim3((unsigned)units), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename ET, int DP> hipError_t attend(const attn_args& a, hipStream_t st)
{
    // or few rows a sequence, whatever their number: up to 16, or 32 of heads that share nothing, over 4096 keys, 32 and 8 heads of 128, us, small | large blocks:
    // 8 rows 88 | 119, 16 86 | 120, 32 136 | 121; over 1024, 32 and 32 heads of 64: 32 rows 117 | 126, 64 158 | 132.  It is the average that counts: a sequence of
    // 16384 and 1023 empty ones, 32 and 8 heads of 128, take 4620 us so, 1710 where the call has one sequence
    if ((long long)a.q_rows <= (a.group == 1 ? 32ll : 16ll) * a.seqs || is_small<ET, DP>(((long long)a.q_rows / SIDE + a.seqs) * a.heads, false)) return launch_few<ET, DP>(a, st);
    return launch_rows<ET, DP>(a, st);
}

}  // namespace

// The kept parts of a forward call of few rows, or the rows' statistics and the kept parts of a small backward call; of this or any smaller call.
size_t attn_workspace_bytes(const moe_attn_t& c)
{
    const size_t row = 32 * (c.d <= 64 ? 64 : 128);
    const long long group = c.heads / c.kv_heads, units = ((long long)c.q_rows * group / 32 + c.seqs) * c.kv_heads, units_k = ((long long)c.k_rows / 32 + c.seqs) * c.kv_heads;
    auto most = [](long long units, long long each, long long all) { return (size_t)(units < all && units * each < all ? units * each : all); };
    const size_t fwd = most(units, c.k_rows / (FEW_KEYS * 4) + 1, ATTN_PARTS) * (row + PARTIAL_MORE) * sizeof(float);
    const size_t dq = most(units, c.k_rows / (32 * ATTN_PART_TILES) + 1, ATTN_BWD_PARTS) * row * sizeof(float);
    const size_t dkv = most(units_k, group * c.q_rows / (32 * ATTN_PART_TILES) + 1, ATTN_BWD_PARTS) * 2 * row * sizeof(float);
    const size_t bwd = attn_stats_bytes(c.heads, c.q_rows) + (dq > dkv ? dq : dkv);            // one after the other
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
