// Gradient of the attention: P is formed again from the scores and the kept logarithms of the rows' sums, never stored.
//
//   dQ_i = scale sum_j ds_ij k_j,   dK_j = scale sum_i ds_ij q_i,   dV_j = sum_i p_ij dO_i,   ds_ij = p_ij (<dO_i, v_j> - D_i),   D_i = <dO_i, O_i>
//
// Two kernels, so that no sum needs atomics and the same bits come out every time: a wave of the first has 32 queries and goes over their keys, a wave of
// the second has 32 keys and goes over the queries of all heads that share them.  Scores and <dO, v> are formed in both, 7 products for the 5 of the formulas.
#include "attn.h"

namespace {

constexpr int KEYS = 64, QUERIES = 64;                     // rows of a tile
constexpr int stages_for(int stage_bytes) { return 4 * stage_bytes <= 156 * 1024 ? 4 : 2; }

// 4 bytes a lane from a buffer into LDS at lds_base + lane * 4.
__device__ __forceinline__ void dma4(rsrc_t r, uint32_t lds_base, uint32_t voff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(lds_base), "v"(voff), "s"(r) : "memory");
}

template <typename ET, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : 1) void attend_dq_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, KEYS, WAVES> request;
    typedef typename Frag<ET>::type frag;
    constexpr int SIDE = WAVES * 32;
    constexpr uint32_t STAGE = 2 * request::BYTES;
    constexpr int STAGES = stages_for(STAGE);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int head, slot;
    head_and_slot(blockIdx.x, a.heads, head, slot);
    const Sequence s = find_sequence<SIDE>(a, a.offsets, a.q_rows, 1, gridDim.x / a.heads - 1 - slot, lane);
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.n) return;
    const int shift = s.m - s.n, first = s.tile * SIDE + wave * 32, row = first + col;
    const int block_keys = a.causal ? min(s.m, max(0, min(s.n, (s.tile + 1) * SIDE) + shift)) : s.m;
    const int wave_keys = first >= s.n ? 0 : a.causal ? min(s.m, max(0, min(s.n, first + 32) + shift)) : s.m;
    const int limit = (a.causal ? min(s.m, row + shift + 1) : s.m) - 1, least = (a.causal ? min(s.m, first + shift + 1) : s.m) - 1;
    const int tiles = (block_keys + KEYS - 1) / KEYS;

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
            if (hi == 0) a.D[at] = D;
        }
    }
    f32x16 g[tile::DB];
#pragma unroll
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) g[b][i] = 0.0f;
    if (tiles > 0) {
#pragma unroll
        for (int j = 0; j < STAGES - 1; ++j) ask(j);
        arrived(q);
        arrived(dO);
        asm volatile("" :: "v"(D), "v"(lse2));
        for (int j = 0; j < tiles; ++j) {
            WAIT_VMCNT((STAGES - 2) * 2 * request::P);     // tile j has arrived
            LDS_BARRIER();                                 // everyone's part of it, and nobody reads tile j - 1 any more
            ask(j + STAGES - 1);
            const uint32_t at = ring + (j % STAGES) * STAGE;
            const auto rows = t.rows_at(at);
            const auto keys = t.keys_at(at);
#pragma unroll
            for (int h = 0; h < KEYS / 32; ++h) {
                const int key = j * KEYS + 32 * h;
                if (key >= wave_keys) break;
                f32x16 x, y;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = y[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < tile::T; ++k) {
                    x = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k), q[k], x);
                    y = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k, request::BYTES), dO[k], y);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = exp2_fast(fmaf(x[i], a.scale2, -lse2)) * (y[i] - D);
                if (key + 31 > least) {
                    RARELY();
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = key + 8 * (i >> 2) + 4 * hi + (i & 3) > limit ? 0.0f : x[i];
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const frag ds = Frag<ET>::pack(x, k);
#pragma unroll
                    for (int b = 0; b < tile::DB; ++b) g[b] = Frag<ET>::mma(tile::by_keys(keys, 32 * h + 16 * k, b), ds, g[b]);
                }
            }
        }
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

template <typename ET, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : 1) void attend_dkv_kernel(attn_args a)
{
    typedef Tile<ET, DP> tile;
    typedef Request<ET, DP, QUERIES, WAVES> request;
    typedef typename Frag<ET>::type frag;
    constexpr int SIDE = WAVES * 32;
    constexpr uint32_t STATS = QUERIES * 4, STAGE = 2 * request::BYTES + WAVES * 2 * STATS;      // each wave has the rows' statistics to itself
    constexpr int STAGES = stages_for(STAGE);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t ring = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    int kv, slot;
    head_and_slot(blockIdx.x, a.kv_heads, kv, slot);
    const Sequence s = find_sequence<SIDE>(a, a.k_begin, a.k_rows, 1, slot, lane);
    if (s.tile < 0 || (long long)s.tile * SIDE >= s.m) return;
    const int shift = s.m - s.n, block = s.tile * SIDE, first = block + wave * 32, key = first + col;
    // the first query that sees the block's first key, this lane's, the wave's last
    const int from = a.causal ? max(0, block - shift) : 0, mine = a.causal ? key - shift : 0, last = a.causal ? first + 31 - shift : 0;
    const int start = from / QUERIES, tiles = max(0, (s.n + QUERIES - 1) / QUERIES - start), steps = tiles * a.group;

    const tile t(lane);
    const request ask_q(lane, wave, a.Q.row, a.d), ask_o(lane, wave, a.dO.row, a.d);
    int next_head = kv * a.group, next = start, slot_at = 0;
    auto ask = [&]() {                                     // the step after the last one asked for; past the end: zeros that nobody reads
        const bool there = next_head < (kv + 1) * a.group;
        const uint32_t at = ring + slot_at * STAGE;
        const int h = there ? next_head : kv * a.group, rows = there ? s.n - next * QUERIES : 0;
        const long long q = s.q0 + (long long)next * QUERIES;
        ask_q(row_of(a.Q, h, q), rows, a.Q.row, a.d, at, wave);
        ask_o(row_of(a.dO, h, q), rows, a.dO.row, a.d, at + request::BYTES, wave);
        const long long stats = (long long)h * a.q_rows + q, bytes = rows > 0 ? min(rows, QUERIES) * 4 : 0;
        dma4(make_rsrc(a.lse + stats, bytes), at + 2 * request::BYTES + wave * 2 * STATS, lane * 4);
        dma4(make_rsrc(a.D + stats, bytes), at + 2 * request::BYTES + wave * 2 * STATS + STATS, lane * 4);
        if (++next == start + tiles) { next = start; ++next_head; }
        if (++slot_at == STAGES) slot_at = 0;
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
    for (int b = 0; b < tile::DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dK[b][i] = dV[b][i] = 0.0f;
    if (steps > 0) {
#pragma unroll
        for (int j = 0; j < STAGES - 1; ++j) ask();
        arrived(K);
        arrived(V);
        int j = start, read_at = 0;
        for (int u = 0; u < steps; ++u) {
            WAIT_VMCNT((STAGES - 2) * (2 * request::P + 2));
            LDS_BARRIER();
            ask();
            const uint32_t at = ring + read_at * STAGE, stats = at + 2 * request::BYTES + wave * 2 * STATS;
            if (++read_at == STAGES) read_at = 0;
            const auto rows = t.rows_at(at);
            const auto keys = t.keys_at(at);
            const int tile_first = j * QUERIES;
            if (++j == start + tiles) j = start;
#pragma unroll 1
            for (int h = 0; h < QUERIES / 32; ++h) {
                const int query = tile_first + 32 * h;
                if (query >= s.n || query + 31 < first - shift && a.causal) continue;
                f32x16 x, y;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = y[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < tile::T; ++k) {
                    x = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k), K[k], x);
                    y = Frag<ET>::mma(tile::by_rows(rows, 32 * h, k, request::BYTES), V[k], y);
                }
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const uint32_t row = stats + (32 * h + 8 * i4 + 4 * hi) * 4;
                    const f32x4 lse = *(const LDS_PTR(f32x4))(uintptr_t)row, D = *(const LDS_PTR(f32x4))(uintptr_t)(row + STATS);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * i4 + e;
                        x[i] = exp2_fast(fmaf(x[i], a.scale2, -lse[e] * LOG2E));
                        y[i] = x[i] * (y[i] - D[e]);
                    }
                }
                if (query < last) {
                    RARELY();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const bool hidden = query + 8 * (i >> 2) + 4 * hi + (i & 3) < mine;
                        x[i] = hidden ? 0.0f : x[i];
                        y[i] = hidden ? 0.0f : y[i];
                    }
                }
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
        if (row >= s.m) continue;
        char* pk = a.dK.p + (long long)kv * a.dK.head + (long long)(s.k0 + row) * a.dK.row;
        char* pv = a.dV.p + (long long)kv * a.dV.head + (long long)(s.k0 + row) * a.dV.row;
#pragma unroll
        for (int b = 0; b < tile::DB; ++b) {
            const int c = 32 * b + col;
            if (c < a.d) {
                store_one<ET>(pk + c * sizeof(ET), dK[b][i] * a.scale);
                store_one<ET>(pv + c * sizeof(ET), dV[b][i]);
            }
        }
    }
}

template <typename ET, int DP, int WAVES> hipError_t attend_bwd(const attn_args& a, hipStream_t st)
{
    constexpr int stage_q = 2 * Request<ET, DP, KEYS, WAVES>::BYTES, stage_k = 2 * Request<ET, DP, QUERIES, WAVES>::BYTES + WAVES * 2 * QUERIES * 4;
    constexpr size_t bytes_q = (size_t)stage_q * stages_for(stage_q), bytes_k = (size_t)stage_k * stages_for(stage_k);
    static PerDeviceOnce once_q, once_k;
    hipError_t e = allow_lds(attend_dq_kernel<ET, DP, WAVES>, bytes_q, once_q);
    if (e == hipSuccess) e = allow_lds(attend_dkv_kernel<ET, DP, WAVES>, bytes_k, once_k);
    if (e != hipSuccess) return e;
    const long long slots_q = a.q_rows / (WAVES * 32) + a.seqs, slots_k = a.k_rows / (WAVES * 32) + a.seqs;
    if (a.q_rows > 0) {
        hipLaunchKernelGGL((attend_dq_kernel<ET, DP, WAVES>), dim3((unsigned)(slots_q * a.heads)), dim3(WAVES * 64), bytes_q, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.k_rows == 0) return hipSuccess;
    hipLaunchKernelGGL((attend_dkv_kernel<ET, DP, WAVES>), dim3((unsigned)(slots_k * a.kv_heads)), dim3(WAVES * 64), bytes_k, st, a);
    return hipGetLastError();
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
    a.lse = const_cast<float*>(lse), a.D = (float*)ws;
    a.offsets = offsets, a.k_begin = k_begin, a.k_end = k_end;
    if (c.dtype == MOE_BF16) return c.d <= 64 ? attend_bwd<bf16_t, 64, 8>(a, st) : attend_bwd<bf16_t, 128, 8>(a, st);
    return c.d <= 64 ? attend_bwd<float, 64, 4>(a, st) : attend_bwd<float, 128, 4>(a, st);
}
