// What the kernels that stage tiles of 16-bit operands through LDS for the matrix cores have in common: geometries, LDS layouts,
// fragment reads, and the requests that go from memory straight into LDS.
#pragma once

#include "internal.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
#define LDS_PTR(T) __attribute__((address_space(3))) T*

// Tile geometries.  Contraction slices of 32 are staged through a ring of LDS buffers.
//   Large: 256 x 256 outputs per block of 8 waves of 128 x 64, one block per CU (a 5-deep ring of 32 KB: all of LDS).
//   Small: 128 x 128 outputs per block of 4 waves of 64 x 64, two blocks per CU (5-deep rings of 16 KB).
constexpr int BK = 32;
template <int WGM_, int WGN_, int TM_, int TN_, int STAGES_, int BLOCKS_> struct Geometry {
    static constexpr int WGM = WGM_, WGN = WGN_, TM = TM_, TN = TN_, STAGES = STAGES_, BLOCKS = BLOCKS_;
    static constexpr int NWAVES = WGM * WGN, THREADS = NWAVES * 64;
    static constexpr int WM = 32 * TM, WN = 32 * TN, BM = WM * WGM, BN = WN * WGN;
    static constexpr uint32_t A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int PA = A_BYTES / 1024 / NWAVES, PB = B_BYTES / 1024 / NWAVES;   // 1-KB DMA pieces per wave and slice
    static constexpr int EP_PITCH = WN * 4 + 16;           // epilogue patch: bytes per staged row of WN floats (padded against bank conflicts)
    static constexpr int EP_ROWS = 32;                     // rows a wave stages at a time: two rows of fragments
    static constexpr int EP_WAVE = EP_ROWS * EP_PITCH;
    static constexpr size_t LDS_BYTES = (size_t)STAGES * STAGE_BYTES;
    static constexpr bool TWO_PHASE = BLOCKS == 1 && NWAVES == 8;      // the rows of waves of a block alternate; else the blocks of a CU do
    static constexpr int UNIT_BYTES = BM * BN * 4;         // a partial tile of a K-split round
    static_assert(LDS_BYTES >= (size_t)NWAVES * EP_WAVE && BLOCKS * LDS_BYTES <= 160 * 1024, "patches inside the ring, rings inside LDS");
    static_assert(WGM == 2 && WGN % 2 == 0, "the two halves of a K-contiguous operand's rows belong to one row of waves or half the columns");
};
typedef Geometry<2, 4, 4, 2, 5, 1> Large;
typedef Geometry<2, 2, 2, 2, 5, 2> Small;

// ---- LDS layouts (byte offsets inside one operand buffer) --------------------------------------
// K-contiguous operand (NN and NT fetch it in whole 128-byte lines): a buffer holds 128 rows x 64 steps (two
// slices of 32), 128 bytes per row, its eight 16-byte pieces XOR-swizzled by the row so that 16 consecutive rows of
// one piece cover all banks.
__device__ __forceinline__ uint32_t halfpair_off(int row, int piece8) { return row * 128 + ((piece8 ^ ((row >> 1) & 7)) << 4); }
// K-major operand, 32 steps x COLS columns: two steps beside each other, 64 columns (a 128-byte line of memory) of one and of
// the other in turn, the four 16-column chunks of a line XOR-swizzled by bits 1 and 3 of the step.  A transposing load takes
// four steps of every lane block, and its lane blocks are eight steps apart: the eight steps that 32 lanes touch differ in
// bits 0, 1 and 3, and their chunks of one column group cover all banks.
__device__ __forceinline__ int kmajor_swizzle(int krow) { return ((krow >> 1) & 1) | ((krow >> 2) & 2); }
template <int COLS>
__device__ __forceinline__ uint32_t kmajor_off(int krow, int col)
{
    return (krow >> 1) * (COLS * 4) + (col >> 6) * 256 + (krow & 1) * 128 + ((((col >> 4) & 3) ^ kmajor_swizzle(krow)) << 5) + (col & 15) * 2;
}
// The inverse for the DMA: byte offset in memory of the 16-byte piece that belongs at slot L of such a buffer.
template <int COLS>
__device__ __forceinline__ uint32_t kmajor_source(int L, long ld)
{
    constexpr int PER_PAIR = COLS / 4;                     // slots of two steps
    const int in_pair = L % PER_PAIR, part = L & 7, krow = L / PER_PAIR * 2 + ((in_pair >> 3) & 1);
    const int col = (in_pair >> 4) * 64 + (((part >> 1) ^ kmajor_swizzle(krow)) << 4) + (part & 1) * 8;
    return (uint32_t)((krow * ld + col) * 2);
}

// Fragment = 16 rows (or columns) x 32 contraction steps; lane l holds row l%16, steps 8*(l/16)..+7.
// Fragment reads are issued as assembly and waited for by hand (WAIT_FRAGS below): the compiler's
// own wait insertion cannot express "the set loaded one iteration ago is complete" and would stall
// every MFMA group on the fragments that were only just requested for the next iteration.
template <int IMM, typename FRAG>
__device__ __forceinline__ void lds_frag_kcontig_at(FRAG& f, uint32_t addr)
{
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f) : "v"(addr), "n"(IMM));
}
// The transposing load works on blocks of 16 lanes: lane s of a block points at 4 consecutive columns
// of step s/4; lane i of the block receives column i of steps 0..3.  Two loads give the 8 steps of a
// lane in the same order as the K-contiguous fragment.  IMM: a constant distance added to the address.
template <int STEP4_BYTES, int IMM, typename FRAG>
__device__ __forceinline__ void lds_frag_kmajor_at(FRAG& f, uint32_t addr)
{
    s16x4 lo, hi;
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n\tds_read_b64_tr_b16 %1, %2 offset:%4"
                 : "=&v"(lo), "=&v"(hi) : "v"(addr), "n"(IMM), "n"(IMM + STEP4_BYTES));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    f = __builtin_bit_cast(FRAG, v);
}

typedef __attribute__((ext_vector_type(4))) int rsrc_t;     // raw buffer resource (4 scalar registers)
typedef __amdgpu_buffer_rsrc_t buf_rsrc_t;                   // the same thing as the store builtin wants it
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

__device__ __forceinline__ rsrc_t make_rsrc(const void* base, long long bytes)
{
    if (bytes < 0) bytes = 0;
    if (bytes > 0xffffffffll) bytes = 0xffffffffll;
    const unsigned long long b = (unsigned long long)base;
    rsrc_t r;
    r[0] = (int)(unsigned)(b & 0xffffffffull);
    r[1] = (int)(unsigned)((b >> 32) & 0xffffull);         // stride 0: raw buffer, byte offsets
    r[2] = (int)(unsigned)bytes;                           // bytes past this limit read as zero
    r[3] = 0x00020000;
    return r;
}

// 16 bytes per lane from a buffer straight into LDS at lds_base + lane*16 (lds_base is uniform and
// goes through M0); bytes past the end of the buffer arrive as zeros.  Issued as assembly so that
// the compiler does not serialise later LDS reads of other ring slots behind it; completion is
// tracked by hand with WAIT_VMCNT before the barrier that publishes the slot.
template <bool NT = false>
__device__ __forceinline__ void dma16(rsrc_t r, uint32_t lds_base, uint32_t voff, uint32_t soff)
{
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                     :: "s"(lds_base), "v"(voff), "s"(r), "s"(soff) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(lds_base), "v"(voff), "s"(r), "s"(soff) : "memory");
}

#define WAIT_VMCNT(n) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(n) : "memory")
#define BLOCK_BARRIER() asm volatile("s_barrier" ::: "memory")

}  // namespace
