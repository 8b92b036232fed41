"""The attention's large kernels exchange tiles through rings in LDS that hardware fills on its own (requests, waited for by count) and barriers publish.  Here their bodies, as
they stand in the sources, are compiled for the host with every operation replaced by a note of it, and the notes of a block's waves are put side by side: what a wave
reads from LDS has arrived, for every wave that asked for a part of it, before a barrier that lies ahead of the read; nothing is asked for into a place that is still read;
tiles come in their order; all waves meet as often.  What the compiler adds (waits of its own for registers) does not count: the sources say the order by themselves.  No GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2411_10003_amd import build as hip_build

STUBS = r"""
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <type_traits>
#include <vector>
using std::max;
using std::min;
#define __global__
#define __device__
#define __shared__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define INLINE
#define RARELY(condition) if (condition)
#define APART()
#define LDS_PTR(T) T*
#define __builtin_amdgcn_sched_barrier(n)
#define __builtin_amdgcn_s_setprio(n)
#define PHASE_END() printf("B ")
#define LDS_BARRIER() printf("B ")
#define WAIT_VMCNT(n) printf("W%d ", (int)(n))
static uint32_t lds_at;
static void note_read(uint32_t at) { printf("R%u ", at - lds_at); }
static void note_request(uint32_t at, uint32_t bytes, int pieces) { printf("Q%u,%u,%d ", at - lds_at, bytes, pieces); }
struct { unsigned x; } threadIdx, blockIdx, gridDim = {2};
struct bf16_t { uint16_t v; };
struct f32x16 { float v[16]; float& operator[](int i) { return v[i]; } const float& operator[](int i) const { return v[i]; } };
struct float2 { float x, y; };
static float2 make_float2(float x, float y) { return {x, y}; }
struct heads_t { char* p; uint32_t row; long long head; };
struct attn_args {
    heads_t Q, K, V, O, dO, dQ, dK, dV;
    float* lse;
    float2* stats;
    const int32_t *offsets, *k_begin, *k_end;
    int q_rows, k_rows, seqs, heads, kv_heads, group, d, causal, splits, chunk;
    float scale, scale2;
    float *partial, *partial_k;
};
struct Sequence { int q0, n, k0, m, tile; };
static Sequence the_sequence;
template <int SIDE> Sequence find_sequence(const attn_args&, const int32_t*, int, int, int, int) { return the_sequence; }
static void head_and_slot(int, int, int& head, int& slot) { head = slot = 0; }
static int uniform(int v) { return v; }
static const char* row_of(const heads_t& t, int, long long) { return t.p; }
struct Halves { float low, high; };
static Halves halves_of(float v) { return {v, v}; }
static float highest_of(float a, float b, float c) { return max(a, max(b, c)); }
static float sum_of_halves(float v) { return v; }
static float exp2_fast(float x) { return x; }
static bool __any(bool b) { return b; }
#define __log2f log2f
constexpr float LOG2E = 1.0f, LN2 = 1.0f, LOWEST = -1.0f;
struct Fragment {};
template <typename ET> struct Frag {
    typedef Fragment type;
    static f32x16 mma(Fragment, Fragment, f32x16 c) { return c; }
    static Fragment pack(const f32x16&, int) { return {}; }
    static Fragment load(const char*) { return {}; }
    static Fragment zero() { return {}; }
    static float at(const Fragment&, int) { return 0.0f; }
};
template <typename ET, int DP> struct Tile {
    static constexpr int ROW = DP * (int)sizeof(ET), PPR = ROW / 16, T = DP / 16, DB = DP / 32;
    typedef Fragment frag;
    Tile(int) {}
    struct RowsAt { uint32_t at[T]; };
    struct KeysAt { uint32_t at; };
    RowsAt rows_at(uint32_t base) const { RowsAt r; for (auto& v : r.at) v = base; return r; }
    KeysAt keys_at(uint32_t base) const { return {base}; }
    static frag by_rows(const RowsAt& r, int row0, int t, int beyond = 0) { note_read(r.at[t] + row0 * ROW + beyond); return {}; }
    static frag by_keys(const KeysAt& k, int row0, int, int beyond = 0) { note_read(k.at + row0 * ROW + beyond); return {}; }
};
template <typename ET, int DP, int ROWS, int WAVES> struct Request {
    typedef Tile<ET, DP> tile;
    static constexpr int P = ROWS * tile::PPR / 64 / WAVES;
    static constexpr uint32_t BYTES = ROWS * tile::ROW;
    Request(int, int, uint32_t, int) {}
    void operator()(const char*, int, uint32_t, int, uint32_t base, int) const { note_request(base, BYTES, P); }
};
typedef int rsrc_t;
static rsrc_t tile_rsrc(const char*, uint32_t) { return 0; }
static void dma4(rsrc_t, uint32_t base, uint32_t) { note_request(base, 256, 1); }
template <typename T, int N> void arrived(const T (&)[N]) {}
template <typename READS, int N, int AHEAD> void pace() {}
template <int ROWS> struct RowsThenKeys {};
template <int KEYS> struct KeysThenRows {};
template <typename ET> void store_four(char*, float, float, float, float) {}
template <typename ET> void store_keys(const attn_args&, const Sequence&, int, int, int, float, float) {}
static void weigh(f32x16&, f32x16&, uint32_t stats, float, int) { note_read(stats); }
static void hide_queries(f32x16&, f32x16&, int, int, int) {}
"""

MAIN = r"""
int main(int argc, char** argv)
{
    const int n = atoi(argv[2]), m = atoi(argv[3]);
    attn_args a = {};
    a.q_rows = n, a.k_rows = m, a.seqs = 1, a.heads = a.group = 2, a.kv_heads = 1, a.d = 64, a.causal = atoi(argv[4]);
    a.scale = a.scale2 = 1.0f;
    std::vector<float> lse(2 * n + 1);
    std::vector<float2> stats(2 * n + 1);
    a.lse = lse.data(), a.stats = stats.data();
    the_sequence = {0, n, 0, m, atoi(argv[5])};
    const int waves = atoi(argv[6]);
    for (int w = 0; w < waves; ++w) {
        threadIdx.x = w * 64;
        switch (atoi(argv[1])) {
            KERNELS
        }
        printf("\n");
    }
}
"""

# kernel, waves and rows of a block, places of its ring
KERNELS = [("fwd::attend_kernel<bf16_t, 64>", 8, 256, 5), ("fwd::attend_kernel<bf16_t, 128>", 8, 256, 5), ("fwd::attend_kernel<float, 64>", 8, 256, 5), ("fwd::attend_kernel<float, 128>", 8, 256, 5),
           ("bwd::attend_dq_kernel<bf16_t, 64>", 8, 256, 5), ("bwd::attend_dq_kernel<bf16_t, 128>", 8, 256, 5), ("bwd::attend_dq_kernel<float, 64>", 8, 256, 5),
           ("bwd::attend_dq_kernel<float, 128>", 8, 256, 5), ("bwd::attend_dkv_kernel<64>", 8, 256, 5), ("bwd::attend_dkv_kernel<128>", 8, 256, 5),
           ("bwd::attend_dkv_f32_kernel<64>", 4, 128, 2), ("bwd::attend_dkv_f32_kernel<128>", 4, 128, 2)]


def _piece(text, name, above="template"):
    """A struct or function of the source, from the line above it on that begins so (None: from its name)."""
    at = text.index(name)
    start, i, depth = at if above is None else text.rindex("\n" + above, 0, at), text.index("{", at), 0
    while True:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
        if depth == 0:
            return text[start:i] + (";" if name.startswith("struct") else "")


def _constants(text):
    return "\n".join(re.findall(r"^(?:constexpr int (?:STAGES|AHEAD)\b.*|template <typename ET, int DP> constexpr int keys_of.*)$", text, re.M))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    read = lambda name: open(os.path.join(hip_build.CSRC, name)).read()  # noqa: E731
    fwd, bwd = read("attn.hip"), read("attn_bwd.hip")
    parts = [STUBS, "namespace fwd { alignas(1024) char lds[1024];", _constants(fwd), _piece(fwd, "struct Rows"), _piece(fwd, "attend_kernel(attn_args a)"), "}",
             "namespace bwd { alignas(1024) char lds[1024];", _constants(bwd), _piece(bwd, "void clear(f32x16& x)", "__device__"), _piece(bwd, "attend_dq_kernel(attn_args a)"),
             _piece(bwd, "struct Walk"), _piece(bwd, "attend_dkv_f32_kernel(attn_args a)"), _piece(bwd, "struct DkvReads", None),
             _piece(bwd, "struct DkvOrder"), _piece(bwd, "struct Dkv "), _piece(bwd, "attend_dkv_kernel(attn_args a)"), "}"]
    cases = "\n".join(f"case {i}: lds_at = (uint32_t)(uintptr_t){k[0][:3]}::lds; {k[0]}(a); break;" for i, k in enumerate(KERNELS))
    folder = tmp_path_factory.mktemp("phases")
    source, binary = str(folder / "phases.cpp"), str(folder / "phases")
    with open(source, "w") as f:
        f.write("\n".join(parts) + MAIN.replace("KERNELS", cases))
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-w", source, "-o", binary], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:4000]
    return binary


def _notes(program, kernel, n, m, causal, tile):
    """A list of notes of each wave of a block: ("B",), ("W", count), ("Q", place, bytes, pieces), ("R", address)."""
    waves = KERNELS[kernel][1]
    r = subprocess.run([program, *map(str, (kernel, n, m, int(causal), tile, waves))], capture_output=True, text=True)
    assert r.returncode == 0
    out = []
    for line in r.stdout.splitlines():
        notes = []
        for word in line.split():
            note = (word[0], *(int(v) for v in word[1:].split(",") if v))
            if not notes or notes[-1] != note or note[0] != "R":
                notes.append(note)
        out.append(notes)
    assert len(out) == waves
    return out


class Asked:
    def __init__(self, wave, segment):
        self.wave, self.segment, self.arrived = wave, segment, None        # between which of the wave's barriers it was asked for, and waited for


def check(waves, places, skips=False):
    """Raises AssertionError where the order that the notes say leaves a read or a request to chance.  skips: a wave may pass over tiles that are hidden from its rows."""
    assert len({sum(note[0] == "B" for note in notes) for notes in waves}) == 1, "waves that meet a different number of times"
    asked, reads = {}, []                                  # per place (address, bytes) all requests; (wave, segment, address, own requests so far)
    for w, notes in enumerate(waves):
        segment, under_way, own = 0, [], {}
        for note in notes:
            if note[0] == "B":
                segment += 1
            elif note[0] == "Q":
                one = Asked(w, segment)
                asked.setdefault(note[1:3], []).append(one)
                own[note[1:3]] = own.get(note[1:3], 0) + 1
                under_way += [one] * note[3]
            elif note[0] == "W":
                done = len(under_way) - note[1]
                for one in under_way[:max(done, 0)]:
                    one.arrived = segment if one not in under_way[max(done, 0):] else one.arrived
                under_way = under_way[max(done, 0):]
            else:
                reads.append((w, segment, note[1], dict(own), [id(one) for one in under_way]))
        assert not under_way, f"wave {w} ends with requests under way"
    last, rings = {}, {}
    for place in asked:
        rings.setdefault(place[1], []).append(place[0])
    rings = {size: sorted(of_size) for size, of_size in rings.items() if len(of_size) % places == 0}
    for w, segment, address, own, own_under_way in reads:
        place, = [p for p in asked if p[0] <= address < p[0] + p[1]] or [None]
        assert place is not None, f"wave {w} reads {address}: nobody asks for it"
        versions = []
        for x in sorted({one.wave for one in asked[place]}):
            of_x, before = [one for one in asked[place] if one.wave == x], 0
            for i, one in enumerate(of_x):
                if x == w:
                    if i < own.get(place, 0):
                        before += 1
                        assert id(one) not in own_under_way, f"wave {w} reads {place} ahead of its own wait"
                    else:
                        assert one.segment > segment, f"wave {w} asks into {place} in the segment in which it reads it"
                else:
                    assert one.segment != segment, f"wave {x} asks into {place} while wave {w} reads it (segment {segment})"
                    if one.segment < segment:
                        before += 1
                        assert one.arrived is not None and one.arrived < segment, f"wave {w} reads {place} in segment {segment}: wave {x}'s part is not waited for"
            versions.append(before)
        assert len(set(versions)) == 1 and versions[0] > 0, f"wave {w} reads {place}: asked for {versions} times"
        # tiles in their order: the places of a ring lie one behind the other, all with the same parts
        ring = rings.get(place[1])
        if ring:
            parts = len(ring) // places
            tile, part = (versions[0] - 1) * places + ring.index(place[0]) // parts, ring.index(place[0]) % parts
            before = last.get((w, place[1], part))
            assert before is None or tile in (before, before + 1) or (skips and tile > before), f"wave {w}: tile {tile} after {before}"
            last[w, place[1], part] = tile
    return len(reads)


LENGTHS = [(256, 256), (44, 300), (100, 300), (128, 1000), (1, 700), (129, 700), (160, 500), (200, 64), (225, 193), (300, 300), (513, 700), (700, 100), (300, 33), (31, 4000), (96, 161), (256, 288)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kernel", range(len(KERNELS)), ids=[k[0] for k in KERNELS])
def test_order_of_requests_and_reads(program, kernel, causal):
    name, _, side, places = KERNELS[kernel]
    seen = 0
    for n, m in LENGTHS:
        for tile in range(((m if "dkv" in name else n) + side - 1) // side):
            seen += check(_notes(program, kernel, n, m, causal, tile), places, skips="f32" in name)
    assert seen > 1000


def test_the_check_itself(program):
    """Mistakes put into the notes are found: a wait left out, a barrier, a request too early."""
    for kernel, earlier in ((0, 3), (4, 1), (9, 2)):
        notes = _notes(program, kernel, 256, 2000, False, 0)
        assert check(notes, 5)
        waits = [i for i, note in enumerate(notes[6]) if note[0] == "W"]
        wrong = [list(w) for w in notes]
        for i in waits[:-1]:
            wrong[6][i] = ("W", 1000)
        with pytest.raises(AssertionError, match="is not waited for|ahead of its own wait"):
            check(wrong, 5)
        wrong = [list(w) for w in notes]
        wrong[3].remove(("B",))
        with pytest.raises(AssertionError, match="different number"):
            check(wrong, 5)
        wrong = [list(w) for w in notes]
        for w in wrong:                                    # a request of the loop so many phases earlier that its place is still read (keys are read two phases ahead of values)
            barriers = [i for i, note in enumerate(w) if note[0] == "B"]
            i = next(i for i, note in enumerate(w) if note[0] == "Q" and i > barriers[6])
            w.insert([b for b in barriers if b < i][-earlier], w.pop(i))
        with pytest.raises(AssertionError, match="while wave|in the segment"):
            check(wrong, 5)
