"""Attention of packed sequences, forward, against the formulas in 64 bits (attn_util: values and bounds): widths, groups of heads, lengths from none to more
than a block's rows, keys more and fewer than queries, layouts, keys in a cache, rows that see nothing, values that no row may see."""
import math
import os
import re

import pytest
import torch

import attn_util as A
import gpu_util as G
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu


def _parts(lens, keys=None, begin=None):
    q = k = 0
    out = []
    for i, n in enumerate(lens):
        m = n if keys is None else keys[i]
        out.append((q, n, k if begin is None else begin[i], m))
        q, k = q + n, k + m
    return out


def _run(at, Q, K, V, off, where=None, stats=True):
    O = torch.full((Q.shape[0], Q.shape[1], Q.shape[2]), 7.0, dtype=Q.dtype, device=G.DEV)
    lse = torch.full((Q.shape[1], Q.shape[0]), 7.0, device=G.DEV) if stats else None
    b, e = where if where is not None else (None, None)
    at.fwd(Q, K, V, O, off, k_begin=b, k_end=e, lse=lse)
    return O, lse


def _check(Q, K, V, lens, dtype, *, causal=True, keys=None, begin=None, scale=None):
    parts = _parts(lens, keys, begin)
    heads, kv, d = Q.shape[1], K.shape[1], Q.shape[2]
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=Q.shape[0], k_rows=K.shape[0], seqs=len(lens), causal=causal, scale=scale, device=G.DEV)
    where = None
    if keys is not None:
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=G.DEV)  # noqa: E731
        where = i32([p[2] for p in parts]), i32([p[2] + p[3] for p in parts])
    O, lse = _run(at, Q, K, V, A.offsets(lens), where)
    wO, bO, wl, bl = A.forward(Q, K, V, parts, scale or d ** -0.5, causal)
    assert A.near(O, wO, bO), ("O", float(((O.double() - wO).abs() / bO).nan_to_num().max()))
    assert A.near(lse, wl, bl), ("lse", float(((lse.double() - wl).abs() / bl).nan_to_num().max()))
    O2, _ = _run(at, Q, K, V, A.offsets(lens), where, stats=False)         # nothing kept, and again: the same bits
    assert torch.equal(O, O2)
    return O, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 56, 64, 72, 80, 96, 104, 120, 128])
def test_widths(d, dtype):
    lens = [1, 37, 64, 65, 0, 130, 300]
    Q, K, V = A.tensors(sum(lens), (4, 2, 2), d, A.TYPES[dtype], "fused", d)
    _check(Q, K, V, lens, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 8), (16, 8), (8, 1)])
def test_groups_of_heads(heads, kv, dtype):
    lens = [5, 257, 33, 512]
    Q, K, V = A.tensors(sum(lens), (heads, kv, kv), 64, A.TYPES[dtype], "apart", heads * 10 + kv)
    _check(Q, K, V, lens, dtype)


# More blocks of 256 queries, or of 256 keys, than there are CUs: fewer are worked on by the kernels of few rows.
MANY = [300, 1, 0, 257, 64, 513, 31, 700, 256]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,keys", [([44, 100], [300, 700]), ([1, 128], [500, 1000]), ([300, 96], [300, 161])])
def test_blocks_whose_later_waves_have_no_rows(lens, keys, d, causal, dtype):
    """At most half of a large block's rows are there, over enough keys for every place of the ring."""
    heads = 264 // len(lens)
    Q, = A.tensors(sum(lens), (heads,), d, A.TYPES[dtype], "apart", 21)
    K, V = A.tensors(sum(keys), (heads, heads), d, A.TYPES[dtype], "fused", 22)
    _check(Q, K, V, lens, dtype, causal=causal, keys=keys)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,d,layout", [(18, 18, 128, "fused"), (36, 18, 64, "heads"), (20, 20, 72, "apart"), (40, 20, 32, "fused"), (24, 24, 8, "heads")])
def test_many_blocks(heads, kv, d, layout, causal, dtype):
    Q, K, V = A.tensors(sum(MANY), (heads, kv, kv), d, A.TYPES[dtype], layout, heads + d)
    _check(Q, K, V, MANY, dtype, causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_many_blocks_more_and_fewer_keys(causal, dtype):
    keys = [500, 70, 64, 0, 64, 512, 300, 65, 1000]
    Q, = A.tensors(sum(MANY), (20,), 64, A.TYPES[dtype], "apart", 3)
    K, V = A.tensors(sum(keys), (20, 20), 64, A.TYPES[dtype], "fused", 4)
    K[500:570], V[500:570] = math.nan, math.inf            # the keys of one sequence, whose only query is not looked at
    at = binding.Attention(heads=20, kv_heads=20, d=64, dtype=dtype, rows=sum(MANY), k_rows=sum(keys), seqs=len(MANY), causal=causal, device=G.DEV)
    O, lse = _run(at, Q, K, V, A.offsets(MANY), _where(keys))
    wO, bO, wl, bl = A.forward(Q, K, V, [p for i, p in enumerate(_parts(MANY, keys)) if i != 1], 64 ** -0.5, causal)
    assert A.near(O, wO, bO) and A.near(lse, wl, bl)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[1], [2, 1], [255], [256], [257], [31, 32, 33], [63, 64, 65, 66], [0, 0, 129, 0], [511, 513], [1] * 70 + [200], [1500, 3]])
def test_lengths(lens, causal):
    Q, K, V = A.tensors(sum(lens), (4, 2, 2), 128, torch.bfloat16, "heads", len(lens))
    _check(Q, K, V, lens, "bf16", causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,keys", [([300, 200, 1], [500, 100, 40]), ([300, 65], [0, 64]), ([260], [3]), ([100, 400], [1000, 463])])
def test_more_and_fewer_keys_than_queries(lens, keys, causal, dtype):
    """With fewer keys the first queries of a causal sequence see nothing: zero, and a sum of nothing."""
    Q, = A.tensors(sum(lens), (6,), 64, A.TYPES[dtype], "apart", 3)
    K, V = A.tensors(sum(keys), (2, 2), 64, A.TYPES[dtype], "fused", 4)
    O, lse = _check(Q, K, V, lens, dtype, causal=causal, keys=keys)
    for (q, n, _, m) in _parts(lens, keys):
        nothing = n if m == 0 else max(0, n - m) if causal else 0
        assert not O[q:q + nothing].any() and (lse[:, q:q + nothing] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d", [(8, 8, 128), (12, 4, 64), (8, 1, 128), (40, 1, 32), (9, 3, 80)])
@pytest.mark.parametrize("lens,keys,cache", [([1] * 5, [1, 33, 700, 4096, 257], 4096), ([1], [6000], 6100), ([3, 0, 1, 2, 8], [900, 5, 0, 1, 4], 1000), ([2] * 40, [50 * i % 1201 for i in range(40)], 1201)])
def test_tokens_over_a_cache(lens, keys, cache, heads, kv, d, dtype):
    t = A.TYPES[dtype]
    Q, = A.tensors(sum(lens), (heads,), d, t, "fused", 5)
    K, V = A.tensors(len(lens) * cache, (kv, kv), d, t, "apart", 6)
    begin = [i * cache for i in range(len(lens))]
    for b, m in zip(begin, keys):                          # what lies behind a sequence's keys is never looked at
        K[b + m:b + cache] = math.nan
        V[b + m:b + cache] = math.inf
    _check(Q, K, V, lens, dtype, keys=keys, begin=begin)
    order = list(reversed(range(len(lens))))               # sequences in other places of the cache
    _check(Q, K, V, lens, dtype, keys=[keys[i] for i in order], begin=[begin[i] for i in order])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d", [(2, 1, 64), (3, 3, 128)])
@pytest.mark.parametrize("seqs", [1, 3, 5, 63, 64, 65, 80])
def test_cut_by_the_sum_of_the_lengths(seqs, heads, kv, d, dtype):
    """Ragged caches whose sequences are cut into none to many parts each, empty places between them, up to three tokens a sequence; the workspace is as long as it has to be."""
    g = torch.Generator().manual_seed(seqs)
    keys = torch.randint(0, 700, (seqs,), generator=g).tolist()
    lens = torch.randint(0, 4, (seqs,), generator=g).tolist()
    keys[seqs // 2], lens[seqs // 2], keys[-1], lens[-1] = 9000, 2, 2500, 1
    cache = 9000
    Q, = A.tensors(sum(lens), (heads,), d, A.TYPES[dtype], "apart", seqs)
    K, V = A.tensors(cache * seqs if seqs < 10 else 1000 * seqs + 9000, (kv, kv), d, A.TYPES[dtype], "fused", seqs + 1)
    begin = [s * cache for s in range(seqs)] if seqs < 10 else [1000 * s + (8000 if s > seqs // 2 else 0) for s in range(seqs)]
    begin[-1] = min(begin[-1], K.shape[0] - 2500)
    _check(Q, K, V, lens, dtype, keys=keys, begin=begin)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["fused", "apart", "heads"])
def test_layouts_and_rows_of_no_sequence(layout, dtype):
    """Rows in front of the first sequence and behind the last one are left as they were; outputs in the middle of something wider."""
    t, lens, heads, kv, d = A.TYPES[dtype], [70, 300], 4, 2, 72
    rows = sum(lens) + 20
    Q, K, V = A.tensors(rows, (heads, kv, kv), d, t, layout, 9)
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=rows, seqs=2, device=G.DEV)
    wide = torch.full((rows, heads + 2, d), 7.0, dtype=t, device=G.DEV)
    O, lse = wide[:, 1:-1], torch.full((heads, rows), 7.0, device=G.DEV)
    off = A.offsets(lens) + 11
    at.fwd(Q, K, V, O, off, lse=lse)
    parts = [(11, 70, 11, 70), (81, 300, 81, 300)]
    wO, bO, wl, bl = A.forward(Q, K, V, parts, d ** -0.5, True)
    assert A.near(O, wO, bO) and A.near(lse, wl, bl)
    for r in (slice(0, 11), slice(381, rows)):
        assert (wide[r] == 7.0).all() and (lse[:, r] == 7.0).all()
    assert (wide[:, 0] == 7.0).all() and (wide[:, -1] == 7.0).all()
    q = Q.clone()                                          # over the queries
    at.fwd(q, K, V, q, off)
    assert torch.equal(q[11:381], O[11:381])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,heads", [(3, 2), (400, 2), (400, 44)])
def test_values_out_of_the_ordinary(n, heads, dtype):
    """Scores far apart, equal ones, all zeros; a NaN or an infinity in a query stays in its row, one in a key in the rows that see it, one of another
    sequence or behind the end nowhere."""
    t, kv, d, m = A.TYPES[dtype], 1, 64, 400
    lens, keys = [n, n, n], [m, m, m]
    Q, = A.tensors(3 * n, (heads,), d, t, "apart", 11)
    K, V = A.tensors(3 * m, (kv, kv), d, t, "apart", 12)
    Q[0] *= 60.0
    Q[1] = 0.0
    K[m:2 * m] = math.nan                                  # the sequence between
    V[m:2 * m] = math.inf
    O, _ = _check_some(Q, K, V, lens, keys, dtype, [0, 2])
    # the last key and its value: only the last query sees it
    K2, Q2 = K.clone(), Q.clone()
    K2[m - 1] = math.nan
    Q2[2 * n] = math.nan
    O2 = _run(binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=3 * n, k_rows=3 * m, seqs=3, device=G.DEV), Q2, K2, V, A.offsets(lens), _where(keys))[0]
    assert torch.equal(O2[:n - 1], O[:n - 1]) and torch.isnan(O2[n - 1]).all()
    assert torch.isnan(O2[2 * n]).all() and torch.equal(O2[2 * n + 1:], O[2 * n + 1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,heads,d", [(1, 32, 64), (3, 6, 128), (400, 2, 64), (400, 2, 128), (400, 134, 64), (400, 134, 128)])
def test_bits_of_a_row_are_its_own(n, heads, d, causal, dtype):
    """What lies in one query, scores that outgrow the maximum in use or infinities, changes no bit of the others, its neighbours in a wave among them."""
    t, m = A.TYPES[dtype], 700
    Q, = A.tensors(n, (heads,), d, t, "apart", 31)
    K, V = A.tensors(m, (1, 1), d, t, "apart", 32)
    K *= torch.linspace(0.2, 3.0, m, device=G.DEV)[:, None, None].to(t)    # later keys have the higher scores
    at = binding.Attention(heads=heads, kv_heads=1, d=d, dtype=dtype, rows=n, k_rows=m, seqs=1, causal=causal, device=G.DEV)
    off, where = A.offsets([n]), _where([m])
    O, lse = _run(at, Q, K, V, off, where)
    for factor in (30.0, -30.0, 0.0, math.inf, -math.inf):
        for row, head in ((0, 0), (n // 2, heads - 1), (n - 1, heads // 2)):
            Q2 = Q.clone()
            Q2[row, head] = Q2[row, head] * factor
            O2, lse2 = _run(at, Q2, K, V, off, where)
            O2[row, head], lse2[head, row] = O[row, head], lse[head, row]
            assert torch.equal(O, O2) and torch.equal(lse, lse2), (factor, row, head)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,d", [(2, 64), (2, 128), (134, 64), (134, 128)])
def test_reach_of_a_value_that_is_no_number(heads, d, dtype):
    """A NaN in V: in all rows that see it, in no row that is further from it than the header says, where the bits are those without it."""
    reach, n, m, t = _said(r"hides it from by up to (\d+) keys"), 400, 401, A.TYPES[dtype]
    Q, = A.tensors(n, (heads,), d, t, "apart", 41)
    K, V = A.tensors(m, (1, 1), d, t, "apart", 42)
    at = binding.Attention(heads=heads, kv_heads=1, d=d, dtype=dtype, rows=n, k_rows=m, seqs=1, device=G.DEV)
    O, lse = _run(at, Q, K, V, A.offsets([n]), _where([m]))
    furthest = 0
    for key in (0, 63, 64, 95, 127, 191, 255, 256, 300, 383, 400):
        for bad in (math.nan, math.inf):
            V2 = V.clone()
            V2[key] = bad
            O2, lse2 = _run(at, Q, K, V2, A.offsets([n]), _where([m]))
            hidden_by = key - (torch.arange(n, device=G.DEV) + m - n)          # keys between the last one that a row sees and this one
            assert not torch.isfinite(O2[hidden_by <= 0]).any() and torch.equal(lse, lse2)
            changed = ~(O2 == O).flatten(1).all(1)
            furthest = max(furthest, int(hidden_by[changed].max()))
    assert furthest <= reach
    if heads > 100 and dtype == "bf16":
        assert furthest == reach                           # tiles of 64 keys: the header says no more than there is


def _said(pattern):
    """A number that the header says."""
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "moehot.h")
    return int(re.search(pattern, " ".join(line.strip(" *") for line in open(header).read().splitlines())).group(1))


def _where(keys):
    ends = A.offsets(keys)
    return ends[:-1].contiguous(), ends[1:].contiguous()


def _check_some(Q, K, V, lens, keys, dtype, which):
    heads, kv, d = Q.shape[1], K.shape[1], Q.shape[2]
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype=dtype, rows=Q.shape[0], k_rows=K.shape[0], seqs=len(lens), device=G.DEV)
    O, lse = _run(at, Q, K, V, A.offsets(lens), _where(keys))
    parts = [_parts(lens, keys)[i] for i in which]
    wO, bO, wl, bl = A.forward(Q, K, V, parts, d ** -0.5, True)
    assert A.near(O, wO, bO) and A.near(lse, wl, bl)
    return O, lse


@pytest.mark.parametrize("heads", [4, 64])
def test_offsets_that_are_wrong(heads):
    """Held inside the tensors, whatever they are: sequences that are right stay right, nothing outside is written."""
    t, d, rows = torch.bfloat16, 64, 600
    Q, K, V = A.tensors(rows, (heads, heads, heads), d, t, "apart", 13)
    at = binding.Attention(heads=heads, kv_heads=heads, d=d, dtype="bf16", rows=rows, seqs=4, device=G.DEV)
    guard = torch.full((rows + 40, heads, d), 7.0, dtype=t, device=G.DEV)
    O = guard[20:20 + rows]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=G.DEV)  # noqa: E731
    for off, right in (([0, 100, 2 ** 31 - 1, 5000, 2 ** 31 - 1], [(0, 100, 0, 100), (100, 500, 100, 500)]), ([-2 ** 31, 100, 50, -7, 70], [(0, 100, 0, 100)]), ([900] * 5, [])):
        at.fwd(Q, K, V, O, i32(off))
        torch.cuda.synchronize()
        wO, bO, _, _ = A.forward(Q, K, V, right, d ** -0.5, True)
        assert A.near(O, wO, bO)
        assert (guard[:20] == 7.0).all() and (guard[20 + rows:] == 7.0).all()


@pytest.mark.parametrize("offsets,begin,end", [([0, 8, 0, 8, 0, 8], [0] * 5, [6000] * 5), ([0, 1, 2, 3, 4, 8], [0, 5000, 4000, -7, 2 ** 30], [6000, 100, 9000, 6000, 2 ** 31 - 1]),
                                               ([8, 6, 4, 2, 0, 0], [0] * 5, [6000] * 5)])
def test_wrong_offsets_of_cut_sequences(offsets, begin, end):
    """Sequences that overlap or fall: what they leave in O is theirs to say, nothing behind the workspace or outside the tensors changes, and no row of no sequence."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=G.DEV)  # noqa: E731
    Q, = A.tensors(8, (4,), 128, torch.bfloat16, "apart", 1)
    K, V = A.tensors(6000, (2, 2), 128, torch.bfloat16, "apart", 2)
    at = binding.Attention(heads=4, kv_heads=2, d=128, dtype="bf16", rows=8, k_rows=6000, seqs=5, device=G.DEV, alloc_workspace=False)
    room = torch.full((at.workspace_bytes + 65536,), 0x5a, dtype=torch.uint8, device=G.DEV)
    at.ws = room[:at.workspace_bytes]
    O = torch.full((24, 4, 128), 7.0, dtype=torch.bfloat16, device=G.DEV)
    at.fwd(Q, K, V, O[8:16], i32(offsets), k_begin=i32(begin), k_end=i32(end))
    assert bool((room[at.workspace_bytes:] == 0x5a).all()) and bool((O[:8] == 7.0).all()) and bool((O[16:] == 7.0).all())


@pytest.mark.parametrize("lens,heads", [([700, 33, 0, 600], 8), ([700, 33, 0, 600], 32), ([1] * 8, 8)])
def test_captured(lens, heads):
    """A graph replayed on new inputs and new lengths among eager calls: each replay what the eager call gives."""
    kv, d, rows = heads // 4, 128, sum(lens)
    keys = [n + 500 for n in lens]
    Q, = A.tensors(rows, (heads,), d, torch.bfloat16, "apart", 1)
    K, V = A.tensors(sum(keys), (kv, kv), d, torch.bfloat16, "apart", 2)
    at = binding.Attention(heads=heads, kv_heads=kv, d=d, dtype="bf16", rows=rows, k_rows=sum(keys), seqs=len(lens), device=G.DEV)
    off, (b, e) = A.offsets(lens), _where(keys)
    O, lse, O2, lse2 = torch.empty_like(Q), torch.empty(heads, rows, device=G.DEV), torch.empty_like(Q), torch.empty(heads, rows, device=G.DEV)
    at.fwd(Q, K, V, O, off, k_begin=b, k_end=e, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at.fwd(Q, K, V, O, off, k_begin=b, k_end=e, lse=lse)
    for k in range(4):
        Q.copy_(A.tensors(rows, (heads,), d, torch.bfloat16, "apart", 10 + k)[0])
        e.copy_(b + torch.tensor([max(1, m - 97 * k) for m in keys], dtype=torch.int32, device=G.DEV))
        graph.replay()
        at.fwd(Q, K, V, O2, off, k_begin=b, k_end=e, lse=lse2)
        torch.cuda.synchronize()
        assert torch.equal(O, O2) and torch.equal(lse, lse2), k


def test_two_streams():
    """Two objects, a stream each, at the same time."""
    heads, d, lens = 4, 64, [1] * 30
    keys = [3000] * 30
    Q, = A.tensors(30, (heads,), d, torch.bfloat16, "apart", 1)
    K, V = A.tensors(90000, (2, 2), d, torch.bfloat16, "apart", 2)
    make = lambda: binding.Attention(heads=heads, kv_heads=2, d=d, dtype="bf16", rows=30, k_rows=90000, seqs=30, device=G.DEV)  # noqa: E731
    off, where = A.offsets(lens), _where(keys)
    want = _run(make(), Q, K, V, off, where)[0]
    streams, ats = [torch.cuda.Stream() for _ in range(2)], [make() for _ in range(2)]
    outs = [torch.empty_like(Q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, at, o in zip(streams, ats, outs):
            with torch.cuda.stream(st):
                at.fwd(Q, K, V, o, off, k_begin=where[0], k_end=where[1])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("n,heads", [(2, 2), (300, 2), (300, 160)])
def test_keys_past_32_bits(n, heads):
    """A cache whose rows lie 4 MB apart: the last of them more than 2^32 bytes in."""
    d, m, row = 64, 2500, 2 ** 21 - 8
    whole = torch.empty(m * row, dtype=torch.bfloat16, device=G.DEV)
    K, V = (whole.as_strided((m, 1, d), (row, d, 1), o) for o in (0, 1024))
    for x, y in zip((K, V), A.tensors(m, (1, 1), d, torch.bfloat16, "apart", 3)):
        x.copy_(y)
    Q, = A.tensors(n, (heads,), d, torch.bfloat16, "apart", 4)
    _check(Q, K, V, [n], "bf16", keys=[m], begin=[0])


def test_long_sequence():
    """16384 keys for the last 600 queries, and one query for all of them."""
    Q, = A.tensors(600, (88,), 128, torch.bfloat16, "apart", 3)
    K, V = A.tensors(16384, (2, 2), 128, torch.bfloat16, "apart", 4)
    _check(Q, K, V, [600], "bf16", keys=[16384])
    _check(Q[:, :4], K, V, [600], "bf16", keys=[16384])
    _check(Q[:1], K, V, [1], "bf16", keys=[16384])


def test_nothing_to_do():
    at = binding.Attention(heads=2, kv_heads=1, d=64, dtype="bf16", rows=0, k_rows=16, seqs=3, device=G.DEV)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    K = torch.zeros(16, 1, 64, dtype=torch.bfloat16, device=G.DEV)
    z = torch.zeros(4, dtype=torch.int32, device=G.DEV)
    at.fwd(none, K, K, none, z, k_begin=z[:3], k_end=z[:3])
    at.fwd(none, K, K, none, z[:1], k_begin=z[:0], k_end=z[:0])


def test_refusals_of_the_binding():
    at = binding.Attention(heads=2, kv_heads=1, d=64, dtype="bf16", rows=8, seqs=2, device=G.DEV)
    Q, K = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device=G.DEV), torch.zeros(8, 1, 64, dtype=torch.bfloat16, device=G.DEV)
    off = torch.zeros(3, dtype=torch.int32, device=G.DEV)
    at.fwd(Q, K, K, Q.clone(), off)
    bad = [lambda: at.fwd(Q.float(), K, K, Q.clone(), off), lambda: at.fwd(Q[:, :1], K, K, Q.clone(), off), lambda: at.fwd(Q[:4], K, K, Q.clone(), off),
           lambda: at.fwd(Q, K, K, Q.clone().transpose(1, 2).contiguous().transpose(1, 2), off), lambda: at.fwd(Q, K, K, Q.clone(), off.long()),
           lambda: at.fwd(Q.cpu(), K, K, Q.clone(), off), lambda: at.fwd(Q, K, K, Q.clone(), off, k_begin=off[:2]),
           lambda: at.fwd(Q, K, K, Q.clone(), torch.zeros(4, dtype=torch.int32, device=G.DEV)), lambda: at.fwd(Q, K, K, Q.clone(), off, lse=torch.empty(2, 4, device=G.DEV)),
           lambda: at.fwd(Q, K[:4], K[:4], Q.clone(), off)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    odd = torch.zeros(8 * 2 * 64 + 1, dtype=torch.bfloat16, device=G.DEV)[1:].view(8, 2, 64)
    for call in (lambda: at.fwd(odd, K, K, Q.clone(), off), lambda: at.fwd(Q, K, K, Q[:1].expand(8, 2, 64), off), lambda: at.fwd(Q, K[:1].expand(8, 1, 64), K, Q.clone(), off)):
        with pytest.raises(binding.MoeError):
            call()
