"""The other half of a pre-norm block, attention, as cases that can be timed and checked: the rotation of queries and keys (with the norm of each
head in the same pass, and the place of a token's keys and values in a cache) and causal attention over packed sequences, both with their gradients.

A case is a dict of plain values; `op` says which operator one pass runs:

  rotary      rows x (heads + kv_heads) x d queries and keys of `dtype`, as a projection of the stream leaves them beside each other (`fused`) or
              in tensors of their own; `norm`: each head is divided by its root mean square first; the first `rot` columns of a head are rotated, in
              pairs of neighbours (`interleaved`) or of halves; `place`: the keys and the values go to rows of a cache, a padded row nowhere;
              `last`: positions run up to it; `long`: frequencies scaled for a long context, with an amplitude
  rotary_bwd  its gradient
  attend      softmax(scale Q K^T) V; `lens` and `keys` are the lengths of the sequences' queries and keys, end to end in their tensors, or
              (`cache` > 0) each sequence's keys in `cache` rows of its own; causal, the last query sees the last key; `layout`: where a
              token's heads lie
  attend_bwd  its gradient
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS, BASE = 1e-6, 10000.0
# for `long`: a context of TRAINED positions stretched by FACTOR, slow frequencies divided by it, fast ones left, those between by parts
TRAINED, FACTOR, FAST, SLOW = 4096, 8.0, 32.0, 1.0
AMPLITUDE = 0.1 * math.log(FACTOR) + 1.0


def listed():
    return [
        # one token of each of 16 sequences that are being answered, one place in the batch empty: norm, rotation, the way into the cache
        _rotary("rotary_token", rows=16, heads=32, kv=8, d=128, rot=128, dtype="bf16", norm=True, place=True, last=30000),
        # a ragged prompt of a model that rotates half of a narrow head, neighbours together, and has no norm there
        _rotary("rotary_ragged", rows=7999, heads=12, kv=4, d=80, rot=40, dtype="bf16", interleaved=True, last=7998),
        # a training step at the largest configuration's tokens and width, long context
        _rotary("rotary_wide", rows=32768, heads=32, kv=8, d=128, rot=128, dtype="bf16", norm=True, long=True, last=32767),
        # the tiny fp32 configuration's tokens and width, and the largest again, on the way back
        _rotary("rotary_bwd_tiny_f32", op="rotary_bwd", rows=512, heads=2, kv=2, d=32, rot=32, dtype="f32", norm=True, last=511),
        _rotary("rotary_bwd_wide", op="rotary_bwd", rows=32768, heads=32, kv=8, d=128, rot=128, dtype="bf16", norm=True, long=True, last=32767),
        # the tiny fp32 configuration's tokens and width in four sequences
        _attend("attend_tiny_f32", lens=[128] * 4, heads=2, kv=2, d=32, dtype="f32"),
        # a token of each of 16 sequences over what they have in the cache, the training steps' heads
        _attend("attend_token", lens=[1] * 16, keys=[1, 17, 300, 1024, 2047, 4096, 5000, 8191, 8192, 9000, 12000, 12345, 15000, 16000, 16384, 16383],
                cache=16384, heads=32, kv=8, d=128, dtype="bf16", stats=False),
        # documents of many lengths packed into one step of the mid-size GELU configurations
        _attend("attend_packed", lens=[4096, 1, 1777, 640, 2048, 0, 333, 64, 4000, 1500, 1925], heads=16, kv=4, d=128, dtype="bf16", layout="fused"),
        # one long sequence: all tokens of a mid-size configuration's step, the largest configuration's heads
        _attend("attend_long", lens=[16384], heads=32, kv=8, d=128, dtype="bf16", layout="fused"),
        # the way back: ragged in fp32; a step of the mid-size configuration with narrow heads; the largest configuration's in sequences of a quarter
        _attend("attend_bwd_ragged_f32", op="attend_bwd", lens=[700, 1, 0, 901, 257, 144], heads=6, kv=2, d=64, dtype="f32"),
        _attend("attend_bwd_packed", op="attend_bwd", lens=[2048, 1021, 3, 4096, 1500, 2500, 1120, 4096], heads=32, kv=32, d=64, dtype="bf16", layout="fused"),
        _attend("attend_bwd_wide", op="attend_bwd", lens=[8192] * 4, heads=32, kv=8, d=128, dtype="bf16", layout="fused"),
    ]


def _rotary(name=None, *, op="rotary", rows, heads, kv, d, rot, dtype, norm=False, interleaved=False, long=False, place=False, last, fused=True):
    c = dict(op=op, rows=rows, heads=heads, kv=kv, d=d, rot=rot, dtype=dtype, norm=norm, interleaved=interleaved, long=long, last=last, fused=fused)
    if op == "rotary":
        c["place"] = place
    if name is not None:
        c["name"] = name
    return c


def _attend(name=None, *, op="attend", lens, keys=None, cache=0, heads, kv, d, dtype, layout="apart", stats=True):
    c = dict(op=op, lens=" ".join(map(str, lens)), keys=" ".join(map(str, lens if keys is None else keys)), cache=cache, heads=heads, kv=kv, d=d, dtype=dtype, layout=layout)
    if op == "attend":
        c["stats"] = stats
    if name is not None:
        c["name"] = name
    return c


def _numbers(text):
    return [int(n) for n in text.split()]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case: sizes over the whole range of its operator."""
    op = rng.choice(["rotary", "rotary_bwd", "attend", "attend", "attend_bwd", "attend_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 8 * rng.randint(1, 16)])
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    heads = min(heads, 32 // kv * kv)
    if op.startswith("rotary"):
        rows = max(1, int(min(_log(rng, 1, 65536), 32768 * 40 * 64 // ((heads + kv) * d))))
        place = {"place": rng.random() < 0.4} if op == "rotary" else {}
        return _rotary(op=op, rows=rows, heads=heads, kv=kv, d=d, rot=rng.choice([d, d, d // 8 * 4, 2 * rng.randint(1, d // 2)]), dtype=dtype, norm=rng.random() < 0.5,
                       interleaved=rng.random() < 0.4, long=rng.random() < 0.4, last=int(_log(rng, max(rows, 2), 1000000)), fused=rng.random() < 0.7, **place)
    most = 4096 if dtype == "f32" else 8192 if op == "attend_bwd" else 16384    # of one sequence
    if op == "attend" and rng.random() < 0.4:               # answering: one token each, or a few, over a cache
        n = int(_log(rng, 1, 65))
        longest = int(_log(rng, 16, most + 1))
        keys = [max(8, int(longest * rng.random())) for _ in range(n)]
        lens = [1] * n if rng.random() < 0.7 else [1] + [rng.randint(0, 8) for _ in range(n - 1)]
        return _attend(lens=lens, keys=keys, cache=max(keys) + rng.choice([0, 1, 100]), heads=heads, kv=kv, d=d, dtype=dtype, stats=rng.random() < 0.3)
    total = int(_log(rng, 16, 16385 if dtype == "bf16" else 4097))
    lens = []
    while sum(lens) < total and len(lens) < 48:
        lens.append(min(total - sum(lens), most, int(_log(rng, 1, total + 1))))
    return _attend(op=op, lens=lens, heads=heads, kv=kv, d=d, dtype=dtype, layout=rng.choice(["fused", "apart", "heads"]))


def _heads_of(layout, rows, counts, d, t):
    """Tensors [rows, n, d] for each n of counts: beside each other in one, each of its own, or each with a head's rows together."""
    if layout == "fused":
        return list(torch.zeros(rows, sum(counts), d, dtype=t, device=DEV).split(counts, 1))
    if layout == "heads":
        return [torch.zeros(n, rows, d, dtype=t, device=DEV).transpose(0, 1) for n in counts]
    return [torch.zeros(rows, n, d, dtype=t, device=DEV) for n in counts]


def _frequencies(case):
    """Radians a position, in 64 bits."""
    r = case["rot"]
    f = BASE ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    if case["long"]:
        turns = TRAINED * f / (2 * math.pi)
        keep = ((turns - SLOW) / (FAST - SLOW)).clamp(0.0, 1.0)
        f = f * keep + f / FACTOR * (1.0 - keep)
    return f


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    s = dict(case)
    t, heads, kv, d = TYPES[case["dtype"]], case["heads"], case["kv"], case["d"]
    new = lambda rows, *counts: _heads_of(case.get("layout", "fused" if case.get("fused") else "apart"), rows, counts, d, t)  # noqa: E731
    if case["op"].startswith("rotary"):
        rows = case["rows"]
        s["Q"], s["K"], s["V"] = new(rows, heads, kv, kv)
        for x in (s["Q"], s["K"], s["V"]):                  # columns of different size, none centred
            x.copy_(randn(*x.shape) * torch.exp(0.5 * randn(x.shape[1], d)) + 0.3 * randn(x.shape[1], d))
        s["gq"], s["gk"] = (1.0 + 0.2 * randn(d), 1.0 + 0.2 * randn(d)) if case["norm"] else (None, None)
        s["frequencies"] = _frequencies(case)
        s["amplitude"] = AMPLITUDE if case["long"] else 1.0
        # sequences end to end, or a token each of sequences of any length
        s["positions"] = torch.randint(0, case["last"] + 1, (rows,), generator=g, device=DEV, dtype=torch.int32) if case.get("place") else \
            torch.arange(case["last"] - rows + 1, case["last"] + 1, device=DEV).clamp(min=0).to(torch.int32)
        if case["op"] == "rotary":
            s["Qo"], = _heads_of("apart", rows, [heads], d, t)
            s["slots"], s["Vo"] = None, None
            if case["place"]:
                s["Ko"], s["Vo"] = _heads_of("apart", 2 * rows, [kv, kv], d, t)
                s["slots"] = torch.randperm(2 * rows, generator=g, device=DEV)[:rows].to(torch.int32)
                s["slots"][rows // 2] = -1
            else:
                s["Ko"], = _heads_of("apart", rows, [kv], d, t)
        else:
            s["dQo"], s["dKo"] = _heads_of("apart", rows, [heads, kv], d, t)
            s["dQo"].copy_(0.02 * randn(rows, heads, d))
            s["dKo"].copy_(0.02 * randn(rows, kv, d))
            s["dQ"], s["dK"], _ = new(rows, heads, kv, kv)
            s["dgq"], s["dgk"] = (torch.empty(d, device=DEV), torch.empty(d, device=DEV)) if case["norm"] else (None, None)
        return s
    lens, keys, cache = _numbers(case["lens"]), _numbers(case["keys"]), case["cache"]
    rows, krows = sum(lens), len(keys) * cache if cache else sum(keys)
    if cache or case["layout"] != "fused":
        s["Q"], = new(rows, heads)
        s["K"], s["V"] = new(krows, kv, kv)
    else:
        s["Q"], s["K"], s["V"] = new(rows, heads, kv, kv)
    # what a rotation with a norm leaves: heads of even length, some columns larger, a direction that queries and keys share
    size, shared = torch.exp(0.3 * randn(d)), 0.4 * randn(d)
    s["Q"].copy_(randn(rows, heads, d).mul_(size).add_(shared))
    s["K"].copy_(randn(krows, kv, d).mul_(size).add_(shared))
    s["V"].copy_(randn(krows, kv, d))
    int32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s["offsets"] = int32([sum(lens[:i]) for i in range(len(lens) + 1)])
    begin = [i * cache if cache else sum(keys[:i]) for i in range(len(keys))]
    s["k_begin"], s["k_end"] = (int32(begin), int32([b + n for b, n in zip(begin, keys)])) if cache or keys != lens else (None, None)
    s["parts"] = [(sum(lens[:i]), n, begin[i], keys[i]) for i, n in enumerate(lens)]
    s["scale"] = 1.0 / math.sqrt(d)
    s["O"], = _heads_of("apart", rows, [heads], d, t)
    s["lse"] = torch.empty(heads, rows, device=DEV) if case.get("stats", True) else None
    if case["op"] == "attend_bwd":
        O, lse = _plain_attend(s)
        s["O"].copy_(O)
        s["lse"].copy_(lse)
        s["dO"], = _heads_of("apart", rows, [heads], d, t)
        s["dO"].copy_(0.02 * randn(rows, heads, d))
        s["dQ"], s["dK"], s["dV"] = new(rows, heads, kv, kv)
    return s


_kept = {}      # what a program makes once and keeps: the rotation and the attention of a model's heads


def _own_rotary(s):
    from paper_2411_10003_amd import binding
    key = ("rotary", s["heads"], s["kv"], s["d"], s["rot"], s["dtype"], s["norm"], s["interleaved"], s["amplitude"])
    if key not in _kept:
        _kept[key] = binding.Rotary(heads=s["heads"], kv_heads=s["kv"], d=s["d"], rot=s["rot"], dtype=s["dtype"], norm=s["norm"], interleaved=s["interleaved"],
                                    eps=EPS, amplitude=s["amplitude"], device=DEV)
    return _kept[key]


def _own_attention(s):
    from paper_2411_10003_amd import binding
    rows, krows, seqs = s["Q"].shape[0], s["K"].shape[0], len(s["parts"])
    key = ("attend", s["heads"], s["kv"], s["d"], s["dtype"], rows, krows, seqs)
    if key not in _kept:
        _kept[key] = binding.Attention(heads=s["heads"], kv_heads=s["kv"], d=s["d"], dtype=s["dtype"], causal=True, rows=rows, k_rows=krows, seqs=seqs, device=DEV)
    return _kept[key]


def run(s):
    if s["op"] == "rotary":
        if own:
            _own_rotary(s).fwd(s["Q"], s["K"], s["positions"], s["frequencies"], s["Qo"], s["Ko"], gamma_q=s["gq"], gamma_k=s["gk"],
                               V=s["V"] if s["place"] else None, Vo=s["Vo"], slots=s["slots"])
            return [s["Qo"], s["Ko"], s["Vo"]]
        return _plain_rotary(s)
    if s["op"] == "rotary_bwd":
        if own:
            more = dict(Q=s["Q"], K=s["K"], gamma_q=s["gq"], gamma_k=s["gk"], dgamma_q=s["dgq"], dgamma_k=s["dgk"]) if s["norm"] else {}
            _own_rotary(s).bwd(s["dQo"], s["dKo"], s["positions"], s["frequencies"], s["dQ"], s["dK"], **more)
            return [s["dQ"], s["dK"], s["dgq"], s["dgk"]]
        return _plain_rotary_bwd(s)
    if s["op"] == "attend":
        if own:
            _own_attention(s).fwd(s["Q"], s["K"], s["V"], s["O"], s["offsets"], k_begin=s["k_begin"], k_end=s["k_end"], lse=s["lse"])
            return [s["O"], s["lse"]]
        O, lse = _plain_attend(s)
        return [O, lse if s["stats"] else None]
    if own:
        _own_attention(s).bwd(s["dO"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["offsets"], s["dQ"], s["dK"], s["dV"], k_begin=s["k_begin"], k_end=s["k_end"])
        return [s["dQ"], s["dK"], s["dV"]]
    return _plain_attend_bwd(s)


def _turn(x, s, sign):
    """The rotation of heads x [rows, n, d] by the positions, or back, in 32 bits; the angles in 64."""
    a = s["positions"].double()[:, None, None] * s["frequencies"]
    c, w = (torch.cos(a) * s["amplitude"]).float(), (torch.sin(a) * (sign * s["amplitude"])).float()
    r, y = s["rot"], x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    y[..., first] = x[..., first] * c - x[..., second] * w
    y[..., second] = x[..., second] * c + x[..., first] * w
    return y


def _plain_rotary(s):
    out = []
    for x, gamma in ((s["Q"], s["gq"]), (s["K"], s["gk"])):
        x = x.float()
        if s["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma
        out.append(_turn(x, s, 1.0).to(s["Q"].dtype))
    if not s["place"]:
        return out + [None]
    kept = s["slots"] >= 0
    to = s["slots"][kept].long()
    s["Ko"][to], s["Vo"][to] = out[1][kept], s["V"][kept]
    return [out[0], s["Ko"], s["Vo"]]


def _plain_rotary_bwd(s):
    grads, dgammas = [], []
    for dy, x, gamma in ((s["dQo"], s["Q"], s["gq"]), (s["dKo"], s["K"], s["gk"])):
        dy = _turn(dy.float(), s, -1.0)
        if s["norm"]:
            x = x.float()
            rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            xh = x * rstd
            dgammas.append((dy * xh).sum((0, 1)))
            dy = dy * gamma
            dy = rstd * (dy - xh * (dy * xh).mean(-1, keepdim=True))
        grads.append(dy.to(s["Q"].dtype))
    return grads + (dgammas if s["norm"] else [None, None])


def _scores(s, part):
    """Masked, scaled scores [kv, group * n, m] of one sequence in 32 bits, with its keys and values [kv, m, d]."""
    r0, n, k0, m = part
    kv, d = s["kv"], s["d"]
    q = s["Q"][r0:r0 + n].float().reshape(n, kv, -1, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
    k, v = (s[x][k0:k0 + m].float().transpose(0, 1).contiguous() for x in "KV")
    p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(s["scale"]).view(kv, -1, n, m)
    hidden = torch.arange(m, device=DEV) > torch.arange(n, device=DEV)[:, None] + (m - n)
    return q, k, v, p.masked_fill_(hidden, -math.inf).view(kv, -1, m)


def _rows_of(x, s, n):
    return x.view(s["kv"], -1, n, s["d"]).permute(2, 0, 1, 3).reshape(n, s["heads"], s["d"])


def _plain_attend(s):
    O, lse = torch.zeros_like(s["O"]), torch.empty(s["heads"], s["Q"].shape[0], device=DEV)
    for part in s["parts"]:
        r0, n, _, m = part
        if not n or not m:
            lse[:, r0:r0 + n] = -math.inf
            continue
        _, _, v, p = _scores(s, part)
        most = p.max(-1, keepdim=True).values.clamp(min=-1e30)
        p = p.sub_(most).exp_()
        total = p.sum(-1, keepdim=True)
        O[r0:r0 + n] = _rows_of(torch.matmul(p, v) / total.clamp(min=1e-30), s, n).to(O.dtype)
        lse[:, r0:r0 + n] = (most + torch.log(total)).view(s["heads"], n)
    return O, lse


def _plain_attend_bwd(s):
    dQ, dK, dV = (torch.zeros_like(s[x]) for x in "QKV")
    for part in s["parts"]:
        r0, n, k0, m = part
        if not n or not m:
            continue
        q, k, v, p = _scores(s, part)
        lse = s["lse"][:, r0:r0 + n].reshape(s["kv"], -1, 1)
        p = p.sub_(lse.clamp(min=-1e30)).exp_()
        do, o = (s[x][r0:r0 + n].float().reshape(n, s["kv"], -1, s["d"]).permute(1, 2, 0, 3).reshape(s["kv"], -1, s["d"]) for x in ("dO", "O"))
        dV[k0:k0 + m] = torch.matmul(p.transpose(1, 2).contiguous(), do).transpose(0, 1).to(dV.dtype)
        dp = torch.matmul(do, v.transpose(1, 2).contiguous())
        ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
        dQ[r0:r0 + n] = _rows_of(torch.matmul(ds, k), s, n).to(dQ.dtype)
        dK[k0:k0 + m] = torch.matmul(ds.transpose(1, 2).contiguous(), q).transpose(0, 1).to(dK.dtype)
    return [dQ, dK, dV]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    heads, kv, d = case["heads"], case["kv"], case["d"]
    if case["op"].startswith("rotary"):
        rows, n = case["rows"], case["rows"] * (heads + kv) * d
        parameters = 4 * case["rot"] + 4 * rows + (8 * d if case["norm"] else 0)
        if case["op"] == "rotary":
            moved = 2 * n + (2 * rows * kv * d if case["place"] else 0)
            return {"bytes": moved * size + parameters + (4 * rows if case["place"] else 0), "flops": (7 if case["norm"] else 3) * n}
        return {"bytes": n * size * (3 if case["norm"] else 2) + parameters + (8 * d if case["norm"] else 0), "flops": (14 if case["norm"] else 3) * n}
    lens, keys = _numbers(case["lens"]), _numbers(case["keys"])
    # query i of n sees the first m - n + i + 1 of m keys
    pairs = sum(n * m - n * (n - 1) // 2 if m >= n else m * (m + 1) // 2 for n, m in zip(lens, keys))
    q, k = sum(lens) * heads * d * size, sum(keys) * kv * d * size
    if case["op"] == "attend":
        return {"bytes": 2 * q + 2 * k + (4 * heads * sum(lens) if case["stats"] else 0), "flops": 4 * d * heads * pairs}
    return {"bytes": 4 * q + 4 * k + 4 * heads * sum(lens), "flops": 10 * d * heads * pairs}


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    back = case["op"].endswith("bwd")
    if case["op"].startswith("rotary"):
        # neighbours or halves as complex numbers, turned by exp(i angle)
        turn = torch.polar(torch.full_like(s["frequencies"], s["amplitude"]).expand(case["rows"], -1), torch.outer(s["positions"].double(), s["frequencies"]))
        outs, leaves = [], []
        for x, gamma in ((s["Q"], s["gq"]), (s["K"], s["gk"])):
            x = x.double().requires_grad_(back)
            gamma = gamma.double().requires_grad_(back) if case["norm"] else None
            leaves.append((x, gamma))
            y = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * gamma if case["norm"] else x
            head, rest = y[..., :case["rot"]], y[..., case["rot"]:]
            pairs = head.unflatten(-1, (-1, 2) if case["interleaved"] else (2, -1))
            z = (torch.view_as_complex(pairs.contiguous()) if case["interleaved"] else torch.complex(pairs[..., 0, :], pairs[..., 1, :])) * turn[:, None]
            z = torch.view_as_real(z)
            outs.append(torch.cat(((z if case["interleaved"] else z.mT).flatten(-2), rest), -1))
        if back:
            torch.autograd.backward(outs, [s["dQo"].double(), s["dKo"].double()])
            return [x.grad for x, _ in leaves] + [gamma.grad if case["norm"] else None for _, gamma in leaves]
        if not case["place"]:
            return outs + [None]
        K, V = torch.zeros(s["Ko"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["Vo"].shape, dtype=torch.float64, device=DEV)
        for i, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                K[slot], V[slot] = outs[1][i], s["V"][i].double()
        return [outs[0], K, V]
    wide = {x: s[x].double() for x in ("Q", "K", "V", *(["dO"] if back else []))}
    O, lse = torch.zeros_like(wide["Q"]), torch.full((case["heads"], wide["Q"].shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    grads = {x: torch.zeros_like(wide[x]) for x in "QKV"}
    group = case["heads"] // case["kv"]
    for h in range(case["heads"]):
        for r0, n, k0, m in s["parts"]:
            for i0 in range(0, n, 4096):                    # some queries and all the keys that the last of them sees
                i1 = min(n, i0 + 4096)
                seen = min(m, max(0, m - n + i1))
                if not seen:
                    continue
                q = wide["Q"][r0 + i0:r0 + i1, h].clone().requires_grad_(back)
                k, v = (wide[x][k0:k0 + seen, h // group].clone().requires_grad_(back) for x in "KV")
                visible = torch.ones(i1 - i0, seen, dtype=torch.bool, device=DEV).tril(m - n + i0)
                rows = visible.any(1)
                a = torch.where(visible, q @ k.T / math.sqrt(case["d"]), -math.inf)
                e = torch.logsumexp(a, 1)
                o = torch.where(visible, torch.exp(a - torch.where(rows, e, 0.0)[:, None]), 0.0) @ v
                if back:
                    o.backward(wide["dO"][r0 + i0:r0 + i1, h])
                    grads["Q"][r0 + i0:r0 + i1, h] += q.grad
                    grads["K"][k0:k0 + seen, h // group] += k.grad
                    grads["V"][k0:k0 + seen, h // group] += v.grad
                else:
                    O[r0 + i0:r0 + i1, h], lse[h, r0 + i0:r0 + i1] = o, e
    if back:
        return [grads["Q"], grads["K"], grads["V"]]
    return [O, lse if case["stats"] else None]
