"""Cases of the operators at the two ends of a recurrent language model and between them: the embedding lookup with its
gradient, the gated delta rule, and the loss from labels and a teacher's top logits, with what each computes in plain torch
operations.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges,
`prepare(case, seed)` what a program holds before the call, `run(state)` one pass: in the plain form where `own` is
false, through the framework's entry points where it is true.  `work(case)` is the bytes and operations a pass cannot
do without, `exact(case, seed)` what a pass gives from the definition in 64 bits.

Kinds:
  embed    ard_embedding_fwd and, with "grad", ard_embedding_bwd: rows of a table by token, scaled, with dp > 1 over the columns
           that a row pattern keeps; the gradient of the whole table, or, with "tied", added to what the output layer's
           product left there
  delta    ard_delta_forward and, with "grad", ard_delta_backward: the gated delta rule over [T][B][heads], queries and keys
           normalised, gates from pre-activations, padded batches
  distill  ard_distill_loss: cross entropy with the labels and divergence from a teacher's top logits, with its gradient
"""
import functools
import math

import numpy as np
import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
CHUNK = 64                                   # time steps between two states that a backward pass starts from
EPS = 1e-6                                   # added to the squared lengths of queries and keys


# ---- cases --------------------------------------------------------------------------------------
def listed():
    return [
        # Serving: the next token of 64 sequences, the 8800-word dictionary into 1500 units.
        {"name": "embed_token", "kind": "embed", "dtype": "bf16", "rows": 64, "V": 8800, "N": 1500, "dp": 1, "pad": False, "tied": False,
         "grad": False},
        # The 20 x 35 positions of a training batch of the 1500-wide layers, half of the units kept.
        {"name": "embed_700x1500_kept", "kind": "embed", "dtype": "bf16", "rows": 700, "V": 8800, "N": 1500, "dp": 2, "pad": False, "tied": False,
         "grad": True},
        # A large batch over a large dictionary, some positions padded.
        {"name": "embed_16384x2048", "kind": "embed", "dtype": "bf16", "rows": 16384, "V": 32000, "N": 2048, "dp": 1, "pad": True, "tied": False,
         "grad": True},
        # Serving: the next token of 64 sequences, 8 heads of 128 x 128.
        {"name": "delta_token", "kind": "delta", "T": 1, "B": 64, "heads": 8, "Dk": 128, "Dv": 128, "ragged": False, "grad": False},
        # The recurrent layer's training batch, 35 steps of 64 sequences, 1024 units.
        {"name": "delta_35x64x8", "kind": "delta", "T": 35, "B": 64, "heads": 8, "Dk": 128, "Dv": 128, "ragged": False, "grad": True},
        # Odd sizes, sequences of different lengths.
        {"name": "delta_777x5x3_odd", "kind": "delta", "T": 777, "B": 5, "heads": 3, "Dk": 40, "Dv": 99, "ragged": True, "grad": True},
        # Reading one long document before an answer.
        {"name": "delta_16384x1x8", "kind": "delta", "T": 16384, "B": 1, "heads": 8, "Dk": 128, "Dv": 128, "ragged": False, "grad": False},
        # Training on long padded sequences.
        {"name": "delta_2048x8x8", "kind": "delta", "T": 2048, "B": 8, "heads": 8, "Dk": 128, "Dv": 128, "ragged": True, "grad": True},
        # The ten classes of the MNIST network, distilled from a larger one's three best.
        {"name": "distill_64x10_f32", "kind": "distill", "dtype": "f32", "rows": 64, "V": 10, "k": 3, "tau": 2.0, "hard": 0.5, "soft": 0.5},
        # The 20 x 35 positions of a training batch over the 8800-word dictionary.
        {"name": "distill_700x8800", "kind": "distill", "dtype": "bf16", "rows": 700, "V": 8800, "k": 16, "tau": 2.0, "hard": 0.3, "soft": 0.7},
        # A large dictionary whose size is odd, so that no two rows begin on the same boundary; labels alone.
        {"name": "distill_1023x100003", "kind": "distill", "dtype": "bf16", "rows": 1023, "V": 100003, "k": 0, "tau": 1.0, "hard": 1.0, "soft": 0.0},
        # A large batch over a large dictionary.
        {"name": "distill_8192x32000", "kind": "distill", "dtype": "bf16", "rows": 8192, "V": 32000, "k": 64, "tau": 1.0, "hard": 0.5, "soft": 0.5},
    ]


def _spread(rng, low, high):
    """A whole number of low..high, spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    kind = rng.choice(["embed", "delta", "distill"])
    if kind == "embed":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        N = _spread(rng, 8, 8192)
        size = 1 if dtype == "bf16" else 2
        rows = _spread(rng, 1, min(65536, 16384 * 2048 // (N * size)))
        return {"kind": kind, "dtype": dtype, "rows": rows, "V": _spread(rng, 2, min(200000, 32000 * 2048 // N)), "N": N,
                "dp": rng.choice([1, 1, 2, 5]) if N >= 64 else 1, "pad": rng.random() < 0.5, "tied": rng.random() < 0.3, "grad": rng.random() < 0.7}
    if kind == "delta":
        heads, Dk, Dv = _spread(rng, 1, 16), rng.choice([128, 64, _spread(rng, 8, 128)]), rng.choice([128, 64, _spread(rng, 8, 128)])
        B = _spread(rng, 1, 64)
        T = _spread(rng, 1, max(1, min(16384, 2048 * 8 * 8 // (B * heads))))
        return {"kind": kind, "T": T, "B": B, "heads": heads, "Dk": Dk, "Dv": Dv, "ragged": rng.random() < 0.5, "grad": rng.random() < 0.6}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = _spread(rng, 4, 200000)
    rows = _spread(rng, 1, min(65536, 8192 * 32000 // (V * (1 if dtype == "bf16" else 2))))
    k = rng.choice([0, 1, _spread(rng, 1, 128), _spread(rng, 1, 128)])
    hard = rng.choice([0.0, 0.5, 1.0]) if k else 1.0
    return {"kind": kind, "dtype": dtype, "rows": rows, "V": V, "k": min(k, V), "tau": rng.choice([1.0, 2.0, round(rng.uniform(0.5, 4.0), 3)]),
            "hard": hard, "soft": 1.0 if hard == 0.0 else 0.5 if k else 0.0}


def _kept(units, dp):
    """The kept units of a row pattern with period dp and offset 1 + dp // 2 (zero-based numbers)."""
    return range(dp // 2, units, dp)


def _bytes(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    if case["kind"] == "embed":
        es, rows, n, V = _bytes(case), case["rows"], len(_kept(case["N"], case["dp"])), case["V"]
        used = min(V, rows)
        moved, flops = 4 * rows + es * n * (used + rows), rows * n
        if case["grad"]:
            table = used * n * 8 if case["tied"] else V * case["N"] * 4
            moved, flops = moved + 4 * rows + es * rows * n + table, flops + 2 * rows * n
        return {"bytes": moved, "flops": flops}
    if case["kind"] == "delta":
        B, heads, Dk, Dv = case["B"], case["heads"], case["Dk"], case["Dv"]
        full = case["T"] * B * heads
        cells = int(_lens(case, 0).sum()) * heads           # the padding is written, never read
        moved = 2 * (cells * (2 * Dk + Dv + 2) + full * Dv) + 8 * B * heads * Dk * Dv
        flops = cells * 6 * Dk * Dv
        if case["grad"]:
            moved += 2 * (cells * (2 * Dk + 2 * Dv + 2) + full * (2 * Dk + Dv + 2)) + 8 * B * heads * Dk * Dv
            flops += cells * 14 * Dk * Dv
        return {"bytes": moved, "flops": flops}
    rows, V, k = case["rows"], case["V"], case["k"]
    return {"bytes": rows * (2 * V * _bytes(case) + 8 * k + 12), "flops": rows * V * (8 if case["tau"] == 1.0 else 12)}


# ---- inputs -------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, scale=1.0, shift=0.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(dtype)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _tokens(g, rows, V):
    """Tokens by falling frequency: the first ones come up often, most seldom or never."""
    return ((V + 1.0) ** _uniform(g, rows) - 1.0).to(torch.int32).clamp_(0, V - 1)


def _lens(case, seed):
    """Lengths of the sequences of a padded batch: the longest fills it."""
    if not case["ragged"]:
        return np.full(case["B"], case["T"], np.int32)
    lens = np.random.RandomState(case["T"] * 31 + case["B"]).randint(case["T"] // 4, case["T"] + 1, case["B"]).astype(np.int32)
    lens[0] = case["T"]
    return np.roll(lens, seed % case["B"])


@functools.lru_cache(None)
def _context():
    from paper_2203_05705_b200 import ard
    return ard.ard_create(0, 0)


def _pattern(units, dp):
    """The framework's handle for the kept units, as a layer's program keeps it."""
    from paper_2203_05705_b200 import ard
    pat = ard.ard_pattern_create(_context(), ard.ARD_ROW, units, units, 0)
    ard.ard_pattern_set(_context(), pat, dp, 1 + dp // 2)
    return pat


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    s = {"case": dict(case), "kind": kind}
    if kind == "embed":
        rows, V, N = case["rows"], case["V"], case["N"]
        s["td"] = F32 if case["dtype"] == "f32" else BF16
        s["n"], s["pat"] = len(_kept(N, case["dp"])), None
        if own and case["dp"] > 1:
            s["pat"] = _pattern(N, case["dp"])
        s["alpha"] = math.sqrt(N) * case["dp"]
        s["ids"] = _tokens(g, rows, V)
        if case["pad"]:
            s["ids"].masked_fill_(_uniform(g, rows) < 0.05, -1)
        s["table"] = _normal(g, V, N, scale=N ** -0.5, dtype=s["td"])
        s["y"] = torch.empty((rows, N), dtype=s["td"], device="cuda")
        if case["grad"]:
            s["dy"] = _normal(g, rows, N, scale=0.1, dtype=s["td"])
            s["left"] = _normal(g, V, N, scale=0.1) if case["tied"] else None      # the output layer's gradient
            s["dtable"] = torch.empty((V, N), device="cuda")
    elif kind == "delta":
        T, B, h, Dk, Dv = (case[x] for x in ("T", "B", "heads", "Dk", "Dv"))
        # blocks of one matrix, as one product over all of them leaves it
        s["ld"] = h * (2 * Dk + Dv)
        s["qkv"] = _normal(g, T * B, s["ld"], dtype=BF16)
        s["z"] = torch.cat([_normal(g, T * B, h, scale=1.5, shift=4.0), _normal(g, T * B, h)], 1).to(BF16)   # a long memory
        s["scale"] = Dk ** -0.5
        s["h0"] = _normal(g, B, h, Dk, Dv, scale=0.3)
        s["lens"] = torch.from_numpy(_lens(case, seed)).cuda() if case["ragged"] else None
        s["y"], s["hT"] = torch.empty((T * B, h * Dv), dtype=BF16, device="cuda"), torch.empty_like(s["h0"])
        s["S"] = None
        if case["grad"]:
            s["dy"], s["dhT"] = _normal(g, T * B, h * Dv, scale=0.1, dtype=BF16), _normal(g, B, h, Dk, Dv, scale=0.1)
            s["S"] = torch.empty((-(-T // CHUNK), B, h, Dk, Dv), device="cuda")
            s["dqkv"], s["dz"], s["dh0"] = torch.empty_like(s["qkv"]), torch.empty_like(s["z"]), torch.empty_like(s["h0"])
        if own:
            from paper_2203_05705_b200 import ard
            s["work"] = torch.empty(ard.ard_delta_work_bytes(T, B, h, Dk, Dv, case["grad"]), dtype=torch.uint8, device="cuda")
    else:
        rows, V, k = case["rows"], case["V"], case["k"]
        s["td"] = F32 if case["dtype"] == "f32" else BF16
        s["z"] = _normal(g, rows, V, scale=2.0, dtype=s["td"])
        s["labels"] = None
        if case["hard"]:
            s["labels"] = _tokens(g, rows, V).masked_fill_(_uniform(g, rows) < 0.05, -1)     # some positions are padded
            s["z"].scatter_add_(1, s["labels"].clamp_min(0)[:, None].long(), torch.full((rows, 1), 4.0, dtype=s["td"], device="cuda"))
        s["teacher_ids"], s["teacher"] = None, None
        if k:
            # the teacher's best, other tokens in every row, which the student finds likelier than most
            start = (_uniform(g, rows, 1) * V).long()
            stride = next(p for p in (7919, 104729, 1299709) if V % p)
            s["teacher_ids"] = ((start + torch.arange(k, device="cuda") * stride) % V).to(torch.int32)
            s["z"].scatter_add_(1, s["teacher_ids"].long(), torch.full((rows, k), 3.0, dtype=s["td"], device="cuda"))
            s["teacher"] = (_normal(g, rows, k, scale=1.5) + 6.0).sort(1, descending=True)[0].contiguous()
        s["weight"] = torch.full((rows,), 1.0 / rows, device="cuda")
        s["loss"], s["total"], s["dz"] = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(s["z"])
    return s


# ---- one pass -----------------------------------------------------------------------------------
def run(s):
    if s["kind"] == "embed":
        return _own_embed(s) if own else _plain_embed(s)
    if s["kind"] == "delta":
        return _own_delta(s) if own else _plain_delta(s)
    return _own_distill(s) if own else _plain_distill(s)


def _own_embed(s):
    from paper_2203_05705_b200 import ard
    c = s["case"]
    rows, V, N, dt = c["rows"], c["V"], c["N"], ard.ARD_F32 if c["dtype"] == "f32" else ard.ARD_BF16
    ard.ard_embedding_fwd(_context(), s["pat"], dt, rows, V, N, s["alpha"], s["ids"], s["table"], N, s["y"], N)
    out = {"y": s["y"][:, :s["n"]]}
    if c["grad"]:
        if c["tied"]:
            s["dtable"].copy_(s["left"])     # stands for the product that leaves its own gradient there
        ard.ard_embedding_bwd(_context(), s["pat"], dt, rows, V, N, s["alpha"], s["ids"], s["dy"], N, s["dtable"], N, c["tied"])
        out["dtable"] = s["dtable"]
    return out


def _plain_embed(s):
    c, n, td = s["case"], s["n"], s["td"]
    keep = slice(c["dp"] // 2, None, c["dp"])
    ids = s["ids"].long()
    there = (ids >= 0)[:, None]
    ids = ids.clamp_min(0)
    y = s["table"][:, keep][ids].float() * s["alpha"]
    out = {"y": torch.where(there, y, 0.0).to(td)}
    if c["grad"]:
        dtable = s["left"].clone() if c["tied"] else torch.zeros_like(s["dtable"])
        part = torch.zeros((c["V"], n), device="cuda")
        part.index_add_(0, ids, torch.where(there, s["dy"][:, :n].float(), 0.0))
        dtable[:, keep] += part * s["alpha"]
        out["dtable"] = dtable
    return out


def _own_delta(s):
    from paper_2203_05705_b200 import ard
    c = s["case"]
    T, B, h, Dk, Dv, ld, dt = c["T"], c["B"], c["heads"], c["Dk"], c["Dv"], s["ld"], ard.ARD_BF16
    at = lambda t, k: t.data_ptr() + 2 * k  # noqa: E731
    q, k, v = (at(s["qkv"], x) for x in (0, h * Dk, 2 * h * Dk))
    ard.ard_delta_forward(_context(), dt, T, B, h, Dk, Dv, s["scale"], EPS, q, ld, k, ld, v, ld, s["z"], at(s["z"], h), 2 * h, s["lens"], s["h0"],
                          s["y"], h * Dv, s["hT"], s["S"], s["work"], s["work"].numel())
    out = {"y": s["y"], "hT": s["hT"]}
    if c["grad"]:
        dq, dk, dv = (at(s["dqkv"], x) for x in (0, h * Dk, 2 * h * Dk))
        ard.ard_delta_backward(_context(), dt, T, B, h, Dk, Dv, s["scale"], EPS, q, ld, k, ld, v, ld, s["z"], at(s["z"], h), 2 * h, s["lens"],
                               s["S"], s["dy"], h * Dv, s["dhT"], dq, ld, dk, ld, dv, ld, s["dz"], at(s["dz"], h), 2 * h, s["dh0"],
                               s["work"], s["work"].numel())
        out.update(_delta_gradients(s, s["dqkv"], s["dz"], s["dh0"]))
    return out


def _delta_gradients(s, dqkv, dz, dh0):
    c = s["case"]
    a, b, h = c["heads"] * c["Dk"], 2 * c["heads"] * c["Dk"], c["heads"]
    return {"dq": dqkv[:, :a], "dk": dqkv[:, a:b], "dv": dqkv[:, b:], "dzf": dz[:, :h], "dzb": dz[:, h:], "dh0": dh0}


def _by_head(x, s, D):
    """[T*B][heads * D] as [B * heads][chunks][CHUNK][D] in fp32, zeros behind the last step."""
    T, B, h = (s["case"][k] for k in ("T", "B", "heads"))
    C = -(-T // CHUNK)
    x = x.reshape(T, B, h, D).float().permute(1, 2, 0, 3).reshape(B * h, T, D)
    return torch.nn.functional.pad(x, (0, 0, 0, C * CHUNK - T)).view(B * h, C, CHUNK, D)


def _by_row(x, s):
    """The way back, without what is behind the last step."""
    T, B, h = (s["case"][k] for k in ("T", "B", "heads"))
    return x.reshape(B, h, -1, x.shape[-1])[:, :, :T].permute(2, 0, 1, 3).reshape(T * B, -1)


def _plain_delta(s):
    """Chunk by chunk: within one, the steps' updates u solve a triangular system, and the state moves by products."""
    c, scale = s["case"], s["scale"]
    T, B, h, Dk, Dv = (c[x] for x in ("T", "B", "heads", "Dk", "Dv"))
    n, C = B * h, -(-T // CHUNK)
    a, b = h * Dk, 2 * h * Dk
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), T, device="cuda")
    inside = (torch.arange(C * CHUNK, device="cuda") < lens.repeat_interleave(h)[:, None]).view(n, C, CHUNK, 1)
    of = lambda x, D: torch.where(inside, _by_head(x, s, D), 0.0)  # noqa: E731
    q, k, v = of(s["qkv"][:, :a], Dk), of(s["qkv"][:, a:b], Dk), of(s["qkv"][:, b:], Dv)
    zf, zb = of(s["z"][:, :h], 1), of(s["z"][:, h:], 1)
    rq, rk = 1.0 / torch.sqrt((q * q).sum(-1, keepdim=True) + EPS), 1.0 / torch.sqrt((k * k).sum(-1, keepdim=True) + EPS)
    q, k = q * rq, k * rk
    beta = torch.where(inside, 1.0 / (1.0 + torch.exp(-zb)), 0.0)
    log_f = torch.where(inside, -torch.log1p(torch.exp(-zf.double())), 0.0)
    G = log_f.cumsum(2)                                            # in 64 bits: differences of sums
    low = torch.ones((CHUNK, CHUNK), device="cuda").tril()
    span = torch.exp((G - G.transpose(2, 3)).masked_fill(low == 0, -math.inf)).float()
    first, last = torch.exp(G).float(), torch.exp(G[:, :, -1:] - G).float()
    whole = first[:, :, -1:]
    A = (beta * span * (k @ k.transpose(2, 3))).tril(-1)
    P = span * (q @ k.transpose(2, 3))
    inv = torch.eye(CHUNK, device="cuda").expand(n, C, CHUNK, CHUNK).clone()
    for i in range(1, CHUNK):
        inv[:, :, i, :i] = -(A[:, :, i:i + 1, :i] @ inv[:, :, :i, :i]).squeeze(2)
    S, states, us = s["h0"].view(n, Dk, Dv), [], []
    ys = torch.empty((n, C, CHUNK, Dv), device="cuda")
    for i in range(C):
        states.append(S)
        u = inv[:, i] @ (beta[:, i] * (v[:, i] - first[:, i] * (k[:, i] @ S)))
        ys[:, i] = scale * (first[:, i] * (q[:, i] @ S) + P[:, i] @ u)
        S = whole[:, i] * S + (last[:, i] * k[:, i]).transpose(1, 2) @ u
        us.append(u)
    out = {"y": _by_row(torch.where(inside, ys, 0.0), s).to(BF16), "hT": S.reshape(B, h, Dk, Dv)}
    if not c["grad"]:
        return out
    dy = of(s["dy"], Dv) * scale
    D = s["dhT"].view(n, Dk, Dv)
    at_end = (D * S).sum((1, 2))
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dzf, dzb = torch.empty_like(zf), torch.empty_like(zb)
    for i in reversed(range(C)):
        ki, qi, u, S0, do = k[:, i], q[:, i], us[i], states[i], dy[:, i]
        du = P[:, i].transpose(1, 2) @ do + last[:, i] * (ki @ D)
        x = inv[:, i].transpose(1, 2) @ du
        dr = beta[:, i] * x
        dv[:, i] = dr
        dP, dA = span[:, i] * (do @ u.transpose(1, 2)), (beta[:, i] * span[:, i] * (x @ u.transpose(1, 2))).tril(-1)
        dq[:, i] = first[:, i] * (do @ S0.transpose(1, 2)) + dP @ ki
        dk[:, i] = (dP.transpose(1, 2) @ qi - dA @ ki - dA.transpose(1, 2) @ ki - first[:, i] * (dr @ S0.transpose(1, 2))
                    + last[:, i] * (u @ D.transpose(1, 2)))
        dzb[:, i] = (x * u).sum(-1, keepdim=True) * (1.0 - beta[:, i])
        # what a step's decay sees is what the later steps' queries read and their values did not replace
        seen = ((qi * dq[:, i]).sum(-1) - (v[:, i] * dr).sum(-1)).flip(1).cumsum(1).flip(1) + at_end[:, None]
        dzf[:, i] = (seen * (1.0 / (1.0 + torch.exp(zf[:, i, :, 0]))))[..., None]
        D = whole[:, i] * D + (first[:, i] * qi).transpose(1, 2) @ do - (first[:, i] * ki).transpose(1, 2) @ dr
        at_end = (D * S0).sum((1, 2))
    dq, dk = rq * (dq - q * (q * dq).sum(-1, keepdim=True)), rk * (dk - k * (k * dk).sum(-1, keepdim=True))
    to = lambda x: _by_row(torch.where(inside, x, 0.0), s).to(BF16)  # noqa: E731
    out.update(_delta_gradients(s, torch.cat([to(dq), to(dk), to(dv)], 1), torch.cat([to(dzf), to(dzb)], 1), D.reshape(B, h, Dk, Dv)))
    return out


def _own_distill(s):
    from paper_2203_05705_b200 import ard
    c = s["case"]
    rows, V, k, dt = c["rows"], c["V"], c["k"], ard.ARD_F32 if c["dtype"] == "f32" else ard.ARD_BF16
    ard.ard_distill_loss(_context(), dt, rows, V, s["z"], V, s["labels"], k, s["teacher_ids"], s["teacher"], k, c["tau"], c["hard"], c["soft"],
                         s["weight"], s["loss"], s["total"], s["dz"], V)
    return {"loss": s["loss"], "total": s["total"], "dz": s["dz"]}


def _plain_distill(s):
    c, rows = s["case"], s["case"]["rows"]
    z, tau = s["z"].float(), c["tau"]
    loss, dz = torch.zeros(rows, device="cuda"), torch.zeros_like(z)
    m = z.amax(1, keepdim=True)
    d = z - m
    at = torch.arange(rows, device="cuda")
    if s["labels"] is not None:
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        label = s["labels"].clamp_min(0).long()
        there = c["hard"] * (s["labels"] >= 0).float()
        loss += there * (torch.log(total) - d.gather(1, label[:, None]))[:, 0]
        dz += there[:, None] * (e / total)
        dz[at, label] -= there
    if c["k"]:
        e = torch.exp(d / tau)
        total = e.sum(1, keepdim=True)
        ids, t = s["teacher_ids"].long(), s["teacher"] / tau
        t = t - t.amax(1, keepdim=True)
        mass = torch.exp(t).sum(1, keepdim=True)
        p = torch.exp(t) / mass
        loss += c["soft"] * tau * tau * (p * (t - torch.log(mass) - d.gather(1, ids) / tau + torch.log(total))).sum(1)
        dz += c["soft"] * tau * (e / total)
        dz.scatter_add_(1, ids, -c["soft"] * tau * p)
    dz *= s["weight"][:, None]
    return {"loss": loss, "total": (s["weight"].double() * loss.double()).sum().float().view(1), "dz": dz.to(s["td"])}


# ---- the definitions in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    return {"embed": _exact_embed, "delta": _exact_delta, "distill": _exact_distill}[case["kind"]](case, s)


def _exact_embed(case, s):
    kept = torch.tensor(list(_kept(case["N"], case["dp"])), device="cuda")
    ids = s["ids"].long()
    rows = torch.nonzero(ids >= 0)[:, 0]
    y = torch.zeros((case["rows"], len(kept)), dtype=F64, device="cuda")
    y[rows] = s["alpha"] * s["table"].index_select(1, kept)[ids[rows]].double()
    out = {"y": y}
    if case["grad"]:
        dtable = torch.zeros((case["V"], case["N"]), dtype=F64, device="cuda")
        wide = torch.zeros((len(rows), case["N"]), dtype=F64, device="cuda")
        wide[:, kept] = s["dy"][rows][:, :len(kept)].double()
        dtable.index_add_(0, ids[rows], wide, alpha=s["alpha"])
        out["dtable"] = dtable if s["left"] is None else dtable + s["left"]
    return out


def _exact_delta(case, s):
    """Step by step, as the recurrence is written."""
    T, B, h, Dk, Dv = (case[x] for x in ("T", "B", "heads", "Dk", "Dv"))
    x = s["qkv"].double().view(T, B, -1)
    raw_q, raw_k, v = x[..., :h * Dk].view(T, B, h, Dk), x[..., h * Dk:2 * h * Dk].view(T, B, h, Dk), x[..., 2 * h * Dk:].view(T, B, h, Dv)
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), T, device="cuda")
    inside = torch.arange(T, device="cuda")[:, None] < lens
    length = lambda x: (x.square().sum(-1, keepdim=True) + EPS).sqrt()  # noqa: E731
    q, k = raw_q / length(raw_q), raw_k / length(raw_k)
    z = s["z"].double().view(T, B, 2 * h)
    f, beta = torch.sigmoid(z[..., :h]), torch.sigmoid(z[..., h:])
    S = s["h0"].double()
    states, misses, ys = [S], [], []
    for t in range(T):
        miss = v[t] - f[t][..., None] * torch.einsum("bhkv,bhk->bhv", S, k[t])
        new = f[t][..., None, None] * S + torch.einsum("bhk,bhv->bhkv", k[t], beta[t][..., None] * miss)
        S = torch.where(inside[t][:, None, None, None], new, S)
        ys.append(torch.einsum("bhkv,bhk->bhv", S, q[t]))
        if case["grad"]:
            states.append(S)
            misses.append(miss)
    on = inside[..., None, None]
    out = {"y": torch.where(on, s["scale"] * torch.stack(ys), 0.0).reshape(T * B, h * Dv), "hT": S}
    if not case["grad"]:
        return out
    dy = torch.where(on, s["scale"] * s["dy"].double().view(T, B, h, Dv), 0.0)
    D = s["dhT"].double()
    dq, dk, dv, df, dbeta = (torch.zeros(a.shape, dtype=F64, device="cuda") for a in (q, k, v, f, beta))
    for t in reversed(range(T)):
        before, here = states[t], inside[t][:, None, None, None]
        E = D + torch.einsum("bhk,bhv->bhkv", q[t], dy[t])
        du = torch.einsum("bhkv,bhk->bhv", E, k[t])
        u = beta[t][..., None] * misses[t]
        dq[t] = torch.einsum("bhkv,bhv->bhk", states[t + 1], dy[t])
        db = beta[t][..., None] * du
        dk[t] = torch.einsum("bhkv,bhv->bhk", E, u) - f[t][..., None] * torch.einsum("bhkv,bhv->bhk", before, db)
        dv[t], dbeta[t] = db, (du * misses[t]).sum(-1)
        E = E - torch.einsum("bhk,bhv->bhkv", k[t], db)
        df[t] = (E * before).sum((-1, -2))
        D = torch.where(here, f[t][..., None, None] * E, D)
    through = lambda d, x, raw: (d - x * (x * d).sum(-1, keepdim=True)) / length(raw)  # noqa: E731
    masked = lambda d, on: torch.where(on, d, 0.0).reshape(T * B, -1)  # noqa: E731
    out.update(dq=masked(through(dq, q, raw_q), on), dk=masked(through(dk, k, raw_k), on), dv=masked(dv, on),
               dzf=masked(df * f * (1 - f), inside[..., None]), dzb=masked(dbeta * beta * (1 - beta), inside[..., None]), dh0=D)
    return out


def _exact_distill(case, s):
    z, rows, tau = s["z"].double(), case["rows"], case["tau"]
    loss, dz = torch.zeros(rows, dtype=F64, device="cuda"), torch.zeros(z.shape, dtype=F64, device="cuda")
    if s["labels"] is not None:
        log_p = torch.log_softmax(z, 1)
        live = torch.nonzero(s["labels"] >= 0)[:, 0]
        label = s["labels"][live].long()
        loss[live] -= case["hard"] * log_p[live, label]
        log_p.exp_()
        log_p[live, label] -= 1.0
        dz[live] = case["hard"] * log_p[live]
    if case["k"]:
        teacher = torch.softmax(s["teacher"].double() / tau, 1)
        log_q = torch.log_softmax(z / tau, 1)
        ids = s["teacher_ids"].long()
        loss += case["soft"] * tau ** 2 * torch.xlogy(teacher, teacher).sum(1)
        loss -= case["soft"] * tau ** 2 * (teacher * log_q.gather(1, ids)).sum(1)
        dz += case["soft"] * tau * log_q.exp_().scatter_add_(1, ids, -teacher)
    w = s["weight"].double()
    return {"loss": loss, "total": (w * loss).sum().view(1), "dz": dz * w[:, None]}
