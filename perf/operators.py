"""Cases of the operators around a layer's products: layer normalisation, the gated linear recurrence and the
optimiser's step, with what each computes in plain torch operations.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges,
`prepare(case, seed)` what a program holds before the call, `run(state)` one pass: in the plain form where `own` is
false, through the framework's entry points where it is true.  `work(case)` is the bytes and operations a pass cannot
do without, `exact(case, seed)` what a pass gives from the definition in 64 bits.

Kinds:
  norm   ard_layer_norm_fwd and ard_layer_norm_bwd over [rows][N], the reduction of the weight's and bias's gradient
         included; with dp > 1 over the compact columns of the neurons that a row pattern keeps
  glr    ard_glr_forward and, with "grad", ard_glr_backward: c_t = f_t c_{t-1} + (1 - f_t) g_t over [T][B][H], gates
         from pre-activations, with or without an output gate, padded batches, kept units
  adamw  ard_adamw_step over many tensors, states in 32 bits or in 8, with "clip" behind ard_grad_norm
"""
import functools
import math

import numpy as np
import torch

own = False

BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
EPS = 1e-5                                   # layer norm
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
MAX_NORM = 1.0
STATE_BLOCK = 128                            # elements that share a scale where states are held in 8 bits
CHUNK = 64                                   # time steps between two states that a backward pass starts from
E4M3_MAX, TINY = 448.0, 2.0 ** -110          # a block whose largest value is below TINY is held as zeros


# ---- cases --------------------------------------------------------------------------------------
MLP = "2048x784,2048,2048x2048,2048,10x2048,10"        # weights and biases of the 784-2048-2048-10 network
LSTM_1500 = "6000x3000,6000,6000x3000,6000,1500,1500"  # two layers of 1500 units, and a norm's weight and bias


def listed():
    return [
        # The tiny fp32 layer of the MNIST network's shape, normalised: launches and latency.
        {"name": "norm_64x256_f32", "kind": "norm", "dtype": "f32", "rows": 64, "N": 256, "dp": 1},
        # Between the 1500-wide layers over the 20 x 35 positions of a batch, half of the neurons kept: odd rows.
        {"name": "norm_700x1500_kept", "kind": "norm", "dtype": "bf16", "rows": 700, "N": 1500, "dp": 2},
        # Behind the hidden layers of the MLP at a large batch.
        {"name": "norm_16384x2048", "kind": "norm", "dtype": "bf16", "rows": 16384, "N": 2048, "dp": 1},
        # The large layer: 8192 neurons at batch 4096.
        {"name": "norm_4096x8192", "kind": "norm", "dtype": "bf16", "rows": 4096, "N": 8192, "dp": 1},
        # Serving: the next token of 64 sequences.
        {"name": "glr_token", "kind": "glr", "dtype": "bf16", "T": 1, "B": 64, "H": 1024, "dp": 1, "gate": True,
         "ragged": False, "grad": False},
        # The recurrent layer's training batch, 35 steps of 64 sequences, dropout on the hidden units.
        {"name": "glr_35x64x1024_kept", "kind": "glr", "dtype": "bf16", "T": 35, "B": 64, "H": 1024, "dp": 2, "gate": True,
         "ragged": False, "grad": True},
        # Odd sizes in fp32, sequences of different lengths, no output gate.
        {"name": "glr_777x5x1500_f32", "kind": "glr", "dtype": "f32", "T": 777, "B": 5, "H": 1500, "dp": 1, "gate": False,
         "ragged": True, "grad": True},
        # Reading one long document before an answer: few channels, many steps.
        {"name": "glr_16384x1x1024", "kind": "glr", "dtype": "bf16", "T": 16384, "B": 1, "H": 1024, "dp": 1, "gate": True,
         "ragged": False, "grad": False},
        # Training on long padded sequences.
        {"name": "glr_2048x8x2048", "kind": "glr", "dtype": "bf16", "T": 2048, "B": 8, "H": 2048, "dp": 1, "gate": True,
         "ragged": True, "grad": True},
        # The MLP's weights and biases after ard_mlp_step, gradients clipped by their norm.
        {"name": "adamw_mlp_clip", "kind": "adamw", "tensors": MLP, "grad_dtype": "f32", "bits": 32, "clip": True},
        # One 8192 x 8192 weight with a bf16 gradient.
        {"name": "adamw_8192", "kind": "adamw", "tensors": "8192x8192", "grad_dtype": "bf16", "bits": 32, "clip": False},
        # The recurrent layers' weights, states in 8 bits.
        {"name": "adamw8_lstm_1500", "kind": "adamw", "tensors": LSTM_1500, "grad_dtype": "f32", "bits": 8, "clip": True},
    ]


def _spread(rng, low, high):
    """A whole number of low..high, spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    kind = rng.choice(["norm", "glr", "adamw"])
    if kind == "norm":
        N = _spread(rng, 8, 16384)
        rows = _spread(rng, 1, min(65536, 4096 * 8192 // N))
        return {"kind": kind, "dtype": rng.choice(["f32", "bf16", "bf16"]), "rows": rows if N > 64 else min(rows, 16384), "N": N,
                "dp": rng.choice([1, 1, 2, 5]) if N >= 64 else 1}
    if kind == "glr":
        H = _spread(rng, 1, 4096)
        B = _spread(rng, 1, 64)
        T = _spread(rng, 1, max(1, min(16384, 2048 * 8 * 2048 // (B * H))))
        f32 = rng.random() < 0.3
        return {"kind": kind, "dtype": "f32" if f32 else "bf16", "T": max(1, T // 2) if f32 else T, "B": B, "H": H,
                "dp": rng.choice([1, 1, 2, 3]) if H >= 16 else 1, "gate": rng.random() < 0.6, "ragged": rng.random() < 0.5,
                "grad": rng.random() < 0.6}
    bits = rng.choice([32, 32, 8])
    room = (8192 * 8192 if bits == 32 else 2 * 6000 * 3000) // 4
    shapes = []
    for _ in range(_spread(rng, 1, 40)):
        rows, cols = _spread(rng, 1, 4096), _spread(rng, 1, 4096)
        if rows * cols > room:
            continue
        room -= rows * cols
        shapes.append("%dx%d" % (rows, cols))
        if rng.random() < 0.5:
            shapes.append("%d" % rows)
    return {"kind": kind, "tensors": ",".join(shapes or ["17"]), "grad_dtype": rng.choice(["f32", "bf16"]), "bits": bits,
            "clip": rng.random() < 0.5}


def _shapes(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["tensors"].split(",")]


def _kept(units, dp):
    """The kept units of a row pattern with period dp and offset 1 + dp // 2 (zero-based numbers)."""
    return range(dp // 2, units, dp)


def work(case):
    if case["kind"] == "norm":
        es, n = 4 if case["dtype"] == "f32" else 2, len(_kept(case["N"], case["dp"]))
        return {"bytes": case["rows"] * (n * es * (2 + 3) + 4 * 4) + 4 * (3 * n + 2 * case["N"]),
                "flops": case["rows"] * n * (8 + 14)}
    if case["kind"] == "glr":
        es, n = 4 if case["dtype"] == "f32" else 2, len(_kept(case["H"], case["dp"]))
        gates, cells = 3 if case["gate"] else 2, case["T"] * case["B"] * n
        if case["ragged"]:
            cells = int(_lens(case, 0).sum()) * n    # the padding is written, never read
        full = case["T"] * case["B"] * n
        moved = es * (cells * gates + full) + 8 * case["B"] * n
        flops = cells * (16 if case["gate"] else 10)
        if case["grad"]:
            moved += es * (cells * (gates + 1) + full * gates) + 8 * case["B"] * n
            flops += cells * (40 if case["gate"] else 26)
        return {"bytes": moved, "flops": flops}
    n = sum(math.prod(s) for s in _shapes(case))
    g = 4 if case["grad_dtype"] == "f32" else 2
    states = 16 if case["bits"] == 32 else 4 + 16 / STATE_BLOCK
    return {"bytes": n * (8 + g + 2 + states), "flops": n * ((3 if case["clip"] else 0) + (15 if case["bits"] == 32 else 60))}


# ---- inputs -------------------------------------------------------------------------------------
def _generator(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, scale=1.0, shift=0.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(dtype)


def _lens(case, seed):
    """Lengths of the sequences of a padded batch: the longest fills it, one may be empty."""
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
    s = {"case": dict(case), "kind": kind, "pat": None}
    if kind in ("norm", "glr"):
        units = case["N"] if kind == "norm" else case["H"]
        s["td"] = F32 if case["dtype"] == "f32" else BF16
        s["n"] = len(_kept(units, case["dp"]))
        if own and case["dp"] > 1:
            s["pat"] = _pattern(units, case["dp"])
    if kind == "norm":
        rows, N, td = case["rows"], case["N"], s["td"]
        s["x"] = _normal(g, rows, N, scale=1.5, shift=0.3, dtype=td)
        s["dy"] = _normal(g, rows, N, scale=0.1, dtype=td)
        s["weight"], s["bias"] = _normal(g, N, scale=0.2, shift=1.0), _normal(g, N, scale=0.2)
        s["y"], s["dx"] = torch.empty((rows, N), dtype=td, device="cuda"), torch.empty((rows, N), dtype=td, device="cuda")
        s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        s["dweight"], s["dbias"] = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    elif kind == "glr":
        T, B, H, td = case["T"], case["B"], case["H"], s["td"]
        s["zf"] = _normal(g, T, B, H, scale=1.5, shift=2.0, dtype=td)       # forget gates near one: a long memory
        s["zg"] = _normal(g, T, B, H, dtype=td)
        s["zo"] = _normal(g, T, B, H, dtype=td) if case["gate"] else None
        s["h0"] = _normal(g, B, H)
        s["lens"] = torch.from_numpy(_lens(case, seed)).cuda() if case["ragged"] else None
        s["y"], s["hT"] = torch.empty((T, B, H), dtype=td, device="cuda"), torch.zeros((B, H), device="cuda")
        if case["grad"]:
            s["dy"], s["dhT"] = _normal(g, T, B, H, scale=0.1, dtype=td), _normal(g, B, H, scale=0.1)
            s["S"] = torch.empty((-(-T // CHUNK), B, H), device="cuda")
            s["dzf"], s["dzg"] = torch.empty_like(s["zf"]), torch.empty_like(s["zf"])
            s["dzo"] = torch.empty_like(s["zf"]) if case["gate"] else None
            s["dh0"] = torch.zeros((B, H), device="cuda")
    else:
        # every tensor begins at a multiple of 128 elements of one buffer
        shapes = _shapes(case)
        starts, total = [], 0
        for sh in shapes:
            starts.append(total)
            total += -(-math.prod(sh) // STATE_BLOCK) * STATE_BLOCK
        gd = F32 if case["grad_dtype"] == "f32" else BF16
        s["p"], s["g"] = _normal(g, total, scale=0.02), _normal(g, total, scale=1e-3)
        s["g"] *= torch.exp(_normal(g, total // STATE_BLOCK, 1)).expand(-1, STATE_BLOCK).reshape(-1)   # rows of different sizes
        m, v = _normal(g, total, scale=3e-4), _normal(g, total, scale=1e-3).square_()
        s["w"] = torch.zeros(total, dtype=BF16, device="cuda")
        s["g"] = s["g"].to(gd)
        s["spans"] = [(a, math.prod(sh), 0.0 if len(sh) == 1 else DECAY, sh) for a, sh in zip(starts, shapes)]
        s["norm"] = torch.zeros(2, device="cuda")
        s["seed"], s["step"] = 1000 + int(seed), 7
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for a, n, _, _ in s["spans"]:
            inside[a:a + n] = True
        for t in (s["p"], s["g"], m, v):
            t.mul_(inside)
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
        if case["bits"] == 8:
            for k, x in (("m", m), ("v", v.sqrt())):
                blocks = x.view(-1, STATE_BLOCK)
                scale = blocks.abs().amax(1) / E4M3_MAX
                s[k] = (blocks / scale.clamp_min(TINY)[:, None]).to(E4M3).view(-1)
                s[k + "_scale"] = scale
        if own:
            s["tensors"] = _tensors(s)
    return s


def _tensors(s):
    """The framework's table of the tensors, as a program makes it once."""
    from paper_2203_05705_b200 import ard
    table = []
    for a, n, decay, shape in s["spans"]:
        rows, cols = (1,) * (2 - len(shape)) + shape
        part = lambda x, e=1: None if x is None else x[a // e:a // e + -(-n // e)]  # noqa: E731
        table.append({"rows": rows, "cols": cols, "p": part(s["p"]), "g": part(s["g"]), "w": part(s["w"]), "m": part(s["m"]), "v": part(s["v"]),
                      "m_scale": part(s["m_scale"], STATE_BLOCK), "v_scale": part(s["v_scale"], STATE_BLOCK), "weight_decay": decay})
    return ard.adamw_tensors(table)


# ---- one pass -----------------------------------------------------------------------------------
def run(s):
    if s["kind"] == "norm":
        return _own_norm(s) if own else _plain_norm(s)
    if s["kind"] == "glr":
        return _own_glr(s) if own else _plain_glr(s)
    return _own_adamw(s) if own else _plain_adamw(s)


def _norm_outputs(s, y, mean, rstd, dx, dw, db):
    n = s["n"]
    return {"y": y[:, :n], "mean": mean, "rstd": rstd, "dx": dx[:, :n], "dweight": dw, "dbias": db}


def _own_norm(s):
    from paper_2203_05705_b200 import ard
    c = s["case"]
    rows, N, dt = c["rows"], c["N"], ard.ARD_F32 if c["dtype"] == "f32" else ard.ARD_BF16
    ard.ard_layer_norm_fwd(_context(), s["pat"], dt, rows, N, EPS, s["x"], N, s["weight"], s["bias"], s["y"], N, s["mean"], s["rstd"])
    ard.ard_layer_norm_bwd(_context(), s["pat"], dt, rows, N, s["dy"], N, s["x"], N, s["weight"], s["mean"], s["rstd"], s["dx"], N,
                           s["dweight"], s["dbias"], 1)
    return _norm_outputs(s, s["y"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"])


def _plain_norm(s):
    c, n, td = s["case"], s["n"], s["td"]
    keep = slice(c["dp"] // 2, None, c["dp"])
    x, dy = s["x"][:, :n].float(), s["dy"][:, :n].float()
    w, b = s["weight"][keep], s["bias"][keep]
    mean = x.sum(1) / n
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / n + EPS)
    xh = d * rstd[:, None]
    y = xh * w + b
    e = dy * w
    dx = rstd[:, None] * (e - e.sum(1, keepdim=True) / n - xh * ((e * xh).sum(1, keepdim=True) / n))
    dw, db = torch.zeros_like(s["weight"]), torch.zeros_like(s["bias"])
    dw[keep], db[keep] = (dy * xh).sum(0), dy.sum(0)
    return _norm_outputs(s, y.to(td), mean, rstd, dx.to(td), dw, db)


def _glr_outputs(s, y, hT, dzf=None, dzg=None, dzo=None, dh0=None):
    n = s["n"]
    out = {"y": y[..., :n], "hT": hT}
    if s["case"]["grad"]:
        out.update(dzf=dzf[..., :n], dzg=dzg[..., :n], dzo=None if dzo is None else dzo[..., :n], dh0=dh0)
    return out


def _own_glr(s):
    from paper_2203_05705_b200 import ard
    c = s["case"]
    T, B, H, dt, grad = c["T"], c["B"], c["H"], ard.ARD_F32 if c["dtype"] == "f32" else ard.ARD_BF16, c["grad"]
    alpha = float(c["dp"])
    ard.ard_glr_forward(_context(), s["pat"], dt, T, B, H, alpha, s["zf"], s["zg"], s["zo"], H, s["lens"], s["h0"], s["y"], H, s["hT"],
                        s["S"] if grad else None)
    if not grad:
        return _glr_outputs(s, s["y"], s["hT"])
    ard.ard_glr_backward(_context(), s["pat"], dt, T, B, H, alpha, s["zf"], s["zg"], s["zo"], H, s["lens"], s["S"], s["dy"], H, s["dhT"],
                         s["dzf"], s["dzg"], s["dzo"], H, s["dh0"])
    return _glr_outputs(s, s["y"], s["hT"], s["dzf"], s["dzg"], s["dzo"], s["dh0"])


def _scan(a, b, first):
    """x_t = a_t x_{t-1} + b_t along the first axis from x_{-1} = first, by doubling: after the k-th pass an entry holds the
    composition of 2^k steps."""
    b = b.clone()
    b[0] += a[0] * first
    a = a.clone()
    k = 1
    while k < a.shape[0]:
        b[k:] = b[k:] + a[k:] * b[:-k]
        a[k:] = a[k:] * a[:-k]
        k *= 2
    return b


def _plain_glr(s):
    c, n, td = s["case"], s["n"], s["td"]
    keep = slice(c["dp"] // 2, None, c["dp"])
    alpha = float(c["dp"])
    inside = None
    if s["lens"] is not None:
        inside = (torch.arange(c["T"], device="cuda")[:, None] < s["lens"][None, :])[..., None]
    zf, zg = s["zf"][..., :n].float(), s["zg"][..., :n].float()
    f, i = 1.0 / (1.0 + torch.exp(-zf)), 1.0 / (1.0 + torch.exp(zf))
    fs, b = f, i * zg
    if inside is not None:
        fs, b = torch.where(inside, f, 1.0), torch.where(inside, b, 0.0)
    h0 = s["h0"][:, keep]
    state = _scan(fs, b, h0)
    o = alpha / (1.0 + torch.exp(-s["zo"][..., :n].float())) if c["gate"] else torch.full((), alpha, device="cuda")
    y = o * state
    if inside is not None:
        y = torch.where(inside, y, 0.0)
    hT = torch.zeros_like(s["h0"])
    hT[:, keep] = state[-1]
    if not c["grad"]:
        return _glr_outputs(s, y.to(td), hT)
    dy = s["dy"][..., :n].float()
    if inside is not None:
        dy = torch.where(inside, dy, 0.0)
    e = dy * o
    e[-1] += s["dhT"][:, keep]
    back = torch.cat([torch.ones_like(fs[:1]), fs.flip(0)[:-1]])
    d = _scan(back, e.flip(0), torch.zeros_like(h0)).flip(0)
    before = torch.cat([h0[None], state[:-1]])
    dzf, dzg = d * (before - zg) * f * i, d * i
    dzo = dy * state * o * (1.0 - o / alpha) if c["gate"] else None
    if inside is not None:
        dzf, dzg = torch.where(inside, dzf, 0.0), torch.where(inside, dzg, 0.0)
    dh0 = torch.zeros_like(s["h0"])
    dh0[:, keep] = fs[0] * d[0]
    return _glr_outputs(s, y.to(td), hT, dzf.to(td), dzg.to(td), None if dzo is None else dzo.to(td), dh0)


def _adamw_outputs(s):
    out = {"p": s["p"], "w": s["w"], "m": s["m"], "v": s["v"]}
    if s["case"]["bits"] == 8:      # an element's value is its 8 bits times its block's scale; v holds the root
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["case"]["clip"]:
        out["norm"] = s["norm"]
    return out


def _own_adamw(s):
    from paper_2203_05705_b200 import ard
    c, n = s["case"], len(s["spans"])
    if c["clip"]:
        ard.ard_grad_norm(_context(), s["tensors"], n, MAX_NORM, s["norm"])
    ard.ard_adamw_step(_context(), s["tensors"], n, LR, BETA1, BETA2, ADAM_EPS, c["bits"], s["seed"], s["step"], None, None,
                       s["norm"][1:] if c["clip"] else None)
    return _adamw_outputs(s)


def _philox(seed, step, number, quads):
    """Philox4x32-10 with the key `seed` and the counters (step low, step high, quad, 1 + number of the tensor), as four words
    for each quad in 64-bit integers."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, seed >> 32 & low
    c = [torch.full_like(quads, step & low), torch.full_like(quads, step >> 32), quads, torch.full_like(quads, 1 + number)]
    for _ in range(10):
        x, y = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57     # the low 64 bits, whatever the sign
        c = [(y >> 32 & low) ^ c[1] ^ k0, y & low, (x >> 32 & low) ^ c[3] ^ k1, x & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack(c, 1)


def _to_e4m3(x, random16):
    """|x| rounded to 8-bit floats (3 bits of mantissa, down to 2^-9), up with the probability of what is cut off."""
    a = x.abs()
    low = a < 2.0 ** -6
    bits = torch.where(low, a + 2.0 ** -6, a).view(torch.int32) + ((random16 << 4) + 8).to(torch.int32)
    q = (bits & ~0xFFFFF).view(F32)
    return torch.where(low, q - 2.0 ** -6, q).clamp_max(E4M3_MAX)


def _pack(x, random16, positive):
    """(8-bit floats, scales) of the blocks of x [blocks][128]."""
    big = x.abs().amax(1)
    fine = big >= TINY
    q = _to_e4m3(x * torch.where(fine, E4M3_MAX / big, 0.0)[:, None], random16)
    if positive:                                        # a root that is not zero is not held as zero
        q = torch.where((x > 0) & fine[:, None], q.clamp_min(2.0 ** -9), q)
    return torch.copysign(q, x), torch.where(fine, big / E4M3_MAX, 0.0)


def _plain_adamw(s):
    c, factor = s["case"], 1.0
    if c["clip"]:
        norm = torch.sqrt(sum(s["g"][a:a + n].double().square().sum() for a, n, _, _ in s["spans"]))
        factor = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
        s["norm"].copy_(torch.stack([norm, factor]))
        factor = s["norm"][1]
    lift1, lift2 = 1.0 / (1.0 - BETA1 ** s["step"]), 1.0 / (1.0 - BETA2 ** s["step"])
    for k, (a, n, decay, _) in enumerate(s["spans"]):
        part = slice(a, a + n)
        g = s["g"][part].float() * factor
        if c["bits"] == 32:
            m, v = s["m"][part], s["v"][part]
        else:
            whole = slice(a, a + -(-n // STATE_BLOCK) * STATE_BLOCK)
            blocks = slice(a // STATE_BLOCK, whole.stop // STATE_BLOCK)
            m = (s["m"][whole].float().view(-1, STATE_BLOCK) * s["m_scale"][blocks, None]).view(-1)[:n]
            v = (s["v"][whole].float().view(-1, STATE_BLOCK) * s["v_scale"][blocks, None]).view(-1)[:n].square()
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g * g
        p = s["p"][part]
        p.copy_(p * (1.0 - LR * decay) - LR * (m * lift1) / (torch.sqrt(v * lift2) + ADAM_EPS))
        s["w"][part] = p.to(BF16)
        if c["bits"] == 32:
            s["m"][part], s["v"][part] = m, v
            continue
        words = _philox(s["seed"], s["step"], k, torch.arange((whole.stop - a) // 4, device="cuda")).view(-1, STATE_BLOCK)
        fill = whole.stop - a - n
        pad = lambda x: torch.cat([x, x.new_zeros(fill)]).view(-1, STATE_BLOCK)  # noqa: E731
        for key, x, r, positive in (("m", m, words & 0xFFFF, False), ("v", torch.sqrt(v), words >> 16, True)):
            q, scale = _pack(pad(x), r, positive)
            s[key][whole] = q.view(-1).to(E4M3)
            s[key + "_scale"][blocks] = scale
    return _adamw_outputs(s)


# ---- the definitions in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    return {"norm": _exact_norm, "glr": _exact_glr, "adamw": _exact_adamw}[case["kind"]](case, s)


def _exact_norm(case, s):
    kept = torch.tensor(list(_kept(case["N"], case["dp"])), device="cuda")
    n = len(kept)
    x, dy = s["x"][:, :n].double(), s["dy"][:, :n].double()
    w, b = s["weight"].double()[kept], s["bias"].double()[kept]
    mean, var = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
    rstd = (var + EPS).rsqrt()
    xh = (x - mean) * rstd
    # the Jacobian of a row's (x - mean) / std is (I - 1/n - xh xh^T / n) / std
    e = dy * w
    dx = (e - e.mean(1, keepdim=True) - xh * (e * xh).mean(1, keepdim=True)) * rstd
    dw, db = torch.zeros(case["N"], dtype=F64, device="cuda"), torch.zeros(case["N"], dtype=F64, device="cuda")
    dw.index_add_(0, kept, (dy * xh).sum(0))
    db.index_add_(0, kept, dy.sum(0))
    return {"y": xh * w + b, "mean": mean[:, 0], "rstd": rstd[:, 0], "dx": dx, "dweight": dw, "dbias": db}


def _exact_glr(case, s):
    """Step by step, as the recurrence is written."""
    kept = torch.tensor(list(_kept(case["H"], case["dp"])), device="cuda")
    n, T, alpha = len(kept), case["T"], float(case["dp"])
    lens = s["lens"] if s["lens"] is not None else torch.full((case["B"],), T, device="cuda")
    c = s["h0"].double()[:, kept]
    f, g = torch.sigmoid(s["zf"][..., :n].double()), s["zg"][..., :n].double()
    o = torch.sigmoid(s["zo"][..., :n].double()) if case["gate"] else None
    states = [c]
    for t in range(T):
        c = torch.where((t < lens)[:, None], g[t] + f[t] * (c - g[t]), c)
        states.append(c)
    inside = (torch.arange(T, device="cuda")[:, None] < lens)[..., None]
    after = torch.stack(states[1:])
    y = torch.where(inside, alpha * after if o is None else alpha * o * after, 0.0)
    hT = torch.zeros(s["h0"].shape, dtype=F64, device="cuda")
    hT[:, kept] = c
    out = {"y": y, "hT": hT}
    if not case["grad"]:
        return out
    dy = torch.where(inside, alpha * s["dy"][..., :n].double(), 0.0)
    d = s["dhT"].double()[:, kept]
    ds = [None] * T
    for t in reversed(range(T)):
        d = d + (dy[t] if o is None else dy[t] * o[t])
        ds[t] = d
        d = torch.where((t < lens)[:, None], d * f[t], d)
    ds = torch.where(inside, torch.stack(ds), 0.0)
    i = torch.sigmoid(-s["zf"][..., :n].double())
    out["dzf"], out["dzg"] = ds * (torch.stack(states[:-1]) - g) * f * i, ds * i
    out["dzo"] = None if o is None else dy * after * o * (1 - o)
    out["dh0"] = torch.zeros(s["h0"].shape, dtype=F64, device="cuda")
    out["dh0"][:, kept] = d
    return out


def _words(seed, step, number, quads):
    """Philox4x32-10 over numpy's unsigned integers."""
    u = np.uint64
    half = u(32)
    c0, c1, c2, c3 = (np.full(quads, x, u) for x in (step % 2 ** 32, step >> 32, 0, 1 + number))
    c2 += np.arange(quads, dtype=u)
    k0, k1 = seed % 2 ** 32, seed >> 32
    for _ in range(10):
        a, b = c0 * u(0xD2511F53), c2 * u(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> half) ^ c1 ^ u(k0), b & u(0xFFFFFFFF), (a >> half) ^ c3 ^ u(k1), a & u(0xFFFFFFFF)
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return np.stack([c0, c1, c2, c3], 1).astype(np.int64).reshape(-1)


def _rounded(x, random16, floor):
    """x / scale on the grid of the 8-bit floats, and the scale."""
    big = x.abs().amax(1, keepdim=True)
    x = torch.where(big >= TINY, x / (big / E4M3_MAX).clamp_min(1e-300), 0.0)
    exponent = torch.floor(torch.log2(x.abs().clamp_min(1e-300))).clamp_min(-6.0)
    quantum = torch.exp2(exponent - 3)
    q = torch.floor(x.abs() / quantum + (random16 + 0.5) / 65536) * quantum
    q = torch.where((x != 0) & (q == 0), floor, q).clamp_max(E4M3_MAX)
    return q * torch.sign(x), torch.where(big >= TINY, big / E4M3_MAX, 0.0)[:, 0]


def _exact_adamw(case, s):
    wide = {k: (s[k].float() if s[k].dtype == E4M3 else s[k]).double() for k in ("p", "g", "m", "v")}
    factor, out = 1.0, {}
    if case["clip"]:
        norm = math.sqrt(sum(float((wide["g"][a:a + n] ** 2).sum()) for a, n, _, _ in s["spans"]))
        factor = min(1.0, MAX_NORM / (norm + 1e-6))
        out["norm"] = torch.tensor([norm, factor], dtype=F64)
    for k in ("m", "v"):
        if case["bits"] == 8:
            wide[k] = wide[k] * s[k + "_scale"].double().repeat_interleave(STATE_BLOCK)
    if case["bits"] == 8:
        wide["v"] = wide["v"] ** 2
    g = wide["g"] * factor
    m, v = BETA1 * wide["m"] + (1 - BETA1) * g, BETA2 * wide["v"] + (1 - BETA2) * g ** 2
    decay = torch.zeros_like(g)
    for a, n, x, _ in s["spans"]:
        decay[a:a + n] = x
    t = s["step"]
    p = wide["p"] - LR * (decay * wide["p"] + m / (1 - BETA1 ** t) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS))
    out.update(p=p, w=p, m=m, v=v)
    if case["bits"] == 8:
        words = np.concatenate([_words(s["seed"], t, k, -(-n // STATE_BLOCK) * STATE_BLOCK // 4) for k, (_, n, _, _) in enumerate(s["spans"])])
        words = torch.from_numpy(words).cuda().view(-1, STATE_BLOCK)
        for key, x, r, floor in (("m", m, words & 0xFFFF, 0.0), ("v", v.sqrt(), words >> 16, 2.0 ** -9)):
            q, scale = _rounded(x.view(-1, STATE_BLOCK), r, floor)
            out[key], out[key + "_scale"] = q.view(-1), scale
    return out
