"""What the operators around the products refuse before anything is launched (no GPU: a context that is never looked into, since
arguments are judged first)."""
import ctypes as C

import pytest

from paper_2203_05705_b200 import ard

# memory that stands for a context and for device buffers; no call gets so far as to use either
_CTX = C.create_string_buffer(8192)
CTX = C.c_void_p(C.addressof(_CTX))
P = [4096 * (k + 1) for k in range(16)]
INVALID, SHAPE, UNSUPPORTED = ard.ARD_ERR_INVALID_ARG, ard.ARD_ERR_SHAPE, ard.ARD_ERR_UNSUPPORTED
NAN, INF = float("nan"), float("inf")

LN_FWD = dict(pat=None, dtype=1, rows=4, N=8, eps=1e-5, X=P[0], ldx=8, weight=None, bias=None, Y=P[1], ldy=8, mean=None, rstd=None)
LN_BWD = dict(pat=None, dtype=0, rows=4, N=8, dY=P[0], lddy=8, X=P[1], ldx=8, weight=None, mean=P[2], rstd=P[3], dX=P[4], lddx=8,
              dweight=None, dbias=None, zero=0)
GLR_FWD = dict(pat=None, dtype=1, T=3, B=2, H=8, alpha=1.0, Zf=P[0], Zg=P[1], Zo=None, ldz=8, lens=None, h0=None, Y=P[2], ldy=8,
               hT=None, S=None)
GLR_BWD = dict(pat=None, dtype=1, T=3, B=2, H=8, alpha=1.0, Zf=P[0], Zg=P[1], Zo=P[2], ldz=8, lens=None, S=P[3], dY=P[4], lddy=8,
               dhT=None, dZf=P[5], dZg=P[6], dZo=P[7], lddz=8, dh0=None)


@pytest.mark.parametrize("name,good,change,status", [
    (name, good, dict([change[:2]]), change[2]) for name, good, changes in [
        ("ard_layer_norm_fwd", LN_FWD, [("dtype", 2, INVALID), ("rows", -1, INVALID), ("N", -1, INVALID), ("eps", -1.0, INVALID),
                                        ("eps", NAN, INVALID), ("eps", INF, INVALID), ("X", None, INVALID), ("Y", None, INVALID),
                                        ("Y", P[0], INVALID), ("ldx", 7, SHAPE), ("ldy", 7, SHAPE), ("rows", 2 ** 31 - 1, UNSUPPORTED)]),
        ("ard_layer_norm_bwd", LN_BWD, [("dtype", -1, INVALID), ("rows", -1, INVALID), ("N", -1, INVALID), ("dY", None, INVALID),
                                        ("X", None, INVALID), ("mean", None, INVALID), ("rstd", None, INVALID), ("dX", P[0], INVALID),
                                        ("dX", P[1], INVALID), ("lddy", 7, SHAPE), ("ldx", 7, SHAPE), ("lddx", 7, SHAPE)]),
        ("ard_glr_forward", GLR_FWD, [("dtype", 3, INVALID), ("T", -1, INVALID), ("B", -1, INVALID), ("H", -1, INVALID),
                                      ("Zf", None, INVALID), ("Zg", None, INVALID), ("Y", None, INVALID), ("Y", P[0], INVALID),
                                      ("Y", P[1], INVALID), ("ldz", 7, SHAPE), ("ldy", 7, SHAPE), ("T", 2 ** 31 - 1, UNSUPPORTED)]),
        ("ard_glr_backward", GLR_BWD, [("dtype", 3, INVALID), ("T", -1, INVALID), ("S", None, INVALID), ("dY", None, INVALID),
                                       ("dZf", None, INVALID), ("dZg", None, INVALID), ("dZo", None, INVALID), ("Zo", None, INVALID),
                                       ("dZf", P[0], INVALID), ("dZo", P[4], INVALID), ("ldz", 7, SHAPE), ("lddy", 7, SHAPE),
                                       ("lddz", 7, SHAPE)]),
    ] for change in changes])
def test_layer_norm_and_recurrence(name, good, change, status):
    call = getattr(ard, name)
    for ctx in (None, CTX):
        args = {**good, **change}
        with pytest.raises(ard.ArdError) as e:
            call(ctx, *args.values(), stream=0)
        assert e.value.status == (INVALID if ctx is None else status)


TENSOR = dict(rows=3, cols=8, p=P[0], ldp=8, g=P[1], ldg=8, g_dtype=0, w=P[2], ldw=8, m=P[3], v=P[4], m_scale=P[5], v_scale=P[6],
              weight_decay=0.1)
STEP = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, bits=8, seed=1, step=1)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(p=None), INVALID), (dict(g=None), INVALID), (dict(m=None), INVALID),
    (dict(v=None), INVALID), (dict(m_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(g_dtype=2), INVALID),
    (dict(weight_decay=-0.1), INVALID), (dict(weight_decay=NAN), INVALID), (dict(ldp=7), SHAPE), (dict(ldg=7), SHAPE), (dict(ldw=7), SHAPE),
    (dict(rows=2 ** 20, cols=2 ** 20), SHAPE), (dict(rows=2 ** 62, cols=2 ** 62), SHAPE)])
def test_optimiser_tensors(change, status):
    good = ard.adamw_tensors([TENSOR, TENSOR])
    bad = ard.adamw_tensors([TENSOR, {**TENSOR, **change}])   # the second one: nothing may start on the first
    with pytest.raises(ard.ArdError) as e:
        ard.ard_adamw_step(CTX, bad, 2, *STEP.values(), stream=0)
    assert e.value.status == status
    if set(change) & {"rows", "cols", "g", "g_dtype", "ldg"}:
        with pytest.raises(ard.ArdError) as e:
            ard.ard_grad_norm(CTX, bad, 2, 1.0, P[8], stream=0)
        assert e.value.status == status
    for call in (lambda t: ard.ard_adamw_step(None, t, 2, *STEP.values(), stream=0), lambda t: ard.ard_grad_norm(None, t, 2, 1.0, P[8], stream=0)):
        with pytest.raises(ard.ArdError) as e:
            call(good)
        assert e.value.status == INVALID


@pytest.mark.parametrize("change", [dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                                    dict(beta2=NAN), dict(eps=-1.0), dict(eps=NAN), dict(bits=16), dict(bits=0)])
def test_optimiser_numbers(change):
    with pytest.raises(ard.ArdError) as e:
        ard.ard_adamw_step(CTX, ard.adamw_tensors([TENSOR]), 1, *{**STEP, **change}.values(), stream=0)
    assert e.value.status == INVALID


def test_optimiser_tables():
    t = ard.adamw_tensors([TENSOR])
    for call in (lambda n, t: ard.ard_adamw_step(CTX, t, n, *STEP.values(), stream=0), lambda n, t: ard.ard_grad_norm(CTX, t, n, 1.0, P[8], stream=0)):
        for n, table in ((-1, t), (1, None)):
            with pytest.raises(ard.ArdError) as e:
                call(n, table)
            assert e.value.status == INVALID
    for out, most in ((None, 1.0), (P[8], NAN)):
        with pytest.raises(ard.ArdError) as e:
            ard.ard_grad_norm(CTX, t, 1, most, out, stream=0)
        assert e.value.status == INVALID


def test_table_of_tensors():
    import torch
    g = torch.zeros(4, 6, dtype=torch.bfloat16)
    t = ard.adamw_tensors([{"rows": 4, "cols": 6, "p": 64, "g": g, "m": 128, "v": 256, "ldg": 7}])[0]
    assert (t.g, t.g_dtype, t.ldg, t.ldp, t.w, t.weight_decay) == (g.data_ptr(), ard.ARD_BF16, 7, 6, None, 0.0)
    assert ard.adamw_tensors([{"rows": 1, "cols": 6, "p": 64, "g": g.float(), "m": 1, "v": 2}])[0].g_dtype == ard.ARD_F32
    for bad in ({"g": 64}, {"g": torch.zeros(2, dtype=torch.float16)}, {"g": g, "decay": 0.1}):
        with pytest.raises(ValueError):
            ard.adamw_tensors([{"rows": 1, "cols": 2, "p": 64, "m": 1, "v": 2, **bad}])
    with pytest.raises(KeyError):
        ard.adamw_tensors([{"rows": 1, "p": 64}])
    assert len(ard.adamw_tensors([])) == 1   # a table that no call looks into


@pytest.mark.parametrize("name,good,change", [
    ("ard_layer_norm_fwd", LN_FWD, dict(mean=P[5], rstd=P[5])), ("ard_layer_norm_bwd", LN_BWD, dict(dweight=P[5], dbias=P[5])),
    ("ard_glr_backward", GLR_BWD, dict(dZf=P[6])), ("ard_glr_backward", GLR_BWD, dict(dZo=P[5])), ("ard_glr_backward", GLR_BWD, dict(dZo=P[6])),
    ("ard_glr_backward", GLR_BWD, dict(Zo=None, dZo=None, dZg=P[5]))])
def test_outputs_in_the_same_place(name, good, change):
    with pytest.raises(ard.ArdError) as e:
        getattr(ard, name)(CTX, *{**good, **change}.values(), stream=0)
    assert e.value.status == INVALID


@pytest.mark.parametrize("eps", [1e-40, 1e-50, 5e-324])
def test_an_eps_that_fp32_holds_only_as_a_subnormal(eps):
    with pytest.raises(ard.ArdError) as e:
        ard.ard_adamw_step(CTX, ard.adamw_tensors([TENSOR]), 1, *{**STEP, "eps": eps}.values(), stream=0)
    assert e.value.status == INVALID
