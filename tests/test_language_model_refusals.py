"""What the embedding, the gated delta rule and the loss refuse before anything is launched (no GPU: see test_operator_refusals.py)."""
import pytest

from paper_2203_05705_b200 import ard
from test_operator_refusals import CTX, INF, INVALID, NAN, P, SHAPE, UNSUPPORTED

NOMEM, ALIGN = ard.ARD_ERR_NOMEM, ard.ARD_ERR_ALIGNMENT
BIG = 1 << 40
EMB_FWD = dict(pat=None, dtype=1, rows=4, V=9, N=8, alpha=1.0, ids=P[0], table=P[1], ldt=8, Y=P[2], ldy=8)
EMB_BWD = dict(pat=None, dtype=1, rows=4, V=9, N=8, alpha=1.0, ids=P[0], dY=P[1], lddy=8, dtable=P[2], lddt=8, accumulate=0)
LOSS = dict(dtype=1, rows=4, V=9, Z=P[0], ldz=9, labels=P[1], k=2, teacher_ids=P[2], teacher_logits=P[3], ldk=2, tau=2.0, hard=0.5, soft=0.5,
            row_weight=P[4], loss=P[5], total=P[6], dZ=P[7], lddz=9)
DELTA_FWD = dict(dtype=1, T=70, B=2, heads=2, Dk=8, Dv=4, scale=1.0, eps=1e-6, Q=P[0], ldq=16, K=P[1], ldk=16, V=P[2], ldv=8, Zf=P[3], Zb=P[4], ldz=2,
                 lens=P[5], h0=P[6], Y=P[7], ldy=8, hT=P[8], S=P[9], work=P[10], work_bytes=BIG)
DELTA_BWD = dict(dtype=1, T=70, B=2, heads=2, Dk=8, Dv=4, scale=1.0, eps=1e-6, Q=P[0], ldq=16, K=P[1], ldk=16, V=P[2], ldv=8, Zf=P[3], Zb=P[4], ldz=2,
                 lens=P[5], S=P[6], dY=P[7], lddy=8, dhT=P[8], dQ=P[9], lddq=16, dK=P[10], lddk=16, dV=P[11], lddv=8, dZf=P[12], dZb=P[13], lddz=2,
                 dh0=P[14], work=P[15], work_bytes=BIG)
CALLS = {
    "ard_embedding_fwd": (EMB_FWD, [("dtype", 2, INVALID), ("rows", -1, INVALID), ("V", -1, INVALID), ("N", -1, INVALID), ("ids", None, INVALID),
                                    ("table", None, INVALID), ("Y", None, INVALID), ("Y", P[1], INVALID), ("ldt", 7, SHAPE), ("ldy", 7, SHAPE),
                                    ("rows", 2 ** 31 - 1, UNSUPPORTED)]),
    "ard_embedding_bwd": (EMB_BWD, [("dtype", -1, INVALID), ("rows", -1, INVALID), ("V", -1, INVALID), ("N", -1, INVALID), ("ids", None, INVALID),
                                    ("dY", None, INVALID), ("dtable", None, INVALID), ("dtable", P[1], INVALID), ("lddy", 7, SHAPE), ("lddt", 7, SHAPE),
                                    ("rows", 2 ** 31 - 1, UNSUPPORTED)]),
    "ard_distill_loss": (LOSS, [("dtype", 2, INVALID), ("rows", -1, INVALID), ("V", -1, INVALID), ("Z", None, INVALID), ("k", -1, INVALID),
                                ("teacher_ids", None, INVALID), ("teacher_logits", None, INVALID), ("tau", 0.0, INVALID), ("tau", -1.0, INVALID),
                                ("tau", NAN, INVALID), ("tau", INF, INVALID), ("tau", 1e-39, INVALID), ("hard", NAN, INVALID), ("hard", INF, INVALID),
                                ("soft", INF, INVALID), ("soft", 3e38, INVALID), ("loss", None, INVALID), ("loss", P[6], INVALID), ("ldz", 8, SHAPE),
                                ("lddz", 8, SHAPE), ("ldk", 1, SHAPE), ("rows", 2 ** 31 - 1, UNSUPPORTED)]),
    "ard_delta_forward": (DELTA_FWD, [("dtype", 3, INVALID), ("dtype", 0, UNSUPPORTED), ("T", -1, INVALID), ("B", -1, INVALID), ("heads", -1, INVALID),
                                      ("Dk", -1, INVALID), ("Dv", -1, INVALID), ("scale", NAN, INVALID), ("eps", INF, INVALID), ("Q", None, INVALID),
                                      ("K", None, INVALID), ("V", None, INVALID), ("Zf", None, INVALID), ("Zb", None, INVALID), ("Y", None, INVALID),
                                      ("Y", P[0], INVALID), ("Y", P[2], INVALID), ("Y", P[4], INVALID), ("S", P[6], INVALID), ("S", P[8], INVALID),
                                      ("ldq", 15, SHAPE), ("ldk", 15, SHAPE), ("ldv", 7, SHAPE), ("ldz", 1, SHAPE), ("ldy", 7, SHAPE),
                                      ("Dk", 129, UNSUPPORTED), ("Dv", 129, UNSUPPORTED), ("T", 2 ** 31 - 1, UNSUPPORTED), ("B", 2 ** 30, UNSUPPORTED),
                                      ("work", None, INVALID), ("work_bytes", 100, NOMEM)]),
    "ard_delta_backward": (DELTA_BWD, [("dtype", 3, INVALID), ("dtype", 0, UNSUPPORTED), ("T", -1, INVALID), ("S", None, INVALID), ("S", P[14], INVALID),
                                       ("dY", None, INVALID), ("dQ", None, INVALID), ("dK", None, INVALID), ("dV", None, INVALID), ("dZf", None, INVALID),
                                       ("dZb", None, INVALID), ("dQ", P[0], INVALID), ("dV", P[7], INVALID), ("dZb", P[12], INVALID), ("dK", P[9], INVALID),
                                       ("lddq", 15, SHAPE), ("lddk", 15, SHAPE), ("lddv", 7, SHAPE), ("lddz", 1, SHAPE), ("lddy", 7, SHAPE),
                                       ("Dk", 200, UNSUPPORTED), ("work", None, INVALID), ("work_bytes", 0, NOMEM)]),
}


@pytest.mark.parametrize("name,change,status", [(n, c[:2], c[2]) for n, (_, changes) in CALLS.items() for c in changes])
def test_refused(name, change, status):
    for ctx in (None, CTX):
        with pytest.raises(ard.ArdError) as e:
            getattr(ard, name)(ctx, *{**CALLS[name][0], change[0]: change[1]}.values(), stream=0)
        assert e.value.status == (INVALID if ctx is None else status)


def test_the_teachers_entries_are_bounded():
    with pytest.raises(ard.ArdError) as e:
        ard.ard_distill_loss(CTX, *{**LOSS, "k": 1025, "ldk": 1025}.values(), stream=0)
    assert e.value.status == UNSUPPORTED


def test_a_gradient_in_place_has_the_logits_rows():
    with pytest.raises(ard.ArdError) as e:
        ard.ard_distill_loss(CTX, *{**LOSS, "dZ": LOSS["Z"], "lddz": 10}.values(), stream=0)
    assert e.value.status == SHAPE


@pytest.mark.parametrize("name,key", [(n, k) for n, (good, _) in CALLS.items() for k, v in good.items() if v in P and k not in ("work",)])
def test_pointers_inside_an_element(name, key):
    good = CALLS[name][0]
    wide = {"ids", "dtable", "labels", "teacher_ids", "teacher_logits", "row_weight", "loss", "total", "lens", "h0", "hT", "S", "dhT", "dh0"}
    for off in (1, 2, 3):
        if off == 2 and key not in wide:
            continue          # a whole element
        with pytest.raises(ard.ArdError) as e:
            getattr(ard, name)(CTX, *{**good, key: good[key] + off}.values(), stream=0)
        assert e.value.status == ALIGN


def test_columns_of_a_table_are_bounded():
    n = (1 << 30) + 1
    for name, good, lds in (("ard_embedding_fwd", EMB_FWD, ("ldt", "ldy")), ("ard_embedding_bwd", EMB_BWD, ("lddy", "lddt"))):
        with pytest.raises(ard.ArdError) as e:
            getattr(ard, name)(CTX, *{**good, "N": n, lds[0]: n, lds[1]: n}.values(), stream=0)
        assert e.value.status == UNSUPPORTED


def test_work_of_the_delta_rule():
    size = ard.ard_delta_work_bytes
    assert size(1, 64, 8, 128, 128, False) == 0            # decoding takes none
    assert 0 < size(100, 2, 2, 64, 64, False) < size(100, 2, 2, 64, 64, True)
    assert size(1, 2, 2, 64, 64, True) > 0
    for bad in ((-1, 1, 1, 8, 8), (10, -1, 1, 8, 8), (10, 1, 1, 129, 8), (0, 1, 1, 8, 8), (10, 0, 1, 8, 8)):
        assert size(*bad, True) == 0
    assert size(16384, 64, 16, 128, 128, True) > 1 << 32
