"""Argument checks of the token scores and of the orthogonalised updates through
the C ABI, without a GPU: what is refused is refused before any device work."""
import ctypes

import pytest

from paper_2609_36662_gb300 import aloco as A
from paper_2609_36662_gb300 import build as B

BASE = 1 << 40


def _name(kw):
    return "-".join(f"{k}={v}" if isinstance(v, (int, float, tuple, type(None))) else k
                    for k, v in kw.items())  # (no addresses: names are the same in every process)


GAP = 1 << 28


@pytest.fixture(scope="module")
def lib():
    B.build()
    return A.load()


def _at(i):
    return BASE + i * GAP


def _tokens(**kw):
    f = dict(logits=_at(0), targets=_at(1), batch=2, rows=3, vocab=100, batch_stride=300,
             row_stride=100, temperature=1.0, dtype=A.F32, target_bytes=8)
    f.update(kw)
    return A.Tokens(**f)


def _scores(lib, tok=None, top=4, **kw):
    p = dict(logp=_at(2), entropy=_at(3), ids=_at(4), best=_at(5), stats=_at(6)) | kw
    return lib.aloco_token_scores(ctypes.byref(tok or _tokens()), top, p["logp"], p["entropy"],
                                  p["ids"], p["best"], p["stats"], None)


def _grad(lib, tok=None, top=4, grad=True, **kw):
    p = dict(stats=_at(2), entropy=_at(3), d_logp=_at(4), d_entropy=_at(5), ids=_at(6),
             d_top=_at(7), data=_at(8), bs=300, rs=100) | kw
    g = ctypes.byref(A.LogitsGrad(p["data"], p["bs"], p["rs"])) if grad else None
    return lib.aloco_token_scores_grad(ctypes.byref(tok or _tokens()), p["stats"], p["entropy"],
                                       p["d_logp"], p["d_entropy"], top, p["ids"], p["d_top"], g,
                                       None)


@pytest.mark.parametrize("kw", [dict(top=-1), dict(top=33), dict(top=101), dict(logp=None),
                                dict(ids=None), dict(best=None), dict(stats=_at(6) + 4),
                                dict(entropy=_at(3) + 2),
                                dict(tok=_tokens(vocab=3, row_stride=3, batch_stride=9)),
                                dict(tok=_tokens(temperature=0.0)), dict(tok=_tokens(dtype=3)),
                                dict(tok=_tokens(row_stride=99))], ids=_name)
def test_scores_refuse(lib, kw):
    assert _scores(lib, **kw) == A.ERR_ARG and A.last_error()


@pytest.mark.parametrize("kw", [dict(top=-1), dict(top=33), dict(grad=False), dict(stats=None),
                                dict(entropy=None), dict(ids=None), dict(data=None),
                                dict(rs=99), dict(stats=_at(2) + 4), dict(d_logp=_at(4) + 1)],
                         ids=_name)
def test_scores_gradients_refuse(lib, kw):
    assert _grad(lib, **kw) == A.ERR_ARG and A.last_error()


def test_scores_refuse_outputs_that_overlap(lib):
    assert _scores(lib, logp=_at(0)) == A.ERR_ALIAS
    assert _scores(lib, best=_at(4) + 16) == A.ERR_ALIAS
    assert _grad(lib, data=_at(0) + 4) == A.ERR_ALIAS
    assert _grad(lib, data=_at(2)) == A.ERR_ALIAS


def test_scores_of_no_rows(lib):
    assert _scores(lib, tok=_tokens(rows=0)) == A.OK
    assert _grad(lib, tok=_tokens(batch=0)) == A.OK


def _matrices(parts):
    return (A.Matrix * len(parts))(*parts)


def _muon(lib, parts=((0, 10, 20), (300, 30, 5), (500, 130, 140)), N=20000, M=2, cfg=None, pdt=A.F32, gdt=A.BF16,
          scratch=_at(20), bytes_=None, x=None, g=None, b=None):
    mats = _matrices(parts)
    vec = ctypes.c_void_p * 64
    x = x or vec(*[_at(i) for i in range(1, 1 + max(M, 1))])
    g = g or vec(*[_at(40 + i) for i in range(max(M, 1))])
    b = b or vec(*[_at(80 + i) for i in range(max(M, 1))])
    need = lib.aloco_muon_scratch_bytes(mats, len(parts), M) if bytes_ is None else bytes_
    return lib.aloco_muon_step(x, g, b, N, M, pdt, gdt, mats, len(parts),
                               ctypes.byref(cfg or A.muon_cfg()), scratch, need, None)


BAD_MUON = [dict(M=0), dict(M=33), dict(pdt=5), dict(gdt=-1), dict(N=18699),
            dict(parts=((-1, 2, 2),)), dict(parts=((0, -2, 2),)),
            dict(parts=((0, 2, A.MAX_LONG_SIDE + 1),), N=1 << 40),
            dict(parts=((0, A.MAX_SIDE + 1, A.MAX_SIDE + 1),), N=1 << 40),
            dict(scratch=None), dict(scratch=_at(20) + 16), dict(bytes_=100), dict(N=1 << 62)]


@pytest.mark.parametrize("kw", BAD_MUON, ids=_name)
def test_steps_refuse(lib, kw):
    assert _muon(lib, **kw) == A.ERR_ARG and A.last_error()


@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(lr=float("nan")), dict(momentum=1.0),
                                dict(momentum=-0.1), dict(weight_decay=-1.0), dict(eps=0.0),
                                dict(eps=float("inf")), dict(nesterov=2), dict(scale=3),
                                dict(steps=0), dict(steps=17),
                                dict(coefficients=[(101.0, 0, 0)]),
                                dict(coefficients=[(float("nan"), 0, 0)])], ids=_name)
def test_steps_refuse_settings(lib, kw):
    assert _muon(lib, cfg=A.muon_cfg(**kw)) == A.ERR_ARG and A.last_error()


def test_steps_refuse_what_overlaps(lib):
    assert _muon(lib, parts=((0, 10, 20), (199, 3, 3))) == A.ERR_ALIAS
    assert _muon(lib, parts=((50, 3, 3), (0, 10, 20))) == A.ERR_ALIAS
    vec = ctypes.c_void_p * 64
    assert _muon(lib, x=vec(_at(1), _at(1) + 2000)) == A.ERR_ALIAS
    assert _muon(lib, b=vec(_at(1), _at(9))) == A.ERR_ALIAS
    assert _muon(lib, g=vec(_at(20), _at(9))) == A.ERR_ALIAS


def test_no_matrices_is_no_work(lib):
    assert _muon(lib, parts=()) == A.OK
    assert _muon(lib, parts=((5, 0, 7), (20000, 3, 0))) == A.OK


def test_settings_by_name():
    with pytest.raises(TypeError):
        A.muon_cfg(learning_rate=1.0)
    with pytest.raises(ValueError):
        A.muon_cfg(coefficients=[])
    with pytest.raises(ValueError):
        A.muon_cfg(coefficients=[(1.0, 2.0)])
    with pytest.raises(TypeError):
        A.Matrices([(0, 2.5, 4)])
    assert list(A.muon_cfg(steps=16).coefficients[15]) == list(A.NEWTON_SCHULZ)
    c = A.muon_cfg(coefficients=[(1.5, -0.5, 0.0)] * 3, lr=0.1)
    assert c.steps == 3 and list(c.coefficients[2]) == [1.5, -0.5, 0.0] and c.lr == 0.1


def test_scratch_is_bounded(lib):
    """Scratch grows with the matrices up to a pass's, never beyond what its
    largest matrix needs."""
    assert lib.aloco_muon_scratch_bytes(_matrices([(0, 64, 64)]), 1, 1) == 0
    assert 0 < lib.aloco_muon_scratch_bytes(_matrices([(0, 129, 129)]), 1, 1) < 1 << 20
    many = [(i * 2048 * 5632, 2048, 5632) for i in range(60)]
    assert lib.aloco_muon_scratch_bytes(_matrices(many), 60, 8) <= 3 << 30
    assert lib.aloco_muon_scratch_bytes(_matrices(many), 60, 0) == 0
    assert lib.aloco_orthogonalize_scratch_bytes(0, 4, 4) == 0
    assert lib.aloco_orthogonalize_scratch_bytes(1, A.MAX_SIDE + 1, A.MAX_SIDE + 1) == 0


def _ortho(lib, **kw):
    p = dict(x=_at(1), batch=2, rows=130, cols=140, bs=18200, rs=140, dtype=A.F32, out=_at(2), steps=5,
             eps=1e-7, scratch=_at(3), bytes=1 << 24, coefficients=True) | kw
    co = (ctypes.c_double * 48)(*([1.5, -0.5, 0.0] * 16)) if p["coefficients"] else None
    return lib.aloco_orthogonalize(p["x"], p["batch"], p["rows"], p["cols"], p["bs"], p["rs"],
                                   p["dtype"], p["out"], co, p["steps"], p["eps"], p["scratch"],
                                   p["bytes"], None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(batch=-1), dict(rows=-1), dict(rs=-1),
                                dict(bs=-140), dict(bs=1 << 62), dict(steps=0), dict(steps=17), dict(eps=0.0),
                                dict(coefficients=False), dict(scratch=None), dict(bytes=1),
                                dict(x=None), dict(out=None), dict(out=_at(2) + 1),
                                dict(rows=A.MAX_SIDE + 1, cols=A.MAX_SIDE + 1, rs=1 << 20)],
                         ids=_name)
def test_factors_refuse(lib, kw):
    assert _ortho(lib, **kw) == A.ERR_ARG and A.last_error()


def test_factors_refuse_what_overlaps(lib):
    assert _ortho(lib, out=_at(1) + 40) == A.ERR_ALIAS
    assert _ortho(lib, scratch=_at(1)) == A.ERR_ALIAS


def test_factors_of_nothing(lib):
    assert _ortho(lib, batch=0) == A.OK and _ortho(lib, rows=0) == A.OK
