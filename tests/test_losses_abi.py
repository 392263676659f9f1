"""Argument checks of the post-training entry points through the C ABI, without
a GPU: what is refused is refused before any device work."""
import ctypes

import pytest

from paper_2609_36662_gb300 import aloco as A
from paper_2609_36662_gb300 import build as B

BASE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    B.build()
    return A.load()


def _tokens(**kw):
    f = dict(logits=BASE, targets=BASE + (1 << 24), batch=2, rows=3, vocab=100, batch_stride=300,
             row_stride=100, temperature=1.0, dtype=A.F32, target_bytes=8)
    f.update(kw)
    return A.Tokens(**f)


def _policy(lib, tok=None, cfg=None, grad=None, **kw):
    at = {k: BASE + ((i + 2) << 24) for i, k in enumerate(
        ("adv", "old", "ref", "w", "terms", "logp", "scratch"))}
    at.update(kw)
    tok = tok or _tokens()
    cfg = cfg or A.PolicyCfg(0.2, 0.2, 0.0)
    return lib.aloco_policy_loss(ctypes.byref(tok), at["adv"], at["old"], at["ref"], at["w"],
                                 ctypes.byref(cfg), at["terms"], at["logp"],
                                 ctypes.byref(grad) if grad else None, at["scratch"],
                                 at.get("bytes", 1 << 16), None)


BAD_TOKENS = [dict(dtype=7), dict(target_bytes=2), dict(vocab=0), dict(vocab=A.MAX_VOCAB + 1),
              dict(batch=-1), dict(rows=-1), dict(rows=1 << 40), dict(temperature=0.0),
              dict(temperature=float("nan")), dict(temperature=1e9), dict(row_stride=99),
              dict(batch_stride=299), dict(row_stride=-100), dict(batch_stride=1 << 62),
              dict(logits=None), dict(targets=None), dict(logits=BASE + 2),
              dict(targets=BASE + (1 << 24) + 4)]


@pytest.mark.parametrize("bad", BAD_TOKENS, ids=lambda b: "-".join(f"{k}={v}" for k, v in b.items()))
def test_tokens_are_checked(lib, bad):
    tok = _tokens(**bad)
    assert lib.aloco_token_logprobs(ctypes.byref(tok), BASE + (1 << 25), None) == A.ERR_ARG
    assert A.last_error()
    assert _policy(lib, tok) == A.ERR_ARG


def test_rows_may_lie_position_by_position(lib):
    """Sequence strides below row strides are fine (the call goes on to the
    device, which is not here)."""
    for strides in ((100, 200), (300, 100), (64_000, 128)):
        tok = _tokens(batch_stride=strides[0], row_stride=strides[1])
        lib.aloco_token_logprobs(ctypes.byref(tok), BASE + (1 << 25), None)
        assert "overlap" not in A.last_error()
    tok = _tokens(batch_stride=100, row_stride=150)
    assert lib.aloco_token_logprobs(ctypes.byref(tok), BASE + (1 << 25), None) == A.ERR_ARG
    assert "overlap" in A.last_error()


def test_policy_arguments(lib):
    nan, inf = float("nan"), float("inf")
    for cfg in (A.PolicyCfg(-0.1, 0.2, 0), A.PolicyCfg(0.2, nan, 0), A.PolicyCfg(inf, 0.2, 0),
                A.PolicyCfg(0.2, 0.2, -1), A.PolicyCfg(0.2, 0.2, nan)):
        assert _policy(lib, cfg=cfg) == A.ERR_ARG
    assert _policy(lib, cfg=A.PolicyCfg(0.2, 0.2, 0.1), ref=None) == A.ERR_ARG
    for name in ("adv", "old", "w", "terms", "logp", "scratch"):
        assert _policy(lib, **{name: None}) == A.ERR_ARG and name[:3] in A.last_error()
    assert _policy(lib, bytes=lib.aloco_loss_scratch_bytes(6) - 1) == A.ERR_ARG and "scratch" in A.last_error()
    assert _policy(lib, scratch=BASE + (9 << 24) + 8) == A.ERR_ARG
    assert _policy(lib, logp=BASE) == A.ERR_ALIAS
    assert _policy(lib, terms=BASE + (7 << 24)) == A.ERR_ALIAS  # over logp
    assert _policy(lib, grad=A.LogitsGrad(None, 300, 100)) == A.ERR_ARG
    assert _policy(lib, grad=A.LogitsGrad(BASE + (1 << 30), 300, 64)) == A.ERR_ARG
    assert _policy(lib, grad=A.LogitsGrad(BASE + 400, 300, 100)) == A.ERR_ALIAS
    assert _policy(lib, grad=A.LogitsGrad(BASE, 600, 200)) == A.ERR_ALIAS
    # over the logits themselves: past the checks, as far as the device
    assert _policy(lib, grad=A.LogitsGrad(BASE, 300, 100)) in (A.ERR_CUDA, A.ERR_ARG)
    assert "overlap" not in A.last_error()


def test_preference_arguments(lib):
    def call(pairs=1, cu_bytes=8, cfg=None, cu=BASE + (3 << 24), tok=None, loss=BASE + (4 << 24)):
        cfg = cfg or A.PreferenceCfg(0.1, 0.0)
        tok = tok or _tokens()
        return lib.aloco_preference_loss(
            ctypes.byref(tok), None, cu, cu_bytes, pairs, ctypes.byref(cfg), loss,
            BASE + (5 << 24), BASE + (6 << 24), None, BASE + (7 << 24), 1 << 16, None)
    for kw in (dict(pairs=-1), dict(pairs=1 << 40), dict(cu_bytes=3), dict(cu=None),
               dict(cu=BASE + (3 << 24) + 4), dict(loss=None), dict(cfg=A.PreferenceCfg(0.0, 0.0)),
               dict(cfg=A.PreferenceCfg(float("inf"), 0.0)), dict(cfg=A.PreferenceCfg(0.1, 1.0)),
               dict(cfg=A.PreferenceCfg(0.1, float("nan")))):
        assert call(**kw) == A.ERR_ARG, kw
    assert call(loss=BASE + (6 << 24)) == A.ERR_ALIAS


def test_gradient_lists(lib):
    out = ctypes.c_void_p()

    def create(ptrs, sizes, dtypes):
        n = len(ptrs)
        return lib.aloco_grads_create((ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*sizes),
                                      (ctypes.c_int32 * n)(*dtypes), n, ctypes.byref(out))
    for ptrs, sizes, dtypes in (([None], [4], [A.F32]), ([BASE], [-1], [A.F32]),
                                ([BASE], [1 << 62], [A.F32]), ([BASE], [4], [5]),
                                ([BASE + 2], [4], [A.F32]), ([BASE + 1], [4], [A.BF16])):
        assert create(ptrs, sizes, dtypes) == A.ERR_ARG
        assert not out.value
    assert lib.aloco_grads_create(None, None, None, 1, ctypes.byref(out)) == A.ERR_ARG
    assert lib.aloco_grads_create(None, None, None, -1, ctypes.byref(out)) == A.ERR_ARG
    assert lib.aloco_grads_create(None, None, None, 0, None) == A.ERR_ARG
    assert lib.aloco_grad_norm(None, BASE, None) == A.ERR_ARG
    assert lib.aloco_clip_grads(None, 1.0, None, 0, BASE, None) == A.ERR_ARG
    lib.aloco_grads_destroy(None)


def test_scratch_sizes(lib):
    assert lib.aloco_loss_scratch_bytes(0) == 0 and lib.aloco_loss_scratch_bytes(-3) == 0
    assert lib.aloco_loss_scratch_bytes(1000) >= 12_000


def test_struct_layouts_match_c(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "probe.c"
    src.write_text(r'''
#include <stdio.h>
#include <stddef.h>
#include "aloco.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu\n", sizeof(aloco_tokens_t), sizeof(aloco_logits_grad_t),
         sizeof(aloco_policy_cfg_t), sizeof(aloco_preference_cfg_t),
         offsetof(aloco_tokens_t, temperature), offsetof(aloco_tokens_t, target_bytes),
         offsetof(aloco_logits_grad_t, row_stride));
  return 0;
}
''')
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True,
                                       check=True).stdout.split()))
    assert got == [ctypes.sizeof(A.Tokens), ctypes.sizeof(A.LogitsGrad),
                   ctypes.sizeof(A.PolicyCfg), ctypes.sizeof(A.PreferenceCfg),
                   A.Tokens.temperature.offset, A.Tokens.target_bytes.offset,
                   A.LogitsGrad.row_stride.offset]
