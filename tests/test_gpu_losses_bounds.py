"""What the post-training losses write around their outputs: nothing."""
import ctypes

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu


def _inputs(n, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(n, V, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    f = lambda s: torch.randn(n, generator=g, device="cuda") * s
    return x, t, f(1.0), f(0.1) - 10.0, torch.full((n,), 1.0 / n, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(1, 300), (5, 5003), (3, 128256), (300, 40)])
def test_nothing_is_written_around_the_outputs(n, V, dtype):
    """Outputs and scratch of exactly the sizes asked for, between sentinels."""
    x, t, adv, old, w = _inputs(n, V, dtype, 9)
    lib = A.load()
    need = lib.aloco_loss_scratch_bytes(n)
    word = need // 4
    sizes = {"terms": 4, "logp": n, "scratch": word, "loss": 1, "ratios": 2}
    big = {k: torch.full((m + 128,), -7.25, device="cuda") for k, m in sizes.items()}
    at = {k: v[64:64 + sizes[k]].data_ptr() for k, v in big.items()}
    grad = torch.full((n * V + 64,), -7.25, dtype=dtype, device="cuda")
    g = A.LogitsGrad(grad[32:].data_ptr(), 0, V)
    tok = A._tokens(x, t, 1.0)
    cfg, pcfg = A.PolicyCfg(0.2, 0.2, 0.1), A.PreferenceCfg(0.1, 0.1)
    opts = A.Opts(stream=torch.cuda.current_stream().cuda_stream)
    r = ctypes.byref
    assert lib.aloco_policy_loss(r(tok), adv.data_ptr(), old.data_ptr(), old.data_ptr(), w.data_ptr(),
                                 r(cfg), at["terms"], at["logp"], r(g), at["scratch"], need,
                                 r(opts)) == A.OK
    cu = torch.tensor([0, n // 2, n], device="cuda")
    assert lib.aloco_preference_loss(r(tok), old.data_ptr(), cu.data_ptr(), 8, 1, r(pcfg), at["loss"],
                                     at["ratios"], at["logp"], r(g), at["scratch"], need,
                                     r(opts)) == A.OK
    assert lib.aloco_token_logprobs(r(tok), at["logp"], r(opts)) == A.OK
    torch.cuda.synchronize()
    for k, v in big.items():
        assert bool((v[:64] == -7.25).all()) and bool((v[64 + sizes[k]:] == -7.25).all()), k
    assert bool((grad[:32] == -7.25).all()) and bool((grad[32 + n * V:] == -7.25).all())
