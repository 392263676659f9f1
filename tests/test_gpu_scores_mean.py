"""Log-probabilities of many rows have no error in common: log ratios of hundreds of
tokens are sums of them.

The rows have one largest value and V others some 10 below, with 1.3 times its
weight together: log2(e) / tau in one float (off by up to 2^-24 of itself, 5e-8 at
these temperatures) puts that of all their powers on the sum, 5e-8 * 10 * 1.3 / 2.3 =
2.8e-7 on every row's log-probability.  What may remain on average is the logarithm's
error, one ulp at most (2^-24 between 1/2 and 1).  A row's own roundings (some
additions on its way, the division: 6 of 2^-24 at most, without a common sign) have a
standard deviation of at most 2^-24 * sqrt(6) * 0.58 = 0.85e-7; 5 of these over
sqrt(rows) are allowed.  The largest values lie anywhere between powers of two, so
that what 2^t is off there averages out too."""
import math

import pytest
import torch

from paper_2609_36662_gb300 import aloco as A

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("temp", [0.69, 1.25, 2.79])
@pytest.mark.parametrize("rows,v,dtype", [(1300, 32000, F32), (400, 32000, F32), (1300, 8192, BF16),
                                          (1300, 32000, BF16)],
                         ids=["ctas", "clusters", "warps", "ctas_bf16"])
def test_no_error_in_common(rows, v, dtype, temp):
    gen = torch.Generator("cuda").manual_seed(v)
    # the mean of exp(u), u uniform in [-1, 1], is sinh(1)
    down = math.log(v * math.sinh(1) / 1.3)
    y = torch.empty(rows, v, device="cuda").uniform_(-1, 1, generator=gen) - down
    t = torch.randint(0, v, (rows,), generator=gen, device="cuda")
    y.scatter_(1, t[:, None], 0.0)
    x = ((y + torch.empty(rows, 1, device="cuda").uniform_(-8, 8, generator=gen)) * temp).to(dtype)
    want = torch.log_softmax(x.double() / temp, -1).gather(1, t[:, None])[:, 0]
    r = A.token_scores(x, t, temperature=temp, top=2)
    for logp in (r.logp, r.top_logp[:, 0]):
        assert abs(float((logp - want).mean())) <= 2.0**-24 + 5 * 0.85e-7 / math.sqrt(rows)
