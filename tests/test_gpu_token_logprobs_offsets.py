"""Log probabilities of logits with a large common offset, which the definition cancels."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [0.0, 1000.0, -4096.5, 3.0e5])
@pytest.mark.parametrize("T,V", [(1, 1000), (5, 4099), (600, 515), (2, 300007)])
@pytest.mark.parametrize("top", [0, 7])
def test_an_offset_costs_no_digits(rq, ctx, T, V, offset, top):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn((T, V), generator=g, device="cuda") * 3 + offset
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    r = rq.token_logprobs(ctx, z, y, top=top, entropy=True)
    want = ref.logprobs(z, y, top)
    # z - max: one rounding of at most |logp| + log S; log S: the sum's float32 error and its own rounding, log S <= log V
    sums = (V / 256 + 64) * ref.F

    def bound(logp):
        return sums + 4 * ref.F * (logp.abs() + math.log(V))
    ref.close(r.logp, want["logp"], bound(want["logp"]), "logp")
    ref.close(r.lse, want["lse"], sums + 4 * ref.F * (want["lse"].abs() + math.log(V)), "lse")
    if top:
        assert torch.equal(r.top_ids, want["top_ids"])
        ref.close(r.top_logp, want["top_logp"], bound(want["top_logp"]), "top_logp")
