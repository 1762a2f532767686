"""Log-probabilities and losses where a row's own token, a gap or an address goes to its limit."""
import math

import numpy as np
import pytest
import torch

import loss_ref as R
from test_gpu_loss import Case, _close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2407_08103_amd as T
    assert torch.cuda.is_available()
    return T


def _dead_tokens(c, every):
    """-inf and NaN in turn as the logit of the token of every row but one in `every`."""
    rows = [i for i in range(c.n) if 0 <= c.t[i] < c.v and i % every]
    for k, i in enumerate(rows):
        c.x[i, int(c.t[i])] = -math.inf if k % 2 else math.nan
    c.z = c.logits.double().cpu().numpy()
    return rows


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("groups", [60, 700, 2500, 5000, 9000, 17000])
def test_gradient_in_place_of_rows_that_take_no_part(T, dtype, constrained, groups):
    """Tokens that are allowed and have logits of -inf or NaN, the gradient over the logits: such rows are zero throughout, whatever
    part of them is written first, and the others are what they are by themselves."""
    v, n = groups * (4 if dtype == "f32" else 8) + 3, 48
    c = Case(T, n, v, dtype, 41, constrained)
    dead = _dead_tokens(c, 4)
    lp64, live, logp = R.token_logprobs(c.z, c.on, c.t, 1.0)
    assert not live[dead].any() and live.any()
    rng = np.random.default_rng(groups)
    base = np.where(live, lp64, 0.0)
    old, adv = (base - 0.1).astype(np.float32), rng.normal(0, 1, size=n).astype(np.float32)
    ref = (base + rng.normal(0, 0.3, size=n)).astype(np.float32)
    ones = np.ones(n)

    def buffers():
        return c.x.clone(), torch.full((1,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")

    def check(x, lp, down, tol_down, what):
        _close(lp, lp64, R.tol_lp(lp64), what)
        g = R.gradient(logp, c.t, live, down, 1.0)
        _close(x[:, :v], g, R.tol_gradient(g, logp, c.t, live, down, tol_down, 1.0, dtype == "bf16"), what)
        assert bool((x[torch.from_numpy(~live).cuda()][:, :v] == 0).all()), what

    x, loss, lp = buffers()
    T.policy_loss(c.table, x[:, :v], c.states, c.tokens, c.f32(old), c.f32(adv), loss, lp, grad_logits=x[:, :v], ref_logprobs=c.f32(ref), kl_coef=0.1)
    want, down, size = R.policy(lp64, live, *(a.astype(np.float64) for a in (old, ref, adv)), ones, 0.2, 0.2, 0.1)
    tol = size * (R.tol_lp(lp64) + 12 * R.U)
    check(x, lp, down, tol, "policy loss")
    _close(loss, np.array([want]), np.array([tol.sum() + 2 * R.U * abs(want)]), "policy loss")

    x, _, lp = buffers()
    stats = torch.full((n, 2), 9.0, device="cuda")
    T.token_logprobs(c.table, x[:, :v], c.states, c.tokens, lp, stats=stats)
    T.token_logprobs_backward(c.table, x[:, :v], c.states, c.tokens, stats, c.f32(adv), x[:, :v])
    check(x, lp, adv.astype(np.float64), np.zeros(n), "backward")

    begin = [0, 11, 25, 40, 48]
    x, loss, lp = buffers()
    T.preference_loss(c.table, x[:, :v], c.states, c.tokens, c.f32(ref), torch.tensor(begin, dtype=torch.int32, device="cuda"), loss,
                      torch.zeros(4, device="cuda"), lp, grad_logits=x[:, :v], beta=0.5)
    want, _, down = R.preference(lp64, live, ref.astype(np.float64), begin, 0.5, 0.0)
    tol = 0.5 * np.where(live, R.tol_lp(lp64), 0.0).sum()
    check(x, lp, down, np.full(n, tol) + 2 * R.U * np.abs(down), "preference loss")
    _close(loss, np.array([want]), np.array([2 * tol + 2 * R.U * abs(want)]), "preference loss")
