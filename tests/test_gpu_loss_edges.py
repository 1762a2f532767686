"""Log-probabilities and losses where a row's own token, a gap or an address goes to its limit."""
import math
import types

import numpy as np
import pytest
import torch

import loss_ref as R
from test_gpu_loss import TYPES, Case, _close, _run_preference

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


def _all_gradients(T, c, temperature, down, old=None):
    """[(what, lp, gradient, d loss / d lp)] of every call that writes a gradient, with a slope of `down` for every row."""
    n, v, out = c.n, c.v, []
    lp, stats, g = torch.full((n,), 9.0, device="cuda"), torch.full((n, 2), 9.0, device="cuda"), torch.full_like(c.x, 7.0)
    T.token_logprobs(*c.args(), lp, temperature=temperature, stats=stats)
    T.token_logprobs_backward(*c.args(), stats, torch.full((n,), down, device="cuda"), g[:, :v], temperature=temperature)
    out.append(("backward", lp, g[:, :v], np.full(n, down)))
    # the ratio is 1 where the old log-probability is lp, and nothing is clipped
    lp2, g, loss = torch.full((n,), 9.0, device="cuda"), torch.full_like(c.x, 7.0), torch.zeros(1, device="cuda")
    T.policy_loss(*c.args(), lp, torch.full((n,), -down, device="cuda"), loss, lp2, grad_logits=g[:, :v], temperature=temperature, clip=(1.0, math.inf))
    out.append(("policy loss", lp2, g[:, :v], np.full(n, down)))
    # rows against an empty sequence each, rewards of zero: every slope is -beta / (2 pairs)
    begin = torch.from_numpy(np.repeat(np.arange(n + 1), 2)[1:].astype(np.int32)).cuda()
    lp3, g, rewards = torch.full((n,), 9.0, device="cuda"), torch.full_like(c.x, 7.0), torch.zeros(2 * n, device="cuda")
    T.preference_loss(*c.args(), lp, begin, loss, rewards, lp3, grad_logits=g[:, :v], temperature=temperature, beta=2.0 * n * abs(down))
    out.append(("preference loss", lp3, g[:, :v], np.full(n, -abs(down))))
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("n,v", [(6, 67), (6, 4099), (40, 9001), (6, 40001), (40, 70003), (6, 140003)])
def test_own_element_of_a_likely_token(T, dtype, constrained, n, v):
    """1 - p_t relative to itself, with p_t down to some 10^-6 below 1 and logits at which a folded exponent has few bits left; the token
    in the first and the last group and behind it; a NaN among the logits of some rows."""
    for logit, temperature in ((3.0, 1.0), (30.0, 1.0), (200.0, 1.0), (600.0, 1.0), (30.0, 0.1)):
        c = Case(T, n, v, dtype, 42, constrained)
        rng = np.random.default_rng([v, int(logit)])
        x = c.x.float()
        x[:, :v] = logit - temperature * (12.0 + math.log(v / 512) + 3.0 * torch.rand((n, v), device="cuda", generator=torch.Generator("cuda").manual_seed(v)))
        allowed = [np.flatnonzero(c.on[i]) for i in range(n)]
        for i in range(n):
            if len(allowed[i]):
                c.t[i] = allowed[i][[0, -1, len(allowed[i]) // 2][i % 3]] if len(allowed[i]) > 1 or i % 2 else allowed[i][0]
                x[i, int(c.t[i])] = logit
                other = int(rng.choice(allowed[i]))
                if i % 4 == 3 and other != c.t[i]:
                    x[i, other] = math.nan
            else:
                c.t[i] = -1
        c.tokens = torch.from_numpy(c.t.astype(np.int32)).cuda()
        c.x = x.to(c.x.dtype)
        c.logits = c.x[:, :v]
        c.z = c.logits.double().cpu().numpy()
        _, live, logp = R.token_logprobs(c.z, c.on, c.t, temperature)
        at = np.where(live, c.t, 0)
        p = np.exp(np.where(np.isnan(logp), -np.inf, logp))
        rows = np.arange(n)
        others = p.copy()
        others[rows, at] = 0.0
        rest = others.sum(axis=1)
        assert live.any() and rest[live].max() < 0.1
        for what, lp, g, down in _all_gradients(T, c, temperature, 1 / 3):
            scale = np.where(live, down / temperature, 0.0)
            g = g.double().cpu().numpy()
            # a sum of others is off by REL_SUM of itself at most; exponents of some |x| = 30 in binary32 add 3 u |x|, the inverse
            # temperature, d and the two functions of it a few u; then the rounding to the gradient's type
            rel = R.REL_SUM + 128 * R.U + (2.0 ** -8 if dtype == "bf16" else 2 * R.U)
            want = scale * rest
            off = np.abs(g[rows, at] - want)
            assert (off[live] <= rel * np.abs(want[live])).all(), (what, logit, float((off / np.abs(want))[live].max()))
            assert (off[live & (rest == 0)] == 0).all()
            want = -scale[:, None] * others
            g[rows[live], at[live]] = 0.0
            # a folded exponent is off by some 2^-14 of p in 16 bits
            assert (np.abs(g - want) <= (rel + 2.0 ** -13) * np.abs(want) + 1e-37).all(), (what, logit)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(5, 40), (70, 515), (70, 9000), (5, 40001), (5, 140003)])
def test_forced_tokens_have_no_gradient(T, dtype, n, v):
    """In a state that allows one token its log-probability and the whole gradient are zero, not a rounding of them."""
    c = Case(T, n, v, dtype, 43)
    only = int(torch.nonzero(c.delta[2] >= 0)[0, 0])
    assert int((c.delta[2] >= 0).sum()) == 1
    c.states[:] = 2
    c.tokens[:] = only
    for k, sigma in enumerate((1.0, 100.0)):
        c.x[:, :v] = (c.x[:, :v].float() * sigma).to(c.x.dtype)
        for temperature in (1.0, 0.7):
            for what, lp, g, _ in _all_gradients(T, c, temperature, 1 / 3):
                assert bool((lp == 0).all()), (what, lp)
                assert bool((g == 0).all()), (what, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(200, 515), (200, 5000), (20, 32003), (200, 32003), (100, 70003), (400, 70003)])
def test_unlikely_tokens(T, dtype, n, v):
    """Tokens up to 80 below the largest logit: neither log-probabilities nor the gradients of the likely tokens lose bits by it."""
    for far in (0, 10, 25, 80):
        c = Case(T, n, v, dtype, 44, constrained=False)
        c.t = np.arange(n) * 7 % v
        c.tokens = torch.from_numpy(c.t.astype(np.int32)).cuda()
        at = c.tokens.long()[:, None]
        x = c.logits.float()
        c.logits.scatter_(1, at, (x.amax(1, keepdim=True) - far).to(c.x.dtype))
        logp = torch.log_softmax(c.logits.double(), dim=1)
        lp64 = logp.gather(1, at)[:, 0]
        top = c.logits.double().amax(1)
        ls = torch.logsumexp(c.logits.double(), 1) - top
        likely = logp.scatter(1, at, -math.inf).topk(20, dim=1).indices
        below = float((top[:, None] - c.logits.double().gather(1, likely)).max())
        drawn = None
        for what, lp, g, down in _all_gradients(T, c, 1.0, 0.5 / n):
            down = torch.from_numpy(down).cuda()
            if what == "preference loss":        # beta is 1, and the reference the first call's lp as it was rounded to binary32
                down = -1.0 / n / (1.0 + torch.exp(lp64 - drawn.double()))
            drawn = lp if drawn is None else drawn
            # lp is rounded once to binary32; the logarithm, and sums whose roundings have no common sign, add some u.  In 16 bits the
            # exponents are relative to the token and off by u of their size, up to |lp|, as well
            bound = R.U * (lp64.abs() * (1 if dtype == "f32" else 3) + 8)
            off = (lp.double() - lp64).abs()
            assert bool((off <= bound).all()), (what, far, float((off / bound).max()))
            if dtype == "f32":
                # ln s is rounded to binary32, the exponents are off by 2 u of their size, the functions and products by a few u; the
                # slope of a preference loss follows the 8 u of lp with at most half of them and has an exponential of its own
                bound = R.U * (float(ls.max()) + 2 * below + 8 + (8 if what == "preference loss" else 0))
                off = (g.double().gather(1, likely) / (-down[:, None] * logp.exp().gather(1, likely)) - 1).abs()
                assert bool((off <= bound).all()), (what, far, float((off / bound).max()))
                assert float(off.square().mean().sqrt()) <= bound / 2, (what, far, float(off.square().mean().sqrt()) / R.U)


@pytest.mark.parametrize("pairs", [4, 70])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_infinite_gaps(T, pairs, grad, smoothing):
    """A reference that gives a token probability zero has -inf there: the pair's gap is infinite, its loss the limit (0 on the side of
    weight zero), its slopes finite, and the other pairs' are what they are by themselves; rewards of inf - inf stay NaN."""
    n, v = 2 * pairs, 64
    c = Case(T, n, v, "f32", 45, constrained=False)
    c.t = np.arange(n) % v
    c.tokens = torch.from_numpy(c.t.astype(np.int32)).cuda()
    lp64, live, logp = R.token_logprobs(c.z, c.on, c.t, 1.0)
    begin = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    for at, both in (([0], False), ([3], False), ([0, 3], False), ([4, 5], True)):
        ref = lp64 + c.rng.normal(0, 0.3, size=n)
        ref = ref.astype(np.float32)
        ref[at] = -math.inf
        loss, rewards, lp = torch.full((1,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        g = torch.full_like(c.x, 7.0)
        T.preference_loss(None, c.logits, None, c.tokens, c.f32(ref), begin, loss, rewards, lp, grad_logits=g[:, :v] if grad else None, beta=0.5,
                          smoothing=smoothing)
        reward = 0.5 * (lp64 - ref.astype(np.float64))
        assert np.array_equal(np.isinf(rewards.cpu().numpy()), np.isinf(reward))
        with np.errstate(invalid="ignore"):
            gap = reward[0::2] - reward[1::2]
        if both:
            assert math.isnan(float(loss))
            continue
        each = sum((w * np.logaddexp(0.0, s * gap) for w, s in ((1.0 - smoothing, -1.0), (smoothing, 1.0)) if w), np.zeros(pairs))
        want = float(each.mean())
        tol = 0.0 if math.isinf(want) else float(R.tol_lp(lp64).max()) + 4 * R.U * abs(want)
        _close(loss, np.array([want]), np.array([tol]), "loss")
        if grad:
            with np.errstate(over="ignore"):
                slope = (smoothing / (1.0 + np.exp(-gap)) - (1.0 - smoothing) / (1.0 + np.exp(gap))) * 0.5 / pairs
            down = np.stack([slope, -slope], 1).reshape(-1)
            want = R.gradient(logp, c.t, live, down, 1.0)
            _close(g[:, :v], want, R.tol_gradient(want, logp, c.t, live, down, np.abs(down) * 8 * R.U + 0.5 / pairs * R.tol_lp(lp64), 1.0, False), "gradient")


def test_gradient_rows_between_the_logits_rows(T):
    """One buffer for both, row by row beside one another or one behind the other, is no overlap; rows that share an element are."""
    c = Case(T, 6, 200, "bf16", 46)
    lp, stats, d = torch.zeros(6, device="cuda"), torch.zeros((6, 2), device="cuda"), torch.ones(6, device="cuda")
    want = torch.zeros_like(c.x)
    T.token_logprobs(*c.args(), lp, stats=stats)
    T.token_logprobs_backward(*c.args(), stats, d, want[:, :200])
    buf = torch.empty((14, 464), dtype=torch.bfloat16, device="cuda")

    def run(x, g):
        buf.fill_(5.0)
        x.copy_(c.logits)
        T.token_logprobs_backward(c.table, x, c.states, c.tokens, stats, d, g)
        assert torch.equal(g, want[:, :200]) and torch.equal(x, c.logits)
        kept = buf.clone()
        for part in (x, g):
            torch.as_strided(kept, part.shape, part.stride(), part.storage_offset()).fill_(5.0)
        assert bool((kept == 5.0).all())

    for first, second in ((0, 200), (200, 0), (8, 256), (264, 0)):
        run(buf[:6, first:first + 200], buf[:6, second:second + 200])
        run(buf[:6, first:first + 200], buf[8:14, second:second + 200])
        run(buf[4:10, first:first + 200], buf[:6, second:second + 200])
    run(buf[:6, :200], buf[6:12, :200])                              # behind the last row
    run(buf[:6, 264:], buf[7:13, :200])
    x = buf[:6, :200]
    for g in (buf[:6, 192:392], buf[1:7, :200], buf[5:11, 8:208]):
        for a, b in ((x, g), (g, x)):
            with pytest.raises(T.TdfaError, match="overlaps"):
                T.token_logprobs_backward(c.table, a, c.states, c.tokens, stats, d, b)
    flat = buf.view(-1)
    far, near = torch.as_strided(flat, (6, 200), (464, 1)), torch.as_strided(flat, (6, 200), (464, 1), 272)       # 272 + 200 > 464
    for a, b in ((far, near), (near, far), (far, torch.as_strided(flat, (6, 200), (472, 1), 208))):               # (another stride between the rows)
        with pytest.raises(T.TdfaError, match="overlaps"):
            T.token_logprobs_backward(c.table, a, c.states, c.tokens, stats, d, b)


def _stream_forms(stream):
    return {"stream": stream, "handle": stream.cuda_stream, "object with a handle": types.SimpleNamespace(cuda_stream=stream.cuda_stream)}


@pytest.mark.parametrize("form", ["stream", "handle", "object with a handle", "default handle"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_on_another_stream(T, form, dtype):
    """All calls on a stream of the caller's, with workspaces from torch on that stream: scoring of rows that want one, both losses, and the
    gradient from statistics; the same bits as on the current stream."""
    c = Case(T, 20, 70003 if dtype == "f32" else 140003, dtype, 47)
    n, v = c.n, c.v
    begin, ones = torch.tensor([0, 5, 9, 14, 20], dtype=torch.int32, device="cuda"), torch.ones(n, device="cuda")
    side = torch.cuda.current_stream() if form == "default handle" else torch.cuda.Stream()
    given = side.cuda_stream if form == "default handle" else _stream_forms(side)[form]

    def run(stream):
        out = [torch.full((n,), 9.0, device="cuda"), torch.full((n, 2), 9.0, device="cuda"), torch.full_like(c.x, 7.0), torch.full((1,), 9.0, device="cuda"),
               torch.full((n,), 9.0, device="cuda"), torch.full_like(c.x, 7.0), torch.full((1,), 9.0, device="cuda"), torch.full((4,), 9.0, device="cuda"),
               torch.full((n,), 9.0, device="cuda"), torch.full_like(c.x, 7.0)]
        lp, stats, g, loss, lp2, g2, loss2, rewards, lp3, g3 = out
        side.wait_stream(torch.cuda.current_stream())
        T.token_logprobs(*c.args(), lp, stats=stats, stream=stream)
        T.token_logprobs_backward(*c.args(), stats, ones, g[:, :v], stream=stream)
        T.policy_loss(*c.args(), ones, ones, loss, lp2, grad_logits=g2[:, :v], ref_logprobs=ones, kl_coef=0.0, stream=stream)
        T.preference_loss(*c.args(), ones, begin, loss2, rewards, lp3, grad_logits=g3[:, :v], stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        return out

    want, got = run(None), run(given)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert bool(torch.isfinite(got[3]).all()) and not bool((got[0] == 9.0).any())


@pytest.mark.parametrize("n,v", [(6, 515), (40, 9001), (40, 70003)])
def test_folded_exponents_at_their_largest(T, n, v):
    """16-bit gradients of logits between 512 and 1,023 in units of the exponent, with slopes down to 10^-30."""
    for sign, far in ((1.0, 0.0), (-1.0, 0.0), (1.0, 60.0), (-1.0, 60.0)):
        c = Case(T, n, v, "bf16", 48, constrained=False)
        g = torch.Generator("cuda").manual_seed(v)
        level = torch.linspace(380.0, 690.0 if sign > 0 else 690.0 - far, n, device="cuda")[:, None]
        x = sign * level + 8.0 * torch.rand((n, v), device="cuda", generator=g)
        c.t = np.arange(n) * 11 % v
        at = torch.from_numpy(c.t).cuda()[:, None]
        x.scatter_(1, at, x.amax(1, keepdim=True) - far)
        c.x[:, :v] = x.to(c.x.dtype)
        c.tokens = at[:, 0].int()
        z2 = (c.logits.float().gather(1, at).abs() * 1.4427).cpu().numpy()
        assert (z2 < 1024).all() and z2.max() > 870 and z2.min() > 450
        p = torch.softmax(c.logits.double(), dim=1)
        for down in (1.0, -1e-10, 1e-30):
            lp, stats, got = torch.zeros(n, device="cuda"), torch.zeros((n, 2), device="cuda"), torch.zeros_like(c.x)
            T.token_logprobs(*c.args(), lp, stats=stats)
            T.token_logprobs_backward(*c.args(), stats, torch.full((n,), down, device="cuda"), got[:, :v])
            want = (-down * p).scatter(1, at, 0.0)
            want.scatter_(1, at, -want.sum(1, keepdim=True))
            # exponents off by 2^-15 + 2^-14 + 2^-17 (the difference itself), sums by REL_SUM and what their own exponents lose, 3 u 2^7;
            # a result below the normal numbers is off by half of the smallest
            rel = 2.0 ** -8 + 1.02 * math.log(2) * (2.0 ** -15 + 2.0 ** -14 + 2.0 ** -17) + 2 * R.REL_SUM + 384 * R.U
            off = (got[:, :v].double() - want).abs()
            assert bool((off <= rel * want.abs() + 1.2e-38).all()), (sign, far, down, float((off / want.abs().clamp(min=1e-37)).max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,pairs", [(256, 1), (257, 1), (512, 2), (513, 2), (1000, 1), (1024, 64), (1025, 64), (1000, 65)])
def test_preference_pairs_of_any_length(T, dtype, n, pairs):
    """Around the numbers of rows and pairs at which the launch between scores and gradients is left out; one pair holds most rows."""
    cut = sorted({0, n, *range(n - 2 * pairs + 1, n)})
    cut = [0] * (2 * pairs + 1 - len(cut)) + cut
    _run_preference(T, Case(T, n, 515, dtype, 49), 1.0, 0.2, 0.1, cut)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,groups", [(64, 16400), (65, 16400), (256, 16400), (257, 16400), (100, 49152), (100, 49153)])
def test_long_rows_around_their_parts(T, dtype, n, groups):
    """Around the numbers of long rows that are shared out by parts, by scoring with its gradient and by the losses."""
    v = groups * (4 if dtype == "f32" else 8) + 1
    g = torch.Generator("cuda").manual_seed(n)
    x = (2.0 * torch.randn(n, -(-v // 8) * 8, device="cuda", generator=g)).to(TYPES[dtype])
    tokens = torch.randint(0, v, (n,), device="cuda", generator=g, dtype=torch.int32)
    at = tokens.long()[:, None]
    lp64 = torch.cat([torch.log_softmax(x[i:i + 32, :v].double(), dim=1).gather(1, at[i:i + 32]) for i in range(0, n, 32)])[:, 0]
    lp, stats, lp2, lp3 = torch.zeros(n, device="cuda"), torch.zeros((n, 2), device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    T.token_logprobs(None, x[:, :v], None, tokens, lp, stats=stats)
    bound = R.U * (3 * lp64.abs() + 8)
    assert bool(((lp.double() - lp64).abs() <= bound).all())
    down, loss, grads = torch.full((n,), 0.5, device="cuda"), torch.zeros(1, device="cuda"), [torch.zeros_like(x) for _ in range(2)]
    T.token_logprobs_backward(None, x[:, :v], None, tokens, stats, down, grads[0][:, :v])
    T.policy_loss(None, x[:, :v], None, tokens, lp, -down, loss, lp2, grad_logits=grads[1][:, :v], clip=(1.0, math.inf))
    T.preference_loss(None, x[:, :v], None, tokens, lp, torch.tensor([0, n, n], dtype=torch.int32, device="cuda"), loss, torch.zeros(2, device="cuda"), lp3)
    for other in (lp2, lp3):
        assert bool(((other.double() - lp64).abs() <= bound).all())
    for i in range(0, n, 32):
        p = torch.softmax(x[i:i + 32, :v].double(), dim=1)
        want = (-0.5 * p).scatter(1, at[i:i + 32], 0.0)
        want.scatter_(1, at[i:i + 32], -want.sum(1, keepdim=True))
        for got in grads:
            # exponents of some 20, off by 3 u of their size, a folded one by 2^-13.8 of p in 16 bits, and the rounding to the type
            rel = 2 * R.REL_SUM + 64 * R.U + (2.0 ** -8 + 2.0 ** -13.7 if dtype == "bf16" else 2 * R.U)
            assert bool(((got[i:i + 32, :v].double() - want).abs() <= rel * want.abs() + 1.2e-38).all())


def test_states_without_a_table_are_not_read(T):
    """So that log-probabilities may be written over them."""
    x, tokens = torch.randn(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    f, loss, rewards = torch.ones(4, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
    want, states = torch.zeros(4, device="cuda"), torch.full((4,), 9, dtype=torch.int32, device="cuda")
    T.token_logprobs(None, x, None, tokens, want)
    T.policy_loss(None, x, states, tokens, f, f, loss, states.view(torch.float32))
    assert torch.equal(states.view(torch.float32), want)
    states.fill_(9)
    T.preference_loss(None, x, states, tokens, f, torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), loss, rewards, states.view(torch.float32))
    assert torch.equal(states.view(torch.float32), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_tokens(T, dtype):
    """A vocabulary of no tokens: no row takes part, and nothing is written behind it."""
    x = torch.full((5, 64), 3.0, dtype=TYPES[dtype], device="cuda")
    tokens = torch.tensor([-1, 0, 3, -1, -7], dtype=torch.int32, device="cuda")
    f, loss, rewards = torch.ones(5, device="cuda"), torch.full((1,), 9.0, device="cuda"), torch.full((2,), 9.0, device="cuda")
    want = [0.0, -math.inf, -math.inf, 0.0, -math.inf]
    lp, stats = torch.full((5,), 9.0, device="cuda"), torch.full((5, 2), 9.0, device="cuda")
    T.token_logprobs(None, x[:, :0], None, tokens, lp, stats=stats)
    assert lp.tolist() == want and stats.tolist() == [[0.0, math.inf]] * 5
    T.token_logprobs_backward(None, x[:, :0], None, tokens, stats, f, x[:, :0])
    for grad in (None, x[:, :0]):
        lp.fill_(9.0)
        T.policy_loss(None, x[:, :0], None, tokens, f, f, loss, lp, grad_logits=grad)
        assert lp.tolist() == want and float(loss) == 0.0
        lp.fill_(9.0)
        T.preference_loss(None, x[:, :0], None, tokens, f, torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda"), loss, rewards, lp, grad_logits=grad)
        assert lp.tolist() == want and rewards.tolist() == [0.0, 0.0] and abs(float(loss) - math.log(2.0)) < 1e-6
    assert bool((x == 3.0).all())
