"""Log-probabilities, policy loss and preference loss against their plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

import gpu_util as G
import loss_ref as R

pytestmark = pytest.mark.gpu
DEAD = NO_TOKEN = -1
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def T():
    import paper_2407_08103_amd as T
    assert torch.cuda.is_available()
    return T


class Case:
    """Rows with a token each under a random constraint.  States: 0 wide, 1 sparse, 2 one token, 3 nothing, 4 all."""

    def __init__(self, T, n, v, dtype, seed, constrained=True, pad=64, special=False, kind="wrapped", sigma=2.0):
        rng = np.random.default_rng([n, v, seed])
        self.n, self.v, self.dtype = n, v, dtype
        stride = -(-max(v, 1) // pad) * pad
        x = (rng.normal(0, sigma, size=(n, stride))).astype(np.float32)
        self.table, self.states, allow = None, None, np.ones((n, v), dtype=bool)
        on = np.zeros((5, v), dtype=bool)
        if v:
            on[0] = rng.random(v) < 0.7
            on[1] = rng.random(v) < min(1.0, 6.0 / v)
            on[2, rng.integers(0, v)] = True
            on[4] = True
            on[1, rng.integers(0, v)] = True
        if constrained:
            table = np.where(on, rng.integers(0, 5, size=on.shape), DEAD).astype(np.int32)
            self.delta = torch.from_numpy(table).cuda()
            self.allow = torch.from_numpy(G.bits_from_table(table, T.allow_row_words(v)).view(np.int32)).cuda()
            self.table = T.table_wrap(self.delta, self.allow)
            if kind == "owned":
                self.table = T.table_concat([self.table])[0]
            elif kind == "packed":
                self.table = T.table_pack(self.table)
            q = rng.integers(-1, 6, size=n)
            q = np.where(rng.random(n) < 0.5, rng.integers(0, 2, size=n), q)
            allow = np.where(((q >= 0) & (q < 5))[:, None], on[np.clip(q, 0, 4)], False)
            self.states = torch.from_numpy(q.astype(np.int32)).cuda()
        if special and v:
            bad = rng.random((n, v))
            view = x[:, :v]
            view[(bad < 0.02) & ~allow] = np.nan
            view[(bad > 0.98) & ~allow] = np.inf
            view[(bad > 0.4) & (bad < 0.42)] = -np.inf
            view[(bad > 0.5) & (bad < 0.52)] = np.nan
            view[(bad > 0.6) & (bad < 0.62)] = -0.0
            view[(bad > 0.7) & (bad < 0.72)] = np.finfo(np.float32).min if dtype == "f32" else -3.38e38
        self.x = torch.from_numpy(x).cuda().to(TYPES[dtype])
        self.logits = self.x[:, :v]
        self.z = self.logits.double().cpu().numpy()
        # mostly allowed tokens
        score = np.where(allow, rng.random((n, v)), -1.0)
        t = score.argmax(axis=1) if v else np.zeros(n, dtype=np.int64)
        t = np.where(allow.any(axis=1) if v else False, t, NO_TOKEN)
        t = np.where(rng.random(n) < 0.08, rng.integers(-3, v + 3, size=n), t)
        self.t = t
        self.tokens = torch.from_numpy(t.astype(np.int32)).cuda()
        self.on = allow
        self.rng = rng

    def f32(self, a):
        return torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda()

    def args(self):
        return self.table, self.logits, self.states, self.tokens


def _close(got, want, tol, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), what
    off = np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0)) - np.broadcast_to(tol, want.shape)
    worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off)), off.shape) if off.size else None
    assert worst is None or off[worst] <= 0, f"{what} at {worst}: got {got[worst]}, want {want[worst]}, tolerance {np.broadcast_to(tol, want.shape)[worst]}"


def _check_logprobs(T, c, temperature, backward=True, inplace=False, stream=None):
    lp = torch.full((c.n,), 9.0, device="cuda")
    stats = torch.full((c.n, 2), 9.0, device="cuda")
    T.token_logprobs(*c.args(), lp, temperature=temperature, stats=stats, stream=stream)
    want, live, logp = R.token_logprobs(c.z, c.on, c.t, temperature)
    if stream is not None:
        stream.synchronize()
    _close(lp, want, R.tol_lp(want), "log-probabilities")
    st = stats.cpu().numpy()
    assert np.array_equal(np.isposinf(st[:, 1]), ~live) and (st[~live, 0] == 0).all()
    again = torch.full((c.n,), 9.0, device="cuda")
    T.token_logprobs(*c.args(), again, temperature=temperature, stream=stream)
    if not backward:
        torch.cuda.synchronize()
        assert torch.equal(lp, again)
        return want, live, logp
    down = c.rng.normal(0, 1, size=c.n).astype(np.float32)
    down[c.rng.random(c.n) < 0.1] = 0.0
    x = c.x.clone()
    buf = x if inplace else torch.full_like(c.x, 7.0)
    behind = buf[:, c.v:].clone()
    d = c.f32(down)
    if stream is not None:
        torch.cuda.synchronize()
    T.token_logprobs_backward(c.table, x[:, :c.v], c.states, c.tokens, stats, d, buf[:, :c.v], temperature=temperature, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(lp, again)
    g = R.gradient(logp, c.t, live, down.astype(np.float64), temperature)
    _close(buf[:, :c.v], g, R.tol_gradient(g, logp, c.t, live, down, np.zeros(c.n), temperature, c.dtype == "bf16"), "gradient")
    assert torch.equal(buf[:, c.v:], behind), "columns behind the vocabulary were written"
    return want, live, logp


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("n,v", [(1, 1), (5, 7), (3, 8), (70, 9), (33, 63), (4, 512), (300, 1000), (1, 4099), (37, 16385), (20, 32003), (2, 65537),
                                 (300, 8193)])
def test_logprobs_and_gradient(T, dtype, constrained, n, v):
    c = Case(T, n, v, dtype, 1, constrained)
    _check_logprobs(T, c, 0.7 if n % 2 else 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(1, 128256), (2, 131073), (17, 100003), (2, 256000), (3, 131072), (3, 65536)])
def test_long_rows(T, dtype, n, v):
    for constrained in (False, True):
        _check_logprobs(T, Case(T, n, v, dtype, 2, constrained), 1.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("n,v", [(40, 77), (9, 4100), (5, 40001), (300, 600)])
def test_special_values(T, dtype, constrained, n, v):
    """NaN and infinities outside the allowed set, NaN, -inf and the type's lowest value inside."""
    c = Case(T, n, v, dtype, 3, constrained, special=True)
    if not constrained:
        c.x[:, :v] = torch.where(torch.isposinf(c.x[:, :v]), 0.0, c.x[:, :v].float()).to(c.x.dtype)
        c.z = c.logits.double().cpu().numpy()
    _check_logprobs(T, c, 0.9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [9, 5000, 40000])
@pytest.mark.parametrize("fill", ["lowest", "largest", "-inf", "nan", "zero", "ascending", "far"])
def test_uniform_and_extreme_rows(T, dtype, v, fill):
    """Rows of one value, the type's lowest among them; rows with nothing but -inf or NaN take no part."""
    c = Case(T, 6, v, dtype, 4, True)
    info = torch.finfo(TYPES[dtype])
    value = {"lowest": info.min, "largest": info.max, "-inf": -math.inf, "nan": math.nan, "zero": 0.0}.get(fill)
    if fill == "ascending":                                          # every group of a lane has a new maximum
        c.x[:, :v] = torch.linspace(-30, 30, v, device="cuda").to(c.x.dtype)
    elif fill == "far":                                              # offsets that no binary32 difference of products survives
        c.x[:, :v] = (c.x[:, :v].float() + 3.0e4).to(c.x.dtype)
    else:
        c.x[:, :v] = value
    c.z = c.logits.double().cpu().numpy()
    for temperature in (1.0, 0.25, 4.0):
        _check_logprobs(T, c, temperature)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(5, 300), (40, 5000), (3, 40001), (140, 9000), (2, 140001)])
def test_low_temperatures(T, dtype, n, v):
    """Tokens whose probability is far below what a sum of exponentials relative to them can hold (lp below -87)."""
    _check_logprobs(T, Case(T, n, v, dtype, 31, sigma=3.0), 0.02)
    _run_policy(T, Case(T, n, v, dtype, 32, sigma=3.0), 0.02, (0.2, 0.2), 0.05)
    _run_policy(T, Case(T, n, v, dtype, 33, constrained=False, sigma=3.0), 0.02, (0.2, 0.2), 0.05)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [255, 256, 257, 512, 513, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385])
def test_rows_at_the_edges_of_launch_shapes(T, dtype, groups):
    """Whole numbers of 16-byte groups, and an element or two more, around every length at which another launch shape is taken."""
    v = groups * (4 if dtype == "f32" else 8) + groups % 3
    for n in (3, 40):
        if n * v > 3_000_000:
            n = 34
        c = Case(T, n, v, dtype, 34)
        _check_logprobs(T, c, 1.0)
        _run_policy(T, Case(T, n, v, dtype, 35), 1.0, (0.2, 0.2), 0.05)
    _run_preference(T, Case(T, 4, v, dtype, 36), 1.0, 0.3, 0.0, [0, 1, 4])


@pytest.mark.parametrize("n,v", [(129, 16400), (513, 9000), (385, 65601), (384, 65601)])
def test_many_rows_at_the_edges_of_launch_shapes(T, n, v):
    c = Case(T, n, v, "f32", 37)
    _check_logprobs(T, c, 1.0)
    _run_policy(T, c, 1.0, (0.2, 0.2), 0.05)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_logit_is_loud(T, dtype):
    c = Case(T, 3, 2000, dtype, 5, False)
    c.x[1, 77] = math.inf
    lp, stats = torch.zeros(3, device="cuda"), torch.zeros((3, 2), device="cuda")
    c.tokens[:] = 5
    T.token_logprobs(*c.args(), lp, stats=stats)
    g = torch.zeros_like(c.x)
    T.token_logprobs_backward(*c.args(), stats, torch.ones(3, device="cuda"), g[:, :2000])
    assert torch.isnan(lp).tolist() == [False, True, False]
    assert bool(torch.isnan(g[1, :2000]).all()) and bool(torch.isfinite(g[0]).all())


@pytest.mark.parametrize("kind", ["owned", "packed"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(50, 3001), (300, 20000), (6, 70000)])
def test_tables_the_library_made(T, kind, dtype, n, v):
    _check_logprobs(T, Case(T, n, v, dtype, 6, kind=kind), 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_in_place(T, dtype):
    for n, v in ((7, 5003), (300, 700), (3, 140001)):
        _check_logprobs(T, Case(T, n, v, dtype, 7), 1.0, inplace=True)


def _run_policy(T, c, temperature, clip, kl, use_weights=True, grad=True, inplace=False, **more):
    lp64, live, logp = R.token_logprobs(c.z, c.on, c.t, temperature)
    x = np.where(np.isfinite(lp64), lp64, 0.0)
    step = c.rng.normal(0, 0.2, size=c.n)
    for b in (1.0 - clip[0], 1.0 + clip[1]):
        if 0 < b < math.inf:                                         # the gradient jumps at a bound of the clip
            step = np.where(np.abs(step - math.log(b)) < 1e-3, step + 0.01, step)
    old, ref, adv = x - step, x + c.rng.normal(0, 0.3, size=c.n), c.rng.normal(0, 1, size=c.n)
    w = np.where(c.rng.random(c.n) < 0.15, 0.0, c.rng.random(c.n)) if use_weights else np.ones(c.n)
    old, ref, adv, w = (np.asarray(a, dtype=np.float32) for a in (old, ref, adv, w))
    loss, lp = torch.full((1,), 9.0, device="cuda"), torch.full((c.n,), 9.0, device="cuda")
    logits = c.x.clone()
    buf = logits if inplace else torch.full_like(c.x, 7.0)
    behind = buf[:, c.v:].clone()
    T.policy_loss(c.table, logits[:, :c.v], c.states, c.tokens, c.f32(old), c.f32(adv), loss, lp, grad_logits=buf[:, :c.v] if grad else None,
                  ref_logprobs=c.f32(ref) if kl else None, weights=c.f32(w) if use_weights else None, temperature=temperature, clip=clip,
                  kl_coef=kl, **more)
    torch.cuda.synchronize()
    w64 = w.astype(np.float64)
    lp64, live, logp = R.token_logprobs(c.z, c.on, c.t, temperature, w64)
    want, down, size = R.policy(lp64, live, *(a.astype(np.float64) for a in (old, ref, adv)), w64, *clip, kl)
    _close(lp, lp64, R.tol_lp(lp64), "log-probabilities")
    # a term and its slope follow lp with at most the row's size, and have some ten roundings of their own
    tol = size * (R.tol_lp(lp64) + 12 * R.U)
    _close(loss, np.array([want]), np.array([tol.sum() + 2 * R.U * abs(want) + 1e-37]), "loss")
    if grad:
        g = R.gradient(logp, c.t, live, down, temperature)
        _close(buf[:, :c.v], g, R.tol_gradient(g, logp, c.t, live, down, tol, temperature, c.dtype == "bf16"), "gradient")
        assert torch.equal(buf[:, c.v:], behind), "columns behind the vocabulary were written"
    return loss, lp, buf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("n,v,kl", [(1, 1, 0.0), (1, 130, 0.1), (4, 512, 0.05), (24, 32000, 0.04), (70, 9, 0.3), (300, 1003, 0.0), (600, 515, 0.1),
                                    (257, 8200, 0.1), (260, 4097, 0.1)])
def test_policy_loss(T, dtype, constrained, n, v, kl):
    _run_policy(T, Case(T, n, v, dtype, 8, constrained), 1.0 if n % 2 else 0.8, (0.2, 0.28), kl, use_weights=n != 24)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(3, 128256), (2, 131073), (2, 256000), (2, 262145), (530, 16384), (515, 33000), (300, 70001)])
def test_policy_loss_long_rows(T, dtype, n, v):
    """Rows on both sides of what a workgroup can hold, in few and many rows."""
    _run_policy(T, Case(T, n, v, dtype, 9, kind="owned"), 1.0, (0.1, 0.3), 0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(1, 130), (9, 40001), (290, 3000), (560, 260)])
def test_policy_loss_forms(T, dtype, n, v):
    """Special values, gradient in place, no gradient, an open upper bound, a negative KL coefficient."""
    _run_policy(T, Case(T, n, v, dtype, 10, special=True), 0.9, (0.2, 0.2), 0.05)
    _run_policy(T, Case(T, n, v, dtype, 11), 1.0, (0.2, 0.2), 0.05, inplace=True)
    _run_policy(T, Case(T, n, v, dtype, 12), 1.0, (0.0, math.inf), -0.05, grad=False)
    _run_policy(T, Case(T, n, v, dtype, 13, constrained=False), 1.0, (1.0, 0.0), 0.05)


def _run_preference(T, c, temperature, beta, smoothing, begin, grad=True, inplace=False):
    lp64, live, logp = R.token_logprobs(c.z, c.on, c.t, temperature)
    ref = (np.where(np.isfinite(lp64), lp64, 0.0) + c.rng.normal(0, 0.3, size=c.n)).astype(np.float32)
    pairs = (len(begin) - 1) // 2
    loss, rewards = torch.full((1,), 9.0, device="cuda"), torch.full((2 * pairs,), 9.0, device="cuda")
    lp = torch.full((c.n,), 9.0, device="cuda")
    logits = c.x.clone()
    buf = logits if inplace else torch.full_like(c.x, 7.0)
    T.preference_loss(c.table, logits[:, :c.v], c.states, c.tokens, c.f32(ref), torch.tensor(begin, dtype=torch.int32, device="cuda"), loss, rewards, lp,
                      grad_logits=buf[:, :c.v] if grad else None, temperature=temperature, beta=beta, smoothing=smoothing)
    torch.cuda.synchronize()
    want, rw, down = R.preference(lp64, live, ref.astype(np.float64), begin, beta, smoothing)
    _close(lp, lp64, R.tol_lp(lp64), "log-probabilities")
    tol_row = np.where(live, R.tol_lp(lp64) + R.U * np.abs(np.where(live, lp64, 0.0)), 0.0)
    tol_rw = beta * np.array([tol_row[a:b].sum() for a, b in zip(begin[:-1], begin[1:])]) + 2 * R.U * np.abs(rw)
    _close(rewards, rw, tol_rw, "rewards")
    tol_gap = tol_rw[0::2] + tol_rw[1::2]
    # |d loss_pair / d gap| <= 1, and the slope's own derivative is at most 1/4
    _close(loss, np.array([want]), np.array([(tol_gap.mean() if pairs else 0.0) + 2 * R.U * abs(want) + 1e-37]), "loss")
    if grad:
        tol_down = np.zeros(c.n)
        for k in range(2 * pairs):
            tol_down[begin[k]:begin[k + 1]] = 0.25 * tol_gap[k // 2] * beta / pairs
        tol_down += 2 * R.U * np.abs(down)
        g = R.gradient(logp, c.t, live, down, temperature)
        _close(buf[:, :c.v], g, R.tol_gradient(g, logp, c.t, live, down, tol_down, temperature, c.dtype == "bf16"), "gradient")
    return loss, rewards, lp, buf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("constrained", [False, True])
@pytest.mark.parametrize("n,v,begin", [(2, 5, [0, 1, 2]), (1, 300, [0, 0, 1]), (9, 1000, [0, 3, 3, 3, 9]), (90, 32000, [0, 20, 31, 60, 90]),
                                       (300, 515, [2, 100, 101, 250, 290]), (700, 130, list(range(0, 700, 5)) + [700]), (5, 77, [2, 2, 2])])
def test_preference_loss(T, dtype, constrained, n, v, begin):
    if len(begin) % 2 == 0:
        begin = begin[:-1]
    _run_preference(T, Case(T, n, v, dtype, 14, constrained), 1.0, 0.3, 0.1 if n % 2 else 0.0, begin)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_preference_loss_forms(T, dtype):
    _run_preference(T, Case(T, 40, 3003, dtype, 15, special=True), 0.8, 0.1, 0.0, [0, 11, 25, 40, 40])
    _run_preference(T, Case(T, 40, 3003, dtype, 16), 1.0, 0.1, 0.5, [0, 11, 25, 30, 40], inplace=True)
    _run_preference(T, Case(T, 40, 3003, dtype, 17, constrained=False), 1.0, 5.0, 0.0, [0, 11, 25], grad=False)
    _run_preference(T, Case(T, 6, 150001, dtype, 18), 1.0, 0.1, 0.0, [0, 2, 6])


def test_far_apart_pairs(T):
    """Gaps at which exp overflows: the loss is linear in the gap on one side and its slope zero on the other."""
    c = Case(T, 2, 64, "f32", 19, constrained=False)
    c.x[:] = 0.0
    c.x[0, 3] = 600.0
    c.tokens[:] = 3
    loss, rewards, lp = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    ref = torch.zeros(2, device="cuda")
    for order, want in (([0, 1, 2], 0.0), ([1, 2, 2], None)):
        g = torch.full((2, 64), 9.0, device="cuda")
        ref[:] = torch.tensor([-5000.0, 5000.0], device="cuda") if want == 0.0 else 5000.0
        T.preference_loss(None, c.x[:, :64], None, c.tokens, ref, torch.tensor(order, dtype=torch.int32, device="cuda"), loss, rewards, lp, grad_logits=g, beta=1.0)
        if want == 0.0:
            assert float(loss) == 0.0 and float(g.abs().max()) == 0.0
        else:
            assert abs(float(loss) - (5000.0 + math.log(64))) < 1e-2 and bool((g[0] == 0).all()) and abs(float(g[1, 3]) + 1 - 1 / 64) < 1e-6


@pytest.mark.parametrize("constrained", [False, True])
def test_gradient_against_differences(T, constrained):
    """Losses of the kernels themselves at logits moved along a direction, and the gradient's product with it."""
    rng = np.random.default_rng(20)
    c = Case(T, 24, 300, "f32", 20, constrained)
    u = torch.from_numpy(rng.normal(0, 1, size=c.x.shape).astype(np.float32)).cuda()
    lp = torch.zeros(24, device="cuda")
    T.token_logprobs(*c.args(), lp)
    base = torch.where(torch.isfinite(lp), lp, 0.0)
    old, ref = base - c.f32(rng.choice([-0.4, 0.05, 0.5], size=24)), base + c.f32(rng.normal(0, 0.3, size=24))
    adv, w = c.f32(rng.normal(0, 1, size=24)), c.f32(rng.random(24) / 24)
    begin = torch.tensor([0, 5, 12, 20, 24], dtype=torch.int32, device="cuda")
    rewards = torch.zeros(4, device="cuda")

    def losses(x, grad):
        out = []
        for kind in ("policy", "preference"):
            loss, g = torch.zeros(1, device="cuda"), torch.zeros_like(x) if grad else None
            gv = None if g is None else g[:, :300]
            if kind == "policy":
                T.policy_loss(c.table, x[:, :300], c.states, c.tokens, old, adv, loss, lp, grad_logits=gv, ref_logprobs=ref, weights=w, kl_coef=0.1)
            else:
                T.preference_loss(c.table, x[:, :300], c.states, c.tokens, ref, begin, loss, rewards, lp, grad_logits=gv, beta=0.5)
            out.append((float(loss), g))
        return out

    h = 0.01
    here, up, down = losses(c.x, True), losses(c.x + h * u, False), losses(c.x - h * u, False)
    for (value, g), (a, _), (b, _) in zip(here, up, down):
        slope = float((g.double() * u.double()).sum())
        # central differences: the losses are off by some 1e-6 each (over 2 h: 1e-4), the third derivative's part is h^2 / 6 of
        # about |u|^3-sized sums over the softmax: below 1e-3
        assert abs((a - b) / (2 * h) - slope) < 2e-3 * max(1.0, abs(slope)), (value, a, b, slope)
        assert abs(slope) > 1e-3


def test_rows_beyond_32_bit_offsets(T):
    """Row offsets that pass 2^31 elements and 2^32 bytes, in logits and gradient."""
    v, stride, n = 1003, 600_000_000, 5
    x = torch.empty(stride * (n - 1) + 1024, dtype=torch.bfloat16, device="cuda")
    g = torch.empty_like(x)
    logits = torch.as_strided(x, (n, v), (stride, 1))
    grad = torch.as_strided(g, (n, v), (stride, 1))
    c = Case(T, n, v, "bf16", 21)
    logits.copy_(c.logits)
    lp, stats = torch.zeros(n, device="cuda"), torch.zeros((n, 2), device="cuda")
    T.token_logprobs(c.table, logits, c.states, c.tokens, lp, stats=stats)
    T.token_logprobs_backward(c.table, logits, c.states, c.tokens, stats, torch.ones(n, device="cuda"), grad)
    want, live, logp = R.token_logprobs(c.z, c.on, c.t, 1.0)
    _close(lp, want, R.tol_lp(want), "log-probabilities")
    gw = R.gradient(logp, c.t, live, np.ones(n), 1.0)
    _close(grad, gw, R.tol_gradient(gw, logp, c.t, live, np.ones(n), np.zeros(n), 1.0, True), "gradient")
    loss = torch.zeros(1, device="cuda")
    grad.zero_()
    T.policy_loss(c.table, logits, c.states, c.tokens, torch.where(torch.isfinite(lp), lp, 0.0), -torch.ones(n, device="cuda"), loss, lp, grad_logits=grad)
    _close(grad, gw, R.tol_gradient(gw, logp, c.t, live, np.ones(n), R.tol_lp(want) + 12 * R.U, 1.0, True), "policy gradient")


def test_another_stream(T):
    c = Case(T, 40, 20000, "bf16", 22)
    torch.cuda.synchronize()
    _check_logprobs(T, c, 1.0, stream=torch.cuda.Stream())


def test_views_and_repeats(T):
    """Rows inside a larger buffer, at an offset of 16 bytes; the same call twice gives the same bits."""
    c = Case(T, 64, 2500, "bf16", 23)
    big = torch.zeros((64, 2576), dtype=torch.bfloat16, device="cuda")
    big[:, 8:2508] = c.logits
    c.x = big[:, 8:]
    c.logits = c.x[:, :2500]
    _check_logprobs(T, c, 1.0)
    runs = []
    for _ in range(2):
        c.rng = np.random.default_rng(5)
        loss, lp, g = _run_policy(T, c, 1.0, (0.2, 0.2), 0.1)
        runs.append((loss, lp, g))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_recorded_graph(T):
    """All calls recorded once and replayed on new logits, with eager work between the replays."""
    c = Case(T, 48, 9000, "bf16", 24)
    n, v = c.n, c.v
    lp, stats = torch.zeros(n, device="cuda"), torch.zeros((n, 2), device="cuda")
    lp2, lp3 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    loss, loss2, rewards = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(4, device="cuda")
    g1, g2, g3 = (torch.zeros((n, v + 8 - v % 8), dtype=torch.bfloat16, device="cuda")[:, :v] for _ in range(3))
    ones, old = torch.ones(n, device="cuda"), torch.full((n,), -8.0, device="cuda")
    begin = torch.tensor([0, 10, 20, 30, 48], dtype=torch.int32, device="cuda")
    ws = torch.empty(T.loss_workspace_bytes(n, 2), dtype=torch.uint8, device="cuda")

    def work():
        T.token_logprobs(*c.args(), lp, stats=stats, workspace=ws)
        T.token_logprobs_backward(*c.args(), stats, ones, g1)
        T.policy_loss(*c.args(), old, ones, loss, lp2, grad_logits=g2, ref_logprobs=old, kl_coef=0.1, workspace=ws)
        T.preference_loss(*c.args(), old, begin, loss2, rewards, lp3, grad_logits=g3, workspace=ws)
        return lp, stats, lp2, lp3, loss, loss2, rewards, g1, g2, g3

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(4):
        c.x.copy_(torch.randn(c.x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(k)))
        want = [t.clone() for t in work()]
        for t in (lp, stats, lp2, lp3, loss, loss2, rewards, g1, g2, g3):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip((lp, stats, lp2, lp3, loss, loss2, rewards, g1, g2, g3), want)):
            assert torch.equal(a, b), (k, i)


def test_no_rows(T):
    x = torch.zeros((0, 64), device="cuda")
    e, i = torch.zeros(0, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    loss, rewards = torch.full((1,), 9.0, device="cuda"), torch.full((2,), 9.0, device="cuda")
    T.token_logprobs(None, x, None, i, e)
    T.token_logprobs_backward(None, x, None, i, e, e, x.clone())
    T.policy_loss(None, x, None, i, e, e, loss, e, grad_logits=x.clone())
    assert float(loss) == 0.0
    begin = torch.zeros(3, dtype=torch.int32, device="cuda")
    T.preference_loss(None, x, None, i, e, begin, loss, rewards, e, grad_logits=x.clone())
    assert abs(float(loss) - math.log(2)) < 1e-6 and rewards.tolist() == [0.0, 0.0]
    T.preference_loss(None, x, None, i, e, begin[:1], loss, rewards, e)
    assert float(loss) == 0.0


def test_sequences_outside_the_rows_are_cut(T):
    c = Case(T, 10, 50, "f32", 25, constrained=False)
    c.t = np.arange(10)
    c.tokens = torch.arange(10, dtype=torch.int32, device="cuda")
    out = []
    for begin in ([-5, 4, 1000], [0, 4, 10]):
        loss, rewards, lp = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(10, device="cuda")
        g = torch.zeros((10, 50 + 2), device="cuda")
        T.preference_loss(None, c.logits, None, c.tokens, torch.zeros(10, device="cuda"), torch.tensor(begin, dtype=torch.int32, device="cuda"),
                          loss, rewards, lp, grad_logits=g[:, :50])
        out.append((loss, rewards, lp, g))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_refusals(T):
    """What the calls refuse, before anything is launched."""
    c = Case(T, 4, 100, "bf16", 26)
    lp, stats, loss, rewards = (torch.zeros(k, device="cuda") for k in (4, 8, 1, 2))
    ones = torch.ones(4, device="cuda")
    begin = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    x = c.x
    half = x[:, :100].half()
    odd = torch.zeros((4, 101), dtype=torch.bfloat16, device="cuda")
    g = torch.zeros_like(x)

    def logprobs(table=c.table, logits=c.logits, states=c.states, tokens=c.tokens, out=lp, **kw):
        T.token_logprobs(table, logits, states, tokens, out, **kw)

    def policy(**kw):
        T.policy_loss(c.table, c.logits, c.states, c.tokens, ones, ones, kw.pop("loss", loss), lp, **kw)

    def preference(**kw):
        T.preference_loss(c.table, c.logits, c.states, c.tokens, ones, kw.pop("begin", begin), loss, kw.pop("rewards", rewards), lp, **kw)

    refused = [
        (TypeError, lambda: logprobs(logits=half)),
        (ValueError, lambda: logprobs(logits=c.logits.t())),
        (ValueError, lambda: logprobs(logits=c.logits.cpu())),
        (ValueError, lambda: logprobs(logits=x[:, :99])),
        (ValueError, lambda: logprobs(states=None)),
        (ValueError, lambda: logprobs(tokens=c.tokens.long())),
        (ValueError, lambda: logprobs(tokens=c.tokens[:3])),
        (ValueError, lambda: logprobs(tokens=c.tokens.cpu())),
        (ValueError, lambda: logprobs(out=lp[::2])),
        (ValueError, lambda: logprobs(stats=lp)),
        (T.TdfaError, lambda: logprobs(temperature=0.0)),
        (T.TdfaError, lambda: logprobs(temperature=-1.0)),
        (T.TdfaError, lambda: logprobs(temperature=math.nan)),
        (T.TdfaError, lambda: logprobs(temperature=math.inf)),
        (T.TdfaError, lambda: logprobs(temperature=1e-39)),
        (T.TdfaError, lambda: logprobs(logits=odd)),
        (T.TdfaError, lambda: logprobs(logits=x[:, 1:])),
        (T.TdfaError, lambda: logprobs(workspace=torch.empty(T.loss_workspace_bytes(4) - 1, dtype=torch.uint8, device="cuda"))),
        (T.TdfaError, lambda: logprobs(workspace=torch.empty(T.loss_workspace_bytes(4) + 4, dtype=torch.uint8, device="cuda")[4:])),
        (ValueError, lambda: policy(grad_logits=g.float())),
        (ValueError, lambda: policy(grad_logits=g[:, :50])),
        (ValueError, lambda: policy(loss=None)),
        (T.TdfaError, lambda: policy(kl_coef=0.1)),
        (T.TdfaError, lambda: policy(kl_coef=math.inf, ref_logprobs=ones)),
        (T.TdfaError, lambda: policy(clip=(-0.1, 0.2))),
        (T.TdfaError, lambda: policy(clip=(1.1, 0.2))),
        (T.TdfaError, lambda: policy(clip=(0.2, -0.1))),
        (T.TdfaError, lambda: policy(clip=(0.2, math.nan))),
        (ValueError, lambda: preference(begin=begin[:2])),
        (ValueError, lambda: preference(rewards=rewards[:1])),
        (T.TdfaError, lambda: preference(beta=0.0)),
        (T.TdfaError, lambda: preference(beta=math.inf)),
        (T.TdfaError, lambda: preference(smoothing=1.5)),
        (T.TdfaError, lambda: preference(smoothing=math.nan)),
        (ValueError, lambda: T.token_logprobs_backward(c.table, c.logits, c.states, c.tokens, stats, ones, None)),
        (T.TdfaError, lambda: T.token_logprobs_backward(c.table, x[:2, :100], c.states, c.tokens, stats, ones, x[1:3, :100])),
    ]
    lib, addr = T.lib(), [x.data_ptr(), c.states.data_ptr(), c.tokens.data_ptr(), lp.data_ptr()]
    assert lib.tdfa_token_logprobs(None, addr[0], 1, 4, (1 << 24) + 1, 1 << 25, None, addr[2], 1.0, addr[3], None, None, 0, None) == -1
    assert lib.tdfa_token_logprobs(c.table._h, addr[0], 1, 4, 99, 128, addr[1], addr[2], 1.0, addr[3], None, None, 0, None) == -1
    assert lib.tdfa_token_logprobs(c.table._h, addr[0], 2, 4, 100, 128, addr[1], addr[2], 1.0, addr[3], None, None, 0, None) == -1
    assert lib.tdfa_token_logprobs(c.table._h, addr[0], 1, -1, 100, 128, addr[1], addr[2], 1.0, addr[3], None, None, 0, None) == -1
    assert lib.tdfa_token_logprobs(c.table._h, None, 1, 4, 100, 128, addr[1], addr[2], 1.0, addr[3], None, None, 0, None) == -1
    assert lib.tdfa_token_logprobs(None, addr[0], 1, 1, 1 << 20, 1 << 20, None, addr[2], 1.0, addr[3], None, None, 0, None) == -1      # wants a workspace
    assert lib.tdfa_policy_loss(None, addr[0], 1, 4, 100, 128, None, addr[2], 1.0, addr[3], None, addr[3], None, 0.2, 0.2, 0.0, loss.data_ptr(),
                                addr[3], None, 0, None, 0, None) == -1
    assert b"workspace" in lib.tdfa_last_error()
    assert lib.tdfa_loss_workspace_bytes(-1, 0) == -1 and lib.tdfa_loss_workspace_bytes(0, -1) == -1
    for k, (error, call) in enumerate(refused):
        with pytest.raises(error):
            call()
            print("not refused:", k)
    torch.cuda.synchronize()
    _check_logprobs(T, c, 1.0)


def _many_rows(T, rows, v=8):
    """Rows of few tokens, in 64 bits on the GPU: (logits, tokens, lp, p)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, v, generator=g, device="cuda").bfloat16()
    tokens = torch.randint(-1, v, (rows,), generator=g, device="cuda", dtype=torch.int32)
    logp = torch.log_softmax(x.double(), dim=1)
    live = tokens >= 0
    lp = torch.where(live, logp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0], 0.0)
    return x, tokens, live, lp, logp.exp()


def _slopes_close(grad, p, tokens, live, down, tol_down):
    """Against down ([j = t] - p_j), in bf16."""
    want = -p
    want[torch.arange(len(tokens), device="cuda")[live], tokens[live].long()] += 1.0
    want *= torch.where(live, down, 0.0)[:, None]
    tol = torch.where(live, down.abs(), 0.0)[:, None] * (2 * R.REL_SUM + 64 * R.U) + tol_down
    tol = tol + 2.0 ** -8 * (want.abs() + tol) + 1e-37
    assert bool(((grad.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("rows", [8193, 16385, (1 << 21) + 3])
def test_more_rows_than_a_launch_has_workgroups(T, rows):
    x, tokens, live, lp, p = _many_rows(T, rows)
    tol = R.REL_SUM + 4 * R.U * lp.abs()
    got, stats = torch.full((rows,), 9.0, device="cuda"), torch.full((rows, 2), 9.0, device="cuda")
    T.token_logprobs(None, x, None, tokens, got, stats=stats)
    assert bool(((got.double() - lp).abs() <= tol).all())
    g = torch.Generator(device="cuda").manual_seed(1)
    down = torch.randn(rows, generator=g, device="cuda")
    grad = torch.full_like(x, 7.0)
    T.token_logprobs_backward(None, x, None, tokens, stats, down, grad)
    _slopes_close(grad, p, tokens, live, down.double(), 0.0)

    old, adv = (lp + 0.05 * torch.randn(rows, generator=g, device="cuda")).float(), torch.randn(rows, generator=g, device="cuda")
    loss, grad = torch.full((1,), 9.0, device="cuda"), torch.full_like(x, 7.0)
    T.policy_loss(None, x, None, tokens, old, adv, loss, got, grad_logits=grad, clip=(1.0, math.inf))      # nothing is clipped
    each = torch.where(live, -torch.exp(lp - old.double()) * adv.double(), 0.0)
    size = float(each.abs().sum())
    assert abs(float(loss) - float(each.sum())) <= size * (R.REL_SUM + 4 * R.U * float(lp.abs().max()) + 16 * R.U) + 1e-6 * abs(float(each.sum()))
    assert bool(((got.double() - lp).abs() <= tol).all())
    _slopes_close(grad, p, tokens, live, each, (each.abs() * (tol + 16 * R.U))[:, None])

    cut = [0, rows // 3, rows - 9, rows - 1, rows]
    begin, ref = torch.tensor(cut, dtype=torch.int32, device="cuda"), (lp + 0.01 * torch.randn(rows, generator=g, device="cuda")).float()
    rewards, grad, beta = torch.full((4,), 9.0, device="cuda"), torch.full_like(x, 7.0), 4.0 / rows
    T.preference_loss(None, x, None, tokens, ref, begin, loss, rewards, got, grad_logits=grad, beta=beta)
    over = torch.where(live, lp - ref.double(), 0.0)
    want = [beta * float(over[a:b].sum()) for a, b in zip(cut, cut[1:])]
    # the sums' errors add up at worst
    off = beta * rows * (R.REL_SUM + 4 * R.U * float(lp.abs().max())) + 8 * R.U
    assert all(abs(float(a) - b) <= off for a, b in zip(rewards, want))
    gap = [want[0] - want[1], want[2] - want[3]]
    assert abs(float(loss) - sum(math.log1p(math.exp(-y)) for y in gap) / 2) <= 2 * off + 16 * R.U
    down = torch.empty(rows, dtype=torch.float64, device="cuda")
    for k, (a, b) in enumerate(zip(cut, cut[1:])):
        down[a:b] = (beta if k % 2 else -beta) / 2 / (1.0 + math.exp(gap[k // 2]))
    _slopes_close(grad, p, tokens, live, down, beta / 2 * (2 * off + 16 * R.U))


def test_refusals_of_overlaps_and_strides(T):
    x = torch.randn(4, 64, device="cuda").bfloat16()
    tokens, f = torch.zeros(4, dtype=torch.int32, device="cuda"), [torch.ones(8, device="cuda") for _ in range(4)]
    loss, rewards, begin = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    kept = [t.clone() for t in (x, tokens, *f)]
    for old, adv, ref, weights, lp in [(0, 1, 2, 3, 0), (0, 1, 2, 3, 1), (0, 1, 2, 3, 2), (0, 1, 2, 3, 3)]:
        with pytest.raises(T.TdfaError, match="overlaps"):
            T.policy_loss(None, x, None, tokens, f[old][:4], f[adv][:4], loss, f[lp][3:7], ref_logprobs=f[ref][:4], weights=f[weights][:4], kl_coef=0.1)
    with pytest.raises(T.TdfaError, match="overlaps"):
        T.preference_loss(None, x, None, tokens, f[0][:4], begin, loss, rewards, f[0][:4])
    with pytest.raises(T.TdfaError, match="overlaps"):
        T.policy_loss(None, x, None, tokens, f[0][:4], f[1][:4], loss, tokens.view(torch.float32))
    # next to one another is fine, and so is what is not read
    T.policy_loss(None, x, None, tokens, f[0][:4], f[1][:4], loss, f[0][4:], ref_logprobs=f[0][4:])
    f[0][4:] = 1.0
    lib, far = T.lib(), (1 << 35)                          # elements of 2 bytes: 2^36 bytes
    a = [x.data_ptr(), tokens.data_ptr(), f[0].data_ptr(), f[1].data_ptr()]
    assert lib.tdfa_token_logprobs(None, a[0], 1, 2, 64, far, None, a[1], 1.0, a[2], None, None, 0, None) == -1
    assert b"stride" in lib.tdfa_last_error()
    assert lib.tdfa_token_logprobs_backward(None, a[0], 1, 2, 64, 64, None, a[1], 1.0, a[2], a[3], a[0], far, None) == -1
    assert b"stride" in lib.tdfa_last_error()
    assert lib.tdfa_token_logprobs(None, a[0], 1, 1, 64, far, None, a[1], 1.0, f[2].data_ptr(), None, None, 0, None) == 0       # one row has none
    torch.cuda.synchronize()
    f[2][:1] = 1.0
    assert all(torch.equal(s, t) for s, t in zip(kept, (x, tokens, *f)))
