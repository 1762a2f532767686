"""Draws and lists where a row's allowed tokens, its logits or its settings lie at an edge of how they are worked out."""
import numpy as np
import pytest
import torch

import draw_ref as R
import gpu_util as G
from test_gpu_draw import DEAD, NO_TOKEN, TYPES, Rows, check_draw, check_top, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2407_08103_amd as T
    assert torch.cuda.is_available()
    return T


class Given(Rows):
    """Given rows of logits, each under a state of its own or (on None) without a constraint."""

    def __init__(self, T, z, on, dtype, seed=0):
        self.rng = np.random.default_rng([seed, *np.shape(z)])
        self.n, self.v = np.shape(z)
        x = np.full((self.n, -(-self.v // 64) * 64), np.nan, dtype=np.float32)
        x[:, :self.v] = z
        self.x = torch.from_numpy(x).cuda().to(TYPES[dtype])
        self.logits = self.x[:, :self.v]
        self.z = self.logits.double().cpu().numpy()
        self.table, self.states, self.delta, self.on = None, None, None, np.ones((self.n, self.v), dtype=bool)
        if on is not None:
            self.on, self.q = np.asarray(on), np.arange(self.n)
            self.delta = np.where(self.on, self.rng.integers(0, 5, size=self.on.shape), DEAD).astype(np.int32)
            allow = torch.from_numpy(G.bits_from_table(self.delta, T.allow_row_words(self.v)).view(np.int32)).cuda()
            self.keep = torch.from_numpy(self.delta).cuda(), allow
            self.table = T.table_wrap(*self.keep)
            self.states = torch.arange(self.n, dtype=torch.int32, device="cuda")

    def after(self, token, i):
        return i if token == NO_TOKEN else self.delta[i, token]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [4001, 9001, 33001, 70001])
def test_few_wavefronts_have_a_token(T, v, dtype):
    """Allowed tokens at one place of a row, about as many as are put in order without another look: most wavefronts have none, and are far ahead of those
    that do."""
    n = 24
    rng = np.random.default_rng([v, 1])
    on = np.zeros((n, v), dtype=bool)
    for i in range(n):
        count = 254 + i % 6
        at = [0, v - count, (v // 2) // 8 * 8][i % 3]
        on[i, at:at + count] = True
    r = Given(T, rng.normal(0, 2, (n, v)), on, dtype)
    for _ in range(4):
        check_draw(T, r, r.uniforms(), temperature=0.8, top_p=0.9)
        check_draw(T, r, r.uniforms(), top_k=20, min_p=0.01)
        check_top(T, r, 30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v,copies", [(3001, 1), (9001, 1), (33001, 1), (33001, 60), (66001, 1), (66001, 60)])
@pytest.mark.parametrize("beside", [50.0, 3.0e38, np.inf, np.nan])
def test_larger_logits_that_are_not_allowed(T, beside, v, copies, dtype):
    """The first token of a row has logits above its own in its group of 16 bytes, of tokens that the constraint does not allow; and ties: the lowest id of
    the largest allowed logit is in such a group or not."""
    n = 8
    rng = np.random.default_rng([v, 2])
    on = rng.random((n, v)) < 0.6
    z = rng.normal(0, 2, (n, v))
    want = np.zeros(n, dtype=np.int64)
    for i in range(n):
        at = [0, 1, 3, v // 8 * 8 + (v % 8 - 1), v // 2, v // 3, v // 16 * 8 + 5, v // 4 * 4 - 1][i]
        z[i, at], on[i, at], want[i] = 20.0, True, at
        for other in {at ^ 1, at ^ 2, at ^ 3} - {at}:
            if other < v:
                z[i, other], on[i, other] = beside, False
        if i % 2 and at + 100 < v:
            z[i, at + 100], on[i, at + 100] = 20.0, True              # a tie behind it
    r = Given(T, z, on, dtype)
    for s in (dict(temperature=0.0), dict(top_k=1), dict(temperature=0.7, top_p=0.9), dict(min_p=0.2)):
        check_draw(T, r, r.uniforms(), **s)
    # the same rows in a batch of as many as take other launch shapes
    x, q = r.x.repeat(copies, 1)[:, :v], r.states.repeat(copies)
    tokens, after = (torch.full((n * copies,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    T.draw_step(r.table, x, q, torch.rand(n * copies, device="cuda"), tokens, after, temperature=0.0)
    assert np.array_equal(tokens.cpu().numpy(), np.tile(want, copies))
    assert np.array_equal(after.cpu().numpy(), np.tile(r.delta[np.arange(n), want], copies))
    check_top(T, r, 5)


@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("temperature,largest", [(1.5, 3.0), (1.5, 0.1875), (0.75, 20.25), (0.75, 24.0), (0.4, 3.2), (0.4, 0.2), (1.0, 2.5), (0.25, 6.0), (2.0, 12.0),
                                                 (1.25, 5.0), (0.5, 0.5)])
def test_zeros_at_a_border(T, temperature, largest, table):
    """Many logits of exactly 0, or next to it, where the distance of the largest logit from 0 is a whole number of 80ths of the temperature or so: tokens that share out
    a search are found however near its end they lie."""
    n, v = 48, 4001
    rng = np.random.default_rng([int(largest * 1000), 5])
    z = np.minimum(rng.normal(0, 2, (n, v)), largest * 0.99)
    z[rng.random((n, v)) < 0.2] = 0.0
    tiny = (rng.random((n, v)) < 0.02)
    z[tiny] = (rng.choice([-1.0, 1.0], (n, v)) * 10.0 ** rng.uniform(-30, -14, (n, v)))[tiny]
    z[np.arange(n), rng.integers(0, v, n)] = largest
    on = None
    if table:
        on = (rng.random((n, v)) < 0.7) | (z == largest)
    r = Given(T, z, on, "f32")
    zeros = [int(np.count_nonzero(r.on[i] & (r.z[i] > 0))) for i in range(n)]
    u = np.linspace(0.0, 0.9999, n).astype(np.float32)
    far = np.exp(-np.float64(np.float32(largest)) / np.float64(np.float32(temperature)))
    for s in (dict(), dict(top_k=zeros[0] + 5), dict(top_k=zeros[n // 2] + 60, top_p=0.95), dict(min_p=float(far * 0.999)), dict(min_p=float(far * 0.999), top_p=0.9), dict(top_p=0.6)):
        for i in range(2):
            check_draw(T, r, np.roll(u, i), temperature=temperature, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [300, 4099, 33001, 262147])
def test_lists_keep_their_bits(T, v, dtype):
    """Log-probabilities as near to the definition as weights and sums of 64 bits and one rounding leave them: where the largest token has nearly all of the probability,
    its logarithm is what all the others add up to.  With 32-bit logits and more than 256 allowed tokens a weight 2^x below the largest, which is 1, may be off: its exponent is a
    difference, times a constant that was rounded, each off by 2^-24 of itself, ln 2 * 3 * 2^-24 |x| of the weight, and the exponential by 2^-23."""
    n = 10
    rng = np.random.default_rng([v, 6])
    z = rng.normal(0, 2, (n, v))
    on = rng.random((n, v)) < 0.7
    at = rng.integers(0, v, n)
    z[np.arange(n), at] = rng.uniform(5, 45, n)
    on[np.arange(n), at] = True
    z[0] = rng.normal(0, 0.1, v)
    for r in (Given(T, z, on, dtype), Given(T, z, None, dtype)):
        for k, t in ((1, 1.0), (40, 0.7), (256, 1.9)):
            ids, lp = torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda")
            T.top_logprobs(r.table, r.logits, r.states, ids, lp, temperature=t)
            for i in range(n):
                want, want_lp = R.top(r.z[i], r.on[i], k, float(np.float32(t)))
                assert np.array_equal(ids[i].cpu().numpy(), want), i
                lost = 0.0
                if dtype == "f32" and np.count_nonzero(r.on[i]) > 256:
                    x = (r.z[i][r.on[i]] - r.z[i][r.on[i]].max()) / float(np.float32(t)) / np.log(2)
                    lost = np.sum(np.where(x < 0, 2.0 ** x * (1 + 3 / 2 * np.log(2) * -x) * 2.0 ** -23, 0.0)) / np.sum(2.0 ** x)
                assert all(close(a, b) or abs(a - b) <= lost + 2.0 ** -39 + abs(b) * 2.0 ** -23 for a, b in zip(lp[i].cpu().numpy(), want_lp)), (i, k, lp[i], want_lp)


def draw_long(z, allow, u, temperature, top_k=0, top_p=1.0):
    """draw_ref.draw with sums of 64-bit mantissas: one by one, 2^22 weights of 2^-41 beside one of 1 are off by 2^-31 of it with 53."""
    temperature, top_p, u = (float(np.float32(x)) for x in (temperature, top_p, u))
    ids, x = R.ordered(z, allow)
    w = R.weights(x, temperature).astype(np.longdouble)
    w = w[:R.kept(x, w, top_k, top_p, 0.0)]
    upto = np.cumsum(w)
    total, last = upto[-1], int(np.flatnonzero(w)[-1])
    lo, hi = (min(int(np.searchsorted(upto, np.longdouble(u) * total + e * total, side="right")), last) for e in (-R.BORDER, R.BORDER))
    return {int(ids[i]): float(np.log(w[i] / total)) for i in range(lo, hi + 1)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [131077, (1 << 22) + 3])
def test_many_tokens_of_next_to_no_weight(T, v, dtype):
    """Tokens that weigh less than a rounding of the largest's weight each, but more than 2^-40 of the whole together: numbers next to 1 draw them."""
    n = 12
    each = -32.1 if v < 1 << 20 else -28.2                      # their weights are 2^-46.3 and 2^-40.7
    z = np.full((n, v), 400.0 + 10.0 * np.floor(each * 5) / 5)
    z[np.arange(n), np.arange(n) * 977] = 400.0
    z[:, 5::1001] = 400.0 - 620.0
    r = Given(T, z, None, dtype)
    u = np.float32(1.0 - 2.0 ** -np.linspace(18, 24, n))
    u[:2] = 1.0
    tokens, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    for s in (dict(), dict(top_k=v - 7), dict(top_p=1.0 - 2.0 ** -24)):
        T.draw_step(None, r.logits, None, torch.from_numpy(u).cuda(), tokens, None, temperature=10.0, logprobs=lp, **s)
        for i in range(n):
            want = draw_long(r.z[i], r.on[i], u[i], 10.0, **s)
            assert int(tokens[i]) in want, (i, s, u[i], tokens[i], want)
            assert close(float(lp[i]), want[int(tokens[i])]), (i, s, lp[i], want)
    check_top(T, r, 3, 10.0)


def test_top_k_of_any_size(T):
    """A top_k beyond 32 bits cuts nothing off, and below 0 it is refused, whatever it is modulo 2^32."""
    r = Rows(T, "open", 30, 3001, "f32", 91, table=None)
    u = torch.from_numpy(r.uniforms()).cuda()
    want, got = torch.empty(30, dtype=torch.int32, device="cuda"), torch.empty(30, dtype=torch.int32, device="cuda")
    T.draw_step(None, r.logits, None, u, want, None)
    for k in (3001, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 2 ** 63 + 2, 10 ** 30):
        T.draw_step(None, r.logits, None, u, got, None, top_k=k)
        assert torch.equal(got, want), k
    for k in (-1, -2 ** 31, 1 - 2 ** 32, -2 ** 32, -10 ** 30):
        with pytest.raises(T.TdfaError):
            T.draw_step(None, r.logits, None, u, got, None, top_k=k)


@pytest.mark.parametrize("beside", [2.0, 3.0e38, np.inf])
def test_lists_beside_larger_logits_that_are_not_allowed(T, beside):
    """The first tokens have a larger logit each in its group of 16 bytes that the constraint does not allow: its distance below the largest is no step."""
    n, v = 6, 9004
    rng = np.random.default_rng(12)
    z = rng.normal(-3, 1, (n, v))
    on = rng.random((n, v)) < 0.6
    for i in range(n):
        at = rng.choice(v // 4, 40, replace=False) * 4 + rng.integers(0, 4, 40)
        z[i, at], on[i, at] = 1.0 - np.arange(40) / 64, True
        z[i, at ^ 1], on[i, at ^ 1] = beside, False
    r = Given(T, z, on, "f32")
    for k in (1, 40, 200):
        check_top(T, r, k)


@pytest.mark.parametrize("table", [None, "owned"])
@pytest.mark.parametrize("dtype,v,rows", [("bf16", 66001, 800), ("bf16", 131081, 770), ("f32", 17003, 470), ("f32", 33003, 470), ("f32", 70001, 470)])
def test_many_long_rows(T, dtype, v, rows, table):
    """Shapes of launches that many rows take, with a constraint and without one: a row gives the same wherever it lies, what the definition says."""
    r = Rows(T, "peaked", 5, v, dtype, 92, table=table)
    rep = -(-rows // 5)
    x, q = r.x.repeat(rep, 1)[:rows], None if table is None else r.states.repeat(rep)[:rows].contiguous()
    u = torch.from_numpy(r.uniforms()).cuda()
    t, lp, ids, top = (torch.empty(s, dtype=d, device="cuda") for s, d in ((rows, torch.int32), (rows, torch.float32), ((rows, 33), torch.int32), ((rows, 33), torch.float32)))
    after = None if table is None else torch.empty_like(t)
    for s in (dict(temperature=0.8, top_p=0.9), dict(top_k=900, min_p=0.001), dict(temperature=0.0)):
        T.draw_step(r.table, x[:, :v], q, u.repeat(rep)[:rows].contiguous(), t, after, logprobs=lp, **s)
        for i in range(5):
            want = R.draw(r.z[i], r.on[i], float(u[i]), s.get("temperature", 1.0), s.get("top_k", 0), s.get("top_p", 1.0), s.get("min_p", 0.0))
            assert int(t[i]) in want and close(float(lp[i]), want[int(t[i])]), (i, s)
            assert after is None or int(after[i]) == r.after(int(t[i]), i), (i, s)
        for a in (t, lp, after):
            assert a is None or torch.equal(a, a[:5].repeat(rep)[:rows])
    T.top_logprobs(r.table, x[:, :v], q, ids, top)
    assert torch.equal(ids, ids[:5].repeat(rep, 1)[:rows]) and torch.equal(top, top[:5].repeat(rep, 1)[:rows])
    check_top(T, r, 33)
    for i in range(5):
        assert np.array_equal(ids[i].cpu().numpy(), R.top(r.z[i], r.on[i], 33, 1.0)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_a_launch(T, dtype):
    n, v = (1 << 21) + 77, 9
    x = torch.randn((n, 16), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(TYPES[dtype])
    u = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    t, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    ids, top = torch.empty((n, 2), dtype=torch.int32, device="cuda"), torch.empty((n, 2), device="cuda")
    T.draw_step(None, x[:, :v], None, u, t, None, logprobs=lp)
    T.top_logprobs(None, x[:, :v], None, ids, top)
    want = torch.log_softmax(x[:, :v].double(), 1)
    # a rounding, and 2^-20 for weights of 32 bits
    assert (lp - want.gather(1, t.long()[:, None])[:, 0]).abs().max() <= 2.0 ** -19
    value, order = torch.sort(x[:, :v].float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), order[:, :2]) and (top - want.gather(1, order[:, :2])).abs().max() <= 2.0 ** -19
    upto = torch.cumsum(want.gather(1, order).exp(), 1)
    at = (order == t.long()[:, None]).to(torch.int8).argmax(1, keepdim=True)
    last, before = upto.gather(1, at)[:, 0], torch.where(at > 0, upto.gather(1, (at - 1).clamp(min=0)), 0.0)[:, 0]
    assert ((before - 2.0 ** -39 <= u) & (u <= last + 2.0 ** -39)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [30, 89, 201, 256, 3001])
def test_tokens_of_no_weight_are_not_drawn(T, v, dtype):
    """Many logits so low that their weights are 0 in 64 bits: the number 1 draws the last token that has one."""
    n = 150
    rng = np.random.default_rng([v, 9])
    z = rng.normal(0, 3, (n, v))
    z[rng.random((n, v)) < 0.5] = -1.0e4
    z[:, 1] = 2.0
    on = None if v <= 256 else (rng.random((n, v)) < 200 / v) | (np.arange(v) == 1)
    r = Given(T, z, on, dtype)
    for temperature in (0.7, 0.5, 1.3):
        for u in (1.0, 1.0 - 2.0 ** -24):
            check_draw(T, r, np.full(n, u, dtype=np.float32), temperature=temperature)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [200, 2873, 9001])
@pytest.mark.parametrize("kind", ["open", "grid", "upcast"])
def test_the_last_token_of_what_is_left(T, kind, v, dtype):
    """The number 1 draws the last token that the cuts leave, and none behind it, however the sums up to there were rounded."""
    n = 60
    rng = np.random.default_rng([v, 10])
    z = rng.normal(0, 3, (n, v))
    if kind == "grid":
        z = np.round(z * 16) / 16
    elif kind == "upcast":
        z = torch.from_numpy(z).bfloat16().double().numpy()
    r = Given(T, z, None, dtype)
    u = np.float32([1.0, 1.0, 1.0 - 2.0 ** -24] * (n // 3))
    for s in (dict(temperature=2.0, top_k=v // 2, min_p=0.05), dict(temperature=5.0, top_k=v // 3, top_p=0.95), dict(temperature=5.0, top_k=v // 3, top_p=0.9),
              dict(temperature=0.9, top_p=0.8), dict(top_p=0.9, min_p=0.01), dict(temperature=1.5, top_k=50, top_p=0.97, min_p=0.02), dict(min_p=0.3), dict(top_k=20)):
        check_draw(T, r, u, **s)
