"""Draws from given numbers and lists of the most likely tokens against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import draw_ref as R
import gpu_util as G

pytestmark = pytest.mark.gpu
DEAD = NO_TOKEN = -1
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def T():
    import paper_2407_08103_amd as T
    assert torch.cuda.is_available()
    return T


def logits_of(kind, n, v, rng):
    """Rows of one kind: open and predictable text, few values that many tokens share, extremes."""
    x = rng.normal(0, 2, size=(n, v))
    if kind == "peaked":
        for r in range(n):
            at = rng.integers(0, v, size=min(v, 30))
            x[r, at] += rng.random(len(at)) * 14
    elif kind == "ties":
        x = np.round(x)
    elif kind == "equal":
        x = np.repeat(rng.normal(0, 2, size=(n, 1)), v, axis=1)
    elif kind == "zeros":                                       # about zero: the smallest numbers, both zeros
        x = rng.normal(0, 1, size=(n, v)) * 10.0 ** rng.integers(-42, -1, size=(n, v))
        x[rng.random((n, v)) < 0.2] = -0.0
        x[rng.random((n, v)) < 0.2] = 0.0
    elif kind == "special":
        r = rng.random((n, v))
        x[r < 0.1] = np.nan
        x[(r > 0.2) & (r < 0.3)] = -np.inf
        x[(r > 0.4) & (r < 0.41)] = -3.38e38
        x[(r > 0.5) & (r < 0.51)] = -0.0
    elif kind == "wide":                                        # far from zero on both sides
        x = rng.normal(0, 300, size=(n, v))
    elif kind == "low":                                         # log-probabilities, the largest next to zero
        x = -np.abs(rng.normal(0, 9, size=(n, v))) - 1e-3 * rng.random((n, v))
        x[:, rng.integers(0, v)] = -1e-6
    elif kind == "infinite":
        x[rng.random((n, v)) < 3.0 / v] = np.inf
    elif kind == "none":
        x[:] = -np.inf
        x[rng.random((n, v)) < 0.5] = np.nan
    return x.astype(np.float32)


class Rows:
    """Rows of logits under a random constraint.  States: 0 wide, 1 sparse, 2 one token, 3 nothing, 4 all."""

    def __init__(self, T, kind, n, v, dtype, seed, table="owned", pad=64):
        rng = np.random.default_rng([n, v, seed])
        self.n, self.v, self.rng = n, v, rng
        x = np.full((n, -(-max(v, 1) // pad) * pad), np.nan, dtype=np.float32)
        if v:
            x[:, :v] = logits_of(kind, n, v, rng)
        self.x = torch.from_numpy(x).cuda().to(TYPES[dtype])
        self.logits = self.x[:, :v]
        self.z = self.logits.double().cpu().numpy()
        self.table, self.states, self.on, self.delta = None, None, np.ones((n, v), dtype=bool), None
        if table is not None:
            on = np.zeros((5, v), dtype=bool)
            if v:
                on[0] = rng.random(v) < 0.7
                on[1] = rng.random(v) < min(1.0, 6.0 / v)
                on[2, rng.integers(0, v)] = True
                on[4] = True
            self.delta = np.where(on, rng.integers(0, 5, size=on.shape), DEAD).astype(np.int32)
            d = torch.from_numpy(self.delta).cuda()
            allow = torch.from_numpy(G.bits_from_table(self.delta, T.allow_row_words(v)).view(np.int32)).cuda()
            self.keep = d, allow
            self.table = T.table_wrap(d, allow)
            if table == "owned":
                self.table = T.table_concat([self.table])[0]
            elif table == "packed":
                self.table = T.table_pack(self.table)
            q = rng.integers(-2, 7, size=n)
            q = np.where(rng.random(n) < 0.5, rng.integers(0, 2, size=n), q)
            q[rng.random(n) < 0.2] = 4
            self.q = q
            self.on = np.where(((q >= 0) & (q < 5))[:, None], on[np.clip(q, 0, 4)], False)
            self.states = torch.from_numpy(q.astype(np.int32)).cuda()

    def uniforms(self):
        u = self.rng.random(self.n).astype(np.float32)
        u[self.rng.random(self.n) < 0.1] = 0.0
        u[self.rng.random(self.n) < 0.1] = 1.0
        return u

    def after(self, token, i):
        if not 0 <= self.q[i] < 5:
            return DEAD
        return self.q[i] if token == NO_TOKEN else self.delta[self.q[i], token]


def close(got, want):
    """A log-probability in binary32: the definition's value, rounded, and what the sums lose (2^-40 of them)."""
    if np.isnan(want) or np.isinf(want):
        return (np.isnan(want) and np.isnan(got)) or got == want
    return abs(got - want) <= abs(want) * 2.0 ** -23 + 2.0 ** -39


def check_draw(T, r, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, params=None, in_place=False):
    n = r.n
    tokens = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((n,), 7.0, device="cuda")
    after = None
    if r.table is not None:
        after = r.states.clone() if in_place else torch.full((n,), -7, dtype=torch.int32, device="cuda")
    p = None if params is None else torch.from_numpy(params).cuda()
    T.draw_step(r.table, r.logits, after if in_place else r.states, torch.from_numpy(u).cuda(), tokens, after, temperature=temperature, top_k=top_k,
                top_p=top_p, min_p=min_p, params=p, logprobs=lp)
    tokens, lp = tokens.cpu().numpy(), lp.cpu().numpy()
    for i in range(n):
        s = (temperature, top_k, top_p, min_p) if params is None else params[i]
        want = R.draw(r.z[i], r.on[i], u[i], s[0], int(s[1]), s[2], s[3])
        assert int(tokens[i]) in want, (i, s, u[i], tokens[i], want)
        assert close(lp[i], want[int(tokens[i])]), (i, s, lp[i], want)
        if after is not None:
            assert int(after[i]) == r.after(int(tokens[i]), i), i
    return tokens


SETTINGS = [dict(), dict(temperature=0.7, top_p=0.9), dict(top_k=50, top_p=0.8), dict(temperature=1.3, min_p=0.05), dict(temperature=0.0),
            dict(temperature=0.9, top_k=700, top_p=0.95, min_p=0.01), dict(top_k=1), dict(top_p=0.0), dict(min_p=1.0)]
KINDS = ["open", "peaked", "ties", "equal", "zeros", "special", "wide", "low", "infinite", "none"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 63, 65, 512, 2047, 2049, 4099])
def test_draw_sizes(T, v, dtype):
    r = Rows(T, "peaked", 24, v, dtype, 1)
    for s in SETTINGS:
        check_draw(T, r, r.uniforms(), **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_draw_kinds(T, kind, dtype):
    for v, table in ((3001, "owned"), (9001, None)):
        r = Rows(T, kind, 12, v, dtype, 2, table=table)
        for s in SETTINGS:
            check_draw(T, r, r.uniforms(), **s)


@pytest.mark.parametrize("table", ["wrapped", "owned", "packed", None])
def test_draw_tables(T, table):
    r = Rows(T, "open", 40, 5003, "bf16", 3, table=table)
    for s in SETTINGS[:4]:
        check_draw(T, r, r.uniforms(), in_place=table is not None, **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [32003, 128256, 262147])
def test_draw_long_rows(T, v, dtype):
    for kind, table in (("open", None), ("peaked", "owned"), ("ties", None)):
        r = Rows(T, kind, 5, v, dtype, 4, table=table)
        for s in SETTINGS[:4] + SETTINGS[5:6]:
            check_draw(T, r, r.uniforms(), **s)


def test_draw_params(T):
    """A setting for every row, and values outside their ranges: they are clamped, NaN is no cut."""
    r = Rows(T, "peaked", 64, 2500, "bf16", 5)
    p = np.stack([r.rng.choice([0.0, 0.5, 1.0, 2.0], 64), r.rng.choice([0, 1, 7, 40], 64), r.rng.choice([0.5, 0.9, 1.0], 64),
                  r.rng.choice([0.0, 0.1, 0.5], 64)], 1).astype(np.float32)
    check_draw(T, r, r.uniforms(), params=p)
    u = r.uniforms()
    odd = p.copy()
    for i, row in enumerate([(-1.0, -3.0, 2.0, -1.0), (np.nan, np.nan, np.nan, np.nan), (1.0, 0.5, -1.0, 0.0), (1.0, 3e9, 1.0, 7.0), (np.inf, 5.0, 1.0, 0.0)]):
        odd[i] = row
    plain = p.copy()
    for i, row in enumerate([(0.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 1.0), (np.finfo(np.float32).max, 5, 1.0, 0.0)]):
        plain[i] = row
    got = [torch.empty(64, dtype=torch.int32, device="cuda") for _ in range(2)]
    for t, q in zip(got, (odd, plain)):
        T.draw_step(r.table, r.logits, r.states, torch.from_numpy(u).cuda(), t, torch.empty_like(t), params=torch.from_numpy(q).cuda())
    assert torch.equal(*got)


def test_draw_numbers_outside(T):
    r = Rows(T, "open", 6, 700, "f32", 6, table=None)
    got = []
    for u in ([-1.0, np.nan, 2.0, np.inf, -np.inf, 0.5], [0.0, 0.0, 1.0, 1.0, 0.0, 0.5]):
        t = torch.empty(6, dtype=torch.int32, device="cuda")
        T.draw_step(None, r.logits, None, torch.tensor(u, device="cuda"), t, None)
        got.append(t)
    assert torch.equal(*got)


def test_draw_is_distributed_as_the_softmax(T):
    """Numbers spread evenly over 0 .. 1 draw every token as often as its probability says, to one number."""
    v, n = 300, 4096
    z = torch.randn(v, device="cuda") * 1.5
    u = (torch.arange(n, device="cuda") + 0.5) / n
    t = torch.empty(n, dtype=torch.int32, device="cuda")
    T.draw_step(None, z.expand(n, v).contiguous().view(n, v) if v % 4 == 0 else z.expand(n, v).contiguous(), None, u, t, None)
    share = torch.bincount(t.long(), minlength=v).double()
    assert (share - n * torch.softmax(z.double(), 0)).abs().max().item() <= 1.0 + 1e-6


def test_draw_leaves_what_is_not_its_own(T):
    r = Rows(T, "open", 10, 1000, "bf16", 7)
    t, q, lp = (torch.full((16,), 5, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32))
    T.draw_step(r.table, r.logits, r.states, torch.rand(10, device="cuda"), t, q, logprobs=lp)
    for x in (t, q, lp):
        assert torch.equal(x[10:], torch.full_like(x[10:], 5))
    empty = torch.empty((0, 1000), device="cuda")
    T.draw_step(None, empty, None, torch.empty(0, device="cuda"), t, None)
    assert int(t[10]) == 5


def test_draw_no_tokens(T):
    x = torch.zeros((3, 8), device="cuda")[:, :0]
    t, lp = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    T.draw_step(None, x, None, torch.rand(3, device="cuda"), t, None, logprobs=lp)
    assert t.tolist() == [NO_TOKEN] * 3 and lp.tolist() == [0.0] * 3


def check_top(T, r, k, temperature=1.0):
    ids = torch.full((r.n, k), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((r.n, k), 7.0, device="cuda")
    T.top_logprobs(r.table, r.logits, r.states, ids, lp, temperature=temperature)
    ids, lp = ids.cpu().numpy(), lp.cpu().numpy()
    for i in range(r.n):
        want, want_lp = R.top(r.z[i], r.on[i], k, float(np.float32(temperature)))
        assert np.array_equal(ids[i], want), (i, ids[i], want)
        for x, y in zip(lp[i], want_lp):
            # the sum may be taken in binary32 (2^-21 of it), and so its logarithm
            assert close(x, y) or abs(x - y) <= 2.0 ** -21 + abs(y) * 2.0 ** -22, (i, x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 65, 512, 2049, 4099, 32003, 128256])
def test_top_sizes(T, v, dtype):
    r = Rows(T, "peaked", 12, v, dtype, 11)
    for k in (1, 5, 64, 256):
        check_top(T, r, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_top_kinds(T, kind, dtype):
    for v, table in ((3001, "packed"), (9001, None)):
        r = Rows(T, kind, 8, v, dtype, 12, table=table)
        for k, t in ((1, 1.0), (20, 0.6), (200, 1.4)):
            check_top(T, r, k, t)


def test_top_is_what_token_logprobs_gives(T):
    r = Rows(T, "peaked", 30, 7001, "bf16", 13)
    ids = torch.empty((30, 8), dtype=torch.int32, device="cuda")
    lp = torch.empty((30, 8), device="cuda")
    T.top_logprobs(r.table, r.logits, r.states, ids, lp, temperature=0.8)
    one = torch.empty(30, device="cuda")
    for j in range(8):
        T.token_logprobs(r.table, r.logits, r.states, ids[:, j].contiguous(), one, temperature=0.8)
        some = ids[:, j] != NO_TOKEN
        assert torch.allclose(one[some], lp[:, j][some], rtol=2.0 ** -20, atol=2.0 ** -20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured(T, dtype):
    """Both calls in one graph, replayed with new logits and numbers between eager work."""
    rows = [Rows(T, "peaked", 9, 6007, dtype, 20 + i) for i in range(3)]
    x, states = rows[0].x.clone(), rows[0].states.clone()
    table = rows[0].table
    u = torch.zeros(9, device="cuda")
    t, q, lp = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, device="cuda")
    ids, top = torch.empty((9, 30), dtype=torch.int32, device="cuda"), torch.empty((9, 30), device="cuda")
    ws = torch.empty(max(16, T.select_workspace_bytes(9, 6007)), dtype=torch.uint8, device="cuda")

    def call():
        T.draw_step(table, x[:, :6007], states, u, t, q, temperature=0.9, top_k=3000, top_p=0.9, logprobs=lp, workspace=ws)
        T.top_logprobs(table, x[:, :6007], states, ids, top, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.copy_(rows[i % 3].x)
        u.copy_(torch.from_numpy(rows[i % 3].uniforms()))
        for out in (t, q, lp, ids, top):
            out.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in (t, q, lp, ids, top)]
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, (t, q, lp, ids, top)):
            assert torch.equal(a, b)


def test_two_streams(T):
    r = [Rows(T, "peaked", 30, 20011, "bf16", 30 + i) for i in range(2)]
    u = [torch.from_numpy(x.uniforms()).cuda() for x in r]
    torch.cuda.synchronize()
    out = [[torch.empty(30, dtype=torch.int32, device="cuda") for _ in range(2)] for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i in range(2):
            T.draw_step(r[i].table, r[i].logits, r[i].states, u[i], *out[i], top_p=0.9, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        T.draw_step(r[i].table, r[i].logits, r[i].states, u[i], *out[2 + i], top_p=0.9)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i][0], out[2 + i][0]) and torch.equal(out[i][1], out[2 + i][1])


def test_refusals(T):
    x = torch.zeros((4, 64), device="cuda")
    t, lp, u = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda"), torch.zeros(4, device="cuda")
    draw = lambda *a, **k: T.draw_step(None, *a, **k)
    for bad in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=1.5), dict(top_p=-0.1),
                dict(top_p=float("nan")), dict(min_p=2.0), dict(min_p=float("nan"))):
        with pytest.raises(T.TdfaError):
            draw(x, None, u, t, None, **bad)
    with pytest.raises(TypeError):
        draw(x.half(), None, u, t, None)
    with pytest.raises(ValueError):
        draw(x.t(), None, u, t, None)
    with pytest.raises(ValueError):
        draw(x, None, u[:3], t, None)
    with pytest.raises(ValueError):
        draw(x, None, u.double(), t, None)
    with pytest.raises(ValueError):
        draw(x, None, u, t.long(), None)
    with pytest.raises(ValueError):
        draw(x, None, u, t, None, params=torch.zeros(15, device="cuda"))
    with pytest.raises(T.TdfaError):
        draw(x[:, 1:], None, u, t, None)                        # not aligned
    with pytest.raises(T.TdfaError):
        draw(x, None, u, u.view(torch.int32), None)             # the tokens lie over the numbers
    with pytest.raises(T.TdfaError):
        draw(x, None, u, t, None, logprobs=x[0, :4])            # the log-probabilities lie over the logits
    with pytest.raises(ValueError):
        draw(x.cpu(), None, u, t, None)
    ids, top = torch.empty((4, 5), dtype=torch.int32, device="cuda"), torch.empty((4, 5), device="cuda")
    with pytest.raises(T.TdfaError):
        T.top_logprobs(None, x, None, ids, top, temperature=0.0)
    with pytest.raises(ValueError):
        T.top_logprobs(None, x, None, ids, top[:, :4])
    with pytest.raises(T.TdfaError):
        T.top_logprobs(None, x, None, torch.empty((4, 257), dtype=torch.int32, device="cuda"), torch.empty((4, 257), device="cuda"))
    r = Rows(T, "open", 4, 64, "f32", 1)
    with pytest.raises(ValueError):
        T.draw_step(r.table, r.logits, None, u, t, t.clone())
    with pytest.raises(ValueError):
        T.draw_step(r.table, r.logits, r.states, u, t, None)
    with pytest.raises(ValueError):
        T.draw_step(r.table, r.logits[:, :32], r.states, u, t, t.clone())
    with pytest.raises(T.TdfaError):
        T.draw_step(r.table, r.logits, r.states, u, r.states, t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(T, dtype):
    """Rows whose offsets pass 32 bits, and other strides than the tested ones."""
    v = 3001
    stride = (1 << 30) + 64
    x = torch.empty(2 * stride + 4096, dtype=TYPES[dtype], device="cuda").as_strided((3, v), (stride, 1))
    near = torch.randn((3, 3008), device="cuda").mul_(2).to(TYPES[dtype])[:, :v]
    x.copy_(near)
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    got = []
    for z in (x, near):
        t, lp = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
        ids, top = torch.empty((3, 9), dtype=torch.int32, device="cuda"), torch.empty((3, 9), device="cuda")
        T.draw_step(None, z, None, u, t, None, top_p=0.9, logprobs=lp)
        T.top_logprobs(None, z, None, ids, top)
        got.append((t, lp, ids, top))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 300, 600, 900])
@pytest.mark.parametrize("v", [9001, 33001, 66001])
def test_shapes_agree(T, v, rows, dtype):
    """A row gives the same whatever the rows around it, which the launch shapes go by."""
    if v * rows > 40_000_000:
        pytest.skip("the shapes of fewer tokens cover it")
    r = Rows(T, "peaked", 6, v, dtype, 60)
    rep = -(-rows // 6)
    x = r.x.repeat(rep, 1)[:rows]
    q = r.states.repeat(rep)[:rows].contiguous()
    u = torch.from_numpy(r.uniforms()).cuda().repeat(rep)[:rows].contiguous()
    t, q2, lp = (torch.empty(rows, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32))
    ids, top = torch.empty((rows, 33), dtype=torch.int32, device="cuda"), torch.empty((rows, 33), device="cuda")
    for s in (dict(temperature=0.8, top_p=0.9), dict(top_k=900, min_p=0.001)):
        T.draw_step(r.table, x[:, :v], q, u, t, q2, logprobs=lp, **s)
        for i in range(min(6, rows)):
            want = R.draw(r.z[i], r.on[i], float(u[i]), s.get("temperature", 1.0), s.get("top_k", 0), s.get("top_p", 1.0), s.get("min_p", 0.0))
            assert int(t[i]) in want and close(float(lp[i]), want[int(t[i])])
        for a in (t, q2, lp):
            assert torch.equal(a, a[:6].repeat(rep)[:rows])
    T.top_logprobs(r.table, x[:, :v], q, ids, top)
    assert torch.equal(ids, ids[:6].repeat(rep, 1)[:rows]) and torch.equal(top, top[:6].repeat(rep, 1)[:rows])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1e-3, 0.02, 30.0, 1e4, 1e30])
def test_draw_temperatures(T, dtype, temperature):
    r = Rows(T, "open", 12, 5003, dtype, 61, table=None)
    for s in (dict(), dict(top_p=0.5), dict(top_k=3), dict(min_p=0.3)):
        check_draw(T, r, r.uniforms(), temperature=temperature, **s)
    if temperature > 1e-4:
        check_top(T, r, 10, temperature)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_top_k_ends_in_ties(T, dtype):
    """More tokens share the k-th logit than fit the list: those of the lowest ids, and a draw among all of them."""
    r = Rows(T, "open", 4, 7001, dtype, 62, table=None)
    r.x[:, 100:5100] = 3.0
    r.x[:, 50] = 9.0
    r.z = r.logits.double().cpu().numpy()
    for k in (1, 2, 40, 256):
        check_top(T, r, k)
    for s in (dict(top_k=2), dict(top_k=5000, top_p=0.7), dict(min_p=0.001)):
        check_draw(T, r, r.uniforms(), **s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1e-40, 1e-30, 1e30, 3e38])
def test_top_temperatures_at_the_ends(T, dtype, temperature):
    """Next to no temperature: all of the probability is the largest logit's; a huge one: every token has the same, logits that differ by more
    than binary32 reaches excepted."""
    r = Rows(T, "open", 3, 5003, dtype, 63, table=None)
    r.x[:, 77], r.x[:, 78], r.x[2, 79] = 20.0, 19.0, -3.0e38
    ids, lp = (torch.empty((3, 5), dtype=t, device="cuda") for t in (torch.int32, torch.float32))
    T.top_logprobs(None, r.logits, None, ids, lp, temperature=temperature)
    ids, lp = ids.cpu().numpy(), lp.cpu().numpy()
    assert (ids[:, :2] == [77, 78]).all()
    if temperature < 1:
        assert (lp[:, 0] == 0).all()
        t = float(np.float32(temperature))
        assert np.allclose(lp[:, 1], np.float32(-1 / t) if 1 / t < 3.4e38 else -np.inf, rtol=1e-6)
    else:
        far = 1.0 if temperature == 1e30 else 1.0 - np.exp(-3.0e38 / 3e38)
        want = -np.log(np.array([5003, 5003, 5003 - far]))[:, None]
        # the rounding of the result, and of 5,003 weights next to 1 and their sum by threads: a few units in the last place
        assert np.abs(lp - want).max() <= 1e-6 * 8.6
