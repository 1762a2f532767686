"""The distillation loss and its gradient against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import distill_ref as R
from test_gpu_draw import KINDS, Rows

pytestmark = pytest.mark.gpu
DEAD = NO_TOKEN = -1
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}              # a rounding to the type, relative


@pytest.fixture(scope="module")
def T():
    import paper_2407_08103_amd as T
    assert torch.cuda.is_available()
    return T


def slots(r, k, rng, odd=True):
    """A teacher near the student: its k likeliest tokens, mostly allowed, and what a list may hold besides."""
    n, v = r.n, r.v
    ids = np.full((n, k), NO_TOKEN, dtype=np.int32)
    values = np.full((n, k), -np.inf, dtype=np.float32)
    for i in range(n):
        y = np.where(np.isfinite(r.z[i]) & r.on[i], np.clip(r.z[i], -30, 30), -np.inf) + rng.normal(0, 1, v)
        m = min(k, int(np.isfinite(y).sum()))
        if m:
            t = np.argsort(-y, kind="stable")[:m]
            ids[i, :m] = t
            values[i, :m] = y[t] - np.logaddexp.reduce(y[np.isfinite(y)])
        if odd and k > 3 and v:
            what = rng.integers(0, 8)
            if what == 0:
                ids[i, 1] = rng.integers(0, v)                # any token, allowed or not, perhaps named already
                values[i, 1] = -2.0
            elif what == 1:
                ids[i, 2], values[i, 2] = v + rng.integers(0, 3), -1.0
            elif what == 2:
                values[i, 0] = np.nan
            elif what == 3:
                values[i, 0] = np.inf
            elif what == 4:
                ids[i, :] = NO_TOKEN
            elif what == 5:
                ids[i, 1:4] = ids[i, 0]                       # one token in four slots
                values[i, 0:4] = -3.0
            elif what == 6:
                values[i, 0] = -np.inf
    return ids, values


def run(T, r, ids, values, weights, temperature, tail, grad="new"):
    n = r.n
    dev = lambda a: torch.from_numpy(a).cuda()
    loss, losses = torch.full((1,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    x = r.x.clone()
    logits = x[:, :r.v]
    g = None
    if grad == "new":
        g = torch.full_like(r.x, 7.0)[:, :r.v]
    elif grad == "in place":
        g = logits
    T.distill_loss(r.table, logits, r.states, dev(ids), dev(values), loss, losses, grad_logits=g, weights=None if weights is None else dev(weights),
                   temperature=temperature, tail=tail)
    torch.cuda.synchronize()
    if grad == "new":
        assert torch.equal(x.view(torch.uint8), r.x.view(torch.uint8))
    return float(loss), losses.cpu().numpy(), None if g is None else g.double().cpu().numpy()


def check(T, r, dtype, k, temperature=1.0, tail=False, grad="new", weighted=True, odd=True):
    rng = np.random.default_rng([r.n, r.v, k])
    ids, values = slots(r, k, rng, odd)
    weights = rng.random(r.n).astype(np.float32) + 0.1 if weighted else None
    if weighted:
        weights[rng.random(r.n) < 0.15] = 0.0
    w = np.ones(r.n, dtype=np.float32) if weights is None else weights
    loss, losses, g = run(T, r, ids, values, weights, temperature, tail, grad)
    want, each, want_g = R.loss(r.z, r.on, ids, values, w.astype(np.float64), temperature, tail)
    # The sum over the tail is in binary32, 16 to 64 terms by a thread and then a tree, each off by an exponential of 2 units and the
    # rounding of its exponent, which is below 2^-23 of it: 2^-18 of the sum, and so is the part of its logarithm that counts.
    # Beside it the result is rounded.
    lost = 2.0 ** -18
    for i in range(r.n):
        if np.isnan(each[i]):
            assert np.isnan(losses[i]), i
        else:
            assert abs(losses[i] - each[i]) <= lost + abs(each[i]) * 2.0 ** -23, (i, losses[i], each[i])
    if not np.isnan(want):
        assert abs(loss - want) <= lost * np.sum(w) + abs(want) * 2.0 ** -23
    if g is None:
        return
    c = 1.0 / float(np.float32(temperature))
    for i in range(r.n):
        if np.isnan(want_g[i]).any():
            assert np.isnan(g[i]).any(), i
            continue
        inside = (ids[i] >= 0) & (ids[i] < r.v) & np.isfinite(values[i])
        if w[i] == 0 or not (r.on[i] & (r.z[i] > -np.inf))[np.where(inside, ids[i], 0)][inside].any():
            assert (g[i] == 0).all(), i                       # the row takes no part
            continue
        # each of the two terms of a gradient, whose difference it is, is off by 2^-18 of itself (also where they are equal), and the
        # result is rounded
        size = np.abs(want_g[i]) + 2 * w[i] * c * upper(r, i, temperature, ids[i], values[i], tail)
        bad = np.abs(g[i] - want_g[i]) > HALF[dtype] * np.abs(want_g[i]) + lost * size + 2.0 ** -126
        assert not bad.any(), (i, np.flatnonzero(bad)[:5], g[i][bad][:5], want_g[i][bad][:5])
        assert (g[i][~r.on[i]] == 0).all(), i


def upper(r, i, temperature, ids, values, tail):
    """p of every token, and its part of r where there is a tail: what its gradient is a difference of."""
    z = np.where(r.on[i] & ~np.isnan(r.z[i]), r.z[i], -np.inf)
    x = (z - z.max()) / float(np.float32(temperature))
    p = np.exp(x) / np.exp(x).sum()
    if not tail:
        return p
    named = np.zeros(len(p), dtype=bool)
    inside = (ids >= 0) & (ids < len(p)) & np.isfinite(values)
    named[ids[inside]] = True
    y = np.where(named, -np.inf, x)
    if y.max() == -np.inf:
        return p
    y = np.exp(y - y.max())
    return p + y / y.sum()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 65, 512, 2049, 4099, 33001])
def test_sizes(T, v, dtype, tail):
    r = Rows(T, "peaked", 24 if v < 10000 else 8, v, dtype, 41)
    for k in (1, 5, 64, 256):
        check(T, r, dtype, k, tail=tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_kinds(T, kind, dtype, tail):
    for v, table in ((3001, "packed"), (9001, None)):
        r = Rows(T, kind, 10, v, dtype, 42, table=table)
        for k, t in ((1, 1.0), (20, 0.6), (200, 1.7)):
            check(T, r, dtype, k, t, tail)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [65528, 65541, 128256, 131072, 131079, 262147])
def test_long_rows(T, v, dtype):
    for table, tail in (("owned", True), (None, False)):
        r = Rows(T, "peaked", 4, v, dtype, 43, table=table)
        check(T, r, dtype, 100, 0.8, tail)
        check(T, r, dtype, 256, 1.0, True, grad="in place")


@pytest.mark.parametrize("table", ["wrapped", "owned", "packed", None])
def test_tables_and_gradients(T, table):
    r = Rows(T, "open", 30, 5003, "bf16", 44, table=table)
    for grad in ("new", "in place", None):
        check(T, r, "bf16", 40, tail=True, grad=grad)
    check(T, r, "bf16", 40, weighted=False)


def test_many_rows(T):
    r = Rows(T, "open", 3000, 130, "f32", 45)
    check(T, r, "f32", 16, tail=True)


def test_tail_of_next_to_nothing(T):
    """A student that is sure of the listed tokens: what it gives the tail is below the smallest binary32."""
    r = Rows(T, "open", 4, 5000, "f32", 46, table=None)
    r.x[:, :3] = 200.0
    r.z = r.logits.double().cpu().numpy()
    ids = np.tile(np.arange(3, dtype=np.int32), (4, 1))
    values = np.full((4, 3), np.log(0.25), dtype=np.float32)
    _, losses, g = run(T, r, ids, values, None, 1.0, True)
    for i in range(4):
        l, want = R.row(r.z[i], r.on[i], ids[i], values[i], 1.0, True)
        assert abs(losses[i] - l) <= 2.0 ** -18 + abs(l) * 2.0 ** -23
        assert np.abs(g[i] - want).max() <= 2.0 ** -18
    assert l > 40


def test_gradient_is_that_of_differences(T):
    r = Rows(T, "peaked", 3, 40, "f32", 47)
    r.states[:] = 0
    r.q[:] = 0
    r.on[:] = r.delta[0] >= 0
    rng = np.random.default_rng(1)
    ids, values = slots(r, 6, rng, odd=False)
    for tail in (False, True):
        _, _, g = run(T, r, ids, values, None, 0.8, tail)
        for i in range(3):
            for j in range(40):
                # central differences of the definition, off by h^2 / 6 times a third derivative below 2
                h = 1e-4
                up, down = r.z[i].copy(), r.z[i].copy()
                up[j] += h
                down[j] -= h
                d = (R.row(up, r.on[i], ids[i], values[i], 0.8, tail)[0] - R.row(down, r.on[i], ids[i], values[i], 0.8, tail)[0]) / (2 * h)
                assert abs(d - g[i, j]) <= 1e-6, (tail, i, j, d, g[i, j])


def test_no_difference_no_loss(T):
    """A student that is its own teacher: top_logprobs of its logits, with the tail, lose nothing and move nothing."""
    r = Rows(T, "peaked", 20, 4099, "bf16", 48)
    ids, lp = torch.empty((20, 50), dtype=torch.int32, device="cuda"), torch.empty((20, 50), device="cuda")
    T.top_logprobs(r.table, r.logits, r.states, ids, lp, temperature=0.9)
    _, losses, g = run(T, r, ids.cpu().numpy(), lp.cpu().numpy(), None, 0.9, True)
    assert np.abs(losses).max() <= 2.0 ** -17 and np.abs(g).max() <= 2.0 ** -17 / 0.9


def test_draw_list_distill(T):
    """The three calls as they are used: a student draws, the teacher lists on what it has drawn, the student learns."""
    n, v, k, steps = 16, 3001, 20, 6
    r = Rows(T, "peaked", n, v, "bf16", 49)
    states = torch.randint(0, 5, (n,), dtype=torch.int32, device="cuda")
    tokens, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    student = [torch.randn((n, 3008), generator=gen, device="cuda").mul_(2).to(torch.bfloat16) for _ in range(steps)]
    before = []
    for x in student:
        before.append(states.clone())
        T.draw_step(r.table, x[:, :v], states, torch.rand(n, generator=gen, device="cuda"), tokens, states, temperature=0.8, top_p=0.95, logprobs=lp)
    q = torch.cat(before)
    teacher = (torch.cat(student).float() + torch.randn((n * steps, 3008), generator=gen, device="cuda"))
    ids, values = torch.empty((n * steps, k), dtype=torch.int32, device="cuda"), torch.empty((n * steps, k), device="cuda")
    T.top_logprobs(r.table, teacher[:, :v], q, ids, values)
    z = torch.cat(student).float()
    loss, losses = torch.empty(1, device="cuda"), torch.empty(n * steps, device="cuda")
    seen = []
    for _ in range(5):
        grad = torch.zeros_like(z)
        T.distill_loss(r.table, z[:, :v], q, ids, values, loss, losses, grad_logits=grad[:, :v], tail=True)
        seen.append(float(loss))
        z -= 1.0 * grad
    assert seen[0] > 0 and all(np.isfinite(seen))
    on = np.where(((q.cpu().numpy() >= 0) & (q.cpu().numpy() < 5))[:, None], r.delta[np.clip(q.cpu().numpy(), 0, 4)] >= 0, False)
    assert (grad[:, :v].cpu().numpy()[~on] == 0).all() and (grad[:, v:] == 0).all()


def test_captured(T):
    r = [Rows(T, "peaked", 9, 6007, "bf16", 50 + i) for i in range(3)]
    lists = [slots(x, 30, np.random.default_rng(i)) for i, x in enumerate(r)]
    x, ids, values = r[0].x.clone(), torch.from_numpy(lists[0][0]).cuda(), torch.from_numpy(lists[0][1]).cuda()
    loss, losses, grad = torch.empty(1, device="cuda"), torch.empty(9, device="cuda"), torch.zeros_like(x)
    ws = torch.empty(T.distill_workspace_bytes(9, 6007, 30), dtype=torch.uint8, device="cuda")

    def call():
        T.distill_loss(r[0].table, x[:, :6007], r[0].states, ids, values, loss, losses, grad_logits=grad[:, :6007], tail=True, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.copy_(r[i % 3].x)
        ids.copy_(torch.from_numpy(lists[i % 3][0]))
        values.copy_(torch.from_numpy(lists[i % 3][1]))
        for out in (loss, losses, grad):
            out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in (loss, losses, grad)]
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, (loss, losses, grad)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_leaves_what_is_not_its_own(T):
    r = Rows(T, "open", 10, 1001, "bf16", 53)
    ids, values = slots(r, 8, np.random.default_rng(0))
    loss, losses = torch.full((3,), 5.0, device="cuda"), torch.full((16,), 5.0, device="cuda")
    grad = torch.full((12, 1088), 5.0, dtype=torch.bfloat16, device="cuda")
    T.distill_loss(r.table, r.logits, r.states, torch.from_numpy(ids).cuda(), torch.from_numpy(values).cuda(), loss, losses, grad_logits=grad[:10, :1001])
    assert (losses[10:] == 5).all() and (loss[1:] == 5).all() and (grad[10:] == 5).all() and (grad[:, 1001:] == 5).all()


def test_nothing(T):
    loss, losses = torch.full((1,), 5.0, device="cuda"), torch.empty(3, device="cuda")
    none = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    T.distill_loss(None, torch.empty((0, 64), device="cuda"), None, none, none.float(), loss, losses)
    assert float(loss) == 0.0
    x = torch.zeros((3, 8), device="cuda")[:, :0]
    ids = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    loss.fill_(5.0)
    T.distill_loss(None, x, None, ids, ids.float(), loss, losses, grad_logits=x.clone())
    assert float(loss) == 0.0 and losses.tolist() == [0.0] * 3


def test_refusals(T):
    x = torch.zeros((4, 64), device="cuda")
    ids, values = torch.zeros((4, 6), dtype=torch.int32, device="cuda"), torch.zeros((4, 6), device="cuda")
    loss, losses = torch.empty(1, device="cuda"), torch.empty(4, device="cuda")
    call = lambda *a, **k: T.distill_loss(None, *a, **k)
    for bad in (dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=1e-45), dict(grad_logits=x.view(-1)[4:].view(-1)[:240].view(4, 60))):
        with pytest.raises((T.TdfaError, ValueError)):
            call(x, None, ids, values, loss, losses, **bad)
    for a in ((x, None, ids.long(), values, loss, losses), (x, None, ids, values.double(), loss, losses), (x, None, ids, values[:, :5], loss, losses),
              (x, None, ids[:3], values[:3], loss, losses), (x, None, ids, values, loss, losses[:3]), (x, None, ids.t(), values.t(), loss, losses)):
        with pytest.raises(ValueError):
            call(*a)
    with pytest.raises(T.TdfaError):
        call(x, None, torch.zeros((4, 257), dtype=torch.int32, device="cuda"), torch.zeros((4, 257), device="cuda"), loss, losses)
    with pytest.raises(T.TdfaError):
        call(x, None, ids, values, loss, values.view(-1)[:4])                       # the losses lie over the values
    with pytest.raises(ValueError):
        call(x, None, ids, values, loss, losses, grad_logits=x.bfloat16())
    wide = torch.zeros((5, 64), device="cuda")
    with pytest.raises(T.TdfaError):
        call(wide[:4], None, ids, values, loss, losses, grad_logits=wide[1:])       # over the logits, a row later
    with pytest.raises(T.TdfaError):
        call(x, None, ids, values, loss, losses, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(T, dtype):
    """Rows whose offsets pass 32 bits, of the logits and of the gradient."""
    import test_gpu_draw as D
    v, stride = 3001, (1 << 30) + 64
    far = [torch.empty(2 * stride + 4096, dtype=D.TYPES[dtype], device="cuda").as_strided((3, v), (stride, 1)) for _ in range(2)]
    near = torch.randn((3, 3008), device="cuda").mul_(2).to(D.TYPES[dtype])[:, :v]
    far[0].copy_(near)
    ids, lp = torch.empty((3, 9), dtype=torch.int32, device="cuda"), torch.empty((3, 9), device="cuda")
    T.top_logprobs(None, near, None, ids, lp, temperature=1.3)
    got = []
    for z, g in ((far[0], far[1]), (near, torch.empty((3, 3008), dtype=near.dtype, device="cuda")[:, :v])):
        loss, losses = torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
        T.distill_loss(None, z, None, ids, lp, loss, losses, grad_logits=g, tail=True)
        got.append((loss, losses, g))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 41, 600])
@pytest.mark.parametrize("v", [9001, 33001, 70001])
def test_shapes_agree(T, v, rows, dtype):
    """Rows by parts and rows in registers give the same to what their sums' orders leave."""
    r = Rows(T, "peaked", 3, v, dtype, 63)
    ids, values = slots(r, 60, np.random.default_rng(9))
    rep = -(-rows // 3)
    x, q = r.x.repeat(rep, 1)[:rows], r.states.repeat(rep)[:rows].contiguous()
    i2, v2 = torch.from_numpy(ids).cuda().repeat(rep, 1)[:rows].contiguous(), torch.from_numpy(values).cuda().repeat(rep, 1)[:rows].contiguous()
    loss, losses, g = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    T.distill_loss(r.table, x[:, :v], q, i2, v2, loss, losses, grad_logits=g[:, :v], tail=True)
    want, each, want_g = R.loss(r.z, r.on, ids, values, np.ones(3), 1.0, True)
    for i in range(3):
        assert abs(float(losses[i]) - each[i]) <= 2.0 ** -18 + abs(each[i]) * 2.0 ** -23
        got = g[i, :v].double().cpu().numpy()
        size = np.abs(want_g[i]) + 2 * (upper(r, i, 1.0, ids[i], values[i], True) if r.on[i].any() else 0.0)
        assert (np.abs(got - want_g[i]) <= HALF[dtype] * np.abs(want_g[i]) + 2.0 ** -18 * size + 2.0 ** -126).all()
    assert torch.equal(losses, losses[:3].repeat(rep)[:rows])
    assert torch.equal(g[:, :v], g[:3, :v].repeat(rep, 1)[:rows])


def test_two_streams(T):
    r = [Rows(T, "peaked", 30, 20011, "bf16", 64 + i) for i in range(2)]
    lists = [[torch.from_numpy(a).cuda() for a in slots(x, 20, np.random.default_rng(i))] for i, x in enumerate(r)]
    out = [[torch.empty(1, device="cuda"), torch.empty(30, device="cuda"), torch.zeros_like(r[i % 2].x)] for i in range(4)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in range(6):
        for i in range(2):
            T.distill_loss(r[i].table, r[i].logits, r[i].states, *lists[i], out[i][0], out[i][1], grad_logits=out[i][2][:, :20011], tail=True, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        T.distill_loss(r[i].table, r[i].logits, r[i].states, *lists[i], out[2 + i][0], out[2 + i][1], grad_logits=out[2 + i][2][:, :20011], tail=True)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(out[i], out[2 + i]))
