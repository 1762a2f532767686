"""The draw from given random numbers, the top log-probabilities and the distillation loss of the library as
cases that can be timed and compared.

A server draws a token for every sequence under its constraint, cut by top-k, top-p and min-p as each
request asks, from random numbers that it brings.  It reports the most likely tokens with their
log-probabilities; a teacher model reports them for texts that its student has drawn, and the student learns from
them: distillation from a teacher's top logits, with the gradient of the student's logits.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes
the call (or computes the same in elementary torch operations), `work` says what a pass cannot do
without, and `exact` gives the outputs from the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

STATES = 128                     # states of the constraint's table
DEAD = NO_TOKEN = -1
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ----------------------------------------------------------------- the cases
def listed():
    return [
        # a draw in a notebook: nothing but latency and launches
        dict(name="draw_call_4", path="draw", vocab=512, rows=4, dtype="f32", free=False, temperature=1.0, top_k=0, top_p=0.9, min_p=0.0, each=False),
        # a server with one sequence and no constraint
        dict(name="draw_token_1", path="draw", vocab=128256, rows=1, dtype="bf16", free=True, temperature=0.8, top_k=0, top_p=0.95, min_p=0.0, each=False),
        # a decode step of a full batch under a constraint
        dict(name="draw_step_256", path="draw", vocab=128256, rows=256, dtype="bf16", free=False, temperature=0.7, top_k=0, top_p=0.9, min_p=0.0, each=False),
        # many requests without a constraint, each with a temperature and cuts of its own
        dict(name="draw_requests_1000", path="draw", vocab=128256, rows=1000, dtype="bf16", free=True, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, each=True),
        # fp32 logits, rows of an odd length, all three cuts
        dict(name="draw_f32_300", path="draw", vocab=32003, rows=300, dtype="f32", free=True, temperature=0.9, top_k=2000, top_p=0.97, min_p=0.002, each=False),
        # what a server reports beside one drawn token
        dict(name="top_token_1", path="top", vocab=128256, rows=1, dtype="bf16", free=True, temperature=1.0, k=20),
        # a teacher reports on the drafts of a student, under the constraint
        dict(name="top_teacher_2048", path="top", vocab=128256, rows=2048, dtype="bf16", free=False, temperature=1.0, k=64),
        # the same with fp32 logits, a smaller vocabulary and longer lists
        dict(name="top_f32_500", path="top", vocab=32000, rows=500, dtype="f32", free=False, temperature=0.7, k=200),
        # one short answer by itself, where latency counts
        dict(name="distill_answer_24", path="distill", vocab=32000, rows=24, dtype="bf16", free=False, temperature=1.0, k=20, tail=False),
        # the ordinary update of a batch of constrained answers, and the largest case
        dict(name="distill_batch_4096", path="distill", vocab=128256, rows=4096, dtype="bf16", free=False, temperature=1.0, k=64, tail=True),
        # answers without a constraint, at a higher temperature, over the listed tokens alone
        dict(name="distill_free_1024", path="distill", vocab=128256, rows=1024, dtype="bf16", free=True, temperature=2.0, k=128, tail=False),
        # fp32 logits of the largest vocabulary
        dict(name="distill_f32_256000", path="distill", vocab=256000, rows=300, dtype="f32", free=False, temperature=1.0, k=32, tail=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    path = rng.choice(["draw", "draw", "top", "distill", "distill"])
    c = dict(path=path, vocab=spread(512, 256000), rows=spread(1, 2048 if path == "draw" else 4096), dtype=rng.choice(["bf16", "bf16", "f32"]),
             free=rng.random() < 0.4, temperature=rng.choice([1.0, round(rng.uniform(0.5, 1.5), 2)]))
    if path == "draw":
        c.update(top_k=rng.choice([0, 0, spread(1, 5000)]), top_p=rng.choice([1.0, round(rng.uniform(0.5, 0.99), 2)]),
                 min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 3)]), each=rng.random() < 0.3)
    else:
        c.update(k=spread(1, 256))
        if path == "distill":
            c.update(tail=rng.random() < 0.5)
    # no more than a third of the largest case, whose inputs take the plain form long enough to sort
    most = max(work(x)["bytes"] for x in listed()) / (1 if path == "distill" else 3)
    while work(c)["bytes"] > most:
        c["rows"] = max(1, c["rows"] * 3 // 4)
    return c


# ----------------------------------------------------------------- inputs
def _allowed_share(vocab):
    """The share of the vocabulary that each state allows: in two of five states one token to 64 (the rest of a
    name, punctuation), in one of four up to a tenth (numbers, identifiers), in the others 0.3 to 0.95 (text in
    quotes); the last state is that of a complete text and allows nothing."""
    share = []
    for s in range(STATES - 1):
        u = (s + 0.5) / (STATES - 1)
        if u < 0.4:
            share.append(min(1.0, 64 ** (u / 0.4) / vocab))
        elif u < 0.65:
            share.append(0.005 * 20 ** ((u - 0.4) / 0.25))
        else:
            share.append(0.3 + 0.65 * (u - 0.65) / 0.35)
    return share + [0.0]


def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 16 + what)


def _constraint(case, seed):
    """Targets of all edges [STATES, vocab] (DEAD: none) and the allowed bits in rows of whole 16 bytes."""
    v, g = case["vocab"], _generator(seed, 1)
    share = torch.tensor(_allowed_share(v), device="cuda")
    on = torch.rand((STATES, v), generator=g, device="cuda") < share[:, None]
    on[torch.arange(STATES - 1), torch.randint(0, v, (STATES - 1,), generator=g, device="cuda")] = True
    delta = torch.randint(0, STATES, (STATES, v), generator=g, device="cuda", dtype=torch.int32)
    delta = torch.where(on, delta, DEAD)
    words = torch.zeros((STATES, -(-v // 128) * 128), dtype=torch.int64, device="cuda")
    words[:, :v] = on
    words = (words.view(STATES, -1, 32) << torch.arange(32, device="cuda")).sum(2)
    return delta, torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _allowed(allow, states, vocab):
    """The allowed tokens of each row's state, as truth values; rows in no state allow nothing."""
    live = (states >= 0) & (states < allow.shape[0])
    words = allow[torch.where(live, states, 0).long()]
    bits = (words[:, :, None] >> torch.arange(32, dtype=torch.int32, device=words.device)) & 1
    return (bits.view(len(states), -1)[:, :vocab] != 0) & live[:, None]


def _language_model(case, g):
    """Rows of logits: most of the vocabulary lies around zero; two rows of three have a few dozen tokens far above the
    others, as where a text goes on predictably, the rest are open."""
    v, n = case["vocab"], case["rows"]
    x = torch.randn((n, -(-v // 64) * 64), generator=g, device="cuda") * 2.0      # rows padded to a multiple of 64 columns, as a head leaves them
    at = torch.randint(0, v, (n, 48), generator=g, device="cuda")
    up = torch.rand((n, 48), generator=g, device="cuda") * 14.0
    return x.scatter_add_(1, at, torch.where((torch.arange(n, device="cuda") % 3 != 2)[:, None], up, 0.0))


def prepare(case, seed):
    v, n, g = case["vocab"], case["rows"], _generator(seed, 2)
    s = {"case": case, "table": None, "allow": None, "states": None, "delta": None}
    x = _language_model(case, _generator(seed, 3))
    s["logits"] = x.to(TYPES[case["dtype"]])
    if not case["free"]:
        s["delta"], s["allow"] = _constraint(case, seed)
        s["states"] = torch.randint(0, STATES, (n,), generator=g, device="cuda", dtype=torch.int32)
        if own:                                                      # the handle that a program keeps beside its constraint
            import paper_2407_08103_amd as T
            s["table"] = T.table_concat([T.table_wrap(s["delta"], s["allow"])])[0]
    if case["path"] == "draw":
        s["uniforms"] = torch.rand(n, generator=g, device="cuda")
        s["params"] = None
        if case["each"]:
            # what requests ask for: plain, greedy, top-p, top-k with top-p, min-p
            kind = torch.randint(0, 5, (n,), generator=g, device="cuda")
            some = torch.rand((n, 4), generator=g, device="cuda")
            s["params"] = torch.stack([torch.where(kind == 1, 0.0, 0.4 + some[:, 0]),
                                       torch.where(kind == 3, (4.0 + 96.0 * some[:, 1]).floor(), 0.0),
                                       torch.where((kind == 2) | (kind == 3), 0.7 + 0.29 * some[:, 2], 1.0),
                                       torch.where(kind == 4, 0.01 + 0.19 * some[:, 3], 0.0)], 1)
        s["tokens"], s["next"] = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        s["logprobs"] = torch.empty(n, device="cuda")
    elif case["path"] == "top":
        s["ids"] = torch.empty((n, case["k"]), dtype=torch.int32, device="cuda")
        s["logprobs"] = torch.empty((n, case["k"]), device="cuda")
    else:
        # the teacher agrees with the student for the most part; it has seen the constraint
        k = min(case["k"], v)
        ids, values = torch.empty((n, k), dtype=torch.int64, device="cuda"), torch.empty((n, k), device="cuda")
        for i in range(0, n, 512):
            y = (x[i:i + 512, :v] * 0.9 + torch.randn((min(512, n - i), v), generator=g, device="cuda")) * (1.0 / case["temperature"])
            if s["allow"] is not None:
                y = y.masked_fill(~_allowed(s["allow"], s["states"][i:i + 512], v), -math.inf)
            ids[i:i + 512] = y.topk(k, 1).indices
            values[i:i + 512] = torch.log_softmax(y, 1).gather(1, ids[i:i + 512])
        ids = torch.where(torch.isfinite(values), ids, NO_TOKEN)
        values = torch.where(ids == NO_TOKEN, -math.inf, values)
        # in one row of sixteen the list is shorter, and its last slot may name a token that the constraint does not allow, or none
        row, slot = torch.arange(n, device="cuda")[:, None], torch.arange(k, device="cuda")
        other = torch.randint(0, v + 2, (n, 1), generator=g, device="cuda")
        other = torch.where((other == ids).any(1, keepdim=True), NO_TOKEN, other)
        ids = torch.where((row % 16 == 5) & (slot >= k - k // 8), torch.where(slot == k - 1, other, NO_TOKEN), ids)
        s["ids"], s["values"] = ids.to(torch.int32), values
        # answers end at different lengths: one row in twelve is padding
        active = (row[:, 0] % 12 != 11).float()
        s["weights"] = active / active.sum().clamp(min=1.0)
        s["loss"], s["losses"], s["grad"] = torch.empty(1, device="cuda"), torch.empty(n, device="cuda"), torch.zeros_like(s["logits"])
    return s


# ----------------------------------------------------------------- the plain form
def _logits(s):
    """Logits as fp32, -inf where a token is not allowed or NaN."""
    x = s["logits"][:, :s["case"]["vocab"]].float()
    x = torch.where(torch.isnan(x), -math.inf, x + 0.0)
    return x if s["allow"] is None else torch.where(_allowed(s["allow"], s["states"], s["case"]["vocab"]), x, -math.inf)


def _plain_draw(s):
    case, n = s["case"], s["case"]["rows"]
    p = s["params"]
    if p is None:
        p = torch.tensor([[case["temperature"], case["top_k"], case["top_p"], case["min_p"]]], device="cuda").expand(n, 4)
    temperature, top_k, top_p, min_p = (p[:, i:i + 1].double() for i in range(4))
    value, order = torch.sort(_logits(s), dim=1, descending=True, stable=True)
    place = torch.arange(value.shape[1], device="cuda")[None]
    top = value[:, :1].double()
    # in 64 bits: where the running sum passes the random number is a border
    z = (value.double() - torch.where(torch.isinf(top), 0.0, top)) / torch.where(temperature > 0, temperature, 1.0)
    w = torch.where((temperature > 0) | (place == 0), torch.exp(z), 0.0)          # at temperature 0 nothing but the first
    kth = value.gather(1, (torch.where(top_k > 0, top_k, math.inf).clamp(max=value.shape[1]) - 1).long())
    w = torch.where(value >= kth, w, 0.0)
    running = torch.cumsum(w, 1)
    # a token stays while the tokens of a larger logit hold less than top_p; the first place of its logit says what they hold
    new = torch.cat([torch.ones_like(value[:, :1], dtype=torch.bool), value[:, 1:] != value[:, :-1]], 1)
    above = (running - w).gather(1, torch.cummax(torch.where(new, place, 0), 1).values)
    kept = ((above < top_p * running[:, -1:]) | (value == value[:, :1])) & (w >= min_p)
    w = torch.where(kept, w, 0.0)
    running = torch.cumsum(w, 1)
    total = running[:, -1:]
    at = (running <= s["uniforms"][:, None].double() * total).sum(1, keepdim=True)
    at = torch.minimum(at, torch.where(w > 0, place, 0).amax(1, keepdim=True))
    some = value[:, :1] > -math.inf
    token = torch.where(some, order.gather(1, at), NO_TOKEN)[:, 0]
    lp = torch.where(some, torch.log(w.gather(1, at) / total), 0.0)[:, 0].float()
    if s["delta"] is None:
        return [token.to(torch.int32), lp]
    after = torch.where(some[:, 0], s["delta"][s["states"].long(), torch.where(some[:, 0], token, 0)], s["states"])
    return [token.to(torch.int32), after, lp]


def _plain_top(s):
    case = s["case"]
    k = case["k"]
    x = _logits(s)
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    top = value[:, :1]
    z = (value - torch.where(torch.isinf(top), 0.0, top)) * (1.0 / case["temperature"])
    lp = (z - torch.log(torch.exp(z).sum(1, keepdim=True)))[:, :k]
    some = value[:, :k] > -math.inf
    ids, lp = torch.where(some, order[:, :k], NO_TOKEN).to(torch.int32), torch.where(some, lp, -math.inf)
    short = k - ids.shape[1]                                         # a vocabulary of fewer tokens
    if short > 0:
        ids = torch.cat([ids, ids.new_full((len(ids), short), NO_TOKEN)], 1)
        lp = torch.cat([lp, lp.new_full((len(ids), short), -math.inf)], 1)
    return [ids, lp]


def _plain_distill(s):
    case, inv = s["case"], 1.0 / s["case"]["temperature"]
    x = _logits(s)
    top = x.amax(1, keepdim=True)
    z = (x - torch.where(torch.isinf(top), 0.0, top)) * inv
    e = torch.exp(z)
    ids = s["ids"].long()
    known = (ids >= 0) & (ids < case["vocab"])
    at = torch.where(known, ids, 0)
    live = known & torch.isfinite(s["values"]) & (x.gather(1, at) > -math.inf)
    a = torch.where(live, s["values"], -math.inf).double()
    if case["tail"]:
        q = torch.exp(a.clamp(max=0.0))
        rest = (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0)
    else:
        q = torch.where(live, torch.exp(a - torch.where(live.any(1, keepdim=True), a.amax(1, keepdim=True), 0.0)), 0.0)
        q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
        rest = torch.zeros_like(q[:, :1])
    mark = torch.zeros_like(e).scatter_add_(1, at, live.float()) > 0
    total, others = e.sum(1, keepdim=True).double(), torch.where(mark, 0.0, e).sum(1, keepdim=True).double()
    rest = torch.where(others > 0, rest, 0.0)
    part = live.any(1, keepdim=True)
    lp = z.gather(1, at).double() - torch.log(total)
    each = torch.where(q > 0, q * (torch.log(q) - lp), 0.0).sum(1)
    each = each + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(others / total)), 0.0)[:, 0]
    w = s["weights"][:, None].double()
    part = part & (w != 0)
    each = torch.where(part[:, 0], each, 0.0)
    loss = (w[:, 0] * each).sum()
    mass = q.sum(1, keepdim=True) + rest
    down = torch.where(part, w * inv, 0.0)
    per = torch.where(part, mass / total, 0.0)
    tail = torch.where(rest > 0, per - rest / others, per)
    grad = e * torch.where(mark, (down * per).float(), (down * tail).float())
    grad.scatter_add_(1, at, torch.where(live & part, -down * q, 0.0).float())
    return [loss.float()[None], each.float(), grad.to(s["logits"].dtype)]


def _plain(s):
    return {"draw": _plain_draw, "top": _plain_top, "distill": _plain_distill}[s["case"]["path"]](s)


def run(s):
    if not own:
        return _plain(s)
    import paper_2407_08103_amd as T
    case = s["case"]
    logits = s["logits"][:, :case["vocab"]]
    if case["path"] == "draw":
        after = None if s["table"] is None else s["next"]
        T.draw_step(s["table"], logits, s["states"], s["uniforms"], s["tokens"], after, temperature=case["temperature"], top_k=case["top_k"],
                    top_p=case["top_p"], min_p=case["min_p"], params=s["params"], logprobs=s["logprobs"])
        return [s["tokens"], s["logprobs"]] if after is None else [s["tokens"], after, s["logprobs"]]
    if case["path"] == "top":
        T.top_logprobs(s["table"], logits, s["states"], s["ids"], s["logprobs"], temperature=case["temperature"])
        return [s["ids"], s["logprobs"]]
    grad = s["grad"][:, :case["vocab"]]
    T.distill_loss(s["table"], logits, s["states"], s["ids"], s["values"], s["loss"], s["losses"], grad_logits=grad, weights=s["weights"],
                   temperature=case["temperature"], tail=case["tail"])
    return [s["loss"], s["losses"], grad]


# ----------------------------------------------------------------- the definition in 64 bits
def _rows64(s, i, count):
    """Rows i .. i + count as float64, -inf for what is not allowed or not a number."""
    x = s["logits"][i:i + count, :s["case"]["vocab"]].double()
    x[torch.isnan(x)] = -math.inf
    if s["allow"] is not None:
        bits = s["allow"][s["states"][i:i + count].long()].cpu().numpy().view(np.uint8)
        on = np.unpackbits(bits, axis=1, bitorder="little")[:, :s["case"]["vocab"]].astype(bool)
        x[torch.from_numpy(~on).cuda()] = -math.inf
    return x


def _exact_draw(s, row, x, settings):
    """One row by its distinct logits, the largest first: how many tokens have each, and what these weigh."""
    temperature, top_k, top_p, min_p = settings
    value, inverse, count = torch.unique(x, return_inverse=True, return_counts=True)
    value, count = value.flip(0).cpu().numpy(), count.flip(0).cpu().numpy()
    if value[0] == -math.inf:
        return NO_TOKEN, 0.0
    if temperature == 0:
        return int(x.eq(x.amax()).nonzero()[0]), 0.0
    w = np.exp((value - value[0]) / temperature)
    mass = w * count
    before = np.cumsum(count) - count                                # tokens of a larger logit
    if top_k > 0:
        mass[before >= top_k] = 0.0
    above = np.cumsum(mass) - mass
    stays = (above < top_p * mass.sum()) & (w >= min_p) & (mass > 0)
    stays[0] = True
    mass[~stays] = 0.0
    upto = np.cumsum(mass)
    target = s["uniforms"][row].item() * upto[-1]
    d = min(int((upto <= target).sum()), int(np.flatnonzero(mass)[-1]))
    nth = min(int((target - (upto[d] - mass[d])) / w[d]), int(count[d]) - 1)
    ids = torch.nonzero(inverse == len(value) - 1 - d)[:, 0]
    return int(ids[nth]), math.log(w[d] / upto[-1])


def exact(case, seed):
    s = prepare(case, seed)
    v, n = case["vocab"], case["rows"]
    if case["path"] == "draw":
        if n > 1500:
            return None
        settings = [(case["temperature"], case["top_k"], case["top_p"], case["min_p"])] * n
        settings = np.array(settings, dtype=np.float32) if s["params"] is None else s["params"].cpu().numpy()
        got = [_exact_draw(s, i, _rows64(s, i, 1)[0], settings[i].astype(np.float64)) for i in range(n)]
        tokens = torch.tensor([t for t, _ in got], dtype=torch.int32)
        lp = torch.tensor([x for _, x in got], dtype=torch.float64)
        if s["delta"] is None:
            return [tokens, lp]
        states, delta = s["states"].cpu(), s["delta"].cpu()
        after = torch.where(tokens == NO_TOKEN, states, delta[states.long(), tokens.clamp(min=0).long()])
        return [tokens, after, lp]
    if case["path"] == "top":
        ids, lp = np.full((n, case["k"]), NO_TOKEN, dtype=np.int32), np.full((n, case["k"]), -math.inf)
        k = min(case["k"], v)
        for i in range(0, n, 256):
            x = _rows64(s, i, 256)
            # ties go to the lowest id: every token whose logit reaches the k-th largest, by logit and then by id
            kth = x.topk(k, 1).values[:, -1:]
            norm = torch.logsumexp(x / case["temperature"], 1).cpu().numpy()
            for r in range(len(x)):
                t = torch.nonzero((x[r] >= kth[r]) & (x[r] > -math.inf))[:, 0]
                y = x[r, t].cpu().numpy()
                t = t.cpu().numpy()
                order = np.lexsort((t, -y))[:k]
                ids[i + r, :len(order)] = t[order]
                lp[i + r, :len(order)] = y[order] / case["temperature"] - norm[r]
        return [torch.from_numpy(ids), torch.from_numpy(lp)]
    losses, grad = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros((n, v), dtype=torch.float64, device="cuda")
    ids, values, weights = s["ids"].long(), s["values"].double(), s["weights"].double()
    for i in range(0, n, 256):
        x = _rows64(s, i, 256) / case["temperature"]
        b = len(x)
        lp = torch.nan_to_num(x - torch.logsumexp(x, 1, keepdim=True), nan=-math.inf, neginf=-math.inf)
        t, a = ids[i:i + b], values[i:i + b]
        inside = (t >= 0) & (t < v)
        mine = torch.where(inside, lp.gather(1, t.clamp(0, v - 1)), -math.inf)
        live = inside & torch.isfinite(mine) & torch.isfinite(a)
        a = torch.where(live, a, -math.inf)
        if case["tail"]:
            q = torch.exp(torch.clamp(a, max=0.0))
        else:
            q = torch.nan_to_num(torch.softmax(a, 1), nan=0.0)
        teacher = torch.zeros_like(lp).scatter_add_(1, torch.where(live, t, 0), torch.where(live, q, 0.0))
        named = torch.zeros_like(lp).scatter_add_(1, torch.where(live, t, 0), live.double()) > 0
        other = torch.where(named, -math.inf, lp)
        ln_tail = torch.logsumexp(other, 1)
        rest = (1.0 - q.sum(1)).clamp(min=0.0) if case["tail"] else torch.zeros(b, dtype=torch.float64, device="cuda")
        rest = torch.where(torch.isfinite(ln_tail), rest, 0.0)
        each = torch.where(live & (q > 0), torch.xlogy(q, q) - q * torch.where(live, mine, 0.0), 0.0).sum(1)
        each += torch.where(rest > 0, torch.xlogy(rest, rest) - rest * torch.where(rest > 0, ln_tail, 0.0), 0.0)
        # the teacher as a distribution over all tokens, its rest in the student's own proportions: the gradient is the difference
        teacher += torch.where((rest > 0)[:, None], rest[:, None] * torch.exp(other - torch.where(rest > 0, ln_tail, 0.0)[:, None]), 0.0)
        on = live.any(1) & (weights[i:i + b] != 0)
        losses[i:i + b] = torch.where(on, each, 0.0)
        g = (torch.exp(lp) * teacher.sum(1, keepdim=True) - teacher) * (weights[i:i + b] / case["temperature"])[:, None]
        grad[i:i + b] = torch.where(on[:, None], g, 0.0)
    return [(weights * losses).sum()[None], losses, grad]


# ----------------------------------------------------------------- what a pass cannot do without
def work(case):
    v, n, size = case["vocab"], case["rows"], 2 if case["dtype"] == "bf16" else 4
    share = [1.0] if case["free"] else _allowed_share(v)
    elements = sum(share) / len(share)
    # logits come in groups of 16 bytes: those with an allowed token among them
    groups = sum(1.0 - (1.0 - f) ** (16 // size) for f in share) / len(share)
    read = n * (11 / 12 if case["path"] == "distill" and n >= 12 else 1.0)               # rows that are not padding
    moved = read * v * size * groups + (0 if case["free"] else min(n, STATES) * v / 8) + 24 * n
    flops = 4 * read * v * elements                                                       # compared, made a weight, added up
    if case["path"] != "draw":
        moved += 8 * n * case["k"]
    if case["path"] == "distill":
        moved += n * v * size
        flops += 4 * read * v * elements
    return {"bytes": moved, "flops": flops}
