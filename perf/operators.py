"""The log-probability and loss operators of the library as cases that can be timed and compared.

A policy that decodes under a constraint draws its tokens from the softmax over the tokens that the
constraint's state allows.  Three operators train and score such a policy on the logits of its
language model: the log-probability of given tokens (with its gradient), the clipped policy loss
with a KL term, and the preference loss of paired sequences.

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
        # one short call scored in a notebook: nothing but latency and launches
        dict(name="logprob_call_4", path="logprob", vocab=512, rows=4, dtype="f32", free=False, temperature=1.0),
        # one sequence, one new token: what a server reports beside the token it has drawn
        dict(name="logprob_token_1", path="logprob", vocab=128256, rows=1, dtype="bf16", free=True, temperature=1.0),
        # a decode step of rollouts: the log-probability of every drawn token, kept for the update
        dict(name="logprob_step_256", path="logprob", vocab=128256, rows=256, dtype="bf16", free=False, temperature=0.7),
        # a reference model scores finished rollouts, logits in fp32, rows of an odd length
        dict(name="logprob_score_f32", path="logprob", vocab=32003, rows=2047, dtype="f32", free=False, temperature=1.0),
        # supervised tuning on answers that follow the constraint: log-probabilities and their gradient
        dict(name="tune_2048", path="tune", vocab=128256, rows=2048, dtype="bf16", free=False, temperature=1.0),
        # the same with a small vocabulary and fp32 logits
        dict(name="tune_f32_700", path="tune", vocab=32000, rows=700, dtype="f32", free=False, temperature=1.0),
        # policy updates: a short answer by itself, where latency counts
        dict(name="policy_answer_24", path="policy", vocab=32000, rows=24, dtype="bf16", free=False, temperature=1.0, low=0.2, high=0.2, kl=0.04),
        # the ordinary update of a group of constrained answers, and the largest case
        dict(name="policy_group_4096", path="policy", vocab=128256, rows=4096, dtype="bf16", free=False, temperature=1.0, low=0.2, high=0.28, kl=0.04),
        # answers without a constraint, and without a KL term
        dict(name="policy_free_1024", path="policy", vocab=128256, rows=1024, dtype="bf16", free=True, temperature=1.0, low=0.2, high=0.2, kl=0.0),
        # fp32 logits of the largest vocabulary
        dict(name="policy_f32_256000", path="policy", vocab=256000, rows=300, dtype="f32", free=False, temperature=0.8, low=0.1, high=0.3, kl=0.1),
        # preferences: a few short pairs, and a batch of ragged ones
        dict(name="preference_4_pairs", path="preference", vocab=32000, rows=90, pairs=4, dtype="bf16", free=False, temperature=1.0, beta=0.1, smoothing=0.0),
        dict(name="preference_32_pairs", path="preference", vocab=128256, rows=2900, pairs=32, dtype="bf16", free=False, temperature=1.0, beta=0.1,
             smoothing=0.1),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    path = rng.choice(["logprob", "tune", "policy", "policy", "preference", "preference"])
    c = dict(path=path, vocab=spread(512, 256000), rows=spread(1, 4096), dtype=rng.choice(["bf16", "bf16", "f32"]), free=rng.random() < 0.3,
             temperature=rng.choice([1.0, round(rng.uniform(0.5, 1.4), 2)]))
    if path == "policy":
        c.update(low=round(rng.uniform(0.1, 0.3), 2), high=round(rng.uniform(0.1, 0.4), 2), kl=rng.choice([0.0, round(rng.uniform(0.01, 0.2), 3)]))
    elif path == "preference":
        c.update(rows=max(2, c["rows"]), beta=round(rng.uniform(0.05, 0.5), 2), smoothing=rng.choice([0.0, 0.1]))
    most = max(work(x)["bytes"] for x in listed())
    while work(c)["bytes"] > most:
        c["rows"] = max(2, c["rows"] * 3 // 4)
    if path == "preference":
        c["pairs"] = min(spread(1, 256), c["rows"] // 2)
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


def prepare(case, seed):
    v, n, g = case["vocab"], case["rows"], _generator(seed, 2)
    s = {"case": case, "table": None, "allow": None, "states": None}
    # as a language model's head leaves them: rows padded to a multiple of 64 columns
    s["logits"] = (torch.randn((n, -(-v // 64) * 64), generator=_generator(seed, 3), device="cuda") * 2.0).to(TYPES[case["dtype"]])
    if not case["free"]:
        delta, s["allow"] = _constraint(case, seed)
        s["states"] = torch.randint(0, STATES, (n,), generator=g, device="cuda", dtype=torch.int32)
        if own:                                                      # the handle that a program keeps beside its constraint
            import paper_2407_08103_amd as T
            s["table"] = T.table_concat([T.table_wrap(delta, s["allow"])])[0]
    # the tokens that such a policy draws, and their log-probabilities as it drew them
    inv = 1.0 / case["temperature"]
    tokens = torch.empty(n, dtype=torch.int64, device="cuda")
    drawn = torch.empty(n, device="cuda")
    for i in range(0, n, 512):
        x = s["logits"][i:i + 512, :v].float() * inv
        if s["allow"] is not None:
            x = x.masked_fill(~_allowed(s["allow"], s["states"][i:i + 512], v), -math.inf)
        u = torch.rand(x.shape, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)
        t = (x - torch.log(-torch.log(u))).argmax(1)
        tokens[i:i + 512] = torch.where(torch.isinf(x.amax(1)), NO_TOKEN, t)
        drawn[i:i + 512] = torch.where(torch.isinf(x.amax(1)), 0.0, torch.log_softmax(x, 1).gather(1, t[:, None])[:, 0])
    row = torch.arange(n, device="cuda")

    def noise(scale):
        return scale * torch.randn(n, generator=g, device="cuda")

    if case["path"] in ("logprob", "tune", "preference") and n >= 64:
        # tokens that come from elsewhere: one in a hundred is not allowed, or not even a token
        other = torch.randint(0, v + 2, (n,), generator=g, device="cuda")
        tokens = torch.where(row % 100 == 63, other, tokens)
    if case["path"] in ("tune", "policy") and n >= 16:
        # answers end at different lengths: one row in twelve is padding
        tokens = torch.where(row % 12 == 11, NO_TOKEN, tokens)
    s["tokens"] = tokens.to(torch.int32)
    s["logprobs"] = torch.empty(n, device="cuda")
    if case["path"] != "logprob":
        s["grad"] = torch.zeros_like(s["logits"])
    active = (tokens != NO_TOKEN).float()
    weights = active / active.sum().clamp(min=1.0)
    if case["path"] == "tune":
        s["stats"] = torch.empty((n, 2), device="cuda")
        s["down"] = -weights
    elif case["path"] == "policy":
        s["weights"] = weights
        # no ratio within rounding of a bound of the clip, where the gradient jumps
        step = noise(0.15)
        for bound in (1.0 - case["low"], 1.0 + case["high"]):
            step = torch.where((step - math.log(bound)).abs() < 1e-3, step + 0.01, step)
        s["old"] = drawn - step
        s["ref"] = drawn + noise(0.3) if case["kl"] else None
        s["advantages"] = torch.randn(-(-n // 64), generator=g, device="cuda").repeat_interleave(64)[:n].contiguous()
        s["loss"] = torch.empty(1, device="cuda")
    elif case["path"] == "preference":
        s["ref"] = drawn + noise(0.3)
        cuts = torch.randint(0, n + 1, (2 * case["pairs"] - 1,), generator=g, device="cuda")
        cuts = torch.cat([cuts.new_zeros(1), cuts.sort().values, cuts.new_full((1,), n)])
        s["begin"] = cuts.to(torch.int32)
        s["loss"], s["rewards"] = torch.empty(1, device="cuda"), torch.empty(2 * case["pairs"], device="cuda")
    return s


# ----------------------------------------------------------------- the plain form
def _distribution(s):
    """The softmax of every row over its allowed tokens: probabilities, and the log-probability of the row's token:
    0 where no token was chosen, -inf where its probability is zero."""
    case = s["case"]
    v, inv = case["vocab"], 1.0 / case["temperature"]
    x = s["logits"][:, :v].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    if s["allow"] is not None:
        x = torch.where(_allowed(s["allow"], s["states"], v), x, -math.inf)
    top = x.amax(1, keepdim=True)
    z = (x - torch.where(torch.isinf(top), 0.0, top)) * inv
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    tokens = s["tokens"].long()
    known = (tokens >= 0) & (tokens < v)
    at = torch.where(known, tokens, 0)[:, None]
    lp = z.gather(1, at)[:, 0] - torch.log(total[:, 0])
    lp = torch.where(known & (x.gather(1, at)[:, 0] > -math.inf), lp, -math.inf)
    lp = torch.where(tokens == NO_TOKEN, 0.0, lp)
    return e / torch.where(total > 0, total, 1.0), lp, torch.isfinite(lp) & (tokens != NO_TOKEN), at


def _gradient(s, p, at, down):
    """down * d lp / d logits, in the type of the logits."""
    g = -p
    g.scatter_add_(1, at, torch.ones_like(g[:, :1]))
    return (g * (down * (1.0 / s["case"]["temperature"]))[:, None]).to(s["logits"].dtype)


def _plain(s):
    case = s["case"]
    p, lp, live, at = _distribution(s)
    if case["path"] == "logprob":
        return [lp]
    if case["path"] == "tune":
        return [lp, _gradient(s, p, at, torch.where(live, s["down"], 0.0))]
    known = torch.where(live, lp, 0.0)
    if case["path"] == "policy":
        live = live & (s["weights"] != 0)
        ratio = torch.exp(known - s["old"])
        free = ratio * s["advantages"]
        clipped = torch.clamp(ratio, 1.0 - case["low"], 1.0 + case["high"]) * s["advantages"]
        each = -torch.minimum(free, clipped)
        down = torch.where(free <= clipped, -free, 0.0)
        if s["ref"] is not None:
            d = s["ref"] - known
            each = each + case["kl"] * (torch.expm1(d) - d)
            down = down - case["kl"] * torch.expm1(d)
        loss = torch.where(live, s["weights"] * each, 0.0).sum()
        lp = torch.where(s["weights"] != 0, lp, 0.0)
        return [loss[None], lp, _gradient(s, p, at, torch.where(live, s["weights"] * down, 0.0))]
    rows = torch.arange(case["rows"], device="cuda")
    inside = (rows >= s["begin"][:-1, None]) & (rows < s["begin"][1:, None])
    rewards = case["beta"] * torch.where(inside, torch.where(live, known - s["ref"], 0.0), 0.0).sum(1)
    gap = rewards[0::2] - rewards[1::2]

    def softplus(x):
        return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-torch.abs(x)))

    eps, n = case["smoothing"], case["pairs"]
    loss = ((1.0 - eps) * softplus(-gap) + eps * softplus(gap)).sum() / n
    down = (eps / (1.0 + torch.exp(-gap)) - (1.0 - eps) / (1.0 + torch.exp(gap))) * (case["beta"] / n)
    down = (torch.stack([down, -down], 1).view(-1, 1) * inside).sum(0)
    return [loss[None], rewards, lp, _gradient(s, p, at, torch.where(live, down, 0.0))]


def run(s):
    if not own:
        return _plain(s)
    import paper_2407_08103_amd as T
    case, v = s["case"], s["case"]["vocab"]
    logits, t = s["logits"][:, :v], case["temperature"]
    if case["path"] == "logprob":
        T.token_logprobs(s["table"], logits, s["states"], s["tokens"], s["logprobs"], temperature=t)
        return [s["logprobs"]]
    grad = s["grad"][:, :v]
    if case["path"] == "tune":
        T.token_logprobs(s["table"], logits, s["states"], s["tokens"], s["logprobs"], temperature=t, stats=s["stats"])
        T.token_logprobs_backward(s["table"], logits, s["states"], s["tokens"], s["stats"], s["down"], grad, temperature=t)
        return [s["logprobs"], grad]
    if case["path"] == "policy":
        T.policy_loss(s["table"], logits, s["states"], s["tokens"], s["old"], s["advantages"], s["loss"], s["logprobs"], grad_logits=grad,
                      ref_logprobs=s["ref"], weights=s["weights"], temperature=t, clip=(case["low"], case["high"]), kl_coef=case["kl"])
        return [s["loss"], s["logprobs"], grad]
    T.preference_loss(s["table"], logits, s["states"], s["tokens"], s["ref"], s["begin"], s["loss"], s["rewards"], s["logprobs"], grad_logits=grad,
                      temperature=t, beta=case["beta"], smoothing=case["smoothing"])
    return [s["loss"], s["rewards"], s["logprobs"], grad]


# ----------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    v, n = case["vocab"], case["rows"]
    tokens = s["tokens"].cpu().numpy().astype(np.int64)
    weights = s["weights"].double().cpu().numpy() if "weights" in s else np.ones(n)
    chosen = (tokens >= 0) & (tokens < v) & (weights != 0)
    probability_zero = (tokens != NO_TOKEN) & (weights != 0)          # unless found otherwise below
    rows_on = None
    if s["allow"] is not None:
        bits = np.unpackbits(s["allow"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :v]
        rows_on = torch.from_numpy(np.concatenate([bits, np.zeros_like(bits[:1])]).astype(bool)).cuda()
        q = s["states"].cpu().numpy().astype(np.int64)
        q = torch.from_numpy(np.where((q < 0) | (q >= STATES), STATES, q)).cuda()
    at = torch.from_numpy(np.where(chosen, tokens, 0)).cuda()

    def log_softmax(i):
        """log p of rows i .. i + 256, -inf for every token of probability zero."""
        x = s["logits"][i:i + 256, :v].double() / case["temperature"]
        dead = torch.isnan(x) if rows_on is None else torch.isnan(x) | ~rows_on[q[i:i + 256]]
        x[dead] = -math.inf
        x -= torch.logsumexp(x, 1, keepdim=True)
        return torch.nan_to_num_(x, nan=-math.inf, neginf=-math.inf)

    lp = np.concatenate([log_softmax(i).gather(1, at[i:i + 256, None])[:, 0].cpu().numpy() for i in range(0, n, 256)])
    lp = np.where(chosen, lp, np.where(probability_zero, -math.inf, 0.0))
    live = chosen & np.isfinite(lp)
    out = [torch.from_numpy(lp)]
    if case["path"] == "logprob":
        return out
    if case["path"] == "tune":
        down = s["down"].double().cpu().numpy()
    elif case["path"] == "policy":
        old, adv = s["old"].double().cpu().numpy(), s["advantages"].double().cpu().numpy()
        r = np.exp(np.where(live, lp, 0.0) - old)
        bounded = np.minimum(np.maximum(r, 1.0 - case["low"]), 1.0 + case["high"])
        each = np.maximum(-r * adv, -bounded * adv)
        down = np.where(r * adv <= bounded * adv, -r * adv, 0.0)
        if s["ref"] is not None:
            back = np.exp(s["ref"].double().cpu().numpy() - np.where(live, lp, 0.0))
            each = each + case["kl"] * (back - np.log(back) - 1.0)
            down = down + case["kl"] * (1.0 - back)
        down = weights * down
        out.insert(0, torch.tensor([float((weights * each)[live].sum())], dtype=torch.float64))
    else:
        begin, ref = s["begin"].cpu().numpy(), s["ref"].double().cpu().numpy()
        over = np.where(live, np.where(live, lp, 0.0) - ref, 0.0)
        rewards = case["beta"] * np.array([over[a:b].sum() for a, b in zip(begin[:-1], begin[1:])])
        gap = rewards[0::2] - rewards[1::2]
        eps, pairs = case["smoothing"], case["pairs"]
        loss = np.mean((1.0 - eps) * np.logaddexp(0.0, -gap) + eps * np.logaddexp(0.0, gap))
        slope = (1.0 / (1.0 + np.exp(-gap)) - (1.0 - eps)) * case["beta"] / pairs
        down = np.zeros(n)
        for k in range(2 * pairs):
            down[begin[k]:begin[k + 1]] = slope[k // 2] if k % 2 == 0 else -slope[k // 2]
        out = [torch.tensor([loss], dtype=torch.float64), torch.from_numpy(rewards)] + out
    down = torch.from_numpy(np.where(live, down, 0.0) / case["temperature"]).cuda()
    grad = torch.empty((n, v), dtype=torch.float64, device="cuda")
    for i in range(0, n, 256):
        g = -torch.exp(log_softmax(i))
        g[torch.arange(len(g), device="cuda"), at[i:i + 256]] += 1.0
        grad[i:i + 256] = torch.where(down[i:i + 256, None] != 0, g * down[i:i + 256, None], 0.0)
    return out + [grad]


# ----------------------------------------------------------------- what a pass cannot do without
def work(case):
    v, n, size = case["vocab"], case["rows"], 2 if case["dtype"] == "bf16" else 4
    share = [1.0] if case["free"] else _allowed_share(v)
    elements = sum(share) / len(share)
    # logits come in groups of 16 bytes: those with an allowed token among them
    groups = sum(1.0 - (1.0 - f) ** (16 // size) for f in share) / len(share)
    read = n * (11 / 12 if case["path"] in ("tune", "policy") and n >= 16 else 1.0)     # rows that are not padding
    moved = read * v * size * groups + (0 if case["free"] else min(n, STATES) * v / 8) + 24 * n
    flops = 4 * read * v * elements
    if case["path"] != "logprob":
        moved += n * v * size
        flops += 4 * read * v * elements
    return {"bytes": moved, "flops": flops}
