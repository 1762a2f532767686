"""Tunes a small policy that answers under a constraint, from rollouts to both losses.

The policy is a linear head over features of the constraint's state; its answers are calls of one
function, [a-z]{1,8}\\(x="[a-z]*"\\), and the reward of an answer is the share of the letter e in it.
Every round draws answers from the masked softmax (sample_step) and keeps the log-probabilities of
the drawn tokens (token_logprobs), takes policy-gradient steps on them (policy_loss), and then one
step that prefers the better answer of each pair (preference_loss).  The gradients that the library
writes for the logits go on through torch's own backward pass.

    python examples/tune_constrained_policy.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2407_08103_amd as T
from workloads import configs

LENGTH, WIDTH = 16, 64


class Policy:
    """Logits of every state: features of the state times a trained head."""

    def __init__(self, n_states: int, n_tokens: int, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.features = torch.randn((n_states, WIDTH), device="cuda", generator=g) / WIDTH ** 0.5
        self.head = torch.zeros((WIDTH, (n_tokens + 7) // 8 * 8), device="cuda", requires_grad=True)
        self.n_tokens = n_tokens

    def logits(self, states: torch.Tensor) -> torch.Tensor:
        """[rows, n_tokens] in bfloat16, rows 16-byte aligned; a state outside the automaton has those of state 0."""
        return (self.features[states.clamp(min=0).long()] @ self.head).to(torch.bfloat16)[:, :self.n_tokens]


def rollouts(table: T.Table, policy: Policy, start: int, batch: int, seed: int):
    """States, tokens and log-probabilities of `batch` answers, [batch, LENGTH] each."""
    states = torch.full((batch,), start, dtype=torch.int32, device="cuda")
    seen = torch.empty((LENGTH, batch), dtype=torch.int32, device="cuda")
    tokens, logprobs = torch.empty_like(seen), torch.empty((LENGTH, batch), device="cuda")
    for step in range(LENGTH):
        seen[step] = states
        with torch.no_grad():
            x = policy.logits(states)
        T.sample_step(table, x, states, 1.0, seed, step, tokens[step], states)          # a complete answer draws NO_TOKEN
        T.token_logprobs(table, x, seen[step], tokens[step], logprobs[step])
    return seen.t().contiguous(), tokens.t().contiguous(), logprobs.t().contiguous()


def rewards_of(tokens: torch.Tensor, letters: torch.Tensor, wanted: torch.Tensor) -> torch.Tensor:
    live = tokens >= 0
    at = tokens.clamp(min=0).long()
    return (wanted[at] * live).sum(1) / (letters[at] * live).sum(1).clamp(min=1)


def run(rounds: int = 12, batch: int = 64, seed: int = 1, verbose: bool = True):
    w = configs.get("c1")
    dfa = w.dfas[0]
    data, offsets = np.asarray(w.vocab.data), np.asarray(w.vocab.offsets).astype(np.int64)
    vocab = T.Vocab(w.vocab.data, w.vocab.offsets)
    table = T.compile_token_dfa(vocab, T.CharDFA(dfa.trans, dfa.accept, dfa.start))
    counts = [np.add.reduceat(np.append(hit, 0), offsets[:-1]) * (np.diff(offsets) > 0)
              for hit in ((data >= ord("a")) & (data <= ord("z")), data == ord("e"))]
    letters, wanted = (torch.from_numpy(c.astype(np.float32)).cuda() for c in counts)

    policy = Policy(dfa.trans.shape[0], vocab.n_tokens, seed)
    optimizer = torch.optim.Adam([policy.head], lr=0.15)
    history = []
    for k in range(rounds):
        seen, tokens, old = rollouts(table, policy, dfa.start, batch, seed * 1000 + k)
        reward = rewards_of(tokens, letters, wanted)
        history.append(float(reward.mean()))
        rows = seen.view(-1), tokens.view(-1)
        n = rows[0].numel()
        advantages = ((reward - reward.mean()) / (reward.std() + 1e-3)).repeat_interleave(LENGTH).contiguous()
        active = (rows[1] >= 0).float()
        weights = active / active.sum()
        loss, logprobs = torch.empty(1, device="cuda"), torch.empty(n, device="cuda")
        for _ in range(2):
            x = policy.logits(rows[0])
            grad = torch.empty_like(x)
            T.policy_loss(table, x.detach(), *rows, old.view(-1), advantages, loss, logprobs, grad_logits=grad,
                          ref_logprobs=old.view(-1), weights=weights, clip=(0.2, 0.3), kl_coef=0.02)
            optimizer.zero_grad()
            x.backward(grad)
            optimizer.step()
        # the better half of the answers against the worse half, pair by pair; the policy that drew them is the reference
        order = reward.argsort(descending=True)
        pairs = torch.stack([order[:batch // 2], order.flip(0)[:batch // 2]], 1).view(-1)
        seen2, tokens2, ref2 = (a[pairs].reshape(-1).contiguous() for a in (seen, tokens, old))
        begin = torch.arange(0, n + 1, LENGTH, dtype=torch.int32, device="cuda")[:2 * (batch // 2) + 1].contiguous()
        preference, margins = torch.empty(1, device="cuda"), torch.empty(2 * (batch // 2), device="cuda")
        x = policy.logits(seen2)
        grad = torch.empty_like(x)
        T.preference_loss(table, x.detach(), seen2, tokens2, ref2, begin, preference, margins, logprobs[:seen2.numel()], grad_logits=grad, beta=0.2)
        optimizer.zero_grad()
        x.backward(grad)
        optimizer.step()
        if verbose:
            text = b"".join(data[offsets[t]:offsets[t + 1]].tobytes() for t in tokens[int(order[0])].tolist() if t >= 0)
            print(f"round {k}: reward {history[-1]:.3f}  policy loss {float(loss):+.4f}  preference loss {float(preference):.4f}  best {text.decode()}")
    return history, tokens, seen, table


if __name__ == "__main__":
    run()
