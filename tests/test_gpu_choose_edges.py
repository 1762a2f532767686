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
