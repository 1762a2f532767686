"""Arguments that the calls which choose tokens of rows refuse before they touch the device."""
import ctypes as C

import pytest

A, B, D, E = 0x10000, 0x20000, 0x30000, 0x40000          # addresses that nothing reads
ROWS, N = 4, 64


@pytest.fixture(scope="module")
def lib():
    import paper_2407_08103_amd as T
    return T.lib()


def draw(lib, logits=A, dtype=0, rows=ROWS, n=N, stride=N, uniforms=B, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, params=None, tokens=D, lp=None, table=None):
    return lib.tdfa_draw_step(table, logits, dtype, rows, n, stride, None, uniforms, temperature, top_k, top_p, min_p, params, tokens, None, lp, 0x800000, 1 << 40, None)


def top(lib, logits=A, dtype=0, rows=ROWS, n=N, stride=N, temperature=1.0, k=5, ids=B, lp=D):
    return lib.tdfa_top_logprobs(None, logits, dtype, rows, n, stride, None, temperature, k, ids, lp, 0x800000, 1 << 40, None)


COMMON = [(dict(dtype=2), b"dtype"), (dict(rows=-1), b"rows"), (dict(n=-1), b"n_tokens"), (dict(n=(1 << 24) + 1, stride=1 << 25), b"n_tokens"),
          (dict(stride=N - 1), b"row_stride"), (dict(stride=1 << 40), b"too large"), (dict(logits=None), b"NULL"), (dict(logits=A + 8), b"aligned"),
          (dict(stride=N + 1), b"aligned"), (dict(temperature=-1.0), b"temperature"), (dict(temperature=float("nan")), b"temperature"),
          (dict(temperature=float("inf")), b"temperature")]


@pytest.mark.parametrize("bad,says", COMMON + [(dict(uniforms=None), b"NULL"), (dict(tokens=None), b"NULL"), (dict(top_k=-1), b"top_k"), (dict(top_p=1.01), b"top_p"),
                                               (dict(top_p=float("nan")), b"top_p"), (dict(min_p=-0.1), b"min_p"), (dict(min_p=float("nan")), b"min_p"),
                                               (dict(params=E + 4), b"aligned"), (dict(tokens=B + 8), b"overlaps"), (dict(lp=D + 12), b"overlaps"),
                                               (dict(tokens=A + 4 * N * ROWS - 4), b"overlaps"), (dict(params=E, lp=E + 60), b"overlaps")])
def test_draw(lib, bad, says):
    assert draw(lib, **bad) == -1 and says in lib.tdfa_last_error(), lib.tdfa_last_error()


@pytest.mark.parametrize("bad,says", COMMON + [(dict(temperature=0.0), b"temperature"), (dict(k=0), b"k 0"), (dict(k=257), b"k 257"), (dict(ids=None), b"NULL"),
                                               (dict(lp=None), b"NULL"), (dict(lp=B + 4 * ROWS * 5 - 4), b"overlaps"), (dict(ids=A), b"overlaps")])
def test_top(lib, bad, says):
    assert top(lib, **bad) == -1 and says in lib.tdfa_last_error(), lib.tdfa_last_error()


def test_nothing_to_do(lib):
    """No rows: nothing is read or launched."""
    assert draw(lib, rows=0, logits=None, uniforms=None, tokens=None) == 0
    assert top(lib, rows=0, logits=None, ids=None, lp=None) == 0
    # settings of every row replace those of the call, which are not looked at
    assert draw(lib, rows=0, temperature=-1.0, params=E) == 0


def test_workspace(lib):
    assert lib.tdfa_select_workspace_bytes(0, 0) == 0
    assert lib.tdfa_select_workspace_bytes(-1, 5) == -1 and lib.tdfa_select_workspace_bytes(5, -1) == -1
    assert lib.tdfa_select_workspace_bytes(4096, 1 << 24) >= 0


def distill(lib, logits=A, dtype=0, rows=ROWS, n=N, stride=N, temperature=1.0, k=5, ids=B, values=D, weights=None, tail=0, loss=E, losses=E + 64, grad=None, grad_stride=N,
            ws=0x800000, ws_bytes=4096):
    return lib.tdfa_distill_loss(None, logits, dtype, rows, n, stride, None, temperature, k, ids, values, weights, tail, loss, losses, grad, grad_stride, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,says", COMMON + [(dict(temperature=0.0), b"temperature"), (dict(temperature=1e-45), b"temperature"), (dict(k=0), b"k 0"), (dict(k=257), b"k 257"),
                                               (dict(tail=2), b"tail"), (dict(tail=-1), b"tail"), (dict(ids=None), b"NULL"), (dict(values=None), b"NULL"),
                                               (dict(loss=None), b"NULL"), (dict(losses=None), b"NULL"), (dict(ws=None), b"workspace"), (dict(ws_bytes=31), b"workspace"),
                                               (dict(ws=0x800008), b"aligned"), (dict(losses=D + 16), b"overlaps"), (dict(loss=B), b"overlaps"), (dict(losses=E), b"overlaps"),
                                               (dict(grad=0x90008), b"aligned"), (dict(grad=0x90000, grad_stride=N - 4), b"grad_stride"),
                                               (dict(grad=A + 16), b"overlaps"), (dict(grad=B), b"overlaps"), (dict(grad=0x800000 - 4 * N), b"overlaps")])
def test_distill(lib, bad, says):
    assert distill(lib, **bad) == -1 and says in lib.tdfa_last_error(), lib.tdfa_last_error()


def test_distill_workspace(lib):
    size = lib.tdfa_distill_workspace_bytes
    assert size(0, 0, 1) == 0 and size(-1, 0, 1) == -1 and size(1, -1, 1) == -1 and size(1, 1, -1) == -1
    assert size(2 ** 31 - 1, 1 << 24, 256) >= (2 ** 31 - 1) * (8 + 16 + 8 * 256)
