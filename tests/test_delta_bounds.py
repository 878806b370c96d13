"""The bound on whole gradients of the gated delta rule tells fp32 arithmetic from arithmetic that loses a third of an operand's bits:
the chunk form in fp64, with one operand at a time kept to two bf16 terms (16 bits) of its three."""
import numpy as np
import pytest
import torch

from tests.block_parity import stored
from tests.delta_bounds import CHUNK, excess, references


def case(N, dk, dv, seed):
    r = np.random.RandomState(seed)
    unit = lambda x: x / np.sqrt((x * x).sum(-1, keepdims=True))
    c = {"dims": (1, 1, 1, N, dk, dv), "scale": dk ** -0.5}
    wide = {"q": unit(r.randn(1, 1, N, dk) + 0.3), "k": unit(r.randn(1, 1, N, dk) + 0.3), "v": r.randn(1, 1, N, dv), "dout": r.randn(1, 1, N, dv),
            "g": -np.exp(r.uniform(-7, 0.5, (1, 1, N))), "beta": r.uniform(0.01, 1, (1, 1, N)), "state": 0.3 * r.randn(1, 1, dk, dv),
            "dstate": 0.1 * r.randn(1, 1, dk, dv)}
    return c | {n: stored(x, "f32")[1] for n, x in wide.items()}


def two_terms(x):
    bf = lambda y: torch.from_numpy(np.ascontiguousarray(y)).float().bfloat16().double().numpy()
    high = bf(x)
    return high + bf(x - high)


def by_chunks(c, short=None):
    """The gradients by chunks of tokens, with the operand `short` at 16 bits."""
    q, k, v, g, beta, dout, dstate = (c[n][0, 0] for n in ("q", "k", "v", "g", "beta", "dout", "dstate"))
    keep = lambda name, x: two_terms(x) if name == short else x
    state, held = c["state"][0, 0], []
    for a in range(0, len(g), CHUNK):
        Q, K, V, G, b = (t[a:a + CHUNK] for t in (q, k, v, g, beta))
        at = np.cumsum(G)
        decay = np.tril(np.exp(np.minimum(at[:, None] - at[None], 0.0)))
        since, left = np.exp(at)[:, None], np.exp(at[-1] - at)[:, None]
        T = np.linalg.inv(np.eye(len(G)) + np.tril(b[:, None] * (K @ K.T) * decay, -1))
        W = T @ (K * b[:, None] * since)
        U = T @ (V * b[:, None]) - W @ state
        new = since[-1] * state + (K * left).T @ U
        held.append((a, Q, K, V, b[:, None], decay, since, left, T, W, U, state, new))
        state = new
    d = {n: np.zeros((1, 1) + t.shape) for n, t in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta))}
    for a, Q, K, V, b, decay, since, left, T, W, U, S0, S1 in reversed(held):
        here, do = slice(a, a + len(Q)), c["scale"] * dout[a:a + len(Q)]
        dU = keep("P", (Q @ K.T) * decay).T @ do + (K * left) @ keep("dS", dstate)
        dX = T.T @ keep("dU", dU)
        dV = b * dX
        M, E = -np.tril((dV @ keep("U", U).T) * decay, -1), keep("E", (do @ keep("U", U).T) * decay)
        dQ = since * (do @ S0.T) + E @ K
        dK = left * (U @ keep("dS1", dstate).T) - since * (dV @ S0.T) + E.T @ Q + M @ K + M.T @ K
        sums = (Q * dQ).sum(-1) - (V * dV).sum(-1)
        for n, t in (("q", dQ), ("k", dK), ("v", dV), ("beta", (dX * U / b).sum(-1)), ("g", np.cumsum(sums[::-1])[::-1] + (dstate * S1).sum())):
            d[n][0, 0, here] = t
        dstate = since[-1] * dstate + (Q * since).T @ do - W.T @ dU
    return d


SHAPES = [(130, 64, 64), (200, 32, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_the_chunk_form_is_the_recurrence(shape):
    c = case(*shape, seed=3)
    worst = excess(c, by_chunks(c), *references(c))
    assert max(worst.values()) < 1e-6, worst


@pytest.mark.parametrize("short,seen", [("P", "v"), ("P", "g"), ("P", "beta"), ("dU", "v"), ("dU", "beta"), ("U", "q"), ("U", "k"), ("E", "q"), ("E", "k")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_an_operand_at_16_bits_is_seen(shape, short, seen):
    c = case(*shape, seed=3)
    assert excess(c, by_chunks(c, short), *references(c))[seen] > 1


@pytest.mark.parametrize("short,seen", [("dS", "v"), ("dS1", "k")])
def test_a_states_gradient_at_16_bits_is_seen(short, seen):
    c = case(130, 64, 64, seed=3)
    assert excess(c, by_chunks(c, short), *references(c))[seen] > 1
