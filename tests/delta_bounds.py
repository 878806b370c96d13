"""How near fp32 gradients of the gated delta rule have to come as a whole (2-norm over all elements).

A result is reached through at most n roundings one after the other, n the length of its chain of sums as in the bounds of single
elements.  A rounding is off by up to half a step, 2^-24 relative, evenly spread, so by 2^-24 / sqrt(3) in the root mean square; n of
them, each independent of the others, by sqrt(n / 3) 2^-24.  Relative to what the sums run over: for dq, dk and dv the results of
the single value heads; for dbeta, a sum over value channels, the root of its terms' squares; for dg likewise, over q dq and v dv of
the chunk's tokens from its own on and over dS1 S1, element by element."""
import numpy as np

from oracle import block_oracle as orc

CHUNK = 64


def chain(dk, dv):
    return 3 * (64 + dk + dv)


def references(c):
    """The fp64 gradients dq, dk, dv, dg, dbeta, and the norms to which their errors are related."""
    B, H, Hk, N, dk, dv = c["dims"]
    group = H // Hk
    wide = [np.repeat(c[n], group, 1) for n in ("q", "k")] + [c["v"], c["g"], c["beta"]]
    q, k, v, g, beta = wide
    _, last, held = orc.delta(*wide, c["scale"], c["state"])
    each = orc.delta_gradients(*wide, c["scale"], held, c["dout"], c["dstate"])
    shared = lambda t: t.reshape(B, Hk, group, N, dk).sum(2)
    ref = {"q": shared(each[0]), "k": shared(each[1]), "v": each[2], "g": each[3], "beta": each[4]}
    scale = {n: np.sqrt((t ** 2).sum()) for n, t in zip(("q", "k", "v"), each)}
    rest = v - np.einsum("bhtk,bhtkv->bhtv", k, held * np.exp(g)[..., None, None])
    scale["beta"] = np.sqrt(((each[2] / beta[..., None] * rest) ** 2).sum())
    terms = ((q * each[0]) ** 2).sum(-1) + ((v * each[2]) ** 2).sum(-1)
    total = 0.0
    for a in range(0, N, CHUNK):
        b = min(a + CHUNK, N)
        if b < N:
            after = [t[:, :, b:] for t in wide]
            end, dend = held[:, :, b], orc.delta_gradients(*after, c["scale"], held[:, :, b:], c["dout"][:, :, b:], c["dstate"])[5]
        else:
            end, dend = last, c["dstate"]
        from_here = np.cumsum(terms[:, :, a:b][:, :, ::-1], 2)
        total += (from_here + ((end * dend) ** 2).sum((2, 3))[..., None]).sum()
    scale["g"] = np.sqrt(total)
    return ref, scale


def excess(c, got, ref, scale):
    """Per gradient, its error over what is allowed."""
    n = chain(*c["dims"][4:])
    return {m: float(np.sqrt(((np.asarray(got[m]) - ref[m]) ** 2).sum()) / (np.sqrt(n / 3) * 2.0 ** -24 * scale[m])) for m in ref}
