"""Log probabilities of given tokens, entropy and best alternatives of rows of logits (fp64, NumPy): the plain definition of
bs_token_logprobs."""
import numpy as np


def row(z, token, temperature, n_top):
    """(log p(token), entropy, tokens of the n_top best, their log p) of one row."""
    z = np.asarray(z, dtype=np.float64)
    rank = [j for j in np.argsort(-z, kind="stable") if z[j] > -np.inf][:n_top]      # NaN fails the comparison
    top = np.full(n_top, -1, dtype=np.int32)
    top[:len(rank)] = rank
    lp_top = np.full(n_top, -np.inf)
    if np.isnan(z).any() or np.isposinf(z).any():
        lp_top[:len(rank)] = np.nan
        return np.nan, np.nan, top, lp_top
    m = z.max()
    if m == -np.inf:
        return -np.inf, 0.0, top, lp_top
    y = np.where(z == -np.inf, -np.inf, (z - m) / temperature)
    e = np.exp(y)
    lse = np.log(e.sum())
    entropy = lse - (e * np.where(e > 0, y, 0.0)).sum() / e.sum()
    lp_top[:len(rank)] = (y - lse)[rank]
    return y[token] - lse, entropy, top, lp_top
