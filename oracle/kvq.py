"""8-bit KV cache and attention over it (fp64, NumPy): the plain definition of bs_kvq_write / read / attention.

A block is 64 tokens of one KV head (K and V apart) with e4m3 codes and a scale 2^e; it is kept here as the values held
(code * 2^e, exact in float64) and e."""
import numpy as np

PAGE = 64
E_MIN, E_MAX = -15, 7
MOST = 448.0 * 2.0 ** E_MAX


def round_e4m3(x):
    """Nearest e4m3 value of |x| <= 448, ties to even: four significant bits, steps of 2^-9 below 2^-6."""
    x = np.asarray(x, dtype=np.float64)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


def exponent(a):
    """Least e in [E_MIN, E_MAX] with a <= 448 * 2^e."""
    for e in range(E_MIN, E_MAX):
        if a <= 448.0 * 2.0 ** e:
            return e
    return E_MAX


def bounded(x):
    """(values with NaN -> 0 and |x| <= MOST, whether any had to be changed)."""
    x = np.asarray(x, dtype=np.float64)
    y = np.clip(np.where(np.isnan(x), 0.0, x), -MOST, MOST)
    return y, bool(np.any(np.isnan(x) | (np.abs(x) > MOST)))


class Slot:
    """One sequence's K or V: rows [n, H, D] in, values held out."""

    def __init__(self, H, D, capacity):
        pages = (capacity + PAGE - 1) // PAGE
        self.value = np.zeros((pages * PAGE, H, D))
        self.e = np.full((pages, H), E_MIN)

    def write(self, pos0, rows):
        rows, out_of_range = bounded(rows)
        n = rows.shape[0]
        for p in range(pos0 // PAGE, (pos0 + n - 1) // PAGE + 1 if n else 0):
            lo, hi = max(pos0, p * PAGE), min(pos0 + n, (p + 1) * PAGE)
            new = rows[lo - pos0:hi - pos0]
            for h in range(rows.shape[1]):
                e = exponent(np.abs(new[:, h]).max())
                if lo > p * PAGE:
                    e = max(e, self.e[p, h])
                    s = 2.0 ** e
                    self.value[p * PAGE:lo, h] = round_e4m3(self.value[p * PAGE:lo, h] / s) * s
                s = 2.0 ** e
                self.value[lo:hi, h] = round_e4m3(new[:, h] / s) * s
                self.e[p, h] = e
        return out_of_range

    def read(self, pos0, n):
        return self.value[pos0:pos0 + n]


def attention(q, k, v, ctx):
    """q [n, Hq, D], k / v [ctx + n, Hkv, D]: (out, sum_t p_t |v_t|, largest sum_d |q_d k_d| / sqrt(D) of a row's scores)."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, mag, most = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq, 1))
    for i in range(n):
        t = ctx + i + 1
        for j in range(Hq):
            z = k[:t, j // G] @ q[i, j] / np.sqrt(D)
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, j], mag[i, j] = p @ v[:t, j // G], p @ np.abs(v[:t, j // G])
            most[i, j] = (np.abs(k[:t, j // G]) @ np.abs(q[i, j])).max() / np.sqrt(D)
    return out, mag, most
