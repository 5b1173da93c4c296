"""The 4-bit cache from its definition, in 64 bits on the host: quantisation of rows, the bytes of the layout, attention."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
PAGE = 256


def quantise(x):
    """x [..., d] -> (codes [..., d] 0..15, scale bytes [..., d / 32])."""
    y = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    ok = np.isfinite(y).all(-1)
    y = np.where(ok[..., None], y, 0.0)
    top = np.abs(y).max(-1)
    m, e = np.frexp(top)                                   # top = m 2^e, m in [0.5, 1)
    byte = np.where(top > 0, np.clip(e - 1 - 2 + (m >= 0.875) + 127, 0, 252), 0)
    z = y / 2.0 ** (byte[..., None] - 127.0)
    dist = np.abs(np.abs(z)[..., None] - VALUES)
    near = dist.min(-1, keepdims=True)
    tied = dist == near                                    # one candidate, or two neighbours: the even code
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), tied.argmax(-1)) + 8 * np.signbit(y)
    code = np.where(ok[..., None], code, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(ok, byte, 255).astype(np.uint8)


def values(code, byte):
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def rounded(x):
    return values(*quantise(x))


class Bytes:
    """The four arrays of one layer, written by the layout's definition."""

    def __init__(self, blocks, n_kv, slots, d, fill=0):
        self.d, self.slots = d, slots
        shapes = ((blocks, n_kv, slots, d // 2), (blocks, n_kv, slots, d // 32),
                  (blocks, n_kv, slots // 8, d // 4, 8, 2), (blocks, n_kv, slots // 8, d // 32, 8))
        self.arrays = [np.full(s, fill, np.uint8) for s in shapes]

    def write(self, block, slot, k, v):
        """Rows k, v [n_kv, d] into one slot."""
        kc, ks, vc, vs = self.arrays
        for x, put in ((k, "k"), (v, "v")):
            c, s = quantise(x)
            two = c[:, 0::2] | (c[:, 1::2] << 4)
            if put == "k":
                kc[block, :, slot], ks[block, :, slot] = two, s
            else:
                vc[block, :, slot // 8, :, slot % 8] = two.reshape(len(x), self.d // 4, 2)
                vs[block, :, slot // 8, :, slot % 8] = s


def place(table, b, slot):
    """(block, slot in it) of a sequence's slot."""
    return (b, slot) if table is None else (int(table[b, slot // PAGE]), slot % PAGE)


def root_paths(parents):
    """[nodes, nodes] truth values: the second is on the first one's path to the root, itself included."""
    m = len(parents)
    a = np.eye(m, dtype=bool)
    for i in range(m):
        if parents[i] >= 0:
            a[i] |= a[parents[i]]
    return a


def attend(q, k_ctx, v_ctx, k, v, parents):
    """One sequence: q [m, heads, d], k_ctx, v_ctx [n, kv, d] as read back, k, v [m, kv, d] or None.  -> (out [m, heads, d], and the
    pieces of a bound on what rounding may do to it: sum p |v|, and the largest over keys of sum |q| |k| / sqrt(d))."""
    m, heads, d = q.shape
    kv = k_ctx.shape[1]
    own = k is not None
    sees = np.ones((m, len(k_ctx)), bool)
    if own:
        k_ctx, v_ctx = np.concatenate((k_ctx, k)), np.concatenate((v_ctx, v))
        sees = np.concatenate((sees, root_paths(parents)), 1)
    out, mass, spread = np.zeros((m, heads, d)), np.zeros((m, heads, d)), np.zeros((m, heads, 1))
    if k_ctx.shape[0] == 0:
        return out, mass, spread
    for h in range(heads):
        kh, vh = k_ctx[:, h // (heads // kv)], v_ctx[:, h // (heads // kv)]
        for i in range(m):
            at = sees[i]
            with np.errstate(all="ignore"):
                s = kh[at] @ q[i, h] / np.sqrt(d)
                p = np.exp(s - s.max())
                p = p / p.sum()
                out[i, h] = p @ vh[at]
                mass[i, h] = p @ np.abs(vh[at])
                spread[i, h] = (np.abs(kh[at]) @ np.abs(q[i, h])).max() / np.sqrt(d)
    return out, mass, spread


def tolerance(out, mass, spread, n_keys, d, bf16):
    """How far a result may be off, by arithmetic.  fp32 sums of d products: a score is off by (d + 8) 2^-24 of sum |q| |k| / sqrt(d) (the
    scale and the subtraction of the maximum among the 8), and by 2^-16 of it where a query goes as bf16 high + low part (2^-8 of the rest,
    which is 2^-8 of it).  A weight is then off by as much, relatively, twice (numerator, and sum of weights), by 2^-16 or, rounded to
    bf16, 2^-8, and by the exponentials' and the sums' (n + 64) 2^-24; 2^-8 for a bf16 result.  A factor of 2 for second-order terms."""
    score = ((d + 8) * 2.0 ** -24 + (0 if bf16 else 2.0 ** -16)) * spread
    weight = 2 * score + (2.0 ** -8 if bf16 else 2.0 ** -16) + (n_keys + 64) * 2.0 ** -24
    return 2 * weight * mass + (2.0 ** -8 * np.abs(out) if bf16 else 2.0 ** -24 * np.abs(out)) + 1e-30
