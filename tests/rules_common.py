"""The decoding rules written out from their definition: once in fp32 with every step rounded (what the adjusted logits must equal
bit for bit) and once in 64 bits."""
import numpy as np


def adjust(x, history, n_prompt, rho=1.0, freq=0.0, pres=0.0, temp=1.0, bias=(), mask=None, dtype=np.float32):
    """One row of logits [vocab]; bias: (token, value) pairs, the last of a token counts; mask: truth values or None."""
    t = dtype
    x = np.asarray(x, t).copy()
    V = len(x)
    old = np.zeros(V, bool)
    new = np.zeros(V, np.int64)
    for i, tok in enumerate(history):
        if 0 <= tok < V:
            if i < n_prompt:
                old[tok] = True
            else:
                new[tok] += 1
    seen = old | (new > 0)
    with np.errstate(all="ignore"):
        x = np.where(seen, np.where(x > 0, x / t(rho), x * t(rho)), x)
        x = np.where(seen, x - t(freq) * new.astype(t), x)
        x = np.where(new > 0, x - t(pres), x)
        add = np.zeros(V, t)
        for tok, v in bias:
            if 0 <= tok < V:
                add[tok] = t(v)
        x = (x + add) / t(temp)
    if mask is not None:
        x = np.where(mask, x, t(-np.inf))
    return x


def softmax(z):
    z = np.asarray(z, np.float64)
    m = z.max() if len(z) else -np.inf
    if m == -np.inf:
        return np.zeros_like(z)
    e = np.exp(z - m)
    return e / e.sum()


def pick(z):
    """The lowest id of the highest value, -1 if nothing is above -inf."""
    return int(np.argmax(z)) if z.max() > -np.inf else -1


def pack(mask):
    """Truth values [rows, vocab] -> int32 words [rows, ceil(vocab / 32)]."""
    mask = np.asarray(mask, bool)
    words = (mask.shape[1] + 31) // 32
    m = np.pad(mask, ((0, 0), (0, words * 32 - mask.shape[1])))
    return np.packbits(m, axis=1, bitorder="little").view("<i4")
