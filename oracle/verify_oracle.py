"""The verification operators in 64 bits, one definition per function: edits of logits, the paged cache's 8-bit form and its
places, attention of the newest tokens.  numpy only; shares nothing with the library."""
import numpy as np

LARGEST = {"e4m3": 448.0, "int8": 127.0}


def edit_row(z, history, prompt, drafted, repetition=1.0, presence=0.0, frequency=0.0, bias=(), allowed=None):
    """One row of logits: `history` token ids, the first `prompt` of them the prompt; `drafted` the block's tokens before the
    row; `bias` (id, value) pairs, the last one of an id counts; `allowed` truth values."""
    x = np.asarray(z, dtype=np.float64).copy()
    vocab = len(x)
    inside = lambda ids: np.asarray([w for w in ids if 0 <= w < vocab], dtype=np.int64)  # noqa: E731
    after = inside(list(history[prompt:]) + list(drafted))
    for w in set(inside(list(history) + list(drafted)).tolist()):
        x[w] = x[w] / repetition if x[w] > 0 else x[w] * repetition
    ids, counts = np.unique(after, return_counts=True)
    x[ids] -= frequency * counts + presence
    for w, v in dict(bias).items():
        if 0 <= w < vocab:
            x[w] += v
    if allowed is not None:
        x[~np.asarray(allowed, dtype=bool)] = -np.inf
    return x


def held(x, store):
    """(held values, scale) of the 8-bit form of rows x [..., dim]."""
    x = np.asarray(x, dtype=np.float64)
    most = LARGEST[store]
    scale = np.maximum((np.abs(x).max(-1) / most), 2.0 ** -100).astype(np.float32)
    t = x / scale.astype(np.float64)[..., None]
    if store == "int8":
        return np.clip(np.rint(t), -127, 127), scale
    _, e = np.frexp(t)
    unit = np.ldexp(1.0, np.maximum(e, -5) - 4)
    return np.clip(np.rint(t / unit) * unit, -448, 448), scale


def place(position, table_row, page_size, pages):
    """(page, place in it) of a position, or None."""
    if position < 0 or position // page_size >= len(table_row):
        return None
    page = int(table_row[position // page_size])
    return (page, position % page_size) if 0 <= page < pages else None


def attend_row(q, position, k, v, there, scale, window=0):
    """(row, log-sum, sum of p |v|, largest sum of scale |q| |k| over the seen keys) of one query at `position`; k, v [length,
    dim], `there` the keys that have a place."""
    j = np.arange(len(k))
    see = (j <= position) & there
    if window:
        see &= j > position - window
    dim = k.shape[1] if len(k) else len(q)
    if not see.any():
        return np.zeros(dim), -np.inf, np.zeros(dim), 0.0
    s = scale * (k[see] @ q)
    top = s.max()
    e = np.exp(s - top)
    p = e / e.sum()
    return p @ v[see], top + np.log(e.sum()), p @ np.abs(v[see]), abs(scale) * float((np.abs(k[see]) @ np.abs(q)).max())
