"""CPU oracle of the 8-bit cache: plain float64 definitions, one head at a time.  Test infrastructure only.

A head's cache is (k_codes, v_codes [C, d] uint8, k_scale, v_scale [blocks], weight [C] float32, position [C] int32); the
functions change numpy arrays in place or return new ones as they say."""
import math

import numpy as np

NAN_CODE = 0x7F
LARGEST = 448.0


def _code_values():
    out = np.empty(256)
    for c in range(256):
        sign, e, m = (-1.0) ** (c >> 7), (c >> 3) & 15, c & 7
        out[c] = math.nan if (e, m) == (15, 7) else sign * (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


VALUES = _code_values()  # of the 256 e4m3 codes


def scale_for(amax):
    """The smallest power of two, at least 2^-126, with amax / scale <= 448."""
    e = -126
    while amax > LARGEST * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x):
    """Nearest e4m3 codes of |x| <= 448, ties to the even code; not finite: the NaN code."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    grid = VALUES[:127]  # ascending
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(a == grid[hi], hi, code) + np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, NAN_CODE).astype(np.uint8)


def decode(codes, scale, block_tokens):
    """Values of [n, d] codes."""
    return VALUES[codes] * np.repeat(scale, block_tokens)[:len(codes), None]


def finite_amax(x):
    a = np.abs(x[np.isfinite(x)])
    return a.max() if a.size else 0.0


def put_rows(codes, scale, block_tokens, rows, values, staying):
    """In place: `values` into `rows`; a block that takes rows in gets the larger of what they need and, where rows of
    `staying` are in it, what it was."""
    T = block_tokens
    rows, staying = np.asarray(rows, dtype=np.int64), np.asarray(staying, dtype=np.int64)
    for j in np.unique(rows // T):
        mine, old = rows // T == j, staying[staying // T == j]
        now = scale_for(finite_amax(values[mine]))
        was = float(scale[j])
        if old.size:
            now = max(now, was)
            if now > was:
                codes[old] = encode(VALUES[codes[old]] * was / now)
        codes[rows[mine]] = encode(values[mine] / now)
        scale[j] = now


def append(cache, block_tokens, n_old, k_new, v_new, first_position):
    k, v, ks, vs, weight, position = cache
    rows = n_old + np.arange(len(k_new))
    put_rows(k, ks, block_tokens, rows, k_new, np.arange(n_old))
    put_rows(v, vs, block_tokens, rows, v_new, np.arange(n_old))
    weight[rows] = 0.0
    position[rows] = rows if first_position is None else first_position + np.arange(len(rows))


def attention(q, k, v, scale, last):
    """q [R, d]; k, v [n, d] values; row r sees keys 0 .. last[r].  -> out [R, d], lse [R], weights [R, n]."""
    R, n = len(q), len(k)
    out, lse, w = np.zeros((R, v.shape[1])), np.full(R, -math.inf), np.zeros((R, n))
    for r in range(R):
        m = min(last[r] + 1, n)
        with np.errstate(invalid="ignore"):
            z = (k[:m] * q[r]).sum(axis=1) * scale
        top = z.max() if m else -math.inf
        if top == -math.inf:
            continue
        e = np.exp(z - top)
        lse[r] = top + math.log(e.sum())
        w[r, :m] = e / e.sum()
        out[r] = (w[r, :m, None] * v[:m]).sum(axis=0)
    return out, lse, w


def order(x):
    """Integers in the order of IEEE-754 totals, all positive NaNs alike."""
    u = int(np.float32(x).view(np.uint32))
    i = u if u < 1 << 31 else -(u - (1 << 31)) - 1
    return min(i, 0x7F800001)


def choose(weight, position, n, budget, n_recent):
    """(n_kept, row_from [n_kept]): the latest rows, then the heaviest, ties to the lower row; kept rows from n_kept on fill
    the places of those that go."""
    keep = min(budget, n)
    latest = max((int(p) for p in position[:n]), default=0)
    rank = sorted(range(n), key=lambda i: (not int(position[i]) > latest - n_recent, -order(weight[i]) if
                                           not int(position[i]) > latest - n_recent else 0, i))
    kept = set(rank[:keep])
    sources = [i for i in range(keep, n) if i in kept]
    row_from = [i if i in kept else sources.pop(0) for i in range(keep)]
    return keep, np.array(row_from, dtype=np.int32)


def evict(cache, block_tokens, n, budget, n_recent):
    """In place; -> (n_kept, row_from)."""
    k, v, ks, vs, weight, position = cache
    keep, row_from = choose(weight, position, n, budget, n_recent)
    rows = np.arange(keep)
    to = rows[row_from != rows]
    came = row_from[to]
    stay = rows[row_from == rows]
    for codes, scale in ((k, ks), (v, vs)):
        values = VALUES[codes[came]] * scale[came // block_tokens][:, None].astype(np.float64)
        put_rows(codes, scale, block_tokens, to, values, stay)
    weight[to], position[to] = weight[came], position[came]
    return keep, row_from
