"""Plain numpy float64 definitions of what the target model needs around a verification: its cache in 8 bits (e4m3 codes, a power of
two as scale per block of 32 positions and head), tree attention over it, its distributions from its logits.  Written from the
definitions; shares no code with the GPU path.  The method's tree attention: Section 3 (token tree verification)."""
import math

import numpy as np

BLOCK = 32
LARGEST = 448.0
LEAST_EXP = -100


# ---------------------------------------------------------------------------------------- e4m3
def e4m3_values():
    """float64 [256]: what each code stands for (sign, 4 exponent bits with bias 7, 3 fraction bits; 0x7F and 0xFF are NaN)."""
    out = np.empty(256)
    for code in range(256):
        exp, frac = (code >> 3) & 15, code & 7
        v = frac * 2.0 ** -9 if exp == 0 else (8 + frac) * 2.0 ** (exp - 10)
        out[code] = math.nan if code & 127 == 127 else -v if code & 128 else v
    return out


VALUES = e4m3_values()


def e4m3_round(x):
    """The nearest e4m3 values of x (|x| <= 448 or NaN), of two equally near ones the one with an even fraction."""
    grid = VALUES[:127]                                       # ascending
    mag = np.abs(x)
    at = np.clip(np.searchsorted(grid, np.nan_to_num(mag)), 1, 126)
    lo, hi = grid[at - 1], grid[at]
    up = (mag - lo > hi - mag) | ((mag - lo == hi - mag) & (at % 2 == 0))
    return np.where(np.isnan(x), math.nan, np.copysign(np.where(up, hi, lo), x))


def scale_of(x):
    """The block's scale: the least power of two, 2^-100 or more, with |x| <= 448 scale for every finite x."""
    finite = np.abs(x[np.isfinite(x)])
    largest = finite.max() if finite.size else 0.0
    e = LEAST_EXP
    while largest > LARGEST * 2.0 ** e:
        e += 1
    return 2.0 ** e


# ---------------------------------------------------------------------------------------- cache
def write(values, scales, first_block, length, rows):
    """rows [n, heads, d] behind the `length` positions of the sequence whose blocks start at first_block.
    values [blocks, heads, 32, d]: what the codes stand for without their scales; scales [blocks, heads].  Both are changed."""
    n, heads, _ = rows.shape
    rows = np.where(np.isfinite(rows), rows, math.nan)
    done = 0
    while done < n:
        block, t = first_block + (length + done) // BLOCK, (length + done) % BLOCK
        part = rows[done:done + BLOCK - t]
        for h in range(heads):
            s = scale_of(part[:, h])
            if t:
                s = max(s, scales[block, h])
                values[block, h, :t] = e4m3_round(values[block, h, :t] * (scales[block, h] / s))
            values[block, h, t:t + len(part)] = e4m3_round(part[:, h] / s)
            values[block, h, t + len(part):] = 0.0
            scales[block, h] = s
        done += len(part)


def read(values, scales, first_block, start, n):
    """[n, heads, d]: positions start .. start + n - 1 of a sequence."""
    at = np.arange(start, start + n)
    block, t = first_block + at // BLOCK, at % BLOCK
    return values[block, :, t] * scales[block][:, :, None]


def place(kind, t, j):
    """The byte of dim j of position t in its block ("k" or "v")."""
    if kind == "k":
        return ((j // 32 * 2 + j // 16 % 2) * 32 + t) * 16 + j % 16
    return ((j // 32 * 2 + t // 4 % 2) * 32 + j % 32) * 16 + t // 8 * 4 + t % 4


def path_rows(n_accepted, path, rows):
    """The tree's rows that a write takes: node 0 and the accepted path, up to an entry that is no row."""
    if n_accepted < 0:
        return []
    take = [0]
    for node in path[:n_accepted]:
        if not 0 <= node < rows:
            break
        take.append(int(node))
    return take


# ---------------------------------------------------------------------------------------- attention
def tree_attention(parent, q, key, value, own_k, own_v, scale):
    """q [nodes, n_heads, d]; key, value [len, n_kv_heads, d]: what is cached; own_k, own_v [nodes, n_kv_heads, d] or None.
    Returns out [nodes, n_heads, d], lse [nodes, n_heads]; rows are independent, a hidden row is not looked at."""
    nodes, nq, d = q.shape
    grp = nq // key.shape[1]
    out, lse = np.zeros((nodes, nq, d)), np.full((nodes, nq), -math.inf)
    for s in range(nodes):
        seen, u = [], s
        while u != -1:
            seen.append(u)
            u = parent[u]
        for h in range(nq):
            k, v = key[:, h // grp], value[:, h // grp]
            if own_k is not None:
                k, v = np.concatenate((k, own_k[seen, h // grp])), np.concatenate((v, own_v[seen, h // grp]))
            if not len(k):
                continue
            x = scale * (k @ q[s, h])
            m = x.max()
            p = np.exp(x - m)
            out[s, h], lse[s, h] = (p / p.sum()) @ v, m + math.log(p.sum())
    return out, lse


# ---------------------------------------------------------------------------------------- distributions
def distribution(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(p, margin) of one row: the kept tokens' probabilities, and how near (relative to the whole mass) another choice of them was."""
    x = np.asarray(logits, dtype=np.float64)
    n = len(x)
    if np.isnan(x).any() or (x == math.inf).any():
        return np.full(n, math.nan), math.inf
    if (x == -math.inf).all():
        return np.zeros(n), math.inf
    if not temperature > 0:
        temperature, top_k = 1.0, 1
    order = np.lexsort((np.arange(n), -x))
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.where(x > -math.inf, np.exp((x - x.max()) / temperature), 0.0)
    margin = math.inf
    if 1 <= top_k < n:
        order = order[:top_k]
    if top_p < 1:
        so_far = np.cumsum(e[order].astype(np.longdouble))
        short = so_far < top_p * so_far[-1]
        margin = float(np.abs(so_far - top_p * so_far[-1]).min() / so_far[-1])
        order = order[:max(1, int(short.sum()) + 1)]
    if min_p > 0:
        least = min(min_p, 1.0)
        away = np.abs(e[order[1:]] - least)
        margin = min(margin, away[away > 0].min(initial=math.inf))
        order = order[e[order] >= least]
    p = np.zeros(n)
    p[order] = e[order] / math.fsum(e[order])
    return p, margin


def draw(p, r):
    """(id, margin): the number of ids whose cumulative sum is <= r * sum, at most the last one with mass; the distance of the nearest sum."""
    if not p.sum() > 0:
        return -1, math.inf
    c = np.cumsum(p)
    at = min(int((c <= r * c[-1]).sum()), int(np.nonzero(p)[0][-1]))
    return at, float(np.abs(c[p > 0] - r * c[-1]).min() / c[-1]) if (p > 0).sum() > 1 else math.inf
