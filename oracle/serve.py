"""TEST INFRASTRUCTURE ONLY: plain forms of the serving operators in 64 bits (numpy), products with
4-bit weights, the paged key/value cache's writes, attention and eviction.
Arrays of 16-bit types come and go as float64; a cache is a dict of arrays (k, v,
with k_books, v_books where it holds symbols; table, lens, mass, pos)."""
import numpy as np

from oracle import philox


def matvec(symbols, codebook, scales, group, x):
    """y and the sum of the terms' absolute values, [m, n_out] each."""
    t = len(codebook)
    w = np.asarray(codebook, dtype=np.float64)[np.minimum(symbols, t - 1)]
    w = w * np.repeat(scales, group, axis=1)[:, : symbols.shape[1]]
    return x @ w.T, np.abs(x) @ np.abs(w).T


def _capacity(c):
    return c["table"].shape[1] * c["k"].shape[2]


def length(c, b):
    return int(min(max(int(c["lens"][b]), 0), _capacity(c)))


def place(c, b, slot):
    """(page, offset) of a slot, or None where it has no page."""
    size = c["k"].shape[2]
    page = int(c["table"][b, slot // size])
    return (page, slot % size) if 0 <= page < c["k"].shape[0] else None


def _rows(c, name, b, head, slots):
    out = []
    for s in slots:
        page, off = place(c, b, s)
        x = c[name][page, head, off]
        if name + "_books" in c:
            x = np.stack((x & 15, x >> 4), -1).reshape(-1)
            x = c[name + "_books"][page, head, off][x]
        out.append(x)
    return np.array(out, dtype=np.float64).reshape(len(slots), -1)


def attention(c, q, scale):
    """out [batch, q_heads, dim], the slots' weights [batch, heads, slots], and
    for tolerances the weighted absolute values (as out) and the largest sum of
    a score's absolute terms per [batch, q_heads]."""
    batch, q_heads, dim = q.shape
    heads = c["k"].shape[1]
    group = q_heads // heads
    out, absolute = np.zeros(q.shape), np.zeros(q.shape)
    mass, terms = np.zeros((batch, heads, _capacity(c))), np.zeros((batch, q_heads))
    for b in range(batch):
        slots = [s for s in range(length(c, b)) if place(c, b, s) is not None]
        for g in range(heads if slots else 0):
            k, v = _rows(c, "k", b, g, slots), _rows(c, "v", b, g, slots)
            for h in range(g * group, (g + 1) * group):
                with np.errstate(invalid="ignore"):
                    z = scale * (k @ q[b, h])
                    terms[b, h] = abs(scale) * (np.abs(k) @ np.abs(q[b, h])).max()
                    if np.all(z == -np.inf):
                        continue
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    out[b, h], absolute[b, h] = p @ v, p @ np.abs(v)
                mass[b, g, slots] += p
    return out, mass, absolute, terms


def round_rows(x, books, counts, seed, word):
    """Symbols of the rows x [n, dim] under codebooks [n, s] (counts of them each;
    0 where that is not 2 to 16)."""
    n, dim = x.shape
    e = np.arange(n * dim, dtype=np.uint64)
    h = e // np.uint64(2)
    w = philox.philox4x32_10(h, h >> np.uint64(32), np.full_like(h, word), np.zeros_like(h),
                             seed, seed >> 32)
    odd = e % np.uint64(2) == 1
    lo, hi = np.where(odd, w[2], w[0]), np.where(odd, w[3], w[1])
    u = (((hi << np.uint64(32)) | lo) >> np.uint64(11)).astype(np.float64).reshape(n, dim)
    u *= 2.0 ** -53
    sym = np.zeros((n, dim), dtype=np.int64)
    for r in range(n):
        t = int(counts[r])
        if t < 2 or t > 16:
            continue
        q = books[r, :t]
        a = np.clip((q[None, :] < x[r][:, None]).sum(1) - 1, 0, t - 2)
        with np.errstate(divide="ignore", invalid="ignore"):
            sym[r] = a + (u[r] < (x[r] - q[a]) / (q[a + 1] - q[a]))
    return sym


def new_slots(c, starts, rows):
    """Sequence and slot of every new row, None for rows that are left out."""
    out = []
    for i in range(rows):
        at = None
        for b in range(len(c["lens"])):
            if starts[b] <= i < starts[b + 1]:
                slot = int(c["lens"][b]) - int(starts[b + 1]) + i
                if 0 <= slot < _capacity(c):
                    at = (b, slot)
        out.append(at)
    return out


def evict(c, keep, recent):
    """mass, pos and lens after it (slots that it does not write as they were),
    and the moves as (sequence, head, from, to)."""
    mass, pos, lens = c["mass"].copy(), c["pos"].copy(), c["lens"].copy()
    moves = []
    for b in range(len(lens)):
        n = length(c, b)
        lens[b] = min(n, keep)
        for h in range(mass.shape[1] if n > keep else 0):
            m, p = mass[b, h], pos[b, h]
            newest = int(p[:n].max())
            key = [(2, 0.0) if int(p[i]) > newest - recent else
                   (0, 0.0) if np.isnan(m[i]) else (1, float(m[i])) for i in range(n)]
            order = sorted(range(n), key=lambda i: (-key[i][0], -key[i][1], i))
            kept = set(order[:keep])
            to = [i for i in range(keep) if i not in kept]
            at = [i for i in range(keep, n) if i in kept]
            for f, t in zip(at, to):
                m[t], p[t] = m[f], p[f]
                moves.append((b, h, f, t))
    return mass, pos, lens, moves
