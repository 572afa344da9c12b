"""Caches whose attention is known in closed form, so that a unit of work that is lost, doubled or read from another
page shows in full however long the context is.

Unit u (32 tokens) of request r under cache head h has one value column other than zero, column (u + 5 r + 3 h) mod dv,
and in it a number of 1 to 7.  A column then holds few units of a context, and a unit is a large part of its column.
Scores are whole powers of two: even query heads score every token alike, odd ones by 0 to 15, the same for all
units of a column.  Heads of the first kind add up whole numbers only: exact in 32 bits, the weights' rounding included.

The bounds.  u: half a step of the output's type, relative.
  even heads   lse: log2 and the product with log(2), 2^-22 (1 + |lse|).  out: one division, one product, u: u + 2^-22
  odd heads    a weight is 2^(score (1 + 2^-22) - base): 16 * 2^-22 from the exponent, 2^-22 from the exponential; the sum
               of the weights goes through 8 additions a unit of a lane's run and fewer than 100 where sums meet:
               (8 units + 100) 2^-24.  Once in the sum of values, where all weights of a column are equal, once in
               that of the weights.
A column without a token is exactly zero.
"""
import numpy as np
import torch

UNIT = 32
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
SCALE = float(np.float32(np.log(2.0)))


def column(u, r, h, dv):
    return (u + 5 * r + 3 * h) % dv


def value(u, dv):
    return 1 + (u // dv) % 7


def score(c):
    return (7 * c) % 16


def expected(lens, H, group, dv, window=0, there=None):
    """out [R][H group][dv] and lse [R][H group] in 64 bits.  there[r]: which of request r's tokens have a page."""
    R = len(lens)
    out, lse = np.zeros((R, H * group, dv)), np.full((R, H * group), -np.inf)
    for r, n in enumerate(lens):
        at = np.arange(max(0, n - window) if window else 0, max(0, n))
        if there is not None:
            at = at[there[r][at]]
        if not len(at):
            continue
        tokens = np.bincount(at // UNIT)
        u = np.arange(len(tokens))
        for h in range(H):
            c = column(u, r, h, dv)
            for odd in range(min(2, group * H)):
                w = tokens * (2.0 ** score(c) if odd else 1.0)
                row = np.bincount(c, w * value(u, dv), dv) / w.sum()
                heads = [i for i in range(h * group, (h + 1) * group) if i % 2 == odd]
                out[r, heads], lse[r, heads] = row, np.log(w.sum())
    return out, lse


def rejected(out, lse, want, want_lse, dtype, units):
    """What of a result is outside the bounds above: text, empty if nothing.  units: the most of a lane's run."""
    odd = np.arange(want.shape[1]) % 2 == 1
    off = np.where(odd, 17 * 2.0 ** -22 + (8 * units + 100) * 2.0 ** -24, 0.0)
    bad = np.abs(out - want) > (U[dtype] + 2.0 ** -22 + 2 * off)[None, :, None] * np.abs(want)
    bad |= ~np.isfinite(out)
    empty = np.isneginf(want_lse)
    finite = np.where(empty, 0.0, want_lse)
    bad_lse = np.where(empty, ~np.isneginf(lse), ~(np.abs(np.where(empty, 0.0, lse) - finite) <= off + 2.0 ** -22 * (1 + np.abs(finite))))
    if not bad.any() and not bad_lse.any():
        return ""
    return f"{int(bad.sum())} outputs, first at {np.argwhere(bad)[:3].tolist()}, {int(bad_lse.sum())} lse, first at {np.argwhere(bad_lse)[:3].tolist()}"


# ---- the cut of the work among runs, as the kernels make it (csrc/attention_common.h)

def units_of(n, window=0):
    first = max(0, n - window) if window else 0
    return max(1, -(-n // UNIT) - first // UNIT)


def cut(lens, per_request, cost, most, least, window=0):
    """For every run, the parts of items in it: (request, item, first unit, end), units counted in the item."""
    lens = [max(0, int(n)) for n in lens]
    total = sum((units_of(n, window) + cost) * per_request for n in lens)
    n_runs = min(most, -(-total // least))
    each, more = divmod(total, n_runs)
    runs = [[] for _ in range(n_runs)]
    w, at = 0, 0
    end = each + (1 if more else 0)
    for r, n in enumerate(lens):
        for item in range(per_request):
            begin, stop = at, at + units_of(n, window) + cost
            while at < stop:
                to = min(stop, end)
                u0, u1 = max(0, at - begin - cost), max(0, to - begin - cost)
                if u1 > u0:
                    runs[w].append((r, item, u0, u1))
                at = to
                if at == end and w + 1 < n_runs:
                    w += 1
                    end += each + (1 if w < more else 0)
    return runs


def ordinary_runs(lens, fmt, heads, group, dk, dv, P, cus, window=0):
    """Runs of the kernel of ordinary rows: one per wave, four waves a workgroup.  None: a workgroup an item."""
    d = max(dk, dv)
    pad = 64 if d <= 64 else 128 if d <= 128 else 256 if d <= 256 else 576
    unit = UNIT * 2 * pad * {"f32": 4, "bf16": 2, "e4m3": 1}[fmt]
    groups = 1 if unit >= 65536 else 2 if P < 16 else 1 if unit >= 16384 else 2 if unit >= 8192 else 4
    workers, per_request = min(4096, groups * cus), heads * -(-group // 16)
    if len(lens) <= 256 and len(lens) * per_request <= workers and max(units_of(max(0, int(n)), window) for n in lens) <= 24:
        return None
    return cut(lens, per_request, 2, 4 * workers, 2, window)


def latent_runs(lens, heads, group, cus, window=0):
    """Runs of the kernel of latent rows, one per workgroup, and how many there may be."""
    workers = max(1, cus // -(-group // 64))
    workers = workers // 8 * 8 if workers >= 8 else workers
    return cut(lens, heads, 8, workers, 6, window), workers


def most_units(runs):
    return max(u1 - u0 for run in runs for _, _, u0, u1 in run)


def most_pages(runs, lens, P, window=0):
    """The most pages of one item that one run goes through."""
    most = 0
    for run in runs:
        for r, _, u0, u1 in run:
            first = (max(0, lens[r] - window) if window else 0) // UNIT
            t0, t1 = (first + u0) * UNIT, min((first + u1) * UNIT, lens[r])
            most = max(most, (t1 - 1) // P - t0 // P + 1)
    return most


def most_workgroups(runs, waves):
    """The most workgroups that one item is cut among."""
    seen = {}
    for w, run in enumerate(runs):
        for r, item, _, _ in run:
            seen.setdefault((r, item), set()).add(w // waves)
    return max(map(len, seen.values()))
