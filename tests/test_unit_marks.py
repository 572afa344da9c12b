"""The closed forms and bounds of unit_marks, on the CPU: results right up to their rounding are taken, and results
that lack a unit of work, or have one twice, are not, wherever it lies in however long a context."""
import math

import numpy as np
import pytest
import torch

import unit_marks as marks


def rounded(out, dtype):
    return torch.from_numpy(out).to(dtype).double().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("n,dv", [(33, 64), (1000, 64), (9000, 128), (40000, 128), (131071, 128), (60000, 256), (300000, 512)])
def test_a_lost_or_doubled_unit_is_seen(n, dv, dtype):
    want, want_lse = marks.expected([n], 1, 2, dv)
    assert not marks.rejected(rounded(want, dtype), want_lse, want, want_lse, dtype, 100)
    count = np.minimum(marks.UNIT, n - np.arange(-(-n // marks.UNIT)) * marks.UNIT).astype(float)
    u = np.arange(len(count))
    c, v = marks.column(u, 0, 0, dv), marks.value(u, dv)
    for odd in (0, 1):
        w = count * (2.0 ** marks.score(c) if odd else 1.0)
        num, den = np.bincount(c, w * v, dv), w.sum()
        assert np.allclose(num / den, want[0, odd]) and np.isclose(math.log(den), want_lse[0, odd])
        for k in (u if len(u) < 400 else np.unique(np.r_[u[:50], u[-50:], u[::max(1, len(u) // 300)]])):
            for sign in (-1, 1):
                other, total = num.copy(), den + sign * w[k]
                other[c[k]] += sign * w[k] * v[k]
                out, lse = want.copy(), want_lse.copy()
                out[0, odd], lse[0, odd] = other / total, math.log(total)
                # by the outputs alone as well as by lse of the head that scores all alike
                assert marks.rejected(rounded(out, dtype), want_lse, want, want_lse, dtype, 100)
                if not odd:
                    assert marks.rejected(rounded(want, dtype), lse, want, want_lse, dtype, 100)


def test_the_closed_form_is_the_attention():
    lens, H, group, dv, window = [70, 0, 200], 2, 3, 16, 90
    there = [np.arange(n) % 37 != 5 for n in lens]
    out, lse = marks.expected(lens, H, group, dv, window, there)
    for r, n in enumerate(lens):
        for head in range(H * group):
            h = head // group
            ks, vs = [], []
            for i in range(max(0, n - window), n):
                if there[r][i]:
                    row = np.zeros(dv)
                    c = marks.column(i // 32, r, h, dv)
                    row[c] = marks.value(i // 32, dv)
                    ks.append(marks.score(c) if head % 2 else 0)
                    vs.append(row)
            if not ks:
                assert np.isneginf(lse[r, head]) and not out[r, head].any()
                continue
            w = np.exp(np.log(2.0) * np.array(ks))
            assert np.allclose((w[:, None] * np.array(vs)).sum(0) / w.sum(), out[r, head]) and np.isclose(np.log(w.sum()), lse[r, head])


def test_values_scores_and_rows_are_exact_in_every_format():
    u = np.arange(5000)
    for dv in (8, 16, 64, 128, 256, 512):
        x = np.r_[marks.value(u, dv), marks.score(marks.column(u, 3, 2, dv))].astype(np.float64)
        for td in (torch.bfloat16, torch.float8_e4m3fn):
            assert np.array_equal(torch.from_numpy(x).to(td).double().numpy(), x)


@pytest.mark.parametrize("lens,per,cost,most,least,window", [([40000], 1, 2, 1024, 2, 0), ([5, 0, 3000, 70], 6, 8, 128, 6, 0), ([1] * 500, 3, 2, 64, 2, 0),
                                                             ([900, 20000], 2, 8, 256, 6, 4096)])
def test_runs_take_every_unit_once(lens, per, cost, most, least, window):
    runs = marks.cut(lens, per, cost, most, least, window)
    assert len(runs) <= most
    seen = [(r, item, u) for run in runs for r, item, u0, u1 in run for u in range(u0, u1)]
    assert len(seen) == len(set(seen)) == sum(marks.units_of(n, window) * per for n in lens)
