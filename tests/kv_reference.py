"""Plain 64-bit forms of the paged-cache operators, on the host, and the bounds their outputs are held to."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step, relative to the value


def tables(lens, add, table, ring, pool, page_size, max_new):
    """One step, request by request.  Returns the outputs as a dict of numpy arrays."""
    P, M, N = page_size, table.shape[1], len(ring)
    cap = M * P
    lens = [min(max(int(n), 0), cap) for n in lens]
    table, ring = table.copy(), ring.copy()
    take, back = int(pool[0]), int(pool[1])
    spare = min(max(back - take, 0), N)
    slots, positions, off, after = [], [], [0], []
    want_pages = want_tokens = 0
    for r, n in enumerate(lens):
        a, got = int(add[r]), 0
        if a > 0 and n + a <= cap:
            pages = -(-(n + a) // P) - -(-n // P)
            want_pages += pages
            want_tokens += a
            if want_pages <= spare and want_tokens <= max_new:
                got = a
                for c in range(-(-n // P), -(-(n + a) // P)):
                    table[r, c] = ring[take % N]
                    take += 1
                for p in range(n, n + a):
                    page = int(table[r, p // P])
                    slots.append(page * P + p % P if 0 <= page < N else -1)
                    positions.append(p)
        after.append(0 if a < 0 else n + got)
        off.append(off[-1] + got)
    for r, n in enumerate(lens):
        if add[r] < 0:
            for c in range(-(-n // P)):
                ring[back % N] = table[r, c]
                back += 1
    rest = [-1] * (max_new - len(slots))
    i32 = lambda x: np.asarray(x, dtype=np.int32)  # noqa: E731
    return dict(slots=i32(slots + rest), positions=i32(positions + rest), token_off=i32(off), lens=i32(after).reshape(len(lens)), table=table,
                ring=ring, pool=np.asarray([take, back], dtype=np.int64))


def rows_of(pages, scale, table, lens, r, h, lo):
    """The cached rows of request r's tokens lo .. lens[r] under head h as float64, and which of them have a page."""
    P = pages.shape[2]
    at = torch.arange(lo, lens)
    page = table[r, at // P].long()
    there = (page >= 0) & (page < pages.shape[0])
    page = torch.where(there, page, 0)
    x = pages[page, h, at % P].double()
    if scale is not None:
        x = x * scale[page, h, at % P].double()[:, None]
    return x, there


def attention(q, k, v, k_scale, v_scale, lens, table, scale, window=0, dv=None):
    """out, lse and the bound on the error of out, all float64 on the host.

    The bound, per output element, with A = sum p |V| / sum p and u a relative rounding:
      scores   a sum of dk products in 32 bits, and the scale: (dk + 4) 2^-24 scale sum |q K| =: e, and 4 2^-24 in the
               exponential; both in the numerator and in the denominator: 2 (e + 2^-22) A
      sums     of n terms in 32 bits, rescaled at most n times on the way: 4 (n + 8) 2^-24 A
      weights  rounded to bf16 in front of the second product (16- and 8-bit values): 2^-8 A
      result   rounded to its type: u |out|
    """
    q, k, table = q.cpu().double(), k.cpu(), table.cpu()
    v = None if v is None else v.cpu()
    k_scale = None if k_scale is None else k_scale.cpu()
    v_scale = None if v_scale is None else v_scale.cpu()
    R, Hq, dk = q.shape
    H, P = k.shape[1], k.shape[2]
    group = Hq // H
    dv = v.shape[3] if v is not None else dv
    f32 = k.dtype == torch.float32
    out, bound = torch.zeros((R, Hq, dv), dtype=torch.float64), torch.zeros((R, Hq, dv), dtype=torch.float64)
    lse, lse_bound = torch.full((R, Hq), -math.inf, dtype=torch.float64), torch.zeros((R, Hq), dtype=torch.float64)
    for r in range(R):
        n = min(int(lens[r]), table.shape[1] * P)
        if n <= 0:
            continue
        lo = max(0, n - window) if window else 0
        for h in range(H):
            kk, there = rows_of(k, k_scale, table, n, r, h, lo)
            vv = rows_of(v, v_scale, table, n, r, h, lo)[0] if v is not None else kk[:, :dv]
            kk, vv = kk[there], vv[there]
            if not len(kk):
                continue
            hs = slice(h * group, (h + 1) * group)
            s = q[r, hs] @ kk.T * scale
            e = ((dk + 4) * 2.0 ** -24 * abs(scale) * (q[r, hs].abs() @ kk.abs().T)).amax(dim=1, keepdim=True)
            p = torch.softmax(s, dim=1)
            out[r, hs] = p @ vv
            A = p @ vv.abs()
            m = len(kk)
            sums = 4 * (m + 8) * 2.0 ** -24
            u = U[torch.float32 if f32 else torch.bfloat16]
            bound[r, hs] = (2 * (e + 2.0 ** -22) + sums + (0 if f32 else 2.0 ** -8)) * A + u * out[r, hs].abs()
            lse[r, hs] = torch.logsumexp(s, dim=1)
            lse_bound[r, hs] = e[:, 0] + sums + 2.0 ** -22 * (1 + lse[r, hs].abs())
    return out, lse, bound, lse_bound
