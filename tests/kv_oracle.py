"""Plain 64-bit (or bit-exact) forms of the cache's operators, on the host, and
the layout of a page: what the tests of the key/value cache compare with."""
import numpy as np
import torch

NP = {torch.bfloat16: np.uint16, torch.float16: np.uint16}


def pages_of(heads, dim, block, layers=1):
    """Elements of a block of one layer, and log2 of the bytes of a page that holds ``layers`` of them."""
    elems = 2 * heads * block * dim
    return elems, max(10, (2 * layers * elems - 1).bit_length())


def k_index(page_elems, block, dim, page, off, head, d):
    """Element index of K's dimension ``d`` of a token in a layer's pool."""
    return page * page_elems + head * 2 * block * dim + (d // 8 * block + off) * 8 + d % 8


def v_index(page_elems, block, dim, page, off, head, d):
    return page * page_elems + head * 2 * block * dim + block * dim + (off // 8 * dim + d) * 8 + off % 8


def rows(flat, index, page_elems, block, heads, dim, slots):
    """[len(slots), heads, dim] of K or V (``index``) at token slots of one layer's pool."""
    slots = torch.as_tensor(slots)[:, None, None]
    h, d = torch.arange(heads)[:, None], torch.arange(dim)
    return flat[index(page_elems, block, dim, slots // block, slots % block, h, d)]


def put_rows(flat, index, page_elems, block, heads, dim, slots, values):
    slots = torch.as_tensor(slots)[:, None, None]
    h, d = torch.arange(heads)[:, None], torch.arange(dim)
    flat[index(page_elems, block, dim, slots // block, slots % block, h, d)] = values


def kv_map(block, ring, ring_pos, held, lens, new, table, n_tokens):
    """Request after request; returns the new state and the token columns, with
    ``table`` and ``ring`` updated in place, and whether anything was out of range."""
    width, size = table.shape[1], len(ring)
    taken, put = (int(x) for x in ring_pos)
    flag = not 0 <= put - taken <= size
    avail = 0 if flag else put - taken
    room = 0 if flag else size - avail
    want, used, back, given = 0, 0, 0, 0
    held_out, lens_out, starts, cols = [], [], [0], []
    old = np.array(table)
    for r, (h, n, m) in enumerate(zip(held.tolist(), lens.tolist(), new.tolist())):
        ok = n >= 0 and 0 <= h <= width and n <= h * block and n + max(m, 0) <= width * block
        starts.append(starts[-1] + max(m, 0))
        flag = flag or not ok
        if m < 0:
            if ok:
                back += h
                ok = h == 0 or back <= room
                flag = flag or not ok
            if ok and h:
                for b in range(h):
                    ring[(put + given + b) % size] = old[r, b]
                given = back
            held_out.append(0 if ok else h)
            lens_out.append(0 if ok else n)
            continue
        need = max(0, -(-(n + m) // block) - h) if ok else 0
        served = ok and (need == 0 or want + need <= avail)
        if served and starts[-1] > n_tokens:
            served = False
        flag = flag or (ok and starts[-1] > n_tokens and starts[-1] != starts[-2])
        if served:
            for b in range(need):
                table[r, h + b] = ring[(taken + want + b) % size]
            used = max(used, want + need) if need else used
        want += need
        held_out.append(h + need if served else h)
        lens_out.append(n + m if served else n)
        for p in range(n, n + min(m, n_tokens - len(cols))):
            slot = int(table[r, p // block]) * block + p % block if served else -1
            cols.append((slot, r, p))
    cols += [(-1, -1, -1)] * (n_tokens - len(cols))
    cols = np.array(cols, dtype=np.int64).reshape(n_tokens, 3)
    return {"ring_pos": [taken + used, put + given], "held": held_out, "lens": lens_out,
            "q_start": [min(s, n_tokens) for s in starts], "slots": cols[:, 0], "request": cols[:, 1],
            "position": cols[:, 2], "flag": flag}


def attend(q, k, v, seen, scale, cap):
    """One request's heads in 64 bits.  q [n, H, D], k, v [t, G, D], seen
    [n, t] bool.  Returns o, lse and, for the error bounds, sum of weights times |v|
    and the largest sum |q_d k_d| scale of a row."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    o = torch.zeros(n, heads, dim, dtype=torch.float64)
    mass, dots = o.clone(), torch.zeros(n, heads, dtype=torch.float64)
    lse = torch.full((n, heads), -torch.inf, dtype=torch.float64)
    for i in range(n):
        on = seen[i].nonzero()[:, 0]
        if not len(on):
            continue
        for h in range(heads):
            kk, vv = k[on, h // group].double(), v[on, h // group].double()
            qq = q[i, h].double()
            s = kk @ qq * scale
            dots[i, h] = (kk.abs() @ qq.abs()).max() * scale
            if cap:
                s = cap * torch.tanh(s / cap)
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.exp(s - lse[i, h])
            o[i, h] = (w[:, None] * vv).sum(0)
            mass[i, h] = (w[:, None] * vv.abs()).sum(0)
    return o, lse, mass, dots


# unit roundoff of a type (round to nearest): 8 and 11 bits
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend_bounds(dtype, dim, tokens, o, lse, mass, dots, cap):
    """How far o and lse may be off.  A score is a sum of ``dim`` exact products
    in fp32, scaled: off by at most (dim + 4) 2^-24 of its sum of magnitudes; a
    capped one also by 8 roundings of the cap.  A weight's relative error is
    twice that (numerator and sum).  Weights are rounded to the type once, o
    once; sums of ``tokens`` terms in fp32 and the joins add (tokens + 64) 2^-24."""
    u, e = ROUND[dtype], 2.0 ** -24
    ds = (dim + 4) * e * dots + 8 * e * cap + 4 * e * torch.where(torch.isinf(lse), 0, lse).abs()
    rest = 2 * ds + (tokens + 64) * e
    ob = u * o.abs() + (u * (1 + u) + rest[..., None]) * mass + 2.0 ** -24
    return ob, ds + (tokens + 64) * e + 4 * e * torch.where(torch.isinf(lse), 0, lse).abs()
