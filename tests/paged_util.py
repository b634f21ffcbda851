"""A plain 64-bit implementation of the paged cache's calls, and seeded inputs
for their tests.  Importing this module does not touch the GPU."""
from __future__ import annotations

import numpy as np
import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # unit roundoff
NAN_CODE = 0x7F  # e4m3's NaN; 127 as an int8


def codes(shape, dtype, g):
    x = torch.randn(shape, generator=g) * (LARGEST[dtype] / 4.5)
    x = x.clamp(-LARGEST[dtype], LARGEST[dtype])
    return (x.round() if dtype is torch.int8 else x).to(dtype)


class Setup:
    """A cache with shuffled pages, requests of the given lengths (tokens in the
    cache, the rows' own among them) and rows that see what `seen` says."""

    def __init__(self, lens, rows, page=16, kv=2, heads=8, dim=64, code=torch.float8_e4m3fn,
                 act=torch.bfloat16, seed=0, values=True, spare_pages=3, seen=None, q_scale=2.5):
        g = torch.Generator().manual_seed(seed)
        self.page, self.kv, self.heads, self.dim, self.act = page, kv, heads, dim, act
        self.lens = lens
        n = len(lens)
        need = [-(-L // page) for L in lens]
        self.n_pages = sum(need) + spare_pages
        order = torch.randperm(self.n_pages, generator=g).tolist()
        width = max([1, *need])
        self.table = torch.full((n, width), -1, dtype=torch.int32)
        self.k, self.v = (codes((self.n_pages, kv, page, dim), code, g) for _ in range(2))
        self.ks, self.vs = (torch.exp(0.5 * torch.randn((self.n_pages, kv), generator=g)) * 4.5 / LARGEST[code]
                            for _ in range(2))
        used = torch.zeros((self.n_pages, page), dtype=torch.bool)
        for r, L in enumerate(lens):
            for j in range(need[r]):
                p = order.pop()
                self.table[r, j] = p
                used[p, :max(0, min(page, L - j * page))] = True
        # what no request holds is NaN where the type has it
        if code is torch.float8_e4m3fn:
            for x in (self.k, self.v):
                x.view(torch.uint8).masked_fill_(~used[:, None, :, None], NAN_CODE)
        if not values:
            self.v = self.vs = None
        # rows: a count for each request; row j of a request's rows sees up to its own token
        self.row_starts = torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32)
        self.row_request = torch.repeat_interleave(torch.arange(n), torch.tensor(rows, dtype=torch.int64)).int()
        length = []
        for r, c in enumerate(rows):
            length += [max(0, lens[r] - c + 1 + j) for j in range(c)]
        self.row_lengths = torch.tensor(length if seen is None else seen, dtype=torch.int32)
        self.n_rows = len(self.row_lengths)
        self.q = (q_scale * torch.randn((self.n_rows, heads, dim), generator=g)).to(act)
        self.scale = dim ** -0.5

    def cuda(self):
        for name, x in list(vars(self).items()):
            if isinstance(x, torch.Tensor):
                setattr(self, name, x.cuda())
        return self

    def cache(self):
        from paper_2609_08450_amd import paged

        return paged.PagedCache.of(self.k, self.ks, self.v, self.vs)

    def tokens(self, side, r, length):
        """Values of the first tokens of request r [kv, length, dim] in 64 bits, and which are in the cache."""
        x, s = (self.k, self.ks) if side == "k" else (self.v, self.vs)
        pages = self.table[r, :-(-length // self.page)].long()
        there = (pages >= 0) & (pages < self.n_pages)
        p = torch.where(there, pages, 0)
        y = x.view(torch.uint8)[p].view(x.dtype).float().double() * s[p].double()[..., None, None]
        y = y.transpose(0, 1).flatten(1, 2)[:, :length]
        return y, there.repeat_interleave(self.page)[:length]


def attention(s: Setup, picked=None):
    """out, lse and the bound's ingredient sum p |v|, all in 64 bits; `picked`: a
    list of tokens for each row, or None for all that it sees."""
    G = s.heads // s.kv
    out = torch.zeros((s.n_rows, s.heads, s.dim), dtype=torch.float64, device=s.q.device)
    mass = torch.zeros_like(out)
    lse = torch.full((s.n_rows, s.heads), -torch.inf, dtype=torch.float64, device=s.q.device)
    request, lengths = s.row_request.tolist(), s.row_lengths.tolist()
    cap = s.table.shape[1] * s.page
    known = {}
    for i in range(s.n_rows):
        r = request[i] if i < len(request) else -1
        L = min(max(lengths[i], 0), cap)
        if r < 0 or r >= len(s.lens) or L == 0:
            continue
        top = max([min(max(x, 0), cap) for x, y in zip(lengths, request) if y == r])
        if r not in known:
            known = {r: (s.tokens("k", r, top), s.tokens("v", r, top))}
        (k, there), (v, _) = known[r]
        at = torch.arange(L, device=k.device)
        if picked is not None:
            at = picked[i].long()
            at = at[(at >= 0) & (at < L)]
        at = at[there[at]]
        if at.numel() == 0:
            continue
        q = s.q[i].double().view(s.kv, G, s.dim)
        x = s.scale * torch.matmul(q, k[:, at].transpose(1, 2))
        z = torch.logsumexp(x, -1)
        p = torch.exp(x - z[..., None])
        out[i] = torch.matmul(p, v[:, at]).reshape(s.heads, s.dim)
        mass[i] = torch.matmul(p, v[:, at].abs()).reshape(s.heads, s.dim)
        lse[i] = z.reshape(s.heads)
    return out, lse, mass


def assert_attention(got, lse, ref, where=""):
    """Elementwise.  Keys, values and queries are exact in the products; what is
    rounded is each weight (2^-11 of it, and 2^-25 of the largest where it is
    tiny), the FP32 sums (below 2^-12 for these sizes), and the result (half a
    unit in the last place of its type)."""
    out, ref_lse, mass = ref
    tol = UNIT[got.dtype] * out.abs() + 2.0 ** -10 * mass + 2.0 ** -18 * (mass > 0) * mass.amax()
    off = (got.double() - out).abs()
    assert bool(torch.isfinite(got.float()).all()), f"{where}: not finite"
    bad = off > tol
    assert not bool(bad.any()), (f"{where}: {int(bad.sum())} of {bad.numel()} out of bounds, first at "
                                 f"{bad.nonzero()[0].tolist()}: {float(off[bad][0]):.3g} > {float(tol[bad][0]):.3g}")
    if lse is not None:
        empty = ref_lse == -torch.inf
        assert bool((lse[empty] == -torch.inf).all()), f"{where}: lse of an empty row"
        # FP32 products and sums: below 2^-16 of the largest score's size here
        d = (lse.double() - ref_lse)[~empty].abs()
        assert bool((d <= 2.0 ** -15 * (1 + ref_lse[~empty].abs())).all()), f"{where}: lse off by {float(d.max()):.3g}"


def e4m3_round(x):
    """Nearest e4m3 value, ties to even, of values within its range (float64)."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 4, -9).astype(np.float64))
    return np.round(x / step) * step


def store_oracle(k, scale, x, slots, dtype):
    """paged_kv_store of one side, from its definition: (values of codes, scale),
    codes as numbers.  k float32 [pages, kv, page, dim] holds the codes' numbers."""
    k, scale = k.copy(), scale.copy()
    P = k.shape[2]
    n_slots = k.shape[0] * P
    f32 = np.float32
    big = f32(LARGEST[dtype])

    def code(y):
        y = np.clip(np.nan_to_num(y.astype(f32), nan=0.0, posinf=big, neginf=-big), -big, big)
        return (np.rint(y) if dtype is torch.int8 else e4m3_round(y)).astype(f32)

    i = 0
    while i < len(slots):
        if not 0 <= slots[i] < n_slots:
            i += 1
            continue
        j = i + 1
        while j < len(slots) and slots[j] == slots[i] + (j - i) and slots[j] // P == slots[i] // P:
            j += 1
        page, place = divmod(int(slots[i]), P)
        new = x[i:j].astype(f32).transpose(1, 0, 2)  # [kv, tokens, dim]
        with np.errstate(invalid="ignore"):
            top = np.where(np.isfinite(new), np.abs(new), 0).max(axis=(1, 2)).astype(f32)
        if dtype is torch.int8:
            s = np.maximum(top * (f32(1) / f32(127)), f32(2.0 ** -100))
        else:
            s = np.array([2.0 ** -100] * len(top), f32)
            for h, t in enumerate(top):
                while f32(448) * s[h] < t:
                    s[h] *= 2
        for h in range(len(top)):
            old = scale[page, h]
            if place > 0:
                s[h] = max(s[h], old)
                if s[h] > old:
                    k[page, h, :place] = code((k[page, h, :place] * old).astype(f32) / s[h])
            with np.errstate(invalid="ignore", over="ignore"):
                k[page, h, place:place + j - i] = code(new[h] / s[h])
            scale[page, h] = s[h]
        i = j
    return k, scale


def tables_oracle(ring, pool, lens, new, table, page, rows):
    """paged_kv_tables from its definition, on lists."""
    ring, table = list(ring), [list(t) for t in table]
    size, (head, free) = len(ring), pool[:2]
    queue = [ring[(head + i) % size] for i in range(free)]
    end = head + free
    up = lambda a: -(-a // page)  # noqa: E731
    to = [max(0, a + b) for a, b in zip(lens, new)]
    for r in range(len(lens)):
        for j in range(up(to[r]), up(lens[r])):
            queue.append(table[r][j])
            ring[end % size] = table[r][j]
            end += 1
    out, starts, who, length, slots, refused, asked, used = [], [0], [], [], [], 0, 0, 0
    for r in range(len(lens)):
        more = max(0, up(to[r]) - up(lens[r]))
        wide = up(to[r]) > len(table[r])
        asked += 0 if wide else more
        no = more > 0 and (wide or asked > len(queue))
        refused += no
        for j in range(up(lens[r]), up(to[r]) if not no else 0):
            table[r][j] = queue[used]
            used += 1
        out.append(lens[r] if no else to[r])
        for j in range(max(0, new[r])):
            p = lens[r] + j
            who.append(r)
            length.append(0 if no else p + 1)
            slots.append(-1 if no else table[r][p // page] * page + p % page)
        starts.append(len(who))
    who, length, slots = who[:rows], length[:rows], slots[:rows]
    fill = rows - len(who)
    return dict(pool_out=[(head + used) % size, len(queue) - used, refused, 0], lens_out=out, row_starts=starts,
                row_request=who + [-1] * fill, row_lengths=length + [0] * fill, slots=slots + [-1] * fill,
                table=table, ring=ring)


def scores(s: Setup, w):
    """Score rows in 64 bits, and the sums of magnitudes for the bound."""
    rows, bound = [], []
    for i in range(s.n_rows):
        r, L = int(s.row_request[i]), int(s.row_lengths[i])
        L = min(max(L, 0), s.table.shape[1] * s.page)
        if r < 0 or r >= len(s.lens) or L == 0:
            rows.append(None)
            bound.append(None)
            continue
        k, there = s.tokens("k", r, L)
        k = torch.where(there[:, None], k[0], 0.0)
        q = s.q[i].double()
        x = torch.matmul(q, k.t()).clamp(min=0)
        y = s.scale * (w[i].double()[:, None] * x).sum(0)
        rows.append(torch.where(there, y, -torch.inf))
        bound.append(s.scale * (w[i].double().abs()[:, None] * torch.matmul(q.abs(), k.abs().t())).sum(0))
    return rows, bound
