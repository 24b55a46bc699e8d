"""Adapter cases whose results are exact in fp32 and need every bit of u and g.

u and g are 24-bit integers (times a power of two).  In the bf16 layers' kernels
they enter the second product as bf16 planes, eight bits of them each: a kernel
that held fewer than three planes would give other results in every row that has
an adapter.  One row of x selects three columns of A, which hold the planes of
the integer, so that the sum that gives u is exact in fp32 in any order.
"""
import torch

from adapter_reference import NONE, forward


def cut(v, planes):
    """What `planes` bf16 planes hold of fp32 values, each cut to its upper 16 bits."""
    kept, rest = torch.zeros_like(v), v.clone()
    for _ in range(planes):
        p = (rest.view(torch.int32) & -65536).view(torch.float32)
        kept, rest = kept + p, rest - p
    return kept


def cut_two_rounded(v):
    """Two planes, the second one rounded."""
    first = cut(v, 1)
    return first + (v - first).bfloat16().float()


def integers(gen, *shape):
    """24-bit integers whose three planes are their three bytes (each with its
    upper bit, so that none reaches into the next, and the last one odd), either sign."""
    v = (torch.randint(2 ** 23, 2 ** 24, shape, generator=gen) | 0x008081).float()
    return torch.where(torch.rand(shape, generator=gen) < 0.5, v, -v)


def make_ids(gen, T, L, how):
    if how == "runs":
        ids = torch.arange(T) * (L + 1) // T
        return torch.where(ids == L, -1, ids).int()
    ids = torch.randint(0, L, (T,), generator=gen).int()
    some = torch.rand(T, generator=gen) < 0.1
    some[0] = False
    ids[some] = torch.tensor(NONE + (L,)).int()[torch.arange(int(some.sum())) % 4]
    return ids


def narrow_operands(gen, T, width, r, L, dt):
    """(v [T][width], W [L][r][width], pick [T]): v W^T is, for row i of adapter l,
    2^e times one of the adapter's integers for each rank.  The ranks go in
    pairs: the second one of a pair is the first's upper 16 bits, negated."""
    K = min(width // 3, 7)
    U = integers(gen, L, K, r)
    U[..., 1::2] = -cut(U[..., 0:r - r % 2:2].contiguous(), 2)
    W = torch.randint(-3, 4, (L, r, width), generator=gen).float()   # columns that no row selects
    for k in range(K):
        rest = U[:, k].clone()
        for d in range(3):
            W[:, :, 3 * k + d] = cut(rest, 1)
            rest -= W[:, :, 3 * k + d]
        assert not rest.any()
    pick = torch.randint(0, K, (T,), generator=gen)
    v = torch.zeros(T, width)
    v.scatter_(1, 3 * pick[:, None] + torch.arange(3)[None, :],
               (2.0 ** torch.randint(-1, 2, (T, 1), generator=gen)).expand(T, 3).contiguous())
    return v.to(dt), W.to(dt), pick


def wide_operand(gen, width, r, L, dt):
    """(W [L][r][width], columns that sum a pair): every column takes one rank times
    +-1, or both of a pair, which leaves the third plane of the first alone."""
    W = torch.zeros(L, r, width)
    pair = torch.zeros(L, width, dtype=torch.bool)
    for l in range(L):
        j = torch.randint(0, r, (width,), generator=gen)
        j[:min(r, width)] = torch.randperm(r, generator=gen)[:width]
        W[l, j, torch.arange(width)] = 1.0
        pair[l] = (torch.rand(width, generator=gen) < 0.5) & (j // 2 * 2 + 1 < r)
        if r > 1 and width > 1:
            pair[l, 0], j[0] = True, 0
            W[l, :, 0] = 0
        W[l, j[pair[l]] // 2 * 2, torch.where(pair[l])[0]] = 1.0
        W[l, j[pair[l]] // 2 * 2 + 1, torch.where(pair[l])[0]] = 1.0
        W[l] *= torch.where(torch.rand(width, generator=gen) < 0.5, 1.0, -1.0)
    return W.to(dt), pair


def base_of(gen, ids, pair, dt):
    """Small integers in the columns that sum a pair (there the sum stays exact)."""
    T, width = ids.numel(), pair.shape[1]
    base = torch.randint(-5, 6, (T, width), generator=gen).float()
    for l in range(pair.shape[0]):
        base[(ids == l)[:, None] & ~pair[l][None, :]] = 0
    return base.to(dt)


def product(T, m, n, r, L, how, dt, odt, seed):
    """x, A, B, ids, base, scale of a forward call."""
    gen = torch.Generator().manual_seed(seed)
    ids = make_ids(gen, T, L, how)
    x, A, _ = narrow_operands(gen, T, m, r, L, dt)
    B, pair = wide_operand(gen, n, r, L, dt)
    scale = (2.0 ** torch.randint(-1, 2, (L,), generator=gen)).float()
    return {"x": x, "A": A, "B": B, "ids": ids, "base": base_of(gen, ids, pair, odt), "scale": scale}


def _spread(rows, count):
    """`count` of these rows (some of them again where there are fewer), over all of them."""
    return rows[(torch.arange(count) * rows.numel() // count) if rows.numel() > count
                else torch.arange(count) % rows.numel()]


def gradients(T, m, n, r, L, how, dt, seed):
    """x, A, B, ids, u, dy, scale of a backward call whose dA and dB are single products:
    each column of an adapter's x is nonzero in one of its rows, and u in one row for each
    triple of columns that dy selects."""
    gen = torch.Generator().manual_seed(seed)
    ids = make_ids(gen, T, L, how)
    dy, B, pick = narrow_operands(gen, T, n, r, L, dt)
    x, u = torch.zeros(T, m), torch.zeros(T, r)
    for l in range(L):
        rows = (ids == l).nonzero()[:, 0]
        if not rows.numel():
            continue
        sign = torch.where(torch.rand(m, generator=gen) < 0.5, 1.0, -1.0)
        x[_spread(rows, m), torch.arange(m)] = sign
        for k in pick[rows].unique():
            at = rows[pick[rows] == k]
            u[at[int(torch.randint(0, at.numel(), (1,), generator=gen))]] = integers(gen, r)
    scale = (2.0 ** torch.randint(-1, 2, (L,), generator=gen)).float()
    return {"x": x.to(dt), "A": torch.zeros(L, r, m, dtype=dt), "B": B, "ids": ids, "u": u, "dy": dy, "scale": scale}


def factor_gradients(c, keep=None):
    """(dA, dB) of such a case in float64, with u and g held as `keep` gives them."""
    g, _ = forward(c["dy"], c["B"], c["A"], c["ids"], None, c["scale"])
    u = c["u"].double()
    if keep is not None:
        g, u = keep(g.float()).double(), keep(c["u"]).double()
    dA = torch.zeros(c["A"].shape, dtype=torch.float64)
    dB = torch.zeros(c["B"].shape, dtype=torch.float64)
    for l in range(dA.shape[0]):
        at = c["ids"] == l
        dA[l], dB[l] = g[at].t() @ c["x"][at].double(), u[at].t() @ c["dy"][at].double()
    return dA, dB
