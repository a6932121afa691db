"""Products by list and of int8 codes in 64 bits on the CPU, and inputs for them."""
import torch

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def lists_from(probes, groups):
    """pair_off and pair_ids of the pairs (query, rank) whose list is probes[query][rank]; -1: in no list.  The pairs of no list
    come last among pair_ids."""
    flat = torch.as_tensor(probes).reshape(-1).long()
    order = torch.argsort(torch.where(flat < 0, groups, flat), stable=True)
    off = torch.zeros(groups + 1, dtype=torch.int64)
    off[1:] = torch.cumsum(torch.bincount(flat[flat >= 0], minlength=groups), 0)
    return off.int(), order.int()


def probes_of(seed, nq, nprobe, groups, empty=0.0, none=0.0):
    """Random lists of every query; a share `empty` of the lists is probed by nobody, a share `none` of the pairs in no list."""
    g = torch.Generator().manual_seed(seed)
    used = torch.nonzero(torch.rand(groups, generator=g) >= empty).flatten()
    if used.numel() == 0:
        used = torch.tensor([groups - 1])
    probes = used[torch.randint(used.numel(), (nq, nprobe), generator=g)]
    return torch.where(torch.rand(nq, nprobe, generator=g) < none, -1, probes)


def numbers(seed, shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


def pairs_of(off, ids, pairs):
    """[(list, pair)] in position order."""
    out = []
    for g in range(len(off) - 1):
        for i in range(int(off[g]), int(off[g + 1])):
            p = i if ids is None else int(ids[i])
            if 0 <= p < pairs:
                out.append((g, p))
    return out


def _by_list(off, ids, pairs, device="cpu"):
    lists = {}
    for g, p in pairs_of(off.tolist(), None if ids is None else ids.tolist(), pairs):
        lists.setdefault(g, []).append(p)
    return {g: torch.tensor(p, device=device) for g, p in lists.items()}


# The 64-bit products run where x and w lie: on the CPU, or, for sizes that take it too long, as the library's fp64 products.


def forward64(x, w, off, ids, nprobe):
    """(out, sum of |products|, named) in 64 bits."""
    x, w = x.double(), w.double()
    pairs = x.shape[0] * nprobe
    y, mag, named = x.new_zeros(pairs, w.shape[1]), x.new_zeros(pairs, w.shape[1]), torch.zeros(pairs, device=x.device).bool()
    for g, p in _by_list(off, ids, pairs, x.device).items():
        y[p], mag[p], named[p] = x[p // nprobe] @ w[g].t(), x[p // nprobe].abs() @ w[g].abs().t(), True
    return y, mag, named


def dx64(dy, w, off, ids, nprobe):
    dy, w = dy.double(), w.double()
    pairs = dy.shape[0]
    d, mag, named = dy.new_zeros(pairs, w.shape[2]), dy.new_zeros(pairs, w.shape[2]), torch.zeros(pairs, device=dy.device).bool()
    for g, p in _by_list(off, ids, pairs, dy.device).items():
        d[p], mag[p], named[p] = dy[p] @ w[g], dy[p].abs() @ w[g].abs(), True
    rows = lambda t: t.reshape(pairs // nprobe, nprobe, -1)
    return rows(d).sum(1), rows(mag).sum(1), named.reshape(-1, nprobe).any(1)


def dw64(dy, x, off, ids, nprobe):
    dy, x = dy.double(), x.double()
    groups = len(off) - 1
    d, mag = dy.new_zeros(groups, dy.shape[1], x.shape[1]), dy.new_zeros(groups, dy.shape[1], x.shape[1])
    for g, p in _by_list(off, ids, dy.shape[0], dy.device).items():
        d[g], mag[g] = dy[p].t() @ x[p // nprobe], dy[p].abs().t() @ x[p // nprobe].abs()
    return d, mag


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_sums(got, want, mag, terms, dtype, what=""):
    """got is an fp32 sum of `terms` products, rounded once to dtype.  Products of two fp32 numbers are rounded (2^-24 of each),
    and every addition, in whatever order, may lose an ulp (2^-23, where the matrix unit does not round to nearest) of a partial sum that is no
    larger than the sum of magnitudes: (terms + 1) 2^-23 mag in all; then half a step of dtype, and of its smallest numbers."""
    err = (got.double().to(want.device) - want).abs()
    sums = (terms + 1) * 2.0 ** -23 * mag
    tol = sums + half_step(dtype) * (want.abs() + sums) + torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    worst = (err - tol).max().item() if err.numel() else -1.0
    assert not torch.isnan(err).any() and worst <= 0, f"{what}: off by {err.max().item():.3e}, {worst:.3e} more than allowed"


def codes64(x):
    """The definition of quantize_rows in 64 bits: (codes, scale)."""
    x64 = x.double()
    top = x64.abs().amax(1)
    scale = (top / 127).float()
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    bad = ~torch.isfinite(x64).all(1)
    codes = torch.where(bad[:, None], torch.zeros_like(x64), torch.round(x64 / scale.double()[:, None]).clamp(-127, 127))
    return codes.to(torch.int8), torch.where(bad, torch.full_like(scale, float("nan")), scale)


def i8_64(a, sa, b, sb):
    return (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()[None, :]


def assert_scaled(got, want, dtype, what=""):
    """got is an exact whole number converted to fp32, multiplied twice and rounded to dtype: three roundings of 2^-24 (their
    product's second order in the 4), and half a step of dtype; where a scale is small, half a step of the smallest numbers
    each time."""
    err = (got.double().to(want.device) - want).abs()
    tol = 4 * 2.0 ** -24 * want.abs() + 1.01 * half_step(dtype) * want.abs() + torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    worst = (err - tol).max().item() if err.numel() else -1.0
    assert not torch.isnan(err).any() and worst <= 0, f"{what}: off by {err.max().item():.3e}, {worst:.3e} more than allowed"


def grouped_i8_64(x, sx, w, sw, off, ids, nprobe):
    """(out, named): whole-number sums, exact in 64 bits, times the scales."""
    y, _, named = forward64(x, w, off, ids, nprobe)
    for g, p in _by_list(off, ids, y.shape[0], y.device).items():
        y[p] *= sx.double()[p // nprobe][:, None] * sw.double()[g][None, :]
    return y, named
