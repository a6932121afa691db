"""Products whose every partial sum fp32 holds exactly, so that results have to be equal and a part that is lost, doubled or out of place shows.

Operands are whole numbers from -2 to 2 (exact in every type): products are at most 4, and fewer than 2^22 of them stay below 2^24,
in whatever order they are added.  The result is then one rounding of the exact sum."""
import torch


def whole(seed, shape, dtype, device="cpu"):
    g = torch.Generator(device=device).manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device=device).to(dtype)


def rows_of_lists(off, ids, pairs):
    """[(list, its pairs)] of the lists that have any."""
    ids = torch.arange(pairs) if ids is None else ids.long()
    o = off.tolist()
    return [(g, ids[o[g]:o[g + 1]]) for g in range(len(o) - 1) if o[g + 1] > o[g]]


def forward_exact(x, w, off, ids, nprobe):
    y = torch.zeros(x.shape[0] * nprobe, w.shape[1], dtype=torch.float64, device=x.device)
    for g, p in rows_of_lists(off, ids, y.shape[0]):
        p = p.to(x.device)
        y[p] = x[p // nprobe].double() @ w[g].double().t().contiguous()
    return y


def dx_exact(dy, w, off, ids, nprobe):
    d = torch.zeros(dy.shape[0], w.shape[2], dtype=torch.float64, device=dy.device)
    for g, p in rows_of_lists(off, ids, dy.shape[0]):
        p = p.to(dy.device)
        d[p] = dy[p].double() @ w[g].double()
    return d.reshape(-1, nprobe, d.shape[1]).sum(1)


def dw_exact(dy, x, off, ids, nprobe):
    d = torch.zeros(len(off) - 1, dy.shape[1], x.shape[1], dtype=torch.float64, device=dy.device)
    for g, p in rows_of_lists(off, ids, dy.shape[0]):
        assert 4 * len(p) < 2 ** 24
        p = p.to(dy.device)
        d[g] = dy[p].double().t().contiguous() @ x[p // nprobe].double()
    return d


def assert_exact(got, want, dtype):
    assert got.dtype == dtype and torch.equal(got, want.to(dtype).to(got.device))
