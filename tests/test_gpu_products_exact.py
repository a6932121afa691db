"""Products on the device against exact sums: long ones in parts, uneven lists, operands far apart, numbers near the type's smallest, rows of
no numbers."""
import ctypes as C
import threading

import pytest
import torch

from paper_2602_23999_amd import rabitq

from product_exact import assert_exact, dw_exact, dx_exact, forward_exact, whole
from product_helpers import TYPES, lists_from, numbers, probes_of

pytestmark = pytest.mark.gpu


def _uneven(seed, nq, nprobe, groups, share, long_list=0):
    """Random lists, a share of the pairs in one of them."""
    probes = probes_of(seed, nq, nprobe, groups)
    g = torch.Generator().manual_seed(seed + 1)
    return lists_from(torch.where(torch.rand(nq, nprobe, generator=g) < share, long_list, probes), groups)


def _parts(groups, nprobe, pairs, n, k):
    """Buffers of n x k sums that dw asks for, from the size of its scratch."""
    ls = rabitq._Lists(groups, nprobe, pairs, n, k, 1 << 20, None)
    return rabitq.load_library().rabitq_grouped_dw_scratch_bytes(C.byref(ls)) // (n * k * 4)


# ---- dw in parts ----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("nq,nprobe,groups,n,k,share,part", [
    (65536, 1, 1, 512, 512, 0, 2048),    # parts longer than the ring of pairs in LDS
    (70001, 1, 1, 500, 390, 0, 2048),    # a last part that ends inside a step, rows that are not whole pieces of 16 bytes
    (40000, 2, 5, 384, 264, 0.4, 1024),
    (30000, 3, 7, 257, 383, 0.7, 1536),
    (200000, 1, 3, 520, 520, 0.5, 9728),
    (70000, 1, 1, 264, 256, 0, 512),
], ids=str)
def test_dw_in_parts(nq, nprobe, groups, n, k, share, part, dtype):
    pairs = nq * nprobe
    assert _parts(groups, nprobe, pairs, n, k) == pairs // part + groups
    off, ids = _uneven(nq, nq, nprobe, groups, share, groups // 2)
    x, dy = whole(1, (nq, k), dtype, "cuda"), whole(2, (pairs, n), dtype, "cuda")
    got = rabitq.grouped_matmul_dw(dy, x, off.cuda(), ids.cuda(), nprobe)
    assert_exact(got, dw_exact(dy, x, off, ids, nprobe), dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("nq,nprobe,groups,n,k", [(20000, 1, 256, 256, 256), (9001, 2, 128, 250, 261), (30000, 1, 8, 1000, 1100)], ids=str)
def test_dw_of_one_long_list_among_many(nq, nprobe, groups, n, k, dtype):
    assert _parts(groups, nprobe, nq * nprobe, n, k) == 0  # the long list too is one part
    off, ids = _uneven(3, nq, nprobe, groups, 0.9, groups - 2)
    x, dy = whole(1, (nq, k), dtype, "cuda"), whole(2, (nq * nprobe, n), dtype, "cuda")
    assert_exact(rabitq.grouped_matmul_dw(dy, x, off.cuda(), ids.cuda(), nprobe), dw_exact(dy, x, off, ids, nprobe), dtype)


# ---- forward and dx -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("nq,nprobe,groups,wide,long,share", [
    (200, 1, 1, 64, 65537, 0),            # groups of wavefronts that share a long contraction
    (64, 2, 3, 40, 70000, 0.5),
    (1500, 2, 40, 512, 1032, 0.9),        # one long list among many short ones
    (4096, 1, 1, 4096, 2056, 0),          # 256 x 256 tiles
    (3000, 2, 3, 1001, 1031, 0.3),
    (6, 2, 5, 130, 100000, 0),            # few rows
], ids=str)
def test_forward_and_dx(nq, nprobe, groups, wide, long, share, dtype):
    off, ids = _uneven(nq, nq, nprobe, groups, share, groups // 2)
    lists = off.cuda(), ids.cuda(), nprobe
    x, w = whole(1, (nq, long), dtype, "cuda"), whole(2, (groups, wide, long), dtype, "cuda")
    assert_exact(rabitq.grouped_matmul(x, w, *lists), forward_exact(x, w, off, ids, nprobe), dtype)
    dy, w = whole(3, (nq * nprobe, long), dtype, "cuda"), whole(4, (groups, long, wide), dtype, "cuda")
    assert_exact(rabitq.grouped_matmul_dx(dy, w, *lists), dx_exact(dy, w, off, ids, nprobe), dtype)


# ---- rows between 2 and 4 GiB from the first, which 32-bit offsets still reach ------------

@pytest.fixture(scope="module")
def memory():
    """8 GiB, of which the tests use the upper half: an offset taken for a negative number would stay inside."""
    return torch.zeros(1 << 33, dtype=torch.uint8, device="cuda")


def _far(memory, t, row_bytes):
    """t [rows, columns] as a view whose rows lie row_bytes apart."""
    flat = memory[1 << 32:].view(t.dtype)
    size = t.element_size()
    assert (t.shape[0] - 1) * row_bytes + t.shape[1] * size <= 1 << 32 and row_bytes % 16 == 0
    view = flat.as_strided(t.shape, (row_bytes // size, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,wide,long", [(1024, 256, 256), (1024, 128, 1024), (4096, 4096, 64), (1000, 4096, 256)], ids=str)
def test_rows_of_the_left_operand_far_apart(memory, rows, wide, long, dtype):
    apart = (1 << 32) // rows - 16 - (1 << 32) // rows % 16
    off = torch.tensor([0, rows // 3, rows], dtype=torch.int32)
    x, w = whole(1, (rows, long), dtype, "cuda"), whole(2, (2, wide, long), dtype, "cuda")
    far = _far(memory, x, apart)
    assert (rows - 1) * apart > 1 << 31 and rows * apart < 1 << 32
    assert_exact(rabitq.grouped_matmul(far, w, off.cuda()), forward_exact(x, w, off, None, 1), dtype)
    w = whole(3, (2, long, wide), dtype, "cuda")
    assert_exact(rabitq.grouped_matmul_dx(far, w, off.cuda()), dx_exact(x, w, off, None, 1), dtype)
    w = whole(4, (rows, 128), dtype, "cuda")
    assert_exact(rabitq.grouped_matmul_dw(far, w, off.cuda()), dw_exact(x, w, off, None, 1), dtype)


@pytest.mark.parametrize("rows,n,k", [(1024, 256, 512), (4096, 4096, 256), (2000, 300, 1040)])
def test_rows_of_codes_far_apart(memory, rows, n, k):
    g = torch.Generator(device="cuda").manual_seed(k)
    a, b = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (rows, n))
    far = _far(memory, a, (1 << 32) // rows // 16 * 16 - 16)
    one = lambda r: torch.ones(r, device="cuda")
    assert torch.equal(rabitq.matmul_i8(far, one(rows), b, one(n)), (a.double() @ b.double().t().contiguous()).float())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_of_a_matrix_far_apart(memory, dtype):
    # 256 rows of a tile over nearly 4 GiB
    long = 1024 // torch.empty(0, dtype=dtype).element_size()
    x, w = whole(1, (65536, long), dtype, "cuda"), whole(2, (256, long), dtype, "cuda")
    off = torch.tensor([0, 65536], dtype=torch.int32)
    far = _far(memory, w, (1 << 24) - 16)
    assert_exact(rabitq.grouped_matmul(x, far[None], off.cuda()), forward_exact(x, w[None], off, None, 1), dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_dw_of_rows_gibibytes_apart(memory, dtype):
    dy, x = whole(1, (2, 128), dtype, "cuda"), whole(2, (2, 64), dtype, "cuda")
    off = torch.tensor([0, 2], dtype=torch.int32)
    far = _far(memory, dy, 3 << 30)
    assert_exact(rabitq.grouped_matmul_dw(far, x, off.cuda()), dw_exact(dy, x, off, None, 1), dtype)


# ---- small numbers, and rows that hold none ----------------------------------------------

@pytest.mark.parametrize("m,n,k", [(4, 16, 64), (300, 256, 64), (600, 64, 1024), (2048, 1024, 256), (4096, 4096, 256)], ids=str)
@pytest.mark.parametrize("dtype,step,factor", [
    (torch.float32, -149, 30), (torch.float32, -149, 0), (torch.float32, -100, -40),
    (torch.bfloat16, -133, 30), (torch.bfloat16, -133, 0), (torch.bfloat16, -93, -40),
    (torch.float16, -24, 4), (torch.float16, -24, 0), (torch.float16, -14, -10)], ids=str)
def test_denormal_numbers(m, n, k, dtype, step, factor):
    # whole multiples (up to 100) of the smallest number of the type, or of one whose products with 2^factor are as small: all sums
    # are whole multiples of 2^(step + factor) below 2^24 of them, exact in fp32, and are rounded once
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    small = lambda *s: (torch.randint(-100, 101, s, generator=g, device="cuda").double() * 2.0 ** step).to(dtype)
    signs = lambda *s: ((torch.randint(0, 2, s, generator=g, device="cuda").double() * 2 - 1) * 2.0 ** factor).to(dtype)
    x, w, dy, y = small(m, k), signs(1, n, k), small(m, n), signs(m, k)
    off = torch.tensor([0, m], dtype=torch.int32)
    assert_exact(rabitq.grouped_matmul(x, w, off.cuda()), forward_exact(x, w, off, None, 1), dtype)
    assert_exact(rabitq.grouped_matmul_dx(dy, w, off.cuda()), dx_exact(dy, w, off, None, 1), dtype)
    assert_exact(rabitq.grouped_matmul_dw(dy, y, off.cuda()), dw_exact(dy, y, off, None, 1), dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,n,k", [(1500, 200, 136), (1500, 201, 131), (1000, 64, 1064), (4096, 4096, 72), (2200, 1032, 264)], ids=str)
def test_infinities_and_nan_stay_in_their_rows_and_lists(rows, n, k, dtype):
    # (the tile kernels: rows of no list, other rows, empty lists, other lists)
    x, w, dy = whole(1, (rows, k), dtype, "cuda"), whole(2, (4, n, k), dtype, "cuda"), whole(3, (rows, n), dtype, "cuda")
    off = torch.tensor([10, rows // 2, rows // 2, rows - 300, rows - 30], dtype=torch.int32)
    want_y, want_dx, want_dw = forward_exact(x, w, off, None, 1), dx_exact(dy, w, off, None, 1), dw_exact(dy, x, off, None, 1)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[10:rows - 30] = True
    x[~inside], dy[~inside], w[1] = float("nan"), float("inf"), float("nan")
    x[15], dy[20], x[rows - 290, 3] = float("inf"), float("nan"), float("-inf")
    fill = lambda *s: torch.full(s, 7.0, dtype=dtype, device="cuda")
    y = rabitq.grouped_matmul(x, w, off.cuda(), out=fill(rows, n))
    good = inside.clone()
    good[15] = good[rows - 290] = False
    assert torch.equal(y[good], want_y[good].to(dtype)) and not torch.isfinite(y[15]).any() and (y[~inside] == 7).all()
    assert not torch.isfinite(y[rows - 290]).any()
    dx = rabitq.grouped_matmul_dx(dy, w, off.cuda(), out=fill(rows, k))
    good = inside.clone()
    good[20] = False
    assert torch.equal(dx[good], want_dx[good].to(dtype)) and dx[20].isnan().all() and (dx[~inside] == 7).all()
    dw = rabitq.grouped_matmul_dw(dy, x, off.cuda())
    assert not torch.isfinite(dw[0]).any() and (dw[1] == 0).all() and torch.equal(dw[2], want_dw[2].to(dtype))
    other = [c for c in range(k) if c != 3]
    assert torch.equal(dw[3][:, other], want_dw[3][:, other].to(dtype)) and not torch.isfinite(dw[3][:, 3]).any()


# ---- graphs and threads -----------------------------------------------------------------

def test_large_tiles_captured_and_replayed():
    # tiles of 256 and 128, shared ones (all of more than 64 KB of LDS) and dw in parts in one graph, on other inputs at every replay
    big, mid, few, long = (4096, 4096, 264), (1200, 4096, 272), (512, 1024, 1040), (20000, 256, 256)
    off = {m: torch.tensor([0, m // 3, m], dtype=torch.int32, device="cuda") for m, _, _ in (big, mid, few, long)}
    data = [(whole(1, (m, k), torch.bfloat16, "cuda"), whole(2, (2, n, k), torch.bfloat16, "cuda"), whole(3, (m, n), torch.bfloat16, "cuda"))
            for m, n, k in (big, mid, few, long)]

    def step():
        out = []
        for x, w, dy in data:
            o = off[x.shape[0]]
            out += [rabitq.grouped_matmul(x, w, o), rabitq.grouped_matmul_dx(dy, w, o), rabitq.grouped_matmul_dw(dy, x, o)]
        return out
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        for i, (x, w, dy) in enumerate(data):
            for j, t in enumerate((x, w, dy)):
                t.copy_(whole(100 * seed + 10 * i + j, t.shape, t.dtype, "cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for (x, w, dy), y, dx, dw in zip(data, got[::3], got[1::3], got[2::3]):
            o = off[x.shape[0]].cpu()
            assert_exact(y, forward_exact(x, w, o, None, 1), torch.bfloat16)
            assert_exact(dx, dx_exact(dy, w, o, None, 1), torch.bfloat16)
            assert_exact(dw, dw_exact(dy, x, o, None, 1), torch.bfloat16)
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_two_host_threads():
    nq, nprobe, groups, n, k = 700, 2, 6, 264, 520
    off, ids = lists_from(probes_of(1, nq, nprobe, groups), groups)
    lists = off.cuda(), ids.cuda(), nprobe
    data = [(whole(s, (nq, k), torch.bfloat16, "cuda"), whole(s + 1, (groups, n, k), torch.bfloat16, "cuda"),
             whole(s + 2, (nq * nprobe, n), torch.bfloat16, "cuda")) for s in (1, 11)]
    torch.cuda.synchronize()
    results, faults = [[], []], []

    def work(i):
        try:
            x, w, dy = data[i]
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    results[i].append((rabitq.grouped_matmul(x, w, *lists), rabitq.grouped_matmul_dx(dy, w, *lists),
                                       rabitq.grouped_matmul_dw(dy, x, *lists)))
                    # each thread reads its own error
                    with pytest.raises(rabitq.RabitqError, match="stride out of range" if i else "k in 1"):
                        rabitq.grouped_matmul(x, w[:1].expand(groups, n, k), *lists) if i else rabitq.quantize_rows(x[:, :0])
                torch.cuda.current_stream().synchronize()
        except BaseException as e:  # (an assertion in a thread would be lost)
            faults.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults, faults
    for (x, w, dy), got in zip(data, results):
        for y, dx, dw in got:
            assert_exact(y, forward_exact(x, w, off, ids, nprobe), torch.bfloat16)
            assert_exact(dx, dx_exact(dy, w, off, ids, nprobe), torch.bfloat16)
            assert_exact(dw, dw_exact(dy, x, off, ids, nprobe), torch.bfloat16)
