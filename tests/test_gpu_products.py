"""Products by list (forward and gradients) and of int8 codes on the device against the same in 64 bits on the CPU."""
import pytest
import torch

from paper_2602_23999_amd import rabitq

from product_helpers import (TYPES, assert_scaled, assert_sums, codes64, dw64, dx64, forward64, grouped_i8_64, i8_64,
                             lists_from, numbers, probes_of)

pytestmark = pytest.mark.gpu

# nq, nprobe, groups, n, k, share of empty lists, share of pairs in no list
SHAPES = [
    (1, 1, 1, 1, 1, 0, 0),
    (1, 1, 3, 17, 33, 0, 0),
    (2, 4, 64, 48, 64, 0, 0),         # a pair or none per list
    (16, 4, 8, 256, 512, 0, 0),
    (37, 3, 5, 65, 129, 0, 0.1),
    (130, 2, 9, 128, 128, 0.5, 0),    # half of the lists empty
    (500, 1, 2, 260, 200, 0, 0.05),
    (700, 2, 3, 512, 320, 0, 0),
    (300, 5, 300, 40, 72, 0.3, 0.2),  # more lists than a wavefront searches at once
    (1000, 1, 1, 128, 96, 0, 0),
    (64, 16, 5000, 16, 32, 0.9, 0),   # three levels of the search for a tile's list
    (1500, 2, 4, 384, 264, 0, 0),
    (40, 1, 2, 100, 2056, 0, 0),
    (33, 2, 3, 1000, 24, 0, 0),
]


def _inputs(shape, dtype, seed=0):
    nq, nprobe, groups, n, k, empty, none = shape
    off, ids = lists_from(probes_of(seed, nq, nprobe, groups, empty, none), groups)
    return numbers(seed + 1, (nq, k), dtype), numbers(seed + 2, (groups, n, k), dtype), numbers(seed + 3, (nq * nprobe, n), dtype), off, ids


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_grouped_matmul(shape, dtype):
    x, w, _, off, ids = _inputs(shape, dtype)
    want, mag, named = forward64(x, w, off, ids, shape[1])
    out = torch.full((shape[0] * shape[1], shape[3]), 7.0, dtype=dtype, device="cuda")
    got = rabitq.grouped_matmul(x.cuda(), w.cuda(), off.cuda(), ids.cuda(), shape[1], out=out)
    assert got is out
    assert_sums(got[named], want[named], mag[named], shape[4], dtype)
    assert (got[~named] == 7.0).all()  # pairs of no list are left as they were


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_grouped_matmul_dx(shape, dtype):
    x, w, dy, off, ids = _inputs(shape, dtype)
    want, mag, named = dx64(dy, w, off, ids, shape[1])
    out = torch.full(x.shape, 7.0, dtype=dtype, device="cuda")
    got = rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), off.cuda(), ids.cuda(), shape[1], out=out)
    assert_sums(got[named], want[named], mag[named], shape[3] * shape[1], dtype)
    assert (got[~named] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_grouped_matmul_dw(shape, dtype):
    x, w, dy, off, ids = _inputs(shape, dtype)
    want, mag = dw64(dy, x, off, ids, shape[1])
    out = torch.full(w.shape, 7.0, dtype=dtype, device="cuda")
    got = rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), off.cuda(), ids.cuda(), shape[1], out=out)
    terms = int((off[1:] - off[:-1]).max())
    assert_sums(got, want, mag, terms, dtype)
    empty = (off[1:] == off[:-1])
    assert (got[empty.cuda()] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_grouped_matmul_i8(shape, dtype):
    nq, nprobe, groups, n, k, _, _ = shape
    x, w, _, off, ids = _inputs(shape, torch.float32)
    cx, sx = codes64(x)
    cw, sw = codes64(w.reshape(-1, k))
    cw, sw = cw.reshape(w.shape), sw.reshape(groups, n)
    want, named = grouped_i8_64(cx, sx, cw, sw, off, ids, nprobe)
    out = torch.full((nq * nprobe, n), 7.0, dtype=dtype, device="cuda")
    got = rabitq.grouped_matmul_i8(cx.cuda(), sx.cuda(), cw.cuda(), sw.cuda(), off.cuda(), ids.cuda(), nprobe, dtype, out)
    assert_scaled(got[named], want[named], dtype)
    assert (got[~named] == 7.0).all()


I8_SHAPES = [(1, 1, 1), (1, 1000, 768), (3, 17, 33), (8, 1024, 1024), (16, 4096, 96), (17, 63, 2049), (64, 64, 64), (100, 300, 127),
             (129, 257, 128), (300, 500, 640), (1000, 333, 48), (513, 1025, 256), (2, 5, 131071)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", I8_SHAPES, ids=str)
def test_matmul_i8(shape, dtype):
    m, n, k = shape
    g = torch.Generator().manual_seed(m + n + k)
    a, b = (torch.randint(-128, 128, (r, k), generator=g).to(torch.int8) for r in (m, n))
    sa, sb = (torch.exp(torch.randn(r, generator=g)) / 127 / k ** 0.5 for r in (m, n))
    got = rabitq.matmul_i8(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), dtype)
    assert_scaled(got, i8_64(a, sa, b, sb), dtype)


@pytest.mark.parametrize("k", [131071, 65536, 255])
def test_matmul_i8_largest_sums(k):
    # 2^14 k, the largest sum there is, and the largest of the other sign
    a = torch.full((2, k), -128, dtype=torch.int8)
    a[1] = 127
    got = rabitq.matmul_i8(a.cuda(), torch.ones(2, device="cuda"), a.cuda(), torch.ones(2, device="cuda"))
    assert_scaled(got, i8_64(a, torch.ones(2), a, torch.ones(2)), torch.float32)


def test_matmul_i8_scales_that_are_no_numbers():
    a = torch.randint(-127, 128, (20, 64), dtype=torch.int8, device="cuda")
    sa, sb = torch.ones(20, device="cuda"), torch.ones(20, device="cuda")
    sa[3], sb[5] = float("nan"), float("inf")
    got = rabitq.matmul_i8(a, sa, a, sb)
    assert got[3].isnan().all()
    rest = [i for i in range(20) if i != 3]
    cols = [j for j in range(20) if j != 5]
    assert torch.isfinite(got[rest][:, cols]).all() and not torch.isfinite(got[rest][:, 5]).any()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (8, 1024), (5, 1000), (300, 96), (2, 20001), (1000, 256), (64, 4096), (7, 1023),
                                    (6, 2048), (6, 2049), (5, 8191), (3, 8193)])
def test_quantize_rows(rows, k, dtype):
    x = numbers(k, (rows, k), torch.float32)
    x[rows // 2] *= 1000.0
    x[0] *= 1e-6
    x = x.to(dtype)
    codes, scale = rabitq.quantize_rows(x.cuda())
    want, want_scale = codes64(x)
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(codes.cpu(), want)  # whole numbers from one definition


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_quantize_rows_ties_zeros_and_no_numbers(dtype):
    x = torch.zeros(9, 40)
    x[0] = torch.arange(40) - 19.5           # scale 19.5 / 127: borders are hit or missed by rounding
    x[1, 0], x[1, 1:] = 127.0, torch.arange(39) + 0.5   # scale 1: every code but the first is a tie
    x[2] = -x[1]
    x[4, 7] = float("inf")
    x[5, 39] = float("nan")
    x[6, 0] = float("-inf")
    x[7] = torch.finfo(dtype).max
    x[8, :2] = torch.tensor([2.0 ** -149, -2.0 ** -149]) if dtype == torch.float32 else torch.tensor([2.0 ** -24, -2.0 ** -24])
    x = x.to(dtype)
    codes, scale = rabitq.quantize_rows(x.cuda())
    want, want_scale = codes64(x)
    assert torch.equal(codes.cpu(), want)
    assert torch.equal(scale.cpu().isnan(), want_scale.isnan()) and scale[4:7].isnan().all()
    ok = ~want_scale.isnan()
    assert torch.equal(scale.cpu()[ok], want_scale[ok])
    assert scale[3] == 1 and (codes[3:7] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_quantize_rows_of_denormal_numbers(dtype):
    # multiples of the smallest number of the type, up to 1000 and up to where the scale is a normal number again
    step = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
    g = torch.Generator().manual_seed(4)
    rows = [torch.randint(-top, top + 1, (200,), generator=g).double() * step for top in (1, 63, 64, 127, 128, 190, 191, 255, 1000)]
    x = torch.stack(rows + [numbers(5, (200,), torch.float32).double() * 2.0 ** -e for e in (100, 120, 126, 130)]).to(dtype)
    codes, scale = rabitq.quantize_rows(x.cuda())
    want, want_scale = codes64(x)
    assert torch.equal(scale.cpu(), want_scale) and torch.equal(codes.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_quantize_rows_near_ties(dtype):
    # quotients next to a half of both parities: x = (h + 1/2) scale moved by a step of its type to either side
    h = torch.arange(-126, 126).double() + 0.5
    rows = []
    for top in (1.0, 3.7, 0.013, 100.0):
        t = torch.tensor(top).to(dtype).double()
        s = (t / 127).float().double()
        x = (h * s).to(dtype)
        near = torch.stack([x, torch.nextafter(x.float(), torch.tensor(1e9)).to(dtype), torch.nextafter(x.float(), torch.tensor(-1e9)).to(dtype)])
        rows.append(torch.cat([t.to(dtype).reshape(1).expand(3, 1), near], 1))
    x = torch.cat(rows)
    codes, scale = rabitq.quantize_rows(x.cuda())
    want, want_scale = codes64(x)
    assert torch.equal(scale.cpu(), want_scale) and torch.equal(codes.cpu(), want)


# ---- larger tiles and long contractions ----------------------------------------------

def _even(dtype):
    """Elements of 16 bytes."""
    return 16 // torch.empty(0, dtype=dtype).element_size()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,groups,odd", [(1200, 8, 0), (1200, 8, 1), (4500, 2, 0)])
def test_large_products(rows, groups, odd, dtype):
    # 128 x 128 tiles (with rows that do not start at multiples of 16 bytes too) and 256 x 256 tiles: lists that end inside a
    # tile, columns that do, a contraction that ends inside a step
    wide, short = 4096 + 3 * _even(dtype) + odd, 264 + _even(dtype) + odd
    off, ids = lists_from(probes_of(rows, rows, 1, groups, 0, 0.02), groups)
    lists = off.cuda(), ids.cuda(), 1
    x, w = numbers(1, (rows, short), dtype).cuda(), numbers(2, (groups, wide, short), dtype).cuda()
    want, mag, named = forward64(x, w, off, ids, 1)
    got = rabitq.grouped_matmul(x, w, *lists, out=torch.full((rows, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], short, dtype)
    assert (got[~named] == 7.0).all()
    w = numbers(3, (groups, short, wide), dtype).cuda()
    want, mag, named = dx64(x, w, off, ids, 1)
    got = rabitq.grouped_matmul_dx(x, w, *lists, out=torch.full((rows, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], short, dtype)
    assert (got[~named] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,groups,wide,short", [
    (4090, 1, 4096, 136),   # 256 tiles of 256 x 256, some not whole
    (6100, 1, 4088, 136),   # 1536 tiles of 128 x 128
    (8192, 4, 2048, 264),   # lists that end inside a tile of 256
    (4090, 1, 4095, 135),   # the same, rows that do not start at multiples of 16 bytes
    (6100, 1, 4081, 77),
    (8192, 4, 2047, 263),
])
def test_rounds_of_tiles(rows, groups, wide, short, dtype):
    off, ids = lists_from(probes_of(rows, rows, 1, groups, 0, 0.02), groups)
    lists = off.cuda(), ids.cuda(), 1
    x, w = numbers(1, (rows, short), dtype).cuda(), numbers(2, (groups, wide, short), dtype).cuda()
    want, mag, named = forward64(x, w, off, ids, 1)
    got = rabitq.grouped_matmul(x, w, *lists, out=torch.full((rows, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], short, dtype)
    assert (got[~named] == 7.0).all()
    w = numbers(3, (groups, short, wide), dtype).cuda()
    want, mag, named = dx64(x, w, off, ids, 1)
    got = rabitq.grouped_matmul_dx(x, w, *lists, out=torch.full((rows, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], short, dtype)
    assert (got[~named] == 7.0).all()
    n, k = 4096 // groups, wide  # (dw of as many tiles, of few positions)
    off, ids = lists_from(probes_of(5, 300, 1, groups, 0, 0.02), groups)
    dy, x = numbers(4, (300, n), dtype).cuda(), numbers(5, (300, k), dtype).cuda()
    want, mag = dw64(dy, x, off, ids, 1)
    got = rabitq.grouped_matmul_dw(dy, x, off.cuda(), ids.cuda())
    assert_sums(got, want, mag, int((off[1:] - off[:-1]).max()), dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("nq,nprobe,groups,wide,long", [
    (300, 2, 3, 130, 1100),
    (301, 1, 3, 129, 1111),     # rows that do not start at multiples of 16 bytes
    (200, 1, 1, 64, 520),       # of four parts of the contraction the last is empty (16-bit types)
    (200, 1, 1, 64, 263),       # ... (f32), and one ends inside a step
    (700, 1, 2, 72, 8200),
    (2200, 1, 1, 150, 1104),    # more than 512 tiles of 16 x 16, fewer than 256 of 32 x 64
    (1100, 3, 3, 80, 1041),
], ids=str)
def test_few_tiles_of_a_long_contraction(nq, nprobe, groups, wide, long, dtype):
    off, ids = lists_from(probes_of(nq, nq, nprobe, groups, 0, 0.05), groups)
    lists = off.cuda(), ids.cuda(), nprobe
    x, w = numbers(1, (nq, long), dtype), numbers(2, (groups, wide, long), dtype)
    want, mag, named = forward64(x, w, off, ids, nprobe)
    got = rabitq.grouped_matmul(x.cuda(), w.cuda(), *lists, out=torch.full((nq * nprobe, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], long, dtype)
    assert (got[~named] == 7.0).all()
    dy, w = numbers(3, (nq * nprobe, long), dtype), numbers(4, (groups, long, wide), dtype)
    want, mag, named = dx64(dy, w, off, ids, nprobe)
    got = rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), *lists, out=torch.full((nq, wide), 7.0, dtype=dtype, device="cuda"))
    assert_sums(got[named], want[named], mag[named], long * nprobe, dtype)
    assert (got[~named] == 7.0).all()
    if dtype == torch.float32:
        (cx, sx), (cw, sw) = codes64(x), codes64(numbers(2, (groups * wide, long), dtype))
        cw, sw = cw.reshape(groups, wide, long), sw.reshape(groups, wide)
        want, named = grouped_i8_64(cx, sx, cw, sw, off, ids, nprobe)
        got = rabitq.grouped_matmul_i8(cx.cuda(), sx.cuda(), cw.cuda(), sw.cuda(), *lists)
        assert_scaled(got[named], want[named], dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("nq,nprobe,groups,n,k", [
    (500, 2, 4, 2048, 2056),    # 256 x 256 tiles
    (900, 1, 8, 1000, 1032),    # 128 x 128 tiles
    (400, 3, 8, 1001, 1029),    # the same, rows that do not start at multiples of 16 bytes
    (5000, 1, 2, 2048, 2048),   # lists longer than what is known of their pairs at a time
    (70000, 1, 1, 264, 256),    # one list in parts of 2048 and more
    (30000, 2, 3, 130, 72),
    (9000, 1, 40, 24, 40),      # most lists in one part, some in two
], ids=str)
def test_large_dw(nq, nprobe, groups, n, k, dtype):
    probes = probes_of(7, nq, nprobe, groups, 0, 0.01)
    if groups > 8:
        probes = torch.where(torch.rand(probes.shape, generator=torch.Generator().manual_seed(8)) < 0.2, 5, probes)  # a long list
    off, ids = lists_from(probes, groups)
    x, dy = numbers(1, (nq, k), dtype).cuda(), numbers(2, (nq * nprobe, n), dtype).cuda()
    want, mag = dw64(dy, x, off, ids, nprobe)
    got = rabitq.grouped_matmul_dw(dy, x, off.cuda(), ids.cuda(), nprobe)
    assert_sums(got, want, mag, int((off[1:] - off[:-1]).max()), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("m,n,k", [(4200, 4100, 528), (1100, 8200, 272), (1030, 8195, 515), (48, 5000, 3000), (40, 70000, 100), (300, 200, 4100),
                                   (290, 190, 4111)])
def test_large_matmul_i8(m, n, k, dtype):
    g = torch.Generator().manual_seed(m)
    a, b = (torch.randint(-128, 128, (r, k), generator=g).to(torch.int8).cuda() for r in (m, n))
    sa, sb = (torch.exp(torch.randn(r, generator=g)).cuda() for r in (m, n))
    assert_scaled(rabitq.matmul_i8(a, sa, b, sb, dtype), i8_64(a, sa, b, sb), dtype)


@pytest.mark.parametrize("rows,nprobe,groups,n,k", [(2300, 2, 2, 4112, 528), (700, 2, 8, 4104, 528), (3000, 3, 5, 515, 260)])
def test_large_grouped_matmul_i8(rows, nprobe, groups, n, k):
    g = torch.Generator().manual_seed(rows)
    off, ids = lists_from(probes_of(rows, rows, nprobe, groups, 0, 0.02), groups)
    x, w = (torch.randint(-128, 128, s, generator=g).to(torch.int8).cuda() for s in ((rows, k), (groups, n, k)))
    sx, sw = torch.rand(rows, generator=g).cuda(), torch.rand(groups, n, generator=g).cuda()
    want, named = grouped_i8_64(x, sx, w, sw, off, ids, nprobe)
    got = rabitq.grouped_matmul_i8(x, sx, w, sw, off.cuda(), ids.cuda(), nprobe, torch.float32,
                                   torch.full((rows * nprobe, n), 7.0, device="cuda"))
    assert_scaled(got[named], want[named], torch.float32)
    assert (got[~named] == 7.0).all()


# ---- layouts ------------------------------------------------------------------------

def _strided(t, pad, shift):
    """t on the device as a view: rows `pad` elements longer, starting `shift` elements into its memory, NaN (codes: 99) around."""
    fill = 99 if t.dtype == torch.int8 else float("nan")
    shape = (*t.shape[:-1], t.shape[-1] + pad)
    flat = torch.full((t.numel() // max(t.shape[-1], 1) * shape[-1] + shift + 64,), fill, dtype=t.dtype, device="cuda")
    view = flat[shift:shift + torch.Size(shape).numel()].view(shape)[..., :t.shape[-1]]
    view.copy_(t)
    return view, flat


def _untouched(view, flat):
    """Nothing but the view's elements was written."""
    keep = view.clone()
    view.fill_(99 if flat.dtype == torch.int8 else float("nan"))
    ok = bool((flat == 99).all() if flat.dtype == torch.int8 else flat.isnan().all())
    view.copy_(keep)
    return ok


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5), (16, 8)])
@pytest.mark.parametrize("shape", [(40, 2, 3, 96, 128), (300, 1, 2, 131, 77), (200, 2, 2, 256, 250)], ids=str)
def test_strides_and_alignment(shape, pad, shift, dtype):
    nq, nprobe, groups, n, k = shape
    x, w, dy, off, ids = _inputs((*shape, 0, 0), dtype, 5)
    (xs, _), (ws, _), (ds, _) = _strided(x, pad, shift), _strided(w, pad, shift), _strided(dy, pad, shift)
    lists = off.cuda(), ids.cuda(), nprobe
    out, flat = _strided(torch.zeros(nq * nprobe, n, dtype=dtype), pad, shift)
    rabitq.grouped_matmul(xs, ws, *lists, out=out)
    want, mag, _ = forward64(x, w, off, ids, nprobe)
    assert_sums(out, want, mag, k, dtype)
    assert _untouched(out, flat)
    out, flat = _strided(torch.zeros_like(x), pad, shift)
    rabitq.grouped_matmul_dx(ds, ws, *lists, out=out)
    want, mag, _ = dx64(dy, w, off, ids, nprobe)
    assert_sums(out, want, mag, n * nprobe, dtype)
    assert _untouched(out, flat)
    out, flat = _strided(torch.zeros_like(w), pad, shift)
    rabitq.grouped_matmul_dw(ds, xs, *lists, out=out)
    want, mag = dw64(dy, x, off, ids, nprobe)
    assert_sums(out, want, mag, int((off[1:] - off[:-1]).max()), dtype)
    assert _untouched(out, flat)


@pytest.mark.parametrize("pad,shift", [(16, 0), (1, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("m,n,k", [(5, 70, 96), (130, 200, 77), (300, 257, 256)])
def test_strides_and_alignment_of_codes(m, n, k, pad, shift):
    g = torch.Generator().manual_seed(k)
    a, b = (torch.randint(-127, 128, (r, k), generator=g).to(torch.int8) for r in (m, n))
    sa, sb = torch.rand(m, generator=g), torch.rand(n, generator=g)
    out, flat = _strided(torch.zeros(m, n), pad, shift)
    rabitq.matmul_i8(_strided(a, pad, shift)[0], sa.cuda(), _strided(b, pad, shift)[0], sb.cuda(), out=out)
    assert_scaled(out, i8_64(a, sa, b, sb), torch.float32)
    assert _untouched(out, flat)
    x = numbers(3, (m, k), torch.bfloat16)
    codes, flat = _strided(torch.zeros(m, k, dtype=torch.int8), pad, shift)
    _, scale = rabitq.quantize_rows(_strided(x, pad, shift)[0], codes=codes)
    want, want_scale = codes64(x)
    assert torch.equal(codes.cpu(), want) and torch.equal(scale.cpu(), want_scale)
    assert _untouched(codes, flat)


@pytest.mark.parametrize("dtype", [*TYPES, torch.int8], ids=str)
@pytest.mark.parametrize("pad,shift", [(0, 0), (16, 16), (1, 0), (5, 3)])
@pytest.mark.parametrize("nq,nprobe,groups,n,k", [
    (1100, 2, 3, 1032, 272),
    (1100, 2, 3, 1031, 77),
    (600, 1, 2, 1000, 1120),  # few tiles of 64 x 64 of a long contraction, but many of 16 x 16
    (600, 1, 2, 1001, 1111),
    (130, 5, 40, 700, 200),   # lists shorter than a tile, and empty ones
    (200, 8, 48, 720, 1040),
], ids=str)
def test_forward_of_many_small_tiles(nq, nprobe, groups, n, k, pad, shift, dtype):
    real = torch.float32 if dtype == torch.int8 else dtype
    x, w, _, off, ids = _inputs((nq, nprobe, groups, n, k, 0.2, 0.05), real, 6)
    lists = off.cuda(), ids.cuda(), nprobe
    out, flat = _strided(torch.full((nq * nprobe, n), 7.0, dtype=real), pad, shift)
    if dtype == torch.int8:
        (cx, sx), (cw, sw) = codes64(x), codes64(w.reshape(-1, k))
        cw, sw = cw.reshape(w.shape), sw.reshape(groups, n)
        rabitq.grouped_matmul_i8(_strided(cx, pad, shift)[0], sx.cuda(), _strided(cw, pad, shift)[0], sw.cuda(), *lists, out=out)
        want, named = grouped_i8_64(cx, sx, cw, sw, off, ids, nprobe)
        assert_scaled(out[named], want[named], real)
    else:
        rabitq.grouped_matmul(_strided(x, pad, shift)[0], _strided(w, pad, shift)[0], *lists, out=out)
        want, mag, named = forward64(x, w, off, ids, nprobe)
        assert_sums(out[named], want[named], mag[named], k, dtype)
    assert (out[~named] == 7.0).all()
    assert _untouched(out, flat)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 0)])
@pytest.mark.parametrize("nq,nprobe,groups,n,k", [(1100, 2, 3, 272, 1032), (200, 8, 48, 1040, 720), (130, 5, 40, 200, 700)], ids=str)
def test_dx_of_many_small_tiles(nq, nprobe, groups, n, k, pad, shift, dtype):
    _, w, dy, off, ids = _inputs((nq, nprobe, groups, n, k, 0.2, 0.05), dtype, 7)
    out, flat = _strided(torch.full((nq, k), 7.0, dtype=dtype), pad, shift)
    rabitq.grouped_matmul_dx(_strided(dy, pad, shift)[0], _strided(w, pad, shift)[0], off.cuda(), ids.cuda(), nprobe, out=out)
    want, mag, named = dx64(dy, w, off, ids, nprobe)
    assert_sums(out[named], want[named], mag[named], n * nprobe, dtype)
    assert (out[~named] == 7.0).all()
    assert _untouched(out, flat)


def test_offsets_behind_32_bits():
    # rows that lie more than 2^31 elements apart, of every operand
    far = (1 << 31) + 64
    flat = torch.zeros(far + 256, dtype=torch.int8, device="cuda")
    rows = flat.as_strided((2, 96), (far, 1))
    g = torch.Generator().manual_seed(0)
    a = torch.randint(-127, 128, (2, 96), generator=g).to(torch.int8)
    rows.copy_(a)
    one = torch.ones(2, device="cuda")
    want = i8_64(a, one.cpu(), a, one.cpu())
    assert_scaled(rabitq.matmul_i8(rows, one, rows, one), want, torch.float32)
    off = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    w = rows.as_strided((2, 3, 32), (far, 32, 1))
    got = rabitq.grouped_matmul_i8(rows[:, :32], one, w, torch.ones(2, 3, device="cuda"), off)
    assert_scaled(got, torch.stack([a[i].reshape(3, 32).double() @ a[i, :32].double() for i in range(2)]), torch.float32)
    del rows, w, flat
    flat = torch.zeros(far + 256, dtype=torch.bfloat16, device="cuda")
    rows = flat.as_strided((2, 128), (far, 1))
    dy, x = numbers(1, (2, 64), torch.bfloat16), numbers(2, (2, 128), torch.bfloat16)
    m = numbers(3, (2, 64, 128), torch.bfloat16)
    off_cpu = off.cpu()
    rabitq.grouped_matmul_dx(dy.cuda(), m.cuda(), off, out=rows)
    want, mag, _ = dx64(dy, m, off_cpu, None, 1)
    assert_sums(rows, want, mag, 64, torch.bfloat16)
    rows.copy_(x)
    want, mag = dw64(dy, x, off_cpu, None, 1)
    assert_sums(rabitq.grouped_matmul_dw(dy.cuda(), rows, off), want, mag, 1, torch.bfloat16)
    want, mag, _ = forward64(x, m, off_cpu, None, 1)
    assert_sums(rabitq.grouped_matmul(rows, m.cuda(), off), want, mag, 128, torch.bfloat16)
    big = flat.as_strided((2, 8, 16), (far, 16, 1))
    rabitq.grouped_matmul_dw(dy[:, :8].contiguous().cuda(), x[:, :16].contiguous().cuda(), off, out=big)
    want, mag = dw64(dy[:, :8], x[:, :16], off_cpu, None, 1)
    assert_sums(big, want, mag, 1, torch.bfloat16)


# ---- lists --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_sorted_rows_and_positions_outside_of_every_list(dtype):
    # no pair_ids: positions are pairs; the first 5 and the last 30 lie in no list, list 1 is empty
    x, w, dy = numbers(1, (200, 72), dtype), numbers(2, (3, 88, 72), dtype), numbers(3, (200, 88), dtype)
    off = torch.tensor([5, 90, 90, 170], dtype=torch.int32)
    out = torch.full((200, 88), 3.0, dtype=dtype, device="cuda")
    rabitq.grouped_matmul(x.cuda(), w.cuda(), off.cuda(), out=out)
    want, mag, named = forward64(x, w, off, None, 1)
    assert_sums(out[named], want[named], mag[named], 72, dtype)
    assert (out[~named] == 3.0).all() and int(named.sum()) == 165
    dx = torch.full((200, 72), 3.0, dtype=dtype, device="cuda")
    rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), off.cuda(), out=dx)
    want, mag, named = dx64(dy, w, off, None, 1)
    assert_sums(dx[named], want[named], mag[named], 88, dtype)
    assert (dx[~named] == 3.0).all()
    want, mag = dw64(dy, x, off, None, 1)
    assert_sums(rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), off.cuda()), want, mag, 85, dtype)


def test_values_of_other_lists_and_rows_do_not_leak():
    # infinities and NaN in rows of no list, in other rows, and in the matrices of empty lists
    x, w, dy = numbers(1, (150, 136), torch.bfloat16), numbers(2, (4, 72, 136), torch.bfloat16), numbers(3, (150, 72), torch.bfloat16)
    off = torch.tensor([10, 60, 60, 100, 130], dtype=torch.int32)
    inside = torch.zeros(150).bool()
    inside[10:130] = True
    x[~inside], dy[~inside], w[1] = float("nan"), float("inf"), float("nan")
    x[15], dy[20] = float("inf"), float("nan")
    got = rabitq.grouped_matmul(x.cuda(), w.cuda(), off.cuda(), out=torch.zeros(150, 72, dtype=torch.bfloat16, device="cuda")).cpu()
    rows = [i for i in range(10, 130) if i != 15]
    assert torch.isfinite(got[rows]).all() and not torch.isfinite(got[15]).any() and (got[~inside] == 0).all()
    dx = rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), off.cuda(), out=torch.zeros(150, 136, dtype=torch.bfloat16, device="cuda")).cpu()
    rows = [i for i in range(10, 130) if i != 20]
    assert torch.isfinite(dx[rows]).all() and dx[20].isnan().all() and (dx[~inside] == 0).all()
    dw = rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), off.cuda()).cpu()
    assert not torch.isfinite(dw[0]).any() and (dw[1] == 0).all() and torch.isfinite(dw[2:]).all()


def test_offsets_and_pairs_out_of_range_stay_inside():
    # offsets are taken as if they lay in 0 .. pairs, ids that are no pair are passed over
    x, w, dy = numbers(1, (60, 40), torch.float32), numbers(2, (5, 24, 40), torch.float32), numbers(3, (60, 24), torch.float32)
    off = torch.tensor([-7, 20, 20, 45, 1000, 2 ** 31 - 1], dtype=torch.int32)
    ids = torch.randperm(60, generator=torch.Generator().manual_seed(1)).int()
    ids[3], ids[30], ids[59] = -1, 60, 2 ** 31 - 1
    clamped = off.clamp(0, 60)
    out = torch.full((60, 24), 2.0, device="cuda")
    rabitq.grouped_matmul(x.cuda(), w.cuda(), off.cuda(), ids.cuda(), out=out)
    want, mag, named = forward64(x, w, clamped, ids, 1)
    assert int(named.sum()) == 57
    assert_sums(out[named], want[named], mag[named], 40, torch.float32)
    assert (out[~named] == 2.0).all()
    want, mag = dw64(dy, x, clamped, ids, 1)
    assert_sums(rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), off.cuda(), ids.cuda()), want, mag, 60, torch.float32)
    # offsets that descend: nothing is promised of the numbers, but every access stays inside
    down = torch.tensor([60, 30, 50, 10, 40, 0], dtype=torch.int32, device="cuda")
    out, flat = _strided(torch.zeros(60, 24), 8, 0)
    rabitq.grouped_matmul(x.cuda(), w.cuda(), down, out=out)
    assert _untouched(out, flat)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_no_pairs(dtype):
    w = numbers(2, (3, 24, 40), dtype).cuda()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    none = torch.empty(0, 40, dtype=dtype, device="cuda")
    assert rabitq.grouped_matmul(none, w, off).shape == (0, 24)
    assert rabitq.grouped_matmul_dx(torch.empty(0, 24, dtype=dtype, device="cuda"), w, off).shape == (0, 40)
    dw = torch.full((3, 24, 40), 5.0, dtype=dtype, device="cuda")
    rabitq.grouped_matmul_dw(torch.empty(0, 24, dtype=dtype, device="cuda"), none, off, out=dw)
    assert (dw == 0).all()
    codes, scale = rabitq.quantize_rows(none)
    assert codes.shape == (0, 40) and scale.shape == (0,)
    assert rabitq.matmul_i8(codes, scale, codes, scale).shape == (0, 0)


# ---- gradients, streams, graphs ------------------------------------------------------

def test_gradients_against_differences():
    # the product is linear in x and in w, so a difference of two forward passes is the gradient's inner product but for rounding
    nq, nprobe, groups, n, k = 90, 3, 4, 56, 72
    x, w, dy, off, ids = _inputs((nq, nprobe, groups, n, k, 0.2, 0.1), torch.float32, 9)
    out = lambda xx, ww: rabitq.grouped_matmul(xx.cuda(), ww.cuda(), off.cuda(), ids.cuda(), nprobe,
                                               out=torch.zeros(nq * nprobe, n, device="cuda")).double().cpu()
    dx = rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), off.cuda(), ids.cuda(), nprobe, out=torch.zeros(nq, k, device="cuda")).double().cpu()
    dw = rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), off.cuda(), ids.cuda(), nprobe).double().cpu()
    ux, uw = numbers(20, x.shape, torch.float32), numbers(21, w.shape, torch.float32)
    for grad, u, moved in ((dx, ux, out(x + ux, w)), (dw, uw, out(x, w + uw))):
        diff = ((moved - out(x, w)) * dy.double()).sum()
        # every output is off by (k + 1) 2^-23 of its magnitudes; x + ux is rounded too; magnitudes summed over all outputs
        _, mag, _ = forward64(x.abs() + ux.abs(), w.abs() + uw.abs(), off, ids, nprobe)
        tol = 4 * (max(k, n * nprobe, nq * nprobe) + 2) * 2.0 ** -23 * (mag * dy.double().abs()).sum()
        assert abs((grad * u.double()).sum() - diff) <= tol
        assert tol < 0.05 * (grad.abs() * u.double().abs()).sum()  # (the test can fail)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_equal_calls_give_equal_bits(dtype):
    shape = (2000, 2, 5, 264, 136, 0, 0)
    x, w, dy, off, ids = [t.cuda() for t in _inputs(shape, dtype)]
    calls = [lambda: rabitq.grouped_matmul(x, w, off, ids, 2), lambda: rabitq.grouped_matmul_dx(dy, w, off, ids, 2),
             lambda: rabitq.grouped_matmul_dw(dy, x, off, ids, 2)]
    for call in calls:
        first = call()
        for _ in range(3):
            assert torch.equal(call(), first)


def test_on_another_stream_and_two_at_once():
    shape = (600, 2, 6, 192, 160, 0, 0)
    x, w, dy, off, ids = [t.cuda() for t in _inputs(shape, torch.bfloat16)]
    want = rabitq.grouped_matmul(x, w, off, ids, 2), rabitq.grouped_matmul_dx(dy, w, off, ids, 2), rabitq.grouped_matmul_dw(dy, x, off, ids, 2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(3):
                got.append((rabitq.grouped_matmul(x, w, off, ids, 2), rabitq.grouped_matmul_dx(dy, w, off, ids, 2),
                            rabitq.grouped_matmul_dw(dy, x, off, ids, 2)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_captured_and_replayed():
    # a step of training and of serving in one graph, replayed on new inputs with eager work between
    nq, nprobe, groups, n, k = 150, 2, 5, 96, 128
    x, w, dy, off, ids = [t.cuda() for t in _inputs((nq, nprobe, groups, n, k, 0, 0), torch.bfloat16)]
    cw, sw = rabitq.quantize_rows(w.reshape(-1, k))
    cw, sw = cw.reshape(w.shape), sw.reshape(groups, n)

    def step():
        y = rabitq.grouped_matmul(x, w, off, ids, nprobe)
        c, s = rabitq.quantize_rows(x)
        return [y, rabitq.grouped_matmul_dx(dy, w, off, ids, nprobe), rabitq.grouped_matmul_dw(dy, x, off, ids, nprobe),
                rabitq.grouped_matmul_i8(c, s, cw, sw, off, ids, nprobe), rabitq.matmul_i8(c, s, cw[0], sw[0], torch.bfloat16)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        nx, nw, nd, noff, nids = _inputs((nq, nprobe, groups, n, k, 0.3 * (seed % 2), 0), torch.bfloat16, 100 + seed)
        for t, v in ((x, nx), (dy, nd), (off, noff), (ids, nids)):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


# ---- refusals that need tensors of the device ------------------------------------------

def test_binding_refusals():
    x, w = torch.zeros(6, 8, device="cuda"), torch.zeros(3, 5, 8, device="cuda")
    off, ids = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    c, s = torch.zeros(6, 8, dtype=torch.int8, device="cuda"), torch.ones(6, device="cuda")
    cw, sw = torch.zeros(3, 5, 8, dtype=torch.int8, device="cuda"), torch.ones(3, 5, device="cuda")
    refused = [
        lambda: rabitq.grouped_matmul(x[:, :7], w, off, ids),
        lambda: rabitq.grouped_matmul(x, w.half(), off, ids),
        lambda: rabitq.grouped_matmul(x, w.transpose(1, 2), off, ids),
        lambda: rabitq.grouped_matmul(x.t(), w, off, ids),
        lambda: rabitq.grouped_matmul(x, w, off[:3], ids),
        lambda: rabitq.grouped_matmul(x, w, off.long(), ids),
        lambda: rabitq.grouped_matmul(x, w, off, ids[:5]),
        lambda: rabitq.grouped_matmul(x, w, off, ids, 2),
        lambda: rabitq.grouped_matmul(x, w, off, ids, 0),
        lambda: rabitq.grouped_matmul(x, w, off, ids, 1.5),
        lambda: rabitq.grouped_matmul(x, w, off, ids, out=torch.zeros(6, 4, device="cuda")),
        lambda: rabitq.grouped_matmul(x, w, off, ids, out=torch.zeros(6, 5, device="cuda", dtype=torch.half)),
        lambda: rabitq.grouped_matmul(x[:1].expand(6, 8), w, off, ids),
        lambda: rabitq.grouped_matmul(x, w[:1].expand(3, 5, 8), off, ids),
        lambda: rabitq.grouped_matmul(x.cpu(), w, off, ids),
        lambda: rabitq.grouped_matmul(x.requires_grad_(), w, off, ids),
        lambda: rabitq.grouped_matmul_dx(x[:, :4], w, off, ids),
        lambda: rabitq.grouped_matmul_dx(x[:5, :5].contiguous(), w, off, None, 2),
        lambda: rabitq.grouped_matmul_dw(x[:5], x.detach(), off, ids),
        lambda: rabitq.grouped_matmul_dw(x.detach(), x.detach(), off, ids, out=w[:2]),
        lambda: rabitq.quantize_rows(c),
        lambda: rabitq.quantize_rows(x.detach(), codes=c[:5]),
        lambda: rabitq.quantize_rows(x.detach(), scale=s[:5]),
        lambda: rabitq.matmul_i8(c, s, c[:, :7], s),
        lambda: rabitq.matmul_i8(c, s[:5], c, s),
        lambda: rabitq.matmul_i8(c, s.double(), c, s),
        lambda: rabitq.matmul_i8(c, s, c, s, torch.int32),
        lambda: rabitq.grouped_matmul_i8(c, s, cw, sw[:2], off, ids),
        lambda: rabitq.grouped_matmul_i8(c, s, cw, sw.t().contiguous().t(), off, ids),
        lambda: rabitq.grouped_matmul_i8(c, s, cw[:, :, :6], sw, off, ids),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(rabitq.RabitqError):
            call()
            pytest.fail(f"call {i} was not refused")
    with torch.no_grad():  # as a program that keeps its weights as parameters calls it
        assert rabitq.grouped_matmul(x.requires_grad_(), w, off, ids, out=torch.zeros(6, 5, device="cuda")).abs().sum() == 0


def test_rows_behind_32_bits_are_refused():
    long = torch.empty(1, (1 << 32) + 16, dtype=torch.int8, device="cuda")  # (16 elements, were the length cut off)
    s = torch.ones(1, device="cuda")
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for call in (lambda: rabitq.matmul_i8(long, s, long, s),
                 lambda: rabitq.grouped_matmul_i8(long, s, long[None], s[None], off),
                 lambda: rabitq.quantize_rows(long.view(torch.bfloat16).new_empty(1, (1 << 32) + 16))):
        with pytest.raises(rabitq.RabitqError, match="too many"):
            call()


# ---- together -------------------------------------------------------------------------

def test_a_layer_of_experts_behind_the_index():
    """The index routes a batch (coarse_probe), regroups it (build_probe_lists), and the lists' matrices are applied, trained
    and served as codes, on the same pairs."""
    import numpy as np

    from paper_2602_23999_amd import synth
    wl = synth.WORKLOADS["l2_128"].scaled(n=6000, nq=200, n_centres=32)
    data, queries = torch.from_numpy(synth.make_base(wl)).cuda(), torch.from_numpy(synth.make_queries(wl)).cuda()
    D, nlist, nprobe, n = data.shape[1], 24, 3, 80
    rot = np.linalg.qr(np.random.default_rng(0).standard_normal((D, D)))[0].astype(np.float32)
    ix = rabitq.Index.build(data, nlist, 4, rot, center=True)
    q = ix.rotate(queries)
    prep = ix.query_prep(q)
    probes = ix.coarse_probe(q, prep["sq_norm"], nprobe)
    off, ids = ix.build_probe_lists(probes["probe_ids"])
    off_c, ids_c = off.cpu(), ids.cpu()
    w = numbers(1, (nlist, n, D), torch.float32) / D ** 0.5
    y = rabitq.grouped_matmul(q, w.cuda(), off, ids, nprobe)
    # row p belongs to query p // nprobe and to the list that the probe chose for it
    want = torch.stack([w[int(l)].double() @ q.cpu()[p // nprobe].double() for p, l in enumerate(probes["probe_ids"].cpu().flatten())])
    mag = torch.stack([w[int(l)].double().abs() @ q.cpu()[p // nprobe].double().abs() for p, l in enumerate(probes["probe_ids"].cpu().flatten())])
    assert_sums(y, want, mag, D, torch.float32)
    dy = numbers(2, tuple(y.shape), torch.float32)
    want, mag, _ = dx64(dy, w, off_c, ids_c, nprobe)
    assert_sums(rabitq.grouped_matmul_dx(dy.cuda(), w.cuda(), off, ids, nprobe), want, mag, n * nprobe, torch.float32)
    want, mag = dw64(dy, q.cpu(), off_c, ids_c, nprobe)
    assert_sums(rabitq.grouped_matmul_dw(dy.cuda(), q, off, ids, nprobe), want, mag, 200 * nprobe, torch.float32)
    c, s = rabitq.quantize_rows(q)
    cw, sw = rabitq.quantize_rows(w.reshape(-1, D).cuda())
    got = rabitq.grouped_matmul_i8(c, s, cw.reshape(w.shape), sw.reshape(nlist, n), off, ids, nprobe)
    want, _ = grouped_i8_64(c.cpu(), s.cpu(), cw.cpu().reshape(w.shape), sw.cpu().reshape(nlist, n), off_c, ids_c, nprobe)
    assert_scaled(got, want, torch.float32)
    # codes of 8 bits: every factor is off by half a step of its row's scale at most
    full, _, _ = forward64(q.cpu(), w, off_c, ids_c, nprobe)
    half = (s.cpu().double()[:, None] / 2).expand(-1, D), (sw.cpu().double().reshape(nlist, n, 1) / 2).expand(-1, -1, D)
    slack = (forward64(half[0], w.abs(), off_c, ids_c, nprobe)[0] + forward64(q.cpu().abs(), half[1], off_c, ids_c, nprobe)[0]
             + forward64(half[0], half[1], off_c, ids_c, nprobe)[0])
    assert ((got.double().cpu() - full).abs() <= slack * (1 + 1e-5) + 1e-6 * full.abs()).all()
    ix.close()
