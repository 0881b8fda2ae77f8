"""mb_matmul_q8 in every form that it takes a product in, each named by the library (mb_matmul_q8_form) and checked, so that
another choice of forms cannot leave one untested: single CTAs with one tile and with several, sums in two, four and eight
parts, stages of one, two and four blocks, pairs of CTAs with one tile and with several, low and high tiles.

Values are whole numbers of at most 2, scales 1/2, 1 or 2: every product is a whole number of quarters below 64 of them, every
sum of K below 2^24 / 64 = 2^18 of those is exact in fp32 whatever its order. So fp32 results have the bits of the product
in 64 bits, and bf16 results those of its one rounding."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

from test_serve_chain_gpu import Chain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _matrix(rows, width, block_rows, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randint(-2, 3, (rows, width), device=DEV, generator=g).float().to(E4M3)
    s = torch.randint(126, 129, (-(-rows // block_rows), mb.mb_q8_scale_stride(width)), device=DEV, generator=g)
    return q, s.to(torch.uint8)


def _wide(q, s, block_rows):
    f = torch.exp2(s.double() - 127).repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.double() * f


def _product(a, sa, w, sw):
    return _wide(a, sa, 1) @ _wide(w, sw, 128).t()


def _inputs(rows, n, width):
    return (*_matrix(rows, width, 1, rows + width), *_matrix(n, width, 128, n + width + 1))


def _is(rows, n, width, dtype, form):
    got = mb.mb_matmul_q8_form(rows, n, width, dtype)
    for k, v in form.items():
        assert (got[k] > 1 if v == "more" else got[k] == v), (k, got)


ONE, MORE = dict(pair=1, parts=1, tiles=1), dict(pair=1, parts=1, tiles="more")
PAIR, PAIRS = dict(pair=2, parts=1, deep=1, tiles=1), dict(pair=2, parts=1, deep=1, tiles="more")
FORMS = [
    # one tile to a CTA: lowest, low, middle, high; stages of 4, 2 and 1 blocks
    (1, 4096, 1024, dict(ONE, height=16, deep=4)), (16, 8, 1296, dict(ONE, height=16, deep=4)), (64, 4608, 2304, dict(ONE, height=32, deep=4)),
    (600, 264, 2320, dict(ONE, deep=4)), (1003, 2072, 1552, dict(ONE, height=128, deep=2)), (2739, 912, 1040, dict(ONE, height=160, deep=1)),
    # several tiles to a CTA: of the lowest, and of the highest (two sums of 224 rows; in fp32 moved in two goes)
    (1, 20976, 400, dict(MORE, height=16, deep=4)), (40, 19720, 1040, dict(MORE, height=64, deep=2)),
    (40000, 128, 272, dict(MORE, height=224, deep=1)), (40100, 120, 1040, dict(MORE, height=224, deep=1)),
    # parts of a sum
    (256, 2304, 4608, dict(parts=2, deep=2)), (585, 424, 3408, dict(parts=2, deep=4)), (500, 2304, 16384, dict(parts=2, deep=2)),
    (129, 5656, 12960, dict(parts=2, deep=1)), (1, 2304, 4608, dict(parts=4, height=16)), (64, 2304, 4608, dict(parts=4, deep=4)),
    (384, 1040, 16384, dict(parts=4, deep=2)), (129, 2584, 12960, dict(parts=4, deep=1)), (1, 264, 9232, dict(parts=8, height=16)),
    (130, 264, 9232, dict(parts=8, deep=4)), (33, 1184, 4736, dict(parts=8, deep=2)), (129, 1992, 9264, dict(parts=4, deep=2)),
    (160, 1816, 9264, dict(parts=8, deep=1)), (1, 1992, 16384, dict(parts=8, deep=1, height=16)), (3588, 8, 24592, dict(parts=8, deep=1, height=192)),
    # pairs of CTAs: one tile, several, in bands of tiles
    (65, 12416, 9264, PAIR), (1600, 1040, 9232, PAIR), (65, 19720, 144, PAIRS), (100, 19592, 640, PAIRS), (300, 20104, 1040, PAIRS),
    (1100, 19592, 656, PAIRS), (2500, 9352, 400, PAIRS), (4100, 2312, 1040, PAIRS),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, n, width, form", FORMS, ids=lambda v: "-".join(f"{k}{x}" for k, x in v.items()) if isinstance(v, dict) else str(v))
def test_exact_sums(rows, n, width, form, dtype):
    _is(rows, n, width, TYPES[dtype], form)
    a, sa, w, sw = _inputs(rows, n, width)
    room = torch.full((rows * n + 4096,), 7.0, dtype=TYPES[dtype], device=DEV)
    room[:rows * n] = float("nan")
    out = room[:rows * n].view(rows, n)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out, ws=ws)
    assert torch.equal(out, _product(a, sa, w, sw).float().to(TYPES[dtype]))
    assert (room[rows * n:] == 7.0).all()
    again = torch.empty_like(out)
    mb.mb_matmul_q8(a, sa, w, sw, again)
    assert torch.equal(out, again) and mb.mb_check(ws) == (mb.MB_OK, -1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, parts, part, width, form", [
    (300, 2, 9856, 1040, PAIRS), (1600, 2, 512, 9232, PAIR), (100, 7, 2816, 272, PAIRS), (40000, 2, 128, 144, dict(pair=2, tiles="more")),
    (30, 2, 9856, 272, MORE)])
def test_groups_of_columns_come_apart(rows, parts, part, width, form, dtype):
    n = parts * part
    _is(rows, n, width, TYPES[dtype], form)
    a, sa, w, sw = _inputs(rows, n, width)
    apart = torch.full((parts, rows, part), float("nan"), dtype=TYPES[dtype], device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, apart)
    want = _product(a, sa, w, sw).float().to(TYPES[dtype])
    assert torch.equal(apart.transpose(0, 1).reshape(rows, n), want)


NUMBERS = [(300, 19848, 640, PAIRS), (1600, 1040, 9232, PAIR), (1100, 20104, 400, PAIRS), (40000, 128, 400, MORE), (40, 19720, 400, MORE),
           (65, 2312, 4624, dict(parts=2)), (64, 2304, 4608, dict(parts=4)), (130, 264, 9232, dict(parts=8)), (256, 2304, 4608, dict(parts=2))]


@pytest.mark.parametrize("rows, n, width, form", NUMBERS, ids=str)
def test_what_is_no_number_stays_in_its_sums(rows, n, width, form):
    _is(rows, n, width, torch.float32, form)
    a, sa, w, sw = _inputs(rows, n, width)
    want = _product(a, sa, w, sw)
    a.view(torch.uint8)[1, width - 3] = 0x7f   # NaN among the values of a row, of W's last; scales that are none
    sa[rows - 1, 2] = 255
    w.view(torch.uint8)[n - 1, 3] = 0xff
    want[1], want[rows - 1], want[:, n - 1] = float("nan"), float("nan"), float("nan")
    out = torch.empty(rows, n, device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out)
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(), want.float().nan_to_num())
    sw[0, 1] = 255   # and one of 128 columns of out
    want[:, :128] = float("nan")
    mb.mb_matmul_q8(a, sa, w, sw, out)
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(), want.float().nan_to_num())


@pytest.mark.parametrize("rows, n, width, form", [(300, 19848, 256, PAIRS), (1600, 1040, 9216, PAIR), (40000, 128, 256, MORE),
                                                  (130, 264, 9216, dict(parts=8))], ids=str)
def test_scales_at_their_ends(rows, n, width, form):
    _is(rows, n, width, torch.float32, form)
    a, w = (torch.ones(k, width, device=DEV).to(E4M3) for k in (rows, n))
    out = torch.empty(rows, n, device=DEV)
    for x, y, want in ((0, 254, float(width)), (254, 0, float(width)), (127, 127, float(width)), (1, 1, 0.0), (254, 254, float("inf")),
                       (64, 190, float(width))):
        sa = torch.full((rows, mb.mb_q8_scale_stride(width)), x, dtype=torch.uint8, device=DEV)
        sw = torch.full((-(-n // 128), mb.mb_q8_scale_stride(width)), y, dtype=torch.uint8, device=DEV)
        mb.mb_matmul_q8(a, sa, w, sw, out)
        assert (out == want).all(), (x, y, out[0, 0])


CHAINS = [(300, 272, 19712, 264), (1100, 512, 9856, 2312)]


def _pairs(size):
    rows, width, inner, vocab = size
    _is(rows, inner, width, torch.bfloat16, PAIRS)


@pytest.mark.parametrize("size", CHAINS, ids=str)
def test_chain_and_graph(size):
    """norm -> product of pairs -> quantise -> product -> draw, without a wait between, then captured and replayed."""
    _pairs(size)
    c = Chain(*size, seed=21)
    for _ in range(5):
        c.run()
    c.want()
    first = [t.clone() for t in c.outputs()]
    c.run()
    assert all(torch.equal(t, f) for t, f in zip(c.outputs(), first)) and mb.mb_check(c.ws)[0] == mb.MB_OK
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    c.residual0.normal_()
    for t in c.outputs():
        t.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    c.want()


def test_streams_at_once():
    """Products of pairs, in parts and of single CTAs on streams of their own: they share SMs and tensor memory."""
    sizes = [CHAINS[0], (64, 2304, 4608, 264), (256, 4608, 2304, 256)]
    _pairs(sizes[0])
    chains = [Chain(*size, seed=31 + i) for i, size in enumerate(sizes)]
    streams = [torch.cuda.Stream() for _ in chains]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s in zip(chains, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c in chains:
        c.want()
