"""Products of 8-bit integers with scales, and products by expert, against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_rows_quantize import HALF, inst, padded  # noqa: E402, F401

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}
STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # half a step, relative
LEAST = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}  # of numbers below the normal ones


def whole(g, *shape, high=127):
    return torch.randint(-high, high + 1, shape, generator=g, dtype=torch.int32).to(torch.int8).cuda()


def starts(counts, first=0):
    return torch.tensor([first] + counts).cumsum(0).int().cuda()


def expected(a, w, a_scale=None, w_scale=None, bias=None, gated=False):
    """(value, what binary32 may lose of it) for rows a and one matrix w."""
    a64, w64 = a.double(), w.double()
    y, size = a64 @ w64.T, a64.abs() @ w64.abs().T
    if a.dtype == torch.int8:
        by = (a_scale.double()[:, None] if a_scale is not None else 1.0) * (w_scale.double() if w_scale is not None else 1.0)
        y = y * by
        lost = 3 * HALF * y.abs()  # the sum itself is exact; to binary32, two scales
    else:
        lost = a.shape[1] * 2 * HALF * size  # a rounding (to whichever side) for each product added
    if bias is not None:
        y = y + bias.double()
        lost = lost + HALF * y.abs()
    if gated:
        n = y.shape[1] // 2
        g, up, lg, lu = y[:, :n], y[:, n:], lost[:, :n], lost[:, n:]
        s = g * torch.sigmoid(g)
        y = s * up
        lost = 1.1 * lg * up.abs() + s.abs() * lu + lg * lu * 1.1 + 24 * HALF * y.abs() + 2.0 ** -126 * (g * up).abs()  # (the slope of silu is below 1.1)
    return y, lost


def close(got, y, lost):
    half = STEP[got.dtype]
    off = (got.double() - y).abs()
    bound = lost * (1 + half) + half * y.abs() + LEAST[got.dtype]
    fine = (off <= bound) | (got.double() == y)  # (infinities of fp16 where y is beyond it are looked at by the caller)
    assert fine.all(), (off / bound).max()


# rows that go through each of the kernels' forms, odd ones among them
ROWS = [1, 2, 16, 17, 40, 64, 65, 130, 300]
SIZES = [(1, 1), (7, 5), (16, 16), (33, 40), (127, 129), (128, 64), (130, 257), (1024, 100), (1990, 300)]


@pytest.mark.parametrize("n_in, n_out", SIZES)
@pytest.mark.parametrize("n", ROWS)
def test_scaled(inst, n, n_in, n_out):  # noqa: F811
    g = torch.Generator().manual_seed(n * 10007 + n_in)
    a, w = padded(whole(g, n, n_in), 16, 55), padded(whole(g, n_out, n_in), 16, -99)
    a_scale, w_scale = torch.rand(n, generator=g).cuda() + 0.1, torch.rand(n_out, generator=g).cuda() * 0.01
    bias = torch.randn(n_out, generator=g).cuda() if n_out % 2 else None
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        out = torch.full((n, n_out + 3), -7.0, dtype=dtype, device="cuda")
        scales = dict(a_scale=a_scale, w_scale=w_scale) if dtype != torch.float32 else dict(w_scale=w_scale * 1e-3) if n % 2 else dict(a_scale=a_scale)
        I.maaso_scaled_product(inst, a=a, w=w, out=out[:, :n_out], bias=bias, **scales)
        y, lost = expected(a, w, bias=bias, **scales)
        keep = y.abs() < 60000 if dtype == torch.float16 else torch.ones_like(y, dtype=torch.bool)
        close(out[:, :n_out][keep], y[keep], lost[keep])
        assert (out[:, n_out:] == -7).all()


@pytest.mark.parametrize("n_in, n_out", [(16, 1), (100, 16), (130, 33), (512, 130), (300, 256)])
@pytest.mark.parametrize("n", ROWS)
def test_scaled_and_gated(inst, n, n_in, n_out):  # noqa: F811
    g = torch.Generator().manual_seed(n * 10007 + n_in)
    a, w = padded(whole(g, n, n_in), 16, 55), padded(whole(g, 2 * n_out, n_in), 16, -99)
    a_scale, w_scale = torch.rand(n, generator=g).cuda() + 0.1, (torch.rand(2 * n_out, generator=g).cuda() + 0.5) / (5000 * n_in ** 0.5)
    bias = torch.randn(2 * n_out, generator=g).cuda() if n_out % 2 else None
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((n, n_out), -7.0, dtype=dtype, device="cuda")
        I.maaso_scaled_product(inst, a=a, w=w, out=out, a_scale=a_scale, w_scale=w_scale, bias=bias, gated=True)
        close(out, *expected(a, w, a_scale, w_scale, bias, True))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n_in", [64, 200, 1000])
@pytest.mark.parametrize("name", ["int8", "bf16"])
def test_large(inst, name, n_in, gated):  # noqa: F811
    """Tiles enough for the largest form; whole numbers, so that 16-bit sums are exact too."""
    n, n_out = 4100, 4097 if not gated else 2050
    g = torch.Generator().manual_seed(n_in)
    a, w = whole(g, n, n_in, high=7), whole(g, n_out * (2 if gated else 1), n_in, high=7)
    out = torch.empty(n, n_out, device="cuda")
    if name == "int8":
        a, w = padded(a, 16, 1), padded(w, 16, 1)
        scale = torch.full((n,), 2.0 ** -11, device="cuda")  # (a power of two: exact)
        I.maaso_scaled_product(inst, a=a, w=w, out=out, a_scale=scale, gated=gated)
        y, lost = expected(a, w, a_scale=scale, gated=gated)
    else:
        a, w = padded(a.to(torch.bfloat16) / 64, 8, math.nan), padded(w.to(torch.bfloat16) / 32, 8, math.nan)
        I.maaso_expert_product(inst, a=a, w=w[None], out=out, start=starts([n]), gated=gated)
        y, lost = expected(a, w, gated=gated)
    if gated:
        close(out, y, lost)
    else:
        assert torch.equal(out.double(), y)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", ["int8", "bf16"])
def test_large_and_ragged(inst, name, gated):  # noqa: F811
    """The largest tiles, some of them hardly filled: whole numbers, exact but for the gate; rows of no expert as they were."""
    counts, n = [700, 3, 0, 1030, 129, 250, 900, 1100], 500
    n_in, n_out, rows = 2000 if name == "int8" else 1000, 2048 if gated else 4096, sum(counts) + 9
    g = torch.Generator().manual_seed(17)
    a, w = whole(g, n, n_in, high=7), whole(g, len(counts), n_out * (2 if gated else 1), n_in, high=7)
    if name == "int8":
        a, w, scales = padded(a, 16, 1), padded(w, 16, 1), dict(a_scale=torch.full((n,), 2.0 ** -11, device="cuda"))
    else:
        a, w, scales = padded(a.to(torch.bfloat16) / 64, 8, math.nan), padded(w.to(torch.bfloat16) / 32, 8, math.nan), {}
    token = torch.randint(n, (rows,), generator=g, dtype=torch.int32).cuda()
    out = torch.full((rows, n_out), -7.0, device="cuda")
    I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts(counts, 4), token=token, gated=gated, **scales)
    assert (out[:4] == -7).all() and (out[4 + sum(counts):] == -7).all()
    at = 4
    for i, c in enumerate(counts):
        t = token[at:at + c].long()
        y, lost = expected(a[t], w[i], gated=gated, **({"a_scale": scales["a_scale"][t]} if scales else {}))
        if gated:
            close(out[at:at + c], y, lost)
        else:
            assert torch.equal(out[at:at + c].double(), y)
        at += c


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n, n_in, n_out", [(1000, 2050, 3900), (1010, 4000, 1900), (1900, 2000, 3900), (130, 8000, 4000), (440, 4000, 8000)])
@pytest.mark.parametrize("name", ["int8", "fp16"])
def test_middling(inst, name, n, n_in, n_out, gated):  # noqa: F811
    """Tiles of 128 in four stages and in two, and of 64, at one matrix; whole numbers as above."""
    g = torch.Generator(device="cuda").manual_seed(n + n_in)
    channels = n_out // 2 * 2
    a = torch.randint(-3, 4, (n, n_in), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-3, 4, (channels, n_in), generator=g, device="cuda", dtype=torch.int8)
    out = torch.full((n, channels // (2 if gated else 1)), -7.0, device="cuda")
    if name == "int8":
        a, w, scale = padded(a, 16, 1), padded(w, 16, 1), torch.full((n,), 2.0 ** -11, device="cuda")
        I.maaso_scaled_product(inst, a=a, w=w, out=out, a_scale=scale, gated=gated)
        y, lost = expected(a, w, a_scale=scale, gated=gated)
    else:
        a, w = padded(a.to(torch.float16) / 64, 8, math.nan), padded(w.to(torch.float16) / 32, 8, math.nan)
        I.maaso_expert_product(inst, a=a, w=w[None], out=out, start=starts([n]), gated=gated)
        y, lost = expected(a, w, gated=gated)
    if gated:
        close(out, y, lost)
    else:
        assert torch.equal(out.double(), y)


@pytest.mark.parametrize("counts", [[3, 0, 40, 17, 64, 1, 9, 30], [150, 33, 0, 400, 260, 190, 1, 250]])
@pytest.mark.parametrize("name", ["int8", "bf16"])
def test_many_weights(inst, name, counts):  # noqa: F811
    """More than the tiles read in one order: they begin at unlike steps, and the rows' end lies inside the last."""
    n, n_out, n_in = 100, 4096, 3210 if name == "int8" else 1610
    g = torch.Generator(device="cuda").manual_seed(23)
    a = torch.randint(-7, 8, (n, n_in), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-7, 8, (len(counts), n_out, n_in), generator=g, device="cuda", dtype=torch.int8)
    if name == "bf16":
        a, w = a.to(torch.bfloat16), w.to(torch.bfloat16)
    a, w = padded(a, 16, 1), padded(w, 16, 1)
    assert w.numel() * w.element_size() >= 96 << 20
    token = torch.randint(n, (sum(counts),), generator=g, device="cuda", dtype=torch.int32)
    out = torch.full((sum(counts), n_out), -7.0, device="cuda")
    I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts(counts), token=token)
    at = 0
    for i, c in enumerate(counts):
        assert torch.equal(out[at:at + c].double(), a[token[at:at + c].long()].double() @ w[i].double().T)
        at += c


COUNTS = {
    "one": [5], "few": [3, 0, 1, 12], "empty": [0, 0, 0], "crowd": [0, 1000, 0, 1], "even": [40] * 6, "many": [k % 5 for k in range(70)], "wide": [150, 33, 0, 260],
    "most": [1 if k % 3 else 0 for k in range(1024)],
}


@pytest.mark.parametrize("name", ["bf16", "fp16", "int8"])
@pytest.mark.parametrize("kind", list(COUNTS))
@pytest.mark.parametrize("n_in, n_out, gated", [(64, 48, False), (200, 33, True), (72, 129, False), (9, 3, False), (530, 64, True)])
def test_experts(inst, kind, n_in, n_out, gated, name):  # noqa: F811
    counts, dtype = COUNTS[kind], TYPES[name]
    e, rows, n = len(counts), sum(counts) + 6, 37
    if e == 1024 and n_in > 100:
        pytest.skip("the same as with fewer elements")
    g = torch.Generator().manual_seed(rows * 131 + n_in)
    channels = n_out * (2 if gated else 1)
    if name == "int8":
        a, w = padded(whole(g, n, n_in), 16, 55), padded(whole(g, e, channels, n_in), 16, -99)
        scales = dict(a_scale=torch.rand(n, generator=g).cuda() / 50, w_scale=torch.rand(e, channels, generator=g).cuda() / n_in ** 0.5 / 50)
    else:
        a, w = padded(torch.randn(n, n_in, generator=g).to(dtype).cuda(), 8, math.nan), padded((torch.randn(e, channels, n_in, generator=g) / n_in ** 0.5).to(dtype).cuda(), 8, math.nan)
        scales = {}
    bias = torch.randn(e, channels, generator=g).cuda() if n_out % 2 else None
    token = torch.randint(n, (rows,), generator=g, dtype=torch.int32).cuda()
    start = starts(counts, 2)
    for out_dtype in (torch.float32, dtype if name != "int8" else torch.bfloat16):
        out = torch.full((rows, n_out), -7.0, dtype=out_dtype, device="cuda")
        I.maaso_expert_product(inst, a=a, w=w, out=out, start=start, token=token, bias=bias, gated=gated, **scales)
        assert (out[:2] == -7).all() and (out[rows - 4:] == -7).all()  # rows of no expert
        at = 2
        for i, c in enumerate(counts):
            if c:
                t = token[at:at + c].long()
                s = dict(a_scale=scales["a_scale"][t], w_scale=scales["w_scale"][i]) if scales else {}
                close(out[at:at + c], *expected(a[t], w[i], bias=bias[i] if bias is not None else None, gated=gated, **s))
            at += c


def test_rows_as_they_are_and_weights_in_a_larger_tensor(inst):  # noqa: F811
    """No tokens: row r is row r; the experts' weights are every other one of a model's, their channels part of it."""
    g = torch.Generator().manual_seed(5)
    a, held = torch.randn(90, 96, generator=g).to(torch.bfloat16).cuda(), torch.randn(6, 80, 104, generator=g).to(torch.bfloat16).cuda()
    w, counts = held[::2, 10:60, :96], [30, 20, 40]
    out = torch.empty(90, 50, dtype=torch.bfloat16, device="cuda")
    I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts(counts))
    for i, part in enumerate(out.split(counts)):
        close(part, *expected(a.split(counts)[i], w[i]))


def test_starts_out_of_order(inst):  # noqa: F811
    """As the nearest that are not; the bit is raised; rows of out are written by one expert each."""
    g = torch.Generator().manual_seed(6)
    a, w = torch.randn(50, 64, generator=g).to(torch.bfloat16).cuda(), torch.randn(5, 32, 64, generator=g).to(torch.bfloat16).cuda()
    for given, taken in (([-5, 10, 7, 30, 40, 45], [0, 10, 10, 30, 40, 45]), ([0, 10, 60, 20, 30, 50], [0, 10, 50, 50, 50, 50]),
                         ([50, 0, 0, 0, 0, 0], [50] * 6), ([-2 ** 31, 2 ** 31 - 1, 0, 0, 0, 0], [0, 50, 50, 50, 50, 50])):
        out = torch.full((50, 32), -7.0, device="cuda")
        I.maaso_expert_product(inst, a=a, w=w, out=out, start=torch.tensor(given, dtype=torch.int32, device="cuda"))
        assert I.maaso_instance_status(inst) == I.BAD_BOUND
        seen = torch.zeros(50, dtype=torch.bool, device="cuda")
        for i in range(5):
            lo, hi = taken[i], taken[i + 1]
            if hi > lo:
                close(out[lo:hi], *expected(a[lo:hi], w[i]))
                seen[lo:hi] = True
        assert (out[~seen] == -7).all()


@pytest.mark.parametrize("rows", [20, 200])
def test_tokens_outside(inst, rows):  # noqa: F811
    g = torch.Generator().manual_seed(7)
    a, w = torch.randn(8, 64, generator=g).to(torch.float16).cuda(), torch.randn(2, 40, 64, generator=g).to(torch.float16).cuda()
    token = torch.randint(8, (rows,), generator=g, dtype=torch.int32).cuda()
    token[3], token[11], token[rows - 1] = -1, 8, 2 ** 31 - 1
    out = torch.full((rows, 40), -7.0, device="cuda")
    I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts([rows // 2, rows - rows // 2]), token=token)
    assert I.maaso_instance_status(inst) == I.BAD_ROW
    bad = (token < 0) | (token >= 8)
    assert (out[bad] == -7).all()
    which = torch.arange(rows, device="cuda") >= rows // 2
    for i in range(2):
        keep = ~bad & (which == bool(i))
        close(out[keep], *expected(a[token[keep].long()], w[i]))


def test_what_is_no_number_stays_in_its_row_and_channel(inst):  # noqa: F811
    g = torch.Generator().manual_seed(8)
    for n in (10, 100):
        a, w = torch.randn(n, 72, generator=g).to(torch.bfloat16).cuda(), torch.randn(1, 48, 72, generator=g).to(torch.bfloat16).cuda()
        a[3, 70], w[0, 5, 0] = math.nan, math.inf
        out = torch.empty(n, 48, device="cuda")
        I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts([n]))
        y = a.double() @ w[0].double().T
        assert out[3].isnan().all() and not out[torch.arange(n) != 3][:, torch.arange(48) != 5].isnan().any()
        assert torch.equal(out[:, 5].isinf(), y[:, 5].isinf())
        q, scale = torch.ones(n, 48, dtype=torch.int8, device="cuda"), torch.ones(n, device="cuda")
        scale[2] = math.nan
        out = torch.empty(n, 30, device="cuda")
        I.maaso_scaled_product(inst, a=q, w=torch.ones(30, 48, dtype=torch.int8, device="cuda"), out=out, a_scale=scale)
        assert out[2].isnan().all() and (out[torch.arange(n) != 2] == 48).all()


def test_extremes_of_eight_bits(inst):  # noqa: F811
    """The largest sums there can be, whole."""
    n_in = 131071
    a, w = torch.full((3, n_in + 1), -128, dtype=torch.int8, device="cuda")[:, :n_in], torch.full((2, n_in + 1), -128, dtype=torch.int8, device="cuda")[:, :n_in]
    w[1] = 127
    out = torch.empty(3, 2, device="cuda")
    I.maaso_scaled_product(inst, a=a, w=w, out=out)
    assert torch.equal(out.double().cpu(), torch.tensor([[128.0 * 128 * n_in, -128.0 * 127 * n_in]]).float().double().expand(3, 2))


def test_nothing_to_do(inst):  # noqa: F811
    a, w = torch.zeros(0, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, 32, dtype=torch.int8, device="cuda")
    I.maaso_scaled_product(inst, a=a, w=w, out=torch.zeros(0, 4, device="cuda"))
    I.maaso_expert_product(inst, a=a, w=w[None], out=torch.zeros(0, 4, device="cuda"), start=starts([0]))


def test_rows_far_apart(inst):  # noqa: F811
    """Offsets beyond 32 bits, in a, w and out."""
    far = (1 << 32) + 64
    held = torch.zeros(far * 2, dtype=torch.int8, device="cuda")
    g = torch.Generator().manual_seed(9)
    a, w = torch.as_strided(held, (3, 64), (far // 2 // 16 * 16, 1)), torch.as_strided(held, (3, 64), (far // 2 // 16 * 16, 1), 4096)
    a.copy_(whole(g, 3, 64))
    w.copy_(whole(g, 3, 64))
    out = torch.as_strided(held.view(torch.float32), (3, 3), (far // 8 // 4 * 4, 1), 4096)
    I.maaso_scaled_product(inst, a=a, w=w, out=out)
    assert torch.equal(out.double(), a.double() @ w.double().T)
    wide = torch.as_strided(held, (3, 3, 64), (far // 2 // 16 * 16, 256, 1), 65536)
    wide.copy_(whole(g, 3, 3, 64))
    y = torch.empty(3, 3, device="cuda")
    I.maaso_expert_product(inst, a=a, w=wide, out=y, start=starts([1, 1, 1]))
    for i in range(3):
        assert torch.equal(y[i].double(), (a[i].double() * wide[i].double()).sum(1))
