"""Routing and joining against plain forms in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_products import LEAST, STEP  # noqa: E402
from tests.test_gpu_rows_quantize import HALF, inst, padded  # noqa: E402, F401

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def plain(logits, k, bias, sigmoid, renorm, scale):
    x = logits.double().cpu()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=torch.finfo(torch.float32).max)
    e = torch.exp(x - torch.where(x.amax(1, keepdim=True) > -math.inf, x.amax(1, keepdim=True), torch.zeros(())))
    p = torch.sigmoid(x) if sigmoid else e / e.sum(1, keepdim=True).clamp(min=1e-300)
    score = x
    if bias is not None:
        score = torch.where(x > -math.inf, p + bias.double().cpu(), x)
        score = torch.where(score.isnan(), -math.inf, score)
    order = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :k]
    there = score.gather(1, order) > -math.inf
    w = torch.where(there, p.gather(1, order), torch.zeros((), dtype=torch.float64))
    if renorm:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total.clamp(min=1e-300), torch.zeros((), dtype=torch.float64))
    return torch.where(there, order, -1), w * scale, p


def check(inst, logits, k, bias=None, sigmoid=False, renorm=True, scale=1.0):  # noqa: F811
    n, e = logits.shape
    expert = torch.full((n, k), -9, dtype=torch.int32, device="cuda")
    weight = torch.full((n, k), -9.0, device="cuda")
    start = torch.full((e + 1,), -9, dtype=torch.int32, device="cuda")
    token, place = torch.full((n * k,), -9, dtype=torch.int32, device="cuda"), torch.full((n, k), -9, dtype=torch.int32, device="cuda")
    I.maaso_expert_route(inst, logits=logits, expert=expert, weight=weight, start=start, token=token, place=place, bias=bias, sigmoid=sigmoid, renorm=renorm, scale=scale)
    want, w, p = plain(logits, k, bias, sigmoid, renorm, scale)
    assert torch.equal(expert.cpu().long(), want)
    # an exponential (two steps), its argument (a difference of numbers up to 88 apart that have an exponential at all, half a step of it), sums of e
    # numbers in parts of 16 and six joins, a quotient; of the sum of the chosen k more; the scale
    rel = (2 * 2 + 88 + 22 + 2 + (88 + 4 + 22 + k + 2 if renorm else 0) + 1) * HALF
    assert ((weight.double().cpu() - w).abs() <= rel * w.abs() + 2.0 ** -126 * (1 if not renorm else abs(scale))).all()
    flat = want.flatten()
    order = torch.sort(torch.where(flat < 0, e, flat), stable=True)[1]
    live = int((flat >= 0).sum())
    assert torch.equal(token.cpu().long(), torch.cat([order[:live] // k, torch.full((n * k - live,), -1)]))
    back = torch.full((n * k,), -1)
    back[order[:live]] = torch.arange(live)
    assert torch.equal(place.cpu().long().flatten(), back)
    assert torch.equal(start.cpu().long(), torch.cat([torch.zeros(1, dtype=torch.long), torch.bincount(flat[flat >= 0], minlength=e).cumsum(0)]))
    again = [torch.empty_like(t) for t in (expert, weight)]
    I.maaso_expert_route(inst, logits=logits, expert=again[0], weight=again[1], bias=bias, sigmoid=sigmoid, renorm=renorm, scale=scale)
    assert torch.equal(again[0], expert) and torch.equal(again[1], weight)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("e, k", [(1, 1), (2, 1), (5, 5), (8, 2), (60, 4), (64, 6), (65, 8), (128, 1), (160, 32), (256, 8), (300, 7), (512, 3), (1000, 10), (1024, 32)])
def test_experts(inst, e, k, name):  # noqa: F811
    g = torch.Generator().manual_seed(e * 37 + k)
    for n in (1, 3, 70, 256, 257, 700):
        logits = padded((torch.randn(n, e, generator=g) * 2).to(TYPES[name]).cuda(), 1, math.inf)
        check(inst, logits, k, renorm=bool(n % 2), scale=2.5 if n == 70 else 1.0)
        check(inst, logits, k, sigmoid=True, renorm=n % 2 == 0)
        check(inst, logits, k, bias=torch.randn(e, generator=g).cuda() * 0.2, sigmoid=True)


def test_many_tokens(inst):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    for n, e, k in ((20000, 8, 2), (16384, 256, 8), (5000, 1024, 4)):
        logits = torch.randn(n, e, generator=g).cuda()
        check(inst, logits, k)
        check(inst, logits, k, bias=torch.randn(e, generator=g).cuda() * 0.2, sigmoid=True)


@pytest.mark.parametrize("n", [5, 300])
def test_equals_go_to_the_lowest(inst, n):  # noqa: F811
    logits = torch.zeros(n, 100, dtype=torch.bfloat16, device="cuda")
    logits[:, 50] = 1
    logits[:, 70] = 1
    check(inst, logits, 6)
    check(inst, logits, 6, bias=torch.zeros(100, device="cuda"), sigmoid=True)
    check(inst, -torch.zeros(n, 100, device="cuda") + 0.0, 3)
    signed = torch.zeros(n, 8, device="cuda")
    signed[:, ::2] = -0.0  # equal to 0
    check(inst, signed, 4)


@pytest.mark.parametrize("n", [7, 400])
def test_experts_that_are_not_chosen(inst, n):  # noqa: F811
    """Masked ones, rows with fewer than k left, rows with none, the types' lowest and largest values."""
    g = torch.Generator().manual_seed(2)
    low = torch.finfo(torch.float32).min
    logits = torch.randn(n, 70, generator=g)
    logits[0] = -math.inf
    logits[1] = math.nan
    logits[2, 3:] = -math.inf
    logits[3] = low
    logits[4, :] = math.inf
    logits[5, ::3] = math.nan
    logits[6, 7], logits[6, 9] = math.inf, -low
    for k in (1, 4, 8):
        check(inst, logits.cuda(), k)
        check(inst, logits.cuda(), k, renorm=False)
        check(inst, logits.cuda(), k, sigmoid=True)
        bias = torch.randn(70, generator=g)
        bias[1], bias[2], bias[3] = math.nan, -math.inf, low
        check(inst, logits.cuda(), k, bias=bias.cuda(), sigmoid=True)


def test_scores_next_to_each_other(inst):  # noqa: F811
    """Sigmoids that are equal in 32 bits and not in 64, and far out where they all are next to 0 or 1."""
    g = torch.Generator().manual_seed(3)
    base = torch.randn(64, 1, generator=g)
    near = (base.double() * (1 + torch.randint(-3, 4, (64, 96), generator=g) * 2.0 ** -23)).float()
    for logits in (near, near - 30, near + 12, near * 20):
        check(inst, logits.cuda(), 8, bias=torch.zeros(96, device="cuda"), sigmoid=True)
        check(inst, logits.cuda(), 8, bias=(torch.randint(-2, 3, (96,), generator=g) * 2.0 ** -24).cuda(), sigmoid=True)


@pytest.mark.parametrize("n", [6, 300])
def test_shares_of_logits_far_below_zero(inst, n):  # noqa: F811
    """Their sigmoids are no numbers of 32 bits any more, the quotients by their sum are; the lowest value is none."""
    g = torch.Generator().manual_seed(4)
    logits = torch.randn(n, 90, generator=g) * 4
    for t, by in enumerate((-60.0, -90.0, -100.0, -200.0, -600.0)):
        logits[t] += by
    logits[5, 1:] -= 75.0  # one expert that is liked and others whose shares are still numbers
    logits[5, 0] = -12.0
    for k in (1, 3, 8):
        check(inst, logits.cuda(), k, sigmoid=True)
        check(inst, logits.cuda(), k, sigmoid=True, bias=(torch.randn(90, generator=g) * 0.1).cuda(), scale=2.5)
        check(inst, logits.cuda(), k, sigmoid=True, renorm=False)
    low = torch.full((n, 90), torch.finfo(torch.float32).min)
    low[0, 7] = -300.0
    check(inst, low.cuda(), 4, sigmoid=True)


def test_no_tokens(inst):  # noqa: F811
    start = torch.full((9,), -9, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    I.maaso_expert_route(inst, logits=torch.empty(0, 8, device="cuda"), expert=none.view(0, 2), weight=torch.empty(0, 2, device="cuda"), start=start, token=none, place=none)
    assert (start == 0).all()


@pytest.mark.parametrize("n, e, k", [((1 << 22) + 1030, 9, 2), ((1 << 23) + 5, 70, 1), ((1 << 26) - 1, 513, 1)])
def test_choosing_by_several_launches(inst, n, e, k):  # noqa: F811
    """More tokens than one launch takes (2^22), up to the most with 64 lanes to each: token t likes expert t % e, then the next."""
    t = torch.arange(n, device="cuda")
    logits = torch.zeros(n, e, dtype=torch.bfloat16, device="cuda")
    for j in range(k):
        logits.view(-1)[t * e + (t + j) % e] = 3.0 - j
    expert, weight = torch.full((n, k), -9, dtype=torch.int32, device="cuda"), torch.full((n, k), -9.0, device="cuda")
    I.maaso_expert_route(inst, logits=logits, expert=expert, weight=weight, renorm=True)
    share = torch.tensor([3.0 - j for j in range(k)], dtype=torch.float64).softmax(0)
    for j in range(k):
        assert torch.equal(expert[:, j], ((t + j) % e).int())
        assert (weight[:, j].double() - share[j].item()).abs().max().item() <= 32 * HALF
    del logits, t, expert, weight
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("n, k, width", [(1, 1, 1), (3, 2, 7), (16, 2, 2048), (33, 8, 100), (5, 32, 130), (200, 3, 513)])
def test_joining(inst, n, k, width, name):  # noqa: F811
    g = torch.Generator().manual_seed(n * 31 + width)
    dtype, rows = TYPES[name], n * k + 3
    y = padded(torch.randn(rows, width, generator=g).to(dtype).cuda(), 8 if k != 3 else 1, math.nan)
    residual = padded(torch.randn(n, width, generator=g).to(dtype).cuda(), 8 if n != 33 else 3, math.nan)
    place = torch.randperm(rows, generator=g)[:n * k].view(n, k).int()
    place[0, 0] = -1
    place = place.cuda()
    weight = torch.randn(n, k, generator=g).cuda()
    weight[0, 0] = math.nan  # of a place that is not there
    for w, r in ((weight, residual), (None, residual), (weight, None)):
        out = padded(torch.full((n, width), -7.0, dtype=dtype, device="cuda"), 8 if k < 3 else 5, 5.0)
        I.maaso_expert_combine(inst, y=y, place=place, out=out, weight=w, residual=r)
        gone = (place < 0)[..., None]
        part = torch.where(gone, 0.0, y[place.clamp(min=0).long()].double() * (w.double()[..., None] if w is not None else 1.0))
        want, size = part.sum(1), part.abs().sum(1)
        if r is not None:
            want, size = want + r.double(), size + r.double().abs()
        assert ((out.double() - want).abs() <= (k + 1) * HALF * size * (1 + STEP[dtype]) + STEP[dtype] * want.abs() + LEAST[dtype]).all()
        if n > 1:
            assert (torch.as_strided(out, (n - 1, out.stride(0)), (out.stride(0), 1))[:, width:] == 5).all()
    held = residual.clone()
    I.maaso_expert_combine(inst, y=y, place=place, out=held, residual=held)
    other = torch.empty_like(held)
    I.maaso_expert_combine(inst, y=y, place=place, out=other, residual=residual)
    assert torch.equal(held, other)


def test_places_outside(inst):  # noqa: F811
    y = torch.ones(6, 16, device="cuda")
    place = torch.tensor([[0, 6], [2 ** 31 - 1, 5], [-1, -2 ** 31]], dtype=torch.int32, device="cuda")
    out = torch.full((3, 16), -7.0, device="cuda")
    I.maaso_expert_combine(inst, y=y, place=place, out=out)
    assert I.maaso_instance_status(inst) == I.BAD_ROW
    assert out[:, 0].tolist() == [1.0, 1.0, 0.0]
    I.maaso_expert_combine(inst, y=torch.empty(0, 16, device="cuda"), place=torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 0).all()


def test_joining_by_several_launches(inst):  # noqa: F811
    """Out of more than 2^33 elements, which takes two launches: the tokens on either side of the seam, and the last."""
    width, n = 1 << 20, (1 << 13) + 3
    y = torch.arange(4 * width, device="cuda").remainder(251).view(4, width).to(torch.bfloat16)  # whole numbers: every step is exact
    place = torch.arange(n, device="cuda", dtype=torch.int32).remainder(4).unsqueeze(1)
    weight = torch.arange(n, device="cuda").remainder(3).sub(1).float().unsqueeze(1)
    out = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    I.maaso_expert_combine(inst, y=y, place=place, out=out, weight=weight)
    for t in (0, 1, 4095, 8190, 8191, 8192, 8193, n - 1):
        assert torch.equal(out[t], y[t % 4] * (t % 3 - 1)), t
