"""Each form of the products with all that a call can ask of it: scales, bias and gate, outputs of 16 and of 32 bits whose rows begin
anywhere, ragged groups beyond 64 experts, weights that are read from unlike steps on, starts out of order.  Whole numbers and powers
of two, so that all is exact in 32 bits but the gate and the output's own rounding."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.product_shapes import DISORDERED, SHAPES  # noqa: E402
from tests.test_gpu_products import close, starts  # noqa: E402
from tests.test_gpu_rows_quantize import HALF, inst, padded  # noqa: E402, F401

TYPES = {"int8": torch.int8, "bf16": torch.bfloat16, "fp16": torch.float16}


def powers(g, low, high, *shape):
    return torch.pow(2.0, torch.randint(low, high + 1, shape, generator=g, device="cuda").float())


def whole(g, name, by, *shape):
    """-7 .. 7, in 16 bits divided by a power of two, with what lies between rows in no sum."""
    t = torch.randint(-7, 8, shape, generator=g, device="cuda", dtype=torch.int8)
    return padded(t, 16, 99) if name == "int8" else padded((t.float() / by).to(TYPES[name]), 8, float("nan"))


def value(a, w, scales, bias, gated):
    """Sums are below 49 * 6500 = 2^18.3 of units of 2^-12 at least (2^-8 in 16 bits) and of 2^-8 at most: exact in 32 bits with their bias."""
    y = a.double() @ w.double().T
    if scales is not None:
        y = y * scales[0].double()[:, None] * scales[1].double()
    y = y + bias.double()
    if not gated:
        return y, torch.zeros_like(y)
    gate, up = y.chunk(2, 1)
    y = gate * torch.sigmoid(gate) * up
    return y, 24 * HALF * y.abs() + 2.0 ** -126 * (gate * up).abs()  # (the gate's exponential, reciprocal and products)


def counts_of(experts, rows):
    """Ragged: every seventh has none, a few many."""
    share = [0 if e % 7 == 3 and experts > 1 else 1 + (e * 37 % 11) ** 2 for e in range(experts)]
    counts = [rows * s // sum(share) for s in share]
    counts[0] += rows - sum(counts)
    return counts


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(int(x)) if isinstance(x, bool) else str(x) for x in s))
def test_every_form(inst, shape, name, gated):  # noqa: F811
    _, _, experts, rows, channels, in_bytes = shape
    if name != "int8" and experts == 0:
        experts = 1
    n_in, n_out, e = in_bytes // (1 if name == "int8" else 2), channels // (2 if gated else 1), max(experts, 1)
    g = torch.Generator(device="cuda").manual_seed(rows + channels)
    n = rows if experts == 0 else 411
    a, w = whole(g, name, 16, n, n_in), whole(g, name, 16, e, channels, n_in)
    scales = (powers(g, -7, -5, n), powers(g, -5, -3, e, channels)) if name == "int8" else None
    bias = torch.randint(-64, 65, (e, channels), generator=g, device="cuda") / 64.0
    given = dict(bias=bias, gated=gated, **(dict(a_scale=scales[0], w_scale=scales[1]) if scales else {}))
    counts = counts_of(e, rows) if experts else [rows]
    token = torch.randint(n, (rows + 5,), generator=g, device="cuda", dtype=torch.int32) if experts else None
    outs = []
    for out_type, step in ((torch.float32, 1), (TYPES[name] if name != "int8" else torch.bfloat16, 8), (TYPES[name] if name != "int8" else torch.float16, 1)):
        if out_type == torch.float16 and gated:
            continue  # (a gate of some 700 times as much is beyond it)
        out = padded(torch.full((rows + 5 if experts else rows, n_out), -7.0, dtype=out_type, device="cuda"), step, -9.0)
        if experts:
            I.maaso_expert_product(inst, a=a, w=w, out=out, start=starts(counts, 2), token=token, **given)
            assert (out[:2] == -7).all() and (out[rows + 2:] == -7).all()
            outs.append(out[2:rows + 2])
        else:
            I.maaso_scaled_product(inst, a=a, w=w[0], out=out, **{k: v[0] if k in ("w_scale", "bias") else v for k, v in given.items()})
            outs.append(out)
        assert (torch.as_strided(out, (out.shape[0] - 1, out.stride(0)), (out.stride(0), 1))[:, n_out:] == -9).all()
    at = 0
    for i, c in enumerate(counts):
        t = token[2 + at:2 + at + c].long() if experts else slice(None)
        y, lost = value(a[t], w[i], (scales[0][t], scales[1][i]) if scales else None, bias[i], gated)
        for out in outs:
            close(out[at:at + c], y, lost)
        at += c
    assert at == rows and I.maaso_instance_status(inst) == 0


def disorder(kind, start, rows):
    """Starts in order, and what is done to them: at the ends, on either side of a group of 64 experts, and far out."""
    s, e = list(start), len(start) - 1
    at = [x for x in (63, 64, 65, 127, 128, 129) if x < e] or [e // 2]
    if kind == "back":
        for x in at:
            s[x] = s[max(0, x - 5)]
        s[0] = -5
    elif kind == "ahead":
        for x in at:
            s[x] = s[min(e, x + 3)]
        s[1] = s[3]
    elif kind == "below":
        for x in at[::2]:
            s[x] = -2 ** 31
        s[e] = 0
    else:
        s[at[-1]] = 2 ** 31 - 1
        s[e] = rows + 1
    return s


@pytest.mark.parametrize("kind", ["back", "ahead", "below", "beyond"])
@pytest.mark.parametrize("shape", DISORDERED, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("name", ["int8", "bf16"])
def test_starts_out_of_order(inst, name, shape, kind):  # noqa: F811
    """As the nearest that are not; the bit is raised; rows of out are written by one expert each, the others left."""
    _, experts, rows, channels, in_bytes = shape
    n_in = in_bytes // (1 if name == "int8" else 2)
    g = torch.Generator(device="cuda").manual_seed(rows + experts)
    a, w = whole(g, name, 16, 300, n_in), whole(g, name, 16, experts, channels, n_in)
    token = torch.randint(300, (rows,), generator=g, device="cuda", dtype=torch.int32)
    given = disorder(kind, starts(counts_of(experts, rows)).tolist(), rows)
    taken, last = [], 0
    for s in given:
        last = max(last, min(max(s, 0), rows))
        taken.append(last)
    assert taken != given
    out = torch.full((rows, channels), -7.0, device="cuda")
    I.maaso_expert_product(inst, a=a, w=w, out=out, start=torch.tensor(given, dtype=torch.int32, device="cuda"), token=token)
    assert I.maaso_instance_status(inst) == I.BAD_BOUND
    assert (out[:taken[0]] == -7).all() and (out[taken[-1]:] == -7).all()
    for i in range(experts):
        lo, hi = taken[i], taken[i + 1]
        if hi > lo:
            assert torch.equal(out[lo:hi].double(), a[token[lo:hi].long()].double() @ w[i].double().T), (i, lo, hi)
