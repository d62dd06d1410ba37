"""The adjustment of logits against the definition: binary32, one rounding per operation, so bit for bit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402


@pytest.fixture(scope="module")
def inst():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only machines)")
    with I.maaso_instance_create() as x:
        yield x


def i32(a):
    return torch.tensor(np.array(a), dtype=torch.int32, device="cuda")


def f32(a):
    return torch.tensor(np.array(a), dtype=torch.float32, device="cuda")


def reference(logits, c):
    """(x before the last rounding, chosen), numpy in float32 (each operation rounded once)."""
    x = logits.float().numpy().copy()
    n, vocab = x.shape
    chosen = np.full(n, -1)
    with np.errstate(all="ignore"):
        for r in range(n):
            if "history" in c:
                times = np.bincount(c["history"][c["history_start"][r]:c["history_start"][r + 1]], minlength=vocab).astype(np.float32)
                said = times > 0
                rep, f, p = (np.float32(c[k][r]) if k in c else np.float32(d) for k, d in (("repetition", 1), ("frequency", 0), ("presence", 0)))
                y = np.where(x[r] > 0, x[r] / rep, x[r] * rep)
                x[r] = np.where(said, y - (f * times + p), x[r])
            if "bias_token" in c:
                b = slice(c["bias_start"][r], c["bias_start"][r + 1])
                x[r][c["bias_token"][b]] += c["bias_value"][b]
            if "temperature" in c:
                x[r] = x[r] / np.float32(c["temperature"][r])
            if "mask" in c:
                row = c["mask_row"][r] if "mask_row" in c else r
                if row >= 0:
                    bits = (c["mask"][row].view(np.uint32)[:, None] >> np.arange(32, dtype=np.uint32)) & 1
                    x[r][bits.reshape(-1)[:vocab] == 0] = -np.inf
            y = np.where(np.isnan(x[r]), -np.inf, x[r])
            if y.max() > -np.inf:
                chosen[r] = int(np.argmax(y))
    return x, chosen


def make(rng, n, vocab, history, biases, masked):
    c = {}
    if history is not None:
        length = [0] + [int(x) for x in rng.integers(0, history + 1, n - 1)] if n > 1 else [history]
        c.update(history=rng.integers(0, max(1, min(vocab, vocab // 3)), sum(length)).astype(np.int32), history_start=np.concatenate([[0], np.cumsum(length)]).astype(np.int32),
                 repetition=(1 + rng.random(n)).astype(np.float32), frequency=rng.random(n).astype(np.float32), presence=rng.random(n).astype(np.float32))
    if biases is not None:
        count = [int(x) for x in rng.integers(0, min(vocab, biases) + 1, n)]
        c.update(bias_token=np.concatenate([np.sort(rng.permutation(vocab)[:k]) for k in count] or [[]]).astype(np.int32), bias_value=rng.normal(size=sum(count)).astype(np.float32),
                 bias_start=np.concatenate([[0], np.cumsum(count)]).astype(np.int32))
    if masked is not None:
        c.update(mask=rng.integers(-2 ** 31, 2 ** 31, (max(1, masked), (vocab + 31) // 32)).astype(np.int32), mask_row=rng.integers(-1, max(1, masked), n).astype(np.int32))
    c["temperature"] = (0.3 + rng.random(n)).astype(np.float32)
    return c


def on_gpu(c):
    return {k: f32(v) if v.dtype == np.float32 else i32(v) for k, v in c.items()}


def check(inst, logits, c, out_type, chosen=True, view=None):
    """logits: on the host; view: the tensor on the GPU that holds them, where it is a view."""
    x = logits.cuda() if view is None else view
    out = torch.full(tuple(logits.shape), 7.0, dtype=out_type, device="cuda")
    got = torch.full((len(logits),), 7, dtype=torch.int32, device="cuda") if chosen else None
    I.maaso_logits_adjust(inst, logits=x, out=out, chosen=got, **on_gpu(c))
    assert I.maaso_instance_status(inst) == 0
    want, which = reference(logits, c)
    want = torch.from_numpy(want)
    same = (out.cpu() == want.to(out_type)) | (want.isnan() & out.cpu().isnan())
    assert same.all(), int((~same).sum())
    if chosen:
        assert got.tolist() == which.tolist()


@pytest.mark.parametrize("dtype, out_type", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32),
                                             (torch.float16, torch.float16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("n, vocab, history, biases, masked", [
    (1, 1, 3, 1, 1), (2, 7, 5, 3, 1), (3, 8, 0, None, None), (5, 33, 40, 9, 2), (1, 8191, 300, 50, None), (4, 8192, 300, 50, 3), (2, 8193, 30, 0, 1),
    (3, 32000, 5000, 100, 2), (2, 50257, 2000, 64, 2), (7, 20011, None, 17, None), (2, 131072, 70000, 300, 1)])
def test_definition(inst, dtype, out_type, n, vocab, history, biases, masked):
    rng = np.random.default_rng(vocab + n)
    logits = (3 * torch.randn(n, vocab, generator=torch.Generator().manual_seed(n))).to(dtype)
    check(inst, logits, make(rng, n, vocab, history, biases, masked), out_type)


def test_one_token_said_very_often(inst):
    c = dict(history=np.full(200000, 5, np.int32), history_start=np.array([0, 200000], np.int32), frequency=np.array([0.01], np.float32))
    check(inst, torch.zeros(1, 100), c, torch.float32)


def test_every_part_alone(inst):
    rng = np.random.default_rng(3)
    logits = torch.randn(4, 1000, generator=torch.Generator().manual_seed(3))
    c = make(rng, 4, 1000, 200, 20, 2)
    history = {k: c[k] for k in ("history", "history_start")}
    for part in ({}, dict(temperature=c["temperature"]), {**history, "repetition": c["repetition"]}, {**history, "frequency": c["frequency"]}, {**history, "presence": c["presence"]},
                 {k: c[k] for k in ("bias_token", "bias_value", "bias_start")}, dict(mask=c["mask"], mask_row=c["mask_row"]), history):
        check(inst, logits, part, torch.float32)
    check(inst, logits, dict(mask=rng.integers(-2 ** 31, 2 ** 31, (4, 32)).astype(np.int32)), torch.float32)  # mask r for row r


def test_ties_go_to_the_lowest_token(inst):
    logits = torch.zeros(5, 40000)
    logits[0, [9000, 30000, 39999]] = 2.0
    logits[1, 39999] = 1.0
    logits[2] = -0.0
    logits[2, 20000] = 0.0
    logits[3] = -5.0
    logits[4, ::2] = -1.0
    check(inst, logits, {}, torch.float32)
    check(inst, logits.bfloat16(), {}, torch.bfloat16)


def test_not_finite(inst):
    inf, nan = float("inf"), float("nan")
    logits = torch.randn(7, 9000)
    logits[0] = -inf
    logits[1] = nan
    logits[2, 8500] = nan
    logits[3, 77] = inf
    logits[4, [5, 8999]] = inf
    logits[5] = -inf
    logits[5, 8998] = -3e38
    mask = np.full((2, 282), -1, np.int32)
    mask[1] = 0
    check(inst, logits, {}, torch.float32)
    check(inst, logits, dict(mask=mask, mask_row=np.array([0, 0, 1, 1, 0, 0, 1], np.int32)), torch.float32)
    check(inst, logits, dict(temperature=np.full(7, 0.5, np.float32)), torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_apart_and_odd_starts(inst, dtype):
    rng = np.random.default_rng(5)
    for pad, start in ((8, 0), (1, 0), (16, 3)):
        flat = torch.randn(3 * (9001 + pad) + start, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        view = flat[start:].view(3, -1)[:, :9001]
        check(inst, view.cpu(), make(rng, 3, 9001, 50, 5, 1), torch.float32, view=view)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_in_place_and_without_outputs(inst, dtype):
    rng = np.random.default_rng(6)
    logits = torch.randn(3, 20000, generator=torch.Generator().manual_seed(1)).to(dtype)
    c = make(rng, 3, 20000, 500, 20, 2)
    want, which = reference(logits, c)
    x, got = logits.cuda(), i32([7] * 3)
    I.maaso_logits_adjust(inst, logits=x, chosen=got, **on_gpu(c))
    assert got.tolist() == which.tolist() and torch.equal(x.cpu(), logits)
    I.maaso_logits_adjust(inst, logits=x, out=x, **on_gpu(c))
    assert torch.equal(x.cpu(), torch.from_numpy(want).to(dtype))


@pytest.mark.parametrize("over, bit", [
    (dict(history=[5, 40, 3]), I.BAD_TOKEN), (dict(history=[5, -1, 3]), I.BAD_TOKEN), (dict(history_start=[0, 4]), I.BAD_BOUND), (dict(history_start=[2, 1]), I.BAD_BOUND),
    (dict(history_start=[-1, 3]), I.BAD_BOUND), (dict(bias_token=[7, 2]), I.BAD_TOKEN), (dict(bias_token=[2, 2]), I.BAD_TOKEN), (dict(bias_token=[2, 40]), I.BAD_TOKEN),
    (dict(bias_start=[0, 3]), I.BAD_BOUND), (dict(mask_row=[2]), I.BAD_ROW)])
def test_out_of_range_is_ignored(inst, over, bit):
    c = dict(history=[5, 5, 3], history_start=[0, 3], bias_token=[2, 7], bias_start=[0, 2], mask_row=[0])
    c.update(over)
    out = torch.empty(1, 40, device="cuda")
    I.maaso_logits_adjust(inst, logits=torch.ones(1, 40, device="cuda"), out=out, chosen=i32([0]), bias_value=f32([1, 1]), mask=i32([[-1, -1], [-1, -1]]),
                          frequency=f32([0.25]), **{k: i32(v) for k, v in c.items()})
    assert I.maaso_instance_status(inst) == bit
    assert out.isfinite().all()


def test_a_graph(inst):
    rng = np.random.default_rng(8)
    logits = torch.randn(3, 20000)
    c = on_gpu(make(rng, 3, 20000, 500, 20, 2))
    x, out, got = logits.cuda(), torch.zeros(3, 20000, device="cuda"), i32([0] * 3)
    I.maaso_logits_adjust(inst, logits=x, out=out, chosen=got, **c)
    want, which = out.clone(), got.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        I.maaso_logits_adjust(inst, logits=x, out=out, chosen=got, **c)
    for _ in range(3):
        out.zero_()
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(got, which)
        I.maaso_logits_adjust(inst, logits=-x, chosen=got)


@pytest.mark.parametrize("biases", [511, 512, 513, 5000])
def test_many_biases(inst, biases):
    rng = np.random.default_rng(biases)
    tokens = np.sort(rng.permutation(20000)[:biases]).astype(np.int32)
    c = dict(bias_token=tokens, bias_value=rng.normal(size=biases).astype(np.float32), bias_start=np.array([0, biases, biases]),
             history=np.concatenate([tokens[:100], tokens[:50]]), history_start=np.array([0, 150, 150]), frequency=np.full(2, 0.5, np.float32))
    check(inst, torch.randn(2, 20000, generator=torch.Generator().manual_seed(2)), {k: v.astype(np.float32 if v.dtype == np.float32 else np.int32) for k, v in c.items()}, torch.float32)


def test_a_history_of_more_than_a_million_tokens(inst):
    history = np.concatenate([np.full(2 ** 20 + 5, 7), np.arange(3000)]).astype(np.int32)
    c = dict(history=history, history_start=np.array([0, len(history)], np.int32), frequency=np.array([1e-5], np.float32), presence=np.array([0.5], np.float32),
             bias_token=np.array([3, 7], np.int32), bias_value=np.array([1.5, 100.0], np.float32), bias_start=np.array([0, 2], np.int32))
    check(inst, torch.randn(1, 5000, generator=torch.Generator().manual_seed(3)), c, torch.float32)


def test_biases_out_of_order_by_several(inst):
    out, tokens = torch.empty(1, 4096, device="cuda"), np.tile([9, 2], 200)
    for _ in range(2):
        I.maaso_logits_adjust(inst, logits=torch.ones(1, 4096, device="cuda"), out=out, chosen=i32([0]), bias_token=i32(tokens), bias_value=f32(np.ones(400)), bias_start=i32([0, 400]))
        assert I.maaso_instance_status(inst) == I.BAD_TOKEN
        assert out.isfinite().all() and (out[0, 10:] == 1).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1.0, 1e30])
@pytest.mark.parametrize("temperature", [1e-9, 0.7, 1.0, 3.0, 1e10])
def test_divisions_over_the_whole_range(inst, scale, temperature):
    logits = torch.randn(2, 6000, generator=torch.Generator().manual_seed(4)) * scale
    logits[0, ::7] *= 1e-4
    logits[1, ::11] = 0
    check(inst, logits, dict(temperature=np.array([temperature, temperature * 1.1], np.float32)), torch.float32)


@pytest.mark.parametrize("n", [1, 3, 900, 1025])
def test_few_and_many_rows(inst, n):
    """Rows whose blocks choose together, and rows whose choices are joined by a launch of their own."""
    rng = np.random.default_rng(n)
    logits = torch.randint(-3, 4, (n, 9001), generator=torch.Generator().manual_seed(n)).float()
    for _ in range(2):
        check(inst, logits, make(rng, n, 9001, 30, 3, 2), torch.float32)
