"""Outputs so large that they are written past the caches: copied pages of more than 32 MiB, queries of more than 32 MiB, logits
of more than 8 MiB.  Formulas and tolerances are those of test_gpu_kv_append.py and test_gpu_logits.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_append import BF16, E4M3, FP16, case  # noqa: E402
from tests.test_gpu_logits import check, i32, inst, make, on_gpu, reference  # noqa: E402, F401

FP32 = torch.float32


@pytest.mark.parametrize("dtype, layers, kv, page, dim, n", [
    (BF16, 4, 8, 64, 128, 40), (E4M3, 2, 5, 64, 64, 450), (FP16, 3, 3, 16, 64, 1100), (BF16, 1, 7, 128, 256, 41), (E4M3, 5, 1, 16, 128, 2000)])
def test_copied_pages(inst, dtype, layers, kv, page, dim, n):  # noqa: F811
    """Pages of whole pieces of 16 KiB, of some and a rest, of less than one; pairs left out among them."""
    pool = 2 * n + 3
    assert n * layers * kv * page * dim * dtype.itemsize * 2 > 32 << 20
    raw = [torch.randint(0, 256, (layers, pool, kv * page * dim * dtype.itemsize), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(s)) for s in (1, 2)]
    k, v = raw[0].view(dtype).view(layers, pool, kv, page, dim), raw[1].view(dtype).view(layers, pool, kv, dim, page)
    pairs = torch.randperm(pool, generator=torch.Generator().manual_seed(3))[:2 * n].view(n, 2).int()
    pairs[5::9] = -1
    kept = pairs[pairs[:, 0] >= 0].long().cuda()
    want = [x.clone() for x in raw]
    for x in want:
        x[:, kept[:, 1]] = x[:, kept[:, 0]]
    I.maaso_kv_copy(inst, I.KvCache(k, v), pairs=pairs.cuda())
    assert I.maaso_instance_status(inst) == 0
    assert all(torch.equal(a, b) for a, b in zip(raw, want))


@pytest.mark.parametrize("over", [{}, dict(odd=True), dict(in_place=True), dict(in_place=True, odd=True)])
@pytest.mark.parametrize("dtype, cache, tokens, heads, kv, dim, rotary, norm, interleaved, page", [
    (BF16, BF16, 4211, 32, 2, 128, 128, True, False, 64), (FP16, E4M3, 2111, 33, 1, 256, 64, True, True, 16), (BF16, BF16, 4111, 65, 1, 64, 64, False, False, 128)])
def test_written_queries(inst, dtype, cache, tokens, heads, kv, dim, rotary, norm, interleaved, page, over):  # noqa: F811
    """At addresses that are multiples of 16 bytes and not, in place and elsewhere."""
    assert tokens * heads * dim * 2 > 32 << 20
    case(inst, dtype, tokens, heads, kv, dim, rotary, norm, interleaved, page, cache=cache, **over)


@pytest.mark.parametrize("dtype, out_type, n, vocab", [
    (FP32, FP32, 17, 131072), (BF16, FP32, 70, 131072), (BF16, BF16, 33, 131072), (FP16, FP16, 70, 131072), (FP16, FP16, 110, 40008), (BF16, FP32, 30, 100004)])
def test_adjusted_logits(inst, dtype, out_type, n, vocab):  # noqa: F811
    """In slices of 1024 tokens and of 4096, with a last one that is not whole, in 16 bits and in 32."""
    assert n * vocab * out_type.itemsize > 8 << 20 and vocab * out_type.itemsize % 16 == 0
    logits = (3 * torch.randn(n, vocab, generator=torch.Generator().manual_seed(n))).to(dtype)
    check(inst, logits, make(np.random.default_rng(n), n, vocab, 400, 30, 2), out_type)


@pytest.mark.parametrize("dtype, n, vocab, stride", [(BF16, 70, 131072, 131072), (FP16, 33, 131071, 131072), (FP32, 30, 100003, 100004), (BF16, 50, 100003, 100008)])
def test_adjusted_logits_in_place(inst, dtype, n, vocab, stride):  # noqa: F811
    """Rows further apart than they are long: what lies between stays."""
    flat = torch.randn(n, stride, generator=torch.Generator().manual_seed(n)).to(dtype)
    c = make(np.random.default_rng(n), n, vocab, 300, 20, 2)
    want, which = reference(flat[:, :vocab], c)
    x, got = flat.cuda(), i32([7] * n)
    view = x[:, :vocab]
    assert n * vocab * dtype.itemsize > 8 << 20 and stride * dtype.itemsize % 16 == 0
    I.maaso_logits_adjust(inst, logits=view, out=view, chosen=got, **on_gpu(c))
    assert I.maaso_instance_status(inst) == 0
    assert torch.equal(view.cpu(), torch.from_numpy(want).to(dtype)) and got.tolist() == which.tolist()
    assert torch.equal(x[:, vocab:].cpu(), flat[:, vocab:])
