"""Entries of a page list that are no page of the pool: none is followed, wherever in the list it stands, and what lies before it
is attended to as if the item's keys ended there.  The tolerances are those of test_gpu_kv_attention.py, whose batches these are."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import BF16, E4M3, FP16, Batch, inst  # noqa: E402, F401


def check_seen(b, i, sees):
    """Sequence i's results where its first queries see the keys of `sees` [queries, held + new]."""
    half, group, at, w = torch.finfo(b.dtype).eps / 2, b.heads // b.kv, sum(b.new[:i]), len(sees)
    q, out, lse = b.q_host[at:at + w].double().cuda(), b.out[at:at + w].double(), b.lse[at:at + w].double()
    K = (b.K[i].float() * b.ks[:, None]).double().cuda().repeat_interleave(group, 1)
    V = (b.V[i].float() * b.vs[:, None]).double().cuda().repeat_interleave(group, 1)
    s = torch.einsum("qhd,khd->qhk", q, K) * b.scale
    d = torch.einsum("qhd,khd->qhk", q.abs(), K.abs()).amax(-1) * abs(b.scale) * (b.dim + 4) * 2.0 ** -24
    s = s.masked_fill(~sees.cuda()[:, None], -math.inf)
    ref_lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(ref_lse == -math.inf, 0.0, ref_lse)[..., None])
    ref, mean = torch.einsum("qhk,khd->qhd", p, V), torch.einsum("qhk,khd->qhd", p, V.abs())
    tol = half * ref.abs() + (half + 2 * d[..., None] + 2.0 ** -18) * mean + 1e-30
    if b.dtype == FP16:
        tol = tol + (len(K) + 1) * 2.0 ** -25 * V.abs().amax()
    assert ((out - ref).abs() <= tol).all(), (i, float((out - ref).abs().max()), float(tol.min()))
    assert ((lse == ref_lse) | ((lse - ref_lse).abs() <= d + 2.0 ** -20 * ref_lse.abs().clamp(min=1))).all(), (i, "lse")


def causal(b, i):
    h, w = b.held[i], b.new[i]
    return torch.arange(h + w) <= (h + torch.arange(w))[:, None]


def spoil(b, i, nth, which):
    b.table[int(b.rows[i]), nth] = (-1, b.k.shape[1], 2 ** 31 - 1)[which % 3]


@pytest.mark.parametrize("page, nth", [(p, n) for p in (16, 32, 64) for n in range(min(7, 256 // p))])
@pytest.mark.parametrize("heads, kv, dim, dtype, cache", [(4, 2, 64, BF16, BF16), (8, 1, 128, FP16, E4M3), (2, 1, 256, FP16, FP16)])
def test_few_rows(inst, nth, page, heads, kv, dim, dtype, cache):  # noqa: F811
    """Four waves to an item; the whole list, up to 256 keys, is one item."""
    pages = min(7, 256 // page)
    b = Batch([pages * page - 3 - i for i in range(3)] + [70], [1, 2, 1, 1], heads, kv, dim, page, dtype, cache)
    for i in range(3):
        spoil(b, i, nth, i)
    b.run(inst)
    assert I.maaso_instance_status(inst) == I.BAD_PAGE
    for i in range(3):
        check_seen(b, i, causal(b, i) & (torch.arange(b.total[i]) < nth * page))
    b.check(which=[3])


@pytest.mark.parametrize("heads, kv, dim, dtype, cache", [(8, 8, 64, BF16, BF16), (16, 8, 128, FP16, E4M3), (8, 8, 256, BF16, BF16)])
@pytest.mark.parametrize("page", [16, 32])
def test_very_many_sequences(inst, page, heads, kv, dim, dtype, cache):  # noqa: F811
    """Bad entries at every place of lists of up to 128 keys, in sequences that share blocks with good ones."""
    n = 513
    b = Batch([128 - 1 - i % 20 for i in range(n)], [1] * n, heads, kv, dim, page, dtype, cache)
    spoiled = {i: i // 9 % (128 // page - 1) for i in range(0, n, 9)}
    for i, nth in spoiled.items():
        spoil(b, i, nth, i)
    b.run(inst)
    assert I.maaso_instance_status(inst) == I.BAD_PAGE
    for i, nth in spoiled.items():
        check_seen(b, i, causal(b, i) & (torch.arange(b.total[i]) < nth * page))
    b.check(which=range(1, n, 9))


@pytest.mark.parametrize("nth", range(7))
@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("heads, kv, dim, dtype, cache", [(8, 2, 64, BF16, BF16), (4, 1, 128, FP16, E4M3), (4, 2, 256, BF16, BF16)])
def test_tiles(inst, nth, page, heads, kv, dim, dtype, cache):  # noqa: F811
    pages = 8 if page == 32 else 9
    b = Batch([pages * page - 45, 10], [43, 40], heads, kv, dim, page, dtype, cache)
    spoil(b, 0, nth, nth)
    b.run(inst)
    assert I.maaso_instance_status(inst) == I.BAD_PAGE
    check_seen(b, 0, causal(b, 0) & (torch.arange(b.total[0]) < nth * page))
    b.check(which=[1])


@pytest.mark.parametrize("nth", range(2, 7))
@pytest.mark.parametrize("shared", [32, 40, 48, 57])
def test_behind_a_shared_beginning(inst, nth, shared):  # noqa: F811
    """Items that begin inside a page or a step: the shared keys are the first sequence's, a bad entry ends the own ones."""
    b = Batch([shared + 60, shared + 55, shared + 50], [1, 1, 1], 4, 2, 64, 16, BF16, groups=[(0, 3, shared)])
    spoil(b, 1, nth, nth)
    b.run(inst)
    at, looked_at = torch.arange(b.total[1]), 16 * nth + 15 >= shared and 16 * nth < b.total[1]
    assert I.maaso_instance_status(inst) == (I.BAD_PAGE if looked_at else 0)
    check_seen(b, 1, causal(b, 1) & ((at < shared) | (at < nth * 16)) if looked_at else causal(b, 1))
    b.check(which=[0, 2])


@pytest.mark.parametrize("nth", [0, 1, 62, 63, 64, 65, 126, 127, 128, 129, 250, 311])
@pytest.mark.parametrize("kv, dim", [(2, 64), (1, 128)])
def test_a_long_row(inst, nth, kv, dim):  # noqa: F811
    """Lists of more than 64 entries, in many parts, in few and in one: the other's results are as without, this one's are
    numbers, and exact where the row is one part."""
    b = Batch([5000, 300], [1, 1], 4 * kv, kv, dim, 16, BF16)
    spoil(b, 0, nth, nth)
    with I.maaso_instance_create(workspace_bytes=1 << 14) as few, I.maaso_instance_create(workspace_bytes=1 << 11) as one:
        for on in (inst, few, one):
            b.out.fill_(math.nan)
            b.run(on)
            assert I.maaso_instance_status(on) == I.BAD_PAGE
            assert b.out[0].isfinite().all()
            b.check(which=[1])
        check_seen(b, 0, causal(b, 0) & (torch.arange(b.total[0]) < nth * 16))
