"""Attention where a row is longer, or a sequence has more queries, than the call's bounds say: what lies beyond is left out, and
the rest is what it is without it.  Batches and tolerances are those of test_gpu_kv_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import BF16, E4M3, FP16, Batch, inst  # noqa: E402, F401
from tests.test_gpu_kv_bad_pages import causal, check_seen  # noqa: E402

FORMS = [(4, 2, 64, 16, BF16, BF16), (8, 1, 128, 64, FP16, E4M3), (6, 2, 256, 32, BF16, BF16)]


@pytest.mark.parametrize("held", [60, 3000])
@pytest.mark.parametrize("heads, kv, dim, page, dtype, cache", FORMS)
@pytest.mark.parametrize("max_q, new", [(1, [3, 1, 0, 2]), (2, [1, 9, 2]), (20, [41, 5, 20, 21, 170])])
def test_more_queries_than_the_bound(inst, heads, kv, dim, page, dtype, cache, held, max_q, new):  # noqa: F811
    b = Batch([held + 5 * i for i in range(len(new))], new, heads, kv, dim, page, dtype, cache)
    b.out.fill_(9.0)
    b.run(inst, max_q=max_q)
    assert I.maaso_instance_status(inst) == I.BAD_BOUND
    for i, w in enumerate(new):
        at, kept = sum(new[:i]), min(w, max_q)
        if kept:
            check_seen(b, i, causal(b, i)[:kept])
        assert (b.out[at + kept:at + w] == 9).all() and (b.lse[at + kept:at + w] == 9).all()


@pytest.mark.parametrize("heads, kv, dim, page, dtype, cache", FORMS)
@pytest.mark.parametrize("max_len, held, new", [(90, [100, 20, 88], [1, 1, 4]), (2000, [1995, 2500, 30], [30, 60, 50]), (64, [30, 63, 0], [64, 2, 3])])
def test_longer_rows_than_the_bound(inst, heads, kv, dim, page, dtype, cache, max_len, held, new):  # noqa: F811
    """Queries whose own keys are left out see all that is before, others what they see otherwise."""
    b = Batch(held, new, heads, kv, dim, page, dtype, cache)
    b.run(inst, max_len=max_len)
    assert I.maaso_instance_status(inst) == I.BAD_BOUND
    for i in range(len(new)):
        check_seen(b, i, causal(b, i) & (torch.arange(b.total[i]) < max_len))


@pytest.mark.parametrize("heads, kv, dim, page, dtype, cache", FORMS)
def test_behind_a_shared_beginning(inst, heads, kv, dim, page, dtype, cache):  # noqa: F811
    new, shared = [1, 4, 2, 1, 5], 200
    b = Batch([shared + 30 * i for i in range(5)], new, heads, kv, dim, page, dtype, cache, groups=[(0, 5, shared)])
    b.out.fill_(9.0)
    b.run(inst, max_q=2, max_len=290)
    assert I.maaso_instance_status(inst) == I.BAD_BOUND
    for i, w in enumerate(new):
        kept = min(w, 2)
        check_seen(b, i, causal(b, i)[:kept] & (torch.arange(b.total[i]) < 290))
        at = sum(new[:i])
        assert (b.out[at + kept:at + w] == 9).all()
