"""Attention where the sequences' queries do not fill n_tok, as in a captured step with idle places: the sequences' results are
those of their formula, and the places of no sequence are left as they are.  Batches and tolerances are those of
test_gpu_kv_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import BF16, E4M3, FP16, Batch, inst  # noqa: E402, F401


def run_and_check(inst, b, before, n_tok, **over):  # noqa: F811
    """The batch's queries from place `before` on among n_tok; the others' places hold 9 before and after."""
    tokens = sum(b.new)
    q, out = (torch.full((n_tok, b.heads, b.dim), 9.0, dtype=b.dtype, device="cuda") for _ in range(2))
    lse = torch.full((n_tok, b.heads), 9.0, device="cuda")
    mine = slice(before, before + tokens)
    q[mine] = b.q
    b.run(inst, q=q, out=out, lse=lse, q_start=b.q_start + before, **over)
    assert I.maaso_instance_status(inst) == 0
    idle = torch.ones(n_tok, dtype=torch.bool, device="cuda")
    idle[mine] = False
    assert (out[idle] == 9).all() and (lse[idle] == 9).all()
    b.out, b.lse = out[mine], lse[mine]
    b.check()


FORMS = [(BF16, BF16, 8, 2, 64, 16), (FP16, E4M3, 4, 1, 128, 64), (BF16, BF16, 8, 2, 256, 32)]


@pytest.mark.parametrize("before", [0, 3])
@pytest.mark.parametrize("held", [50, 3000])
@pytest.mark.parametrize("dtype, cache, heads, kv, dim, page", FORMS)
def test_a_sequence_of_fewer_queries_than_most(inst, dtype, cache, heads, kv, dim, page, held, before):  # noqa: F811
    """n * max_q is n_tok, and yet the last sequences have few rows: 8 of them, 4, none."""
    for new in ([8, 8, 8, 2], [8, 1, 0, 0, 8], [0, 8, 3]):
        b = Batch([held - 7 * i for i in range(len(new))], new, heads, kv, dim, page, dtype, cache)
        run_and_check(inst, b, before, 8 * len(new), max_q=8)


@pytest.mark.parametrize("before", [0, 1])
@pytest.mark.parametrize("held", [40, 3000])
@pytest.mark.parametrize("dtype, cache, heads, kv, dim, page", FORMS)
def test_single_tokens_and_idle_sequences(inst, dtype, cache, heads, kv, dim, page, held, before):  # noqa: F811
    """n_tok is n, and yet token i is not of sequence i."""
    for new in ([1, 0, 1], [0, 1, 1, 1], [1, 1, 0, 0, 1, 0, 1, 0, 0]):
        b = Batch([held - 4 * i for i in range(len(new))], new, heads, kv, dim, page, dtype, cache)
        run_and_check(inst, b, before, len(new), max_q=1)


@pytest.mark.parametrize("shared", [32, 700])
@pytest.mark.parametrize("dtype, cache, heads, kv, dim, page", FORMS)
def test_a_shared_beginning(inst, dtype, cache, heads, kv, dim, page, shared):  # noqa: F811
    for new in ([1, 0, 1, 1, 0, 0, 1], [0, 0, 1, 1, 0, 1, 1] * 3):
        n = len(new)
        b = Batch([shared + 1 + 37 * i % 90 for i in range(n)], new, heads, kv, dim, page, dtype, cache, groups=[(0, n - 2, shared), (n - 2, n, 16)])
        run_and_check(inst, b, 0, n, max_q=1)
        run_and_check(inst, b, 2, n + 5, max_q=1)


@pytest.mark.parametrize("heads, kv, dim", [(8, 8, 64), (16, 8, 128)])
def test_very_many_sequences(inst, heads, kv, dim):  # noqa: F811
    n = 600
    b = Batch([i % 300 for i in range(n)], [i % 3 % 2 for i in range(n)], heads, kv, dim, 16, BF16)
    run_and_check(inst, b, 5, n, max_q=1)


def test_nobody_at_all(inst):  # noqa: F811
    b = Batch([700, 3], [0, 0], 4, 2, 64, 16, BF16)
    run_and_check(inst, b, 0, 2, max_q=1)
    run_and_check(inst, b, 2, 40, max_q=20)
