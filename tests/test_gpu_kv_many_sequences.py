"""Attention for very many short sequences, where a wave takes an item alone (4096 items or more of few keys on average), and the
join of many rows, eight tokens to a block.  Batches and tolerances are those of test_gpu_kv_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import BF16, E4M3, FP16, Batch, inst  # noqa: E402, F401

# sequences, heads, key heads, head dim, page, types; the last items of 1367 * 3 leave three waves of a block without one
FORMS = [(520, 8, 8, 64, 16, BF16, BF16), (1367, 9, 3, 64, 128, FP16, FP16), (1367, 3, 3, 64, 32, BF16, E4M3), (520, 16, 8, 64, 64, FP16, E4M3),
         (1367, 6, 3, 128, 16, BF16, BF16), (520, 8, 8, 128, 64, FP16, FP16), (1030, 20, 4, 128, 32, BF16, E4M3), (1367, 3, 3, 128, 128, FP16, E4M3),
         (1367, 3, 3, 256, 16, BF16, BF16), (1030, 8, 4, 256, 32, FP16, FP16), (520, 24, 8, 256, 64, BF16, E4M3), (1367, 3, 3, 256, 16, FP16, E4M3)]


@pytest.mark.parametrize("n, heads, kv, dim, page, dtype, cache", FORMS)
def test_single_tokens(inst, n, heads, kv, dim, page, dtype, cache):  # noqa: F811
    """Rows of one part each, of nothing but the new token among them: written as they are."""
    assert n * kv >= 4096
    held = [i % 100 if i % 5 == 0 else i % 31 for i in range(n)]
    assert sum(held) + n <= 64 * n
    Batch(held, [1] * n, heads, kv, dim, page, dtype, cache).run(inst).check()
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("n, heads, kv, dim, page, dtype, cache", FORMS)
def test_some_long_rows_and_several_tokens(inst, n, heads, kv, dim, page, dtype, cache):  # noqa: F811
    """Rows of several parts among them, sequences of up to three new tokens and of none."""
    held, new = [900 + i if i % 61 == 7 else i % 41 for i in range(n)], [(1, 1, 3, 1, 0, 2, 1)[i % 7] if heads // kv * 3 <= 16 else 1 for i in range(n)]
    held = [h if h < 900 else 900 + h % 300 for h in held]
    assert sum(held) + sum(new) <= 64 * n
    b = Batch(held, new, heads, kv, dim, page, dtype, cache)
    b.run(inst).check()
    b.out.fill_(9.0)
    b.run(inst, lse=None, total_len=30 * n).check()
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("n, heads, kv, dim, page, dtype, cache", FORMS[::3])
def test_beside_tiles(inst, n, heads, kv, dim, page, dtype, cache):  # noqa: F811
    """A few sequences of many new tokens among them."""
    held, new = [i % 37 for i in range(n)], [1] * n
    for at, w in ((3, 40), (n // 2, 170), (n - 1, 33)):
        new[at] = w
    Batch(held, new, heads, kv, dim, page, dtype, cache).run(inst).check()
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("n, heads, kv, dim, page, dtype, cache", FORMS[1::4])
def test_behind_a_shared_beginning(inst, n, heads, kv, dim, page, dtype, cache):  # noqa: F811
    """Groups of few rows, whose shared keys a wave takes alone as well, and sequences outside every group."""
    per = max(1, 16 // (heads // kv))
    groups = [(f, f + per, 150 + f % 90) for f in range(10, 10 + 30 * per, per)]
    shared = {i: s for f, e, s in groups for i in range(f, e)}
    held = [shared.get(i, 0) + i % 29 for i in range(n)]
    Batch(held, [1] * n, heads, kv, dim, page, dtype, cache, groups=groups).run(inst, max_shared=240).check()
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("heads, kv, dim, dtype, cache, new", [
    (64, 8, 256, BF16, E4M3, [130, 0, 65, 1, 7, 3, 255, 2, 90, 1, 4]), (66, 22, 128, FP16, FP16, [400, 1, 1, 1, 9, 6, 300, 700, 3, 110]),
    (120, 30, 64, BF16, BF16, [501, 900, 5, 1, 64, 2, 70])])
def test_joins_of_many_tokens(inst, heads, kv, dim, dtype, cache, new):  # noqa: F811
    """Blocks of eight tokens: sequences of one part and of several in one block, some that hold nothing else, a last block that is
    not full."""
    tokens, groups = sum(new), -(-heads // (256 // dim))
    held = [(3000, 0, 300, 4500, 5, 0)[i % 6] for i in range(len(new))]
    assert tokens * groups >= 32768 and tokens % 8
    Batch(held, new, heads, kv, dim, 64, dtype, cache).run(inst).check()
    assert I.maaso_instance_status(inst) == 0
