"""The instance's calls on several streams, captures among them."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import BF16, Batch, i32, inst  # noqa: E402, F401


def attend(inst, b, rows, stream):  # noqa: F811
    I.maaso_kv_attention(inst, b.view, b.pages, layer=0, q=b.q, out=b.out, lse=b.lse, q_start=b.q_start, rows=rows, scale=b.scale, max_q=max(b.new),
                         max_len=max(b.total), total_len=sum(b.total), stream=stream)


def test_a_call_elsewhere_while_the_previous_calls_stream_is_captured(inst):  # noqa: F811
    """It runs, and is no part of the capture; the graph replays."""
    one, two = Batch([3000, 40], [1, 2], 4, 2, 64, 16, BF16), Batch([2000, 70, 9], [1, 1, 1], 8, 2, 128, 32, BF16, seed=1)
    rows = [i32(b.rows) for b in (one, two)]
    here, there = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    attend(inst, one, rows[0], here)
    torch.cuda.synchronize()
    one.check()
    two.out.fill_(9.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=here):
        attend(inst, one, rows[0], here)
        attend(inst, two, rows[1], there)
    torch.cuda.synchronize()
    two.check()
    for _ in range(3):
        one.out.fill_(9.0)
        two.out.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        one.check()
        assert (two.out == 9).all()
        attend(inst, two, rows[1], there)
        attend(inst, two, rows[1], here)
        torch.cuda.synchronize()
        two.check()


def test_a_bit_raised_behind_the_status_call_is_kept(inst):  # noqa: F811
    """The clear has been made when the call returns, also for streams that do not wait for the null stream."""
    vocab, streams = 100, [torch.cuda.Stream() for _ in range(3)]
    logits, chosen, start = torch.zeros(1, vocab, device="cuda"), i32([0]), i32([0, 1])
    bad, good = i32([vocab]), i32([5])
    torch.cuda.synchronize()
    for k in range(60):
        for history, want in ((bad, I.BAD_TOKEN), (bad, I.BAD_TOKEN), (good, 0)):
            I.maaso_logits_adjust(inst, logits=logits, chosen=chosen, history=history, history_start=start, stream=streams[k % 3])
            assert I.maaso_instance_status(inst) == want


def test_the_status_call_puts_the_instance_in_order(inst):  # noqa: F811
    """What calls of few rows of logits keep between their blocks, as calls that ran at once may leave it, is cleared."""
    lib, vocab = I._library(), 50257
    logits = torch.randn(3, vocab, generator=torch.Generator().manual_seed(1)).cuda()
    chosen = torch.empty(3, dtype=torch.int32, device="cuda")
    with I.maaso_instance_create() as spoilt:
        assert C.c_int32.from_address(spoilt.handle + 4).value == torch.cuda.get_device_properties(0).multi_processor_count
        status = C.c_void_p.from_address(spoilt.handle + 8).value  # the rows lie 256 bytes behind it, 128 bytes each
        torch.cuda.synchronize()
        assert lib.hipMemset(C.c_void_p(status + 256), 1, C.c_size_t(1024 * 128)) == 0
        torch.cuda.synchronize()
        assert I.maaso_instance_status(spoilt) == 0
        for _ in range(3):
            chosen.fill_(-7)
            I.maaso_logits_adjust(spoilt, logits=logits, chosen=chosen)
            assert torch.equal(chosen.long(), logits.argmax(1))
