"""An instance's operators together, as a program serves requests with them: a prompt, rows forked from it, single tokens,
a compaction between two steps, against the same decoder computed without a cache in 64 bits.

Every tensor of the cached run that is rounded to bf16 is off by at most half a step, 2^-8 of its value: of a layer the
norm's output, q, k, v, the rotated q and k, the weights, the output, its product, the sum, the second norm's output, the two
products and the sum, 14; the embedding needs none, the last norm and the logits two.  Were they all to add up, the logits
would be off by (14 layers + 2) 2^-8 in the mean."""
import sys
from pathlib import Path

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
import measure_instance as M  # noqa: E402


def reference(m, ids):
    """Logits behind the last of the tokens, in 64 bits."""
    t = len(ids)
    x = m.embedding.double()[ids]
    cos, sin = (a[:, None] for a in m.cos_sin.double()[:t].chunk(2, 1))

    def normed(y):
        return y / ((y * y).mean(-1, keepdim=True) + 1e-6).sqrt()

    def turned(y):
        a, b = y.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    for i in range(m.layers):
        y = (normed(x) @ m.qkv[i].double().T).unflatten(1, (-1, m.dim))
        q, k, v = y.split([m.heads, m.kv_heads, m.kv_heads], 1)
        q, k = turned(normed(q) * m.q_norm[i].double()), turned(normed(k) * m.k_norm[i].double())
        k, v = (z.repeat_interleave(m.heads // m.kv_heads, 1).transpose(0, 1).contiguous() for z in (k, v))
        score = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() * m.dim ** -0.5
        score = score.masked_fill(torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        o = (torch.softmax(score, -1) @ v).transpose(0, 1).reshape(t, -1)
        x = x + o @ m.out[i].double().T
        x = x + torch.relu(normed(x) @ m.up[i].double().T) @ m.down[i].double().T
    return normed(x[-1]) @ m.embedding.double().T


@pytest.mark.parametrize("prompt, page", [(1, 16), (37, 16), (130, 64)])
def test_a_prompt_forks_and_tokens(prompt, page):
    m = M.Decoder(layers=2, heads=4, kv_heads=2, dim=64, vocab=500, max_len=256)
    tol = (14 * m.layers + 2) * 2.0 ** -8
    s = M.Serving(m, rows=5, pages=60, page_size=page, width=-(-160 // page))
    rng = np.random.default_rng(prompt)
    text = [rng.integers(0, 500, prompt).tolist() for _ in range(1)] * 4
    said = [list(t) for t in text]

    def close(logits, row):
        ref = reference(m, torch.tensor(said[row], device="cuda"))
        assert float((logits.double() - ref).norm() / ref.norm()) <= tol

    first = s.buffers([0], prompt)
    close(s.step(torch.tensor(text[0], device="cuda"), first)[0], 0)
    b = s.buffers([1, 2, 4], 1)
    I.maaso_kv_fork(s.inst, s.pages, parents=torch.zeros(3, dtype=torch.int32, device="cuda"), children=b["rows"])
    whole = prompt // page * page
    group = (torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([whole], dtype=torch.int32, device="cuda"), whole) if whole else None
    for turn in range(4):
        new = rng.integers(0, 500, 3)
        for i in range(3):
            said[i + 1].append(int(new[i]))
        logits = s.step(torch.tensor(new, device="cuda"), b, group)
        for i in range(3):
            close(logits[i], i + 1)
        if turn == 1:  # the first row leaves, and the pool is packed
            I.maaso_kv_trim(s.inst, s.pages, rows=torch.zeros(1, dtype=torch.int32, device="cuda"), keep=torch.zeros(1, dtype=torch.int32, device="cuda"))
            moves, live = torch.empty(30, 2, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
            I.maaso_kv_compact(s.inst, s.pages, refs_out=s.pages.refs, table_out=s.pages.table, moves=moves, n_live=live)
            I.maaso_kv_copy(s.inst, s.cache, pairs=moves)
            assert int(s.pages.table.max()) < int(live) == int((s.pages.refs > 0).sum())
    assert I.maaso_instance_status(s.inst) == 0


def test_the_measured_profile():
    m = M.Decoder(layers=1, heads=4, kv_heads=2, dim=64, vocab=500, max_len=256)
    assert all(0 < M.measure(m, level, 100, 4, 16) < 1 for level in (1, 3))


def test_a_step_in_a_graph():
    """Replays of a captured step against the same steps one by one, on a second instance of the same state."""
    m = M.Decoder(layers=2, heads=4, kv_heads=2, dim=64, vocab=500, max_len=256)
    both = []
    for captured in (False, True):
        s = M.Serving(m, rows=3, pages=40, page_size=16, width=10)
        s.step(torch.arange(33, device="cuda"), s.buffers([0], 33))
        b, got = s.buffers([1, 2], 1), []
        I.maaso_kv_fork(s.inst, s.pages, parents=torch.zeros(2, dtype=torch.int32, device="cuda"), children=b["rows"])
        group = (torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.tensor([32], dtype=torch.int32, device="cuda"), 32)
        tokens = torch.tensor([7, 9], dtype=torch.int32, device="cuda")

        def one():
            logits = s.step(tokens, b, group)
            tokens.copy_(b["chosen"])
            return logits

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            one()
        torch.cuda.current_stream().wait_stream(side)
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = one()
        for _ in range(4):
            if captured:
                graph.replay()
            else:
                out = one()
            torch.cuda.synchronize()
            got.append((out.clone(), tokens.clone(), s.pages.length.clone(), s.pages.table.clone()))
            torch.randn(100, 100, device="cuda").sum()
        both.append(got)
        assert I.maaso_instance_status(s.inst) == 0
    for a, b in zip(*both):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
