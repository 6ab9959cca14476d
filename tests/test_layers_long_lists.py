"""The embedding's gradient for lists of every length: against sums in 64 bits, whatever the ids, and in a time that grows
as the list does.

Tolerance: n terms of a row in fp32, in any order, are within (n + 2) E times the sum of their magnitudes, E = 2^-24; half
a step of the output's type comes on top."""
import numpy as np
import pytest
import torch

from test_layers_ops import E, close, n64, randn, strided

SORTED_IN_LDS = 16384


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def ids_of(kind, tokens, vocab, seed=0):
    g = np.random.default_rng(seed)
    if kind == "one":                    # a filler id, and a few others
        return np.where(g.random(tokens) < 0.97, vocab // 2, g.integers(0, vocab, tokens))
    if kind == "half":                   # half of them a filler id, the others by rank
        return np.where(g.random(tokens) < 0.5, min(7, vocab - 1), ids_of("rank", tokens, vocab, seed + 1))
    if kind == "rank":                   # falling as one over the id, as ids that a tokenizer has numbered by frequency
        return np.minimum(np.exp(g.random(tokens) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1)
    if kind == "outside":                # few have a row: paddings, ids past the vocabulary, past 32 bits
        some = g.random(tokens)
        return np.where(some < 0.4, -1, np.where(some < 0.8, vocab, np.where(some < 0.9, 2 ** 40 + 1, g.integers(0, vocab, tokens))))
    return g.integers(0, vocab, tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,d,kind", [
    (7169, 300, 8, "one"), (SORTED_IN_LDS, 300, 8, "one"), (SORTED_IN_LDS, 32000, 8, "half"), (SORTED_IN_LDS, 40, 12, "even"),
    (SORTED_IN_LDS, 1, 8, "even"), (SORTED_IN_LDS, 70000, 4, "rank"), (SORTED_IN_LDS + 1, 300, 8, "one"),
    (SORTED_IN_LDS + 1, 1, 8, "even"), (SORTED_IN_LDS + 1, 32000, 9, "rank"), (20479, 256, 8, "even"), (20480, 257, 8, "even"),
    (20481, 65536, 4, "rank"), (40000, 65537, 4, "even"), (70001, 32000, 16, "half"), (100000, 250, 130, "rank"),
    (300000, 70000, 8, "rank"), (1100000, 1000, 4, "rank"), (1100000, 20000000, 1, "even"), (50000, 1000, 8, "outside"),
    (50000, 5, 8, "none")])
def test_long_lists(gl, tokens, vocab, d, kind):
    ids = np.full(tokens, -1) if kind == "none" else ids_of(kind, tokens, vocab)
    dy = strided(randn((tokens, d), 3), 1)
    got = gl.galore_embedding_grad(torch.tensor(ids, device="cuda"), dy, vocab, scale=0.5)
    inside = (ids >= 0) & (ids < vocab)
    rows, where, n = np.unique(ids[inside], return_inverse=True, return_counts=True)
    y = n64(dy)[inside]
    want, mag = np.zeros((len(rows), d)), np.zeros((len(rows), d))
    np.add.at(want, where, 0.5 * y)
    np.add.at(mag, where, 0.5 * np.abs(y))
    at = torch.from_numpy(rows).cuda()
    close(got[at], want, (n[:, None] + 2) * E * mag, torch.float32)
    assert int((got != 0).any(1).sum()) <= len(rows)          # every other row is zero
    if kind != "outside":
        again = gl.galore_embedding_grad(torch.tensor(ids, device="cuda", dtype=torch.int32), dy, vocab, scale=0.5)
        assert torch.equal(got, again)
    G = torch.full((vocab, d), 3.0, device="cuda")
    gl.galore_embedding_grad(torch.tensor(ids, device="cuda"), dy, vocab, scale=0.5, G=G, accumulate=True)
    close(G[at], want + 3.0, (n[:, None] + 3) * E * (mag + 3.0), torch.float32)
    assert int((G != 3.0).any(1).sum()) <= len(rows)


@pytest.mark.gpu
def test_long_lists_in_a_workspace_of_the_stated_size(gl):
    """nothing past the workspace's end is written, narrow rows among them, whose partial sums need less than the sort"""
    for tokens, vocab, d in ((SORTED_IN_LDS, 3000, 1), (SORTED_IN_LDS + 1, 3000, 1), (100000, 100, 2), (30000, 32000, 130)):
        ids, dy = torch.tensor(ids_of("half", tokens, vocab), device="cuda"), randn((tokens, d), 1)
        size = gl.galore_embedding_grad_workspace_size(tokens, vocab, d)
        room = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        got = gl.galore_embedding_grad(ids, dy, vocab, workspace=room[:size])
        assert (room[size:] == 0x5a).all()
        assert torch.equal(got, gl.galore_embedding_grad(ids, dy, vocab))


@pytest.mark.gpu
def test_a_long_list_in_a_graph(gl):
    """every replay on new ids gives what the call gives"""
    tokens, vocab, d = 60000, 5000, 16
    ids, dy, G = torch.zeros(tokens, dtype=torch.int64, device="cuda"), randn((tokens, d), 1), torch.empty((vocab, d), device="cuda")
    ws = torch.empty(gl.galore_embedding_grad_workspace_size(tokens, vocab, d), dtype=torch.uint8, device="cuda")
    gl.galore_embedding_grad(ids, dy, vocab, G=G, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gl.galore_embedding_grad(ids, dy, vocab, G=G, workspace=ws)
    for i, kind in enumerate(("rank", "one", "even", "half", "rank")):
        ids.copy_(torch.from_numpy(ids_of(kind, tokens, vocab, i)))
        dy.copy_(randn(dy.shape, 10 + i))
        graph.replay()
        got = G.clone()
        assert torch.equal(got, gl.galore_embedding_grad(ids, dy, vocab))
        torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rank", "half", "even"])
@pytest.mark.parametrize("vocab", [256, 32000])
def test_time_grows_as_the_list_does(gl, kind, vocab):
    """sixteen times the tokens: at most sixteen times the time, whichever ids there are"""
    def least(tokens, d=64):
        ids = torch.tensor(ids_of(kind, tokens, vocab), device="cuda")
        dy, G = randn((tokens, d), 1, torch.bfloat16), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(gl.galore_embedding_grad_workspace_size(tokens, vocab, d), dtype=torch.uint8, device="cuda")
        times = []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                gl.galore_embedding_grad(ids, dy, vocab, G=G, workspace=ws)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    assert least(1 << 18) <= 16 * least(1 << 14)
