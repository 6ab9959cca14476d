"""The loops of the head norms and of the recurrence past their first trip, against the 64-bit forms, with the tolerances
of test_layers_ops.py: waves that take several tokens and several passes of heads, chains of more than sixteen chunks with
sequences that begin and end around their bounds, workgroups that take all chunks of their channels."""
import numpy as np
import pytest
import torch

import layers_oracle as lo
import test_layers_ops as ops
from test_layers_ops import DTYPES, E, close, gate_logits, n64, randn


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


# forward 16384 waves at most, backward 1536, of 64 / lanes heads each: tokens and heads past both
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,hq,hk,d,rot,inter,how", [
    (16500, 17, 3, 64, 64, False, "product"), (16500, 17, 1, 64, 32, True, "heads"), (16400, 9, 2, 75, 74, False, "odd"),
    (700, 70, 9, 128, 128, False, "heads"), (700, 9, 70, 80, 20, True, "product")])
def test_head_norm_takes_tokens_and_heads_in_turn(gl, dtype, tokens, hq, hk, d, rot, inter, how):
    ops.test_head_norm(gl, dtype, tokens, hq, hk, d, rot, inter, how)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,hq,hk,d,rot,inter,how", [
    (8200, 17, 3, 64, 64, False, "product"), (8200, 17, 2, 64, 64, False, "packed"), (8200, 3, 17, 48, 32, True, "heads"),
    (1700, 9, 9, 75, 74, False, "odd"), (700, 70, 9, 128, 128, False, "heads"), (700, 70, 9, 128, 128, True, "packed"),
    (500, 40, 9, 96, 24, False, "packed")])
def test_head_norm_backward_takes_tokens_and_heads_in_turn(gl, dtype, tokens, hq, hk, d, rot, inter, how):
    ops.test_head_norm_backward(gl, dtype, tokens, hq, hk, d, rot, inter, how)


# a chunk has 128 tokens (fp32 backward 64), a group 16 chunks: bounds on, before and behind both
BOUNDS = [(5000, 6, [0, 1, 127, 128, 129, 255, 257, 1023, 1024, 1025, 2047, 2048, 2049, 2049, 4095, 4097, 4097, 4900]),
          (5000, 70, [3, 4400, 4400, 4990]), (4300, 5, [0, 2048, 4096, 4300]), (4161, 9, [0, 4161]),
          (4500, 4, [2100, 2101, 2101, 4230]), (9000, 3, [0, 40, 8999, 9000])]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,d,bounds", BOUNDS)
@pytest.mark.parametrize("start", [False, True])
def test_packed_sequences_over_groups_of_chunks(gl, dtype, tokens, d, bounds, start):
    ops.test_packed_recurrence(gl, dtype, 1, tokens, d, bounds, start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,d,bounds", BOUNDS + [(700, 24700, [0, 100, 130, 130, 690])])
def test_states_of_packed_sequences(gl, dtype, tokens, d, bounds):
    """before every 64 tokens: the state after the token before them, zeros where that one is of no sequence"""
    x, f, h0 = randn((tokens, d), 1, dtype), gate_logits((tokens, d), 2, dtype), randn((len(bounds) - 1, d), 3)
    states = gl.galore_recurrence(x, f, h0=h0, offsets=torch.tensor(bounds, device="cuda"), states=True)[2]
    h, _, _, age = lo.recurrence(n64(x), n64(f), n64(h0), bounds)
    first = np.zeros((1, d))
    close(states, np.concatenate((first, h[63:tokens - 1:64])), 10 * E * np.concatenate((first, age[63:tokens - 1:64])), torch.float32)


# from 385 tiles of 64 channels on (bf16 backward 257) a workgroup takes all chunks of its tile
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("start", [False, True])
def test_wide_packed_sequences(gl, dtype, start):
    ops.test_packed_recurrence(gl, dtype, 1, 300, 24700, [0, 1, 63, 128, 128, 129, 200, 290], start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("start", [False, True])
def test_many_matrices(gl, dtype, start):
    ops.test_recurrence(gl, dtype, 390, 140, 24, start)
    ops.test_recurrence_backward(gl, dtype, 390, 140, 24, start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("start", [False, True])
def test_long_sequences(gl, dtype, start):
    """dense, over several groups of chunks"""
    ops.test_recurrence(gl, dtype, 2, 4500, 5, start)
    ops.test_recurrence_backward(gl, dtype, 2, 4500, 5, start)
