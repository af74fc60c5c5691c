"""Counts that 32 bits do not hold are refused by the binding, or mean all there is: never their low bits (no GPU;
tensors without memory)."""
import types

import pytest
import torch

import paper_2609_30884_amd as crf

BIG = 1 << 32


def _none(*shape, dtype=torch.int32):
    return torch.empty(*shape, dtype=dtype, device="meta")


def _ctx(got):
    lib = types.SimpleNamespace(crf_token_logprobs=lambda *a: got.append(a) or 0)
    return types.SimpleNamespace(dims=crf.make_dims(2, 128, 4, 2, 64, 64), lib=lib, handle=None, device=-1)


@pytest.mark.parametrize("rows,vocab,tokens,top", [(BIG + 2, 50, 1, 3), (2, BIG + 50, 1, 3), (2, 50, BIG + 1, 3),
                                                   (2, 50, 1, BIG + 3), (1 << 31, 50, 1, 3)])
def test_token_logprobs_refuses_counts_past_32_bits(rows, vocab, tokens, top):
    got, f32 = [], torch.float32
    with pytest.raises(crf.CrfError) as e:
        crf.token_logprobs(_ctx(got), _none(rows, vocab, dtype=f32), _none(rows, tokens), _none(rows, tokens, dtype=f32),
                           top_token=_none(rows, top), top_logprob=_none(rows, top, dtype=f32), stream=1)
    assert e.value.status == 2 and not got


def test_token_logprobs_takes_counts_of_31_bits():
    got = []
    most = (1 << 31) - 1
    crf.token_logprobs(_ctx(got), _none(most, 50, dtype=torch.float32), lse=_none(most, dtype=torch.float32), stream=1)
    assert got[0][4:6] == (most, 50)


@pytest.mark.parametrize("seqs,pages,rows", [(BIG + 3, 2, 6), (3, BIG + 2, 6), (3, 2, BIG + 6), (3, 2, 6 - BIG)])
def test_batches_of_counts_past_32_bits_are_refused(seqs, pages, rows):
    with pytest.raises(crf.CrfError) as e:
        crf.seq_batch(_none(seqs + 1), _none(seqs), _none(seqs, pages), rows)
    assert e.value.status == 2


def test_groups_past_32_bits_are_refused():
    with pytest.raises(crf.CrfError) as e:
        crf.seq_groups(_none(BIG + 3), _none(BIG + 2))
    assert e.value.status == 2


@pytest.mark.parametrize("given,taken", [(0, 0), (7, 7), (1 << 31, (1 << 31) - 1), (BIG + 1, (1 << 31) - 1), (-1, -1)])
def test_bounds_of_new_tokens_past_32_bits(given, taken):
    """max_new is a bound: one that 32 bits do not hold bounds nothing."""
    assert crf.seq_batch(_none(4), _none(3), _none(3, 2), 6, given).max_new == taken
