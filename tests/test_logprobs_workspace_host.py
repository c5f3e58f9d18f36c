"""Sizes of the log probabilities' workspace: one made for an engine's largest batch, vocabulary and
number of alternatives serves every smaller call."""
import ctypes

import pytest

from paper_2609_31395_amd import actkv


def size(rows, vocab, top_k):
    n = ctypes.c_size_t()
    assert actkv.load_library().actkv_token_logprobs_workspace(rows, vocab, top_k, ctypes.byref(n)) == 0
    return n.value


ROWS = [*range(0, 140), 170, 171, 255, 256, 257, 510, 511, 512, 513, 1000, 4000, 1 << 20]


@pytest.mark.parametrize("vocab", [1, 4096, 4097, 16384, 16385, 32000, 50257, 151936, 262144])
@pytest.mark.parametrize("top_k", [0, 1, 5, 20, 64])
def test_it_never_falls_as_rows_grow(vocab, top_k):
    sizes = [size(r, vocab, top_k) for r in ROWS]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("rows", [1, 32, 51, 52, 64, 600])
def test_it_never_falls_as_alternatives_or_the_vocabulary_grow(rows):
    for vocab in (5000, 32000, 151936, 262144):
        sizes = [size(rows, vocab, k) for k in range(65)]
        assert sizes == sorted(sizes)
    for k in (0, 4, 20, 64):
        sizes = [size(rows, v, k) for v in range(1, 262145, 1023)]
        assert sizes == sorted(sizes)


def parts(rows, vocab, top_k, chunk):
    """Bytes of a call in chunks of that many logits: three floats a chunk, then top_k keys each."""
    chunks = rows * -(-vocab // chunk)
    return -(-12 * chunks // 256) * 256 + 8 * chunks * top_k


@pytest.mark.parametrize("rows", ROWS[:-1])
def test_it_holds_what_either_kind_of_chunk_needs(rows):
    for vocab in (1, 16385, 50257, 151936, 262144):
        for k in (0, 1, 20, 64):
            assert size(rows, vocab, k) >= parts(rows, vocab, k, 16384)
            if rows * -(-vocab // 16384) < 512 and -(-vocab // 4096) * k <= 1024:
                assert size(rows, vocab, k) >= parts(rows, vocab, k, 4096)
