"""From how many rows on the vocabulary calls are refused, form by form: where the launch would count 2^32 work items (no GPU)."""
import pytest

from paper_1805_10387_amd import _lib as ML
from test_more_operator_refusals import lib, lp


@pytest.mark.parametrize("vocab,lanes", [(3, 64), (512, 64), (1024, 64), (2048, 64), (4096, 128), (8192, 256), (16384, 256), (32768, 256), (65536, 512)])
@pytest.mark.parametrize("top", [0, 3])
def test_token_logprobs(vocab, lanes, top):
    kw = dict(rows=2 ** 32 // lanes, vocab=vocab, top=top, ld=vocab, ids=256 if top else None, tops=256 if top else None)
    assert lp(**kw) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


@pytest.mark.parametrize("vocab,chunks,lanes", [(131072, 2, 512), (65537, 2, 512), (1 << 20, 16, 512)])
def test_token_logprobs_in_chunks(vocab, chunks, lanes):
    assert lp(rows=2 ** 32 // lanes // chunks, vocab=vocab, ld=vocab, n=(1 << 64) - 1) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()
