"""The serving operators together, as the example of a shared prefix runs them."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import shared_prefix
    return shared_prefix


def _inputs():
    rng = np.random.default_rng(3)
    return rng.integers(0, 1023, 100).tolist(), [rng.integers(0, 1023, n).tolist() for n in (5, 33, 1)]


def test_shared_prefix_equals_requests_alone(ex):
    """The next block's logits of a request under a shared prefix are those of the request by itself, its prefix in
    its own pages: the same attention over the same keys, cut and paged otherwise.  Differences are roundings of
    probabilities and sums that pass two layers: as for the models of two layers elsewhere, relative L2 below 1e-2."""
    prefix, prompts = _inputs()
    together = ex.Batch(prefix, prompts, gen_len=16).block_logits().view(3, ex.BLOCK, ex.VOCAB)
    for b, p in enumerate(prompts):
        alone = ex.Batch([], [prefix + p], gen_len=16, page=64)
        # the prefix before the prompt, so that it sees itself alone
        alone.serve.dllm_serve_reset()
        alone._run([0], [len(prefix)], [prefix])
        alone._run([len(prefix)], [len(p)], [p])
        z = alone.block_logits()
        rel = float((z - together[b]).norm() / together[b].norm())
        assert rel <= 1e-2, rel


def test_blocks_obey_masks_and_repeat_themselves(ex):
    prefix, prompts = _inputs()
    runs = []
    for _ in range(2):
        batch = ex.Batch(prefix, prompts, gen_len=48)
        for _ in range(3):
            tok = batch.decode_block(grammar=range(0, 1022, 3), bias={9: 2.0, 12: -1e4})
            assert (tok % 3 == 0).all() and (tok < 1022).all() and not (tok == 12).any()
        runs.append(batch.tokens)
    assert runs[0] == runs[1] and [len(t) for t in runs[0]] == [5 + 48, 33 + 48, 1 + 48]
    # strong penalties: no id twice in a request's blocks
    batch = ex.Batch(prefix, prompts, gen_len=16)
    tok = batch.decode_block(steps=16, rep=1.0, freq=0.0, pres=1e4)
    assert all(len(set(row)) == len(row) for row in tok.tolist())
