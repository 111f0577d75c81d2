"""The operators for drafts and continuations together, as the example of draft trees runs them."""
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
    import draft_trees
    return draft_trees


def _alone(ex, tokens, seed=0):
    """Logits behind each token of a sequence, from one causal pass over all of it."""
    c = ex.Causal([tokens], -(-len(tokens) // 16), -(-len(tokens) // 16), len(tokens), seed=seed)
    c.serve.dllm_serve_reset()
    c.serve.dllm_serve_plan(ex.i32([0]), ex.i32([len(tokens)]), len(tokens), causal=True)
    z = c.logits(ex.i32(tokens))
    c.serve.dllm_serve_check()
    return z


def _prompts(ex):
    rng = np.random.default_rng(3)
    half = rng.integers(0, ex.VOCAB, 9).tolist()
    return [rng.integers(0, ex.VOCAB, 5).tolist(), half + half, [7], rng.integers(0, ex.VOCAB, 50).tolist()]


def test_trees_decide_as_the_sequence_alone(ex):
    """Logits of the accepted tokens are those of one causal pass over the whole sequence: the same attention over the
    same keys, those of the path moved together after each step.  Differences are roundings that pass two layers: as for
    the models of two layers elsewhere, relative L2 below 1e-2."""
    prompts = _prompts(ex)
    d = ex.Drafted(prompts, 30, seed=1)
    for _ in range(8):
        gained = d.step()
        assert all(len(g) >= 1 for g in gained)
    assert [t[:len(p)] for t, p in zip(d.tokens, prompts)] == prompts
    alone = [_alone(ex, t, seed=1) for t in d.tokens]
    got = torch.stack([z for _, _, z in d.seen])
    want = torch.stack([alone[b][i] for b, i, _ in d.seen])
    rel = (got - want).norm(dim=1) / want.norm(dim=1)
    assert float(rel.max()) <= 1e-2
    # every token but a request's last was decided on by the row before it
    for b, i, z in d.seen:
        if i + 1 < len(d.tokens[b]):
            assert int(z.argmax()) == d.tokens[b][i + 1]


def test_a_right_draft_is_accepted(ex):
    """A tree that holds the continuation found step by step is walked to its end in one pass."""
    prompts = _prompts(ex)
    slow = ex.Drafted(prompts, 30, seed=2)
    for _ in range(6):
        slow.step()
    fast = ex.Drafted(prompts, 30, seed=2)
    chains = [t[len(p):][:6] for t, p in zip(slow.tokens, prompts)]

    def guess(b):  # the chain, between tokens that are none of it
        ids, parent, node = [chains[b][0]], [-1], 0
        for t in chains[b][1:]:
            ids += [(t + 1) % ex.VOCAB, t]
            parent += [node, node]
            node = len(ids) - 1
        while len(ids) < ex.TREE:
            ids.append((chains[b][1] + 1) % ex.VOCAB)
            parent.append(0)
        return parent, ids

    fast.guess = guess
    gained = fast.step()
    # (nearly equal logits may be decided on otherwise, so that a request may stop early)
    assert sum(g == c for g, c in zip(gained, chains)) >= 3 and all(g == c[:len(g)] for g, c in zip(gained, chains))


def test_beams_share_pages_and_score_what_they_say(ex):
    rng = np.random.default_rng(4)
    prompt = rng.integers(0, ex.VOCAB, 45).tolist()
    b = ex.Beams(prompt, 4, 20, seed=3)
    for _ in range(19):
        b.step()
        rows = b.serve.table.cpu()[:, :b.serve.held.max().item()]
        assert bool((rows[:, :2] == rows[:1, :2]).all())  # the prompt's full pages
    assert bool((b.score[:-1] >= b.score[1:]).all()) and len(set(map(tuple, b.tokens.tolist()))) == 4
    for score, t in zip(b.score.tolist(), b.tokens.tolist()):
        z = torch.log_softmax(_alone(ex, prompt + t, seed=3).double(), 1)
        want = sum(float(z[44 + i, v]) for i, v in enumerate(t))
        # logits 1e-2 off relative to their size (about 1.5 rms): 0.015 a log probability, rms, 20 of them
        assert abs(score - want) <= 20 * 0.03
    # all but the pages of the four beams are free, and no page is held and free
    s = b.serve
    held = {p for row, n in zip(s.table.tolist(), s.held.tolist()) for p in row[:n]}
    head, free = s.ring_pos.tolist()
    ring = {s.ring.tolist()[(head + i) % s.cfg.n_pages] for i in range(free)}
    assert len(ring) == free and not held & ring and len(held) + free == s.cfg.n_pages
