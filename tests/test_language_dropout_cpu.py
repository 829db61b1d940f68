"""``Dropout``'s numbers without a device (the stand-ins of ``test_language_calls_cpu.py``)."""
import copy
import pickle

import pytest
import torch

from test_language_calls_cpu import _On0, calls  # noqa: F401

import paper_2606_13894_amd as gf


def _host(drop):
    """The module with its state where the stand-ins say that device 0 is."""
    for m in drop.modules():
        if isinstance(m, gf.Dropout):
            m.state = m.state.as_subclass(_On0)
    return drop


def _pass(drop):
    """(seed, offset) that a training pass takes."""
    before = drop.state.tolist()
    drop(torch.zeros(4, dtype=torch.bfloat16).as_subclass(_On0))
    after = drop.state.tolist()
    assert after[1] == before[1] + 1
    return after[0], before[1]


def test_modules_without_a_seed_differ(calls):  # noqa: F811
    """Each draws a seed of its own at its first training pass, and keeps it."""
    layer = gf.FeedForward(8, 8, dropout=0.1)
    first = [_host(gf.Dropout(0.1)) for _ in range(4)]
    first += [_host(copy.deepcopy(layer)).drop for _ in range(3)]    # layers copied before they ran
    assert all(d.state.tolist() == [0, 0] for d in first)
    torch.manual_seed(5)
    seeds = [_pass(d)[0] for d in first]
    assert len(set(seeds)) == len(seeds) and all(0 < s < 2 ** 63 for s in seeds)
    assert [_pass(d) for d in first] == [(s, 1) for s in seeds]
    torch.manual_seed(5)
    assert [_pass(_host(gf.Dropout(0.1)))[0] for _ in first] == seeds


@pytest.mark.parametrize("seed", [0, 7, -5])
def test_a_given_seed_stays(calls, seed):  # noqa: F811
    for drop in (gf.Dropout(0.1, seed=seed), gf.FeedForward(8, 8, dropout=0.1, seed=seed).drop):
        before = torch.get_rng_state()
        assert _pass(_host(drop)) == (seed, 0) and _pass(drop) == (seed, 1)
        assert torch.equal(torch.get_rng_state(), before)


def test_loaded_states_stay(calls):  # noqa: F811
    """A state that has run resumes in a module with a seed or without, also where that one has run; a
    new state draws again where no seed was given."""
    saved = _host(gf.Dropout(0.1, seed=9))
    _pass(saved)
    own = _host(gf.Dropout(0.1))
    own_seed, _ = _pass(own)
    for other in (_host(gf.Dropout(0.1)), _host(gf.Dropout(0.1, seed=3)), own):
        other.load_state_dict({k: v.clone() for k, v in saved.state_dict().items()})
        assert _pass(other) == (9, 1)
    new = gf.Dropout(0.1).state_dict()
    own.load_state_dict(new)
    seed, at = _pass(own)
    assert seed not in (0, 9, own_seed) and at == 0
    given = _host(gf.Dropout(0.1, seed=4))
    given.load_state_dict(new)
    assert _pass(given) == (0, 0)


def test_evaluation_draws_nothing():
    x = torch.randn(4)
    before = torch.get_rng_state()
    for drop in (gf.Dropout(0.0), gf.Dropout(0.3).eval()):
        assert drop(x) is x
    assert torch.equal(torch.get_rng_state(), before)


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_passes_are_errors(calls, reentrant):  # noqa: F811
    """A second forward pass in the backward pass would drop other elements."""
    from torch.utils.checkpoint import checkpoint
    drop = _host(gf.Dropout(0.1, seed=3))
    x = torch.ones(4, dtype=torch.bfloat16).as_subclass(_On0).requires_grad_()

    def block(v):
        v = drop(v)
        return v * v

    y = checkpoint(block, x, use_reentrant=reentrant, preserve_rng_state=False)
    assert drop.state.tolist() == [3, 1]
    with pytest.raises(RuntimeError, match="run again within a backward pass"):
        y.sum().backward()
    assert drop.state.tolist() == [3, 1]
    drop.eval()
    checkpoint(block, x, use_reentrant=reentrant, preserve_rng_state=False).sum().backward()
    assert torch.equal(x.grad, torch.full_like(x, 2.0))


def test_blocks_pickled_without_dropout():
    """Whole blocks that were saved before they had dropout load and run; others keep theirs."""
    block = gf.FeedForward(8, 8)
    del block.drop
    assert pickle.loads(pickle.dumps(block)).drop is None
    assert pickle.loads(pickle.dumps(gf.FeedForward(8, 8))).drop is None
    assert copy.deepcopy(block).drop is None
    dropping = pickle.loads(pickle.dumps(gf.FeedForward(8, 8, dropout=0.2, seed=4)))
    assert dropping.drop.p == 0.2 and dropping.drop.state.tolist() == [4, 0]
