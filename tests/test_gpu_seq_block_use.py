"""A block of sequence operators in use: parameters laid out again, its steps beside it."""
import pytest
import torch

from paper_1808_05567_amd import seq_block

pytestmark = pytest.mark.gpu


def tokens(M, C, count, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    return [[torch.randn(M, C // 8, 1, 8, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)] for _ in range(count)]


def serve(step, states, pairs):
    """What the tokens give, one after the other, and the states behind them."""
    got = []
    for x, r in pairs:
        got += [t.clone() for t in step(x, r, states)]
    return got + [t.clone() for t in states]


def same(got, want):
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


DIMS = dict(C=136, Ci=200, S=16, W=4)
M = 3


def block_of(params, **more):
    return seq_block.SeqBlock(M, 12, **DIMS, params=params, slots=M, **more)


def params_of(seed):
    return seq_block.init(*(DIMS[k] for k in ("C", "Ci", "S", "W")), seed=seed)


def test_a_step_serves_what_was_laid_out_last():
    """Parameters laid out a second time, and their tensors changed after that: a step built then has those of the second time."""
    new = params_of(2)
    want = block_of(params_of(2))
    block = block_of(params_of(1))
    block.load(new)
    for t in new.values():
        t.zero_()
    pairs = tokens(M, DIMS["C"], 3)
    same(serve(seq_block.SeqBlockStep(block, M), block.states(), pairs), serve(seq_block.SeqBlockStep(want, M), want.states(), pairs))
