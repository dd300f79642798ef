"""A block of sequence operators in use: parameters laid out again, its steps beside it, sequences that end early."""
import numpy as np
import pytest
import torch

from paper_1808_05567_amd import seq, seq_block
from seq_util import Seq, spoil
from test_gpu_seq_block import reference, reference_bwd

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


@pytest.mark.parametrize("dtype", [seq.SEQ_F32, seq.SEQ_BF16])
def test_parameters_stay_in_their_memory(dtype):
    """A recorded forward pass runs with the parameters that were laid out since."""
    N, L, C, Ci, S, W = 2, 20, 40, 56, 8, 4
    make = lambda seed: seq_block.SeqBlock(N, L, C, Ci, S, W, seq_block.init(C, Ci, S, W, seed=seed), dtype)  # noqa: E731
    block, other = make(1), make(2)
    x, res = (torch.randn(N, C // block.v, L, block.v, device="cuda").to(block.u.dtype) for _ in range(2))
    tensors = lambda b: [b.nw, b.taps, b.bias, b.A, b.D, b.dt_bias] + [p.wt for p in (b.w_in, b.w_mid, b.w_mid_t, b.w_out)]  # noqa: E731
    at = [t.data_ptr() for t in tensors(block)]
    block.forward(x, res)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, r = block.forward(x, res)
    block.load(seq_block.init(C, Ci, S, W, seed=2))
    assert at == [t.data_ptr() for t in tensors(block)]
    want = other.forward(x, res)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        same((out, r), want)


def test_parameters_that_do_not_fit_are_refused():
    """... before any of them is laid out."""
    block = block_of(params_of(1))
    pairs = tokens(M, DIMS["C"], 1)
    want = serve(seq_block.SeqBlockStep(block, M), block.states(), pairs)
    for name, bad in (("w_in", torch.zeros(1, 1)), ("taps", torch.zeros(DIMS["Ci"], DIMS["W"])), ("w_out", None)):
        p = params_of(2)
        if bad is None:
            del p[name]
        else:
            p[name] = bad.cuda()
        with pytest.raises((KeyError, ValueError)):
            block.load(p)
    same(serve(seq_block.SeqBlockStep(block, M), block.states(), pairs), want)


def test_steps_follow_the_block():
    """Parameters laid out again: a step that was there serves them too, called or recorded."""
    want = block_of(params_of(2))
    block = block_of(params_of(1))
    step = seq_block.SeqBlockStep(block, M)
    pairs = tokens(M, DIMS["C"], 3)
    serve(step, block.states(), pairs)
    x, r, states = *(torch.empty_like(t) for t in pairs[0]), block.states()
    x.copy_(pairs[0][0])
    r.copy_(pairs[0][1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, after = step(x, r, states)
    block.load(params_of(2))
    expected = serve(seq_block.SeqBlockStep(want, M), want.states(), pairs)
    same(serve(step, block.states(), pairs), expected)
    for t in states:
        t.zero_()
    got = []
    for token in pairs:
        x.copy_(token[0])
        r.copy_(token[1])
        graph.replay()
        torch.cuda.synchronize()
        got += [out.clone(), after.clone()]
    same(got + list(states), expected)


def test_steps_have_the_blocks_eps():
    """The residual stream is small beside eps: 1e-1 and 1e-5 are far apart."""
    params, eps = params_of(1), 1e-1
    block = block_of(params, eps=eps)
    pairs = [[0.1 * t for t in p] for p in tokens(M, DIMS["C"], 2)]
    got = serve(seq_block.SeqBlockStep(block, M), block.states(), pairs)
    same(got, serve(seq_block.SeqBlockStep(block, M, eps=eps), block.states(), pairs))
    other = serve(seq_block.SeqBlockStep(block, M, eps=1e-5), block.states(), pairs)
    assert (other[0].float() - got[0].float()).norm() > 0.1 * got[0].float().norm()


@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_a_training_step_of_sequences_that_end_early(eps, monkeypatch):
    """In fp32, with NaN and infinities behind each end, against the sequences one by one; the bound is that of the whole step (seven operators, each good to
    some 1e-6 of its magnitudes)."""
    N, L, C, Ci, S, W, dtype = 5, 37, 24, 40, 16, 4, seq.SEQ_F32
    ends = [L, 0, 1, 20, L + 3]
    rng = np.random.default_rng(7)
    params = seq_block.init(C, Ci, S, W, seed=1)
    p = {k: t.double().cpu().numpy() for k, t in params.items()}
    x, res, dout, dr = (np.float64(np.float32(rng.standard_normal((N, L, C)))) for _ in range(4))
    block = seq_block.SeqBlock(N, L, C, Ci, S, W, params, dtype, eps=eps)
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    X, RES, DOUT, DR = (Seq(N, C, L, dtype, "dense", spoil(a, ends)).t.contiguous() for a in (x, res, dout, dr))
    before = [t.clone() for t in (X, RES, DOUT, DR)]
    out, r = block.forward(X, RES, lengths=lengths)
    back = lambda t, n: t.permute(0, 2, 1, 3).reshape(N, L, -1)[..., :n].double().cpu().numpy()  # noqa: E731
    out, r = back(out, C), back(r, C)
    dx, g = block.backward(DOUT, DR, lengths=lengths)
    dx = back(dx, C)
    monkeypatch.setattr("test_gpu_seq_block.EPS", eps)
    want, wx, wg = np.zeros_like(out), np.zeros_like(dx), None
    for n, end in enumerate(ends):
        end = min(end, L)
        if end == 0:
            continue
        part = [a[n:n + 1, :end] for a in (x, res, dout, dr)]
        want[n, :end] = reference(p, part[0], part[1], S)[-1]
        wx[n, :end], one = reference_bwd(p, *part, S)
        wg = one if wg is None else {k: wg[k] + one[k] for k in wg}
        assert not out[n, end:].any() and not r[n, end:].any() and not dx[n, end:].any()
    for got, ref, name in [(out, want, "out"), (dx, wx, "dx")] + [(g[k].double().cpu().numpy(), wg[k], k) for k in wg]:
        assert np.linalg.norm(got - ref) <= 1e-4 * np.linalg.norm(ref), name
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip((X, RES, DOUT, DR), before))
    again, g2 = block.backward(DOUT.flatten(), DR.flatten(), lengths=lengths)  # (dense, without dimensions)
    np.testing.assert_array_equal(back(again, C), dx)
    assert all(torch.equal(g[k], g2[k]) for k in g)


def test_gradients_of_another_form_are_refused():
    """What backward is given is as its outputs are: type, extents, strides."""
    block = block_of(params_of(1))
    good = torch.zeros_like(block.out)
    block.forward(good, good)
    turned = good.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    for bad in (good.float(), good[:1].clone(), turned, good.cpu()):
        for args in ((bad, good), (good, bad)):
            with pytest.raises(ValueError):
                block.backward(*args)
    block.backward(good, None)
