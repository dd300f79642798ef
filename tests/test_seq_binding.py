"""What the binding of the sequence operators refuses before a call reaches the library: tensors that stand for ones on the GPU, and a library that
only notes its calls."""
import pytest
import torch

from paper_1808_05567_amd import seq


class OnGpu(torch.Tensor):
    """A tensor in host memory that says it is on the GPU."""
    is_cuda = True


def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's functions as they are called; none runs."""
    done, real = [], seq.load()

    class Noted:
        def __getattr__(self, name):
            if name.endswith("_create") or name in ("seq_query", "seq_destroy"):
                return getattr(real, name)
            return lambda *args: done.append(name) or 0
    monkeypatch.setattr(seq, "load", Noted)
    return done


N, C, L, W = 2, 16, 4, 4  # (two blocks of bf16)


def conv_fwd(views, x, y):
    h = seq.seq_conv_create(N, C, L, W, seq.SEQ_BF16, views=views)
    seq.seq_conv_fwd(h, x, tensor(W, C, dtype=torch.float32), None, y, stream=0)


def test_tensors_of_fewer_places_are_refused(calls):
    """Half of the blocks of a wider tensor: others of the same strides and as many elements, with fewer sequences, blocks or positions."""
    half, dense = tensor(N, 4, L, 8)[:, :2], tensor(N, 2, L, 8)
    fewer = [tensor(1, 4, L, 8), tensor(4, 4, L, 8)[:, :1], tensor(3, 4, L, 8)[:, :2, :3], tensor(N, 4, L, 8)[:, :2, :, :4]]
    assert all(t.stride() == half.stride() for t in fewer) and all(t.numel() >= N * C * L for t in fewer[:3])
    for bad in fewer:
        with pytest.raises(ValueError):
            conv_fwd({"x": half}, bad, dense)
        with pytest.raises(ValueError):
            conv_fwd({"y": half}, dense, bad)
    assert not calls
    conv_fwd({"x": half, "y": half}, half, tensor(3, 4, L, 8)[:, 1:])  # (more of them do)
    with pytest.raises(ValueError):
        conv_fwd(None, tensor(N, L, 2, 8), dense)  # (as many elements in another order)
    # dense ones may have their places in any dimensions
    for good in (dense, dense.flatten(), tensor(1, 4, L, 8), tensor(N + 1, 2, L, 8), tensor(N, 2, L, 1, 8)):
        conv_fwd(None, good, dense)
    assert calls == ["seq_conv_fwd"] * 6


def test_places_of_states_and_of_eight_bits_are_counted_too(calls):
    S, f = 16, torch.float32
    part = tensor(N, 6, L, 8)[:, :2]
    h = seq.seq_scan_create(N, C, L, S, seq.SEQ_BF16, views={"B": part})
    x, A, ws = tensor(N, 2, L, 8), tensor(S, C, dtype=f), tensor(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError):
        seq.seq_scan_fwd(h, x, x, A, tensor(1, 6, L, 8), x, x, ws, stream=0)
    seq.seq_scan_fwd(h, x, x, A, part, x, x, ws, stream=0)
    n = seq.seq_norm_create(N, 32, L, seq.SEQ_BF16, views={"q": tensor(N, 5, L, 16, dtype=torch.int8)[:, :2]})
    x, w, scale = tensor(N, 4, L, 8), tensor(32, dtype=f), tensor(N, L, dtype=f)
    with pytest.raises(ValueError):
        seq.seq_norm_fwd_q8(n, x, None, w, None, tensor(1, 5, L, 16, dtype=torch.int8), scale, stream=0)
    seq.seq_norm_fwd_q8(n, x, None, w, None, tensor(N, 5, L, 16, dtype=torch.int8)[:, 3:], scale, stream=0)
    assert calls == ["seq_scan_fwd", "seq_norm_fwd_q8"]


def test_single_places_have_any_stride(calls):
    one = seq.seq_conv_create(1, 8, 1, W, seq.SEQ_BF16, slots=1)
    x, w, state = tensor(64).as_strided((1, 1, 1, 8), (40, 16, 24, 1)), tensor(W, 8, dtype=torch.float32), tensor(1, 1, W - 1, 8)
    seq.seq_conv_step(one, x, w, None, state, x, stream=0)
    assert calls == ["seq_conv_step"]


def test_views_give_a_stride_for_every_place(calls):
    """A view with one sequence, block or position says nothing of where the second lies."""
    wide = tensor(N, 4, L, 8)
    for view in (wide[:1, :2], wide[:, :1], wide[:, :2, :1]):
        with pytest.raises(ValueError):
            seq.seq_conv_create(N, C, L, W, seq.SEQ_BF16, views={"x": view})
    with pytest.raises(ValueError):
        seq.seq_scan_create(N, C, L, 16, seq.SEQ_BF16, views={"B": wide[:, :1]})
    with pytest.raises(ValueError):
        seq.seq_norm_create(N, 32, L, seq.SEQ_BF16, views={"q": tensor(N, 1, L, 16, dtype=torch.int8)})
    # where the plan has one too, and for tensors of the same strides that have fewer, it may be any
    seq.seq_conv_create(N, 8, 1, W, seq.SEQ_BF16, views={"x": wide[:, :1, :1]})
    conv_fwd({"x": tensor(N + 2, 4, L, 8)[:2, :2, :3]}, wide[:, :2], wide.flatten())
    assert calls == ["seq_conv_fwd"]


def test_views_of_one_block_for_all_places_are_refused(calls):
    """Three distances of zero stand for a dense tensor, which a block that is expanded over all places is not."""
    with pytest.raises(ValueError):
        seq.seq_conv_create(N, C, L, W, seq.SEQ_BF16, views={"x": tensor(1, 1, 1, 8).expand(N, 2, L, 8)})
    # over some of the dimensions it may be, and over all if there is one sequence (whose distance is not zero then)
    for same in (tensor(N, 1, 1, 8).expand(N, 2, L, 8), tensor(1, 2, L, 8).expand(N, 2, L, 8)):
        conv_fwd({"x": same}, same, tensor(N, 2, L, 8))
    seq.seq_conv_create(1, C, L, W, seq.SEQ_BF16, views={"x": tensor(1, 1, 1, 8).expand(1, 2, L, 8)})
    assert calls == ["seq_conv_fwd"] * 2


def test_workspaces_are_dense_and_on_the_gpu(calls):
    h = seq.seq_conv_create(N, C, L, W, seq.SEQ_BF16)
    x, w, size = tensor(N, 2, L, 8), tensor(W, C, dtype=torch.float32), h.info.workspace_bytes
    for bad in (torch.zeros(size, dtype=torch.uint8), tensor(2 * size, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            seq.seq_conv_bwd(h, x, w, None, x, x, w, None, bad, stream=0)
    assert not calls
    seq.seq_conv_bwd(h, x, w, None, x, x, w, None, tensor(size // 4, dtype=torch.float32), stream=0)
    assert calls == ["seq_conv_bwd"]


def test_plans_are_refused_for_launches_that_they_make():
    """States are joined in one launch where there are several runs, by a wave for 16 of them: single positions and short sequences of many states do not need
    as many work-items as the longest."""
    from paper_1808_05567_amd import conv
    b16 = seq.SEQ_BF16
    for n, c, l, s in ((512, 8192, 1, 64), (1024, 8192, 1, 32), (256, 1 << 14, 65, 64), (1 << 12, 1 << 14, 16, 64)):
        seq.seq_scan_create(n, c, l, s, b16, slots=n)
    for n, c, l, s in ((1 << 12, 1 << 14, 65, 64), (1 << 20, 1 << 13, 1, 4), (1 << 19, 1 << 10, 65, 8)):
        with pytest.raises(conv.ConvError) as e:
            seq.seq_scan_create(n, c, l, s, b16)
        assert e.value.status == conv.CONV_EUNSUPPORTED


def test_distances_that_64_bits_do_not_hold_are_refused():
    """Positions 2^40 elements apart: 2^24 of them come back to the first one's place, modulo 2^64."""
    import ctypes
    from paper_1808_05567_amd import conv
    far = 1 << 40
    for name in ("x", "y"):
        for n, l, strides, ok in ((2, (1 << 24) + 1, (far, 8, far), False), (1, (1 << 24) + 1, (8, 8, far), False), (1, 1 << 17, (8, 8, far), True)):
            d = seq.SeqConvDesc(N=n, C=8, L=l, W=W, dtype=seq.SEQ_BF16)
            setattr(d, name, seq.SeqView(*strides))
            h = ctypes.c_void_p()
            status = seq.load().seq_conv_create(ctypes.byref(d), ctypes.byref(h))
            assert (status == conv.CONV_OK) == ok and (ok or status == conv.CONV_EINVAL), (name, n, l)
            if ok:
                seq.load().seq_destroy(h)
