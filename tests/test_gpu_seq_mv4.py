"""Products with 4-bit weights against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import close, nans
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = (seq.SEQ_F32, seq.SEQ_BF16, seq.SEQ_I8)
CASES = [  # M, C, K, group
    (1, 128, 16, 128), (1, 4, 1, 32), (2, 200, 40, 128), (3, 100, 17, 32), (16, 1000, 72, 64), (17, 260, 33, 64), (33, 384, 130, 128),
    (5, 33, 100, 32), (70, 2100, 20, 32), (1, 4096, 300, 128), (2, 300, 8200, 64), (20, 160, 4130, 32), (40, 1200, 4100, 128),
    (48, 1300, 4100, 32), (64, 200, 4128, 64), (70, 170, 4110, 128), (130, 96, 4097, 64), (6, 2200, 8196, 32), (12, 520, 64, 64),
]


def pack(q, K, C):
    """The header's layout, one weight at a time."""
    Kp, Cs = -(-K // 16) * 16, -(-C // 128)
    words = np.zeros((Cs, Kp, 4, 4), dtype=np.uint32)
    for c in range(C):
        words[c // 128, :K, c % 32 // 8, c % 128 // 32] |= (q[:, c].astype(np.int64) & 15).astype(np.uint32) << np.uint32(4 * (c % 8))
    return torch.from_numpy(words.view(np.uint8).reshape(-1)).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,K,group", CASES)
def test_products(M, C, K, group, dtype):
    rng = np.random.default_rng(M + C + K)
    q = rng.integers(-8, 8, (K, C))
    scale = rng.uniform(0.5, 2, (-(-C // group), K)).astype(np.float32)
    bias = rng.standard_normal(K).astype(np.float32) if M % 2 else None
    xscale = None
    if dtype == seq.SEQ_I8:
        x, v, tt = rng.integers(-127, 128, (M, C)).astype(np.float64), 16, torch.int8
        xscale = rng.uniform(0.5, 2, M).astype(np.float32)
    else:
        v, tt = (4, torch.float32) if dtype == seq.SEQ_F32 else (8, torch.bfloat16)
        x = torch.from_numpy(rng.standard_normal((M, C)).astype(np.float32)).to(tt).double().numpy()
    h = seq.seq_mv4_create(M, C, K, group, dtype)
    X = torch.zeros(M, h.info.Cp, dtype=tt, device="cuda")
    X[:, :C] = torch.from_numpy(x).cuda()
    Kp = -(-K // 16) * 16
    sc = nans(scale.shape[0], Kp)  # (scales beyond K are not used)
    sc[:, :K] = torch.from_numpy(scale).cuda()
    vy = 4 if dtype == seq.SEQ_F32 else 8
    Ky = -(-K // vy) * vy
    out = torch.full((M + 2, Ky), float("nan"), dtype=torch.float32 if dtype == seq.SEQ_F32 else torch.bfloat16, device="cuda")
    Y = out[1:M + 1]
    b = None if bias is None else torch.from_numpy(bias).cuda()
    xs = None if xscale is None else torch.from_numpy(xscale).cuda()
    wt = pack(q, K, C)
    assert wt.numel() == h.info.wt_bytes and sc.numel() * 4 == h.info.scale_bytes
    seq.seq_mv4(h, X, wt, sc, Y, xscale=xs, bias=b)
    assert torch.isnan(out[0]).all() and torch.isnan(out[M + 1]).all()
    got = Y.double().cpu().numpy()
    assert not got[:, K:].any()
    args = (x, q.astype(np.float64), scale.astype(np.float64), group, xscale, bias)
    # sums inside a group (32 products a rounding at least), over the groups, scale, scale of the row, bias
    close(got[:, :K], oracle.mv4(*args), (C / 8 + 16) * U * oracle.mv4(*args, mag=True), dtype != seq.SEQ_F32)
    w = nans(K, C)
    seq.seq_mv4_unquant(h, wt, sc, w)
    want = torch.from_numpy((q * np.repeat(scale, group, 0)[:C].T).astype(np.float32))
    assert torch.equal(w.cpu(), want)


def test_whole_numbers_are_exact():
    """8-bit activations, scales of one: every sum is a whole number below 2^24 and comes out exactly (rounded once to bf16)."""
    M, C, K = 4, 1024, 64
    rng = np.random.default_rng(1)
    q, x = rng.integers(-8, 8, (K, C)), rng.integers(-127, 128, (M, C))
    h = seq.seq_mv4_create(M, C, K, 64, seq.SEQ_I8)
    Y = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    one = torch.ones
    seq.seq_mv4(h, torch.from_numpy(x.astype(np.int8)).cuda(), pack(q, K, C), one(16, K, device="cuda"), Y, xscale=one(M, device="cuda"))
    assert torch.equal(Y.cpu(), torch.from_numpy((x @ q.T).astype(np.float32)).to(torch.bfloat16))


def test_rows_do_not_touch_each_other():
    """NaN in one row of activations stays there."""
    M, C, K = 18, 256, 32
    h = seq.seq_mv4_create(M, C, K, 64, seq.SEQ_BF16)
    x = torch.randn(M, C, device="cuda").to(torch.bfloat16)
    x[3, 5] = float("nan")
    q = np.random.default_rng(2).integers(-8, 8, (K, C))
    Y = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    seq.seq_mv4(h, x, pack(q, K, C), torch.ones(4, K, device="cuda"), Y)
    bad = torch.isnan(Y).any(1).cpu()
    assert bad[3] and bad.sum() == 1


def test_infinite_and_tiny_activations():
    """fp32 activations beyond what three bf16 numbers hold: infinities stay infinities, what is tiny is lost at 2^-133 at most."""
    C, K = 128, 16
    x = torch.zeros(3, C, device="cuda")
    x[0, 5], x[1, 7], x[2, 9] = float("inf"), 1e-35, float("nan")
    q = np.full((K, C), 3)
    Y = torch.empty(3, K, device="cuda")
    h = seq.seq_mv4_create(3, C, K, 128, seq.SEQ_F32)
    seq.seq_mv4(h, x, pack(q, K, C), torch.ones(1, K, device="cuda"), Y)
    y = Y.cpu()
    assert torch.isinf(y[0]).all() and torch.isnan(y[2]).all()
    assert np.abs(y[1].double().numpy() - 3 * np.float64(np.float32(1e-35))).max() <= 3 * 2.0 ** -133


@pytest.mark.parametrize("C,K,group", [(128, 16, 128), (200, 40, 128), (100, 17, 32), (1000, 72, 64), (7, 3, 32)])
def test_laying_out_weights(C, K, group):
    rng = np.random.default_rng(C)
    w = rng.standard_normal((K, C)).astype(np.float32)
    w[0] = 0
    h = seq.seq_mv4_create(1, C, K, group, seq.SEQ_BF16)
    wt = torch.full((h.info.wt_bytes,), 0xAB, dtype=torch.uint8, device="cuda")
    sc = nans(h.info.scale_bytes // 4)
    seq.seq_mv4_quant(h, torch.from_numpy(w).cuda(), wt, sc)
    Kp = -(-K // 16) * 16
    groups = -(-C // group)
    padded = np.zeros((K, groups * group), dtype=np.float32)
    padded[:, :C] = w
    want = np.abs(padded.reshape(K, groups, group)).max(-1).T / np.float32(7)
    got = sc.cpu().numpy().reshape(groups, Kp)
    np.testing.assert_array_equal(got[:, :K], want)
    assert not got[:, K:].any()
    per = np.repeat(want, group, 0)[:C].T
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(per > 0, np.rint(w / per), 0)
    assert torch.equal(wt.cpu(), pack(q, K, C).cpu())
    back = nans(K, C)
    seq.seq_mv4_unquant(h, wt, sc, back)
    assert np.all(np.abs(back.cpu().numpy() - w) <= per * (0.5 + 2.0 ** -20))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_groups_without_a_scale(bad):
    """A NaN or an infinity in a group: its scale is NaN, so that its products are, and the others stay as they are."""
    C, K, group = 96, 20, 32
    w = torch.linspace(-1, 1, K * C, device="cuda").reshape(K, C)
    h = seq.seq_mv4_create(1, C, K, group, seq.SEQ_BF16)
    out = []
    for value in (0.0, bad):
        w[3, 40] = value
        wt, sc = torch.empty(h.info.wt_bytes, dtype=torch.uint8, device="cuda"), nans(h.info.scale_bytes // 4)
        back = nans(K, C)
        seq.seq_mv4_quant(h, w, wt, sc)
        seq.seq_mv4_unquant(h, wt, sc, back)
        out.append(back.cpu())
    hit = torch.zeros(K, C, dtype=torch.bool)
    hit[3, 32:64] = True
    assert torch.isnan(out[1][hit]).all() and torch.equal(out[0][~hit], out[1][~hit])
