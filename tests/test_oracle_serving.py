"""Pins of the serving oracle: against torch's own attention arithmetic in 64 bits, by hand-made cases, and its E4M3 against
torch's conversion."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so


def test_attend_is_softmax_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(5, 16)), rng.normal(size=(9, 16)), rng.normal(size=(9, 16))
    seen = rng.random((5, 9)) < 0.6
    seen[2] = False
    seen[3] = True
    o, lse, tol, slack = so.attend(q, k, v, seen)
    s = torch.from_numpy(q @ k.T / 4.0).masked_fill(~torch.from_numpy(seen), -np.inf)
    for r in range(5):
        if r == 2:
            assert (o[r] == 0).all() and lse[r] == -np.inf
            continue
        assert np.allclose(o[r], (torch.softmax(s[r], 0)[:, None] * torch.from_numpy(v)).sum(0).numpy(), atol=1e-13)
        assert np.isclose(lse[r], float(torch.logsumexp(s[r], 0)), atol=1e-13)
        assert (tol[r] > 0).all() and 0 < slack[r] < 1e-3


def test_what_is_not_seen_has_no_effect():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(2, 8)), rng.normal(size=(4, 8)), rng.normal(size=(4, 8))
    seen = np.array([[True, True, False, False], [True, True, True, False]])
    o, lse, _, _ = so.attend(q, k, v, seen)
    k[3], v[3], v[2] = np.nan, np.inf, np.nan
    o2, lse2, _, _ = so.attend(q, k, v, seen)
    assert np.array_equal(o[0], o2[0]) and np.array_equal(lse, lse2) and np.isnan(o2[1]).all()


def test_decode_of_pages_is_attend_of_the_rows_they_hold():
    rng = np.random.default_rng(3)
    hkv, group, page, d = 2, 3, 16, 8
    k, v = rng.normal(size=(2, 40, hkv, d))
    pages = rng.normal(size=(2, 6, hkv, page, d))
    order, pre = [4, 0, 2], [5]
    for i in range(40):
        pages[0, order[i // page], :, i % page] = k[i]
        pages[1, order[i // page], :, i % page] = v[i]
    q = rng.normal(size=(1, hkv * group, 2, d))
    o, lse, _, _ = so.decode(q, pages[0], pages[1], np.array([order + [-1]]), np.array([40]), np.array(pre), 7)
    for h in range(hkv * group):
        for t in range(2):
            ks = np.concatenate([pages[0, 5, h // group, :7], k[:39 + t, h // group]])
            vs = np.concatenate([pages[1, 5, h // group, :7], v[:39 + t, h // group]])
            want = so.attend(q[0, h, t:t + 1], ks, vs, np.ones((1, len(ks)), dtype=bool))
            assert np.allclose(o[0, h, t], want[0][0], atol=1e-14) and np.isclose(lse[0, h, t], want[1][0], atol=1e-13)


def test_holes_and_lengths_beyond_the_table():
    rng = np.random.default_rng(4)
    pages = rng.normal(size=(2, 3, 1, 16, 4))
    q = rng.normal(size=(4, 1, 1, 4))
    table = np.array([[0, 1], [0, 7], [-5, 2], [0, 1]])
    o, lse, _, _ = so.decode(q, pages[0], pages[1], table, np.array([99, 32, 17, -3]), np.array([], dtype=int), 0)
    whole = np.concatenate([pages[0, 0, 0], pages[0, 1, 0]])
    want = [so.attend(q[0, 0], whole, np.concatenate([pages[1, 0, 0], pages[1, 1, 0]]), np.ones((1, 32), dtype=bool)),
            so.attend(q[1, 0], pages[0, 0, 0], pages[1, 0, 0], np.ones((1, 16), dtype=bool)),
            so.attend(q[2, 0], pages[0, 2, 0, :1], pages[1, 2, 0, :1], np.ones((1, 1), dtype=bool))]
    for s in range(3):
        assert np.allclose(o[s, 0], want[s][0], atol=1e-14) and np.allclose(lse[s, 0], want[s][1], atol=1e-13)
    assert (o[3] == 0).all() and lse[3, 0, 0] == -np.inf


def test_positions():
    assert so.positions([3, 0, 1, -2], [2, 1, 3, 1]) == [(0, 0, 1), (0, 1, 2), (2, 2, 0)]


@pytest.mark.parametrize("scale", [1e-4, 0.3, 40.0])
def test_e4m3_is_torchs(scale):
    x = np.concatenate([np.random.default_rng(5).normal(size=20000) * scale, np.arange(-460, 461) * 0.5, [0.0, 2.0 ** -10, 3 * 2.0 ** -10]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert np.array_equal(so.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    assert so.e4m3(np.float32(1e9)) == 448 and so.e4m3(-np.inf) == -448 and np.isnan(so.e4m3(np.nan))
