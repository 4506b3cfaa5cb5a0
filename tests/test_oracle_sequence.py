"""Pins of the plain implementations in oracle/sequence.py on cases worked out by hand, and of pack_weights (CPU only)."""
import numpy as np
import pytest

from oracle import sequence as S


def test_plan_by_hand():
    # pages of 4; stream 0 has 3 tokens on page 9 and gets 2: one more page; stream 1 ends and gives 5, 6 back; stream 2 starts with 5
    table = np.array([[9, -1, -1], [5, 6, -1], [-1, -1, -1]])
    free = np.array([1, 2, -1, -1, -1, -1, -1, -1, -1, -1])
    slots, off, after, count, t, f = S.plan([2, -1, 5], [3, 8, 0], table, free, 2, 4, 9)
    assert f[:4].tolist() == [1, 2, 5, 6] and count == 1
    assert t.tolist() == [[9, 6, -1], [5, 6, -1], [5, 2, -1]]
    assert slots.tolist() == [39, 24, 20, 21, 22, 23, 8, -1, -1] and off.tolist() == [0, 2, 2, 7] and after.tolist() == [5, 0, 5]


def test_plan_refuses_by_running_sums():
    table = np.full((4, 2), -1)
    # 2 free pages: stream 0 needs 2, stream 1 (1 page) comes too late, stream 2 asks for nothing, stream 3 does not fit its row
    slots, off, after, count, t, _ = S.plan([5, 1, 0, 9], [0, 0, 0, 0], table, np.array([7, 3]), 2, 4, 20)
    assert off.tolist() == [0, 5, 5, 5, 5] and after.tolist() == [5, 0, 0, 0] and count == 0
    assert t[0].tolist() == [3, 7] and (t[1:] == -1).all() and slots[:5].tolist() == [12, 13, 14, 15, 28]
    # slots: the second stream's tokens pass the room for them
    _, off, _, _, _, _ = S.plan([2, 2, 1], [0, 0, 0], np.full((3, 2), -1), np.arange(6), 6, 4, 3)
    assert off.tolist() == [0, 2, 2, 2]


def test_e4m3_values():
    v = S.e4m3_values()
    assert v[0x7E] == 448 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1 and v[0xB8] == -1 and np.isnan(v[0x7F])


def test_attend_by_hand():
    k = np.zeros((2, 2, 1, 2)); v = np.arange(8.0).reshape(2, 2, 1, 2)
    k[1, 0, 0] = [1, 0]
    # stream 0: tokens on page 1 then page 0, 3 of them; stream 1 has none; stream 2's page does not exist
    out, lse = S.attend(np.array([[[2.0, 0]]] * 3), k, v, np.array([[1, 0], [0, 0], [5, 5]]), [3, 0, 4], 2, 0.5)
    e = np.exp(1.0)
    assert np.allclose(out[0, 0], (e * v[1, 0, 0] + v[1, 1, 0] + v[0, 0, 0]) / (e + 2)) and np.isclose(lse[0, 0], np.log(e + 2))
    assert (out[1:] == 0).all() and np.isneginf(lse[1:]).all()
    out, _ = S.attend(np.array([[[2.0, 0]]]), k, v, np.array([[1, 0]]), [3], 2, 0.5, window=1)
    assert np.allclose(out[0, 0], v[0, 0, 0])


def test_norm_by_hand():
    s, y, sc = S.norm(np.array([[3.0, 1.0]]), np.array([1.0, 2.0]), np.array([[0.0, 3.0]]), 0.0)
    assert s.tolist() == [[3, 4]] and np.allclose(y, np.array([[3, 8]]) / np.sqrt(12.5)) and np.isclose(sc[0], 8 / np.sqrt(12.5) / 448)


def test_matvec_by_hand():
    w = np.zeros((1, 32), np.uint8); w[0, 0] = 0x72; w[0, 16] = 0x0F       # k=0: 1, k=1: 6; k=32: -6
    sc = np.array([[127, 126]], np.uint8)
    x = np.zeros((1, 40)); x[0, [0, 1, 32]] = [10, 1, 2]
    assert S.matvec(x, w, sc)[0, 0] == 10 + 6 - 6 and S.matvec(-x, w, sc, relu=True)[0, 0] == 0


@pytest.mark.parametrize("n,k", [(1, 1), (3, 31), (4, 32), (5, 33), (7, 200)])
def test_pack_weights_takes_the_nearest_code(n, k):
    from paper_2407_16990_amd import pack_weights
    rng = np.random.default_rng(n * 1000 + k)
    w = rng.standard_normal((n, k)) * np.exp2(rng.integers(-20, 20, (n, 1)))
    w[0, : min(k, 32)] = 0                                     # a block of zeros
    codes, scales = pack_weights(w)
    assert codes.shape == (n, 16 * ((k + 31) // 32)) and scales.shape == (n, (k + 31) // 32)
    got = S.unpack_weights(codes, scales, k)
    factor = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)[:, :k]
    # every value is within half a step of its code's neighbours; the largest of a block is below 8, and what passes 6 becomes 6
    scaled = w / factor
    near = np.abs(scaled[..., None] - S.FP4).min(-1)
    assert (np.abs(got / factor - scaled) <= near + 1e-12).all() and (np.abs(scaled) < 8).all()


def test_pack_weights_keeps_what_the_codes_can_hold():
    from paper_2407_16990_amd import pack_weights
    w = np.array([[0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6] + [0] * 17]) * 2.0 ** -9
    codes, scales = pack_weights(w)
    assert np.array_equal(S.unpack_weights(codes, scales, 32), w)
    with pytest.raises(ValueError):
        pack_weights(np.array([[np.nan]]))
