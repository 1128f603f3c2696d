"""The fp64 oracle of the norm, rotation and 4-bit cache, pinned by hand-computed values and identities."""

import numpy as np
import pytest

from oracle import q4


def test_rotation_keeps_norms_and_relative_angles():
    rng = np.random.default_rng(0)
    P, D = 40, 16
    angle = np.arange(P)[:, None] * 0.3 ** (np.arange(D // 2) / 3)
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    x = rng.standard_normal((P, 2, D))
    for il in (False, True):
        y = q4.norm_rotate(x, cos_sin=table, interleaved=il, pos=np.arange(P))
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
        # q at p and k at p + 3 meet at the angle of their distance alone
        a, b = x[0, 0], x[1, 1]
        both = [q4.norm_rotate(np.stack([a, b])[:, None], cos_sin=table, interleaved=il, pos=np.array([p, p + 3]))[:, 0]
                for p in (0, 20)]
        assert np.isclose(both[0][0] @ both[0][1], both[1][0] @ both[1][1])
    assert np.allclose(q4.norm_rotate(np.array([[[1.0, 0.0]]]), cos_sin=np.array([[0.6, 0.8]]), pos=np.array([0])), [[[0.6, 0.8]]])


def test_norm():
    x = np.array([[3.0, 4.0]])
    assert np.allclose(q4.norm_rotate(x, weight=np.array([2.0, 1.0])), [[6 / np.sqrt(12.5), 4 / np.sqrt(12.5)]])


def test_quantize_by_hand():
    x = np.zeros(16)
    x[:5] = [-1.0, 14.0, 0.5, 1.5, 2.4]     # scale 1, offset -1: quotients 0, 15, 1.5, 2.5, 3.4, and 1 for zeros
    codes, sq, gap = q4.quantize_rows(x)
    assert codes.tolist() == [0, 15, 2, 2, 3] + [1] * 11 and sq.tolist() == [0x3F80, 0xBF80]
    assert gap[2] == 0 and gap[3] == 0 and gap[5] == 0.5
    assert (q4.unpack_codes(q4.pack_codes(codes)) == codes).all()
    codes, sq, _ = q4.quantize_rows(np.full(16, 0.1))
    assert not codes.any() and sq[0] == 0 and sq[1] == q4.to_bf16_bits(0.1)
    for odd in (np.nan, np.inf, -np.inf):
        x[3] = odd
        codes, sq, _ = q4.quantize_rows(x)
        assert not codes.any() and (sq == 0x7FC0).all()


@pytest.mark.parametrize("v,bits", [(1.0, 0x3F80), (1.00390625, 0x3F80), (1.01171875, 0x3F82), (-2.5, 0xC020), (3.4e38, 0x7F80)])
def test_bf16(v, bits):
    assert q4.to_bf16_bits(v) == bits


def test_attend_by_hand():
    kc = np.array([[1, 0], [0, 2]], dtype=np.uint8)
    ksq = np.array([[1.0, 0.0], [0.5, 0.0]])
    vsq = np.array([[1.0, -1.0], [2.0, 0.0]])
    q = np.log(3) * np.array([[[1.0, 0.0]], [[1.0, 0.0]]])
    out, *_ = q4.attend(q, kc, ksq, kc, vsq, np.array([0, 1]), scale=1.0)
    assert np.allclose(out[0, 0], [0, -1])                       # sees the first token alone
    assert np.allclose(out[1, 0], [0, (3 * -1 + 4) / 4])         # logits ln 3 and 0
    out, *_ = q4.attend(q, kc, ksq, kc, vsq, np.array([-1, 1]), window=1, sinks=[0.0], scale=1.0)
    assert not out[0].any() and np.allclose(out[1, 0], [0, 2.0])  # half of the weight goes to the sink
