"""The 64-bit implementation of the 4-bit key/value cache against values worked out by hand."""
import numpy as np

from oracle import kv as O


def test_sixteen_bit_rounding():
    x = np.array([0.0, 1.0, -2.5, 1 + 2 ** -8, 1 + 2 ** -8 + 2 ** -20, 3.0e38, -1e-30])
    back = O.from16(O.to16(x, "bf16"), "bf16")
    assert back[:3].tolist() == [0.0, 1.0, -2.5]
    assert back[3] == 1.0                          # a tie goes to the even neighbour
    assert back[4] == 1 + 2 ** -7
    # eight significant bits: half a unit in the last place is at most 2^-8 of the number
    assert np.all(np.abs(back - x) <= 2.0 ** -8 * np.abs(x))
    assert O.from16(O.to16(np.array([0.1]), "f16"), "f16")[0] == float(np.float16(0.1))


def test_channel_order():
    # word w holds channels 8w..8w+7: even ones in the low half, odd ones in the high half
    bit = O.channel_bit()
    assert bit[:8].tolist() == [0, 16, 4, 20, 8, 24, 12, 28]
    assert bit[8] == 32 and sorted(bit.tolist()) == list(range(0, 256, 4))


def test_block_decodes_as_laid_out():
    page, d = 16, 128
    block = np.zeros(2 * 2 * page * 36, np.uint8)
    # K, slot 3, group 1: channel 64 + 9 has code 5; scale 0.5, low -1
    bit = int(O.channel_bit()[9])
    block[1 * page * 32 + 3 * 32 + bit // 8] = 5 << (bit % 8)
    meta = 2 * page * 32 + (3 * 2 + 1) * 4
    block[meta:meta + 4] = np.array([0x3F00, 0xBF80], np.uint16).view(np.uint8)
    out = O.decode_block(block, page, d, "bf16")
    assert out["k"][3, 64 + 9] == 1.5 and out["k"][3, 64 + 8] == -1.0
    assert out["k"][3, 0] == 0.0 and np.all(out["v"] == 0.0)


def test_quantise_by_hand():
    x = np.zeros(64)
    x[0], x[1], x[2], x[3] = -1.0, 14.0, 0.49, 0.5
    code, scale, low = O.quantise(x, "bf16")
    assert scale == 1.0 and low == -1.0
    assert code[:4].tolist() == [0, 15, 1, 2]      # 1.5 goes to the even 2
    code, scale, low = O.quantise(np.full(64, 3.0), "f16")
    assert scale == 0 and low == 3.0 and not code.any()


def test_attend_by_hand():
    k = np.array([[1.0, 0.0], [0.0, 1.0]])
    v = np.array([[1.0, 2.0], [3.0, 4.0]])
    q = np.array([[np.log(3.0), 0.0], [0.0, 0.0], [5.0, 5.0]])
    sees = np.array([[True, True], [False, True], [False, False]])
    out, lse = O.attend(q, k, v, sees, 1.0)
    assert np.allclose(out[0], [1.5, 2.5]) and np.isclose(lse[0], np.log(4.0))
    assert np.allclose(out[1], [3.0, 4.0]) and lse[1] == 0.0
    assert np.all(out[2] == 0) and lse[2] == -np.inf


def test_evict_by_hand():
    weight = np.array([5.0, 1.0, 1.0, 9.0, 0.0, 2.0])
    pos = np.array([0, 7, 3, 4, 9, 5])
    # position 0 and the newest (9) stay; then 9.0, 2.0: slots 0, 3, 4, 5 kept, 1 and 2 free
    assert O.evict(weight, pos, 10, 4, 1, 1).tolist() == [0, 4, 5, 3]
    # a tie of weights: the lower position stays
    assert O.evict(weight, pos, 100, 5, 0, 0).tolist() == [0, 1, 2, 3, 5]
    assert O.evict(np.array([1.0, 1.0, 1.0]), np.array([8, 2, 5]), 9, 2, 0, 0).tolist() == [2, 1]
