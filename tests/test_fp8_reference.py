"""The 8-bit cache's reference against the format's definition, by enumeration (CPU)."""
import numpy as np
import torch

import fp8_ref as ref
from fp4_ref import E4M3


def test_scale_is_the_smallest_power_that_holds_the_block():
    for e in range(-14, 8):
        top = 448 * 2.0 ** e
        assert ref.scale_of(top) == 2.0 ** e
        if e < 7:
            assert ref.scale_of(np.nextafter(top, np.inf)) == 2.0 ** (e + 1)
    assert ref.scale_of(0.0) == 2.0 ** -15 and ref.scale_of(np.inf) == 2.0 ** 7


def test_codes_are_those_of_the_type():
    """Against torch's conversion, over every bf16 magnitude that the scale reaches."""
    bits = torch.arange(0, 0x7f80, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).double()
    x = x[x <= 448]
    for sign in (1, -1):
        want = (sign * x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        np.testing.assert_array_equal(ref.code_of(sign * x.numpy(), 1.0), want)
    assert ref.code_of(np.array([np.nan, 1e9, -np.inf]), 1.0).tolist() == [127, 126, 254]


def test_every_value_is_exact_in_bf16_and_fp16():
    codes = np.arange(256, dtype=np.uint8)
    codes = codes[(codes & 127) != 127]
    for s in ref.POWERS:
        v = ref.values(codes.reshape(1, 1, -1), np.array([s]))[0, 0]
        assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)
        assert np.array_equal(v.astype(np.float16).astype(np.float64), v)


def test_round_trip_and_second_rounding():
    """A value comes back within half a step of e4m3, and moving to a larger power changes nothing above the subnormals."""
    r = np.random.default_rng(0)
    x = r.standard_normal((16, 64)) * 10.0 ** r.integers(-2, 2, (16, 1))
    s = ref.scale_of(np.abs(x).max())
    v = ref.values(ref.code_of(x, s), s)
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * E4M3[1] / 2)).all()
    up = ref.values(ref.code_of(v, 4 * s), 4 * s)
    normal = np.abs(v) >= 4 * s * E4M3[8]
    assert np.array_equal(up[normal], v[normal])


def test_page_references():
    table = np.array([[5, 6, 7, -1], [-1] * 4, [-1] * 4])
    t, n, sh, st, c = ref.fork([0, 0], [1, 2], table, [40, 0, 0], np.zeros(10, int), [1, 2, 3])
    assert t.tolist() == [[5, 6, 7, -1], [5, 6, 3, -1], [5, 6, 2, -1]] and n.tolist() == [40] * 3
    assert sh[[5, 6, 7]].tolist() == [2, 2, 0] and st == [1] and c == [(7, 3), (7, 2)]
    t2, n2, sh2, st2 = ref.free([1, 2], t, n, sh, st)
    assert t2.tolist() == table.tolist() and st2 == [1, 2, 3] and not sh2.any() and n2.tolist() == [40, 0, 0]
    t3, _, sh3, st3 = ref.free([0], t, n, sh, st)
    assert st3 == [1, 7] and sh3[[5, 6]].tolist() == [1, 1]
    tc, shc, stc, pm, mv = ref.compact(t, sh, [1, 0, 4, 8, 9], 10)
    assert mv == [(5, 0), (6, 1), (7, 4)] and stc == [9, 8, 7, 6, 5] and tc.tolist() == [[0, 1, 4, -1], [0, 1, 3, -1], [0, 1, 2, -1]]
    assert shc[[0, 1]].tolist() == [2, 2]
