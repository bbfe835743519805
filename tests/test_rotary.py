"""Host side of the rotary calls: frequencies, fixed-point table, refusals (no GPU needed)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def _wanted(R, base, scaling, factor, L0, low, high):
    i = np.arange(R // 2, dtype=np.float64)
    f = base ** (-2 * i / R)
    if scaling == "linear":
        return f / factor
    if scaling == "ntk":
        return (base * factor ** (R / (R - 2))) ** (-2 * i / R)
    if scaling == "parts":
        w = np.clip((L0 * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return f * w + f / factor * (1 - w)
    if scaling == "ramp":
        at = lambda r: R * math.log(L0 / (2 * math.pi * r)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), R - 1)
        w = 1 - np.clip((i - lo) / (hi - lo), 0, 1)
        return f * w + f / factor * (1 - w)
    return f


@pytest.mark.parametrize("R", [2, 16, 50, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "parts", "ramp"])
def test_frequencies_are_the_formulas(lib, R, scaling):
    if scaling == "ntk" and R == 2:
        with pytest.raises(binding.OptGqaError):
            binding.rotary_frequencies(R, 1e4, scaling, 4.0)
        return
    got = binding.rotary_frequencies(R, 1e4, scaling, 4.0, 4096.0, 1.0, 32.0).numpy()
    want = _wanted(R, 1e4, scaling, 4.0, 4096.0, 1.0, 32.0)
    # a handful of 64-bit operations of at most an ulp each, the power amplifying its argument's by 2 ln(base) < 19
    np.testing.assert_allclose(got, want, rtol=64 * 2.0 ** -52, atol=0)


def test_scaled_frequencies_keep_the_fast_pairs_and_divide_the_slow_ones(lib):
    plain = binding.rotary_frequencies(128, 1e4)
    for scaling in ("parts", "ramp"):
        f = binding.rotary_frequencies(128, 1e4, scaling, 8.0, 8192.0, 1.0, 32.0)
        assert f[0] == plain[0] and torch.allclose(f[-1], plain[-1] / 8, rtol=1e-14)
        assert bool((f[1:] < f[:-1]).all())


def test_table_is_the_fraction_of_a_turn(lib):
    f = torch.tensor([1.0, 0.0, 2 * math.pi, -2 * math.pi / 4, 1e-9, 2 * math.pi * 3.25, 123.456], dtype=torch.float64)
    got = [int(x) & (2 ** 64 - 1) for x in binding.rotary_table(f, "cpu")]
    turns = (f.numpy() / (2 * math.pi)) % 1.0
    for g, w in zip(got, turns):
        d = abs(g - int(w * 2.0 ** 64)) % 2 ** 64
        # one division and one subtraction in 64 bits, of at most 20 turns: 20 * 2^-52 turns
        assert min(d, 2 ** 64 - d) <= 20 * 2 ** 12
    # multiples of 2pi by powers of two divide out exactly; 3.25 * 2pi is rounded when it is formed and again when it is
    # divided, by at most half an ulp of a value below 4 each time: 2^-51 turns in all
    assert got[1] == 0 and got[2] == 0 and got[3] == 3 << 62 and abs(got[5] - (1 << 62)) <= 2 ** 13
    # the angle at a position wraps without a rounding: position 2^31 - 1 of a quarter turn back
    assert (((2 ** 31 - 1) * got[3]) % 2 ** 64) >> 62 == (3 * (2 ** 31 - 1)) % 4


def test_frequency_and_table_refusals(lib):
    f, n = lib.opt_gqa_rotary_frequencies, np.zeros(64).ctypes.data
    assert f(None, 64, 1e4, 0, 1, 0, 0, 0) == -1
    assert f(n, 63, 1e4, 0, 1, 0, 0, 0) == -2 and f(n, 0, 1e4, 0, 1, 0, 0, 0) == -2
    for base in (0.0, -1.0, math.nan, math.inf):
        assert f(n, 64, base, 0, 1, 0, 0, 0) in ((-2,) if base != math.inf else (0, -2))
    assert f(n, 64, 1e4, 5, 1, 0, 0, 0) == -2 and f(n, 64, 1e4, -1, 1, 0, 0, 0) == -2
    assert f(n, 64, 1e4, 1, 0.0, 0, 0, 0) == -2 and f(n, 64, 1e4, 1, math.nan, 0, 0, 0) == -2
    for kind in (3, 4):
        assert f(n, 64, 1e4, kind, 8, 0.0, 1, 32) == -2
        assert f(n, 64, 1e4, kind, 8, 4096, 32, 32) == -2
        assert f(n, 64, 1e4, kind, 8, 4096, 0, 32) == -2
        assert f(n, 64, 1e4, kind, 8, 4096, 1, 32) == 0
    assert f(n, 64, 1.0, 4, 8, 4096, 1, 32) == -2
    t = lib.opt_gqa_rotary_table
    assert t(n, n, -1) == -2 and t(None, None, 0) == 0 and t(None, n, 4) == -1 and t(n, None, 4) == -1
    bad = np.array([0.5, math.nan])
    assert t(n, bad.ctypes.data, 2) == -2 and t(n, np.array([math.inf]).ctypes.data, 1) == -2


def test_rotary_argument_checks_run_before_any_cuda_call(lib):
    one, odd = ctypes.c_void_p(256), ctypes.c_void_p(264)

    def rotary(q_out=one, q=one, k_out=one, k=one, pos=one, freq=one, R=128, layout=0, T=2, Hq=4, Hkv=2, D=128,
               qos=512, qs=512, kos=256, ks=256, dtype=1):
        return lib.opt_gqa_rotary(q_out, q, k_out, k, pos, freq, R, layout, 1.0, 0, T, Hq, Hkv, D, qos, qs, kos, ks,
                                  dtype, None)

    assert rotary(dtype=2) == -3
    for bad in (dict(R=0), dict(R=3), dict(R=130), dict(layout=2), dict(layout=-1), dict(T=-1), dict(Hq=-1), dict(Hkv=-1),
                dict(D=96), dict(qs=504), dict(qs=0), dict(qs=-512), dict(kos=128), dict(qs=1 << 60), dict(qs=1024),
                dict(ks=512)):
        assert rotary(**bad) == -2, bad
    for bad in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(pos=None), dict(freq=None)):
        assert rotary(**bad) == -1, bad
    for bad in (dict(q=odd), dict(k_out=odd), dict(q_out=odd, qs=516), dict(q_out=odd, ks=260, k=ctypes.c_void_p(512))):
        assert rotary(**bad) == -4, bad
    assert rotary(T=0, q=None, q_out=None, k=None, k_out=None, pos=None, freq=None) == 0
    assert rotary(Hq=0, Hkv=0) == 0

    def append(q_out=one, q=one, k_out=None, k=one, v=one, kc=one, vc=one, slots=one, pos=one, freq=one, R=64, layout=0,
               T=2, Hq=4, Hkv=2, D=64, qs=256, ks=128, vs=128, bs=16, blocks=4, dtype=0):
        return lib.opt_gqa_rotary_append(q_out, q, k_out, k, v, kc, vc, slots, pos, freq, R, layout, 1.0, T, Hq, Hkv, D,
                                         qs, ks, vs, bs, blocks, dtype, None)

    assert append(dtype=9) == -3
    for bad in (dict(R=66), dict(bs=8), dict(blocks=-1), dict(blocks=0), dict(Hkv=0), dict(vs=64), dict(D=100), dict(T=-3),
                dict(blocks=1 << 60)):
        assert append(**bad) == -2, bad
    for bad in (dict(v=None), dict(kc=None), dict(vc=None), dict(slots=None), dict(k=None), dict(q=None), dict(pos=None)):
        assert append(**bad) == -1, bad
    for bad in (dict(v=odd), dict(kc=odd), dict(vc=odd), dict(k_out=odd), dict(vs=130), dict(q=odd)):
        assert append(**bad) == -4, bad
    assert append(T=0, q=None, k=None, v=None, kc=None, vc=None, slots=None, pos=None, freq=None, blocks=0) == 0


def test_binding_refuses_tensors_that_do_not_fit(lib):
    q = torch.zeros(3, 4, 64)
    pos, freq = torch.zeros(3, dtype=torch.int32), torch.zeros(32, dtype=torch.int64)
    for kw in (dict(q_out=torch.zeros(3, 4, 32)), dict(q_out=None), dict(positions=pos.long()), dict(positions=pos[:2]),
               dict(freq=freq.double()), dict(k=torch.zeros(2, 2, 64), k_out=torch.zeros(2, 2, 64)),
               dict(k=torch.zeros(3, 2, 64)), dict()):                  # the last: host tensors
        a = dict(dict(q_out=q, q=q, positions=pos, freq=freq, layout=0), **kw)
        with pytest.raises(ValueError):
            binding.rotary(**a)
    cache = torch.zeros(2, 2, 16, 64)
    k = torch.zeros(3, 2, 64)
    slots = torch.zeros(3, dtype=torch.int64)
    for kw in (dict(v=k[:2]), dict(slot_mapping=slots.int()), dict(slot_mapping=slots[:1]), dict(q=q[:, :, :32], q_out=q),
               dict(q=q, q_out=None), dict(k_cache=cache.bfloat16()), dict(v_cache=cache[:1]), dict(k_out=k[:2]), dict()):
        a = dict(dict(q_out=q, q=q, k=k, v=k, k_cache=cache, v_cache=cache, slot_mapping=slots, positions=pos, freq=freq,
                      layout=0), **kw)
        with pytest.raises(ValueError):
            binding.rotary_append(**a)
