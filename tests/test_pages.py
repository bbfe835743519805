"""Host side of the page operators: workspace size and refusals (no GPU needed)."""
import ctypes
import struct

import pytest
import torch

from paper_2505_02351_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(260)


def addresses(*a):
    return (ctypes.c_void_p * len(a))(*a)


POOLS = addresses(256, 512)


def test_workspace_grows_with_requests_and_pages(lib):
    f = binding.pages_workspace_bytes
    # per request seven words and a 64-bit one, per page one word and, of half the pages, three
    assert 65535 * 36 + 4 * 1000 <= f(65535, 1000) <= 65535 * 36 + 4 * 1000 + 10 * 256
    assert 4 * 100000 + 3 * 4 * 50000 <= f(1, 100000) <= 4 * 100000 + 3 * 4 * 50001 + 36 + 10 * 256
    sizes = [f(n, b) for n, b in ((1, 1), (1, 10), (9, 10), (9, 5000), (300, 5000), (3000, 5000), (3000, 1 << 28))]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for bad in ((0, 10), (-1, 10), (65536, 10), (1, 0), (1, -5), (1, (1 << 28) + 1)):
        assert f(*bad) == 0, bad


def bad_pools():
    yield -2, dict(num=0)
    yield -2, dict(num=-1)
    yield -2, dict(num=257)
    yield -2, dict(Hkv=0)
    yield -2, dict(Hkv=70000)
    yield -2, dict(D=96)
    yield -2, dict(bs=8)
    yield -2, dict(blocks=0)
    yield -2, dict(blocks=(1 << 28) + 1)
    yield -3, dict(dtype=2)
    yield -1, dict(pools=None)
    yield -1, dict(pools=addresses(256, None))
    yield -4, dict(pools=addresses(256, 264))


def test_copy_refuses_before_any_cuda_call(lib):
    def call(pools=POOLS, num=2, src=ONE, dst=ONE, n=3, Hkv=8, D=128, bs=16, blocks=10, dtype=1):
        return lib.opt_gqa_cache_copy_pages(pools, num, src, dst, n, Hkv, D, bs, blocks, dtype, None)

    for want, bad in bad_pools():
        assert call(**bad) == want, bad
    assert call(n=-1) == -2 and call(src=None) == -1 and call(dst=None) == -1
    assert call(n=0, src=None, dst=None) == 0


@pytest.mark.parametrize("entry", ["opt_gqa_cache_fork", "opt_gqa_cache_resize"])
def test_requests_refuse_before_any_cuda_call(lib, entry):
    def call(pools=POOLS, num=2, bt=ONE, W=8, lens=ONE, refs=ONE, a=ONE, b=ONE, n=3, done=ONE, S=4, Hkv=8, D=128, bs=16, blocks=10,
             ws=ONE, wsb=None, dtype=1):
        wsb = binding.pages_workspace_bytes(3, 10) if wsb is None else wsb
        return getattr(lib, entry)(pools, num, bt, W, lens, refs, a, b, n, done, S, Hkv, D, bs, blocks, ws, wsb, dtype, None)

    for want, bad in bad_pools():
        assert call(**bad) == want, bad
    for bad in (dict(n=-1), dict(n=65536), dict(S=0), dict(W=0), dict(W=1 << 27), dict(wsb=binding.pages_workspace_bytes(3, 10) - 1)):
        assert call(**bad) == -2, bad
    for name in ("bt", "lens", "refs", "a", "b", "done", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("refs", "ws"):
        assert call(**{name: ODD}) == -4, name
    assert call(n=0, a=None, b=None, done=None, ws=None) == 0


def test_compact_refuses_before_any_cuda_call(lib):
    def call(pools=POOLS, num=2, bt=ONE, bto=ONE, W=8, lens=ONE, refs=ONE, refs_out=ONE, pm=ONE, used=ONE, S=4, Hkv=8, D=128, bs=16,
             blocks=10, ws=ONE, wsb=None, dtype=1):
        wsb = binding.pages_workspace_bytes(1, 10) if wsb is None else wsb
        return lib.opt_gqa_cache_compact(pools, num, bt, bto, W, lens, refs, refs_out, pm, used, S, Hkv, D, bs, blocks, ws, wsb, dtype, None)

    for want, bad in bad_pools():
        assert call(**bad) == want, bad
    for bad in (dict(S=0), dict(W=0), dict(W=1 << 27), dict(wsb=binding.pages_workspace_bytes(1, 10) - 1)):
        assert call(**bad) == -2, bad
    for name in ("bt", "bto", "lens", "refs", "refs_out", "pm", "used", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("refs", "ws"):
        assert call(**{name: ODD}) == -4, name


def test_binding_refuses_host_tensors_and_no_pools(lib):
    with pytest.raises(ValueError):
        binding.page_pools([])
    with pytest.raises(ValueError):
        binding.page_pools([torch.zeros(2, 2, 16, 64)])


def host(pools):
    return 0 if pools is None else ctypes.addressof(pools)


@pytest.mark.parametrize("entry,where", [(1, "copy"), (2, "fork"), (3, "resize"), (4, "compact")])
def test_a_record_of_the_arguments_is_refused_as_the_call_is(lib, entry, where):
    fixed = dict(Hkv=8, D=128, bs=16, blocks=10)
    n = 1 if where == "compact" else 3
    wsb = binding.pages_workspace_bytes(n, 10)
    last = dict(ws=256, wsb=wsb, dtype=1, stream=0)
    good = dict(pools=POOLS, num=2)
    if where == "copy":
        good |= dict(src=256, dst=256, n=3) | fixed | dict(dtype=1, stream=0)
    elif where == "compact":
        good |= dict(bt=256, bto=256, W=8, lens=256, refs=256, refs_out=256, pm=256, used=256, S=4) | fixed | last
    else:
        good |= dict(bt=256, W=8, lens=256, refs=256, a=256, b=256, n=3, done=256, S=4) | fixed | last

    def call(**kw):
        values = dict(good, **kw)
        values["pools"] = host(values["pools"])
        return lib.opt_gqa_call_record(entry, struct.pack("=%dq" % len(values), *values.values()))

    for want, bad in bad_pools():
        assert call(**bad) == want, bad
    for name in set(good) & {"src", "dst", "bt", "bto", "lens", "refs", "refs_out", "pm", "used", "a", "b", "done", "ws"}:
        assert call(**{name: 0}) == -1, name
    for name in set(good) & {"refs", "ws"}:
        assert call(**{name: 260}) == -4, name
    for bad in (dict(n=-1), dict(S=0), dict(W=0), dict(W=1 << 27), dict(wsb=wsb - 1)):
        if set(bad) <= set(good):
            assert call(**bad) == -2, bad
    for name in set(good) & {"num", "W", "n", "S", "Hkv", "D", "bs", "dtype"}:                  # not cut to 32 bits
        assert call(**{name: good[name] + (1 << 32)}) == -2, name
    if "n" in good:
        assert call(n=0) == 0
