"""Host side of the chunk attention: workspace size and refusals (no GPU needed)."""
import ctypes
import struct

import pytest
import torch

from paper_2505_02351_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def test_workspace_holds_two_parts_per_worker(lib):
    f = binding.chunk_workspace_bytes
    for q, rows in ((1, 32), (8, 32), (9, 64), (17, 96), (25, 128), (32, 128), (33, 128), (100000, 128)):
        need = 2 * 2 * 148 * rows * (128 + 1) * 4       # two CTAs per multiprocessor, two places each
        # and what the merge needs to know of each: a word and two times four; four arrays rounded up to 256 bytes
        assert need + 296 * 36 <= f(32, 8, 128, q) <= need + 296 * 36 + 4 * 256, q
    assert f(32, 8, 128, 2 ** 31 - 1) == f(32, 8, 128, 32) and f(8, 8, 64, 1) > 0
    for bad in ((33, 8, 128, 1), (48, 3, 128, 1), (32, 8, 96, 1), (32, 8, 128, 0), (32, 8, 128, -1), (0, 8, 128, 1)):
        assert f(*bad) == 0, bad


def test_argument_checks_run_before_any_cuda_call(lib):
    one, odd = ctypes.c_void_p(256), ctypes.c_void_p(264)

    def call(out=one, q=one, stride=4096, qsl=one, T=9, most=4, k=one, v=one, bt=one, maxb=8, n=one, sl=one, B=4, Hq=32, Hkv=4,
             D=128, bs=16, blocks=100, window=0, ws=one, wsb=None, dtype=1):
        if wsb is None:
            wsb = binding.chunk_workspace_bytes(32, 4, 128, 4)
        return lib.opt_gqa_paged_attention_chunk(out, q, stride, qsl, T, most, k, v, bt, maxb, n, sl, 1.0, B, Hq, Hkv, D, bs, blocks,
                                                 window, ws, wsb, dtype, None)

    assert call(dtype=0) == -3 and call(dtype=7) == -3
    for bad in (dict(B=-1), dict(B=70000), dict(T=-1), dict(most=-1), dict(Hq=33), dict(Hq=64), dict(D=96), dict(bs=8), dict(maxb=-1),
                dict(maxb=0), dict(blocks=0), dict(blocks=-1), dict(window=-1), dict(stride=4088), dict(stride=1 << 40), dict(stride=-8),
                dict(wsb=0), dict(wsb=binding.chunk_workspace_bytes(32, 4, 128, 4) - 1), dict(most=5)):
        assert call(**bad) == -2, bad
    for name in ("out", "q", "qsl", "k", "v", "bt", "n", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("out", "q", "k", "v", "ws"):
        assert call(**{name: odd}) == -4, name
    assert call(stride=4100) == -4
    for none in (dict(B=0), dict(T=0), dict(most=0)):
        assert call(**none, out=None, q=None, qsl=None, ws=None) == 0


def test_binding_refuses_tensors_that_do_not_fit(lib):
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    cache = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    for kw in (dict(out=q[:2]), dict(v_cache=cache[:1]), dict(k_cache=cache[..., :32]), dict(block_tables=i),
               dict(block_tables=torch.zeros(2, 4, dtype=torch.int32)), dict()):            # the last: host tensors
        a = dict(dict(out=q, q=q, q_start_loc=torch.zeros(4, dtype=torch.int32), max_q_len=1, k_cache=cache, v_cache=cache,
                      block_tables=torch.zeros(3, 4, dtype=torch.int32), context_lens=i, alibi_slopes=None, scale=1.0,
                      workspace=None), **kw)
        with pytest.raises(ValueError):
            binding.paged_attention_chunk(**a)


def test_a_record_of_the_arguments_is_refused_as_the_call_is(lib):
    wsb = binding.chunk_workspace_bytes(32, 4, 128, 4)
    good = dict(out=256, q=256, stride=4096, qsl=256, T=9, most=4, k=256, v=256, bt=256, maxb=8, n=256, sl=256, scale=1.0, B=4, Hq=32, Hkv=4,
                D=128, bs=16, blocks=100, window=0, ws=256, wsb=wsb, dtype=1, stream=0)

    def call(which=0, **kw):
        return lib.opt_gqa_call_record(which, struct.pack("=12qd11q", *dict(good, **kw).values()))

    for code, cases in ((-3, (dict(dtype=0), dict(dtype=7))),
                        (-2, (dict(B=-1), dict(B=70000), dict(T=-1), dict(most=-1), dict(Hq=33), dict(Hkv=3), dict(D=96), dict(bs=8),
                              dict(maxb=0), dict(blocks=0), dict(window=-1), dict(stride=4088), dict(stride=1 << 40), dict(wsb=wsb - 1))),
                        (-1, [{name: 0} for name in ("out", "q", "qsl", "k", "v", "bt", "n", "ws")]),
                        (-4, [{name: 264} for name in ("out", "q", "k", "v", "ws")] + [dict(stride=4100)]),
                        (0, (dict(B=0), dict(T=0), dict(most=0)))):
        for bad in cases:
            assert call(**bad) == code, bad
    for name in ("T", "most", "maxb", "B", "Hq", "Hkv", "D", "bs", "window", "dtype"):          # not cut to 32 bits
        assert call(**{name: good[name] + (1 << 32)}) == -2, name
    assert call(which=5) == -2 and call(which=-1) == -2 and lib.opt_gqa_call_record(0, None) == -1
