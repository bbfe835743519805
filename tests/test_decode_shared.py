"""Host side of the shared-prefix decode: workspace size and refusals (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2505_02351_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def test_workspace_holds_every_piece_of_both_passes(lib):
    B, Hq, Hkv, D, N, P = 256, 64, 8, 128, 12, 20
    G = Hq // Hkv
    rows = Hkv * (N + B * G // 128) * 128 + B * Hq          # of every (group, KV head, block of 128 rows) and every sequence
    need = binding.shared_workspace_bytes(B, Hq, Hkv, D, N, P)
    # and of at most two more pieces of either kind per multiprocessor, 32 bytes per (sequence, KV head), rounding
    assert rows * (D + 1) * 4 <= need
    assert need <= (rows + 2 * 148 * (128 + G)) * (D + 1) * 4 + B * Hkv * 32 + 4096
    # the route of small batches (of up to 32 MB of cache) needs the balanced decode's
    assert binding.shared_workspace_bytes(4, 32, 8, 128, 1, 110) >= (4 * 32 * 110 + 2048 * 4) * 129 * 4
    for bad in ((0, Hq, Hkv, D, N, P), (B, 63, Hkv, D, N, P), (B, Hq, Hkv, 96, N, P), (B, Hq, Hkv, D, 0, P),
                (B, Hq, Hkv, D, 513, P), (B, Hq, Hkv, D, N, 0), (1 << 17, Hq, Hkv, D, N, P), (B, 48, 3, D, N, P)):
        assert binding.shared_workspace_bytes(*bad) == 0, bad


def test_argument_checks_run_before_any_cuda_call(lib):
    one, odd = ctypes.c_void_p(256), ctypes.c_void_p(264)

    def call(out=one, q=one, k=one, v=one, bt=one, maxb=8, n=one, gs=one, pl=one, N=2, sl=one, B=4, Hq=32, Hkv=4, D=128,
             bs=16, blocks=100, P=512, ws=one, wsb=None, maxP=4, dtype=1):
        if wsb is None:
            wsb = binding.shared_workspace_bytes(B, Hq, Hkv, D, N, maxP)
        return lib.opt_gqa_paged_attention_decode_shared(out, q, k, v, bt, maxb, n, gs, pl, N, sl, 1.0, B, Hq, Hkv, D, bs,
                                                         blocks, P, ws, wsb, maxP, dtype, None)

    assert call(dtype=0) == -3 and call(dtype=7) == -3
    for bad in (dict(B=-1), dict(Hq=33), dict(Hq=64), dict(D=96), dict(bs=8), dict(maxb=-1), dict(maxb=0), dict(blocks=0),
                dict(P=0), dict(P=24), dict(P=-16), dict(maxP=0), dict(N=-1), dict(N=0), dict(N=513), dict(B=70000),
                dict(maxP=70000), dict(wsb=0),
                dict(wsb=binding.shared_workspace_bytes(4, 32, 4, 128, 2, 4) - 1)):
        assert call(**bad) == -2, bad
    for name in ("out", "q", "k", "v", "bt", "n", "gs", "pl", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("out", "q", "k", "v", "ws"):
        assert call(**{name: odd}) == -4, name
    assert call(B=0, out=None, q=None, gs=None, ws=None) == 0


def test_binding_refuses_tensors_that_do_not_fit(lib):
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    cache = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    for kw in (dict(out=q[:2]), dict(v_cache=cache[:1]), dict(k_cache=cache[..., :32]), dict(block_tables=i),
               dict(block_tables=torch.zeros(2, 4, dtype=torch.int32)), dict()):            # the last: host tensors
        a = dict(dict(out=q, q=q, k_cache=cache, v_cache=cache, block_tables=torch.zeros(3, 4, dtype=torch.int32),
                      context_lens=i, group_start=i, prefix_lens=i, alibi_slopes=None, scale=1.0, partition_size=16,
                      workspace=None, max_partitions=1), **kw)
        with pytest.raises(ValueError):
            binding.paged_attention_decode_shared(**a)
