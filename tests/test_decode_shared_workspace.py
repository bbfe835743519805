"""Host side of the shared-prefix decode: one workspace serves every smaller call (no GPU needed)."""
import pytest

from paper_2505_02351_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


@pytest.mark.parametrize("Hq,Hkv,D", [(64, 8, 64), (64, 8, 128), (32, 8, 128), (32, 4, 128), (8, 8, 64), (8, 1, 128), (16, 8, 64)])
def test_workspace_never_shrinks_as_the_batch_grows(lib, Hq, Hkv, D):
    """A program allocates for its longest contexts, largest batch and most groups, and calls with less: the size a call asks
    for does not fall as any of them grows, across the bound up to which contexts are read for themselves (32 MB)."""
    size = binding.shared_workspace_bytes
    most = int(32e6 / (16 * Hkv * D * 4))                                       # B * max_partitions at that bound
    counts = sorted({1, 2, 3, 5, 61, 62, 122, 123, 124, 1000, 65535} | {min(max(1, most // b + d), 65535) for b in (1, 2, 4, 8, 9, 33, 300)
                                                                      for d in (-1, 0, 1, 2)})
    for B in (1, 2, 4, 8, 9, 33, 300, 4000):
        for N in (1, 12):
            sizes = [size(B, Hq, Hkv, D, N, P) for P in counts]
            assert sizes[0] > 0 and sizes == sorted(sizes), (B, N)
    batches = sorted({1, 2, 3, 7, 8, 9, 31, 32, 33, 100, 1000, 4000, 65535} | {min(max(1, most // p + d), 65535) for p in (1, 2, 4, 20) for d in (-1, 0, 1)})
    for P in (1, 2, 4, 20, 123):
        sizes = [size(B, Hq, Hkv, D, 3, P) for B in batches]
        assert sizes[0] > 0 and sizes == sorted(sizes), P
    assert [size(8, Hq, Hkv, D, N, 9) for N in range(1, 513)] == sorted(size(8, Hq, Hkv, D, N, 9) for N in range(1, 513))
