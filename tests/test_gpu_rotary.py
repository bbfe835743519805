"""Rotary positions on the GPU against the definition in extended precision."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"


def freq_of(R, base=10000.0):
    f = binding.rotary_frequencies(R, base)
    return f, binding.rotary_table(f, DEV)


def pairs(x, R, layout):
    return (x[..., :R // 2], x[..., R // 2:R]) if layout == 0 else (x[..., 0:R:2], x[..., 1:R:2])


def wanted(x, positions, f, R, layout, amplitude=1.0, inverse=False):
    """(rotated x, bound on the error before the last rounding), in numpy's long double."""
    x = x.detach().float().cpu().numpy().astype(np.longdouble)
    f = f.numpy().astype(np.longdouble)
    t = positions.cpu().numpy().astype(np.longdouble)[:, None] * f
    c, s = np.cos(t)[:, None] * amplitude, np.sin(t)[:, None] * amplitude * (-1 if inverse else 1)
    a, b = pairs(x, R, layout)
    y, err = x.copy(), np.zeros_like(x)
    ya, yb = pairs(y, R, layout)
    ya[...], yb[...] = a * c - b * s, b * c + a * s
    # angle: conversion of 32 bits to fp32, half an ulp of at most 1 half turn (2^-25 pi), the 32 bits dropped
    # (2^-32 2pi), and the table's frequency (two 64-bit roundings and the reference's pi) times the position
    pos = np.abs(positions.cpu().numpy().astype(np.longdouble))[:, None, None]
    angle = np.pi * 2.0 ** -25 + 2 * np.pi * 2.0 ** -32 + pos * 2.0 ** -50 * np.maximum(np.abs(f), 1e-30)
    # sincospi (1 ulp), the amplitude, the product and the sum: at most 2.5 ulp of fp32 on each term
    e = (angle + 2.5 * 2.0 ** -23) * abs(amplitude) * (np.abs(a) + np.abs(b))
    ea, eb = pairs(err, R, layout)
    ea[...], eb[...] = e, e
    return y, err


def check(got, x, positions, f, R, layout, **kw):
    y, err = wanted(x, positions, f, R, layout, **kw)
    half_step = torch.finfo(got.dtype).eps / 2
    bound = err + half_step * (np.abs(y) + err) + 1e-38
    d = np.abs(got.detach().float().cpu().numpy().astype(np.longdouble) - y)
    assert got.shape == x.shape and bool((d <= bound).all()), float((d / bound).max())
    assert torch.equal(got[..., R:], x[..., R:])                       # dims past R pass through bit for bit


def rows(T, H, D, dtype, gen, pad=0):
    """[T, H, D], as a slice of wider rows where pad > 0."""
    x = torch.randn(T, H * D + pad, generator=gen, device=DEV).to(DT[dtype])
    return x[:, :H * D].unflatten(1, (H, D)) if T else torch.empty(0, H, D, device=DEV, dtype=DT[dtype])


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype,D,R", [("bf16", 128, 128), ("bf16", 64, 64), ("bf16", 128, 32), ("bf16", 128, 96), ("bf16", 64, 2),
                                       ("bf16", 128, 50), ("fp32", 128, 128), ("fp32", 64, 16), ("fp32", 64, 8), ("fp32", 128, 126)])
@pytest.mark.parametrize("T", [1, 3, 259, 4099])
def test_rotary_both_layouts_types_and_partial_heads(layout, dtype, D, R, T):
    gen = torch.Generator(DEV).manual_seed(T + R)
    Hq, Hkv = (5, 3) if T < 1000 else (2, 1)
    q, k = rows(T, Hq, D, dtype, gen, pad=16), rows(T, Hkv, D, dtype, gen)
    pos = torch.randint(0, 200000, (T,), generator=gen, device=DEV, dtype=torch.int32)
    f, table = freq_of(R)
    q_out, k_out = torch.full((T, Hq, D), float("nan"), device=DEV, dtype=q.dtype), torch.empty_like(k)
    binding.rotary(q_out, q, pos, table, layout, k_out=k_out, k=k)
    check(q_out, q, pos, f, R, layout)
    check(k_out, k, pos, f, R, layout)
    # in place, bit for bit the same; q alone
    binding.rotary(q, q, pos, table, layout)
    assert torch.equal(q, q_out)
    assert binding.device_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rotary_positions_at_the_ends_of_their_range(dtype):
    gen = torch.Generator(DEV).manual_seed(0)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 20, 123456789], device=DEV, dtype=torch.int32)
    x = rows(pos.numel(), 2, 128, dtype, gen)
    f, table = freq_of(128)
    y = torch.empty_like(x)
    binding.rotary(y, x, pos, table, 0)
    check(y, x, pos, f, 128, 0)
    assert torch.equal(y[0], x[0])                                     # position 0: nothing moves


@pytest.mark.parametrize("scaling", ["linear", "ntk", "parts", "ramp"])
def test_rotary_scaled_frequencies_and_amplitude(scaling):
    gen = torch.Generator(DEV).manual_seed(1)
    f = binding.rotary_frequencies(128, 1e4, scaling, 8.0, 8192.0, 1.0, 32.0)
    pos = torch.randint(0, 65536, (33,), generator=gen, device=DEV, dtype=torch.int32)
    x = rows(33, 4, 128, "fp32", gen)
    y = torch.empty_like(x)
    binding.rotary(y, x, pos, binding.rotary_table(f, DEV), 1, amplitude=1.25)
    check(y, x, pos, f, 128, 1, amplitude=float(np.float32(1.25)))


@pytest.mark.parametrize("layout,R", [(0, 64), (1, 64), (0, 20), (1, 20)])
def test_inverse_is_the_gradient(layout, R):
    """<g, forward(x)> differentiated: by the formula, and by differences along random directions (the map is linear,
    so a difference over any step is the derivative up to rounding)."""
    gen = torch.Generator(DEV).manual_seed(2)
    T, H, D, amp = 37, 3, 64, 1.5
    f, table = freq_of(R)
    pos = torch.randint(0, 5000, (T,), generator=gen, device=DEV, dtype=torch.int32)
    x, g, e = (rows(T, H, D, "fp32", gen) for _ in range(3))
    dx = torch.empty_like(x)
    binding.rotary(dx, g, pos, table, layout, amplitude=amp, inverse=True)
    y, err = wanted(g, pos, f, R, layout, amplitude=amp, inverse=True)
    assert bool((np.abs(dx.cpu().numpy() - y) <= err + 2.0 ** -24 * (np.abs(y) + err) + 1e-38).all())
    up, down = torch.empty_like(x), torch.empty_like(x)
    binding.rotary(up, x + e, pos, table, layout, amplitude=amp)
    binding.rotary(down, x - e, pos, table, layout, amplitude=amp)
    by_difference = ((up.double() - down.double()) / 2 * g.double()).sum()
    by_gradient = (dx.double() * e.double()).sum()
    # every rotated value is within 4 * 2^-23 of its terms, of which there are T H D of size amp * (|x| + |e|) * |g|
    size = (amp * (x.abs() + e.abs()).double() * (g.abs().double() + 1)).sum()
    assert abs(by_difference - by_gradient) <= 8 * 2.0 ** -23 * size


def cache_of(blocks, Hkv, bs, D, dtype, gen):
    return tuple(torch.randn(blocks, Hkv, bs, D, generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype,Hq,Hkv,D,R,bs", [("bf16", 32, 8, 128, 128, 16), ("bf16", 8, 1, 64, 32, 32), ("bf16", 4, 4, 128, 22, 16),
                                                 ("fp32", 4, 2, 64, 64, 16), ("fp32", 3, 3, 128, 62, 32)])
@pytest.mark.parametrize("T,fused", [(1, False), (7, True), (70, False), (4100, True)])
def test_append_rotates_keys_on_the_way_and_copies_values(layout, dtype, Hq, Hkv, D, R, bs, T, fused):
    gen = torch.Generator(DEV).manual_seed(T)
    blocks = T // bs + 3
    kc, vc = cache_of(blocks, Hkv, bs, D, dtype, gen)
    if fused:
        x = torch.randn(T, (Hq + 2 * Hkv) * D, generator=gen, device=DEV).to(DT[dtype])
        q, k, v = (y.unflatten(1, (-1, D)) for y in x.split([Hq * D, Hkv * D, Hkv * D], 1))
    else:
        q, k, v = rows(T, Hq, D, dtype, gen), rows(T, Hkv, D, dtype, gen), rows(T, Hkv, D, dtype, gen)
    slots = torch.randperm(blocks * bs, generator=gen, device=DEV)[:T]
    if T > 4:
        slots[2] = -1                                                  # skipped tokens: nothing stored
        slots[T - 1] = blocks * bs
        slots[T - 2] = -(1 << 62)
    pos = torch.randint(0, 100000, (T,), generator=gen, device=DEV, dtype=torch.int32)
    f, table = freq_of(R)
    k_out = torch.empty(T, Hkv, D, device=DEV, dtype=k.dtype)
    q_out = torch.empty(T, Hq, D, device=DEV, dtype=k.dtype)
    kc0, vc0 = kc.clone(), vc.clone()
    binding.rotary_append(q_out, q, k, v, kc, vc, slots, pos, table, layout, k_out=k_out)
    check(q_out, q, pos, f, R, layout)
    check(k_out, k, pos, f, R, layout)
    live = (slots >= 0) & (slots < blocks * bs)
    page, off = slots[live] // bs, slots[live] % bs
    kc0[page, :, off], vc0[page, :, off] = k_out[live], v[live]
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)               # every other slot as it was
    # the same bits as rotating first and appending afterwards, and without queries or k_out
    kc1, vc1 = torch.zeros_like(kc), torch.zeros_like(vc)
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    binding.rotary_append(None, None, k, v, kc1, vc1, slots, pos, table, layout)
    slots2 = torch.where(live, slots, -1)
    binding.cache_append(k_out, v.contiguous(), kc2, vc2, slots2)
    assert torch.equal(kc1, kc2) and torch.equal(vc1, vc2)
    assert binding.device_status() == 0


def test_empty_calls_launch_nothing():
    _, table = freq_of(64)
    e = torch.empty(0, 4, 64, device=DEV)
    pos, slots = torch.empty(0, device=DEV, dtype=torch.int32), torch.empty(0, device=DEV, dtype=torch.int64)
    kc = torch.ones(2, 4, 16, 64, device=DEV)
    binding.rotary(e, e, pos, table, 0, k_out=e, k=e)
    binding.rotary_append(e, e, e, e, kc, kc.clone(), slots, pos, table, 0)
    torch.cuda.synchronize()
    assert bool((kc == 1).all())


def test_values_that_are_not_finite_stay_in_their_pairs_and_rows():
    _, table = freq_of(128)
    x = torch.ones(3, 2, 128, device=DEV, dtype=torch.bfloat16)
    x[1, 0, 5] = float("nan")
    x[1, 1, 70] = float("inf")
    pos = torch.tensor([3, 4, 5], device=DEV, dtype=torch.int32)
    y = torch.empty_like(x)
    binding.rotary(y, x, pos, table, 0)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, [5, 69]] = True
    want[1, 1, [6, 70]] = True
    assert torch.equal(bad, want)


def test_append_past_32_bit_offsets():
    """A pool of more than 2^31 elements per cache: the last slot lies where a 32-bit offset would wrap."""
    Hkv, bs, D = 8, 32, 128
    blocks = (1 << 31) // (Hkv * bs * D) + 3
    kc, vc = (torch.zeros(blocks, Hkv, bs, D, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    gen = torch.Generator(DEV).manual_seed(3)
    k, v = rows(2, Hkv, D, "bf16", gen), rows(2, Hkv, D, "bf16", gen)
    slots = torch.tensor([blocks * bs - 1, 0], device=DEV)
    pos = torch.tensor([9, 10], device=DEV, dtype=torch.int32)
    f, table = freq_of(128)
    binding.rotary_append(None, None, k, v, kc, vc, slots, pos, table, 0)
    check(kc[-1, :, -1][None], k[:1], pos[:1], f, 128, 0)
    assert torch.equal(vc[-1, :, -1], v[0]) and torch.equal(vc[0, :, 0], v[1])
    assert int((vc.view(blocks, -1) != 0).any(1).sum()) == 2           # two pages touched


def test_rotation_then_append_and_decode_on_another_stream_and_in_a_graph():
    """rotary_append -> decode on a side stream without synchronisation, and the same captured and replayed with new
    inputs in the same buffers: the same bits as with a synchronisation after every call."""
    gen = torch.Generator(DEV).manual_seed(4)
    B, Hq, Hkv, D, bs, n = 6, 8, 2, 64, 16, 75
    pages = -(-n // bs)
    kc, vc = cache_of(B * pages, Hkv, bs, D, "bf16", gen)
    bt = torch.arange(B * pages, device=DEV, dtype=torch.int32).view(B, pages)
    lens = torch.full((B,), n, device=DEV, dtype=torch.int32)
    slots = bt[:, -1].long() * bs + (n - 1) % bs
    pos = lens - 1
    _, table = freq_of(D)
    x = torch.randn(B, (Hq + 2 * Hkv) * D, generator=gen, device=DEV).bfloat16()
    q, k, v = (y.unflatten(1, (-1, D)) for y in x.split([Hq * D, Hkv * D, Hkv * D], 1))
    q_out = torch.empty(B, Hq, D, device=DEV, dtype=torch.bfloat16)
    out = torch.empty_like(q_out)

    def step(stream=None, sync=False):
        binding.rotary_append(q_out, q, k, v, kc, vc, slots, pos, table, 0, stream=stream)
        if sync:
            torch.cuda.synchronize()
        binding.paged_attention_decode(out, q_out, kc, vc, bt, lens, None, D ** -0.5, stream=stream)

    step(sync=True)
    torch.cuda.synchronize()
    first = out.clone()
    out.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        step(stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
    pos.sub_(3)
    graph.replay()
    torch.cuda.synchronize()
    replayed = out.clone()
    step(sync=True)
    torch.cuda.synchronize()
    assert torch.equal(out, replayed) and not torch.equal(out, first)
    assert binding.device_status() == 0
