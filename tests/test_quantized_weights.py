"""4-bit base weights: conversion, the routed linear and the decode step on them, against plain 64-bit forms.

Tolerances of the linears: the weights are exact in bf16, so what is left is the fp32 sums and one rounding to bf16:
|y - ref| <= 2^-8 |ref| + n 2^-24 S, n the length of the longest sum (d1 + rank + 16), S the sum of the magnitudes; rows above 128
take t as two bf16 halves (relative 2^-16 of the low-rank part, covered by 2^-16 S)."""
import ctypes

import pytest
import torch

import oracle
from paper_2410_18035_amd import binding as mb
from paper_2410_18035_amd import synth
from tests import plain
from tests.util import assert_rows_close, oracle_adapters

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------- host side
def test_plain_form_on_hand_worked_values():
    w = torch.zeros(2, 32)
    w[0, :10] = torch.tensor([6.0, 0.25, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, -5.5])
    w[1, 0], w[1, 1] = 7.9, -1.0  # largest in [4, 8): scale 1, 7.9 -> 6
    codes, scales = plain.quantize(w)
    assert scales.tolist() == [[127], [127]]
    assert codes[0, :10].tolist() == [7, 0, 8, 2, 2, 8 + 4, 4, 6, 6, 8 + 7]
    assert codes[1, :2].tolist() == [7, 8 + 2]
    back = plain.dequantize(plain.pack(codes, scales), 32, 2)
    assert back[0, :10].tolist() == [6.0, 0.0, 0.0, 1.0, 1.0, -2.0, 2.0, 4.0, 4.0, -6.0]


def test_sizes_and_refusals():
    L, n = mb.lib(), ctypes.c_void_p(None)
    p, off = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
    assert mb.quantized_weight_bytes(4096, 11008) == 4096 * 11008 * 17 // 32
    assert mb.quantized_weight_bytes(32, 1) == 17
    assert mb.quantized_weight_bytes(48, 16) == 0 and mb.quantized_weight_bytes(32, 0) == 0
    assert L.milora_quantize_weight(n, 0, p, 32, 16, n) == -1 and L.milora_quantize_weight(p, 0, n, 32, 16, n) == -1
    assert L.milora_quantize_weight(p, 2, p, 32, 16, n) == -1 and L.milora_quantize_weight(p, 0, p, 0, 16, n) == -1
    assert L.milora_quantize_weight(p, 0, p, 33, 16, n) == -3 and L.milora_quantize_weight(p, 0, off, 32, 16, n) == -3
    assert L.milora_dequantize_weight(n, p, 0, 32, 16, n) == -1 and L.milora_dequantize_weight(p, p, 5, 32, 16, n) == -1
    assert L.milora_dequantize_weight(p, p, 0, 31, 16, n) == -3 and L.milora_dequantize_weight(off, p, 0, 32, 16, n) == -3
    ad = mb._Adapters(1, 8, 0x1000, 0x1000, 0x1000)
    lin = lambda M, d1, d2, dt, x, w, ws, nb: L.milora_routed_linear(x, M, d1, d2, dt, p, w, 2, n, ctypes.byref(ad), 0, p, p, 1, p, ws, nb, n)
    big = 1 << 30
    assert lin(4, 32, 16, 1, p, p, p, big) == -3  # fp32 activations
    assert lin(4, 48, 16, 0, p, p, p, big) == -3 and lin(4, 32, 24, 0, p, p, p, big) == -3
    assert lin(4, 32, 16, 0, off, p, p, big) == -3 and lin(4, 32, 16, 0, p, off, p, big) == -3
    assert lin(4, 1 << 30, 16, 0, p, p, p, big) == -2
    assert lin(4, 32, 16, 0, p, p, n, 0) == -5 and lin(4, 32, 16, 0, p, p, p, 16) == -5
    assert L.milora_routed_linear(p, 4, 32, 16, 0, p, p, 3, n, ctypes.byref(ad), 0, p, p, 1, p, p, big, n) == -1  # no such layout
    lw = mb._LayerWeights()
    for m in range(7):
        lw.W[m] = 0x1000
    lw.layout = 2
    dec = lambda d, F, dt, x: L.milora_layer_decode(x, 4, d, F, dt, ctypes.byref(lw), ctypes.byref(ad), p, p, 0, n, p, n, p, big, n)
    assert dec(48, 64, 0, p) == -3 and dec(64, 48, 0, p) == -3 and dec(64, 64, 1, p) == -3 and dec(64, 64, 0, off) == -3
    assert L.milora_layer_decode_noalloc(p, 4, 64, 64, 0, ctypes.byref(lw), ctypes.byref(ad), p, p, 0, n, p, n, n) == -3
    slots = (ctypes.c_float * mb.PROFILE_SLOTS)()
    assert mb.quantized_linear_workspace_bytes(4, 1 << 30, 16, 8) == 0
    lw.layout = 3
    assert dec(64, 64, 0, p) == -1
    del slots


def test_kernel_family_and_workspace():
    k, t = mb.milora_routed_linear_kernel, mb.milora_routed_linear_tile
    bf = torch.bfloat16
    assert k(1, 4096, 4096, bf, mb.W_MX4) == mb.KERNEL_STREAM and t(1, 4096, 4096, bf, mb.W_MX4) == 0
    assert k(4000, 4096, 4096, bf, mb.W_MX4) == mb.KERNEL_TILES and t(32768, 4096, 11008, bf, mb.W_MX4) == 256
    assert t(32768, 4128, 11008, bf, mb.W_MX4) in (64, 128)  # no 256 x 256 kernel for a reduction that is no multiple of 64
    assert k(4, 48, 16, bf, mb.W_MX4) == -3 and k(4, 32, 16, torch.float32, mb.W_MX4) == -3
    size = mb.quantized_linear_workspace_bytes
    rows = [1, 16, 17, 32, 33, 64, 65, 127, 128, 129, 200, 300, 512, 513, 1000, 4096, 4097, 9000]
    for d1, d2, r in [(32, 16, 1), (4096, 4096, 32), (4128, 11008, 256), (11008, 4096, 5)]:
        sizes = [size(M, d1, d2, r) for M in rows]
        assert sizes == sorted(sizes) and sizes[0] > 0
        for M in rows:
            assert size(M, d1, d2, r) <= size(M, d1 + 32, d2, r) and size(M, d1, d2, r) <= size(M, d1, d2 + 16, r)
            assert size(M, d1, d2, r) <= size(M, d1, d2, r + 1)
    assert size(0, 32, 16, 1) == 0 and size(4, 32, 16, 0) == 0


def test_sizes_beyond_a_launch_are_refused_before_any_work():
    """What would be left for these is a kernel whose hand-over words a workspace of any contents does not hold, or no launch at all."""
    L, n, p = mb.lib(), ctypes.c_void_p(None), ctypes.c_void_p(0x1000)
    ad = mb._Adapters(1, 8, 0x1000, 0x1000, 0x1000)
    k, t = mb.milora_routed_linear_kernel, mb.milora_routed_linear_tile
    lin = lambda M, d1, d2: L.milora_routed_linear(p, M, d1, d2, 0, p, p, 2, n, ctypes.byref(ad), 0, p, p, 1, p, p, 1 << 60, n)
    for M, d1, d2 in [(600, 8388640, 16), (4096, 96, 4200000), (1, 32, 1 << 28), (128, 1 << 26, 16), (600, 8388608, 16), (1, 32, 2147483632),
                      (128, 32, 2147483632), (600, 32, 2147483632)]:
        assert lin(M, d1, d2) == -2, (M, d1, d2)
        assert k(M, d1, d2, torch.bfloat16, mb.W_MX4) == -2 and t(M, d1, d2, torch.bfloat16, mb.W_MX4) == -2
    assert k(4, 1 << 30, 16, torch.bfloat16, mb.W_MX4) == -2
    for M, d1, d2 in [(600, 8388512, 16), (4000, 96, 4190000), (1, 32, 1 << 26), (700, 48 * 2, 528)]:  # the last ones that fit keep their kernels
        assert k(M, d1, d2, torch.bfloat16, mb.W_MX4) == (mb.KERNEL_STREAM if M == 1 else mb.KERNEL_TILES)
        assert t(M, d1, d2, torch.bfloat16, mb.W_MX4) == 0 if M == 1 else t(M, d1, d2, torch.bfloat16, mb.W_MX4) in (64, 128)
    # whatever a call is told about its kernel, it is never the streaming one on a weight written out
    for M in (129, 513, 600, 4096, 5000, 100000):
        for d1 in (32, 96, 4128, 8388576, 8388640):
            for d2 in (16, 4096, 4194304, 4200000):
                if k(M, d1, d2, torch.bfloat16, mb.W_MX4) == mb.KERNEL_TILES:
                    assert t(M, d1, d2, torch.bfloat16, mb.W_MX4) in (64, 128)
    lw = mb._LayerWeights()
    for m in range(7):
        lw.W[m] = 0x1000
    lw.layout = 2
    assert L.milora_layer_decode(p, 1, 32, 1 << 29, 0, ctypes.byref(lw), ctypes.byref(ad), p, p, 0, n, p, n, p, 1 << 60, n) == -2


def test_binding_checks_quantised_weights():
    with pytest.raises(ValueError):
        mb._check_weight(torch.zeros(16, dtype=torch.uint8), 32, 1, mb.W_MX4, torch.bfloat16)
    with pytest.raises(ValueError):
        mb._check_weight(torch.zeros(17, dtype=torch.int8), 32, 1, mb.W_MX4, torch.bfloat16)
    mb._check_weight(torch.zeros(17, dtype=torch.uint8), 32, 1, mb.W_MX4, torch.bfloat16)


# ---------------------------------------------------------------------------------------------------- conversion
def _same_weight(w):
    d2, d1 = w.shape
    q = mb.milora_quantize_weight(w)
    codes, scales = plain.quantize(w)
    ref = plain.dequantize(plain.pack(codes, scales), d1, d2)
    assert torch.equal(q[d1 * d2 // 2:].cpu().reshape(scales.shape), scales)
    for dt in (torch.bfloat16, torch.float32):
        back = mb.milora_dequantize_weight(q, d1, d2, dt).cpu()
        assert back.dtype == dt and torch.equal(torch.isnan(back), torch.isnan(ref))
        ok = ~torch.isnan(ref)
        assert torch.equal(back[ok].double(), ref[ok])
    return q


@gpu
def test_quantize_every_bf16_value():
    """Each of the 65536 bit patterns, beside a value that sets the group's scale to its own, the next or far larger."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    _same_weight(bits.reshape(-1, 32).to(DEV))  # neighbours share a group
    for factor in (1.0, 3.0, 37.0):
        w = torch.zeros(4096, 16, 32, dtype=torch.bfloat16)
        w[..., 5] = bits.reshape(4096, 16)
        w[..., 17] = (bits.float() * factor).to(torch.bfloat16).reshape(4096, 16)
        _same_weight(w.reshape(4096, -1).to(DEV))


@gpu
@pytest.mark.parametrize("d1,d2,dtype", [(32, 1, torch.float32), (32, 3, torch.bfloat16), (96, 37, torch.float32), (1056, 129, torch.bfloat16),
                                         (4096, 40, torch.float32)])
def test_quantize_shapes(d1, d2, dtype):
    g = torch.Generator().manual_seed(d1 + d2)
    w = torch.randn(d2, d1, generator=g) * torch.exp2(torch.randint(-20, 20, (d2, 1), generator=g).float())
    w[0, :4] = torch.tensor([0.0, -0.0, 1e-42, -1e-30])
    q = _same_weight(w.to(dtype).to(DEV))
    again = mb.milora_quantize_weight(mb.milora_dequantize_weight(q, d1, d2, dtype))
    assert torch.equal(mb.milora_dequantize_weight(again, d1, d2, dtype), mb.milora_dequantize_weight(q, d1, d2, dtype))


@gpu
def test_quantize_fp32_next_to_the_borders():
    """The borders between codes and their fp32 neighbours, for a scale of 1 and a far one."""
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    v = torch.stack([mid, torch.nextafter(mid, mid * 0), torch.nextafter(mid, mid * 9)]).reshape(-1)
    w = torch.zeros(2, 32)
    w[0, :21], w[1, :21] = v, -v
    w[:, 31] = 4.0
    _same_weight(torch.cat([w, w * 2.0 ** -100, w * 2.0 ** 120]).to(DEV))


@gpu
def test_quantize_nonfinite_extreme_and_unaligned():
    g = torch.Generator().manual_seed(3)
    w = torch.randn(6, 64, generator=g)
    w[1, 3], w[2, 40], w[3, 63] = float("inf"), float("-inf"), float("nan")
    w[4] *= 1e-38
    w[5] = torch.finfo(torch.float32).max
    _same_weight(w.to(DEV))
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.randn(1 + 7 * 96, generator=g).to(dtype).to(DEV)
        _same_weight(flat[1:].reshape(7, 96))  # one element past a 16-byte boundary


@gpu
def test_dequantize_takes_every_scale():
    d1, d2 = 32, 256
    codes = torch.arange(16, dtype=torch.uint8).repeat(d2, 2)
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8).reshape(d2, 1)
    q = plain.pack(codes, scales)
    ref = plain.dequantize(q, d1, d2)
    got = mb.milora_dequantize_weight(q.to(DEV), d1, d2, torch.float32).cpu()
    want = torch.where(ref.abs() > 3.4e38, torch.sign(ref) * float("inf"), ref).float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[:255], want[:255])


# ---------------------------------------------------------------------------------------------------- the routed linear
def _assert_linear(Y, x, Wd, c, site, bias=None):
    ten = c.tenants(site)
    ref = plain.linear(x, Wd, c.A[site], c.Bm[site], ten, bias)
    size = plain.linear_size(x, Wd, c.A[site], c.Bm[site], ten, bias)
    n = x.shape[1] + max(c.rank) + 16
    tol = ref.abs() * 2.0 ** -8 + size * (n * 2.0 ** -24 + (2.0 ** -16 if x.shape[0] > 128 else 0.0))
    far = (Y.cpu().double() - ref).abs()
    assert torch.isfinite(Y).all() and (far <= tol).all(), float((far / tol.clamp(min=1e-300)).max())
    return ref


@gpu
@pytest.mark.parametrize("M,d1,d2,rows", [
    (1, 32, 16, "own"), (1, 4096, 64, "own"), (2, 96, 48, "mixed"), (3, 160, 1040, "mixed"), (15, 128, 16, "mixed"), (16, 1056, 80, "sorted"),
    (17, 64, 32, "mixed"), (31, 2080, 208, "own"), (32, 11008, 32, "mixed"), (33, 96, 48, "own"), (100, 224, 272, "mixed"), (128, 512, 2064, "own"),
    (129, 96, 48, "mixed"), (129, 512, 272, "sorted"), (300, 192, 528, "mixed"), (700, 1056, 304, "mixed"), (1100, 512, 1040, "sorted"), (40, 64, 64, "none")])
@pytest.mark.parametrize("ranks", [(8,), (5, 33, 256), (1, 16)])
def test_linear(M, d1, d2, rows, ranks):
    if rows == "own":
        B = M
    else:
        B = min(M, 7)
    site = (M + d1) % 7
    c = plain.Case(M, B, 3, {site: (d1, d2)}, ranks, M * 31 + d1, DEV, rows=rows, sites=[site])
    x, bias = c.rnd(M, d1), c.rnd(d2) if M % 2 else None
    q = mb.milora_quantize_weight(c.rnd(d2, d1, s=d1 ** -0.5))
    tid, route = c.requests()
    guard = torch.full((M + 2, d2), 7.0, dtype=torch.bfloat16, device=DEV)
    Y = mb.milora_routed_linear(x, q, c.tab, site, tid, route, row_to_req=c.rows(), bias=bias, w_layout=mb.W_MX4, d2=d2, out=guard[:M])
    assert (guard[M:] == 7.0).all()
    _assert_linear(Y, x, plain.dequantize(q, d1, d2), c, site, bias)


@gpu
@pytest.mark.parametrize("M,d1,d2,rows", [(2100, 512, 4112, "mixed"), (2049, 640, 4096, "sorted"), (2304, 1152, 4208, "sorted"), (1800, 4224, 2064, "mixed"),
                                           (1800, 4224, 8080, "mixed"), (800, 8320, 2064, "mixed"), (2100, 4352, 8208, "sorted")])
@pytest.mark.parametrize("ranks", [(8,), (5, 33, 256)])
def test_linear_in_large_tiles(M, d1, d2, rows, ranks):
    """256 x 256 tiles read the codes: reductions of one to several groups of scales, the last one not whole; tiles cut along the reduction, all of
    them or those behind full turns."""
    test_linear(M, d1, d2, rows, ranks)


@gpu
@pytest.mark.parametrize("d1", [640, 4224])
def test_large_tiles_keep_nans_where_they_belong(d1):
    M, d2, site = 2100, 4112, 1
    c = plain.Case(M, 4, 3, {site: (d1, d2)}, (8, 40, 16), 53, DEV, rows="mixed", sites=[site])
    c.tid[:] = torch.tensor([0, 1, 2, 1])
    x, w = c.rnd(M, d1), c.rnd(d2, d1)
    tid, route = c.requests()
    run = lambda x, w: mb.milora_routed_linear(x, mb.milora_quantize_weight(w), c.tab, site, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4, d2=d2)
    clean = run(x, w)
    assert torch.isfinite(clean).all()
    w2 = w.clone()
    w2[d2 - 1, 600] = w2[130, 0] = float("nan")
    Y = run(x, w2)
    keep = torch.ones(d2, dtype=torch.bool, device=DEV)
    keep[[130, d2 - 1]] = False
    assert torch.equal(Y[:, keep], clean[:, keep]) and torch.isnan(Y[:, ~keep]).all()
    x2 = x.clone()
    x2[M - 1, d1 - 1] = x2[300, 32] = float("inf")
    Y = run(x2, w)
    keep = torch.ones(M, dtype=torch.bool, device=DEV)
    keep[[300, M - 1]] = False
    assert torch.equal(Y[keep], clean[keep]) and not torch.isfinite(Y[~keep]).all(dim=1).any()
    c.Bm[site][0][3, 7] = float("inf")
    Y = run(x, w)
    mine = (torch.tensor(c.tenants(site)) == 0).to(DEV)
    assert mine.any() and torch.equal(Y[~mine], clean[~mine]) and not torch.isfinite(Y[mine][:, 7]).any()


@gpu
@pytest.mark.parametrize("M", [5, 40, 200])
def test_linear_keeps_infinities_and_nans_where_they_belong(M):
    """A NaN group stays in its column, an Inf of X in its row, a tenant's Inf in its rows."""
    d1, d2, site = 192, 80, 2
    c = plain.Case(M, 4, 3, {site: (d1, d2)}, (8,), 50 + M, DEV, rows="mixed", sites=[site])
    c.tid[:] = torch.tensor([0, 1, 2, 1])
    c.r2r[:4] = torch.tensor([0, 1, 2, -1])
    x, w = c.rnd(M, d1), c.rnd(d2, d1)
    tid, route = c.requests()
    run = lambda x, w: mb.milora_routed_linear(x, mb.milora_quantize_weight(w), c.tab, site, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4, d2=d2)
    clean = run(x, w)
    assert torch.isfinite(clean).all()
    w2 = w.clone()
    w2[33, 100] = float("nan")
    Y = run(x, w2)
    keep = torch.arange(d2, device=DEV) != 33
    assert torch.equal(Y[:, keep], clean[:, keep]) and torch.isnan(Y[:, 33]).all()
    x2 = x.clone()
    x2[1, 191] = float("inf")
    Y = run(x2, w)
    keep = torch.arange(M, device=DEV) != 1
    assert torch.equal(Y[keep], clean[keep]) and not torch.isfinite(Y[1]).all()
    ten = torch.tensor(c.tenants(site))
    c.Bm[site][0][3, 7] = float("inf")
    Y = run(x, w).cpu()
    mine = ten == 0
    assert torch.equal(Y[~mine], clean.cpu()[~mine]) and not torch.isfinite(Y[mine][:, 7]).any()
    assert torch.equal(Y[mine][:, 8:], clean.cpu()[mine][:, 8:])


@gpu
def test_linear_skips_foreign_ids():
    """Rows whose request, tenant or rank is out of range get the base term only."""
    M, d1, d2, site = 24, 128, 48, 3
    c = plain.Case(M, 6, 3, {site: (d1, d2)}, (8, 16, 8), 8, DEV, rows="mixed", sites=[site], r_max=8)
    c.tid[:] = torch.tensor([0, -1, 3, 1, 2, 1 << 30])
    c.route[:] = torch.tensor([site, site, site, site, 255, site])
    c.r2r[:] = torch.tensor([0, 1, 2, 3, 4, 5, 6, -1] * 3)
    assert c.tenants(site) == [0, -1, -1, -1, -1, -1, -1, -1] * 3
    x, q = c.rnd(M, d1), mb.milora_quantize_weight(c.rnd(d2, d1))
    tid, route = c.requests()
    Y = mb.milora_routed_linear(x, q, c.tab, site, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4, d2=d2)
    _assert_linear(Y, x, plain.dequantize(q, d1, d2), c, site)


@gpu
def test_packed_and_quantised_calls_share_a_workspace():
    """The stream kernel's hand-over words stay as they are over calls on 4-bit weights of every kind."""
    M, d1, d2, site = 8, 128, 64, 2
    c = plain.Case(M, 4, 2, {site: (d1, d2)}, (8, 16), 91, DEV, rows="mixed", sites=[site])
    x, w = c.rnd(M, d1), c.rnd(d2, d1)
    wp, (tid, route), r2r = mb.milora_pack_weight(w), c.requests(), c.rows()
    others = [(3, 96, 48), (129, 96, 48), (700, 96, 528), (1100, 512, 1040), (2100, 640, 4112)]
    need = [mb.routed_linear_workspace_bytes(M, d1, d2, 16)] + [mb.quantized_linear_workspace_bytes(m, a, b, 16) for m, a, b in others]
    ws = torch.zeros(max(need), dtype=torch.uint8, device=DEV)
    packed = lambda: mb.milora_routed_linear(x, wp, c.tab, site, tid, route, row_to_req=r2r, w_layout=mb.W_PACKED, d2=d2, workspace=ws)
    first = packed()
    words = ws[:16384].clone()
    for m, a, b in others:
        o = plain.Case(m, 4, 2, {site: (a, b)}, (8, 16), m, DEV, rows="mixed", sites=[site])
        xo, q, ids = o.rnd(m, a), mb.milora_quantize_weight(o.rnd(b, a, s=a ** -0.5)), o.requests()
        Y = mb.milora_routed_linear(xo, q, o.tab, site, *ids, row_to_req=o.rows(), w_layout=mb.W_MX4, d2=b, workspace=ws)
        _assert_linear(Y, xo, plain.dequantize(q, a, b), o, site)
        assert torch.equal(ws[:16384], words), (m, a, b)
    assert torch.equal(packed(), first)
    assert mb.milora_packed_workspace_status(ws) == 0


@gpu
@pytest.mark.parametrize("M", [3, 64, 200])
def test_linear_in_a_graph_and_on_another_stream(M):
    d1, d2, site = 256, 96, 5
    c = plain.Case(M, 4, 2, {site: (d1, d2)}, (16,), 70 + M, DEV, rows="mixed", sites=[site])
    x, q = c.rnd(M, d1), mb.milora_quantize_weight(c.rnd(d2, d1))
    tid, route, r2r = *c.requests(), c.rows()
    ws = torch.full((mb.quantized_linear_workspace_bytes(M, d1, d2, c.tab.r_max),), 255, dtype=torch.uint8, device=DEV)  # any contents
    out = torch.empty(M, d2, dtype=torch.bfloat16, device=DEV)
    call = lambda: mb.milora_routed_linear(x, q, c.tab, site, tid, route, row_to_req=r2r, w_layout=mb.W_MX4, d2=d2, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = call().clone()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        x.copy_(c.rnd(M, d1))
        out.zero_()
        graph.replay()
        got = out.clone()
        ws.fill_(255)
        assert torch.equal(call(), got)
        torch.cuda.synchronize()
    _assert_linear(out, x, plain.dequantize(q, d1, d2), c, site)
    assert not torch.equal(first, out)


# ---------------------------------------------------------------------------------------------------- the decode step
@gpu
@pytest.mark.parametrize("B,d,F,ranks,norm,attn", [(1, 64, 96, (8,), False, False), (7, 256, 704, (5, 16), True, False), (16, 512, 1056, (8,), True, True),
                                                   (17, 96, 160, (4,), False, True), (33, 256, 352, (32, 8), True, False), (128, 256, 704, (64,), False, False)])
def test_layer_decode(B, d, F, ranks, norm, attn):
    """Against the oracle on the bf16 numbers that the codes stand for; the oracle's own rounding points and tolerance."""
    wl = synth.Workload("mx4", "bf16", d, F, 1, max(1, B // 2), B, ranks, (4, 8), tenants="uniform", seed=B, sigma_w=0.05, sigma_lora=0.15)
    q = [mb.milora_quantize_weight(w) for w in synth.base_weights(wl, 0, DEV)]
    W = [mb.milora_dequantize_weight(w, *synth.site_dims(m, d, F)) for m, w in enumerate(q)]
    ad = synth.adapters(wl, 0, DEV)
    tab = mb.AdapterTable.from_tensors(ad.A, ad.B, ad.rank)
    tid = synth.tenant_ids(wl)
    g = torch.Generator().manual_seed(B)
    route = torch.randint(0, 7, (B,), generator=g).to(torch.uint8)
    route[0] = mb.ROUTE_SET | 0b1110111
    x = synth.decode_input(wl, 0, DEV)
    a = synth.decode_input(wl, 1, DEV) if attn else None
    ws = torch.full((mb.layer_decode_workspace_bytes(B, d, F, tab.r_max),), 255, dtype=torch.uint8, device=DEV)
    y, qkv = mb.milora_layer_decode(x, q, tab, tid.to(DEV), route.to(DEV), F, w_layout=mb.W_MX4, rmsnorm=norm, attn_out=a, workspace=ws)
    y_ref, qkv_ref = oracle.layer_decode(synth.as_numpy(x), [synth.as_numpy(w) for w in W], oracle_adapters(ad), tid.numpy(), route.numpy(), F,
                                         flags=oracle.FLAG_RMSNORM if norm else 0, attn_out=None if a is None else synth.as_numpy(a))
    assert_rows_close(y, y_ref, torch.bfloat16, "y")
    assert_rows_close(qkv, qkv_ref, torch.bfloat16, "qkv")
    again, _ = mb.milora_layer_decode(x, q, tab, tid.to(DEV), route.to(DEV), F, w_layout=mb.W_MX4, rmsnorm=norm, attn_out=a, want_qkv=False,
                                      y=x, workspace=ws)  # y may alias x
    assert torch.equal(again, y)


@gpu
@pytest.mark.parametrize("B,d,F", [(1, 2080, 1056), (3, 4128, 352), (8, 2080, 352), (8, 4128, 1056), (9, 4128, 352), (1, 4128, 96), (33, 2080, 352)])
@pytest.mark.parametrize("norm", [False, True])
def test_layer_decode_of_real_width(B, d, F, norm):
    """Several parts of every level's reduction, several trips of the sums of squares."""
    test_layer_decode(B, d, F, (8, 20), norm, B == 8)


def _remainder_layer(B, d, F, seed, sites):
    """A layer whose gate and up projections see only what bf16 cannot hold of h: h is 1 + e with |e| < 2^-9, and inputs 2 k and 2 k + 1 have
    opposite weights (in the adapters too), so that all ones cancel, exactly in the base weights, whose values are small multiples of a power
    of two."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    pairs = lambda w: torch.stack([w, -w], -1).reshape(w.shape[0], -1)
    W = [rnd(d, d) * 0.02 for _ in range(4)] + [pairs(rnd(F, d // 2)) * 64 for _ in range(2)] + [rnd(d, F)]
    q = [mb.milora_quantize_weight(w.to(DEV)) for w in W]
    W = [mb.milora_dequantize_weight(v, *synth.site_dims(m, d, F), torch.float32).double() for m, v in enumerate(q)]
    x = torch.ones(B, d, dtype=torch.bfloat16, device=DEV)
    a = rnd(B, d).to(torch.bfloat16).to(DEV)
    a = (a.double() * 2.0 ** torch.floor(torch.log2(2.0 ** -9 / (a.double() @ W[3].t()).abs().max())).item()).to(torch.bfloat16)
    r, T = 8, 2
    A = [[(pairs(rnd(r, d // 2)).t() * 64 if m in (4, 5) else rnd(synth.site_dims(m, d, F)[0], r)).contiguous().to(torch.bfloat16).to(DEV) for m in range(7)]
         for _ in range(T)]
    Bm = [[(rnd(r, synth.site_dims(m, d, F)[1]) * 0.5).to(torch.bfloat16).to(DEV) for m in range(7)] for _ in range(T)]
    tid = torch.arange(B) % T
    route = torch.full((B,), 0x80 | sum(1 << s for s in sites) if sites else mb.ROUTE_NONE, dtype=torch.uint8)
    return q, W, x, a, A, Bm, tid.to(torch.int32).to(DEV), route.to(DEV)


def _remainder_step(B, d, F, norm, sites):
    q, W, x, a, A, Bm, tid, route = _remainder_layer(B, d, F, B + d, sites)
    tab = mb.AdapterTable.from_tensors(A, Bm, [8] * len(A))
    ws = torch.full((mb.layer_decode_workspace_bytes(B, d, F, 8),), 255, dtype=torch.uint8, device=DEV)
    y, _ = mb.milora_layer_decode(x, q, tab, tid, route, F, w_layout=mb.W_MX4, rmsnorm=norm, attn_out=a, want_qkv=False, workspace=ws)
    e = a.double() @ W[3].t()
    assert e.abs().max() <= 2.0 ** -9
    h = 1 + e
    n = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-5) if norm else h
    z = []
    for s in (4, 5):
        term = torch.stack([(n[b] @ A[int(tid[b])][s].double()) @ Bm[int(tid[b])][s].double() for b in range(B)])
        z.append(n @ W[s].t() + (term if s in sites else 0.0))
    ref = h + plain.gated(*z) @ W[6].t()
    # Independent roundings, each uniform and at most 2^-8 of its value, 2^-8 / sqrt(3) = 2.26e-3 of a norm: the second row of h in g (silu's
    # logarithmic slope: up to 2) and in u, m, y: sqrt(4 + 1 + 1 + 1) 2.26e-3 = 6e-3, 7e-3 with the sums.  Without the second rows z is
    # zero and y is h, at least a tenth of the norm away: that shows.
    assert (ref - h).norm() > 0.1 * ref.norm()
    far = (y.double() - ref).norm(dim=1) / ref.norm(dim=1)
    assert far.max() <= 7e-3, far.tolist()


@gpu
@pytest.mark.parametrize("B,d,F", [(1, 128, 96), (1, 4128, 352), (3, 2080, 352), (4, 4128, 1056), (8, 4128, 352), (8, 4128, 3104)])
@pytest.mark.parametrize("norm", [False, True])
def test_layer_decode_takes_h_beyond_its_first_bf16(B, d, F, norm):
    _remainder_step(B, d, F, norm, ())


@gpu
@pytest.mark.parametrize("B,d,F,sites", [(1, 4128, 352, (4,)), (3, 2080, 352, (5,)), (8, 4128, 1056, (4, 5)), (5, 1056, 352, (4, 5))])
@pytest.mark.parametrize("norm", [False, True])
def test_low_rank_terms_take_h_beyond_its_first_bf16(B, d, F, sites, norm):
    _remainder_step(B, d, F, norm, sites)


@gpu
@pytest.mark.parametrize("B", [2, 8, 9])
def test_an_infinite_input_stays_infinite_through_a_step(B):
    """h + Inf W is Inf where the weights say so: request 1 has an Inf, all weights it meets are positive."""
    d, F = 128, 96
    g = torch.Generator().manual_seed(B)
    W = [torch.rand(*synth.site_dims(m, d, F)[::-1], generator=g) + 0.5 for m in range(7)]
    q = [mb.milora_quantize_weight(w.to(DEV)) for w in W]
    A = [[torch.zeros(synth.site_dims(m, d, F)[0], 8, dtype=torch.bfloat16, device=DEV) for m in range(7)]]
    Bm = [[torch.zeros(8, synth.site_dims(m, d, F)[1], dtype=torch.bfloat16, device=DEV) for m in range(7)]]
    tab = mb.AdapterTable.from_tensors(A, Bm, [8])
    x, a = (torch.rand(B, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    tid, route = torch.zeros(B, dtype=torch.int32, device=DEV), torch.full((B,), 255, dtype=torch.uint8, device=DEV)
    run = lambda: mb.milora_layer_decode(x, q, tab, tid, route, F, w_layout=mb.W_MX4, attn_out=a)
    clean, qkv = run()
    assert torch.isfinite(clean).all()
    x[1, 70] = float("inf")
    y, qkv2 = run()
    keep = torch.arange(B, device=DEV) != 1
    assert torch.equal(y[keep], clean[keep]) and torch.equal(qkv2[keep], qkv[keep])
    assert (y[1] == float("inf")).all() and (qkv2[1] == float("inf")).all()


@gpu
@pytest.mark.parametrize("layout,M,d1,d2", [(mb.W_MX4, 5, 192, 80), (mb.W_MX4, 200, 192, 80), (mb.W_MX4, 700, 1056, 304), (mb.W_MX4, 2100, 640, 4112),
                                            (mb.W_ROWMAJOR, 20, 192, 80), (mb.W_ROWMAJOR, 200, 192, 80), (mb.W_ROWMAJOR, 2100, 640, 4112), (mb.W_PACKED, 8, 192, 80),
                                            (mb.W_PACKED, 200, 192, 80)])
def test_linear_keeps_an_infinite_scale_infinite(layout, M, d1, d2):
    site = 2
    c = plain.Case(M, 4, 3, {site: (d1, d2)}, (8, 40), 50 + M, DEV, rows="mixed", sites=[site])
    c.route[:] = site
    c.tid[:] = torch.tensor([0, 1, 2, 1])
    x, w = c.rnd(M, d1), c.rnd(d2, d1)
    w = mb.milora_quantize_weight(w) if layout == mb.W_MX4 else mb.milora_pack_weight(w) if layout == mb.W_PACKED else w
    tid, route = c.requests()
    run = lambda: mb.milora_routed_linear(x, w, c.tab, site, tid, route, row_to_req=c.rows(), w_layout=layout, d2=d2)
    clean = run()
    c.A[site][1][3, 33] = float("inf")
    assert (x[:, 3] != 0).all() and (c.Bm[site][1][33] != 0).all()
    Y = run()
    mine = (torch.tensor(c.tenants(site)) == 1).to(DEV)
    assert mine.any() and torch.equal(Y[~mine], clean[~mine])
    want = torch.sign(x[mine, 3].float())[:, None] * torch.sign(c.Bm[site][1][33].float()) * float("inf")
    assert torch.equal(Y[mine].float(), want)


@gpu
@pytest.mark.parametrize("B,d,F,sites", [(9, 2080, 352, ()), (16, 4128, 352, (4,)), (17, 1056, 96, (4, 5)), (32, 4128, 352, ()), (33, 2080, 352, (5,)), (64, 128, 96, ()),
                                         (100, 1056, 3104, (4, 5)), (128, 2080, 352, (4, 5))])
@pytest.mark.parametrize("norm", [False, True])
def test_larger_batches_take_h_beyond_its_first_bf16(B, d, F, sites, norm):
    """The precision of a request does not go by the batch that it is in."""
    _remainder_step(B, d, F, norm, sites)
