"""The gated block and its backward pass against plain 64-bit forms.

Tolerances, element by element.  Forward: g and u are off by E = n 2^-24 S + h S (n: terms of the longest sum, S: the sum of magnitudes,
h = 2^-16 where t enters as two bf16 halves), silu's slope is below 1.1 and the exponential good to 2^-20:
|y - ref| <= |u| 1.1 Eg + |silu(g)| Eu + Eg Eu + (eps/2 + 2^-20) |y|.
Backward: dz carries one rounding to the type (eps/2) and what g and u were off, so every product of it is off by as much of its
size; the result's own rounding comes on top: |v - ref| <= c S + eps/2 |ref|, c = eps/2 + n 2^-24 + 2^-12 (fp32: 2^-18, no halves there).
bf16 results are also held to a relative 2-norm: two independent roundings of at most eps/2 each, uniform: sqrt(2) 2^-8 / sqrt(3) = 3.2e-3; 4e-3
leaves room for the sums."""
import ctypes

import pytest
import torch

from paper_2410_18035_amd import binding as mb
from tests import plain

DEV = "cuda:0"
gpu = pytest.mark.gpu
F64 = torch.float64


# ---------------------------------------------------------------------------------------------------- host side
def test_refusals():
    L, n = mb.lib(), ctypes.c_void_p(None)
    p, off, big = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), 1 << 40
    ad, far = mb._Adapters(1, 8, 0x1000, 0x1000, 0x1000), mb._Adapters(1, 300, 0x1000, 0x1000, 0x1000)
    gr = mb._Gradients(0x1000, 0x1000)

    def both(want, M=4, d=64, F=64, dt=0, r2r=p, X=p, Wg=p, Wu=p, lay=0, a=ad, tid=p, route=p, B=2, Y=p, ws=p, nb=big):
        fwd = L.milora_gated_linear(X, M, d, F, dt, r2r, Wg, Wu, lay, ctypes.byref(a), tid, route, B, Y, n, n, ws, nb, n)
        bwd = L.milora_gated_linear_backward(p, X, p, p, M, d, F, dt, r2r, Wg, Wu, lay, ctypes.byref(a), tid, route, B, Y or n,
                                             ctypes.byref(gr), ws, nb, n)
        assert fwd == want, fwd
        assert bwd == want, bwd

    for kw in (dict(M=0), dict(d=0), dict(F=0), dict(B=0), dict(dt=2), dict(lay=3), dict(X=n), dict(Wg=n), dict(Wu=n), dict(tid=n), dict(route=n),
               dict(r2r=n), dict(a=mb._Adapters(1, 8, 0, 0x1000, 0x1000)), dict(a=mb._Adapters(0, 8, 0x1000, 0x1000, 0x1000))):
        both(-1, **kw)
    both(-2, a=far)
    both(-2, F=1 << 30)
    both(-2, d=1 << 30)
    for kw in (dict(lay=1), dict(lay=2, dt=1), dict(lay=2, d=48), dict(lay=2, F=40), dict(lay=2, Wg=off), dict(lay=2, Wu=off)):
        both(-3, **kw)
    both(-5, ws=n)
    both(-5, nb=16)
    args = lambda dY=p, g=p, u=p: (dY, p, g, u, 4, 64, 64, 0, p, p, p, 0, ctypes.byref(ad), p, p, 2, p, None, p, big, n)
    for kw in (dict(dY=n), dict(g=n), dict(u=n)):
        assert L.milora_gated_linear_backward(*args(**kw)) == -1
    assert L.milora_gated_linear(p, 4, 64, 64, 0, p, p, p, 0, ctypes.byref(ad), p, p, 2, n, n, n, p, big, n) == -1
    assert L.milora_gated_linear(off, 4, 64, 64, 0, p, p, p, 2, ctypes.byref(ad), p, p, 2, p, n, n, p, big, n) == -3
    many = mb._Adapters(32768, 8, 0x1000, 0x1000, 0x1000)
    assert L.milora_gated_linear_backward(p, p, p, p, 4, 64, 64, 0, p, p, p, 0, ctypes.byref(many), p, p, 2, p, None, p, big, n) == -2


def test_sizes_beyond_a_launch_are_refused_before_any_work():
    """On a machine without a GPU anything that is enqueued comes back as a failed HIP call."""
    L, n, p, huge = mb.lib(), ctypes.c_void_p(None), ctypes.c_void_p(0x1000), 1 << 60
    ad, many = (mb._Adapters(t, 8, 0x1000, 0x1000, 0x1000) for t in (1, 32768))
    fwd = lambda M, d, F, lay, dt=0: L.milora_gated_linear(p, M, d, F, dt, p, p, p, lay, ctypes.byref(ad), p, p, 2, p, n, n, p, huge, n)
    bwd = lambda M, d, F, lay, dt=0, a=ad: L.milora_gated_linear_backward(p, p, p, p, M, d, F, dt, p, p, p, lay, ctypes.byref(a), p, p, 2, p, None, p, huge, n)
    assert fwd(4096, 32, 1 << 21, 2) == -2 and fwd(600, 8388640, 16, 2) == -2 and fwd(600, 8388608, 16, 2) == -2
    assert fwd(1, 32, 1 << 28, 2) == -2 and fwd(128, 1 << 26, 16, 2) == -2
    for lay, dt in ((0, 0), (0, 1), (2, 0)):
        assert bwd(4194241, 32, 32, lay, dt) == -2
        assert bwd(4, 32, 32, lay, dt, many) == -2
    assert fwd(4194241, 1, 1, 0, 1) == -2


def test_workspaces_never_shrink():
    rows = [1, 16, 17, 64, 100, 128, 129, 300, 1000, 4096, 4097, 8192, 20000]
    for size in (mb.gated_linear_workspace_bytes, mb.gated_linear_backward_workspace_bytes):
        for lay, dt in ((0, torch.bfloat16), (0, torch.float32), (2, torch.bfloat16)):
            for d, F, r in [(64, 64, 1), (4096, 11008, 32), (1024, 2752, 256)]:
                got = [size(M, d, F, dt, lay, r) for M in rows]
                assert got == sorted(got) and got[0] > 0
                for M in rows:
                    assert got[rows.index(M)] <= min(size(M, d + 64, F, dt, lay, r), size(M, d, F + 64, dt, lay, r), size(M, d, F, dt, lay, r + 1))
        assert size(0, 64, 64, torch.float32, 0, 8) == 0 and size(1, 64, 1 << 30, torch.float32, 0, 8) == 0


def test_gradient_table_refusals():
    with pytest.raises(ValueError):
        mb.GradientTable.from_tensors([[None] * 7], [[None] * 7])
    with pytest.raises(ValueError):
        mb.GradientTable.from_tensors([[None] * 6], [[None] * 6])
    with pytest.raises(ValueError):
        mb.GradientTable.from_tensors([[torch.zeros(2)] + [None] * 6], [[None] * 7])  # host memory


def _host_tables(dA, dB, ranks=(4, 6), d=64, F=96):
    """Tables over host memory: what the binding reads of them before any device work."""
    z = torch.zeros(7 * len(ranks), dtype=torch.int64)
    A, B = [[torch.zeros(d, r)] * 7 for r in ranks], [[torch.zeros(r, F)] * 7 for r in ranks]
    return mb.AdapterTable(torch.tensor(ranks, dtype=torch.int32), z, z, max(ranks), len(ranks), (A, B)), mb.GradientTable(z, z, len(dA), torch.float32, (dA, dB))


def test_gradients_have_the_extents_of_their_matrices():
    """A buffer that is smaller than its matrix would be written past its end."""
    row = lambda **kw: [kw.get(f"s{s}") for s in range(7)]
    z = torch.zeros
    fits = lambda dA, dB: (lambda tabs: tabs[1].fits(tabs[0], 64, 96))(_host_tables(dA, dB))
    assert fits([row(s4=z(64, 4)), row(s5=z(64, 6))], [row(s5=z(4, 96)), row()])
    assert fits([row(), row(s4=z(64, 6), s0=z(1, 1))], [row(), row()])  # other sites' are not written
    for a, b in ((z(64, 3), None), (z(63, 4), None), (None, z(4, 95)), (None, z(3, 96)), (z(4, 96), z(64, 4)), (z(64, 6), None), (None, z(6, 96))):
        for s in ("s4", "s5"):
            assert not fits([row(**{s: a}), row()], [row(**{s: b}), row()])
    assert not fits([row(s4=z(64, 4))], [row()])  # a tenant short
    with pytest.raises(ValueError, match="dA must be"):
        _host_tables([row(s4=z(256)), row()], [row(), row()])
    x, w, ids = z(8, 64), z(96, 64), (z(2, dtype=torch.int32), z(2, dtype=torch.uint8))
    tab, short = _host_tables([row(s4=z(64, 2)), row()], [row(), row()])
    m, r2r = z(8, 96), z(8, dtype=torch.int32)
    with pytest.raises(ValueError, match="gradients must be those"):
        mb.milora_gated_linear_backward(m, x, m, m, w, w, tab, *ids, row_to_req=r2r, grads=short)
    narrow, _ = _host_tables([row(), row()], [row(), row()], F=95)
    for call in (lambda: mb.milora_gated_linear(x, w, w, narrow, *ids, row_to_req=r2r),
                 lambda: mb.milora_gated_linear_backward(m, x, m, m, w, w, narrow, *ids, row_to_req=r2r)):
        with pytest.raises(ValueError, match="adapter matrices"):
            call()


def test_adapters_share_the_type_of_x():
    """fp32 rows read from bf16 matrices would be read past their end."""
    z = torch.zeros
    tab, _ = _host_tables([[None] * 7] * 2, [[None] * 7] * 2)
    x, w, m, ids = z(8, 64).bfloat16(), z(96, 64).bfloat16(), z(8, 96), (z(2, dtype=torch.int32), z(2, dtype=torch.uint8))
    r2r = z(8, dtype=torch.int32)
    for call in (lambda: mb.milora_gated_linear(x, w, w, tab, *ids, row_to_req=r2r),
                 lambda: mb.milora_gated_linear_backward(m.bfloat16(), x, m, m, w, w, tab, *ids, row_to_req=r2r)):
        with pytest.raises(TypeError, match="adapter matrices"):
            call()


def test_gradients_may_not_overlap():
    room = torch.zeros(64 * 8 + 64 * 8)
    row = lambda v: [None] * 4 + [v, None, None]
    at = lambda k: room[k:k + 64 * 4].reshape(64, 4)
    _host_tables([row(at(0)), row(None)], [[None] * 7] * 2)
    _host_tables([row(at(0)), row(at(256))], [[None] * 7] * 2, ranks=(4, 4))  # one behind the other
    for k in (0, 1, 255):
        with pytest.raises(ValueError, match="one place"):
            _host_tables([row(at(k)), row(at(256 if k else 0))], [[None] * 7] * 2, ranks=(4, 4))


def test_plain_gradients_against_differences():
    """The formulas of the oracle against central differences in 64 bits (step 1e-6: error about 1e-9 relative)."""
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=F64)
    M, d, F, r = 5, 6, 7, 2
    x, Wg, Wu, dy = rnd(M, d), rnd(F, d), rnd(F, d), rnd(M, F)
    Ag, Bg, Au, Bu = ([rnd(*s), rnd(*s)] for s in ((d, r), (r, F), (d, r), (r, F)))
    tg, tu = [0, 1, -1, 0, 1], [1, 1, 0, -1, -1]
    loss = lambda: (plain.gated(plain.linear(x, Wg, Ag, Bg, tg), plain.linear(x, Wu, Au, Bu, tu)) * dy).sum()
    dx, dAg, dBg, dAu, dBu = plain.gated_backward(dy, x, Wg, Wu, Ag, Bg, Au, Bu, tg, tu)
    for v, dv in [(x, dx)] + [(m[t], dm[t]) for m, dm in ((Ag, dAg), (Bg, dBg), (Au, dAu), (Bu, dBu)) for t in range(2)]:
        num = torch.zeros_like(v)
        for i in range(v.numel()):
            keep = float(v.view(-1)[i])
            v.view(-1)[i] = keep + 1e-6
            up = loss()
            v.view(-1)[i] = keep - 1e-6
            num.view(-1)[i] = (up - loss()) / 2e-6
            v.view(-1)[i] = keep
        assert (num - dv).abs().max() <= 1e-7 * (1 + dv.abs().max())


# ---------------------------------------------------------------------------------------------------- results
def _layer(M, B, T, d, F, ranks, seed, dtype, rows, mx4=False, r_max=None):
    c = plain.Case(M, B, T, {4: (d, F), 5: (d, F)}, ranks, seed, DEV, dtype=dtype, rows=rows, sites=[4, 5], r_max=r_max)
    x = c.rnd(M, d)
    W = [c.rnd(F, d, s=d ** -0.5) for _ in range(2)]
    if mx4:
        W = [mb.milora_quantize_weight(w) for w in W]
        dense = [plain.dequantize(w, d, F) for w in W]
    else:
        dense = [w.cpu() for w in W]
    return c, x, W, dense


def _assert_forward(Y, c, x, dense, gate=None, up=None):
    d, half = x.shape[1], torch.finfo(c.dtype).eps / 2
    n = d + max(c.rank) + 16
    z, E = [], []
    for s in (4, 5):
        ten = c.tenants(s)
        z.append(plain.linear(x, dense[s - 4], c.A[s], c.Bm[s], ten))
        size = plain.linear_size(x, dense[s - 4], c.A[s], c.Bm[s], ten)
        E.append(size * (n * 2.0 ** -24 + (2.0 ** -16 if c.dtype == torch.bfloat16 else 0.0)))
    for saved, ref, e in ((gate, z[0], E[0]), (up, z[1], E[1])):
        if saved is not None:
            assert ((saved.cpu().double() - ref).abs() <= e).all()
    ref = plain.gated(*z)
    tol = z[1].abs() * 1.1 * E[0] + (z[0] * plain.sigmoid(z[0])).abs() * E[1] + E[0] * E[1] + ref.abs() * (half + 2.0 ** -20)
    far = (Y.cpu().double() - ref).abs()
    assert torch.isfinite(Y).all() and (far <= tol).all(), float((far / tol.clamp(min=1e-300)).max())
    return z


def _assert_backward(c, x, dense, dY, dX, dA, dB):
    T, half = c.T, torch.finfo(c.dtype).eps / 2
    ten = [c.tenants(4), c.tenants(5)]
    args = (c.A[4], c.Bm[4], c.A[5], c.Bm[5])
    dx, *grads = plain.gated_backward(dY, x, *dense, *args, *ten)
    # sizes: the same products with the magnitudes of dz and of all factors
    x64, dy = x.cpu().to(F64), dY.cpu().to(F64)
    z = [plain.linear(x, dense[i], c.A[4 + i], c.Bm[4 + i], ten[i]) for i in range(2)]
    s = plain.sigmoid(z[0])
    E = [plain.linear_size(x, dense[i], c.A[4 + i], c.Bm[4 + i], ten[i]) * (x.shape[1] * 2.0 ** -24 + 2.0 ** -16) for i in range(2)]
    grow = lambda v, e: v.abs() + e / half if half > 1e-4 else v.abs() + e * 2.0 ** 17  # what g and u are off, in units of c
    dz = [grow(dy * z[1] * s * (1 + z[0] * (1 - s)), dy.abs() * (1.1 * E[1] + z[1].abs() * 0.5 * E[0])),
          grow(dy * z[0] * s, dy.abs() * 1.1 * E[0])]
    F, n = dense[0].shape[0], 2 * dense[0].shape[0] + x.shape[0] + x.shape[1]
    unit = half + n * 2.0 ** -24 + (2.0 ** -12 if half > 1e-4 else 2.0 ** -18)
    size = sum(dz[i] @ dense[i].to(F64).abs() for i in range(2))
    sizes = [[], [], [], []]
    for i in range(2):
        for t in range(T):
            rows = [m for m, v in enumerate(ten[i]) if v == t]
            A, B = c.A[4 + i][t].cpu().to(F64).abs(), c.Bm[4 + i][t].cpu().to(F64).abs()
            low = dz[i][rows] @ B.t()
            size[rows] += low @ A.t()
            sizes[2 * i].append(x64[rows].abs().t() @ low)
            sizes[2 * i + 1].append((x64[rows].abs() @ A).t() @ dz[i][rows])
    got = [dA[0], dB[0], dA[1], dB[1]]
    pairs = ([("dX", dX, dx, size)] if dX is not None else [])
    pairs += [(f"{'dA' if k % 2 == 0 else 'dB'}{4 + k // 2} of tenant {t}", got[k][t], grads[k][t], sizes[k][t]) for k in range(4) for t in range(T)
              if got[k][t] is not None]
    for what, v, ref, S in pairs:
        v = v.cpu().double()
        far, tol = (v - ref).abs(), unit * S + half * ref.abs()
        assert torch.isfinite(v).all() and (far <= tol).all(), (what, float((far / tol.clamp(min=1e-300)).max()))
        if c.dtype == torch.bfloat16 and ref.numel() >= 1000 and ref.norm() > 0:
            assert far.norm() <= 4e-3 * ref.norm(), (what, float(far.norm() / ref.norm()))


def _room(c, d, F, r_extra=0):
    nan = lambda *s: torch.full(s, float("nan"), dtype=c.dtype, device=DEV)
    return [[nan(d, r) for r in c.rank] for _ in range(2)], [[nan(r, F) for r in c.rank] for _ in range(2)]


def _table(c, dA, dB):
    rows = lambda g: [[None] * 4 + [g[0][t], g[1][t], None] for t in range(c.T)]
    return mb.GradientTable.from_tensors(rows(dA), rows(dB))


SHAPES = [  # M, d, F, rows
    (1, 64, 16, "own"), (2, 64, 48, "mixed"), (17, 128, 80, "mixed"), (45, 192, 272, "mixed"), (63, 1024, 528, "own"), (64, 64, 64, "mixed"),
    (130, 192, 272, "sorted"), (300, 512, 1040, "mixed"), (300, 2048, 2064, "sorted"), (1100, 256, 1040, "mixed"), (513, 4096, 336, "sorted"),
    (1100, 2304, 1040, "mixed"), (2100, 1536, 4112, "sorted")]


@gpu
@pytest.mark.parametrize("M,d,F,rows", SHAPES)
@pytest.mark.parametrize("ranks", [(8,), (5, 33, 256)])
def test_forward_bf16(M, d, F, rows, ranks):
    c, x, W, dense = _layer(M, M if rows == "own" else min(M, 6), 3, d, F, ranks, M + d, torch.bfloat16, rows)
    tid, route = c.requests()
    guard = torch.full((M + 1, F), 7.0, dtype=c.dtype, device=DEV)
    gate, up = (torch.full((M + 1, F), 7.0, device=DEV) for _ in range(2))
    Y = mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), out=guard[:M], gate_out=gate[:M], up_out=up[:M])
    _assert_forward(Y, c, x, dense, gate[:M], up[:M])
    assert all((v[M] == 7.0).all() for v in (guard, gate, up))
    assert torch.equal(mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows()), Y)  # saving changes nothing


@gpu
@pytest.mark.parametrize("M,d,F,rows", [(1, 96, 16, "own"), (5, 1056, 48, "mixed"), (16, 64, 528, "own"), (33, 160, 80, "mixed"), (128, 512, 272, "own"),
                                        (129, 96, 48, "mixed"), (200, 192, 272, "mixed"), (700, 512, 1040, "sorted"), (600, 1056, 304, "mixed"),
                                                        (1100, 512, 2064, "mixed"), (2049, 640, 2064, "sorted"), (1300, 1152, 2048, "mixed"), (1100, 2304, 1040, "mixed")])
@pytest.mark.parametrize("ranks", [(8,), (5, 33, 256)])
def test_forward_quantised(M, d, F, rows, ranks):
    c, x, W, dense = _layer(M, M if rows == "own" else min(M, 6), 3, d, F, ranks, M + d, torch.bfloat16, rows, mx4=True)
    tid, route = c.requests()
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    Y = mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4, F=F, gate_out=gate, up_out=up)
    _assert_forward(Y, c, x, dense, gate, up)
    assert torch.equal(mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4, F=F), Y)


@gpu
@pytest.mark.parametrize("M,d,F,rows,dtype", [
    (1, 1, 1, "own", torch.float32), (3, 3, 5, "mixed", torch.float32), (16, 100, 77, "own", torch.float32), (17, 33, 65, "mixed", torch.float32),
    (300, 250, 683, "mixed", torch.float32), (200, 1000, 130, "sorted", torch.float32), (7, 50, 31, "mixed", torch.bfloat16),
    (100, 70, 90, "mixed", torch.bfloat16), (90, 64, 24, "mixed", torch.bfloat16), (11, 200, 1010, "mixed", torch.float32),
    (70, 66, 700, "sorted", torch.float32), (2100, 1030, 100, "sorted", torch.float32), (130, 90, 650, "mixed", torch.bfloat16)])
@pytest.mark.parametrize("ranks", [(4,), (3, 17, 40)])
def test_any_shape_forward_and_backward(M, d, F, rows, dtype, ranks):
    c, x, W, dense = _layer(M, M if rows == "own" else min(M, 5), 3, d, F, ranks, 3 * M + d, dtype, rows)
    tid, route = c.requests()
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    Y = mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), gate_out=gate, up_out=up)
    _assert_forward(Y, c, x, dense, gate, up)
    assert torch.equal(mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows()), Y)
    dY = c.rnd(M, F)
    dA, dB = _room(c, d, F)
    dX = mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), grads=_table(c, dA, dB))
    _assert_backward(c, x, dense, dY, dX, dA, dB)


@gpu
@pytest.mark.parametrize("M,d,F,rows,mx4", [(1, 64, 64, "own", False), (5, 128, 192, "mixed", False), (64, 64, 128, "own", False), (100, 256, 704, "mixed", False),
                                            (257, 192, 320, "sorted", False), (600, 512, 1088, "mixed", False), (700, 1040, 448, "sorted", False),
                                            (1500, 320, 1024, "sorted", False), (4200, 4128, 704, "sorted", False), (65, 96, 32, "mixed", False), (300, 288, 800, "mixed", True),
                                            (1100, 1056, 1504, "sorted", False), (40, 384, 96, "mixed", True), (1100, 1152, 1504, "sorted", True), (7, 128, 32, "own", True),
                                            (2100, 4352, 512, "sorted", True), (33, 96, 128, "mixed", True), (300, 256, 704, "mixed", True), (64, 160, 48, "mixed", True)])
@pytest.mark.parametrize("ranks", [(8,), (16, 32), (5, 33, 256)])
def test_backward_bf16(M, d, F, rows, mx4, ranks):
    c, x, W, dense = _layer(M, M if rows == "own" else min(M, 6), 3, d, F, ranks, M + d, torch.bfloat16, rows, mx4)
    tid, route = c.requests()
    lay = mb.W_MX4 if mx4 else mb.W_ROWMAJOR
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F, gate_out=gate, up_out=up)
    dY = c.rnd(M, F)
    dA, dB = _room(c, d, F)
    guard = torch.full((M + 1, d), 7.0, dtype=c.dtype, device=DEV)
    dX = mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F, dX=guard[:M],
                                         grads=_table(c, dA, dB))
    assert (guard[M] == 7.0).all()
    _assert_backward(c, x, dense, dY, dX, dA, dB)
    # one wanted output at a time gives the same bits; nothing else is touched
    only = mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F)
    assert torch.equal(only, dX)
    dA2, dB2 = _room(c, d, F)
    rows_of = lambda g, keep: [[None] * 4 + [g[0][t] if keep(0, t) else None, g[1][t] if keep(1, t) else None, None] for t in range(c.T)]
    part = mb.GradientTable.from_tensors(rows_of(dA2, lambda s, t: s == t % 2), rows_of(dB2, lambda s, t: t == 1))
    assert mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F, want_dx=False, grads=part) is None
    for s in range(2):
        for t in range(c.T):
            assert torch.equal(dA2[s][t], dA[s][t]) if s == t % 2 else torch.isnan(dA2[s][t]).all()
            assert torch.equal(dB2[s][t], dB[s][t]) if t == 1 else torch.isnan(dB2[s][t]).all()


@gpu
def test_rows_without_a_tenant_and_tenants_without_rows():
    """No row has a LoRA term: its gradients are zeros, dX that of the base; ranks out of range keep their buffers."""
    M, d, F = 70, 128, 192
    c, x, W, dense = _layer(M, 5, 3, d, F, (8, 16, 8), 9, torch.bfloat16, "none", r_max=8)
    tid, route = c.requests()
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    Y = mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), gate_out=gate, up_out=up)
    _assert_forward(Y, c, x, dense, gate, up)
    dY = c.rnd(M, F)
    dA, dB = _room(c, d, F)
    dX = mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), grads=_table(c, dA, dB))
    assert all(torch.isnan(g[s][1]).all() for g in (dA, dB) for s in range(2))  # rank 16 > r_max 8
    for g in (dA, dB):
        for s in range(2):
            g[s][1] = None
            assert all((g[s][t] == 0).all() for t in (0, 2))
    _assert_backward(c, x, dense, dY, dX, dA, dB)


@gpu
@pytest.mark.parametrize("M,d,F,dtype", [(20, 128, 96, torch.bfloat16), (130, 128, 192, torch.bfloat16), (1100, 256, 1040, torch.bfloat16), (600, 1280, 1040, torch.bfloat16), (40, 30, 50, torch.float32),
                                         (9, 30, 50, torch.float32)])
def test_infinities_and_nans_stay_in_their_tenants_rows(M, d, F, dtype):
    c, x, W, dense = _layer(M, 6, 3, d, F, (8, 16), 40 + M, dtype, "mixed")
    c.route[:] = 0x80 | 0x30
    c.tid[:] = torch.tensor([0, 1, 2, 0, 1, 2])
    c.route[5] = 255
    tid, route = c.requests()
    run = lambda: mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows())
    clean = run()
    assert torch.isfinite(clean).all()
    c.Bm[4][1][3, 7], c.Bm[5][1][0, F - 1] = float("inf"), float("nan")
    Y = run()
    mine = (torch.tensor(c.tenants(4)) == 1).to(DEV)
    assert mine.any() and torch.equal(Y[~mine], clean[~mine])
    assert not torch.isfinite(Y[mine][:, 7].float()).any() or (Y[mine][:, 7] == 0).any()  # silu(-inf) u is NaN, silu(inf) u is Inf
    assert torch.isnan(Y[mine][:, F - 1]).all()
    keep = [j for j in range(F) if j not in (7, F - 1)]
    assert torch.equal(Y[mine][:, keep], clean[mine][:, keep])


@gpu
def test_backward_keeps_a_tenants_infinities_to_its_rows():
    M, d, F = 300, 192, 320
    c, x, W, dense = _layer(M, 6, 3, d, F, (8, 16), 41, torch.bfloat16, "mixed")
    c.route[:] = 0x80 | 0x30
    tid, route = c.requests()
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), gate_out=gate, up_out=up)
    dY = c.rnd(M, F)

    def run():
        dA, dB = _room(c, d, F)
        return mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), grads=_table(c, dA, dB)), dA, dB

    dX, dA, dB = run()
    c.A[4][1][3, 7], c.A[5][1][d - 1, 0] = float("inf"), float("nan")
    bad, dA2, dB2 = run()
    mine = (torch.tensor(c.tenants(4)) == 1).to(DEV)
    assert torch.equal(bad[~mine], dX[~mine]) and torch.isnan(bad[mine][:, d - 1]).all() and not torch.isfinite(bad[mine][:, 3]).any()
    keep = [j for j in range(d) if j not in (3, d - 1)]
    assert torch.equal(bad[mine][:, keep], dX[mine][:, keep])
    for s in range(2):
        for t in (0, 2):
            assert torch.equal(dA2[s][t], dA[s][t]) and torch.equal(dB2[s][t], dB[s][t])


@gpu
@pytest.mark.parametrize("M,d,F,mx4,dtype", [(40, 128, 96, False, torch.bfloat16), (300, 256, 320, False, torch.bfloat16), (24, 128, 96, True, torch.bfloat16),
                                             (300, 256, 320, True, torch.bfloat16), (1100, 1536, 1088, False, torch.bfloat16), (1100, 2304, 1088, True, torch.bfloat16),
                                             (30, 50, 70, False, torch.float32)])
def test_captured_step_replays(M, d, F, mx4, dtype):
    """A training step captured once and replayed with other inputs gives the bits of eager calls, whatever the workspaces hold."""
    c, x, W, dense = _layer(M, 5, 2, d, F, (8, 16), 60 + M, dtype, "mixed", mx4)
    tid, route, r2r = *c.requests(), c.rows()
    lay = mb.W_MX4 if mx4 else mb.W_ROWMAJOR
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    dY, Y, dX = c.rnd(M, F), torch.empty(M, F, dtype=dtype, device=DEV), torch.empty(M, d, dtype=dtype, device=DEV)
    dA, dB = _room(c, d, F)
    table = _table(c, dA, dB)
    r = c.tab.r_max
    ws = torch.full((mb.gated_linear_workspace_bytes(M, d, F, dtype, lay, r),), 255, dtype=torch.uint8, device=DEV)
    ws2 = torch.full((mb.gated_linear_backward_workspace_bytes(M, d, F, dtype, lay, r),), 255, dtype=torch.uint8, device=DEV)

    def step():
        mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=r2r, w_layout=lay, F=F, out=Y, gate_out=gate, up_out=up, workspace=ws)
        mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=r2r, w_layout=lay, F=F, dX=dX, grads=table, workspace=ws2)
        return [v.clone() for v in (Y, dX, *(g[s][t] for g in (dA, dB) for s in range(2) for t in range(2)))]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.copy_(c.rnd(M, d))
        dY.copy_(c.rnd(M, F))
        want = step()
        for v in (Y, dX, gate, up):
            v.fill_(3.0)
        ws.fill_(255)
        ws2.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [Y, dX, *(g[s][t] for g in (dA, dB) for s in range(2) for t in range(2))]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    _assert_backward(c, x, dense, dY, dX, dA, dB)


@gpu
@pytest.mark.parametrize("M", [20, 200])
def test_unaligned_bf16_tensors(M):
    """Row-major tensors at any alignment of their type take the any-shape path."""
    d, F = 128, 96
    c, x, W, dense = _layer(M, 4, 2, d, F, (8,), 80 + M, torch.bfloat16, "mixed")
    shift = lambda v: torch.cat([v.reshape(-1)[:1], v.reshape(-1)])[1:].reshape(v.shape)
    x, W = shift(x), [shift(w) for w in W]
    assert x.data_ptr() % 4 == 2
    tid, route = c.requests()
    gate, up = (torch.empty(M * F + 1, device=DEV)[1:].reshape(M, F) for _ in range(2))
    Y = mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), gate_out=gate, up_out=up)
    _assert_forward(Y, c, x, dense, gate, up)
    dY = shift(c.rnd(M, F))
    dA, dB = _room(c, d, F)
    dX = mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, row_to_req=c.rows(), grads=_table(c, dA, dB))
    _assert_backward(c, x, dense, dY, dX, dA, dB)


@gpu
def test_two_streams_at_once():
    """Training steps and 4-bit linears on two streams at the same time, workspaces apart, give the bits of one after the other."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    steps = []
    for k, (M, d, F, mx4) in enumerate([(1100, 2304, 1088, False), (1100, 1536, 1088, True)]):
        c, x, W, _ = _layer(M, 5, 2, d, F, (8, 16), 95 + k, torch.bfloat16, "mixed", mx4)
        tid, route, r2r = *c.requests(), c.rows()
        lay = mb.W_MX4 if mx4 else mb.W_ROWMAJOR
        dY, gate, up, Y, dX = c.rnd(M, F), *(torch.empty(M, F, device=DEV) for _ in range(2)), torch.empty(M, F, dtype=c.dtype, device=DEV), torch.empty_like(x)
        dA, dB = _room(c, d, F)
        q = mb.milora_quantize_weight(c.rnd(F, d, s=d ** -0.5))
        Z = torch.empty_like(Y)
        size = mb.gated_linear_workspace_bytes, mb.gated_linear_backward_workspace_bytes
        ws = [torch.empty(f(M, d, F, c.dtype, lay, c.tab.r_max), dtype=torch.uint8, device=DEV) for f in size]
        ws.append(torch.empty(mb.quantized_linear_workspace_bytes(M, d, F, c.tab.r_max), dtype=torch.uint8, device=DEV))
        kw = dict(row_to_req=r2r, w_layout=lay, F=F)

        def step(x=x, W=W, c=c, tid=tid, route=route, r2r=r2r, kw=kw, Y=Y, gate=gate, up=up, dY=dY, dX=dX, ws=ws, q=q, Z=Z, F=F, table=_table(c, dA, dB)):
            mb.milora_gated_linear(x, *W, c.tab, tid, route, out=Y, gate_out=gate, up_out=up, workspace=ws[0], **kw)
            mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, dX=dX, grads=table, workspace=ws[1], **kw)
            mb.milora_routed_linear(x, q, c.tab, 4, tid, route, row_to_req=r2r, w_layout=mb.W_MX4, d2=F, out=Z, workspace=ws[2])

        steps.append((step, [Y, gate, up, dX, Z, *dA[0], *dA[1], *dB[0], *dB[1]]))
    alone = []
    for step, outs in steps:
        step()
        alone.append([o.clone() for o in outs])
    torch.cuda.synchronize()
    for _ in range(10):
        for _, outs in steps:
            for o in outs:
                o.fill_(float("nan"))
        torch.cuda.synchronize()
        for side, (step, _) in zip(sides, steps):
            with torch.cuda.stream(side):
                step()
                step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for (_, outs), want in zip(steps, alone) for a, b in zip(outs, want))


@gpu
def test_refuses_another_device_and_gradients_in_one_place(monkeypatch):
    c, x, W, _ = _layer(20, 4, 2, 64, 96, (8,), 90, torch.bfloat16, "mixed", True)
    tid, route = c.requests()
    kw = dict(row_to_req=c.rows(), w_layout=mb.W_MX4, F=96)
    gate, up = (torch.empty(20, 96, device=DEV) for _ in range(2))
    dA, dB = _room(c, 64, 96)
    dA[1][0] = dA[0][0]
    with pytest.raises(ValueError):
        _table(c, dA, dB)
    wide, dy, dx = c.rnd(64, 64), c.rnd(20, 96), torch.empty_like(x)
    q = mb.milora_quantize_weight(wide)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: mb.milora_gated_linear(x, *W, c.tab, tid, route, **kw),
                 lambda: mb.milora_gated_linear_backward(dy, x, gate, up, *W, c.tab, tid, route, dX=dx, **kw),
                 lambda: mb.milora_quantize_weight(wide, out=q), lambda: mb.milora_dequantize_weight(q, 64, 64)):
        with pytest.raises(ValueError, match="current device"):
            call()


@gpu
def test_the_block_is_the_middle_of_a_layer():
    """Chained with the routed down projection: the feed-forward half of a layer, on bf16 and on 4-bit weights of the same values."""
    M, d, F = 200, 256, 704
    c = plain.Case(M, 5, 3, {4: (d, F), 5: (d, F), 6: (F, d)}, (8, 16), 77, DEV, rows="mixed", sites=[4, 5, 6])
    x = c.rnd(M, d)
    q = [mb.milora_quantize_weight(c.rnd(*s, s=s[1] ** -0.5)) for s in ((F, d), (F, d), (d, F))]
    W = [mb.milora_dequantize_weight(q[i], *((d, F) if i < 2 else (F, d))) for i in range(3)]
    # adapters of sites 4, 5 and 6 have shapes of their own
    tab = mb.AdapterTable.from_tensors([[c.A[6 if s == 6 else 4 if s < 5 else 5][t] for s in range(7)] for t in range(3)],
                                       [[c.Bm[6 if s == 6 else 4 if s < 5 else 5][t] for s in range(7)] for t in range(3)], c.rank)
    tid, route = c.requests()
    outs = []
    for lay, w in ((mb.W_ROWMAJOR, W), (mb.W_MX4, q)):
        m = mb.milora_gated_linear(x, w[0], w[1], tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F)
        outs.append((m, mb.milora_routed_linear(m, w[2], tab, 6, tid, route, row_to_req=c.rows(), w_layout=lay, d2=d)))
    ref = plain.gated(*(plain.linear(x, W[i], c.A[4 + i], c.Bm[4 + i], c.tenants(4 + i)) for i in range(2)))
    out = plain.linear(ref, W[2], c.A[6], c.Bm[6], c.tenants(6))
    for m, y in outs:
        assert (m.cpu().double() - ref).norm() <= 2.5e-3 * ref.norm()  # one rounding
        assert (y.cpu().double() - out).norm() <= 4e-3 * out.norm()    # two


# Kernels: few rows in fp32 arithmetic, tiles of 64 and 128 (terms row by row, and by the matrix cores), 256 x 256 (cut too), 4-bit weights of few rows,
# on the codes and written out, any shape.
@gpu
@pytest.mark.parametrize("M,d,F,dtype,mx4", [
    (9, 70, 96, torch.bfloat16, False), (20, 128, 96, torch.bfloat16, False), (63, 1024, 528, torch.bfloat16, False), (130, 128, 192, torch.bfloat16, False),
    (300, 512, 1040, torch.bfloat16, False), (600, 1280, 1040, torch.bfloat16, False), (2100, 1536, 4112, torch.bfloat16, False), (9, 128, 96, torch.bfloat16, True),
    (100, 512, 272, torch.bfloat16, True), (600, 1056, 304, torch.bfloat16, True), (1100, 512, 2064, torch.bfloat16, True), (2049, 640, 2064, torch.bfloat16, True),
    (12, 30, 50, torch.float32, False), (40, 30, 50, torch.float32, False), (300, 250, 683, torch.float32, False)])
def test_an_infinite_scale_stays_infinite_and_in_its_projection(M, d, F, dtype, mx4):
    """x W^A_4 of one rank is Inf for a tenant's rows: g is Inf by the signs of the factors, u is what it was."""
    c, x, W, dense = _layer(M, 6, 3, d, F, (8, 16), 40 + M, dtype, "mixed", mx4)
    c.route[:] = 0x80 | 0x30
    c.tid[:] = torch.tensor([0, 1, 2, 0, 1, 2])
    tid, route = c.requests()
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    run = lambda: mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=mb.W_MX4 if mx4 else mb.W_ROWMAJOR, F=F, gate_out=gate, up_out=up)
    clean, u = run(), up.clone()
    assert torch.isfinite(clean).all()
    c.A[4][1][3, 2] = float("inf")
    assert (x[:, 3] != 0).all() and (c.Bm[4][1][2] != 0).all()
    Y = run()
    mine = (torch.tensor(c.tenants(4)) == 1).to(DEV)
    assert mine.any() and torch.equal(Y[~mine], clean[~mine])
    sign = torch.sign(x[mine, 3].float())[:, None] * torch.sign(c.Bm[4][1][2].float())
    assert torch.equal(gate[mine], sign * float("inf"))
    assert torch.equal(up, u)
    pos = sign > 0
    assert torch.isnan(Y[mine][~pos]).all()  # silu(-Inf) is -Inf / Inf
    assert torch.equal(Y[mine][pos].float(), (torch.sign(u[mine]) * float("inf"))[pos])


@gpu
@pytest.mark.parametrize("M,d,F,mx4", [(40, 128, 96, False), (300, 192, 320, False), (1100, 1536, 1088, False), (300, 256, 704, True), (64, 160, 48, True), (40, 30, 50, False)])
def test_backward_of_an_infinite_scale(M, d, F, mx4):
    """dz (W^B)^T of one rank is Inf for a tenant's rows: dX is Inf by the signs of the factors, other gradients are what they were."""
    dtype = torch.bfloat16 if d % 32 == 0 else torch.float32
    c, x, W, dense = _layer(M, 6, 3, d, F, (8, 16), 41, dtype, "mixed", mx4)
    c.route[:] = 0x80 | 0x30
    c.tid[:] = torch.tensor([0, 1, 2, 0, 1, 2])
    tid, route = c.requests()
    kw = dict(row_to_req=c.rows(), w_layout=mb.W_MX4 if mx4 else mb.W_ROWMAJOR, F=F)
    gate, up = (torch.empty(M, F, device=DEV) for _ in range(2))
    mb.milora_gated_linear(x, *W, c.tab, tid, route, gate_out=gate, up_out=up, **kw)
    dY = c.rnd(M, F)

    def run():
        dA, dB = _room(c, d, F)
        return mb.milora_gated_linear_backward(dY, x, gate, up, *W, c.tab, tid, route, grads=_table(c, dA, dB), **kw), dA, dB

    dX, dA, dB = run()
    c.Bm[5][1][2, 7] = float("inf")
    got, dA2, dB2 = run()
    mine = (torch.tensor(c.tenants(5)) == 1).to(DEV)
    du = dY[:, 7].float() * gate[:, 7] * torch.sigmoid(gate[:, 7])
    assert mine.any() and (du != 0).all() and (c.A[5][1][:, 2] != 0).all()
    assert torch.equal(got[~mine], dX[~mine])
    assert torch.equal(got[mine].float(), torch.sign(du[mine])[:, None] * torch.sign(c.A[5][1][:, 2].float()) * float("inf"))
    for s in range(2):
        for t in range(3):
            assert torch.equal(dB2[s][t], dB[s][t])
            keep = [k for k in range(c.rank[t]) if (s, t, k) != (1, 1, 2)]
            assert torch.equal(dA2[s][t][:, keep], dA[s][t][:, keep])
    assert not torch.isfinite(dA2[1][1][:, 2]).any()


@gpu
@pytest.mark.parametrize("mx4", [False, True])
def test_a_wait_of_cut_tiles_ends(mx4):
    """With a limit of one poll a cut tile whose other sums are not there yet is NaN, the others are what they were, and the launch ends; with the default
    the same call is right again."""
    M, d, F = 1100, 2304, 1040
    c, x, W, dense = _layer(M, 5, 3, d, F, (8, 16), 17, torch.bfloat16, "mixed", mx4)
    tid, route = c.requests()
    lay = mb.W_MX4 if mx4 else mb.W_ROWMAJOR
    ws = torch.full((mb.gated_linear_workspace_bytes(M, d, F, c.dtype, lay, c.tab.r_max),), 255, dtype=torch.uint8, device=DEV)
    run = lambda: mb.milora_gated_linear(x, *W, c.tab, tid, route, row_to_req=c.rows(), w_layout=lay, F=F, workspace=ws)
    clean = run()
    _assert_forward(clean, c, x, dense)
    old = mb.milora_set_wait_limit(1)
    try:
        short = run()
        torch.cuda.synchronize()
    finally:
        assert mb.milora_set_wait_limit(old) == 1
    same = (short == clean) | torch.isnan(short)
    assert same.all()
    assert torch.equal(run(), clean)
