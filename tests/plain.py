"""Plain 64-bit forms of the 4-bit weights and of the gated block, written from their definitions (test infrastructure only)."""
import math

import torch

from paper_2410_18035_amd import binding as mb

F64 = torch.float64
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantize(w: torch.Tensor):
    """[d2, d1] weights -> (codes uint8 [d2, d1], scale bytes uint8 [d2, d1/32]) by search over the eight magnitudes."""
    v = w.detach().cpu().to(F64).reshape(w.shape[0], -1, 32)
    finite = torch.isfinite(v).all(2)
    clean = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    top = clean.abs().amax(2)
    scale = torch.full(top.shape, 2, dtype=torch.int64)
    for i, j in (top >= 2.0 ** -126).nonzero().tolist():
        scale[i, j] = max(2, math.frexp(float(top[i, j]))[1] - 1 - 2 + 127)
    m = clean.abs() * torch.pow(torch.tensor(2.0, dtype=F64), (127 - scale).to(F64))[..., None]
    grid = torch.tensor(E2M1, dtype=F64)
    far = (m[..., None] - grid).abs()
    far[..., 1::2] += far.amin(-1, keepdim=True) * 1e-12  # a tie goes to the even code (distances are exact to far less than that)
    codes = far.argmin(-1) + 8 * torch.signbit(clean)
    codes[~finite] = 0
    scale[~finite] = 255
    return codes.reshape(w.shape).to(torch.uint8), scale.to(torch.uint8)


def pack(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    return torch.cat([(codes[:, 0::2] | (codes[:, 1::2] << 4)).reshape(-1), scales.reshape(-1)])


def dequantize(q: torch.Tensor, d1: int, d2: int) -> torch.Tensor:
    q = q.cpu()
    pair = torch.stack([q[:d1 * d2 // 2] & 15, q[:d1 * d2 // 2] >> 4], 1).reshape(d2, d1 // 32, 32).long()
    s = q[d1 * d2 // 2:].reshape(d2, d1 // 32, 1)
    v = torch.tensor(E2M1 + [-e for e in E2M1], dtype=F64)[pair] * torch.pow(torch.tensor(2.0, dtype=F64), s.to(F64) - 127)
    return torch.where(s == 255, torch.full_like(v, float("nan")), v).reshape(d2, d1)


def routed_to(site, route, tid, n_tenants, ranks, r_max, r2r, M):
    """Tenant of each row with a low-rank term at `site`, -1 for the others."""
    out = []
    for m in range(M):
        b = m if r2r is None else int(r2r[m])
        ten = -1
        if 0 <= b < len(route):
            v = int(route[b])
            has = v == site if v < 7 else (v != 255 and v & 0x80 and (v >> site) & 1)
            t = int(tid[b])
            if has and 0 <= t < n_tenants and 1 <= ranks[t] <= r_max:
                ten = t
        out.append(ten)
    return out


def linear(x, W, A, B, tenants, bias=None):
    """x W^T + bias + (x A) B for the rows of each tenant; W [d2, d1], A and B per tenant."""
    x = x.cpu().to(F64)
    y = x @ W.cpu().to(F64).t()
    if bias is not None:
        y = y + bias.cpu().to(F64)
    for t in sorted(set(tenants)):
        if t >= 0:
            rows = [m for m, u in enumerate(tenants) if u == t]
            y[rows] += (x[rows] @ A[t].cpu().to(F64)) @ B[t].cpu().to(F64)
    return y


def linear_size(x, W, A, B, tenants, bias=None):
    """The same with the magnitudes of all factors: what rounding errors of the sums go by."""
    pos = lambda v: None if v is None else v.cpu().to(F64).abs()
    return linear(pos(x), pos(W), [pos(a) for a in A], [pos(b) for b in B], tenants, pos(bias))


def sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def gated(g, u):
    return g * sigmoid(g) * u


def gated_backward(dy, x, Wg, Wu, Ag, Bg, Au, Bu, ten_g, ten_u):
    """Gradients of x and of the tenants' low-rank matrices at the two sites (a tenant without rows: zeros)."""
    x, dy = x.cpu().to(F64), dy.cpu().to(F64)
    g, u = linear(x, Wg, Ag, Bg, ten_g), linear(x, Wu, Au, Bu, ten_u)
    s = sigmoid(g)
    dx, grads = 0, []
    for dz, W, A, B, ten in ((dy * u * s * (1 + g * (1 - s)), Wg, Ag, Bg, ten_g), (dy * g * s, Wu, Au, Bu, ten_u)):
        part = dz @ W.cpu().to(F64)
        dA, dB = [torch.zeros(a.shape, dtype=F64) for a in A], [torch.zeros(b.shape, dtype=F64) for b in B]
        for t in range(len(A)):
            rows = [m for m, v in enumerate(ten) if v == t]
            if rows:
                low = dz[rows] @ B[t].cpu().to(F64).t()
                part[rows] += low @ A[t].cpu().to(F64).t()
                dA[t] = x[rows].t() @ low
                dB[t] = (x[rows] @ A[t].cpu().to(F64)).t() @ dz[rows]
        dx = dx + part
        grads += [dA, dB]
    return dx, *grads


class Case:
    """A layer's adapters, requests and rows, drawn from a seed."""

    def __init__(self, M, B, T, dims, ranks, seed, dev, dtype=torch.bfloat16, rows="mixed", sites=None, r_max=None):
        self.g = torch.Generator().manual_seed(seed)
        self.M, self.B, self.T, self.dev, self.dtype = M, B, T, dev, dtype
        self.rank = [ranks[t % len(ranks)] for t in range(T)]
        scale = {s: (dims[s][0] * sum(self.rank) / T) ** -0.25 for s in dims}
        self.A = {s: [self.rnd(dims[s][0], r, s=scale[s]) for r in self.rank] for s in dims}
        self.Bm = {s: [self.rnd(r, dims[s][1], s=scale[s]) for r in self.rank] for s in dims}
        any_of = lambda mats, s: mats[s] if s in mats else mats[next(iter(mats))]
        self.tab = mb.AdapterTable.from_tensors([[any_of(self.A, s)[t] for s in range(7)] for t in range(T)],
                                                [[any_of(self.Bm, s)[t] for s in range(7)] for t in range(T)], self.rank, r_max)
        self.tid = torch.randint(0, T, (B,), generator=self.g).to(torch.int32)
        k = torch.randint(1, 5, (B,), generator=self.g)
        sets = torch.rand(B, 7, generator=self.g).argsort(1)
        self.route = torch.tensor([int(sets[b, 0]) if k[b] == 1 else 0x80 | sum(1 << int(s) for s in sets[b, :int(k[b])]) for b in range(B)],
                                  dtype=torch.uint8)
        if sites:  # request 0 has these
            self.route[0] = 0x80 | sum(1 << s for s in sites)
        self.r2r = None
        if rows != "own":
            self.r2r = torch.sort(torch.randint(0, B, (M,), generator=self.g))[0].to(torch.int32)
            if rows == "mixed":
                self.r2r = self.r2r[torch.randperm(M, generator=self.g)]
                self.r2r[torch.rand(M, generator=self.g) < 0.1] = -1
            if rows == "none":
                self.r2r[:] = B
            if M > 1 and rows != "none":
                self.r2r[M // 2] = 0

    def rnd(self, *shape, s=1.0, dtype=None):
        return (torch.randn(*shape, generator=self.g) * s).to(dtype or self.dtype).to(self.dev)

    def tenants(self, site):
        return routed_to(site, self.route, self.tid, self.T, self.rank, self.tab.r_max, self.r2r, self.M)

    def requests(self):
        return self.tid.to(self.dev), self.route.to(self.dev)

    def rows(self):
        return None if self.r2r is None else self.r2r.to(self.dev)
