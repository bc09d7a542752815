"""Residual layer norm and its gradient against the plain fp64 form.

Per value the kernel rounds r - mu (relative to |r| + |mu|, with mu's own error: a sum of d values
in chains of at most ceil(d / 256) additions and a tree), the product with rstd (whose relative
error is that of a sum of squares) and one fused step with w and b.  With c = 24 + d / 128 roundings
of 2^-24 relative to m = max |r| of the row times rstd (at least 1), |u - ref| <= c 2^-24 (m |w| + |b|);
bf16 adds half a step, 2^-8 |u|.
"""
import numpy as np
import pytest

import paper_2605_28283_amd as pp
from oracle import operators as op

pytestmark = pytest.mark.gpu

EPS = 1e-5
HALF = 2.0 ** -24
WIDTHS = [1, 2, 3, 5, 63, 64, 100, 255, 256, 257, 1000, 1023, 1024, 1028, 2048, 4095, 4096, 4100,
          8191, 8192, 8196, 12289, 65536]


def dev(a, lead=0):
    """On the GPU; `lead` elements in front move it off its alignment."""
    import torch
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    buf = torch.full((lead + t.numel() + 3,), -77.0, device="cuda")
    buf[lead:lead + t.numel()] = t.reshape(-1).cuda()
    return buf[lead:lead + t.numel()].view(t.shape)


def out(shape, dtype, lead=0):
    import torch
    n = int(np.prod(shape))
    buf = torch.full((lead + n + 3,), -77.0, dtype=dtype, device="cuda")
    return buf[lead:lead + n].view(shape), buf, lead


def ends_kept(o):
    view, buf, lead = o
    n = view.numel()
    return bool((buf[:lead] == -77).all()) and bool((buf[lead + n:] == -77).all())


def bounds(r, w, b, eps=EPS):
    d = r.shape[1]
    ref, mu, rstd = op.layernorm(r, eps, w, b)
    m = np.maximum(np.abs(r).max(1, keepdims=True) * rstd, 1.0)
    c = (24 + d / 128) * HALF
    wa = 1.0 if w is None else np.abs(w)
    ba = 0.0 if b is None else np.abs(b)
    return ref, c * (m * wa + ba), mu, rstd


def forward(x, y, w, b, f32, alias=None, lead=0, x_out=True, eps=EPS):
    import torch
    T, d = x.shape
    xd, yd = dev(x, lead), dev(y, lead)
    xo = {"x": xd, "y": yd}.get(alias)
    xo_o = None
    if xo is None and x_out:
        xo_o = out((T, d), torch.float32, lead)
        xo = xo_o[0]
    u_o = out((T, d), torch.float32 if f32 else torch.bfloat16, lead)
    st_o = out((T, 2), torch.float32, 1)
    pp.prunepath_residual_layernorm(xd, yd, xo, T, d, eps, dev(w, lead), dev(b, lead), u_o[0],
                                    st_o[0], pp.PP_NORM_F32 if f32 else 0)
    torch.cuda.synchronize()
    assert all(ends_kept(o) for o in (xo_o, u_o, st_o) if o)
    return (None if xo is None else xo.cpu().numpy(), u_o[0].float().cpu().numpy(),
            st_o[0].cpu().numpy())


def check_forward(x, y, w, b, f32, **kw):
    r32 = x if y is None else (x + y).astype(np.float32)
    xo, u, st = forward(x, y, w, b, f32, **kw)
    if xo is not None:
        np.testing.assert_array_equal(xo, r32)
    r = r32.astype(np.float64)
    ref, tol, mu, rstd = bounds(r, w, b, kw.get("eps", EPS))
    assert (np.abs(u - ref) <= tol + (0 if f32 else 2.0 ** -8 * np.abs(ref))).all(), \
        np.abs(u - ref).max()
    c = (24 + x.shape[1] / 128) * HALF
    assert (np.abs(st[:, :1] - mu) <= c * np.abs(r).max(1, keepdims=True)).all()
    # the sum of squares is off by a relative c, and by the error of mu squared
    m = np.maximum(np.abs(r).max(1, keepdims=True) * rstd, 1.0)
    assert (np.abs(st[:, 1:] - rstd) <= (c + (c * m) ** 2) * rstd).all()
    return u, st


def data(T, d, seed, std=4.0):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    return f(T, d) * np.float32(std), f(T, d), 1 + f(d) * np.float32(0.2), f(d) * np.float32(0.3)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("f32", [False, True])
def test_forward(d, f32):
    print("layernorm d=%d f32=%d" % (d, f32), flush=True)
    T = 7 if d < 9000 else 2
    x, y, w, b = data(T, d, d)
    check_forward(x, y, w, b, f32)
    check_forward(x, None, None, None, f32)
    check_forward(x, y, w, None, f32, lead=1)
    check_forward(x, None, None, b, f32, lead=2, x_out=False)


@pytest.mark.parametrize("d", [4, 5, 256, 1024, 4096, 8192, 8200, 12289])
@pytest.mark.parametrize("alias", ["x", "y"])
def test_in_place(d, alias):
    x, y, w, b = data(3, d, d + 1)
    check_forward(x, y, w, b, False, alias=alias)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 63, 257, 5000])
def test_rows_do_not_touch_each_other(T):
    x, y, w, b = data(T, 320, T)
    u, st = check_forward(x, y, w, b, False)
    for t in {0, T // 2, T - 1}:
        u1, s1 = check_forward(x[t:t + 1], y[t:t + 1], w, b, False)
        assert u1.tobytes() == u[t:t + 1].tobytes() and s1.tobytes() == st[t:t + 1].tobytes()


def test_hard_rows():
    """A large common offset, constant rows, tiny and large values, rows that are not finite."""
    x, y, w, b = data(6, 512, 5, 1.0)
    x[0] += 3000.0
    x[1] = 7.5
    y[1] = 0.0
    x[2] *= 1e-20
    y[2] *= 1e-20
    x[3] *= 1e12
    check_forward(x, y, w, b, True)
    x[4, 7] = np.nan
    x[5, 3] = np.inf
    _, u, _ = forward(x, y, w, b, False)
    assert np.isnan(u[4]).all() and np.isnan(u[5]).any()
    assert np.isfinite(u[:4]).all()


# ------------------------------------------------------------------ gradient

def backward(r, du, dres, w, stats, f32, lead=0, alias=False, dw=True, db=True):
    import torch
    T, d = r.shape
    g = dev(du, lead)
    if not f32:
        buf = torch.zeros(lead + T * d, dtype=torch.bfloat16, device="cuda")
        buf[lead:] = g.reshape(-1).bfloat16()
        g = buf[lead:].view(T, d)
    dr = dev(dres, lead)
    o = out((T, d), torch.float32, lead)
    dx = dr if alias else o[0]
    w_o, b_o = out((d,), torch.float32, lead), out((d,), torch.float32, lead)
    n = pp.prunepath_residual_layernorm_grad_workspace(T, d) // 4
    ws = out((n,), torch.float32, 0)
    ws[1][:n] = float("nan")
    pp.prunepath_residual_layernorm_grad(dev(r, lead), g, dr, T, d, dev(w, lead), dev(stats), dx,
                                         w_o[0] if dw else None, b_o[0] if db else None,
                                         ws[0] if dw or db else None, pp.PP_NORM_F32 if f32 else 0)
    torch.cuda.synchronize()
    assert all(ends_kept(a) for a in (o, w_o, b_o, ws))
    return dx.cpu().numpy(), w_o[0].cpu().numpy(), b_o[0].cpu().numpy()


def check_backward(T, d, seed, f32, w=True, dres=True, **kw):
    x, du, wv, _ = data(T, d, seed)
    rng = np.random.default_rng(seed + 1)
    dr = rng.standard_normal((T, d)).astype(np.float32) if dres else None
    wv = wv if w else None
    if not f32:  # what the call gets
        bits = du.view(np.uint32) & np.uint32(0xFFFF0000)
        du = bits.view(np.float32)
    _, mu, rstd = op.layernorm(x, EPS)
    stats = np.concatenate([mu, rstd], 1).astype(np.float32)
    dx, dw, db = backward(x, du, dr, wv, stats, f32, **kw)
    rx, rw, rb = op.layernorm_grad(x, du, dr, EPS, wv)
    # hat carries the rounding of r - mu, of mu and of rstd, at most 4 HALF m (see above) and its own
    # two; a one; the means chains of d / 256 and a tree of 16; the result is a sum of 4 terms
    hat, _, _ = op.layernorm(x, EPS)
    m = np.maximum(np.abs(x).max(1, keepdims=True) * rstd, 1.0)
    a = np.abs(du if wv is None else du * wv.astype(np.float64))
    c = (24 + d / 128) * HALF
    size = a + a.mean(1, keepdims=True) + (np.abs(hat) + m) * (a * (np.abs(hat) + m)).mean(1, keepdims=True)
    tol = 2 * c * rstd * size + HALF * 2 * np.abs(rx)
    assert (np.abs(dx - rx) <= tol).all(), (np.abs(dx - rx) / tol).max()
    # T terms: each product off by 8 HALF m, the sum by its longest chain (at most T additions)
    g = np.abs(du).astype(np.float64)
    if kw.get("dw", True):
        n = (T + 16) * HALF
        assert (np.abs(dw - rw) <= (g * (np.abs(hat) * n + 8 * HALF * m)).sum(0) + 1e-37).all()
    if kw.get("db", True):
        assert (np.abs(db - rb) <= (T + 16) * HALF * g.sum(0) + 1e-37).all()
    return dx, dw, db


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("f32", [False, True])
def test_gradient(d, f32):
    print("layernorm_grad d=%d f32=%d" % (d, f32), flush=True)
    T = 9 if d < 9000 else 2
    check_backward(T, d, d, f32)
    check_backward(T, d, d + 1, f32, w=False, dres=False)
    check_backward(T, d, d + 2, f32, lead=1)
    check_backward(T, d, d + 3, f32, alias=True)


@pytest.mark.parametrize("T", [1, 2, 31, 64, 65, 511, 512, 513, 2047, 6000])
def test_gradient_rows(T):
    a = check_backward(T, 132, T, False)
    b = check_backward(T, 132, T, False)
    assert all(p.tobytes() == q.tobytes() for p, q in zip(a, b))
    check_backward(T, 67, T, True)


@pytest.mark.parametrize("kw", [dict(dw=False), dict(db=False), dict(dw=False, db=False)])
def test_gradient_parts(kw):
    for d in (96, 97, 2048, 5000, 9001):
        check_backward(21, d, d, False, **kw)


def test_gradient_against_differences_of_the_call():
    """sum(u du) of the fp32 call itself, by central differences in x, w and b."""
    T, d = 2, 12
    x, du, w, b = data(T, d, 50, 1.0)
    _, mu, rstd = op.layernorm(x, EPS)
    stats = np.concatenate([mu, rstd], 1).astype(np.float32)
    dx, dw, db = backward(x, du, None, w, stats, True)
    f = lambda x, w, b: float((forward(x, None, w, b, True)[1].astype(np.float64) * du).sum())  # noqa: E731
    h = np.float32(2.0 ** -7)
    # h^2 / 6 of a third derivative: rstd <= 2 here, so below 50 |du|_1; the sums' errors over 2 h
    tol = float(h) ** 2 / 6 * 50 * np.abs(du).sum() + 40 * 2e-7 * np.abs(du).sum() / (2 * float(h))
    tol = min(tol, 0.2)
    for t in range(T):
        for j in (0, 5, 11):
            p, q = x.copy(), x.copy()
            p[t, j] += h
            q[t, j] -= h
            assert abs((f(p, w, b) - f(q, w, b)) / (2 * float(h)) - dx[t, j]) <= tol
    for j in (0, 7):
        e = np.eye(d, dtype=np.float32)[j] * h
        assert abs((f(x, w + e, b) - f(x, w - e, b)) / (2 * float(h)) - dw[j]) <= 1e-3
        assert abs((f(x, w, b + e) - f(x, w, b - e)) / (2 * float(h)) - db[j]) <= 1e-3


def test_replayed_graph_gives_the_eager_bits():
    import torch
    T, d = 700, 1024
    x, y, w, b = (dev(a) for a in data(T, d, 60))
    du, dres = dev(data(T, d, 61)[0]).bfloat16(), dev(data(T, d, 62)[0])
    xo, u = torch.zeros_like(x), torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    st, dx = torch.zeros((T, 2), device="cuda"), torch.zeros_like(x)
    dw, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    ws = torch.zeros(pp.prunepath_residual_layernorm_grad_workspace(T, d), dtype=torch.uint8,
                     device="cuda")

    def both():
        pp.prunepath_residual_layernorm(x, y, xo, T, d, EPS, w, b, u, st)
        pp.prunepath_residual_layernorm_grad(xo, du, dres, T, d, w, st, dx, dw, db, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    outs = (xo, u, st, dx, dw, db)
    for seed in range(3):
        x.copy_(dev(data(T, d, 70 + seed)[0]))
        both()
        eager = [a.clone() for a in outs]
        for a in outs:
            a.fill_(-5)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, e in zip(outs, eager):
            assert torch.equal(a, e)


def test_offsets_past_32_bits():
    """More than 2^31 values: the last rows as in a call of their own, forward and back."""
    import torch
    T, d, n = 525000, 4096, 3
    x = torch.randn((T, d), device="cuda")
    u = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    w, b, st = torch.randn(d, device="cuda"), torch.randn(d, device="cuda"), torch.empty((T, 2), device="cuda")
    pp.prunepath_residual_layernorm(x, None, None, T, d, EPS, w, b, u, st)
    u2, st2 = torch.empty_like(u[:n]), torch.empty_like(st[:n])
    pp.prunepath_residual_layernorm(x[-n:], None, None, n, d, EPS, w, b, u2, st2)
    assert torch.equal(u[-n:], u2) and torch.equal(st[-n:], st2)
    dx, dw, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(pp.prunepath_residual_layernorm_grad_workspace(T, d), dtype=torch.uint8,
                     device="cuda")
    pp.prunepath_residual_layernorm_grad(x, u, None, T, d, w, st, dx, dw, db, ws)
    dx2 = torch.empty_like(x[:n])
    pp.prunepath_residual_layernorm_grad(x[-n:], u2, None, n, d, w, st2, dx2)
    assert torch.equal(dx[-n:], dx2)
    # db: 525000 values of about |b| <= 5, fp32 chains of T / 512 additions and 512 partial sums
    ref = torch.zeros(d, dtype=torch.float64, device="cuda")
    size = torch.zeros(d, dtype=torch.float64, device="cuda")
    for i in range(0, T, 75000):
        ref += u[i:i + 75000].double().sum(0)
        size += u[i:i + 75000].double().abs().sum(0)
    assert ((db.double() - ref).abs() <= (T / 512 + 16) * HALF * size).all()


@pytest.mark.parametrize("T,d", [(20001, 1023), (20001, 1024), (5001, 4095), (5001, 4096),
                                 (2501, 8190), (2501, 8192)])
@pytest.mark.parametrize("f32", [False, True])
def test_long_batches(T, d, f32):
    """Calls that stream past the caches: some rows as in a call of their own, the column sums
    against those of torch in 64 bits."""
    import torch
    torch.manual_seed(d)
    kind, fl = (torch.float32, pp.PP_NORM_F32) if f32 else (torch.bfloat16, 0)
    z = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    x, y, dres, w = (torch.randn((T, d), device="cuda") for _ in range(4))
    w, b = w[0].contiguous(), torch.randn(d, device="cuda")
    du = torch.randn((T, d), device="cuda").to(kind)
    ws = torch.empty(pp.prunepath_residual_layernorm_grad_workspace(T, d), dtype=torch.uint8,
                     device="cuda")

    def both(rows):
        n = rows.stop - rows.start
        xo, u, st, dx = z(n, d), torch.empty((n, d), dtype=kind, device="cuda"), z(n, 2), z(n, d)
        dw, db = z(d), z(d)
        # (rows of the arrays themselves where they are aligned, copies where odd rows are not)
        a = [v[rows] if d % 4 == 0 else v[rows].clone() for v in (x, y, dres, du)]
        pp.prunepath_residual_layernorm(a[0], a[1], xo, n, d, EPS, w, b, u, st, fl)
        pp.prunepath_residual_layernorm_grad(xo, a[3], a[2], n, d, w, st, dx, dw, db, ws, fl)
        return xo, u, st, dx, dw, db
    whole = both(slice(0, T))
    for rows in (slice(0, 3), slice(T - 5, T)):
        for p, q in zip(whole[:4], both(rows)[:4]):
            assert torch.equal(p[rows], q)
    hat = (whole[0].double() - whole[2][:, :1].double()) * whole[2][:, 1:].double()
    g = du.double()
    c = (T / 512 + 32) * HALF
    assert ((whole[5].double() - g.sum(0)).abs() <= c * g.abs().sum(0)).all()
    assert ((whole[4].double() - (g * hat).sum(0)).abs() <= (c + 8 * HALF) * (g * hat).abs().sum(0) +
            8 * HALF * g.abs().sum(0)).all()


@pytest.mark.parametrize("d", [3, 32])
def test_many_short_rows(d):
    T = 150001
    x, y, w, b = data(T, d, d)
    check_forward(x, y, w, b, True)
    check_backward(T, d, d, False)


def test_binding_refuses_short_arrays():
    import torch
    x, u = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 8), dtype=torch.bfloat16, device="cuda")
    w, st = torch.zeros(8, device="cuda"), torch.zeros((4, 2), device="cuda")
    with pytest.raises(ValueError):
        pp.prunepath_residual_layernorm(x, None, None, 5, 8, EPS, w, w, u)
    with pytest.raises(ValueError):
        pp.prunepath_residual_layernorm(x, None, None, 4, 8, EPS, w[:7], w, u)
    with pytest.raises(TypeError):
        pp.prunepath_residual_layernorm(x, None, None, 4, 8, EPS, w, w, u, flags=pp.PP_NORM_F32)
    ws = torch.zeros(1, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        pp.prunepath_residual_layernorm_grad(x, u, None, 4, 8, w, st, torch.zeros_like(x), w.clone(),
                                             None, ws)
