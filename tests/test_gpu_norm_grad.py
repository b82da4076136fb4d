"""sgd_kernel_norm_grad on the GPU, against oracle/ends.py in float64 on the same inputs.

Tolerances, from the kernel's arithmetic (u = 2^-24): a sum over a row has at most S = 40 roundings in a row (16 in a thread and
their products', 5 of the warp, 8 of the warps), so that
  mean is off by S u mean|h|, x = h - mean by that and u |x| (E_x),
  the mean square by (S + 2) u of itself and 2 mean(|x| E_x), rstd by half of that relative and 4 u (rsqrtf is within 2 ulp) (E_r),
  xhat by rstd E_x + |xhat| (E_r + u) (E_xhat),
  mean(dx) by S u mean|dx| (+ 3 u of it: dx has up to two products and a sum), mean(dx xhat) by (S + 6) u mean|dx xhat| + mean(|dx| E_xhat),
  dh by the sum of these through its formula, E_r relative, 8 u of its terms and u of the result.
Sums over rows: E_xhat |dn| of each term, and n + 64 roundings of 2^-24 of the sum of magnitudes (n rows, the workspace's shares and their tree).
"""
import math

import numpy as np
import pytest
import torch

from oracle import ends as oe

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
S = 40
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
KINDS = {"rms": 0, "ln": 1, "ln_plain": 2}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    binding.lib()
    return binding


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(rows, d, dtype, affine, per, residual, seed, wide=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    h = r(rows, d) * (0.5 + torch.rand(rows, 1, generator=g)) + 0.5 * r(rows, 1)
    h[:, d // 3] *= 30.0
    x = dict(h=h, dout=r(rows, d).to(DT[dtype]))
    if "g" in affine:
        x["g"] = (1 + 0.2 * r(d)).bfloat16()
    if "b" in affine:
        x["b"] = (0.2 * r(d)).bfloat16()
    if per:
        n = -(-rows // per)
        x["scale"] = (0.4 * r(n, d + wide))[:, :d] if not wide else 0.4 * r(n, d + wide)
    if residual:
        x["residual"] = r(rows, d)
    x = {k: v.cuda() for k, v in x.items()}
    if wide:
        x["scale"] = x["scale"][:, wide // 2:wide // 2 + d]
    return x


def _outputs(x, per, wide=0):
    rows, d = x["h"].shape
    out = dict(dh=torch.full((rows, d), math.nan, device="cuda"))
    if "g" in x:
        out["dg"] = torch.full((d,), math.nan, device="cuda")
    if "b" in x:
        out["db"] = torch.full((d,), math.nan, device="cuda")
    if per:
        n = x["scale"].shape[0]
        for i, name in enumerate(("dshift", "dscale")):
            out[name] = torch.full((n, d + wide), math.nan, device="cuda")[:, i * (wide // 2):i * (wide // 2) + d]
    return out


def _check(out, x, kind, per, eps=1e-6):
    h, dout, g, b, scale = (_np(x.get(k)) for k in ("h", "dout", "g", "b", "scale"))
    rows, d = h.shape
    want = oe.norm_grad(dout, h, kind, g, b, scale, max(per, 1), eps, _np(x.get("residual")))
    mean = lambda v: v.mean(1, keepdims=True)  # noqa: E731
    mu = np.zeros((rows, 1)) if kind == "rms" else mean(h)
    xc = h - mu
    E_x = U * np.abs(xc) + (0 if kind == "rms" else S * U * mean(np.abs(h)))
    ms = mean(xc * xc)
    rstd = 1 / np.sqrt(ms + eps)
    E_r = 0.5 * ((S + 4) * U * ms + 2 * mean(np.abs(xc) * E_x)) / (ms + eps) + 4 * U
    xhat = xc * rstd
    E_xhat = rstd * E_x + np.abs(xhat) * (E_r + U)
    s = np.arange(rows) // max(per, 1)
    dn = dout if scale is None else dout * (1 + scale[s])
    dx = np.abs(dn if g is None else dn * g)
    E_m1 = 0 if kind == "rms" else (S + 3) * U * mean(dx)
    m1 = 0 if kind == "rms" else np.abs(mean(dn if g is None else dn * g))
    m2 = np.abs(mean((dn if g is None else dn * g) * xhat))
    E_m2 = (S + 6) * U * mean(dx * np.abs(xhat)) + mean(dx * E_xhat)
    terms = rstd * (dx + m1 + np.abs(xhat) * m2)
    E_dh = rstd * (E_m1 + np.abs(xhat) * E_m2 + E_xhat * m2) + terms * (E_r + 8 * U) + U * np.abs(want["dh"])

    def near(name, got, tol):
        err = np.abs(_np(got) - want[name])
        assert np.isfinite(err).all() and (err <= tol).all(), (name, float(np.max(err / np.maximum(tol, 1e-300))))
    near("dh", out["dh"], E_dh)
    if "dg" in out:
        near("dg", out["dg"], (np.abs(dn) * E_xhat).sum(0) + (rows + 64) * U * np.abs(dn * xhat).sum(0))
    if "db" in out:
        near("db", out["db"], (rows + 64) * U * np.abs(dn).sum(0))
    if per:
        n = xhat * (1 if g is None else g)
        E_n = E_xhat * (1 if g is None else np.abs(g))
        b1 = 0 if b is None else np.abs(b)
        tol = {k: np.zeros((len(scale), d)) for k in ("dshift", "dscale")}
        np.add.at(tol["dshift"], s, np.abs(dout) * (min(per, rows) + 64) * U)
        np.add.at(tol["dscale"], s, np.abs(dout) * (E_n + (min(per, rows) + 64) * U * (np.abs(n) + b1)))
        near("dshift", out["dshift"], tol["dshift"])
        near("dscale", out["dscale"], tol["dscale"])


def _run(B, rows, d, dtype, kind, affine="", per=0, residual=False, seed=0, wide=0, eps=1e-6):
    x = _inputs(rows, d, dtype, affine, per, residual, seed, wide)
    out = _outputs(x, per, wide)
    n = B.sgd_kernel_norm_grad_workspace(rows, d, per)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # (NaN)
    B.sgd_kernel_norm_grad(kind=KINDS[kind], rows_per_batch=max(per, 1), workspace=ws, eps=eps, **x, **out)
    _check(out, x, kind, per, eps)
    return x, out


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kind,affine", [("rms", "g"), ("rms", ""), ("ln", "gb"), ("ln", "g"), ("ln_plain", "")])
@pytest.mark.parametrize("d", [4, 8, 60, 128, 132, 256, 288, 512, 516, 1000, 1024, 1028, 1152, 1280, 2048, 2052, 4092, 4096])
def test_widths(B, d, kind, affine, dtype):
    _run(B, 37, d, dtype, kind, affine, residual=d % 8 == 0, seed=d)


@pytest.mark.parametrize("kind,affine", [("rms", "g"), ("ln", "gb")])
@pytest.mark.parametrize("rows,d", [(1, 4096), (2, 64), (303, 4096), (304, 4096), (305, 4096), (700, 4096), (2431, 64), (2433, 64), (5000, 288), (1216, 1152)])
def test_rows(B, rows, d, kind, affine):
    _run(B, rows, d, "bf16", kind, affine, residual=True, seed=rows)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kind,affine", [("ln_plain", ""), ("ln", "gb"), ("rms", "g")])
@pytest.mark.parametrize("rows,per,d", [(1, 1, 64), (5, 1, 8), (5, 2, 256), (7, 100, 1152), (64, 64, 1152), (65, 64, 1152), (512, 256, 1152), (600, 7, 100),
                                        (3000, 1, 64), (40, 8, 4096), (1000, 999, 2048), (2048, 3, 288)])
def test_modulated(B, rows, per, d, kind, affine, dtype):
    _run(B, rows, d, dtype, kind, affine, per=per, residual=rows % 2 == 0, seed=rows + per)


def test_parts_of_a_wider_modulation(B):
    """scale, dshift and dscale as columns of wider tensors, at addresses that are not multiples of 16 bytes."""
    for wide in (2, 6, 130):
        _run(B, 50, 64, "f32", "ln_plain", per=20, wide=wide)


@pytest.mark.parametrize("name", ["dh", "dg", "db", "dshift", "dscale"])
def test_one_output_alone(B, name):
    x, want = _run(B, 90, 256, "f16", "ln", "gb", per=32, residual=False)
    only = {name: torch.full_like(want[name], math.nan)}
    B.sgd_kernel_norm_grad(kind=1, rows_per_batch=32, **x, **only)
    assert torch.equal(only[name], want[name])
    x, want = _run(B, 90, 256, "f16", "ln", "gb")
    if name in want:
        only = {name: torch.full_like(want[name], math.nan)}
        B.sgd_kernel_norm_grad(kind=1, **x, **only)
        assert torch.equal(only[name], want[name])


def test_residual_in_place(B):
    x, want = _run(B, 333, 1152, "bf16", "rms", "g", residual=True)
    dh = x.pop("residual").clone()
    B.sgd_kernel_norm_grad(kind=0, dh=dh, residual=dh, **x)
    assert torch.equal(dh, want["dh"])


@pytest.mark.parametrize("kind", ["rms", "ln"])
def test_rows_of_a_constant_and_of_zeros(B, kind):
    """Rows without variance: eps alone is under the root."""
    h = torch.zeros(6, 64, device="cuda")
    h[2:4] = 3.0
    h[4:] = -1e-3
    x = dict(h=h, dout=torch.randn(6, 64, device="cuda"), g=torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    out = _outputs(x, 0)
    B.sgd_kernel_norm_grad(kind=KINDS[kind], eps=1e-5, **x, **out)
    _check(out, x, kind, 0, eps=1e-5)


def test_nan_stays_in_its_row(B):
    x, want = _run(B, 40, 512, "f16", "ln", "gb")
    x["dout"][7, 3] = math.nan
    x["h"][9, 5] = math.inf
    dh = torch.empty_like(want["dh"])
    B.sgd_kernel_norm_grad(kind=1, dh=dh, **x)
    ok = torch.ones(40, dtype=torch.bool, device="cuda")
    ok[[7, 9]] = False
    assert torch.equal(dh[ok], want["dh"][ok]) and dh[7].isnan().all() and dh[9].isnan().any()


def test_no_rows(B):
    none = torch.empty(0, 64, device="cuda")
    g, dg = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    db = torch.ones(64, device="cuda")
    B.sgd_kernel_norm_grad(none, none, 1, dh=none.clone(), g=g, b=g, dg=dg, db=db)
    assert (dg == 0).all() and (db == 0).all()


def test_against_differences_of_the_forward(B):
    """The gradient of sum(out dout), out as sgd_kernel_norm writes it (fp16: steps of 0.02 keep its rounding, 2^-11 of values up to
    4, below a hundredth of the differences of most columns; their sum over the row is compared)."""
    rows, d = 4, 256
    gen = torch.Generator().manual_seed(3)
    h = torch.randn(rows, d, generator=gen).cuda()
    g = (1 + 0.2 * torch.randn(d, generator=gen)).bfloat16().cuda()
    b = (0.2 * torch.randn(d, generator=gen)).bfloat16().cuda()
    dout = torch.randn(rows, d, generator=gen).cuda()
    direction = torch.randn(rows, d, generator=gen).cuda()
    for kind in ("rms", "ln"):
        kw = dict(g=g, b=b if kind == "ln" else None)
        dh = torch.empty_like(h)
        B.sgd_kernel_norm_grad(dout, h, KINDS[kind], dh=dh, **kw)

        def loss(at):
            out = torch.empty(rows, d, dtype=torch.float16, device="cuda")
            B.sgd_kernel_norm(at.contiguous(), out, rows, d, KINDS[kind], **kw)
            return (out.double() * dout.double()).sum(1)
        e = 0.02
        got = (dh * direction).double().sum(1)
        want = (loss(h + e * direction) - loss(h - e * direction)) / (2 * e)
        # roundings of 2^-11 |out| / 2 at random signs, |out| about 1: sqrt(2 d) 2^-12 |dout| / (2 e) (six of these deviations), and the
        # difference's own error, e^2 / 6 of a third derivative of the order of the terms' sum
        tol = 6 * math.sqrt(2 * d) * 2.0 ** -12 / (2 * e) + e * e * d
        assert (got - want).abs().max() <= tol


def test_same_on_every_run_streams_and_graphs(B):
    x, want = _run(B, 2000, 1152, "bf16", "ln", "gb", per=256, residual=True)
    outs = [_outputs(x, 256) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in outs]
    torch.cuda.synchronize()
    for o, s in zip(outs, streams):
        B.sgd_kernel_norm_grad(kind=1, rows_per_batch=256, stream=s, **x, **o)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(o[k], want[k]) for k in want)
    o = _outputs(x, 256)
    ws = torch.empty(B.sgd_kernel_norm_grad_workspace(2000, 1152, 256), dtype=torch.uint8, device="cuda")
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        B.sgd_kernel_norm_grad(kind=1, rows_per_batch=256, workspace=ws, **x, **o)
    gr.replay()
    assert all(torch.equal(o[k], want[k]) for k in want)


def test_binding_refuses(B):
    h, dout = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, device="cuda")
    g = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(h=h.half()), dict(dout=dout.double()), dict(g=g.float()), dict(dh=h.half()), dict(scale=torch.zeros(4, 64, device="cuda").half())):
        with pytest.raises(TypeError):
            B.sgd_kernel_norm_grad(**{**dict(dout=dout, h=h, kind=0, dh=torch.empty_like(h), g=g), **kw})
    for kw in (dict(dout=dout[:3]), dict(g=g[:32]), dict(dg=torch.zeros(32, device="cuda")), dict(residual=h[:2]), dict(h=h.t()), dict(dh=h.cpu()),
               dict(scale=torch.zeros(3, 64, device="cuda")), dict(scale=torch.zeros(2, 64, device="cuda"), rows_per_batch=0),
               dict(dshift=torch.zeros(4, 64, device="cuda")),
               dict(scale=torch.zeros(4, 64, device="cuda"), dshift=torch.zeros(4, 64, device="cuda"), dscale=torch.zeros(4, 128, device="cuda")[:, :64])):
        with pytest.raises(ValueError):
            B.sgd_kernel_norm_grad(**{**dict(dout=dout, h=h, kind=0, dh=torch.empty_like(h), g=g), **kw})
    with pytest.raises(B.SgdError):
        B.sgd_kernel_norm_grad(dout, h, 0)
    with pytest.raises(B.SgdError, match="workspace"):
        B.sgd_kernel_norm_grad(dout, h, 0, g=g, dg=torch.zeros(64, device="cuda"), workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.SgdError, match="overlaps"):
        B.sgd_kernel_norm_grad(dout, h, 0, dh=h)
