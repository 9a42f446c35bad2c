"""GPU tests of the block operators at sizes where the kernels' loops repeat: CTAs and CTA pairs that take several steps or tiles,
rings that wrap, more tile rows than one group of the tile order.  Expected values come from 64-bit operations on the device.
Tolerances are those of test_gpu_block_ops.py; its count of 96 roundings on any path of a sum over rows holds here too: at most 28 rows
a team, 5 halvings, 37 of the parts a lane and 16 lanes."""
import pytest

from paper_2506_22771_b200 import binding as ffb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": (ffb.FF_F32, 2.0 ** -24, 0.0), "bf16": (ffb.FF_BF16, 2.0 ** -8, 0.0), "f16": (ffb.FF_F16, 2.0 ** -11, 2.0 ** -25)}


def _type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


@pytest.fixture(scope="module")
def ctx():
    c = ffb.Context(workspace_bytes=512 << 20)
    yield c.ctx
    c.close()


@pytest.fixture
def gen():
    import torch
    return torch.Generator(device="cuda").manual_seed(11)


def _pitched(rows, cols, kind, pad, values=None):
    import torch
    t = torch.full((rows, cols + pad), 7.0, dtype=_type(kind), device="cuda")[:, :cols]
    return t if values is None else t.copy_(values)


def _saved(ctx, x):
    """Checkpoint of x and its values in 64 bits."""
    import torch
    rows, cols = x.shape
    c = ffb.Ckpt8(rows, cols, "cuda")
    ffb.ff_ckpt8_save(ctx, x.data_ptr(), x.stride(0), ffb.FF_F32, rows, cols, c.struct)
    unit = torch.exp2(c.e.double() - 127).repeat_interleave(32, dim=1)[:, :cols]
    return c, c.q.double() * unit


def _within(got, want, room, what):
    far = (got.double() - want).abs() - room
    assert float(far.max()) <= 0.0, (what, float(far.max()), int((far > 0).sum()))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(9001, 64, 0), (9001, 200, 1), (6001, 300, 0), (3601, 500, 0), (2401, 784, 8), (2001, 1000, 3), (1101, 2000, 0),
                                           (1001, 2001, 0), (601, 4096, 0), (501, 8192, 0), (301, 8191, 2)])
def test_layernorm_forward_over_many_rows(ctx, gen, rows, cols, pad, kind):
    """Two rows a team, the last one alone.  Without gamma and beta FP32's y is the normalised value, whose checkpoint is then the one that
    ff_ckpt8_save makes of it, in every rounding mode."""
    import torch
    code, w, step = TYPES[kind]
    X = _pitched(rows, cols, kind, pad, torch.randn((rows, cols), generator=gen, device="cuda") + 0.25)
    gamma, beta = 1 + 0.3 * torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    xd = X.double()
    m = xd.mean(dim=1, keepdim=True)
    r = ((xd - m).square().mean(dim=1, keepdim=True) + 1e-5).rsqrt()
    xh, most = (xd - m) * r, xd.abs().amax(dim=1, keepdim=True)
    dxh = 64 * U * (xh.abs() * (2 + r * most) + r * most)
    for mode, affine in ((ffb.FF_ROUND_NEAREST_EVEN, True), (ffb.FF_ROUND_STOCHASTIC, False), (ffb.FF_ROUND_STOCHASTIC | ffb.FF_ROUND_KEEP_SIGN, False)):
        Y, c = _pitched(rows, cols, kind, pad), ffb.Ckpt8(rows, cols, "cuda")
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        b = ffb.ff_layernorm_bufs(X=X.data_ptr(), ld_x=X.stride(0), Y=Y.data_ptr(), ld_y=Y.stride(0), mean=mean.data_ptr(), rstd=rstd.data_ptr(), C=c.struct)
        if affine:
            b.gamma, b.beta = gamma.data_ptr(), beta.data_ptr()
        d = ffb.ff_layernorm_desc(cols=cols, dtype=code, eps=1e-5, round=mode, seed=5, index=2)
        ffb.ff_layernorm_forward(ctx, d, b, rows, 9)
        ffb.ff_poll_status(ctx)
        _within(mean, m[:, 0], 64 * U * most[:, 0], "mean")
        _within(rstd, r[:, 0], (64 * U * r * (2 + r * most))[:, 0], "rstd")
        y = xh * gamma.double() + beta.double() if affine else xh
        dy = dxh * (gamma.double().abs() if affine else 1.0) + 2 * U * y.abs()
        _within(Y, y, dy + w * (y.abs() + dy) + step, "y")
        unit = torch.exp2(c.e.double() - 127).repeat_interleave(32, dim=1)[:, :cols]
        _within(c.q.double() * unit, xh, (0.5 if mode == ffb.FF_ROUND_NEAREST_EVEN else 1.0) * unit * (1 + 2.0 ** -20) + dxh, "held")
        if kind == "f32" and not affine:
            own = ffb.Ckpt8(rows, cols, "cuda")
            ffb.ff_ckpt8_save(ctx, Y.data_ptr(), Y.stride(0), ffb.FF_F32, rows, cols, own.struct, mode, 5, 2, 9)
            assert torch.equal(own.q, c.q) and torch.equal(own.e, c.e)


# rows of the ring kernel in each of its shapes, of the register kernels (narrow, and rows that bulk copies cannot address)
@pytest.mark.parametrize("ckpt", [True, False])
@pytest.mark.parametrize("kind,rows,cols,pad", [("bf16", 8192, 2000, 0), ("f32", 8192, 2000, 0), ("f16", 6000, 1000, 0), ("f32", 4000, 4096, 0),
                                                ("bf16", 3000, 8192, 0), ("f32", 3000, 8192, 0), ("f32", 20000, 64, 0), ("f16", 6000, 500, 0),
                                                ("bf16", 6000, 200, 0), ("f16", 4000, 1000, 3), ("bf16", 4000, 2001, 0), ("f32", 2500, 4099, 1),
                                                ("bf16", 1501, 8191, 0)])
def test_layernorm_backward_over_many_rows(ctx, gen, kind, rows, cols, pad, ckpt):
    import torch
    code, w, step = TYPES[kind]
    new = lambda: torch.randn((rows, cols), generator=gen, device="cuda")
    gamma = 1 + 0.3 * torch.randn(cols, generator=gen, device="cuda")
    X = _pitched(rows, cols, kind, pad, new() + 0.25)
    dY, A = _pitched(rows, cols, kind, pad, new()), _pitched(rows, cols, kind, pad, new())
    xd = X.double()
    mean = xd.mean(dim=1).float()
    rstd = ((xd - mean.double()[:, None]).square().mean(dim=1) + 1e-5).rsqrt().float()
    r = rstd.double()[:, None]
    xh = (xd - mean.double()[:, None]) * r
    exh = torch.zeros((), device="cuda")
    if ckpt:
        c, xh = _saved(ctx, xh.float())
    else:
        exh = 4 * U * r * (xd.abs() + mean.double().abs()[:, None])
    for add in (False, True):
        dX = _pitched(rows, cols, kind, pad)
        dg, db = torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")
        b = ffb.ff_layernorm_bufs(dY=dY.data_ptr(), ld_dy=dY.stride(0), rstd=rstd.data_ptr(), gamma=gamma.data_ptr(), dX=dX.data_ptr(),
                                  ld_dx=dX.stride(0), dgamma=dg.data_ptr(), dbeta=db.data_ptr())
        if add:
            b.dAdd, b.ld_dadd = A.data_ptr(), A.stride(0)
        if ckpt:
            b.C = c.struct
        else:
            b.X, b.ld_x, b.mean = X.data_ptr(), X.stride(0), mean.data_ptr()
        ffb.ff_layernorm_backward(ctx, ffb.ff_layernorm_desc(cols=cols, dtype=code, eps=1e-5), b, rows)
        ffb.ff_poll_status(ctx)
        d = dY.double()
        gy = d * gamma.double()
        dx = r * (gy - gy.mean(dim=1, keepdim=True) - xh * (gy * xh).mean(dim=1, keepdim=True))
        ga = gy.abs()
        room = r * 64 * U * (ga + ga.mean(dim=1, keepdim=True) + xh.abs() * (ga * xh.abs()).mean(dim=1, keepdim=True))
        if not ckpt:
            room += r * (exh * (ga * xh.abs()).mean(dim=1, keepdim=True) + xh.abs() * (ga * exh).mean(dim=1, keepdim=True))
        if add:
            dx = dx + A.double()
            room += U * A.double().abs()
        _within(dX, dx, room + w * (dx.abs() + room) + step, "dX")
        _within(dg, (d * xh).sum(dim=0), 96 * U * (d * xh).abs().sum(dim=0) + (d.abs() * exh).sum(dim=0), "dgamma")
        _within(db, d.sum(dim=0), 96 * U * d.abs().sum(dim=0), "dbeta")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n,cols", [(200, 4500, 4100), (2500, 2300, 2100), (130, 12000, 800)])
def test_weight_gradient_of_more_tiles_than_pairs(ctx, gen, rows, n, cols, kind):
    """More work items than CTA pairs, more than 16 tile rows; with and without the affine, added to and written over."""
    import torch
    dy = (torch.randn((rows, n), generator=gen, device="cuda") * 0.02).to(_type(kind))
    c, held = _saved(ctx, torch.randn((rows, cols), generator=gen, device="cuda"))
    gamma, beta = 1 + 0.3 * torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    start = torch.randn((n, cols), generator=gen, device="cuda")
    d = dy.double()
    for affine, accumulate in ((False, 0), (True, 1)):
        dw, db = start.clone(), start[:, 0].clone()
        b = ffb.ff_ckpt8_wgrad_bufs(dY=dy.data_ptr(), ld_dy=n, C=c.struct, dW=dw.data_ptr(), dbias=db.data_ptr())
        if affine:
            b.gamma, b.beta = gamma.data_ptr(), beta.data_ptr()
        ffb.ff_ckpt8_wgrad(ctx, ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=TYPES[kind][0], accumulate=accumulate), b, rows)
        ffb.ff_poll_status(ctx)
        want, mag, bias = d.t() @ held, d.abs().t() @ held.abs(), d.sum(dim=0)
        if affine:
            want = want * gamma.double() + bias[:, None] * beta.double()
            mag = mag * gamma.double().abs() + d.abs().sum(dim=0)[:, None] * beta.double().abs()
        if accumulate:
            want, mag, bias = want + start.double(), mag + start.double().abs(), bias + start[:, 0].double()
        _within(dw, want, 256 * U * mag, "dW")
        assert float((dw.double() - want).norm() / want.norm()) <= 4e-6
        _within(db, bias, 256 * U * (d.abs().sum(dim=0) + start[:, 0].double().abs()), "dbias")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols", [(3100, 8000), (5003, 2999)])
def test_activation_backward_over_many_values(ctx, gen, rows, cols, act, kind):
    """More groups than the CTAs that fit the device take in one pass."""
    import math
    import torch
    code, w, step = TYPES[kind]
    c, h = _saved(ctx, 3 * torch.randn((rows, cols), generator=gen, device="cuda"))
    dz = torch.randn((rows, cols), generator=gen, device="cuda").to(_type(kind))
    dh = _pitched(rows, cols, kind, 0)
    d = ffb.ff_activation_desc(kind={"relu": ffb.FF_ACT_RELU, "gelu": ffb.FF_ACT_GELU, "silu": ffb.FF_ACT_SILU}[act], cols=cols, dtype=code)
    ffb.ff_activation_backward(ctx, d, ffb.ff_activation_bufs(dZ=dz.data_ptr(), ld_dz=cols, dH=dh.data_ptr(), ld_dh=cols, CH=c.struct), rows)
    ffb.ff_poll_status(ctx)
    if act == "relu":
        slope = (h > 0).double()
    elif act == "gelu":
        slope = 0.5 * (1 + torch.erf(h / math.sqrt(2.0))) + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)
    else:
        s = torch.sigmoid(h)
        slope = s * (1 + h * (1 - s))
    z = dz.double()
    want = z * slope
    room = z.abs() * (16 + 2 * h.abs()) * U if act != "relu" else torch.zeros((), device="cuda")
    _within(dh, want, room + w * (want.abs() + room) + step, act)
