"""GPU tests of the block operators where a call's parts meet: outputs written over inputs, workspaces smaller than the most that a
call can use, infinities beside bias sums.  Tolerances are those of test_gpu_block_ops.py unless a test states its own."""
import numpy as np
import pytest

from oracle import block_ops as O
from paper_2506_22771_b200 import binding as ffb
from tests.test_gpu_block_ops import TYPES, U, Pitched, Saved, _data, _vec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ffb.Context(workspace_bytes=64 << 20)
    yield c.ctx
    c.close()


# ---- layer norm backward in place --------------------------------------------------------------------------------------
@pytest.mark.parametrize("ckpt", [True, False])
@pytest.mark.parametrize("into", ["dy", "add"])
@pytest.mark.parametrize("cols", [64, 500, 2000, 8192, 9000, 20011])
def test_layernorm_parameter_sums_in_place(ctx, cols, into, ckpt):
    """dX over dY or over dAdd leaves all three outputs with the bits of the call that writes elsewhere, and the sums right."""
    import torch
    rows = 37
    g, x = _data(rows, cols, cols + 1)
    dy, add = g.normal(size=(rows, cols)), g.normal(size=(rows, cols))
    _, m, r, xh = O.layernorm_forward(Pitched(rows, cols, "bf16", values=x).np(), None, None, 1e-5)
    X, c, mean, rstd = Pitched(rows, cols, "bf16", values=x), Saved(rows, cols, xh), _vec(m), _vec(r)

    def run(into):
        D, A = Pitched(rows, cols, "bf16", values=dy), Pitched(rows, cols, "bf16", values=add)
        to = {"dy": D, "add": A, None: Pitched(rows, cols, "bf16")}[into]
        dg, db = torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")
        b = ffb.ff_layernorm_bufs(dY=D.ptr, ld_dy=D.ld, dAdd=A.ptr, ld_dadd=A.ld, rstd=rstd.data_ptr(), dX=to.ptr, ld_dx=to.ld,
                                  dgamma=dg.data_ptr(), dbeta=db.data_ptr())
        if ckpt:
            b.C = c.struct
        else:
            b.X, b.ld_x, b.mean = X.ptr, X.ld, mean.data_ptr()
        ffb.ff_layernorm_backward(ctx, ffb.ff_layernorm_desc(cols=cols, dtype=ffb.FF_BF16), b, rows)
        return to.np(), dg.double().cpu().numpy(), db.double().cpu().numpy(), D

    whole, there = run(None), run(into)
    for k in range(3):
        assert np.array_equal(whole[k], there[k])
    d = whole[3].np()
    assert (np.abs(there[2] - d.sum(axis=0)) <= 96 * U * np.abs(d).sum(axis=0)).all()
    if ckpt:
        assert (np.abs(there[1] - (d * c.values).sum(axis=0)) <= 96 * U * np.abs(d * c.values).sum(axis=0)).all()


# ---- weight gradient: infinities ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n,cols,shift", [(70, 40, 96, 0), (70, 40, 95, 0), (70, 40, 96, 1), (5000, 17, 40, 0), (5000, 17, 39, 0)])
def test_infinite_bias_sum_stays_in_the_bias(ctx, rows, n, cols, shift, kind):
    """Without beta, dW does not depend on the sums of dY: an Inf there gives what the products alone give, whether the bias
    gradient is asked for or not, in whole words or value by value, with one split or several."""
    import torch
    g = np.random.default_rng(cols + rows)
    dy = g.normal(size=(rows, n))
    dy[3, 5] = np.inf
    D, c = Pitched(rows, n, kind, values=dy), Saved(rows, cols, g.normal(size=(rows, cols)) + 3.0)
    ga = _vec(1 + 0.3 * g.normal(size=cols))
    want, _ = O.wgrad(D.np(), c.values)
    assert (np.abs(c.values[3]) > 0).all() and np.isinf(want[5]).all()
    for gamma in (False, True):
        out = []
        for bias in (False, True):
            dw, db = torch.full((n * cols + 4,), 7.0, device="cuda"), torch.zeros(n, device="cuda")
            b = ffb.ff_ckpt8_wgrad_bufs(dY=D.ptr, ld_dy=D.ld, C=c.struct, dW=dw[shift:].data_ptr(), dbias=db.data_ptr() if bias else None)
            if gamma:
                b.gamma = ga.data_ptr()
            ffb.ff_ckpt8_wgrad(ctx, ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=TYPES[kind][0]), b, rows)
            ffb.ff_poll_status(ctx)
            out.append(dw[shift:shift + n * cols].double().cpu().numpy().reshape(n, cols))
            if bias:
                b = db.cpu().numpy()
                assert b[5] == np.inf and np.isfinite(np.delete(b, 5)).all()
        assert np.array_equal(out[0], out[1])
        assert np.array_equal(np.isinf(out[1]), np.isinf(want)) and not np.isnan(out[1]).any()
        assert np.array_equal(np.sign(out[1][5]), np.sign(want[5] * (ga.cpu().numpy() if gamma else 1.0)))


# ---- weight gradient: workspaces ---------------------------------------------------------------------------------------
def _wgrad_in(workspace_bytes, rows, n, cols, kind):
    import torch
    g = np.random.default_rng(rows)
    own = ffb.Context(workspace_bytes=workspace_bytes)
    try:
        D, c = Pitched(rows, n, kind, values=g.normal(size=(rows, n))), Saved(rows, cols, g.normal(size=(rows, cols)))
        dw, db = torch.zeros((n, cols), device="cuda"), torch.zeros(n, device="cuda")
        assert own.workspace.numel() == workspace_bytes
        ffb.ff_ckpt8_wgrad(own.ctx, ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=TYPES[kind][0]),
                           ffb.ff_ckpt8_wgrad_bufs(dY=D.ptr, ld_dy=D.ld, C=c.struct, dW=dw.data_ptr(), dbias=db.data_ptr()), rows)
        ffb.ff_poll_status(own.ctx)
        wd, wb = O.wgrad(D.np(), c.values)
        assert (np.abs(dw.double().cpu().numpy() - wd) <= 256 * U * (np.abs(D.np()).T @ np.abs(c.values))).all()
        assert (np.abs(db.double().cpu().numpy() - wb) <= 256 * U * np.abs(D.np()).sum(axis=0)).all()
    finally:
        own.close()


@pytest.mark.parametrize("kind,n,cols,most,rows", [("f32", 500, 784, 1281, 1280), ("f16", 500, 784, 1793, 1792), ("bf16", 300, 200, 2049, 2048),
                                                   ("f32", 40, 24, 4097, 4095)])
def test_workspace_of_the_largest_batch_serves_smaller_ones(kind, n, cols, most, rows):
    """A program allocates for its batch; the last batch of a pass has fewer rows."""
    d = ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=TYPES[kind][0])
    for r in (most, rows, 1):
        _wgrad_in(ffb.ff_ckpt8_wgrad_workspace_bytes(d, most), r, n, cols, kind)


@pytest.mark.parametrize("kind,parts", [("f32", 3), ("f16", 2), ("bf16", 1)])
def test_workspace_without_room_for_splits_still_serves(kind, parts):
    """The input, dY's parts and its column sums have to fit; the splits take what is left, none if nothing is (a device with
    another number of SMs cuts the rows otherwise)."""
    rows, n, cols = 3000, 300, 200
    up = lambda v: -(-v // 256) * 256
    d = ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=TYPES[kind][0])
    header = ffb.ff_ckpt8_wgrad_workspace_bytes(ffb.ff_ckpt8_wgrad_desc(N=1, K=1, dtype=ffb.FF_BF16), 0)
    least = header + up(rows * 208 * 2) + up(parts * rows * 304 * 2) + up(-(-rows // 64) * n * 4)
    asked = ffb.ff_ckpt8_wgrad_workspace_bytes(d, rows)
    assert asked >= least + 2 * n * cols * 4, "the case is one that splits"
    for room in (0, 1, 2 * n * cols * 4 + 256, 3 * n * cols * 4 + 256):
        _wgrad_in(least + room, rows, n, cols, kind)
    with pytest.raises(ffb.FFError) as e:
        _wgrad_in(header + up(rows * 208 * 2), rows, n, cols, "f32")
    assert e.value.code == ffb.FF_ERR_WORKSPACE


# ---- weight gradient: accuracy of FP32 gradients -------------------------------------------------------------------------
@pytest.mark.parametrize("rows,n,cols", [(64, 500, 784), (128, 500, 784), (512, 500, 784), (2048, 300, 520), (8192, 300, 520)])
def test_weight_gradient_of_fp32_is_as_exact_as_fp32_products(rows, n, cols):
    """The lower parts of dY enter a small accumulator, so what truncates is the four steps of the leading part in a stage: 2^-23 of
    the accumulator each at most, half of that on average, 4 * 2^-24 = 2.4e-7 for a chunk.  Chunks are added with rounding to
    nearest (2^-24 each, in both directions): 2^-24 * sqrt(chunks / 3) more, less than 4e-7 altogether at 8192 rows and 2.6e-7 at 128.
    FP32 sums in order have 2^-24 * sqrt(rows / 3) and above."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    dy = torch.randn((rows, n), generator=gen, device="cuda") * 0.02
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    d = ffb.ff_ckpt8_wgrad_desc(N=n, K=cols, dtype=ffb.FF_F32)
    own = ffb.Context(workspace_bytes=ffb.ff_ckpt8_wgrad_workspace_bytes(d, rows))
    c, dw = ffb.Ckpt8(rows, cols, "cuda"), torch.empty((n, cols), device="cuda")
    ffb.ff_ckpt8_save(own.ctx, x.data_ptr(), cols, ffb.FF_F32, rows, cols, c.struct)
    ffb.ff_ckpt8_wgrad(own.ctx, d, ffb.ff_ckpt8_wgrad_bufs(dY=dy.data_ptr(), ld_dy=n, C=c.struct, dW=dw.data_ptr()), rows)
    ffb.ff_poll_status(own.ctx)
    held = c.q.double() * torch.exp2(c.e.double() - 127).repeat_interleave(32, dim=1)[:, :cols]
    want = dy.double().t() @ held
    assert float((dw.double() - want).norm() / want.norm()) <= U * (4 + (rows / 64 / 3) ** 0.5)
    own.close()
