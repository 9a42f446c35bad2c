"""What a LocalBlock holds on the device, read from torch's allocator: between the passes no more than its 8-bit checkpoints and one
number a row; the workspace is shared by blocks of one context.  Counted are the bytes asked for (`requested_bytes`): those of the
blocks that the allocator hands out depend on what it has cached."""
import pytest

from paper_2506_22771_b200 import binding as ffb

pytestmark = pytest.mark.gpu

ROWS, WIDTH, HIDDEN = 2000, 500, 2000
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _type(kind):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _allocated():
    import torch
    return torch.cuda.memory_stats()["requested_bytes.all.current"]


@pytest.mark.parametrize("kind", list(SIZE))
@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_held_between_the_passes(act, kind):
    import torch
    from paper_2506_22771_b200.local_block import LocalBlock
    dtype = _type(kind)
    context = ffb.Context(workspace_bytes=LocalBlock.workspace_bytes(ROWS, WIDTH, HIDDEN, dtype))
    x = torch.randn((ROWS, WIDTH), device="cuda").to(dtype)
    warm = LocalBlock(ROWS, WIDTH, HIDDEN, act=act, dtype=dtype, context=context)     # the matrix products' own workspaces
    warm.forward(x, 0), warm.backward(x)
    del warm
    start = _allocated()
    blocks = [LocalBlock(ROWS, WIDTH, HIDDEN, act=act, dtype=dtype, seed=k, context=context) for k in range(3)]
    made = _allocated() - start
    parameters = 2 * 4 * (2 * WIDTH + 2 * WIDTH * HIDDEN)                              # with their gradients
    assert made <= 3 * (parameters + blocks[0].saved_bytes())
    ys = [x]
    for b in blocks:
        ys.append(b.forward(ys[-1], 1))
    torch.cuda.synchronize()
    between = _allocated() - start - made
    assert between <= 3 * x.numel() * SIZE[kind]                                      # the blocks' outputs
    assert blocks[0].saved_bytes() <= 0.53 * 2 * ROWS * (WIDTH + 2 * HIDDEN)           # of 16-bit activations
    dy = x
    for b in reversed(blocks):
        dy = b.backward(dy)
    ffb.ff_poll_status(context.ctx)
    del ys, dy
    assert _allocated() - start == made
    del blocks, b
    assert _allocated() == start
    context.close()


def test_blocks_of_one_context_compute_what_they_compute_alone():
    import torch
    from paper_2506_22771_b200.local_block import LocalBlock
    sizes = [(300, 500, 784), (300, 500, 96), (120, 500, 300)]
    room = max(LocalBlock.workspace_bytes(*s) for s in sizes)       # the same room everywhere: the same splits, the same bits
    context = ffb.Context(workspace_bytes=room)
    gen = torch.Generator(device="cuda").manual_seed(4)
    shared = [LocalBlock(*s, context=context) for s in sizes]
    xs = [torch.randn((s[0], s[1]), generator=gen, device="cuda").bfloat16() for s in sizes]
    ys = [b.forward(x, 3) for b, x in zip(shared, xs)]
    dxs = [b.backward(x) for b, x in reversed(list(zip(shared, xs)))][::-1]            # all forward passes before the first backward
    for s, x, y, dx, b in zip(sizes, xs, ys, dxs, shared):
        own = ffb.Context(workspace_bytes=room)
        alone = LocalBlock(*s, context=own)
        assert torch.equal(alone.forward(x, 3), y) and torch.equal(alone.backward(x), dx)
        for name in ("dgamma", "dbeta", "dW1", "dW2"):
            assert torch.equal(getattr(alone, name), getattr(b, name)), name
        own.close()
        b.close()                                                                       # the context is not the block's to close
    ffb.ff_poll_status(context.ctx)
    with pytest.raises(ValueError):
        LocalBlock(4 * 300, 500, 784, context=context)
    context.close()
