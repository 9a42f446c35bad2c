"""What a LocalBlock accepts: the kernels see an address and a row pitch only, so everything else is refused before a launch."""
import pytest

from paper_2506_22771_b200.local_block import LocalBlock, _address


def _wrong(torch, rows, cols, dtype, device):
    new = lambda *s, t=dtype, d=device: torch.zeros(s, dtype=t, device=d)
    other = torch.float32 if dtype != torch.float32 else torch.float16
    return [("fewer rows", new(rows - 1, cols)), ("more rows", new(rows + 1, cols)), ("narrower", new(rows, cols - 1)),
            ("wider", new(rows, cols + 1)), ("flat", new(rows * cols)), ("a batch of batches", new(1, rows, cols)),
            ("another type", new(rows, cols, t=other)), ("a wider type", new(rows, cols, t=torch.float64)),
            ("another device", new(rows, cols, d="meta")), ("columns first", new(cols, rows).t()),
            ("every other column", new(rows, 2 * cols)[:, ::2]), ("one row many times", new(1, cols).expand(rows, cols)),
            ("one value many times", new(1, 1).expand(rows, cols))]


def test_addresses_of_inputs():
    import torch
    cpu = torch.device("cpu")
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for name, t in _wrong(torch, 6, 10, dtype, cpu):
            with pytest.raises(ValueError):
                _address(name, t, 6, 10, dtype, cpu)
        whole, wide = torch.zeros(6, 10, dtype=dtype), torch.zeros(6, 16, dtype=dtype)
        assert _address("x", whole, 6, 10, dtype, cpu) == (whole.data_ptr(), 10)
        assert _address("x", wide[:, 3:13], 6, 10, dtype, cpu) == (wide.data_ptr() + 3 * wide.element_size(), 16)
        row = torch.zeros(10, 1, dtype=dtype).t()                      # one row: its pitch says nothing
        assert row.stride() == (1, 1) and _address("x", row, 1, 10, dtype, cpu) == (row.data_ptr(), 10)


@pytest.mark.gpu
def test_block_refuses_wrong_inputs():
    import torch
    from paper_2506_22771_b200 import binding as ffb
    with pytest.raises(ValueError):
        LocalBlock(8, 8, 8, act="tanh")
    with pytest.raises(ValueError):
        LocalBlock(8, 8, 8, dtype=torch.float64)
    for dtype in (torch.float32, torch.bfloat16):
        block = LocalBlock(60, 100, 130, dtype=dtype)
        before = ffb.ff_launch_count(block.ctx.ctx)
        for name, t in _wrong(torch, 60, 100, dtype, "cuda"):
            for call in (lambda: block.forward(t, 0), lambda: block.backward(t)):
                with pytest.raises(ValueError):
                    call()
        assert ffb.ff_launch_count(block.ctx.ctx) == before
        # rows of a wider tensor and one that autograd tracks are taken
        wide = torch.randn((60, 120), device="cuda").to(dtype)
        y = block.forward(wide[:, 8:108], 0)
        dx = block.backward(wide[:, 8:108])
        tracked = wide[:, 8:108].contiguous().requires_grad_()
        again = block.forward(tracked, 0)
        assert torch.equal(again, y) and not again.requires_grad and torch.equal(block.backward(tracked), dx)
        block.close()
