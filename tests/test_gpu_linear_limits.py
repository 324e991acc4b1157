"""The linear layer at the limit on its output tiles: tall products go to a tiling that takes them; a refused call has changed nothing."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_a_refused_backward_pass_leaves_its_outputs():
    """2^29 rows of one element: 2^22 tiles of 128 x 128 for dx, one tile for dw."""
    m = 1 << 29
    dy = torch.ones((m, 1), dtype=BF, device="cuda")
    dx = torch.full((m, 1), 7, dtype=BF, device="cuda")
    w = torch.ones((1, 1), dtype=BF, device="cuda")
    dw, db = torch.full((1, 1), 7, dtype=BF, device="cuda"), torch.full((1,), 7, dtype=BF, device="cuda")
    size = vf._size_of("vf_linear_workspace", vf.VF_BF16, m, 1, 1, 0, 1)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    rc = vf.load_library().vf_linear_backward(vf.VF_BF16, m, 1, 1, dy.data_ptr(), 1, dy.data_ptr(), 1, w.data_ptr(), 1, None, 1, 0, dx.data_ptr(), 1,
                                              dw.data_ptr(), 1, db.data_ptr(), ws.data_ptr(), size, stream)
    torch.cuda.synchronize()
    assert rc == -1 and b"output tiles" in vf.load_library().vf_last_error()
    assert db.item() == 7 and dw.item() == 7 and (dx == 7).all()


def test_more_rows_than_the_smallest_tiles_take():
    """2^28 + 65 rows: 2^22 + 2 tiles of 64 x 64, half as many of 128 x 128.  Small whole numbers, so that everything is exact but dw and db:
    some 2^18 additions one after the other, each off by up to 2^-24 either way, 2^-15 in all, and an output's rounding of 2^-8."""
    m = (1 << 28) + 65
    x = (torch.arange(m, device="cuda", dtype=torch.int32) % 7).to(BF).view(m, 1)
    w = torch.full((1, 1), 3, dtype=BF, device="cuda")
    y = vf.linear(x, w, torch.ones(1, dtype=BF, device="cuda"))
    assert all(torch.equal(y[a:a + (1 << 24)], 3 * x[a:a + (1 << 24)] + 1) for a in range(0, m, 1 << 24))
    del y
    dx, dw, db = vf.linear_backward(x, x, w)
    assert all(torch.equal(dx[a:a + (1 << 24)], 3 * x[a:a + (1 << 24)]) for a in range(0, m, 1 << 24))
    whole, left = divmod(m, 7)
    first, second = 21 * whole + sum(range(left)), 91 * whole + sum(i * i for i in range(left))
    assert abs(db.item() - first) <= 2 ** -7 * first and abs(dw.item() - second) <= 2 ** -7 * second
