"""An error that other code of the thread met and left with the runtime is no error of the library's next call: the calls of the
pages and of the rotary positions do their work and say so, and a handle stays in use."""

from __future__ import annotations

import pytest
import torch

from gpu_pages import BF16, Pool, check_attention
from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu


@pytest.fixture
def left():
    """Makes the runtime refuse a device that does not exist, which it keeps as the thread's last error."""
    L = fsx.lib()

    def leave():
        assert L.hipSetDevice(9999) != 0
        assert L.hipPeekAtLastError() != 0
    yield leave
    L.hipGetLastError()


def clear():
    fsx.lib().hipGetLastError()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_lists_change_and_the_handle_stays_in_use(left, fp8):
    p = Pool(seqs=4, pages=30, most=10, fp8=fp8)
    k, v = p.new(20)
    kd, vd = k.cuda(), v.cuda()
    torch.cuda.synchronize()
    left()
    p.pages.extend([0], [20])
    left()
    p.pages.write(0, p.L, kd, vd, [0], fsx.PackedRows([20]))
    left()
    p.pages.fork([0], [1])
    left()
    p.pages.keep([1], [[(0, 3), (10, 9)]])
    left()
    p.pages.extend([], [])      # nothing to launch
    left()
    p.pages.extend([2], [0])
    left()
    p.pages.free([3])
    left()
    p.pages.keep([], [])
    left()
    p.pages.write(0, p.L, kd, vd, [0], fsx.PackedRows([0]))
    left()
    p.pages.free([2])
    clear()
    p.rows[0] = p.stored(k, v)
    p.rows[1] = p.rows[0][:3] + p.rows[0][10:19]
    p.check()
    left()
    p.pages.free([0])
    clear()
    p.rows[0] = []
    p.check()


def test_attention_rotation_and_a_new_handle(left):
    p = Pool(seqs=3, pages=200, most=150, L=1)
    p.extend([0, 1], [1500, 40])
    q = torch.randn(2, 4, 128, generator=p.g).to(BF16).cuda()
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    ws = torch.empty(p.pages.attention_workspace(q, [0, 1]), dtype=torch.uint8, device="cuda")
    x, y = torch.randn(5, 4, 128, device="cuda"), torch.zeros(5, 4, 128, device="cuda")
    at, plan = torch.zeros(1, 5, dtype=torch.int32, device="cuda"), fsx.RotaryPlan.sections((64,))
    torch.cuda.synchronize()
    left()
    p.pages.attention(0, q, out, [0, 1], lse=lse, workspace=ws)
    left()
    fsx.rotary_rows(x, y, at, plan)  # positions of 0: nothing turns
    left()
    other = fsx.Pages(p.k, p.v, 3, 8)
    left()
    other.extend([0], [5])
    clear()
    check_attention(p, 0, q, out, lse, [0, 1])
    assert torch.equal(x, y)
    assert other.tables()[1].tolist() == [5, 0, 0]
