"""Slots that have no row are left out of a weight gradient, whatever their dy
holds (moe.weight_grad against 64-bit products on the GPU, and against the
gradient of the slots that are left)."""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import STEP, U, gpu, types  # noqa: F401

pytestmark = pytest.mark.gpu
NOWHERE = [-1, -2 ** 31, 2 ** 31 - 1, None]      # None: one past the last row


def compare(torch, got, x, dy, off, row, rows, out):
    """Every expert's gradient against the products of the slots that have a row."""
    for i in range(len(off) - 1):
        at = torch.arange(off[i], off[i + 1], device="cuda")
        at = at[(row[at] >= 0) & (row[at] < rows)]
        left, right = dy[at].double().t().contiguous(), x[row[at].long()]
        want, size = left @ right, left.abs() @ right.abs()
        bound = (len(at) + 8) * U * size + STEP[out] * want.abs() + 1e-37
        assert ((got[i].double() - want).abs() <= bound).all(), i


# short sums; sums of whole steps, in parts; fewer columns than a vector; wide tiles
@pytest.mark.parametrize("slots,experts,n,cols,pad", [(70, 3, 40, 70, 0), (3100, 3, 72, 136, 8), (3000, 2, 5, 33, 0),
                                                      (5003, 12, 130, 97, 1), (49000, 3, 1024, 1000, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_slots_without_a_row(gpu, slots, experts, n, cols, pad, kind):  # noqa: F811
    torch, moe = gpu
    rng = np.random.default_rng(slots)
    rows = 333
    x = torch.from_numpy(rng.normal(0, 1, (rows, cols))).float().cuda()
    saved = moe.save(x)
    off = np.sort(rng.integers(0, slots + 1, experts + 1))
    off[0], off[-1] = 0, slots
    off[1] = off[2] - 40 if off[2] >= 40 else off[1]        # an expert whose slots all have none
    row = rng.integers(0, rows, slots)
    gone = rng.random(slots) < 0.1
    gone[[0, -1]] = True
    gone[off[1]:off[2]] = True
    gone[slots // 2:slots // 2 + 200] = True                # whole steps
    row[gone] = [rows if v is None else v for v in np.array(NOWHERE, dtype=object)[rng.integers(0, 4, gone.sum())]]
    big = torch.full((slots, n + pad), float("nan"), dtype=types(torch)[kind], device="cuda")
    dy = big[:, :n]
    dy.copy_(torch.from_numpy(rng.normal(0, 0.02, (slots, n))))
    at = torch.from_numpy(np.flatnonzero(gone)).cuda()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0], device="cuda").to(dy.dtype)
    dy[at] = bad[torch.from_numpy(rng.integers(0, 4, (len(at), n))).cuda()]
    row = torch.from_numpy(row.astype(np.int32)).cuda()
    for out in ("f32", "bf16"):
        got = moe.weight_grad(saved, dy, torch.from_numpy(off.astype(np.int32)).cuda(), row, out_dtype=types(torch)[out])
        compare(torch, got, moe.restore(saved).double(), dy, off, row, rows, out)
        assert (got[1] == 0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_slots_beyond_the_rows(gpu, kind):  # noqa: F811
    """Without a map slot s has row s: those past the last row have none."""
    torch, moe = gpu
    g = torch.Generator(device="cuda").manual_seed(4)
    saved = moe.save(torch.randn((1500, 60), generator=g, device="cuda"))
    dy = torch.randn((2100, 24), generator=g, device="cuda").to(types(torch)[kind])
    dy[1500:] = float("nan")
    off = np.array([0, 700, 1400, 2100])
    got = moe.weight_grad(saved, dy, torch.from_numpy(off).int().cuda())
    compare(torch, got, moe.restore(saved).double(), dy, off, torch.arange(2100, device="cuda"), 1500, "f32")


def test_oracle_leaves_them_out(gpu):  # noqa: F811
    torch, moe = gpu
    rng = np.random.default_rng(3)
    q, e = plain.save(rng.normal(0, 1, (9, 40)))
    dy = rng.normal(0, 1, (12, 10)).astype(np.float32)
    row = np.array([0, 1, -1, 2, 3, 9, 4, 5, 6, -5, 7, 8])
    dy[[2, 5, 9]] = [[np.nan], [np.inf], [-np.inf]]
    off = np.array([0, 6, 12])
    got = moe.weight_grad(moe.Saved(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda(), 40), torch.from_numpy(dy).cuda(),
                          torch.from_numpy(off).int().cuda(), torch.from_numpy(row).int().cuda()).double().cpu().numpy()
    x = plain.restore(q, e, 40)
    want = plain.weight_grad(x, dy, off, row)
    size = plain.weight_grad(np.abs(x), np.abs(dy), off, row)
    assert np.isfinite(want).all() and (np.abs(got - want) <= 20 * U * size).all()
