"""Every kernel of the microscaled product with an epilogue and as a gated pair: the sizes of test_mx4_plans_cpu.py, which says which of them each gets."""
import pytest
import torch

from test_gpu_mx4_epilogue import ACTS, DEV, DT, act, act_bound, make, run_fused, run_gated
from test_mx4_plans_cpu import SIZES
import lowbit_ref as R

pytestmark = pytest.mark.gpu
CASES = [(size, x_dtype) for size, one, three in SIZES for x_dtype, has in (("bf16", one), ("f32", three)) if has]


def within(got, ref, off, dtype):
    ref, off = (torch.from_numpy(v).to(DEV) for v in (ref, off))
    over = ((got.double() - ref).abs() / (off + ref.abs() * R.HALF[dtype] * 1.01 + 1e-37)).max().item()
    assert over <= 1, f"{over:.2f} of the bound"


def product_on_the_card(w, x):
    """The sums in 64 bits, and how far 32 bits may be from them in any order: three planes are three times as many products."""
    values, x = torch.from_numpy(R.mx4_values(*(t.cpu().numpy() for t in w))).to(DEV).t().contiguous(), x.double()
    return (x @ values).cpu().numpy(), (3 * x.shape[1] + 8) * 2.0 ** -24 * (x.abs() @ values.abs()).cpu().numpy()


@pytest.mark.parametrize("size, x_dtype", CASES)
def test_fused(size, x_dtype):
    n, k, rows = size
    out_dtype = "f32" if rows % 2 else "bf16"
    (w,), x = make(n, k, rows, x_dtype)
    g = torch.Generator(device=DEV).manual_seed(5)
    b, r = torch.randn(n, generator=g, device=DEV).to(DT[out_dtype]), torch.randn(rows, n, generator=g, device=DEV).to(DT[out_dtype])
    y, off = product_on_the_card(w, x)
    bh, rh = b.double().cpu().numpy(), r.double().cpu().numpy()
    y = y + bh
    ref = act(y, "silu")
    off = act_bound(y, ref, off + abs(y) * 2.0 ** -24, "silu") + (abs(ref) + abs(rh)) * 2.0 ** -23
    out = torch.full((rows + 1, n), 7.0, device=DEV, dtype=DT[out_dtype])
    run_fused(w, x, out[:rows], bias=b, activation=ACTS["silu"], residual=r)
    within(out[:rows], ref + rh, off, out_dtype)
    assert (out[rows] == 7).all(), "written behind the last row"


@pytest.mark.parametrize("size, x_dtype", CASES)
def test_gated(size, x_dtype):
    n, k, rows = size[0] // 2, *size[1:]
    out_dtype = "f32" if rows % 2 else "bf16"
    (gate, up), x = make(n, k, rows, x_dtype, matrices=2)
    (y, off), (u, off_u) = product_on_the_card(gate, x), product_on_the_card(up, x)
    a = act(y, "silu")
    off = act_bound(y, a, off, "silu")
    out = torch.full((rows + 1, n), 7.0, device=DEV, dtype=DT[out_dtype])
    run_gated(gate, up, x, out[:rows], activation=ACTS["silu"])
    within(out[:rows], a * u, off * (abs(u) + off_u) + abs(a) * off_u + abs(a * u) * 2.0 ** -23, out_dtype)
    assert (out[rows] == 7).all(), "written behind the last row"
