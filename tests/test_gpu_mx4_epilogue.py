"""The microscaled product with an epilogue, and the gated pair, on the GPU against their 64-bit plain forms."""
import math

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = {"none": sun.SUN_ACT_NONE, "silu": sun.SUN_ACT_SILU, "gelu": sun.SUN_ACT_GELU, "gelu_tanh": sun.SUN_ACT_GELU_TANH}
# up to 16 rows with 16, 32 and 64 columns a workgroup; up to 32, 64 and 128 rows with 64 columns; tiles of 128 x 128; k split in each of the latter (test_mx4_plans_cpu.py has a size for every kernel)
SIZES = [(1, 32, 1), (17, 96, 5), (4500, 160, 7), (8200, 160, 3), (33, 160, 17), (129, 1376, 33), (257, 544, 65), (300, 4096, 20), (300, 4096, 60), (300, 4096, 100), (129, 2080, 130),
         (300, 4096, 200), (515, 352, 700), (1000, 4096, 333)]


def host(t):
    return t.detach().cpu().double().numpy()


def act(y, name):
    """64 bits; erf through math.erfc, which keeps the digits of what is near 0."""
    if name == "silu":
        with np.errstate(over="ignore"):
            return y / (1 + np.exp(-y))
    if name == "gelu_tanh":
        with np.errstate(over="ignore"):
            return y / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if name == "gelu":
        return 0.5 * y * np.vectorize(math.erfc, otypes=[float])(-y / math.sqrt(2))
    return y


def act_bound(y, out, off, name):
    """What an activation makes of a sum that is off by `off` (their slopes are below 1.13), and its own error: an exponential of argument z (|z| <= 1.45 |y|, for
    the tanh form 2.31 |y| + 0.104 |y|^3) in 32 bits is off by 4 |z| 2^-24 + 2^-22 of itself, which the quotient passes on at most; GELU's error function is off by
    1.5e-7 and 8 roundings of a polynomial whose terms stay below 1.46: 0.5 |y| (1.5e-7 + 16 * 2^-24)."""
    if name == "none":
        return off
    a = np.abs(y)
    if name == "gelu":
        own = 0.5 * a * (1.5e-7 + 16 * 2.0 ** -24) + np.abs(out) * 2.0 ** -22
    else:
        z = 1.45 * a if name == "silu" else 2.31 * a + 0.104 * a ** 3
        own = np.abs(out) * (4 * np.minimum(z, 140.0) * 2.0 ** -24 + 2.0 ** -21) + 1e-37
    return 1.13 * off + own


def make(n, k, rows, x_dtype, seed=0, pad=0, matrices=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = [sun.sun_mx4_quantize(torch.randn(n, k, generator=g, device=DEV) * k ** -0.5 * 2) for _ in range(matrices)]
    x = torch.randn(rows, k + pad, generator=g, device=DEV).to(DT[x_dtype])[:, :k]
    return w, x


def product(w, x):
    """The sums, and how far 32 bits may be from them in any order: three planes of 32-bit activations are three times as many products."""
    codes, scales = (t.cpu().numpy() for t in w)
    values, x = R.mx4_values(codes, scales), host(x)
    return x @ values.T, (3 * x.shape[1] + 8) * 2.0 ** -24 * (np.abs(x) @ np.abs(values).T)


def buffer(rows, n, dtype, ld):
    return torch.full((rows, max(ld, n)), 7.0, device=DEV, dtype=DT[dtype])[:, :n]


def workspace(nbytes):
    return torch.full((nbytes + 256,), 0xff, dtype=torch.uint8, device=DEV)


def run_fused(w, x, out, **kw):
    nbytes = sun.sun_mx4_linear_workspace_bytes(w[0].shape[0], x.shape[1], x.shape[0])
    ws = workspace(nbytes)
    sun.sun_mx4_linear_fused(*w, x, out, ws[:nbytes], **kw)
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 0xff).all()
    return out


def run_gated(gate, up, x, out, **kw):
    nbytes = sun.sun_mx4_gated_workspace_bytes(gate[0].shape[0], x.shape[1], x.shape[0])
    ws = workspace(nbytes)
    sun.sun_mx4_gated(*gate, *up, x, out, ws[:nbytes], **kw)
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 0xff).all()
    return out


def check(got, ref, off, dtype):
    over = np.abs(host(got) - ref) / (off + np.abs(ref) * R.HALF[dtype] * 1.01 + 1e-37)
    assert (over <= 1).all(), f"{over.max():.2f} of the bound"


def check_fused(n, k, rows, x_dtype, out_dtype, activation, bias, residual, pad=0, ld=0):
    (w,), x = make(n, k, rows, x_dtype, pad=pad)
    g = torch.Generator(device=DEV).manual_seed(5)
    b = torch.randn(n, generator=g, device=DEV).to(DT[out_dtype]) if bias else None
    out = buffer(rows, n, out_dtype, ld)
    r = None
    if residual:
        r = buffer(rows, n, out_dtype, ld + (8 if ld else 0)) if residual == "apart" else out
        r.copy_(torch.randn(rows, n, generator=g, device=DEV))
    rh = host(r) if residual else 0.0
    y, off = product(w, x)
    if bias:
        y = y + host(b)
        off = off + np.abs(y) * 2.0 ** -24
    ref = act(y, activation)
    off = act_bound(y, ref, off, activation)
    run_fused(w, x, out, bias=b, activation=ACTS[activation], residual=r)
    check(out, ref + rh, off + (np.abs(ref) + np.abs(rh)) * 2.0 ** -23, out_dtype)
    if ld > n:
        assert (out.as_strided((rows, ld - n), (ld, 1), out.storage_offset() + n)[:-1] == 7).all(), "written between rows"


@pytest.mark.parametrize("x_dtype, out_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, k, rows", SIZES)
def test_fused_sizes(n, k, rows, x_dtype, out_dtype):
    check_fused(n, k, rows, x_dtype, out_dtype, "silu", True, "apart")


@pytest.mark.parametrize("rows", [3, 40, 100, 260])
@pytest.mark.parametrize("activation", list(ACTS))
@pytest.mark.parametrize("bias, residual", [(False, None), (True, None), (False, "apart"), (True, "itself")])
def test_fused_parts(bias, residual, activation, rows):
    check_fused(200, 544, rows, "bf16", "f32", activation, bias, residual)


@pytest.mark.parametrize("rows", [1, 40, 260])
@pytest.mark.parametrize("n, ld", [(100, 108), (101, 103), (64, 65)])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_fused_strides(n, ld, rows, out_dtype):
    check_fused(n, 160, rows, "bf16", out_dtype, "gelu", True, "apart", pad=24, ld=ld)
    check_fused(n, 160, rows, "f32", out_dtype, "none", False, "itself", pad=4, ld=ld)


def check_gated(n, k, rows, x_dtype, out_dtype, activation, pad=0, ld=0, stacked=False):
    (gate, up), x = make(n, k, rows, x_dtype, pad=pad, matrices=2)
    if stacked:
        both = [torch.cat([a, b]) for a, b in zip(gate, up)]
        gate, up = [t[:n] for t in both], [t[n:] for t in both]
    (y, off), (u, off_u) = product(gate, x), product(up, x)
    a = act(y, activation)
    off = act_bound(y, a, off, activation)
    out = run_gated(gate, up, x, buffer(rows, n, out_dtype, ld), activation=ACTS[activation])
    check(out, a * u, off * (np.abs(u) + off_u) + np.abs(a) * off_u + np.abs(a * u) * 2.0 ** -23, out_dtype)
    if ld > n:
        assert (out.as_strided((rows, ld - n), (ld, 1), out.storage_offset() + n)[:-1] == 7).all(), "written between rows"


@pytest.mark.parametrize("x_dtype, out_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, k, rows", SIZES)
def test_gated_sizes(n, k, rows, x_dtype, out_dtype):
    check_gated(n, k, rows, x_dtype, out_dtype, "silu")


@pytest.mark.parametrize("rows", [3, 40, 100, 260])
@pytest.mark.parametrize("activation", list(ACTS))
def test_gated_activations(activation, rows):
    check_gated(200, 544, rows, "bf16", "f32", activation, stacked=True)


@pytest.mark.parametrize("rows", [1, 40, 260])
@pytest.mark.parametrize("n, ld", [(100, 108), (101, 103), (64, 65)])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_gated_strides(n, ld, rows, out_dtype):
    check_gated(n, 160, rows, "bf16", out_dtype, "gelu", pad=24, ld=ld)
    check_gated(n, 160, rows, "f32", out_dtype, "silu", pad=4, ld=ld)


@pytest.mark.parametrize("activation", ["silu", "gelu", "gelu_tanh"])
def test_activations_far_from_zero(activation):
    """Sums from -3e4 to 3e4, among them 0: one product each, exact, so that the activation's own error is all there is."""
    k = 32
    w = torch.zeros(64, k, device=DEV)
    w[:, 0] = 1
    codes, scales = sun.sun_mx4_quantize(w)
    y = np.concatenate([np.linspace(-12, 12, 400), np.geomspace(1e-6, 3e4, 200), -np.geomspace(1e-6, 3e4, 200), [0.0]]).astype(np.float32)
    x = torch.zeros(len(y), k, device=DEV)
    x[:, 0] = torch.from_numpy(y)
    out = run_fused((codes, scales), x, torch.empty(len(y), 64, device=DEV), activation=ACTS[activation])
    ref = act(y.astype(np.float64), activation)[:, None]
    check(out, np.repeat(ref, 64, 1), act_bound(y.astype(np.float64)[:, None], ref, 0.0, activation), "f32")
    x[:, 0] = math.inf
    assert (run_fused((codes, scales), x, torch.empty(len(y), 64, device=DEV), activation=ACTS[activation]) == math.inf).all()
    x[:, 0] = -math.inf   # 0 times infinity, as the formula has it
    assert torch.isnan(run_fused((codes, scales), x, torch.empty(len(y), 64, device=DEV), activation=ACTS[activation])).all()


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_not_a_numbers_stay_where_they_belong(rows):
    """A row, a bias, a residual and a block of weights that are not numbers."""
    n, k = 130, 256
    (gate, up), x = make(n, k, rows + 1, "bf16", matrices=2)
    b, r = torch.randn(n, device=DEV), torch.randn(rows + 1, n, device=DEV)
    fused = lambda: run_fused(gate, x, torch.empty(rows + 1, n, device=DEV), bias=b, activation=sun.SUN_ACT_SILU, residual=r)
    pair = lambda: run_gated(gate, up, x, torch.empty(rows + 1, n, device=DEV))
    clean, clean2 = fused().clone(), pair().clone()
    bad, bad2 = torch.zeros(rows + 1, n, dtype=torch.bool, device=DEV), torch.zeros(rows + 1, n, dtype=torch.bool, device=DEV)
    x[rows, 77] = math.nan
    bad[rows], bad2[rows] = True, True
    b[5] = math.nan
    bad[:, 5] = True
    r[0, 9] = math.inf
    gate[1][17, 3] = 255
    bad[:, 17], bad2[:, 17] = True, True
    up[1][18, 3] = 255
    bad2[:, 18] = True
    got, got2 = fused(), pair()
    assert torch.equal(torch.isnan(got), bad) and (bad[0, 9] or got[0, 9] == math.inf)
    bad[0, 9] = True
    assert torch.equal(got[~bad], clean[~bad])
    assert torch.equal(torch.isnan(got2), bad2) and torch.equal(got2[~bad2], clean2[~bad2])


@pytest.mark.parametrize("rows", [4, 64, 300])
def test_again_gives_the_same_bits(rows):
    (gate, up), x = make(300, 4096, rows, "f32", matrices=2)
    first = run_gated(gate, up, x, torch.empty(rows, 300, device=DEV))
    assert torch.equal(first, run_gated(gate, up, x, torch.empty(rows, 300, device=DEV)))
    assert torch.equal(run_fused(gate, x, torch.empty(rows, 300, device=DEV), bias=first[0].contiguous()),
                       run_fused(gate, x, torch.empty(rows, 300, device=DEV), bias=first[0].contiguous()))


def test_binding_refuses_what_does_not_fit():
    (gate, up), x = make(64, 128, 4, "bf16", matrices=2)
    out, ws = torch.empty(4, 64, device=DEV), workspace(1 << 20)

    def refused(call, *args, **kw):
        with pytest.raises(sun.SunError) as e:
            call(*args, **kw)
        assert e.value.status == 2, e.value

    refused(sun.sun_mx4_gated, *gate, up[0][:32], up[1][:32], x, out, ws)
    refused(sun.sun_mx4_gated, *gate, up[0], up[1].float(), x, out, ws)
    refused(sun.sun_mx4_gated, *gate, *up, x, out[:3], ws)
    refused(sun.sun_mx4_gated, *gate, *up, x, out, ws, activation=4)
    refused(sun.sun_mx4_gated, *gate, *up, x, out, ws, activation=1 << 40)
    refused(sun.sun_mx4_gated, *gate, *up, x[0], out, ws)
    refused(sun.sun_mx4_gated, *gate, up[0].cpu(), up[1], x, out, ws)
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, bias=torch.empty(63, device=DEV))
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, bias=torch.empty(64, device=DEV, dtype=torch.bfloat16))
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, residual=torch.empty(4, 64, device=DEV, dtype=torch.bfloat16))
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, residual=torch.empty(5, 64, device=DEV))
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, activation=-1)
    refused(sun.sun_mx4_linear_fused, *gate, x, out, ws, residual=torch.empty(64, 4, device=DEV).t())
