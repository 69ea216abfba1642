"""The microscaled 4-bit format on the GPU against its 64-bit plain form: conversions bit for bit, the product element by element."""
import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().cpu().double().numpy()


def check_quantize(x):
    codes, scales = sun.sun_mx4_quantize(x)
    want_c, want_s = R.mx4_quantize(host(x))
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    for dt in DT.values():
        got = sun.sun_mx4_dequantize(codes, scales, dt)
        assert got.dtype == dt and np.array_equal(host(got), R.mx4_values(want_c, want_s), equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, k", [(1, 32), (3, 64), (7, 96), (129, 1376), (1, 13824), (1000, 32), (5000, 4096)])
def test_quantize_and_values(n, k, dtype):
    g = torch.Generator(device=DEV).manual_seed(n * 7 + k)
    x = torch.randn(n, k, generator=g, device=DEV) * torch.exp2(torch.randint(-20, 20, (n, k // 32, 1), generator=g, device=DEV).float()).expand(-1, -1, 32).reshape(n, k)
    check_quantize(x.to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_edges(dtype):
    """Every bf16 value in a block of its own kind, ties, zeros of both signs, subnormals, the largest numbers, infinities and not-a-numbers."""
    every = (torch.arange(65536, dtype=torch.int32) << 16).view(torch.float32)
    rows = [every.view(-1, 32)]
    grid = torch.tensor([0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.96875])
    for e in (-149, -130, -128, -127, -126, -125, -30, 0, 60, 124):
        rows.append(torch.ldexp(torch.cat([grid, -grid]), torch.tensor(e)).view(1, 32))
    # blocks that mix a large value with small ones
    mixed = every.view(-1, 32).clone()
    mixed[:, 31] = 3.0e38
    mixed[::2, 31] = 1.0
    rows += [mixed, torch.zeros(1, 32), -torch.zeros(1, 32)]
    for bad in (float("inf"), -float("inf"), float("nan")):
        one = torch.ones(1, 32)
        one[0, 17] = bad
        rows.append(one)
    x = torch.cat(rows).to(DEV).to(DT[dtype])
    check_quantize(torch.cat([x, x.flip(0)], 1).contiguous())


def test_values_of_every_code_and_scale():
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).view(16, 16).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8, device=DEV).repeat_interleave(16).view(-1, 1)
    want = R.mx4_values(codes.cpu().numpy(), scales.cpu().numpy())
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)   # 4 and 6 times 2^127 are beyond both types
    for dt in DT.values():
        got = host(sun.sun_mx4_dequantize(codes, scales, dt))
        assert np.array_equal(got, want, equal_nan=True)


def make_linear(n, k, rows, x_dtype, seed=0, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed + n * 31 + k * 7 + rows)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.randint(112, 130, (n, k // 32), generator=g, device=DEV, dtype=torch.uint8)
    x = torch.randn(rows, k + pad, generator=g, device=DEV).to(DT[x_dtype])[:, :k]
    return codes, scales, x


def multiply(codes, scales, x, out_dtype, ld=0):
    n, k, rows = codes.shape[0], codes.shape[1] * 2, x.shape[0]
    whole = torch.full((rows + 1, n + ld), 77.0, device=DEV, dtype=DT[out_dtype])
    out = whole[:rows, :n]
    ws = torch.full((sun.sun_mx4_linear_workspace_bytes(n, k, rows) + 256,), 0xff, device=DEV, dtype=torch.uint8)   # whatever it held
    sun.sun_mx4_linear(codes, scales, x, out, ws)
    torch.cuda.synchronize()
    assert (whole[rows] == 77).all() and (whole[:, n:] == 77).all(), "written behind the rows or columns"
    assert (ws[-256:] == 0xff).all(), "written behind the workspace"
    return out


def check_linear(codes, scales, x, out_dtype, ld=0):
    got = host(multiply(codes, scales, x, out_dtype, ld))
    w, xs = R.mx4_values(codes.cpu().numpy(), scales.cpu().numpy()), host(x)
    ref = xs @ w.T
    over = np.abs(got - ref) / R.linear_bound(xs, w, ref, out_dtype)
    assert (over <= 1).all(), f"{over.max():.2f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


@pytest.mark.parametrize("x_dtype, out_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, k, rows", [(1, 32, 1), (16, 128, 16), (17, 96, 5), (33, 160, 17), (100, 544, 33), (257, 1376, 65), (48, 4096, 1), (129, 2080, 130),
                                        (512, 512, 256), (300, 13824, 3), (4096, 1024, 8), (1000, 256, 300), (1023, 992, 515)])
def test_linear(n, k, rows, x_dtype, out_dtype):
    check_linear(*make_linear(n, k, rows, x_dtype), out_dtype)


@pytest.mark.parametrize("rows", [1, 40, 260])
@pytest.mark.parametrize("x_dtype, out_dtype", [("f32", "bf16"), ("bf16", "f32")])
def test_linear_with_strides(rows, x_dtype, out_dtype):
    check_linear(*make_linear(70, 320, rows, x_dtype, pad=24), out_dtype, ld=5)


@pytest.mark.parametrize("rows", [1, 20, 200, 600])
@pytest.mark.parametrize("x_dtype", ["f32", "bf16"])
def test_linear_not_a_numbers_stay_where_they_belong(rows, x_dtype):
    """A block of scale 255 makes its output column not-a-number, an infinite activation its row, and nothing else."""
    codes, scales, x = make_linear(50, 256, rows, x_dtype)
    scales[7, 3] = 255
    x[rows // 2, 100] = float("inf")
    got = host(multiply(codes, scales, x, "f32"))
    w, xs = R.mx4_values(codes.cpu().numpy(), scales.cpu().numpy()), host(x)
    with np.errstate(invalid="ignore"):
        ref = xs @ w.T
    assert np.isnan(got[:, 7]).all()
    keep = np.ones(rows, bool)
    keep[rows // 2] = False
    cols = np.arange(50) != 7
    assert np.isfinite(got[keep][:, cols]).all()
    assert not np.isfinite(got[rows // 2]).any()
    assert np.array_equal(np.isnan(got[rows // 2]), np.isnan(ref[rows // 2]))


@pytest.mark.parametrize("rows", [3, 64, 300])
def test_linear_extreme_scales(rows):
    """Powers of two from the smallest normal numbers to the largest."""
    codes, scales, x = make_linear(64, 64, rows, "f32")
    scales[:, 0] = torch.arange(4, 68, device=DEV, dtype=torch.uint8)
    scales[:, 1] = torch.arange(4, 68, device=DEV, dtype=torch.uint8)
    check_linear(codes, scales, x * 2.0 ** 20, "f32")
    scales += 150
    check_linear(codes, scales, x * 2.0 ** -20, "f32")


@pytest.mark.parametrize("rows", [1, 9, 100, 400])
def test_linear_again_and_other_rows(rows):
    """The same call twice gives the same bits, and a row does not depend on its neighbours' values."""
    codes, scales, x = make_linear(200, 1056, rows, "bf16")
    a = multiply(codes, scales, x, "f32").clone()
    b = multiply(codes, scales, x, "f32").clone()
    assert torch.equal(a, b)
    y = x.clone()
    y[1:] = torch.randn_like(y[1:].float()).to(y.dtype)
    assert torch.equal(multiply(codes, scales, y, "f32")[0], a[0])


@pytest.mark.parametrize("x_dtype, out_dtype", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, k, rows", [(4500, 160, 7), (8200, 160, 3), (16400, 96, 16), (2000, 4096, 9), (300, 4096, 20), (300, 4096, 60), (300, 4096, 100), (17000, 160, 20), (17000, 288, 60),
                                        (17000, 416, 100), (15000, 160, 2000), (2000, 8192, 500), (4000, 2080, 1100), (6000, 96, 1287), (14700, 160, 642),
                                        (16500, 96, 586), (16900, 160, 687), (5400, 3008, 178), (5500, 3200, 140)])
def test_linear_every_way_of_dealing(n, k, rows, x_dtype, out_dtype):
    """Wide and narrow workgroups, whole and split along k, large and small tiles with and without a last few column tiles."""
    check_linear(*make_linear(n, k, rows, x_dtype), out_dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_many_with_a_ragged_end(dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    check_quantize(torch.randn(1031, 8224, generator=g, device=DEV).to(DT[dtype]))


@pytest.mark.parametrize("dtype, n, k", [("f32", 1873, 32800), ("bf16", 3301, 32800)])
def test_values_past_the_caches(dtype, n, k):
    """Values that leave past the caches, against a table of the codes' values."""
    g = torch.Generator(device=DEV).manual_seed(4)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.randint(100, 140, (n, k // 32), generator=g, device=DEV, dtype=torch.uint8)
    got = sun.sun_mx4_dequantize(codes, scales, DT[dtype])
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    table = torch.cat([table, -table])
    for at in range(0, n, 500):
        c, s = codes[at:at + 500].int(), scales[at:at + 500].float()
        want = torch.stack([table[c & 15], table[c >> 4]], -1).view(-1, k // 32, 32) * torch.exp2(s - 127)[:, :, None]
        assert torch.equal(got[at:at + 500].float(), want.view(-1, k))


def test_offsets_beyond_32_bits():
    """More than 2^32 values to convert, and activations and outputs of more than 2^31 elements: the last rows are like those of a small call."""
    n, k = 131080, 32800
    w = torch.empty(n, k, device=DEV, dtype=torch.bfloat16)
    w[:-9] = 1.0
    w[-9:] = torch.randn(9, k, device=DEV)
    codes, scales = sun.sun_mx4_quantize(w)
    few_codes, few_scales = sun.sun_mx4_quantize(w[-9:].clone())
    assert torch.equal(codes[-9:], few_codes) and torch.equal(scales[-9:], few_scales)
    del w
    values = sun.sun_mx4_dequantize(codes, scales)
    assert torch.equal(values[-9:], sun.sun_mx4_dequantize(few_codes, few_scales)) and (values[:-9:5000] == 1).all()
    del values, codes, scales
    rows, n, k = 70000, 32768, 32
    codes, scales, _ = make_linear(n, k, 1, "bf16")
    x = torch.zeros(rows, n, device=DEV, dtype=torch.bfloat16)[:, :k]
    x[-300:] = torch.randn(300, k, device=DEV).to(x.dtype)
    out = torch.empty(rows, n, device=DEV, dtype=torch.bfloat16)
    sun.sun_mx4_linear(codes, scales, x, out, torch.empty(sun.sun_mx4_linear_workspace_bytes(n, k, rows), device=DEV, dtype=torch.uint8))
    xs, wv = host(x[-300:]), R.mx4_values(codes.cpu().numpy(), scales.cpu().numpy())
    ref = xs @ wv.T
    assert (np.abs(host(out[-300:]) - ref) <= R.linear_bound(xs, wv, ref, "bf16")).all()
    assert (out[:-300:700] == 0).all()


def pool_of(t):
    """The stream whose pool of the allocator the tensor's memory comes from."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_belong_to_the_stream_that_fills_them(dtype, raw):
    """A block of the current stream's pool may still be read by work that is queued there, and would be handed out again while `stream` writes it."""
    x = torch.randn(300, 416, device=DEV).to(DT[dtype])
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    assert side.cuda_stream != here.cuda_stream
    side.wait_stream(here)
    stream = side.cuda_stream if raw else side
    codes, scales = sun.sun_mx4_quantize(x, stream=stream)
    values = sun.sun_mx4_dequantize(codes, scales, DT[dtype], stream=stream)
    assert torch.cuda.current_stream() == here
    here.wait_stream(side)
    assert [pool_of(t) for t in (codes, scales, values)] == [side.cuda_stream] * 3 and pool_of(x) == here.cuda_stream
    want_c, want_s = R.mx4_quantize(host(x))
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(host(values), R.mx4_values(want_c, want_s))
    on = torch.zeros(5, 300, device=DEV)
    workspace = torch.zeros(sun.sun_mx4_linear_workspace_bytes(300, 416, 5), device=DEV, dtype=torch.uint8)
    side.wait_stream(here)
    sun.sun_mx4_linear(codes, scales, x[:5], on, workspace, stream=stream)
    here.wait_stream(side)
    assert torch.equal(on, multiply(codes, scales, x[:5], "f32"))


def test_activations_that_are_no_matrix_are_refused():
    codes, scales, x = make_linear(16, 64, 1, "f32")
    ws, out = torch.zeros(sun.sun_mx4_linear_workspace_bytes(16, 64, 1), device=DEV, dtype=torch.uint8), torch.zeros(1, 16, device=DEV)
    for bad in (x[0, 0], x[0], x[None], x[:, :, None]):
        with pytest.raises(sun.SunError) as e:
            sun.sun_mx4_linear(codes, scales, bad, out, ws)
        assert e.value.status == 2


def test_outputs_dropped_while_the_current_stream_reads_them():
    """What a call on another stream has returned may be dropped once its reader is queued: its memory is not handed out before that is done."""
    xs = [torch.randn(300, 416, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV) for i in range(2)]
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    side.wait_stream(here)
    codes, scales = sun.sun_mx4_quantize(xs[0], stream=side)
    here.wait_stream(side)
    torch.cuda._sleep(50_000_000)   # the reader waits in the queue
    copies = codes.clone(), scales.clone()
    first = {codes.data_ptr(), scales.data_ptr()}
    del codes, scales
    again = sun.sun_mx4_quantize(xs[1], stream=side)
    waiting = not here.query()
    here.wait_stream(side)
    torch.cuda.synchronize()
    assert waiting and not first & {t.data_ptr() for t in again}
    for x, got in zip(xs, (copies, again)):
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, R.mx4_quantize(host(x))))
