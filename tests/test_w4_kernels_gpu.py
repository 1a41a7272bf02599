"""Products with 4-bit weights through each of their two kernels, whatever the sizes: ReLU, residuals, distances, guards, infinities, real numbers, and
CTAs that go from tile to tile.  Inputs and bounds as in tests/test_w4_gpu.py."""
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding
from tests.test_w4_gpu import DT, SIZES, U, exact_inputs, option, weights64  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

PATHS = [1, 2]
# Of the tcgen05 kernel: up to five blocks of 128 inputs are one CTA's; more are split over a cluster when tiles are few.
FORMS = [(40, 256, 150, 64), (150, 512, 1500, 128), (20, 4096, 300, 32), (101, 2176, 129, 128), (200, 1184, 700, 32)]


@pytest.fixture(params=PATHS)
def path(request, option):
    option("w4_path", request.param)
    yield request.param
    assert_ok()


def assert_ok():
    binding.dresd_w4_status(torch.cuda.current_stream().cuda_stream)


def exact64(x, codes, scales, group):
    return x.double() @ weights64(codes, scales, group).T.cuda()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,inputs,outputs,group", SIZES + FORMS)
def test_relu_and_residual(path, rows, inputs, outputs, group, dtype):
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, dtype, rows + inputs)
    w, want = binding.W4(codes, scales, dtype), exact64(x, codes, scales, group)
    residual = torch.randint(-9, 9, (rows, outputs), generator=torch.Generator().manual_seed(1)).to(DT[dtype]).cuda()
    for relu in (False, True):
        y = want.clamp(min=0) if relu else want
        assert torch.equal(w.matmul(x, relu=relu), y.to(DT[dtype]))
        assert torch.equal(w.matmul(x, residual=residual, relu=relu), (y + residual.double()).to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,inputs,outputs,group", SIZES + FORMS)
def test_real_numbers(path, rows, inputs, outputs, group, dtype):
    g = torch.Generator().manual_seed(rows + inputs)
    x = torch.randn((rows, inputs), generator=g).to(DT[dtype]).cuda()
    q = binding.W4.quantise(torch.randn((inputs, outputs), generator=g).to(DT[dtype]).cuda(), group)
    w64, x64 = weights64(q.codes, q.scales, group).cuda(), x.double()
    want, sums = x64 @ w64.T, (inputs + inputs // group + 16) * 2.0 ** -23 * (x64.abs() @ w64.abs().T)
    off = (q.matmul(x).double() - want).abs()
    assert bool((off <= sums + U[dtype] * (want.abs() + sums) + 2.0 ** -25).all())


@pytest.mark.parametrize("rows,inputs,outputs,group", [(1, 256, 150, 64), (17, 4096, 150, 128)] + FORMS)
def test_distances_and_guards(path, rows, inputs, outputs, group):
    """Rows apart from each other on every side; nothing between them is written, and what lies behind the last row is not read."""
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, "f16", 3)
    want = exact64(x, codes, scales, group)
    apart = torch.full((rows + 1, inputs + 40), float("nan"), dtype=torch.float16, device="cuda")
    apart[:rows, 16:16 + inputs] = x
    x = apart[:rows, 16:16 + inputs]
    w = binding.W4(codes, scales, "f16")
    out = torch.full((rows + 2, outputs + 7), 5.0, dtype=torch.float16, device="cuda")
    residual = torch.full((rows, outputs + 3), 2.0, dtype=torch.float16, device="cuda")
    w.matmul(x, residual=residual[:, 1:1 + outputs], out=out[1:-1, 3:3 + outputs])
    assert torch.equal(out[1:-1, 3:3 + outputs], (want + 2).half())
    out[1:-1, 3:3 + outputs] = 5
    assert bool((out == 5).all())
    onto = residual[:, 1:1 + outputs]
    w.matmul(x, residual=onto, relu=True, out=onto)           # onto the residual itself
    assert torch.equal(onto, (want.clamp(min=0) + 2).half())
    onto.fill_(2)
    assert bool((residual == 2).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,inputs,outputs,group", [(1, 512, 140, 128)] + FORMS)
def test_infinities_and_nan_stay_in_their_rows(path, rows, inputs, outputs, group, dtype):
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, dtype, 5)
    x[0, 5], x[rows // 2, inputs - 3] = float("inf"), float("nan")
    residual = torch.ones((rows, outputs), dtype=DT[dtype], device="cuda")
    got = binding.W4(codes, scales, dtype).matmul(x, residual=residual, relu=True)
    assert bool(got[rows // 2].isnan().all()) and not bool(got[0].isfinite().all())
    clean = torch.ones(rows, dtype=torch.bool)
    clean[0] = clean[rows // 2] = False
    want = (exact64(x, codes, scales, group).clamp(min=0) + 1).to(DT[dtype])
    assert torch.equal(got[clean], want[clean])


@pytest.mark.parametrize("rows,inputs,outputs,group", FORMS)
def test_repeated_captured_and_on_another_stream(path, rows, inputs, outputs, group):
    _, codes, scales = exact_inputs(rows, inputs, outputs, group, "f16", 9)
    w, x = binding.W4(codes, scales, "f16"), torch.randn((rows, inputs), device="cuda").half()
    want = w.matmul(x)
    assert all(torch.equal(w.matmul(x), want) for _ in range(5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = w.matmul(x, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = w.matmul(x)
        two = w.matmul(x, residual=one)
    x.mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(one, -want) and torch.equal(two, w.matmul(x, residual=one))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group,inputs", [(32, 416), (64, 448), (128, 640), (128, 128), (32, 32)])       # 13, 7, 5 groups, and one
@pytest.mark.parametrize("rows,outputs", [(300, 15111), (513, 23041)])      # 180 and 455 tiles of 256 outputs
def test_a_cta_goes_from_tile_to_tile(option, rows, outputs, group, inputs, dtype):
    option("w4_path", 2)
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, dtype, group + rows)
    w, want = binding.W4(codes, scales, dtype), exact64(x, codes, scales, group)
    residual = torch.randint(-9, 9, (rows, outputs), generator=torch.Generator().manual_seed(2)).to(DT[dtype]).cuda()
    assert torch.equal(w.matmul(x), want.to(DT[dtype]))
    assert torch.equal(w.matmul(x, residual=residual, relu=True), (want.clamp(min=0) + residual.double()).to(DT[dtype]))
    assert_ok()


@pytest.mark.parametrize("rows,inputs,outputs", [(16, 4096, 11008), (17, 4096, 11008), (32, 4096, 7324), (32, 4096, 7325), (33, 4096, 3662), (33, 4096, 3663),
                                                 (128, 1024, 7324), (128, 1024, 7325)])
def test_either_side_of_the_choice_of_kernel(rows, inputs, outputs):
    """More than 16 rows, and 30 million weights for every 32 of them."""
    x, codes, scales = exact_inputs(rows, inputs, outputs, 128, "bf16", rows)
    w, want = binding.W4(codes, scales, "bf16"), exact64(x, codes, scales, 128)
    residual = torch.randint(-9, 9, (rows, outputs), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    assert torch.equal(w.matmul(x, residual=residual, relu=True), (want.clamp(min=0) + residual.double()).bfloat16())
    assert_ok()
