"""Products with 4-bit weights against float64.

Two kinds of inputs.  Whole numbers with scales that are powers of two: every product and sum is exact in fp32 whatever its order, so the
result is the correctly rounded one, bit for bit; one wrong code, input or scale shows.  Real numbers: with A = sum |w x|, a sum of `inputs`
products, of which an instruction adds 16 at a time with at worst a truncation each, and one more rounding for every group and part, is off by at
most (inputs + inputs / group + 16) 2^-23 A; the result is rounded once (2^-11, 2^-8 of it; fp16 below 2^-14 by 2^-25).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import binding

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def weights64(codes, scales, group):
    c = codes.cpu().to(torch.int64)
    q = torch.stack((c & 15, c >> 4), -1).view(codes.shape[0], -1) - 8
    return q.double() * scales.cpu().double().repeat_interleave(group, 1)


def exact_inputs(rows, inputs, outputs, group, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(256, (outputs, inputs // 2), generator=g, dtype=torch.uint8)
    scales = 2.0 ** torch.randint(-2, 2, (outputs, inputs // group), generator=g)
    x = torch.randint(-2, 3, (rows, inputs), generator=g)
    return x.to(DT[dtype]).cuda(), codes.cuda(), scales.to(DT[dtype]).cuda()


SIZES = [(1, 32, 1, 32), (1, 64, 3, 64), (1, 128, 129, 128), (2, 4096, 513, 128), (3, 352, 31, 32), (8, 1024, 1000, 64), (9, 11008, 130, 128), (16, 2080, 257, 32),
         (17, 704, 65, 64), (33, 1152, 100, 128), (64, 512, 300, 64), (65, 96, 128, 32), (101, 2176, 129, 128), (128, 640, 77, 64), (129, 256, 256, 32),
         (257, 1280, 200, 128), (500, 4224, 139, 64), (1, 65536, 40, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,inputs,outputs,group", SIZES)
def test_whole_numbers_are_exact(rows, inputs, outputs, group, dtype):
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, dtype, rows + inputs + outputs)
    w = binding.W4(codes, scales, dtype)
    want = x.cpu().double() @ weights64(codes, scales, group).T
    assert float((x.cpu().double().abs() @ weights64(codes, scales, group).abs().T).max()) < 2 ** 22      # quarters: 24 bits
    got = w.matmul(x)
    assert torch.equal(got.cpu(), want.to(DT[dtype]))
    residual = torch.randint(-9, 9, (rows, outputs), generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    got = w.matmul(x, residual=residual.cuda(), relu=True)
    assert torch.equal(got.cpu(), (want.clamp(min=0) + residual.double()).to(DT[dtype]))


@pytest.fixture
def option():
    def set_option(name, value):
        binding.dresd_set_global_option(name, value)
    yield set_option
    for name in ("w4_path", "w4_wait_ms", "w4_debug_lose_stage"):
        binding.dresd_set_global_option(name, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("rows,inputs,outputs,group", SIZES + [(1, 4096, 4096, 128), (16, 11008, 4096, 64), (112, 4096, 11008, 32), (700, 1024, 3000, 128), (48, 4096, 4096, 32), (17, 4096, 11008, 64), (2047, 512, 1000, 128)])
def test_either_kernel_at_every_size(option, path, rows, inputs, outputs, group):
    dtype = "f16" if (rows + inputs) % 3 else "bf16"
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, dtype, rows)
    option("w4_path", path)
    got = binding.W4(codes, scales, dtype).matmul(x)
    assert torch.equal(got.cpu(), (x.cpu().double() @ weights64(codes, scales, group).T).to(DT[dtype]))
    binding.dresd_w4_status(torch.cuda.current_stream().cuda_stream)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,stage", [(40, 1), (40, 4), (300, 3)])      # a CTA has at least four stages here: 32 blocks, split by up to 8
def test_a_wait_that_runs_out_is_reported(option, rows, stage):
    """The first CTA never receives a stage: the call comes back, says so, and the next one is right."""
    x, codes, scales = exact_inputs(rows, 4096, 600, 128, "f16", 4)
    w, stream = binding.W4(codes, scales, "f16"), torch.cuda.current_stream().cuda_stream
    option("w4_path", 2)
    want = w.matmul(x)
    binding.dresd_w4_status(stream)
    option("w4_wait_ms", 20)
    option("w4_debug_lose_stage", stage)
    w.matmul(x)
    with pytest.raises(binding.DresdError) as e:
        binding.dresd_w4_status(stream)
    assert e.value.status == -5
    option("w4_debug_lose_stage", 0)
    binding.dresd_w4_status(stream)
    assert torch.equal(w.matmul(x), want)
    binding.dresd_w4_status(stream)


@pytest.mark.parametrize("name,value", [("w4_path", 3), ("w4_path", -1), ("w4_wait_ms", -1), ("w4_wait_ms", 60001), ("w4_debug_lose_stage", -1), ("w4_other", 0)])
def test_options_outside_their_range(name, value):
    from paper_2502_15572_b200 import build
    build.build()
    with pytest.raises(binding.DresdError) as e:
        binding.dresd_set_global_option(name, value)
    assert e.value.status == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,inputs,outputs,group", SIZES)
def test_real_numbers(rows, inputs, outputs, group, dtype):
    g = torch.Generator().manual_seed(rows + inputs)
    x = torch.randn((rows, inputs), generator=g).to(DT[dtype])
    w = torch.randn((inputs, outputs), generator=g).to(DT[dtype]).cuda()
    q = binding.W4.quantise(w, group)
    w64 = weights64(q.codes, q.scales, group)
    got = q.matmul(x.cuda()).cpu().double()
    want, all_ = x.double() @ w64.T, x.double().abs() @ w64.abs().T
    sums = (inputs + inputs // group + 16) * 2.0 ** -23 * all_
    bound = sums + U[dtype] * (want.abs() + sums) + 2.0 ** -25
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("order", ["inputs first", "outputs first", "slices"])
def test_quantise(dtype, group, order):
    g = torch.Generator().manual_seed(group)
    inputs, outputs = 5 * group, 77
    w = torch.randn((inputs, outputs), generator=g) * torch.logspace(-6, 4, outputs)
    w[:group, 3] = 0                                          # a group of zeros
    w[:group, 4] = 1e-7                                       # fp16: a scale that rounds to 0 or to a subnormal
    w[group:2 * group, 5] = torch.arange(group).float() - 7   # codes on halves and ends
    w = w.to(DT[dtype]).cuda()
    if order == "outputs first":
        w = w.t().contiguous().t()
    elif order == "slices":
        w = torch.cat((w, w), 1).repeat_interleave(2, 0)[::2, 10:10 + outputs]
    q = binding.W4.quantise(w, group)
    x = w.t().float().cpu().reshape(outputs, 5, group)
    s = (x.abs().amax(-1) / 7).to(DT[dtype])
    c = torch.where(s[..., None] > 0, (x / s.float()[..., None]).round().clamp(-8, 7), torch.zeros(())).to(torch.int64) + 8
    c = c.view(outputs, -1, 2)
    assert torch.equal(q.scales.cpu(), s) and torch.equal(q.codes.cpu(), (c[..., 0] | c[..., 1] << 4).to(torch.uint8))
    # as they are rounded: within half a step, and what the scale's own rounding adds at the ends
    step = q.scales.cpu().double().repeat_interleave(group, 1)
    off = (weights64(q.codes, q.scales, group) - w.t().cpu().double()).abs()
    fine = step > 2.0 ** -10
    assert bool((off <= step * (0.5 + 8 * U[dtype]))[fine].all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 5, 40, 200])
def test_distances_and_guards(rows):
    """Rows apart from each other on every side; nothing between them is written, and what lies behind the last row is not read."""
    inputs, outputs, group = 256, 150, 64
    x, codes, scales = exact_inputs(rows, inputs, outputs, group, "f16", 3)
    want = (x.cpu().double() @ weights64(codes, scales, group).T)
    apart = torch.full((rows + 1, inputs + 40), float("nan"), dtype=torch.float16, device="cuda")
    apart[:rows, 16:16 + inputs] = x
    w = binding.W4(codes, scales, "f16")
    out = torch.full((rows + 2, outputs + 7), 5.0, dtype=torch.float16, device="cuda")
    residual = torch.full((rows, outputs + 3), 2.0, dtype=torch.float16, device="cuda")
    w.matmul(apart[:rows, 16:16 + inputs], residual=residual[:, 1:1 + outputs], out=out[1:-1, 3:3 + outputs])
    assert torch.equal(out[1:-1, 3:3 + outputs].cpu(), (want + 2).half())
    assert bool((out[0] == 5).all()) and bool((out[-1] == 5).all()) and bool((out[:, :3] == 5).all()) and bool((out[:, 3 + outputs:] == 5).all())
    onto = residual[:, 1:1 + outputs]
    w.matmul(apart[:rows, 16:16 + inputs], residual=onto, out=onto)          # onto the residual itself
    assert torch.equal(onto.cpu(), (want + 2).half())
    assert bool((residual[:, 0] == 2).all()) and bool((residual[:, 1 + outputs:] == 2).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 20, 150])
def test_infinities_and_nan_stay_in_their_rows(rows):
    x, codes, scales = exact_inputs(rows, 512, 140, 128, "bf16", 5)
    x[0, 5], x[rows // 2, 300] = float("inf"), float("nan")
    got = binding.W4(codes, scales, "bf16").matmul(x, relu=True).cpu()
    assert bool(got[rows // 2].isnan().all())
    clean = torch.ones(rows, dtype=torch.bool)
    clean[0] = clean[rows // 2] = False
    want = (x.cpu().double() @ weights64(codes, scales, 128).T).clamp(min=0).bfloat16()
    assert torch.equal(got[clean], want[clean])


@pytest.mark.gpu
def test_offsets_beyond_31_bits():
    """Codes of more than 2^32 weights; activations whose rows lie far apart."""
    inputs, outputs = 32768, 131200
    codes = torch.full((outputs, inputs // 2), 0x88, dtype=torch.uint8, device="cuda")
    codes[-3:] = torch.randint(256, (3, inputs // 2), dtype=torch.uint8, device="cuda")
    scales = torch.ones((outputs, inputs // 128), dtype=torch.float16, device="cuda")
    x = torch.randint(-1, 2, (2, inputs), device="cuda").half()
    got = binding.W4(codes, scales, "f16").matmul(x)
    want = x.cpu().double() @ weights64(codes[-3:], scales[-3:], 128).T
    assert torch.equal(got[:, -3:].cpu(), want.half()) and int(got[:, :-3].abs().max()) == 0
    del codes, scales
    apart = torch.empty((2, 1 << 31), dtype=torch.float16, device="cuda")[:, :256]
    y, codes, scales = exact_inputs(2, 256, 20, 64, "f16", 2)
    apart.copy_(y)
    assert torch.equal(binding.W4(codes, scales, "f16").matmul(apart).cpu(), (y.cpu().double() @ weights64(codes, scales, 64).T).half())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 30, 300])
def test_repeated_captured_and_on_another_stream(rows):
    x, codes, scales = (t.cuda() for t in exact_inputs(rows, 1024, 260, 32, "f16", 9))
    w = binding.W4(codes, scales, "f16")
    x = torch.randn_like(x)
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
    assert torch.equal(one, -want)
    assert torch.equal(two, w.matmul(x, residual=one))


@pytest.mark.gpu
def test_no_rows():
    x, codes, scales = exact_inputs(1, 64, 9, 32, "f16", 0)
    assert binding.W4(codes, scales, "f16").matmul(x[:0]).shape == (0, 9)


@pytest.mark.gpu
def test_refusals():
    x, codes, scales = exact_inputs(2, 256, 10, 64, "f16", 0)
    w = binding.W4(codes, scales, "f16")
    out = torch.empty((2, 10), dtype=torch.float16, device="cuda")
    far = torch.zeros((2, 260), dtype=torch.float16, device="cuda")
    for bad in [lambda: binding.W4(codes.cpu(), scales, "f16"), lambda: binding.W4(codes, scales.cpu(), "f16"), lambda: binding.W4(codes, scales, "bf16"),
                lambda: binding.W4(codes, scales[:, :3].contiguous(), "f16"), lambda: binding.W4(codes, scales[:9], "f16"), lambda: binding.W4(codes[:, ::2], scales, "f16"),
                lambda: w.matmul(x[0]), lambda: w.matmul(x.bfloat16()), lambda: w.matmul(x[:, :128]), lambda: w.matmul(x.cpu()), lambda: w.matmul(far[:, 1:257]),
                lambda: w.matmul(far[:, :256]), lambda: w.matmul(x.t().contiguous().t()), lambda: w.matmul(x, out=out[:1]), lambda: w.matmul(x, out=out.float()),
                lambda: w.matmul(x, residual=out[:, :9]), lambda: w.matmul(x, residual=out[:1].expand(2, 10)), lambda: w.matmul(x, out=out[:1].expand(2, 10)),
                lambda: w.matmul(x[:1].expand(2, 256)), lambda: binding.W4.quantise(x[:1].expand(128, 256), 64), lambda: binding.W4.quantise(x, 32),
                lambda: binding.W4.quantise(x.float(), 32)]:
        with pytest.raises(binding.DresdError) as e:
            bad()
        assert e.value.status == -1
    for bad in [lambda: binding.W4(codes, scales, "f32"), lambda: binding.W4(codes, scales[:, :1].contiguous(), "f16"), lambda: binding.W4.quantise(far.t().contiguous(), 20)]:
        with pytest.raises(binding.DresdError) as e:
            bad()
        assert e.value.status == -2


@pytest.mark.parametrize("change,status", [
    (dict(dtype=0), -2), (dict(dtype=9), -1), (dict(group=16), -2), (dict(group=0), -1), (dict(inputs=96), -1), (dict(outputs=0), -1), (dict(inputs=0), -1),
    (dict(outputs=(1 << 20) + 1, out_row=1 << 21), -2), (dict(rows=-1), -1), (dict(rows=(1 << 20) + 1), -2), (dict(x_row=132), -1), (dict(x_row=120), -1),
    (dict(out_row=9), -1), (dict(residual_row=9), -1), (dict(x_row=1 << 40), -1)])
def test_refusals_need_no_device(change, status):
    from paper_2502_15572_b200 import build
    build.build()
    a = dict(x_row=128, rows=2, inputs=128, outputs=10, dtype=1, group=64, residual_row=10, out_row=10)
    a.update(change)
    with pytest.raises(binding.DresdError) as e:
        binding.dresd_w4_matmul(0x1000, a["x_row"], a["rows"], 0x1000, 0x1000, a["inputs"], a["outputs"], a["dtype"], a["group"], 0, 0x1000, a["residual_row"],
                                0x1000, a["out_row"])
    assert e.value.status == status
    with pytest.raises(binding.DresdError):
        binding.dresd_w4_quantise(0x1000, 0, 1, 128, 10, 1, 64, 0x1000, 0x1000)
