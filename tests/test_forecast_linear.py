"""Matrix product with bias, activation and residual, and its gradients, against 64-bit values:
few rows and many, sizes around the tiles' edges, odd ones, strided and unaligned operands."""
import math

import pytest
import torch

from tests import forecast_ref as R

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])


@pytest.fixture(scope="module")
def F():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2407_14843_b200 import build
    build.build_library()
    from paper_2407_14843_b200 import forecast
    return forecast


def normal(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def terms_of(depth):
    """Roundings of a sum over `depth` products: the tensor core adds 16 products at a time to a
    32-bit accumulator and may cut instead of rounding (two units); the rest is the epilogue's."""
    return 64 + depth // 4


def make(m, n, k, dtype, seed=0, bias=True, residual=True):
    a = {"x": normal(seed, m, k).to(dtype), "weight": (normal(seed + 1, n, k) / math.sqrt(k)).to(dtype)}
    a["bias"] = normal(seed + 2, n) if bias else None
    a["residual"] = normal(seed + 3, m, n).to(dtype) if residual else None
    return a


def reference(a, activation):
    pre = a["x"].double() @ a["weight"].double().t()
    if a["bias"] is not None:
        pre = pre + a["bias"].double()
    y = R.activate(pre, activation)
    return pre, y if a["residual"] is None else y + a["residual"].double()


SIZES = [(1, 1, 1), (1, 16, 8), (3, 17, 40), (8, 100, 64), (9, 64, 33), (16, 33, 300), (17, 130, 72), (32, 48, 1000), (33, 64, 64),
         (64, 8, 16), (100, 130, 72), (128, 256, 64), (129, 257, 136), (200, 1000, 513), (300, 64, 1), (77, 1, 264), (1000, 520, 104),
         (257, 127, 1030)]


@TYPES
@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_against_64_bits(F, size, activation, dtype):
    a = make(*size, dtype, seed=sum(size))
    pre, y = reference(a, activation)
    got, got_pre = F.linear(**a, activation=activation, save_pre=True)
    R.close(got, y, terms=terms_of(size[2]), what="y")
    R.close(got_pre, pre, terms=terms_of(size[2]), what="pre")


@TYPES
@pytest.mark.parametrize("size", [(5, 40, 64), (150, 260, 128), (150, 260, 77)], ids=str)
def test_linear_without_bias_and_residual(F, size, dtype):
    a = make(*size, dtype, bias=False, residual=False)
    R.close(F.linear(**a), reference(a, "none")[1], terms=terms_of(size[2]))


@pytest.mark.parametrize("rows", [7, 250])
@pytest.mark.parametrize("offset", [0, 1, 8], ids=lambda o: f"offset{o}")
@pytest.mark.parametrize("pitch", [0, 3, 8], ids=lambda o: f"pitch{o}")
def test_strided_and_unaligned_operands(F, rows, offset, pitch):
    n, k = 144, 200
    def view(seed, r, c, scale=1.0):
        big = (normal(seed, r, c + offset + pitch) * scale).bfloat16()
        return big[:, offset:offset + c]
    a = {"x": view(1, rows, k), "weight": view(2, n, k, 1 / math.sqrt(k)), "bias": normal(3, n + 1)[1:].clone(), "residual": view(4, rows, n)}
    R.close(F.linear(**a, activation="silu"), reference(a, "silu")[1], terms=terms_of(k))
    dy = view(5, rows, n)
    check_gradients(F, a["x"], a["weight"], dy, "none")
    check_gradients(F, a["x"], a["weight"], dy, "gelu")


def test_many_tiles_per_block(F):
    """More tiles than multiprocessors: both accumulator buffers and every ring position are reused."""
    a = make(128 * 45 + 3, 1032, 328, torch.bfloat16, seed=5)
    R.close(F.linear(**a, activation="silu"), reference(a, "silu")[1], terms=terms_of(328))


# large enough for every kind of tile (pairs of blocks on 256 and 128 columns, single blocks on 128 and
# 64), with and without ragged edges
LARGE = [(2048, 2048, 1024), (1000, 2040, 1000), (100, 16384, 1024), (1021, 1000, 520), (3000, 515, 700)]


@TYPES
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_every_kind_of_tile(F, size, dtype):
    a = make(*size, dtype, seed=sum(size))
    pre, y = reference(a, "gelu")
    got, got_pre = F.linear(**a, activation="gelu", save_pre=True)
    R.close(got, y, terms=terms_of(size[2]), what="y with pre")
    R.close(got_pre, pre, terms=terms_of(size[2]), what="pre")
    assert torch.equal(F.linear(**a, activation="gelu"), got)


@pytest.mark.parametrize("size", LARGE, ids=str)
def test_gradients_with_every_kind_of_tile(F, size):
    m, n, k = size
    a = make(m, n, k, torch.bfloat16, seed=sum(size))
    check_gradients(F, a["x"], a["weight"], normal(4, m, n).bfloat16(), "silu")


def check_gradients(F, x, weight, dy, activation, seed=9):
    m, k = x.shape
    n = weight.shape[0]
    pre = None if activation == "none" else normal(seed, m, n).to(x.dtype)
    got = F.linear_backward(dy, x, weight, pre=pre, activation=activation)
    q = dy.double()
    if pre is not None:
        p = pre.double().requires_grad_()
        q, = torch.autograd.grad(R.activate(p, activation), p, q)
    w, xd, unit = weight.double(), x.double(), R.UNIT[x.dtype]
    rounded = 0 if activation == "none" else 1
    for name, a, b, depth in (("dx", q, w, n), ("dweight", q.t(), xd, m)):
        ref = a @ b
        # q's own rounding to the operands' type: at most `unit` of each term, of either sign; four
        # times the 2-norm of the terms is beyond any sum of such errors that these sizes can show
        spread = rounded * 4 * unit * torch.sqrt((a * a) @ (b * b))
        room = 1.01 * unit * ref.abs() + spread + terms_of(depth) * 2.0 ** -24 * ref.abs().max()
        if x.dtype == torch.float16:
            room = room + 2.0 ** -25 + rounded * 2.0 ** -25 * b.abs().sum(0, keepdim=True)
        off = (got[name].double() - ref).abs()
        assert torch.isfinite(got[name]).all() and (off <= room).all(), (name, (off / room).max().item())
    R.close(got["dbias"], q.sum(0), terms=64 + m // 64, what="dbias")
    return got


@TYPES
@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradients_against_64_bits(F, size, activation, dtype):
    m, n, k = size
    a = make(m, n, k, dtype, seed=sum(size))
    check_gradients(F, a["x"], a["weight"], normal(4, m, n).to(dtype), activation)


@pytest.mark.parametrize("size", [(5000, 70, 40), (4099, 256, 128), (9000, 33, 65), (2000, 1024, 32)], ids=str)
def test_gradients_split_over_many_rows(F, size):
    m, n, k = size
    a = make(m, n, k, torch.bfloat16, seed=sum(size))
    check_gradients(F, a["x"], a["weight"], normal(4, m, n).bfloat16(), "silu")


def test_wanted_gradients_only(F):
    a = make(70, 40, 24, torch.bfloat16)
    dy, pre = normal(1, 70, 40).bfloat16(), normal(2, 70, 40).bfloat16()
    full = F.linear_backward(dy, a["x"], a["weight"], pre=pre, activation="gelu")
    for kw, names in ((dict(bias=False), {"dx", "dweight"}), (dict(need_dx=False), {"dweight", "dbias"}),
                      (dict(need_dweight=False, bias=False), {"dx"}), (dict(need_dx=False, need_dweight=False), {"dbias"})):
        got = F.linear_backward(dy, a["x"], a["weight"], pre=pre, activation="gelu", **kw)
        assert set(got) == names
        assert all(torch.equal(got[k], full[k]) for k in names)


def test_gradients_against_differences(F):
    """Central differences of the forward product along single directions, in fp16 with few, well scaled
    terms: y is off by 2^-11 of itself, so the step is large (0.25) and only smooth activations are used;
    the differences carry (0.25)^2 / 6 of the third derivative and the roundings' 2^-11 / 0.25."""
    m, n, k = 40, 16, 24
    x, w = normal(1, m, k).half(), (normal(2, n, k) / math.sqrt(k)).half()
    bias, dy = normal(3, n), normal(4, m, n).half()
    y, pre = F.linear(x, w, bias, "silu", save_pre=True)
    g = F.linear_backward(dy, x, w, pre=pre, activation="silu")
    value = lambda x, w, b: (F.linear(x, w, b, "silu").double() * dy.double()).sum()  # noqa: E731
    for name, arg in (("dx", 0), ("dweight", 1), ("dbias", 2)):
        args = [x, w, bias]
        v = normal(7 + arg, *args[arg].shape)
        v = v / v.norm()
        lo, hi = list(args), list(args)
        hi[arg], lo[arg] = ((args[arg].float() + s * 0.25 * v).to(args[arg].dtype) for s in (1, -1))
        step = (hi[arg].double() - lo[arg].double())
        slope = value(*hi) - value(*lo)
        along = (g[name].double() * step).sum()
        noise = 2 * 2.0 ** -11 * (y.double() * dy.double()).norm()
        assert abs(slope - along) < 4 * noise + 0.05 * abs(along) + 0.01, (name, slope.item(), along.item())


def test_autograd_function(F):
    a = make(50, 40, 24, torch.bfloat16, seed=3)
    leaves = {k: v.clone().requires_grad_() for k, v in a.items()}
    y = F.Linear.apply(leaves["x"], leaves["weight"], leaves["bias"], "silu", leaves["residual"])
    dy = normal(8, 40, 50).bfloat16().t()             # the last axis is not contiguous
    y.backward(dy)
    _, pre = F.linear(**a, activation="silu", save_pre=True)
    g = F.linear_backward(dy.contiguous(), a["x"], a["weight"], pre=pre, activation="silu")
    assert torch.equal(leaves["x"].grad, g["dx"]) and torch.equal(leaves["weight"].grad, g["dweight"])
    assert torch.equal(leaves["bias"].grad, g["dbias"]) and torch.equal(leaves["residual"].grad, dy)


def test_no_rows(F):
    w = normal(1, 40, 24).bfloat16()
    x = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    assert F.linear(x, w).shape == (0, 40)
    g = F.linear_backward(torch.empty(0, 40, dtype=torch.bfloat16, device="cuda"), x, w)
    assert g["dx"].shape == (0, 24) and (g["dweight"] == 0).all() and (g["dbias"] == 0).all()


def test_not_a_number_stays_in_its_row(F):
    for rows in (9, 200):
        a = make(rows, 300, 100, torch.bfloat16, seed=2)
        clean = F.linear(**a, activation="silu")
        a["x"][4, 7] = float("nan")
        y = F.linear(**a, activation="silu")
        assert torch.isnan(y[4]).all()
        keep = torch.arange(rows, device="cuda") != 4
        assert torch.equal(y[keep], clean[keep])


def test_same_inputs_give_the_same_bits_and_no_timeout(F):
    a = make(3000, 520, 264, torch.bfloat16)
    dy, pre = normal(1, 3000, 520).bfloat16(), normal(2, 3000, 520).bfloat16()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    runs = [(F.linear(**a, activation="gelu", status=status),
             F.linear_backward(dy, a["x"], a["weight"], pre=pre, activation="gelu", status=status)) for _ in range(3)]
    for y, g in runs[1:]:
        assert torch.equal(y, runs[0][0]) and all(torch.equal(g[k], runs[0][1][k]) for k in g)
    assert status.item() == 0


def test_calls_follow_the_current_stream(F):
    a = make(512, 256, 128, torch.bfloat16)
    ref = F.linear(**a)
    late = torch.zeros_like(a["x"])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(a["x"])
        y = F.linear(**{**a, "x": late})
    side.synchronize()
    assert torch.equal(y, ref)


def test_refusals(F):
    a = make(40, 24, 16, torch.bfloat16)
    with pytest.raises(TypeError):
        F.linear(a["x"].float(), a["weight"].float())
    with pytest.raises(TypeError):
        F.linear(a["x"], a["weight"].half())
    with pytest.raises(TypeError):
        F.linear(a["x"], a["weight"][:, :-1])
    with pytest.raises(TypeError):
        F.linear(a["x"].t().contiguous().t(), a["weight"])
    with pytest.raises(TypeError):
        F.linear(a["x"][:1].expand(40, -1), a["weight"])      # overlapping rows
    with pytest.raises(TypeError):
        F.linear(**{**a, "bias": a["bias"].bfloat16()})
    with pytest.raises(TypeError):
        F.linear(**{**a, "residual": a["residual"][:-1]})
    with pytest.raises(ValueError):
        F.linear(**a, activation="tanh")
    with pytest.raises(TypeError):
        F.linear(a["x"], a["weight"].cpu())
    with pytest.raises(TypeError):
        F.linear_backward(a["residual"], a["x"], a["weight"], activation="gelu")      # no pre
    with pytest.raises(F.ThemisError) as e:
        F.linear_backward(a["residual"], a["x"], a["weight"], workspace=torch.empty(256, dtype=torch.uint8, device="cuda")[:0])
    assert e.value.code in (F.E_WORKSPACE_TOO_SMALL, F.E_INVALID_ARG)


def test_an_expired_wait_is_not_lost(F, monkeypatch):
    """Calls without a status, the autograd function's among them, report to one word of pinned host memory; what the
    device writes there (here by a copy) is raised by the next call."""
    a = make(100, 64, 48, torch.bfloat16)
    y = F.linear(**a, activation="silu")
    word = F._status_memory
    assert word.is_pinned() and word.item() == 0
    given = []
    for name, at in (("themis_linear_forward", 7), ("themis_linear_backward", 8)):
        real = getattr(F._lib, name)
        monkeypatch.setattr(F._lib, name, lambda *args, real=real, at=at: (given.append(args[at]), real(*args))[1])
    x = a["x"].clone().requires_grad_()
    out = F.Linear.apply(x, a["weight"], a["bias"], "silu", a["residual"])
    out.sum().backward()
    assert given == [word.data_ptr()] * 2 and torch.equal(out, y)
    torch.cuda.synchronize()
    F.check_status()
    expired = torch.full((1,), F.STATUS_TIMEOUT, dtype=torch.int32, device="cuda")
    for call in (lambda: F.linear(**a), lambda: F.linear_backward(a["residual"], a["x"], a["weight"]),
                 lambda: F.Linear.apply(x, a["weight"]), F.check_status):
        word.copy_(expired)
        with pytest.raises(F.WaitExpired):
            call()
        assert torch.equal(F.linear(**a, activation="silu"), y)
    # a word of the caller's own is used as it is
    own = torch.zeros(1, dtype=torch.int32, device="cuda")
    F.linear(**a, status=own)
    assert given[-1] == own.data_ptr() and own.item() == 0


def test_capture_into_a_graph(F):
    a = make(100, 64, 48, torch.bfloat16)
    y = F.linear(**a, activation="silu")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = F.linear(**a, activation="silu")
    again.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, y)
    F.check_status()


@pytest.mark.parametrize("activation", ["none", "silu"])
def test_second_derivatives_are_refused(F, activation):
    """Alone and in a sum with other terms, where a gradient without a graph would only go missing."""
    a = make(50, 40, 24, torch.bfloat16, seed=3)
    for name in ("x", "weight", "bias"):
        leaves = {k: v.clone().requires_grad_() for k, v in a.items()}
        y = F.Linear.apply(leaves["x"], leaves["weight"], leaves["bias"], activation, leaves["residual"])
        g, = torch.autograd.grad(y.float().square().sum() if name == "x" else y.sum(), leaves[name], create_graph=True)
        plain = {k: v.clone().requires_grad_() for k, v in a.items()}
        y = F.Linear.apply(plain["x"], plain["weight"], plain["bias"], activation, plain["residual"])
        want, = torch.autograd.grad(y.float().square().sum() if name == "x" else y.sum(), plain[name])
        assert torch.equal(g, want) and g.requires_grad
        with pytest.raises(RuntimeError, match="differentiated again"):
            (g.float().square().sum() + leaves["x"].float().sum()).backward()


@TYPES
@pytest.mark.parametrize("rows", [4, 200])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_activations_value_by_value(F, activation, rows, dtype):
    """pre is the bias alone, over -12..12, and every value has its own room: one rounding to the type; for gelu
    1.5e-7 / 2 of v (the error function's) and four roundings of the distribution function, from -6 to -3 also no more
    than 4e-3 of the value; for silu a dozen roundings and the exponent's |v|."""
    v = torch.linspace(-12, 12, 4097, device="cuda")[:4096].contiguous()
    x = torch.ones(rows, 16, dtype=dtype, device="cuda")
    y = F.linear(x, torch.zeros(4096, 16, dtype=dtype, device="cuda"), v, activation).double()
    d = v.double()
    # (1 + erf would cancel in 64 bits too)
    ref = d * 0.5 * torch.special.erfc(-d / math.sqrt(2)) if activation == "gelu" else d / (1 + torch.exp(-d))
    room = 1.01 * R.UNIT[dtype] * ref.abs() + (2.0 ** -25 if dtype == torch.float16 else 1e-36)
    if activation == "gelu":
        wide = d.abs() * (0.75e-7 + 4 * 2.0 ** -24)
        tail = (d >= -6) & (d <= -3)
        room = room + torch.where(tail, torch.minimum(wide, 4e-3 * ref.abs()), wide)
    else:
        room = room + ref.abs() * (12 + d.abs()) * 2.0 ** -24
    assert ((y - ref).abs() <= room).all(), ((y - ref).abs() / room).max().item()


@TYPES
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_slopes_value_by_value(F, activation, dtype):
    """The bias gradient of one row with dy = 1 is the slope in 32 bits: the error function's 0.75e-7 and sixteen
    roundings of values up to 1.13."""
    pre = torch.linspace(-12, 12, 4097, device="cuda")[:4096].to(dtype)[None]
    x, w = torch.zeros(1, 16, dtype=dtype, device="cuda"), torch.zeros(4096, 16, dtype=dtype, device="cuda")
    got = F.linear_backward(torch.ones_like(pre), x, w, pre=pre, activation=activation)["dbias"].double()
    p = pre[0].double().requires_grad_()
    ref, = torch.autograd.grad(R.activate(p, activation).sum(), p)
    assert (got - ref).abs().max() <= 0.75e-7 + 16 * 1.13 * 2.0 ** -24
