"""Selective state space scan (whole histories, one time, gradients) against the plain 64-bit
statement in ``forecast_ref``: every type, head layout, state size and width, lengths from none to
ones that are split over the time axis, ragged rows with NaN behind their end, strided views."""
import math

import pytest
import torch

from tests import forecast_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2407_14843_b200 import build
    build.build_library()
    from paper_2407_14843_b200 import forecast
    return forecast


def make(rows, length, D, N, G=1, W=4, dtype=torch.float32, seed=0, optional=True, states=True, ragged=False, views=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    a = {}
    if views:       # slices of one projection, an odd offset among them
        proj = normal(rows, length, 2 * D + 2 * G * N + 3).to(dtype)
        z, _, x, b, c = proj.split([D, 3, D, G * N, G * N], dim=2)
        b, c = b.unflatten(2, (G, N)), c.unflatten(2, (G, N))
    else:
        x, z, b, c = (normal(*s).to(dtype) for s in ((rows, length, D), (rows, length, D), (rows, length, G, N), (rows, length, G, N)))
    a.update(x=x, B=b, C=c, dt=normal(rows, length, D).to(dtype))
    a["A"] = -torch.exp(0.7 * normal(D, N)) * 3
    a["conv_weight"] = normal(D, W) / math.sqrt(W)
    if optional:
        a.update(z=z, conv_bias=normal(D), skip=normal(D), dt_bias=normal(D) - 3)
    if states:
        a.update(conv_state=normal(rows, W - 1, D).to(dtype), ssm_state=normal(rows, D, N))
    if ragged:
        lengths = torch.randint(0, length + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
        lengths[0] = 0
        lengths[-1] = length
        a["lengths"] = lengths
    return a


def scan_args(a):
    return {k: v for k, v in a.items()}


def spoil(a):
    """NaN and infinities behind every row's end."""
    a = dict(a)
    for k in ("x", "dt", "z", "B", "C"):
        if k in a:
            v = a[k].clone()
            for b, n in enumerate(a["lengths"].tolist()):
                v[b, n:] = float("nan") if b % 2 else float("inf")
            a[k] = v
    return a


SHAPES = [  # rows, length, D, N, G, W
    (2, 1, 5, 16, 1, 4), (3, 2, 1, 1, 1, 2), (2, 3, 130, 4, 1, 3), (1, 17, 33, 8, 1, 4), (2, 63, 12, 16, 3, 4),
    (2, 64, 40, 12, 2, 4), (1, 65, 129, 16, 1, 2), (2, 130, 66, 17, 2, 3), (2, 100, 24, 32, 1, 4), (1, 90, 10, 40, 2, 4),
    (1, 70, 36, 64, 2, 4), (2, 129, 8, 3, 8, 4), (2, 200, 260, 5, 2, 4),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scan_against_the_definition(F, shape, dtype):
    a = make(*shape, dtype=dtype, seed=sum(shape))
    r = F.ssm_scan(**a)
    y, conv, h = R.scan(**a)
    R.close(r.y, y, what="y")
    R.close(r.ssm_state, h, what="state")
    assert torch.equal(r.conv_state.double(), conv)


@pytest.mark.parametrize("length", [1, 2, 64, 200])
def test_without_the_optional_inputs(F, length):
    a = make(2, length, 48, 16, optional=False, states=False, views=False)
    r = F.ssm_scan(**a)
    y, conv, h = R.scan(**a)
    R.close(r.y, y, what="y")
    R.close(r.ssm_state, h, what="state")
    assert torch.equal(r.conv_state.double(), conv)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 33, 40, 16, 2, 4), (4, 2, 130, 8, 1, 4), (6, 1, 20, 4, 1, 3), (4, 150, 20, 40, 1, 2)], ids=str)
def test_ragged_rows_do_not_see_what_is_behind_their_end(F, shape, dtype):
    a = make(*shape, dtype=dtype, ragged=True, seed=7)
    y, conv, h = R.scan(**a)
    r = F.ssm_scan(**spoil(a))
    R.close(r.y, y, what="y")
    R.close(r.ssm_state, h, what="state")
    assert torch.equal(r.conv_state.double(), conv)
    for b, n in enumerate(a["lengths"].tolist()):
        assert (r.y[b, n:] == 0).all()
    clamped = dict(a, lengths=torch.where(a["lengths"] == 0, -3, torch.where(a["lengths"] == shape[1], shape[1] + 9, a["lengths"])).int())
    assert torch.equal(F.ssm_scan(**clamped).y, r.y)


@pytest.mark.parametrize("shape", [(1, 5000, 24, 16, 1, 4), (2, 3001, 130, 8, 2, 3), (1, 2500, 8, 40, 1, 4), (1, 700, 16, 3, 1, 2)], ids=str)
def test_few_rows_are_split_over_the_time_axis(F, shape):
    a = make(*shape, seed=3)
    a["A"] = a["A"] * 0.02                   # long memories, so that the parts depend on each other
    problem, *_ = F._ssm_args(**{k: a.get(k) for k in ("x", "dt", "A", "B", "C", "conv_weight", "conv_bias", "skip", "dt_bias", "z",
                                                       "conv_state", "ssm_state", "lengths")}, step=False)
    assert F.themis_ssm_workspace_bytes(problem, False) > 0          # otherwise nothing is split
    r = F.ssm_scan(**a)
    y, conv, h = R.scan(**a)
    # the state sums up to a few thousand terms whose factors are each rounded
    R.close(r.y, y, terms=512, what="y")
    R.close(r.ssm_state, h, terms=512, what="state")
    assert torch.equal(r.conv_state.double(), conv)
    ragged = dict(a, lengths=torch.tensor([shape[1] // 3] * shape[0], dtype=torch.int32, device="cuda"))
    r = F.ssm_scan(**spoil(ragged))
    y, conv, h = R.scan(**ragged)
    R.close(r.y, y, terms=512, what="ragged y")
    R.close(r.ssm_state, h, terms=512, what="ragged state")
    assert torch.equal(r.conv_state.double(), conv)


def test_empty_inputs(F):
    a = make(3, 0, 20, 8, views=False)
    r = F.ssm_scan(**a)
    assert r.y.shape == (3, 0, 20)
    assert torch.equal(r.ssm_state, a["ssm_state"]) and torch.equal(r.conv_state, a["conv_state"])
    no_states = {k: v for k, v in a.items() if k not in ("ssm_state", "conv_state")}
    r = F.ssm_scan(**no_states, save=True)
    assert (r.ssm_state == 0).all() and (r.conv_state == 0).all()
    g = F.ssm_scan_backward(torch.empty_like(r.y), r.checkpoints, **no_states)
    assert all((g[k] == 0).all() for k in ("dA", "dconv_weight", "dconv_bias", "dskip", "ddt_bias"))
    a = make(0, 7, 20, 8, views=False)
    assert F.ssm_scan(**a).y.shape == (0, 7, 20)


def test_whole_history_follows_its_pieces(F):
    """Not bit for bit: a long history of few rows is split over the time axis, a short piece is not."""
    a = make(3, 150, 40, 16, dtype=torch.bfloat16, seed=5)
    whole = F.ssm_scan(**a)
    states, ys = (a["conv_state"], a["ssm_state"]), []
    for lo, hi in ((0, 1), (1, 3), (3, 67), (67, 150)):
        piece = {k: (v[:, lo:hi] if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items()}
        piece["conv_state"], piece["ssm_state"] = states
        r = F.ssm_scan(**piece)
        states = (r.conv_state, r.ssm_state)
        ys.append(r.y)
    # both are one rounding away from the same values
    y, conv, h = R.scan(**a)
    R.close(torch.cat(ys, 1), y, what="pieces")
    R.close(whole.y, y, what="whole")
    R.close(states[1], h, what="state of the pieces")
    R.close(whole.ssm_state, h, what="state of the whole")
    assert torch.equal(states[0], whole.conv_state) and torch.equal(states[0].double(), conv)


# --- one time ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", [(1, 512, 16, 1, 4), (7, 33, 16, 3, 4), (5, 40, 1, 1, 2), (3, 24, 6, 2, 3), (2, 130, 64, 1, 4),
                                   (300, 20, 40, 2, 4), (4, 6, 12, 1, 2), (9, 65, 4, 1, 3)], ids=str)
def test_step_against_the_definition(F, shape, dtype):
    rows, D, N, G, W = shape
    a = make(rows, 1, D, N, G, W, dtype=dtype, seed=11)
    y, conv, h = R.scan(**a)
    s = {k: (v[:, 0] if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items()}
    new_conv, new_h = torch.full_like(a["conv_state"], 7), torch.full_like(a["ssm_state"], 7)
    kept = a["conv_state"].clone(), a["ssm_state"].clone()
    got = F.ssm_step(**s, new_conv_state=new_conv, new_ssm_state=new_h)
    R.close(got, y[:, 0], what="y")
    R.close(new_h, h, what="state")
    assert torch.equal(new_conv.double(), conv)
    assert torch.equal(a["conv_state"], kept[0]) and torch.equal(a["ssm_state"], kept[1])
    in_place = F.ssm_step(**s)                       # states updated where they are
    assert torch.equal(in_place, got) and torch.equal(a["ssm_state"], new_h) and torch.equal(a["conv_state"], new_conv)


def test_step_leaves_inactive_rows_alone(F):
    a = make(6, 1, 40, 16, seed=2)
    s = {k: (v[:, 0].clone() if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items()}
    y, conv, h = R.scan(**a)
    active = torch.tensor([1, 0, 1, 0, 0, 1], dtype=torch.int32, device="cuda")
    off = active == 0
    before = a["conv_state"].clone(), a["ssm_state"].clone()
    for k in ("x", "dt", "z", "B", "C"):
        s[k][off] = float("nan")
    got = F.ssm_step(**s, active=active)
    assert (got[off] == 0).all()
    assert torch.equal(a["conv_state"][off], before[0][off]) and torch.equal(a["ssm_state"][off], before[1][off])
    R.close(got[~off], y[~off, 0], what="y")
    R.close(a["ssm_state"][~off], h[~off], what="state")


def test_steps_follow_the_scan(F):
    a = make(4, 40, 24, 16, seed=9)
    whole = F.ssm_scan(**a)
    conv, h = a["conv_state"].clone(), a["ssm_state"].clone()
    for t in range(40):
        s = {k: (v[:, t] if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items() if k not in ("conv_state", "ssm_state")}
        y = F.ssm_step(**s, conv_state=conv, ssm_state=h)
        R.close(y, whole.y[:, t].double(), what=f"time {t}")
    R.close(h, whole.ssm_state.double(), what="state")
    assert torch.equal(conv, whole.conv_state)


# --- gradients -----------------------------------------------------------------------------------

NAMES = {"x": "dx", "dt": "ddt", "z": "dz", "B": "dB", "C": "dC", "A": "dA", "conv_weight": "dconv_weight",
         "conv_bias": "dconv_bias", "skip": "dskip", "dt_bias": "ddt_bias"}


def reference_gradients(a, dy):
    leaves = {k: a[k].detach().double().requires_grad_() for k in NAMES if k in a}
    y, _, _ = R.scan(**{**a, **leaves})
    return dict(zip((NAMES[k] for k in leaves), torch.autograd.grad(y, list(leaves.values()), dy.double())))


def check_gradients(F, a, dy, terms=64, spoiled=None):
    given = spoiled or a
    r = F.ssm_scan(**given, save=True)
    states = {k: a[k] for k in ("conv_state", "ssm_state") if k in a}
    got = F.ssm_scan_backward(dy, r.checkpoints, **{k: v for k, v in given.items() if k not in states}, **states)
    ref = reference_gradients(a, dy)
    assert set(got) == set(ref)
    for k in ref:
        R.close(got[k], ref[k], terms=terms, what=k)
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients_against_the_definition(F, shape, dtype):
    a = make(*shape, dtype=dtype, seed=sum(shape) + 1)
    dy = torch.randn(shape[0], shape[1], shape[2], device="cuda").to(dtype)
    check_gradients(F, a, dy, terms=256)         # sums over rows, times, channels and states


@pytest.mark.parametrize("length", [1, 64, 200])
def test_gradients_without_the_optional_inputs(F, length):
    a = make(2, length, 48, 16, optional=False, states=False, views=False)
    check_gradients(F, a, torch.randn(2, length, 48, device="cuda"), terms=256)


@pytest.mark.parametrize("shape", [(5, 33, 40, 16, 2, 4), (4, 2, 130, 8, 1, 4), (3, 150, 20, 40, 1, 2), (4, 260, 70, 16, 1, 4)], ids=str)
def test_gradients_of_ragged_rows(F, shape):
    a = make(*shape, ragged=True, seed=8)
    dy = torch.randn(shape[0], shape[1], shape[2], device="cuda")
    bad_dy = dy.clone()
    for b, n in enumerate(a["lengths"].tolist()):
        bad_dy[b, n:] = float("nan")
    ref = check_gradients(F, a, dy, terms=256)
    states = {k: a[k] for k in ("conv_state", "ssm_state")}
    given = spoil(a)
    r = F.ssm_scan(**given, save=True)
    got = F.ssm_scan_backward(bad_dy, r.checkpoints, **{**given, **states})
    for k in got:
        assert torch.equal(got[k], ref[k]), k
    for b, n in enumerate(a["lengths"].tolist()):
        for k in ("dx", "ddt", "dz", "dB", "dC"):
            assert (got[k][b, n:] == 0).all(), k


@pytest.mark.parametrize("shape", [(1, 3000, 24, 16, 1, 4), (2, 1500, 70, 8, 2, 3), (1, 1281, 8, 40, 1, 2)], ids=str)
def test_gradients_of_few_rows_split_over_the_time_axis(F, shape):
    a = make(*shape, seed=4)
    a["A"] = a["A"] * 0.02
    check_gradients(F, a, torch.randn(shape[0], shape[1], shape[2], device="cuda"), terms=1024)
    ragged = dict(a, lengths=torch.tensor([shape[1] // 3] * shape[0], dtype=torch.int32, device="cuda"))
    check_gradients(F, ragged, torch.randn(shape[0], shape[1], shape[2], device="cuda"), terms=1024, spoiled=spoil(ragged))


def test_gradients_against_differences(F):
    """Central differences of the forward kernel along random directions of length 1.  Step 0.01: the
    cubic term is about 1e-4, the 32-bit noise of the two sums about 1e-6 / 0.02."""
    a = make(2, 9, 6, 3, 2, 3, seed=21, views=False)
    dy = torch.randn(2, 9, 6, device="cuda")
    r = F.ssm_scan(**a, save=True)
    g = F.ssm_scan_backward(dy, r.checkpoints, **a)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    value = lambda b: (F.ssm_scan(**b).y.double() * dy.double()).sum()  # noqa: E731
    for k, name in NAMES.items():
        v = torch.randn(a[k].shape, generator=gen, device="cuda")
        v /= v.norm()
        slope = (value({**a, k: a[k] + 0.01 * v}) - value({**a, k: a[k] - 0.01 * v})) / 0.02
        along = (g[name].double() * v.double()).sum()
        assert abs(slope - along) < 2e-3 * (1 + abs(along)), (k, slope.item(), along.item())


def test_same_inputs_give_the_same_bits(F):
    a = make(3, 300, 200, 16, seed=6)
    dy = torch.randn(3, 300, 200, device="cuda")
    runs = []
    for _ in range(3):
        r = F.ssm_scan(**a, save=True)
        runs.append((r.y, r.ssm_state, F.ssm_scan_backward(dy, r.checkpoints, **a)))
    for y, h, g in runs[1:]:
        assert torch.equal(y, runs[0][0]) and torch.equal(h, runs[0][1])
        assert all(torch.equal(g[k], runs[0][2][k]) for k in g)


def test_autograd_function_with_broadcast_inputs(F):
    """B and C shared by all rows (stride 0): the gradient of the shared tensor is the rows' sum."""
    a = make(3, 40, 24, 8, states=False, views=False, seed=12)
    b1 = a["B"][:1].clone().requires_grad_()
    names = ("x", "dt", "A", "B", "C", "conv_weight", "conv_bias", "skip", "dt_bias", "z")
    leaves = {k: a[k].clone().requires_grad_() for k in names if k != "B"}
    y = F.SsmScan.apply(*(b1.expand(3, -1, -1, -1) if k == "B" else leaves[k] for k in names), None)
    dy = torch.randn_like(y)
    y.backward(dy)
    ref = reference_gradients({**a, "B": a["B"][:1].expand(3, -1, -1, -1)}, dy)
    R.close(b1.grad, ref["dB"].sum(0, keepdim=True), terms=256, what="dB")
    for k, v in leaves.items():
        R.close(v.grad, ref[NAMES[k]], terms=256, what=k)


def test_calls_follow_the_current_stream(F):
    a = make(8, 512, 256, 16, seed=13, views=False)
    ref = F.ssm_scan(**a).y
    side = torch.cuda.Stream()
    late = dict(a, x=torch.zeros_like(a["x"]))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)               # the input arrives late on this stream
        late["x"].copy_(a["x"])
        y = F.ssm_scan(**late).y
    side.synchronize()
    assert torch.equal(y, ref)


def test_rows_beyond_32_bit_offsets(F):
    """A row stride that puts the last row past 2^31 elements."""
    rows, length, D, N = 3, 5, 8, 4
    pitch = 2 ** 30 + 64
    big = torch.zeros(2 * pitch + length * D, dtype=torch.bfloat16, device="cuda")
    a = make(rows, length, D, N, dtype=torch.bfloat16, seed=14, views=False)
    x = big.as_strided((rows, length, D), (pitch, D, 1))
    x.copy_(a["x"])
    assert torch.equal(F.ssm_scan(**{**a, "x": x}).y, F.ssm_scan(**a).y)


def test_refusals(F):
    a = make(2, 8, 16, 8, views=False)
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "x": a["x"].double()})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "x": a["x"].cpu()})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "x": a["x"].transpose(1, 2).contiguous().transpose(1, 2)})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "dt": a["dt"][:, :-1]})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "A": a["A"].half()})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "skip": a["skip"][:-1]})
    with pytest.raises(TypeError):
        F.ssm_scan(**{**a, "lengths": torch.ones(2, device="cuda")})
    with pytest.raises(F.ThemisError) as e:          # 5 taps
        F.ssm_scan(**{**a, "conv_weight": torch.zeros(16, 5, device="cuda"), "conv_state": torch.zeros(2, 4, 16, device="cuda")})
    assert e.value.code == F.E_UNSUPPORTED_SIZE
    big = make(1, 4, 8, 65, views=False)
    with pytest.raises(F.ThemisError) as e:
        F.ssm_scan(**big)
    assert e.value.code == F.E_UNSUPPORTED_SIZE
    three = {**a, "B": torch.zeros(2, 8, 3, 8, device="cuda"), "C": torch.zeros(2, 8, 3, 8, device="cuda")}
    with pytest.raises(F.ThemisError) as e:          # 16 channels in 3 groups
        F.ssm_scan(**three)
    assert e.value.code == F.E_INVALID_ARG
    long = make(1, 4096, 8, 8, views=False)
    with pytest.raises(F.ThemisError) as e:
        F.ssm_scan(**long, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == F.E_WORKSPACE_TOO_SMALL


# --- parts of several tiles ------------------------------------------------------------------------

def parts_of(F, a, backward):
    """Number of parts of the time axis, from the workspace that the call asks for."""
    names = ("x", "dt", "A", "B", "C", "conv_weight", "conv_bias", "skip", "dt_bias", "z", "conv_state", "ssm_state", "lengths")
    problem, _, N, W = F._ssm_args(**{k: a.get(k) for k in names}, step=False)
    (rows, length, D), G = a["x"].shape, a["B"].shape[2]
    tile = 128 if N <= 16 else 64 if N <= 32 else 16                # channels of a block of the gradients' kernel
    def need(s):
        sizes = [rows * s * D * N, rows * s * D] if s > 1 else []
        if backward:
            sizes += [rows * s * D * (N + 8), -(-(D // G) // tile) * rows * length * G * 2 * N]
            sizes += [rows * s * (W - 1) * D] * 2 if s > 1 else []
        return sum(-(-4 * v // 256) * 256 for v in sizes)
    found = [s for s in range(1, -(-length // F.SSM_CHUNK) + 1) if need(s) == F.themis_ssm_workspace_bytes(problem, backward)]
    assert len(found) == 1
    return found[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("state,views", [(1, False), (3, False), (4, False), (4, True), (8, False), (16, False), (16, True), (40, False)],
                         ids=lambda v: str(v))
def test_parts_of_several_tiles(F, state, views, dtype):
    """Parts that take both input buffers, with rows that are copied 16 bytes at a time (contiguous inputs of 136
    channels) and value by value (slices at an odd offset)."""
    a = make(8, 2041, 136, state, dtype=dtype, seed=30 + state, views=views)
    a["A"] = a["A"] * 0.02                   # long memories, so that the parts depend on each other
    chunks = -(-2041 // F.SSM_CHUNK)
    assert 2 <= parts_of(F, a, False) <= chunks // 4 and 2 <= parts_of(F, a, True) <= chunks // 2
    dy = torch.randn(8, 2041, 136, device="cuda").to(dtype)
    leaves = {k: a[k].detach().double().requires_grad_() for k in NAMES}
    y, conv, h = R.scan(**{**a, **leaves})
    ref = dict(zip((NAMES[k] for k in leaves), torch.autograd.grad(y, list(leaves.values()), dy.double())))
    r = F.ssm_scan(**a, save=True)
    got = F.ssm_scan_backward(dy, r.checkpoints, **a)
    R.close(r.y, y.detach(), terms=512, what="y")
    R.close(r.ssm_state, h.detach(), terms=512, what="state")
    assert torch.equal(r.conv_state.double(), conv.detach())
    for k in ref:
        R.close(got[k], ref[k], terms=1024, what=k)
    # rows that end inside a part, and before it
    ragged = dict(a, lengths=torch.tensor([0, 1, 40, 700, 701, 1500, 2040, 2041], dtype=torch.int32, device="cuda"))
    s = F.ssm_scan(**spoil(ragged), states=False)
    for b, n in enumerate(ragged["lengths"].tolist()):
        assert torch.equal(s.y[b, :n], r.y[b, :n]) and (s.y[b, n:] == 0).all()


@pytest.mark.parametrize("name", ["x", "dt", "A", "B", "C", "conv_weight", "conv_bias", "skip", "dt_bias", "z"])
def test_second_derivatives_are_refused(F, name):
    """Alone and in a sum with other terms, where a gradient without a graph would only go missing."""
    a = make(3, 20, 24, 8, states=False, views=False, seed=12)
    names = ("x", "dt", "A", "B", "C", "conv_weight", "conv_bias", "skip", "dt_bias", "z")
    leaves = [a[k].clone().requires_grad_() for k in names]
    at = leaves[names.index(name)]
    want, = torch.autograd.grad(F.SsmScan.apply(*leaves, None).sum(), at)
    g, = torch.autograd.grad(F.SsmScan.apply(*leaves, None).sum(), at, create_graph=True)
    assert torch.equal(g, want) and g.requires_grad
    with pytest.raises(RuntimeError, match="differentiated again"):
        (g.square().sum() + at.sum()).backward()


@pytest.mark.parametrize("length", [1, 6, 61, 700])
def test_states_that_forget_at_once(F, length):
    """A of the lowest value and of -inf: the factors are 0 at every time that exists and 1 at those that do not
    (behind a row's end, and up to the next multiple of the times that a kernel takes at once)."""
    rows = 3
    a = make(rows, length, 24, 8, dtype=torch.bfloat16, seed=40 + length, views=False)
    a["A"][:, 1], a["A"][:, 5], a["A"][3] = torch.finfo(torch.float32).min, -math.inf, -math.inf
    for lengths in (None, torch.tensor([0, max(1, length // 3), length], dtype=torch.int32, device="cuda")):
        b = dict(a) if lengths is None else dict(a, lengths=lengths)
        r = F.ssm_scan(**(b if lengths is None else spoil(b)))
        y, conv, h = R.scan(**b)
        R.close(r.y, y, terms=512, what="y")
        R.close(r.ssm_state, h, terms=512, what="state")
        assert torch.equal(r.conv_state.double(), conv)
    s = {k: (v[:, 0] if k in ("x", "dt", "z", "B", "C") else v.clone()) for k, v in a.items()}
    y, _, h = R.scan(**{k: (v[:, :1] if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items()})
    R.close(F.ssm_step(**s), y[:, 0], what="y of a step")
    R.close(s["ssm_state"], h, what="state of a step")
    # gradients for finite A (those of -inf are not a number by the formula: A exp(s A))
    a["A"] = a["A"].clamp_min(torch.finfo(torch.float32).min)
    lengths = torch.tensor([0, max(1, length // 3), length], dtype=torch.int32, device="cuda")
    dy = torch.randn(rows, length, 24, device="cuda").bfloat16()
    check_gradients(F, dict(a, lengths=lengths), dy, terms=1024, spoiled=spoil(dict(a, lengths=lengths)))


# --- fleets: what many rows run -------------------------------------------------------------------

DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])


@DTYPES
@pytest.mark.parametrize("views", [False, True], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("shape", [(2371, 264, 16, 1, 4), (2371, 263, 16, 1, 4), (2370, 264, 12, 1, 4), (4603, 264, 8, 2, 3), (1151, 264, 32, 1, 4),
                                   (579, 264, 64, 1, 2), (9301, 264, 4, 3, 4)], ids=str)
def test_step_of_many_rows(F, shape, views, dtype):
    """Several rows to a thread (two times 1.2 million lanes and more): whole blocks, the last block of a row, a rest of
    rows, inactive rows with NaN, states in place and elsewhere."""
    rows, D, N, G, W = shape
    a = make(rows, 1, D, N, G, W, dtype=dtype, seed=N, views=views)
    y, conv, h = R.scan(**a)
    s = {k: (v[:, 0] if k in ("x", "dt", "z", "B", "C") else v) for k, v in a.items()}
    kept = a["conv_state"].clone(), a["ssm_state"].clone()
    new_conv, new_h = torch.full_like(kept[0], 7), torch.full_like(kept[1], 7)
    got = F.ssm_step(**s, new_conv_state=new_conv, new_ssm_state=new_h)
    R.close(got, y[:, 0], what="y")
    R.close(new_h, h, what="state")
    assert torch.equal(new_conv.double(), conv)
    assert torch.equal(a["conv_state"], kept[0]) and torch.equal(a["ssm_state"], kept[1])
    active = (torch.arange(rows, device="cuda") * 2654435761 % 7 < 5).int()
    active[-1] = 0
    off = active == 0
    for k in ("x", "dt", "z", "B", "C"):
        s[k][off] = float("nan")
    in_place = F.ssm_step(**s, active=active)
    assert (in_place[off] == 0).all() and torch.equal(in_place[~off], got[~off])
    assert torch.equal(a["ssm_state"][~off], new_h[~off]) and torch.equal(a["conv_state"][~off], new_conv[~off])
    assert torch.equal(a["ssm_state"][off], kept[1][off]) and torch.equal(a["conv_state"][off], kept[0][off])


def check_all(F, a, dy, terms):
    """Forward and gradients against 64 bits."""
    leaves = {k: a[k].detach().double().requires_grad_() for k in NAMES if k in a}
    y, conv, h = R.scan(**{**a, **leaves})
    ref = dict(zip((NAMES[k] for k in leaves), torch.autograd.grad(y, list(leaves.values()), dy.double())))
    given = spoil(a) if "lengths" in a else a
    plain = F.ssm_scan(**given)
    r = F.ssm_scan(**given, save=True)
    assert torch.equal(plain.y, r.y) and torch.equal(plain.ssm_state, r.ssm_state)
    R.close(r.y, y.detach(), what="y")
    R.close(r.ssm_state, h.detach(), what="state")
    assert torch.equal(r.conv_state.double(), conv.detach())
    got = F.ssm_scan_backward(dy, r.checkpoints, **given)
    assert set(got) == set(ref)
    for k in ref:
        R.close(got[k], ref[k], terms=terms, what=k)


# rows, length, D, N, G, W; enough rows for 16 states on a lane (with 1, 2 and 4 lanes to a channel) and 8 (1, 2)
FLEETS = [(90, 37, 504, 16, 1, 4), (90, 37, 505, 13, 1, 3), (124, 40, 264, 8, 1, 4), (204, 35, 136, 5, 1, 2), (124, 40, 136, 16, 1, 4),
          (124, 33, 272, 24, 2, 4), (30, 70, 136, 64, 1, 4)]


@DTYPES
@pytest.mark.parametrize("ragged", [False, True], ids=["whole", "ragged"])
@pytest.mark.parametrize("shape", FLEETS, ids=str)
def test_many_rows(F, shape, ragged, dtype):
    a = make(*shape, dtype=dtype, seed=sum(shape), ragged=ragged, views=ragged)
    dy = torch.randn(shape[0], shape[1], shape[2], device="cuda").to(dtype)
    # parameters' gradients sum rows x times (about 4000) terms of some tens of roundings each: 64 times the square root
    check_all(F, a, dy, terms=1024)


@DTYPES
@pytest.mark.parametrize("views", [False, True], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("shape", [(300, 197, 40, 16, 1, 4), (300, 200, 40, 32, 1, 3), (450, 150, 24, 40, 1, 4), (600, 150, 40, 8, 1, 4),
                                   (600, 150, 40, 4, 1, 4), (600, 131, 40, 3, 1, 2)], ids=str)
def test_gradients_of_many_chunks_in_one_part(F, shape, views, dtype):
    """Rows that fill the GPU are not split: nine to thirteen chunks one after the other in a block."""
    a = make(*shape, dtype=dtype, seed=sum(shape), views=views)
    assert parts_of(F, a, True) == 1
    dy = torch.randn(shape[0], shape[1], shape[2], device="cuda").to(dtype)
    check_all(F, a, dy, terms=1024)
