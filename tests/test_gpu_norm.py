"""The root-mean-square norm against a plain implementation in 64 bits: widths of every kernel, one row to thousands, both types, 8-bit outputs, gradients, in place, replayed."""
import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


def rows(seed, T, n, dtype, scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.empty((T, n), device="cuda").normal_(0.0, scale, generator=gen)
    x[:, ::37] *= 9.0
    return x.to(dtype)


def weight(seed, n, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(n, device="cuda").normal_(1.0, 0.3, generator=gen).to(dtype)


# a width for every form of the kernel, most of them no whole number of vectors of the lanes
WIDTHS = [8, 64, 72, 128, 136, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 5120, 6152, 8192, 8200, 16384, 16392, 32768]


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n", WIDTHS)
def test_forward(n, dtype):
    for T in (1, 7):
        X, R, W = rows(n, T, n, dtype), rows(n + 1, T, n, dtype), weight(n + 2, n, torch.float32 if T == 1 else dtype)
        out = eq.eqat_norm_fwd(X, W, EPS, R=R, want=("S", "Y"))
        S, _, Y = ref.norm(X, W, EPS, R)
        assert torch.equal(out["S"], S)
        ref.within(out["Y"], Y, Y.abs() * (ref.half(dtype) + ref.NORM_ROUNDINGS * ref.F32))
        plain = eq.eqat_norm_fwd(X, None, EPS)["Y"]
        Y = ref.norm(X, None, EPS)[2]
        ref.within(plain, Y, Y.abs() * (ref.half(dtype) + ref.NORM_ROUNDINGS * ref.F32))


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n, group", [(32, 32), (64, -1), (96, 32), (256, 64), (512, 512), (1536, 512), (640, 128), (4096, 256), (5120, -1), (5120, 128), (8192, 32), (32768, -1), (8200, -1), (512, 256)])
def test_eight_bits(n, group, dtype):
    T = 5
    X, R, W = rows(n, T, n, dtype), rows(n + 1, T, n, dtype), weight(3, n, dtype)
    X[2] = 0
    R[2] = 0                             # a row of zeros: scale 2^-126, codes 0
    out = eq.eqat_norm_fwd(X, W, EPS, R=R, group=group, want=("S", "Y", "codes"))
    S, _, Y = ref.norm(X, W, EPS, R)
    assert torch.equal(out["S"], S)
    ref.within(out["Y"], Y, Y.abs() * (ref.half(dtype) + ref.NORM_ROUNDINGS * ref.F32))
    y = Y.unflatten(1, (-1, n if group == -1 else group))
    scale = (y.abs().amax(-1) / 448.0).clamp_min(2.0 ** -126)
    ref.within(out["scales"], scale, scale * (ref.NORM_ROUNDINGS + 1) * ref.F32)
    v = (y / scale[..., None]).flatten(1)
    # half a step, and what Y, its scale, the reciprocal and the product are off by before it is rounded (and with it, at a power of two, the step)
    loose = v.abs() * (2 * ref.NORM_ROUNDINGS + 3) * ref.F32
    ref.within(out["codes"].float(), v, ref.e4m3_step(v.abs() + loose) / 2 + loose)
    assert not out["codes"][2].float().any() and (out["scales"][2] == 2.0 ** -126).all()
    only = eq.eqat_norm_fwd(X, W, EPS, R=R, group=group)
    assert torch.equal(only["codes"].view(torch.uint8), out["codes"].view(torch.uint8)) and torch.equal(only["scales"], out["scales"]) and set(only) == {"S", "codes", "scales"}


def check_back(T, n, dtype, with_ds=True, w_dtype=torch.float32):
    S, W, dY, dS = rows(n, T, n, dtype), weight(n + 2, n, w_dtype), rows(n + 3, T, n, dtype, 0.02), rows(n + 4, T, n, dtype, 0.02) if with_ds else None
    out = eq.eqat_norm_bwd(S, W, EPS, dY, dS)
    dX, dW, bound, terms = ref.norm_back(S, W, EPS, dY, dS)
    ref.within(out["dX"], dX, bound)
    # rows that a workgroup adds up one after the other (a 512th of them), at most 8 of the same workgroup and 48 parts; rstd's and the product's roundings
    ref.within(out["dW"], dW, terms.abs().sum(0) * (T // 512 + 1 + 8 + 48 + ref.NORM_ROUNDINGS + 2) * ref.F32)
    return S, W, dY, dS, out


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n", WIDTHS)
def test_backward(n, dtype):
    check_back(1, n, dtype)
    check_back(13, n, dtype, with_ds=False, w_dtype=dtype)


@pytest.mark.parametrize("T, n", [(515, 4096), (1025, 1024), (5000, 64), (2049, 520), (3, 32768), (8192, 128)])
def test_backward_of_many_rows(T, n):
    S, W, dY, dS, out = check_back(T, n, torch.bfloat16)
    again = eq.eqat_norm_bwd(S, W, EPS, dY, dS)
    assert torch.equal(again["dX"], out["dX"]) and torch.equal(again["dW"], out["dW"])
    one = eq.eqat_norm_bwd(S, W, EPS, dY, dS, want=("dX",))
    other = eq.eqat_norm_bwd(S, W, EPS, dY, dS, want=("dW",))
    assert set(one) == {"dX"} and set(other) == {"dW"} and torch.equal(one["dX"], out["dX"]) and torch.equal(other["dW"], out["dW"])


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("T, n", [(257, 4104), (300, 6152), (300, 8192), (260, 8200), (257, 16384), (259, 1024), (1030, 8)])
def test_more_rows_than_compute_units(T, n, dtype):
    """other forms of the kernels take these"""
    X, R, W = rows(n, T, n, dtype), rows(n + 1, T, n, dtype), weight(n + 2, n, torch.float32)
    out = eq.eqat_norm_fwd(X, W, EPS, R=R, group=-1, want=("S", "Y", "codes"))
    S, _, Y = ref.norm(X, W, EPS, R)
    assert torch.equal(out["S"], S)
    ref.within(out["Y"], Y, Y.abs() * (ref.half(dtype) + ref.NORM_ROUNDINGS * ref.F32))
    scale = Y.abs().amax(-1, keepdim=True) / 448.0
    ref.within(out["scales"], scale, scale * (ref.NORM_ROUNDINGS + 1) * ref.F32)
    check_back(T, n, dtype)


def test_gradient_against_differences():
    T, n, h = 2, 72, 1e-3
    X, R, W, dY, dS = (rows(i, T, n, torch.float32) for i in range(5))
    W = weight(9, n, torch.float32)
    S = eq.eqat_norm_fwd(X, W, EPS, R=R)["S"]
    out = eq.eqat_norm_bwd(S, W, EPS, dY, dS)

    def loss(x, w):
        S, _, Y = ref.norm(x, None, EPS)
        return float((Y * w * dY.double()).sum() + (S.double() * dS.double()).sum())

    for k in range(0, T * n, 11):
        e = torch.zeros(T * n, dtype=torch.float64, device="cuda")
        e[k] = h
        e = e.view(T, n)
        d = (loss(S.double() + e, W.double()) - loss(S.double() - e, W.double())) / (2 * h)
        # the third derivative's share, h^2 / 6 of numbers of some 100, and 1e-12 of the loss over h
        assert abs(d - float(out["dX"].flatten()[k])) <= 1e-4 + 1e-5 * abs(d)
    for k in range(0, n, 7):
        e = torch.zeros(n, dtype=torch.float64, device="cuda")
        e[k] = h
        d = (loss(S.double(), W.double() + e) - loss(S.double(), W.double() - e)) / (2 * h)
        assert abs(d - float(out["dW"][k])) <= 1e-4 + 1e-5 * abs(d)


def test_no_rows():
    X = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    assert eq.eqat_norm_fwd(X, None, EPS, group=32)["scales"].shape == (0, 8)
    out = eq.eqat_norm_bwd(X, None, EPS, X, out={"dW": torch.full((256,), 7.0, device="cuda")})
    assert not out["dW"].any()


@pytest.mark.parametrize("n", (64, 1024, 5120))
def test_in_place(n):
    T, dt = 9, torch.bfloat16
    X, R, W = rows(1, T, n, dt), rows(2, T, n, dt), weight(3, n, dt)
    want = eq.eqat_norm_fwd(X, W, EPS, R=R, want=("S", "Y"))
    for s, y in (("R", "X"), ("X", "R"), ("X", None), ("R", None)):
        t = {"X": X.clone(), "R": R.clone()}
        out = eq.eqat_norm_fwd(t["X"], W, EPS, R=t["R"], want=("S", "Y"), out={"S": t[s], "Y": t[y] if y else torch.empty_like(X)})
        assert torch.equal(out["S"], want["S"]) and torch.equal(out["Y"], want["Y"])
    dY, dS = rows(4, T, n, dt), rows(5, T, n, dt)
    want = eq.eqat_norm_bwd(X, W, EPS, dY, dS)
    for name in ("S", "dY", "dS"):
        t = {"S": X.clone(), "dY": dY.clone(), "dS": dS.clone()}
        out = eq.eqat_norm_bwd(t["S"], W, EPS, t["dY"], t["dS"], out={"dX": t[name]})
        assert torch.equal(out["dX"], want["dX"]) and torch.equal(out["dW"], want["dW"])


def test_rows_that_are_not_numbers_stay_alone():
    T, n = 6, 1032
    X, W = rows(1, T, n, torch.bfloat16), weight(2, n, torch.float32)
    clean = eq.eqat_norm_fwd(X, W, EPS, group=-1, want=("Y", "codes"))
    clean = {k: v.float() for k, v in clean.items()}
    X[1, 5], X[3, 7] = float("nan"), float("inf")
    out = eq.eqat_norm_fwd(X, W, EPS, group=-1, want=("Y", "codes"))
    others = [0, 2, 4, 5]
    for k in ("Y", "codes", "scales"):
        assert torch.equal(out[k].float()[others], clean[k][others])
    assert out["Y"][1].isnan().all() and out["scales"][1].isnan().all() and out["codes"][1].float().isnan().all() and out["Y"][3, 7].isnan()


def test_nothing_beside_the_tensors_is_touched():
    T, n, dt = 3, 1032, torch.bfloat16
    guard = lambda t: torch.nn.functional.pad(t.flatten(), (64, 64), value=77.0)
    X, R, W = rows(1, T, n, dt), rows(2, T, n, dt), weight(3, n, dt)
    whole = {k: guard(torch.zeros((T, n), dtype=d, device="cuda")) for k, d in (("S", dt), ("Y", dt), ("dX", dt))}
    whole["dW"] = guard(torch.zeros(n, device="cuda"))
    inner = {k: v[64:-64].view(-1, n) if k != "dW" else v[64:-64] for k, v in whole.items()}
    eq.eqat_norm_fwd(X, W, EPS, R=R, want=("S", "Y"), out=inner)
    eq.eqat_norm_bwd(X, W, EPS, R, out=inner)
    for v in whole.values():
        assert (v[:64] == 77).all() and (v[-64:] == 77).all()


def test_replayed_and_on_another_stream():
    T, n, dt = 700, 1024, torch.bfloat16
    X, R, W, dY = rows(1, T, n, dt), rows(2, T, n, dt), weight(3, n, torch.float32), rows(4, T, n, dt)
    ws = eq.norm_workspace(T, n)
    fwd, bwd = {"S": torch.empty_like(X), "Y": torch.empty_like(X)}, {"dX": torch.empty_like(X), "dW": torch.empty(n, device="cuda")}

    def step():
        eq.eqat_norm_fwd(X, W, EPS, R=R, want=("S", "Y"), out=fwd)
        eq.eqat_norm_bwd(fwd["S"], W, EPS, dY, out=bwd, ws=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for k in range(3):
        X.copy_(rows(10 + k, T, n, dt))
        W.copy_(weight(20 + k, n, torch.float32))
        want = eq.eqat_norm_fwd(X, W, EPS, R=R, want=("S", "Y"))
        back = eq.eqat_norm_bwd(want["S"], W, EPS, dY)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((fwd, want), (bwd, back)):
            assert all(torch.equal(a[name], b[name]) for name in b)
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert torch.equal(bwd["dW"], back["dW"]) and torch.equal(fwd["Y"], want["Y"])


def test_offsets_beyond_32_bits():
    """4.3 GB a tensor: the last rows are those of a call of their own"""
    T, n, dt = 525_000, 4096, torch.bfloat16
    tail = 3
    X = torch.zeros((T, n), dtype=dt, device="cuda")
    X[-tail:] = rows(1, tail, n, dt)
    W = weight(2, n, torch.float32)
    Y = torch.empty_like(X)
    eq.eqat_norm_fwd(X, W, EPS, want=("Y",), out={"Y": Y})
    assert torch.equal(Y[-tail:], eq.eqat_norm_fwd(X[-tail:], W, EPS)["Y"]) and not Y[:5].any() and not Y[T // 2:T // 2 + 5].any()
    dY = torch.zeros_like(X)
    dY[-tail:] = rows(3, tail, n, dt)
    out = eq.eqat_norm_bwd(X, W, EPS, dY, out={"dX": Y})
    want = eq.eqat_norm_bwd(X[-tail:], W, EPS, dY[-tail:])
    assert torch.equal(Y[-tail:], want["dX"]) and not Y[:-tail].any()
    _, dW, _, terms = ref.norm_back(X[-tail:], W, EPS, dY[-tail:])
    ref.within(out["dW"], dW, terms.abs().sum(0) * (T // 512 + 1 + 8 + 48 + ref.NORM_ROUNDINGS + 2) * ref.F32)
