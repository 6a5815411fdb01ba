"""Dense gated feed-forward block, forward and backward, against the definition in 64 bits.

Tolerances, element by element.  `half` is half a step of the type, finfo.eps / 2; a sum of K products in fp32 is
within K * 2^-23 of the sum of their sizes (each addition may cut off a step); a, dg and du are rounded to the
type before they are multiplied; |silu'| < 1.1, |silu''| <= 0.5, and the exponential's error is below 2^-18 of a
result at the arguments that occur.  These errors are carried through the following products with the operands'
sizes.  The 2-norm of the error is held to `half` as well: one rounding of random values has a 2-norm of
half / sqrt(3) or less, and no output has more than two of them behind it that count in full, plus smaller ones,
while a lost block of 64 of a contraction of n blocks would be off by 1 / sqrt(n)."""
import ctypes

import pytest
import torch

from paper_2402_14800_b200 import binding, build, synth

E23 = 2.0 ** -23
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load_library()


# ------------------------------------------------------------------------------- no device


def test_refuses_bad_arguments_without_a_device(lib):
    p = [ctypes.c_void_p((i + 1) << 24) for i in range(14)]
    odd = ctypes.c_void_p((1 << 24) + 8)
    names = ("x", "W1", "W3", "W2", "residual", "y", "saved", "ws")

    def fwd(T=4, h=64, f=128, dt=0, n=1 << 22, **kw):
        a = {k: p[i] for i, k in enumerate(names)}
        a.update(kw)
        return lib.moe_ffn_forward(a["x"], a["W1"], a["W3"], a["W2"], a["residual"], T, h, f, dt, a["y"], a["saved"],
                                   a["ws"], n, None)

    for k in ("x", "W1", "W3", "W2", "y"):
        assert fwd(**{k: None}) == -1 and "NULL" in binding.last_error(), k
    for k in names:
        assert fwd(**{k: odd}) == -1 and "aligned" in binding.last_error(), k
    assert fwd(ws=None) == -1 and "workspace" in binding.last_error()
    assert fwd(n=4 * 128 * 2 - 1) == -1 and "workspace" in binding.last_error()
    for k in ("x", "W1", "W3", "W2", "saved"):
        assert fwd(y={"x": p[0], "W1": p[1], "W3": p[2], "W2": p[3], "saved": p[6]}[k]) == -1, k
        assert "overlap" in binding.last_error()
    assert fwd(y=ctypes.c_void_p((5 << 24) + 64)) == -1 and "overlap" in binding.last_error()
    for i, k in enumerate(names[:-1]):
        assert fwd(ws=p[i]) == -1 and "workspace overlaps" in binding.last_error(), k
        if k not in ("y", "saved"):
            assert fwd(saved=p[i]) == -1 and "saved overlaps" in binding.last_error(), k
    assert fwd(dt=2) == -1 and "dtype" in binding.last_error()  # the tensor cores' 16-bit types
    assert fwd(h=68) == -2 and fwd(f=4) == -2 and fwd(h=0) == -2 and fwd(f=(1 << 20) + 8) == -2
    assert fwd(T=-1) == -1 and fwd(T=(1 << 24) + 1) == -1
    assert fwd(T=0) == 0

    names_b = ("dy", "x", "W1", "W3", "W2", "saved", "dx", "dW1", "dW3", "dW2", "ws")

    def bwd(T=4, h=64, f=128, dt=0, n=1 << 22, **kw):
        a = {k: p[i] for i, k in enumerate(names_b)}
        a.update(kw)
        return lib.moe_ffn_backward(a["dy"], a["x"], a["W1"], a["W3"], a["W2"], a["saved"], T, h, f, dt, a["dx"],
                                    a["dW1"], a["dW3"], a["dW2"], a["ws"], n, None)

    for k in names_b[:-1]:
        assert bwd(**{k: None}) == -1 and "NULL" in binding.last_error(), k
    for i, k in enumerate(names_b):
        assert bwd(**{k: ctypes.c_void_p(((i + 1) << 24) + 8)}) == -1 and "aligned" in binding.last_error(), k
    for k in ("dx", "dW1", "dW3", "dW2"):
        for i in range(6):
            assert bwd(**{k: p[i]}) == -1 and "overlaps an input" in binding.last_error()
    assert bwd(dW1=p[8]) == -1 and "two gradients" in binding.last_error()
    for i in range(10):
        assert bwd(ws=p[i]) == -1 and "workspace overlaps" in binding.last_error(), names_b[i]
    assert bwd(ws=None) == -1 and bwd(n=100) == -1 and "workspace" in binding.last_error()
    assert bwd(dt=2) == -1 and bwd(h=12) == -2 and bwd(T=-1) == -1
    assert lib.moe_ffn_saved_bytes(0, 64) == 0 and lib.moe_ffn_saved_bytes(3, 60) == 0
    assert lib.moe_ffn_saved_bytes(3, 64) == 3 * 64 * 8 + 3 * 64 * 2
    assert lib.moe_ffn_saved_bytes(1, 8) == 256 + 16
    assert lib.moe_ffn_forward_workspace(0, 64, 64) == 0 and lib.moe_ffn_backward_workspace(3, 60, 64) == 0


@pytest.mark.parametrize("h,f", [(8, 8), (64, 8), (128, 448), (1000, 2728), (2040, 5464), (4096, 14336), (14336, 4096),
                                 (8, 1 << 20), (1 << 20, 8)])
def test_tiles_cover_every_output(lib, h, f):
    """What the kernel's index arithmetic rests on, for every launch and many batch sizes: the tiles cover the outputs,
    no split is empty, rows and columns fit an accumulator, stores of two neighbouring rows do not straddle a tile."""
    out = (ctypes.c_int * 6)()
    for T in (1, 2, 15, 33, 64, 100, 128, 200, 256, 257, 400, 611, 1000, 1024, 2048, 5000, 8192, 100000):
        for pairs in (74, 66, 1):
            for launch in range(5):
                assert lib.moe_test_ffn_plan(launch, T, h, f, pairs, out) == 0
                R, n_tile, S, mt, nt, kb = list(out)
                kbs = -(-kb // S)
                assert 1 <= S <= 16 and (S - 1) * kbs < kb <= S * kbs
                if launch == 4:
                    assert R in (64, 128) and n_tile in (32, 64, 128, 256) and kb == -(-T // 64)
                    assert S == 1 or pairs != 74 or lib.moe_ffn_backward_workspace(T, h, f) >= T * f * 4 + 3 * S * f * h * 4
                    continue
                M = f if launch in (0, 2) else h
                unit = 2 if launch == 0 else 4
                assert 8 <= R <= 128 and R % (64 if launch >= 2 else 8) == 0, (T, launch, list(out))
                assert n_tile % 16 == 0 and 16 <= n_tile <= (128 if T <= 128 else 256)
                assert (mt - 1) * unit * R < M <= mt * unit * R and (nt - 1) * n_tile < T <= nt * n_tile
                if launch == 0:
                    assert S == 1  # the activation needs whole sums
                # a stage of the pipeline fits, and so does what an MMA reads behind the last one
                slot = -(-R // 64) * 8192 if launch >= 2 else -(-R // 8) * 1024
                stage, tail = 2 * slot + n_tile * 64, max(0, 16384 - slot)
                kept = 65536 if launch == 2 else 0  # of the da launch's epilogue; a fourth of it in the slim form
                assert 1024 + tail + 2 * stage + kept <= 230400 and (T > 64 or M * kb * 128 >= 96 << 20 or 1024 + tail + 2 * stage + kept // 4 <= 114688)
                if S > 1:
                    ws = lib.moe_ffn_forward_workspace if launch == 1 else lib.moe_ffn_backward_workspace
                    if pairs == 74:  # without a device the library assumes 148 multiprocessors
                        assert ws(T, h, f) >= T * f * 2 * (1 if launch == 1 else 2) + S * T * M * 4


def test_binding_refuses_host_tensors(lib):
    x, W, V = torch.zeros((4, 64)).bfloat16(), torch.zeros((8, 64)).bfloat16(), torch.zeros((64, 8)).bfloat16()
    with pytest.raises(binding.MoeError):
        binding.ffn_forward(x, W, W, V)
    with pytest.raises(binding.MoeError):
        binding.ffn_backward(x, x, W, W, V, torch.zeros(lib.moe_ffn_saved_bytes(4, 8), dtype=torch.uint8))


@gpu
def test_binding_refuses_wrong_tensors():
    x, W1, W3, W2, dy = make(4, 64, 128, torch.bfloat16)
    saved = binding.ffn_saved(4, 128, DEV)
    bad = [lambda: binding.ffn_forward(x.float(), W1.float(), W3.float(), W2.float()), lambda: binding.ffn_forward(x, W1, W3, W1),
           lambda: binding.ffn_forward(x, W1, W3[:64], W2), lambda: binding.ffn_forward(x, W1, W3, W2.half()),
           lambda: binding.ffn_forward(x[:, :60], W1, W3, W2), lambda: binding.ffn_forward(x, W2.T, W3, W2),
           lambda: binding.ffn_forward(x[0], W1, W3, W2), lambda: binding.ffn_forward(x, W1, W3, W2, saved=saved[:3]),
           lambda: binding.ffn_forward(x, W1, W3, W2, y=x), lambda: binding.ffn_forward(x, W1, W3, W2, residual=x[:3]),
           lambda: binding.ffn_forward(x, W1.cpu(), W3, W2), lambda: binding.ffn_forward(x, None, W3, W2),
           lambda: binding.ffn_backward(dy, x, W1, W3, W2, None), lambda: binding.ffn_backward(dy[:3], x, W1, W3, W2, saved),
           lambda: binding.ffn_backward(dy, x, W1, W3, W2, saved, dW1=W1), lambda: binding.ffn_backward(dy, x, W1, W3, W2, saved, dx=dy)]
    for call in bad:
        with pytest.raises(binding.MoeError):
            call()


# ------------------------------------------------------------------------------- against 64 bits


def make(T, h, f, dt, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)

    return (normal(T, h), normal(f, h, std=1.28 / h ** 0.5), normal(f, h, std=1.28 / h ** 0.5), normal(h, f, std=1.28 / f ** 0.5),
            normal(T, h, std=0.1))


def reference(x, W1, W3, W2, dy=None):
    """Outputs in 64 bits and their tolerances: {name: (value, tolerance)}."""
    dt = x.dtype
    half, least = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    (T, h), f = x.shape, W1.shape[0]
    x, W1, W3, W2 = (t.double() for t in (x, W1, W3, W2))
    g, u = x @ W1.T, x @ W3.T
    eg, eu = h * E23 * (x.abs() @ W1.abs().T), h * E23 * (x.abs() @ W3.abs().T)
    sig = torch.sigmoid(g)
    sw = g * sig
    a = sw * u
    ea = half * a.abs() + least + 1.1 * eg * u.abs() + sw.abs() * eu + 1.1 * eg * eu + 2.0 ** -18 * a.abs()
    y = a @ W2.T
    out = dict(y=(y, half * y.abs() + least + ea @ W2.abs().T + f * E23 * (a.abs() @ W2.abs().T)))
    if dy is None:
        return out
    dy = dy.double()
    da = dy @ W2
    eda = h * E23 * (dy.abs() @ W2.abs())
    slope = sig + sw * (1 - sig)
    dg, du = da * u * slope, da * sw
    edg = half * dg.abs() + least + eda * (u * slope).abs() + da.abs() * (1.1 * eu + u.abs() * 0.5 * eg) + 2.0 ** -18 * (da * u).abs()
    edu = half * du.abs() + least + eda * sw.abs() + da.abs() * 1.1 * eg + 2.0 ** -18 * du.abs()

    def add(name, want, tol):
        out[name] = (want, half * want.abs() + least + tol)

    add("dx", dg @ W1 + du @ W3,
        edg @ W1.abs() + edu @ W3.abs() + 2 * f * E23 * (dg.abs() @ W1.abs() + du.abs() @ W3.abs()))
    add("dW1", dg.T @ x, edg.T @ x.abs() + T * E23 * (dg.abs().T @ x.abs()))
    add("dW3", du.T @ x, edu.T @ x.abs() + T * E23 * (du.abs().T @ x.abs()))
    add("dW2", dy.T @ a, dy.abs().T @ ea + T * E23 * (dy.abs().T @ a.abs()))
    return out


def check(got, want, dt, name):
    value, tol = want
    off = (got.double() - value).abs() - tol * (1 + 1e-6)
    assert bool((off <= 0).all()), "%s: worst excess %.3g at %d" % (name, float(off.max()), int(off.argmax()))
    if value.numel() < 4096:  # too few values for their mean
        return
    rel = float((got.double() - value).norm() / value.norm())
    assert rel < torch.finfo(dt).eps / 2, "%s: 2-norm of the error %.3g" % (name, rel)


SIZES = [(1, 8, 8), (3, 64, 8), (2, 8, 200), (1, 128, 448), (100, 128, 448), (31, 72, 136), (33, 520, 264), (128, 1000, 2728),
         (256, 256, 512), (257, 264, 520), (300, 2048, 4096), (611, 2040, 5464), (1025, 512, 1032), (2500, 136, 72),
         (5000, 64, 64), (8000, 128, 448), (3000, 256, 1032), (1500, 40, 520)]
FEW = [(2, 4096, 14336), (3, 4096, 14336), (4, 40, 24), (5, 128, 448), (7, 4096, 14336), (8, 2040, 5464), (9, 1000, 2728),
       (16, 2048, 4096), (24, 264, 1032), (32, 1024, 2048), (33, 640, 1032), (50, 72, 1528), (64, 512, 1024), (64, 1528, 8),
       (40, 8, 1528), (12, 4096, 72), (6, 72, 14336),
       (5, 2400, 1200), (20, 2400, 1200)]  # blocks of unequal numbers of tiles


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,h,f", SIZES + FEW + [(1, 4096, 14336), (17, 4096, 14336), (128, 4096, 14336), (200, 4096, 14336),
                                           (1000, 4096, 14336)])
def test_forward(T, h, f, dt):
    dt = TYPES[dt]
    x, W1, W3, W2, _ = make(T, h, f, dt, seed=T + h)
    y = binding.ffn_forward(x, W1, W3, W2)
    check(y, reference(x, W1, W3, W2)["y"], dt, "y")
    assert torch.equal(binding.ffn_forward(x, W1, W3, W2), y)  # a fixed order of the sums
    saved = binding.ffn_saved(T, f, DEV)
    y2 = binding.ffn_forward(x, W1, W3, W2, saved=saved)
    check(y2, reference(x, W1, W3, W2)["y"], dt, "y")
    if T > 32:  # few tokens have kernels of their own where nothing is saved
        assert torch.equal(y2, y)
    # what is saved: u silu'(g) and silu(g) in fp32, then a
    g, u = x.double() @ W1.double().T, x.double() @ W3.double().T
    eg, eu = (h * E23 * (x.double().abs() @ W.double().abs().T) for W in (W1, W3))
    sig = torch.sigmoid(g)
    p, q = u * (sig + g * sig * (1 - sig)), g * sig
    kept = saved[: T * f * 8].view(torch.float32).view(T, f, 2).double()
    assert bool(((kept[:, :, 0] - p).abs() <= 1.1 * eu + u.abs() * 0.5 * eg + 0.5 * eu * eg + 2.0 ** -18 * u.abs()).all())
    assert bool(((kept[:, :, 1] - q).abs() <= 1.1 * eg + 2.0 ** -18 * q.abs() + 1e-37).all())
    a = saved[-(-T * f * 8 // 256) * 256:].view(dt).view(T, f).double()
    half = torch.finfo(dt).eps / 2
    assert bool(((a - q * u).abs() <= half * (q * u).abs() * 1.01 + 1.1 * eg * u.abs() + q.abs() * eu + 1.1 * eg * eu + 2.0 ** -17 * a.abs()
                 + torch.finfo(dt).smallest_normal * half * 2).all())
    assert binding.operators_status(DEV) == 0


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,h,f", SIZES + [(1, 4096, 14336), (65, 4096, 14336), (600, 4096, 14336)])
def test_backward(T, h, f, dt):
    dt = TYPES[dt]
    x, W1, W3, W2, dy = make(T, h, f, dt, seed=3 * T + h)
    saved = binding.ffn_saved(T, f, DEV)
    binding.ffn_forward(x, W1, W3, W2, saved=saved)
    got = dict(zip(("dx", "dW1", "dW3", "dW2"), binding.ffn_backward(dy, x, W1, W3, W2, saved)))
    want = reference(x, W1, W3, W2, dy)
    for k, v in got.items():
        check(v, want[k], dt, k)
    again = binding.ffn_backward(dy, x, W1, W3, W2, saved)
    assert all(torch.equal(a, b) for a, b in zip(again, got.values()))
    assert binding.operators_status(DEV) == 0


@gpu
def test_backward_is_the_slope_of_forward():
    # <gradient, direction> against central differences of L = <dy, y> in 64 bits; the gradients carry the roundings of
    # their type: a sum of n products of independent errors is within 4 standard deviations of n's root
    T, h, f = 40, 136, 200
    x, W1, W3, W2, dy = make(T, h, f, torch.float16, seed=2)
    saved = binding.ffn_saved(T, f, DEV)
    binding.ffn_forward(x, W1, W3, W2, saved=saved)
    grads = binding.ffn_backward(dy, x, W1, W3, W2, saved)
    at = [t.double() for t in (x, W1, W3, W2)]

    def loss(x, W1, W3, W2):
        g = x @ W1.T
        return float((((g * torch.sigmoid(g)) * (x @ W3.T)) @ W2.T * dy.double()).sum())

    gen = torch.Generator(DEV).manual_seed(7)
    for k, grad in enumerate(grads):
        d = torch.randn(at[k].shape, generator=gen, device=DEV, dtype=torch.float64)
        d /= d.norm()
        step = 1e-4
        hi, lo = list(at), list(at)
        hi[k], lo[k] = at[k] + step * d, at[k] - step * d
        slope = (loss(*hi) - loss(*lo)) / (2 * step)
        tol = 4 * torch.finfo(torch.float16).eps * float(grad.double().norm()) / grad.numel() ** 0.5 * 2 + 1e-6
        assert abs(slope - float((grad.double() * d).sum())) < tol + 1e-6 * abs(slope), (k, slope)


# ------------------------------------------------------------------------------- edges


@gpu
@pytest.mark.parametrize("T", [1, 2, 6, 40, 300])
@pytest.mark.parametrize("dt", list(TYPES))
def test_residual_is_added_before_the_rounding(T, dt):
    dt = TYPES[dt]
    h, f = 1000, 2728
    x, W1, W3, W2, _ = make(T, h, f, dt, seed=11)
    r = make(T, h, 8, dt, seed=12)[0]
    value, tol = reference(x, W1, W3, W2)["y"]
    half = torch.finfo(dt).eps / 2
    y = binding.ffn_forward(x, W1, W3, W2, residual=r)
    want = value + r.double()
    check(y, (want, tol + half * (want.abs() - value.abs()).clamp_min(0) + 2 * E23 * (value.abs() + r.double().abs())), dt, "y")
    mine = r.clone()
    assert torch.equal(binding.ffn_forward(x, W1, W3, W2, residual=mine, y=mine), y)


@gpu
def test_no_tokens():
    h, f = 64, 128
    x, W1, W3, W2, dy = make(3, h, f, torch.bfloat16)
    assert binding.ffn_forward(x[:0], W1, W3, W2).shape == (0, h)
    bufs = [torch.full_like(t, 7.0) for t in (W1, W3, W2)]
    dx, *grads = binding.ffn_backward(dy[:0], x[:0], W1, W3, W2, binding.ffn_saved(0, f, DEV), dW1=bufs[0], dW3=bufs[1], dW2=bufs[2])
    assert dx.shape == (0, h) and not any(t.any() for t in grads)


@gpu
@pytest.mark.parametrize("T", [3, 5, 40, 300])
def test_a_bad_token_spoils_only_its_own_rows(T):
    h, f = 520, 1032
    x, W1, W3, W2, dy = make(T, h, f, torch.bfloat16, seed=5)
    saved, saved_bad = binding.ffn_saved(T, f, DEV), binding.ffn_saved(T, f, DEV)
    y = binding.ffn_forward(x, W1, W3, W2)
    binding.ffn_forward(x, W1, W3, W2, saved=saved)
    dx, *_ = binding.ffn_backward(dy, x, W1, W3, W2, saved)
    bad = x.clone()
    bad[T // 2, 3], bad[T - 1, 0] = float("nan"), float("inf")
    y_bad = binding.ffn_forward(bad, W1, W3, W2)
    binding.ffn_forward(bad, W1, W3, W2, saved=saved_bad)
    dx_bad, *_ = binding.ffn_backward(dy, bad, W1, W3, W2, saved_bad)
    keep = [t for t in range(T) if t not in (T // 2, T - 1)]
    assert torch.equal(y_bad[keep], y[keep]) and torch.equal(dx_bad[keep], dx[keep])
    assert y_bad[T // 2].isnan().all() and not y_bad[T - 1].isfinite().any()


@gpu
@pytest.mark.parametrize("T", [1, 2, 5, 37, 300])
def test_nothing_is_written_behind_the_outputs(T):
    h, f = 136, 264
    x, W1, W3, W2, dy = make(T, h, f, torch.bfloat16, seed=6)
    pad = 5

    def room(*shape, dtype=torch.bfloat16):
        whole = torch.full((shape[0] + pad, *shape[1:]), 5.0, dtype=dtype, device=DEV)
        return whole, whole[: shape[0]]

    wy, y = room(T, h)
    ws, saved = room(binding.load_library().moe_ffn_saved_bytes(T, f), dtype=torch.uint8)
    binding.ffn_forward(x, W1, W3, W2, y=y, saved=saved)
    rooms = [room(T, h), room(f, h), room(f, h), room(h, f)]
    binding.ffn_backward(dy, x, W1, W3, W2, saved, *[r[1] for r in rooms])
    for whole, part in [(wy, y), (ws, saved), *rooms]:
        assert bool((whole[part.shape[0]:] == 5).all()) and part.isfinite().all()
    # the smallest workspace is enough and nothing is written behind it
    lib = binding.load_library()
    n = lib.moe_ffn_forward_workspace(T, h, f)
    buf = torch.full((n + 512,), 9, dtype=torch.uint8, device=DEV)
    y2 = torch.empty_like(x)
    st = torch.cuda.current_stream().cuda_stream
    assert lib.moe_ffn_forward(x.data_ptr(), W1.data_ptr(), W3.data_ptr(), W2.data_ptr(), None, T, h, f, 0, y2.data_ptr(), None,
                               buf.data_ptr(), n, st) == 0
    check(y2, reference(x, W1, W3, W2)["y"], torch.bfloat16, "y")
    assert bool((buf[n:] == 9).all())
    n = lib.moe_ffn_backward_workspace(T, h, f)
    buf = torch.full((n + 512,), 9, dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(t) for t in (x, W1, W3, W2)]
    assert lib.moe_ffn_backward(dy.data_ptr(), x.data_ptr(), W1.data_ptr(), W3.data_ptr(), W2.data_ptr(), saved.data_ptr(), T, h, f,
                                0, *[o.data_ptr() for o in outs], buf.data_ptr(), n, st) == 0
    assert all(torch.equal(o, r[1]) for o, r in zip(outs, rooms)) and bool((buf[n:] == 9).all())


@gpu
def test_weights_are_read_anew_in_every_call():
    T, h, f = 20, 128, 448
    x, W1, W3, W2, _ = make(T, h, f, torch.bfloat16, seed=1)
    binding.ffn_forward(x, W1, W3, W2)
    other = make(T, h, f, torch.bfloat16, seed=2)
    for t, o in zip((x, W1, W3, W2), other):
        t.copy_(o)
    assert torch.equal(binding.ffn_forward(x, W1, W3, W2), binding.ffn_forward(*other[:4]))


@gpu
@pytest.mark.parametrize("T", [1, 100, 700])
def test_two_streams_at_once_and_graphs(T):
    h, f = 1024, 2048
    sets = [make(T, h, f, torch.bfloat16, seed=s) for s in (1, 2)]

    def step(s, stream=None):
        x, W1, W3, W2, dy = s
        saved = binding.ffn_saved(T, f, DEV)
        y = binding.ffn_forward(x, W1, W3, W2, saved=saved, stream=stream)
        return y, saved, *binding.ffn_backward(dy, x, W1, W3, W2, saved, stream=stream)

    want = [step(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            a = step(sets[0])
        with torch.cuda.stream(streams[1]):
            b = step(sets[1])
        got.append((a, b))
    torch.cuda.synchronize()
    for a, b in got:
        assert all(torch.equal(p, q) for p, q in zip(a, want[0])) and all(torch.equal(p, q) for p, q in zip(b, want[1]))
    side = torch.cuda.Stream()
    saved = binding.ffn_saved(T, f, DEV)
    side.wait_stream(torch.cuda.current_stream())
    y = binding.ffn_forward(*sets[0][:4], saved=saved, stream=side)
    alone = binding.ffn_forward(*sets[0][:4], stream=side)
    side.synchronize()
    assert torch.equal(y, want[0][0]) and torch.equal(alone, binding.ffn_forward(*sets[0][:4]))
    # two graphs, each with its own workspaces, replayed beside each other
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    for k in range(3):
        for s, st in zip(sets, streams):
            s[0].copy_(torch.roll(s[0], 1, 1))
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, o in zip(sets, outs):
            assert all(torch.equal(p, q) for p, q in zip(o, step(s)))


@gpu
def test_rows_beyond_32_bit_offsets():
    # 2^31 and more elements of a, g and u: the last tokens of a batch equal the definition
    T, h, f = 150100, 64, 14336
    assert T * f > 2 ** 31
    x, W1, W3, W2, dy = make(T, h, f, torch.bfloat16, seed=9)
    saved = binding.ffn_saved(T, f, DEV)
    y = binding.ffn_forward(x, W1, W3, W2, saved=saved)
    dx, dW1, dW3, dW2 = binding.ffn_backward(dy, x, W1, W3, W2, saved)
    last = slice(T - 100, T)
    want = reference(x[last].clone(), W1, W3, W2, dy[last].clone())
    check(y[last], want["y"], torch.bfloat16, "y")
    check(dx[last], want["dx"], torch.bfloat16, "dx")
    assert dW1.isfinite().all() and dW3.isfinite().all() and dW2.isfinite().all()


@gpu
def test_an_expired_wait_is_reported_once_and_leaves_the_operators_usable():
    T, h, f = 300, 520, 1032
    x, W1, W3, W2, _ = make(T, h, f, torch.bfloat16, seed=3)
    y = binding.ffn_forward(x, W1, W3, W2)
    lib = binding.load_library()
    assert lib.moe_test_operators_expiry(0, None) == -1 and lib.moe_test_operators_expiry(100001, None) == -1
    assert binding.operators_status(DEV) == 0
    assert lib.moe_test_operators_expiry(1000, torch.cuda.current_stream().cuda_stream) == 0
    assert binding.operators_status(DEV) == -5 and "expired" in binding.last_error()
    assert binding.operators_status() == 0
    assert torch.equal(binding.ffn_forward(x, W1, W3, W2), y) and binding.operators_status() == 0


@gpu
@pytest.mark.parametrize("T", [1, 50, 400])
def test_prenorm_block_beside_routed_experts(T):
    """The operators as they are used together: residual addition and norm, the dense block as a shared expert whose
    output the routed experts are added to, and back through block and norm."""
    h, f, E = synth.TINY["h"], synth.TINY["f"], synth.TINY["E"]
    L = synth.make_layer_weights(h, f, E, seed=0)
    layer = binding.MoeLayer(*[t.to(DEV) for t in (L.W_gate, L.W1, L.W3, L.W2)])
    x, W1, W3, W2, dy = make(T, h, f, torch.bfloat16, seed=4)
    r = make(T, h, 8, torch.bfloat16, seed=5)[0]
    gain = (1 + 0.1 * make(1, h, 8, torch.bfloat16, seed=6)[0][0].float()).bfloat16()
    rstd = torch.empty(T, device=DEV)
    saved = binding.ffn_saved(T, f, DEV)
    n, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
    y = binding.ffn_forward(n, W1, W3, W2, residual=s, saved=saved)
    both = layer.forward(n, 0.0, residual=y)
    routed = layer.forward(n, 0.0)
    # y + routed, each rounded once: off by the rounding of the routed part and of the sum
    want = y.double() + routed.double()
    assert bool(((both.double() - want).abs() <= 2.0 ** -8 * (want.abs() + routed.double().abs()) + 1e-6).all())
    check(y, (reference(n, W1, W3, W2)["y"][0] + s.double(), reference(n, W1, W3, W2)["y"][1] + 2.0 ** -8 * s.double().abs()),
          torch.bfloat16, "y")
    dn, dW1, dW3, dW2 = binding.ffn_backward(dy, n, W1, W3, W2, saved)
    want = reference(n, W1, W3, W2, dy)
    for k, v in (("dx", dn), ("dW1", dW1), ("dW3", dW3), ("dW2", dW2)):
        check(v, want[k], torch.bfloat16, k)
    dx, dgain = binding.add_rmsnorm_backward(dn, s, rstd, gain, d_s=dy)
    root = 1 / torch.sqrt((s.double() ** 2).mean(1, keepdim=True) + 1e-5)
    hat, up = s.double() * root, dn.double() * gain.double()
    want_x = dy.double() + root * (up - hat * (up * hat).mean(1, keepdim=True))
    assert bool(((dx.double() - want_x).abs() <= 2.0 ** -8 * want_x.abs() + 1e-4).all())
    layer.close()


FRESH_PROCESS = """
import torch
from paper_2402_14800_b200 import binding
T, h, f = %d, 256, 512
torch.manual_seed(0)
x, r, dy = (torch.randn((T, h), device="cuda").bfloat16() for _ in range(3))
W1, W3, W2 = (torch.randn(s, device="cuda").mul_(0.06).bfloat16() for s in ((f, h), (f, h), (h, f)))
gain = torch.ones(h, device="cuda").bfloat16()
rstd = torch.empty(T, device="cuda")
torch.cuda.synchronize()

def step():
    n, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
    q, c, _ = binding.add_rmsnorm_e4m3(x, r, gain)
    saved = binding.ffn_saved(T, f, x.device)
    y = binding.ffn_forward(n, W1, W3, W2, residual=s, saved=saved)
    y2 = binding.ffn_forward(n, W1, W3, W2)
    dn, *dW = binding.ffn_backward(dy, n, W1, W3, W2, saved)
    return n, s, q.float(), c, y, y2, dn, *dW, *binding.add_rmsnorm_backward(dn, s, rstd, gain, d_s=dy)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = step()
for _ in range(2):
    x.normal_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, step()))
print("replayed")
"""


@gpu
@pytest.mark.parametrize("T", [1, 5, 100, 300])
def test_the_first_call_of_a_process_may_be_captured(T):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FRESH_PROCESS % T], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "replayed" in r.stdout, r.stdout + r.stderr
