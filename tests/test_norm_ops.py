"""Residual addition with RMS norm (forward, backward, e4m3 output) against the definition in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32.  A row's sum of squares is a chain of at most CHAIN additions of
non-negative terms per thread, shuffles and partial sums included, so its relative error is below CHAIN * u,
that of 1/sqrt half of it, and a handful of roundings follow: every fp32 value before the store is within
(CHAIN + 8) * u of its own size, or of the sum of its terms' sizes where it is a difference.  The store adds half
a step of the type, finfo.eps / 2; e4m3 adds 2^-4 of the value, or half of its smallest step, 2^-10, times the scale."""
import ctypes

import pytest
import torch

from paper_2402_14800_b200 import binding, build

U = 2.0 ** -24
CHAIN = 96
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load_library()


# ------------------------------------------------------------------------------- refusals, no device


def test_refuses_bad_arguments_without_a_device(lib):
    p = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(8)]
    odd = ctypes.c_void_p(0x100008)

    def fwd(x=p[0], r=p[1], g=p[2], T=4, h=64, eps=1e-5, dt=0, out=p[3], s=p[4], rstd=None):
        return lib.moe_add_rmsnorm(x, r, g, T, h, eps, dt, out, s, rstd, None)

    assert fwd(x=None) == -1 and "NULL" in binding.last_error()
    assert fwd(out=None) == -1
    assert fwd(s=None) == -1 and "go together" in binding.last_error()
    assert fwd(r=None) == -1 and "go together" in binding.last_error()
    for k in ("x", "r", "g", "out", "s"):
        assert fwd(**{k: odd}) == -1 and "aligned" in binding.last_error(), k
    assert fwd(dt=3) == -1 and "dtype" in binding.last_error()
    assert fwd(T=-1) == -1 and fwd(T=(1 << 24) + 1) == -1
    assert fwd(h=0) == -2 and fwd(h=(1 << 20) + 1) == -2
    assert fwd(eps=-1.0) == -1 and fwd(eps=float("nan")) == -1
    assert fwd(out=ctypes.c_void_p(0x100000 + 128)) == -1 and "overlap" in binding.last_error()
    assert fwd(s=ctypes.c_void_p(0x100000 + 128)) == -1 and "overlap" in binding.last_error()
    assert fwd(s=p[3]) == -1 and "overlap" in binding.last_error()
    assert fwd(g=p[3]) == -1 and "gain" in binding.last_error()
    for k in range(5):
        assert fwd(rstd=p[k]) == -1 and "rstd" in binding.last_error()
    assert fwd(T=0) == 0 and fwd(T=0, x=None, out=None) == 0

    def q8(group=0, h=256, q=p[3], scales=p[5], s=p[4]):
        return lib.moe_add_rmsnorm_e4m3(p[0], p[1], p[2], 4, h, 1e-5, 0, group, q, scales, s, None)

    assert q8(group=64) == -1 and q8(group=-1) == -1 and q8(group=128, h=200) == -2
    assert q8(scales=None) == -1 and "scales" in binding.last_error()
    assert q8(scales=p[3]) == -1 and q8(scales=p[0]) == -1 and "scales overlaps" in binding.last_error()
    assert q8(q=p[0]) == -1 and "overlap" in binding.last_error()  # no 8-bit output in place

    def bwd(d=p[0], e=p[1], s=p[2], rstd=p[3], g=p[4], T=4, h=64, dt=0, dx=p[5], dg=p[6], ws=p[7], n=1 << 30):
        return lib.moe_add_rmsnorm_backward(d, e, s, rstd, g, T, h, dt, dx, dg, ws, n, None)

    for k in ("d", "s", "rstd", "dx"):
        assert bwd(**{k: None}) == -1 and "NULL" in binding.last_error(), k
    for k in ("d", "e", "s", "g", "dx", "dg", "ws"):
        assert bwd(**{k: odd}) == -1 and "aligned" in binding.last_error(), k
    assert bwd(ws=None) == -1 and "workspace" in binding.last_error()
    assert bwd(n=64 * 4 - 1) == -1 and "workspace" in binding.last_error()
    assert bwd(dx=p[0]) == -1 and bwd(dx=p[2]) == -1 and bwd(dx=ctypes.c_void_p(0x200000 + 128)) == -1
    assert bwd(dg=p[4]) == -1 and bwd(dg=p[5]) == -1
    for k in range(7):
        assert bwd(ws=p[k]) == -1 and "workspace overlaps" in binding.last_error()
    for k in ("dx", "dg"):
        assert bwd(**{k: p[3]}) == -1 and "rstd" in binding.last_error()
    assert bwd(dt=9) == -1 and bwd(h=0) == -2 and bwd(T=-2) == -1
    assert bwd(T=0, dg=None) == 0
    assert lib.moe_add_rmsnorm_backward_workspace(0, 64) == 0 and lib.moe_add_rmsnorm_backward_workspace(4, 0) == 0


def test_binding_refuses_host_tensors(lib):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    for call in (lambda: binding.add_rmsnorm(x), lambda: binding.add_rmsnorm_e4m3(x),
                 lambda: binding.add_rmsnorm_backward(x, x, torch.ones(4))):
        with pytest.raises(binding.MoeError):
            call()


@gpu
def test_binding_refuses_wrong_tensors():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    g = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    rstd = torch.ones(4, device=DEV)
    bad = [lambda: binding.add_rmsnorm(x[:, ::2]), lambda: binding.add_rmsnorm(x.T),
           lambda: binding.add_rmsnorm(x, x[:3]), lambda: binding.add_rmsnorm(x, x.float()),
           lambda: binding.add_rmsnorm(x, x, g.float()), lambda: binding.add_rmsnorm(x, x, g[:63]),
           lambda: binding.add_rmsnorm(x.double()), lambda: binding.add_rmsnorm(x, s=torch.empty_like(x)),
           lambda: binding.add_rmsnorm(x, x, rstd=rstd.double()), lambda: binding.add_rmsnorm(x, x.cpu()),
           lambda: binding.add_rmsnorm(x.view(-1)[4:4 + 192].view(3, 64)),  # not 16-byte aligned
           lambda: binding.add_rmsnorm_e4m3(x, group=32), lambda: binding.add_rmsnorm_e4m3(x, group=128),
           lambda: binding.add_rmsnorm_e4m3(x, scales=rstd),
           lambda: binding.add_rmsnorm_backward(x, x, rstd[:2]), lambda: binding.add_rmsnorm_backward(x, x, rstd, d_s=x[:2]),
           lambda: binding.add_rmsnorm_backward(x, x.clone(), rstd, dx=x)]
    for call in bad:
        with pytest.raises(binding.MoeError):
            call()


# ------------------------------------------------------------------------------- against 64 bits


def make(T, h, dt, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn((T, h), generator=g, device=DEV).to(dt)
    r = (torch.randn((T, h), generator=g, device=DEV) * 3).to(dt)
    gain = (1 + 0.3 * torch.randn(h, generator=g, device=DEV)).to(dt)
    return x, r, gain, g


def norm64(s, gain, eps):
    s = s.double()
    rstd = 1 / torch.sqrt((s * s).mean(1) + eps)
    v = s * rstd[:, None] * (gain.double() if gain is not None else 1.0)
    return v, rstd


def half(dt):
    return torch.finfo(dt).eps / 2


def assert_within(got, want, tol):
    off = (got.double() - want).abs() - tol
    assert bool((off <= 0).all()), "worst excess %.3g at %d" % (float(off.max()), int(off.argmax()))


SHAPES = [(1, 1), (3, 7), (1, 8), (5, 64), (9, 120), (77, 256), (2, 1000), (33, 1001), (64, 1024), (12, 2048), (7, 2056),
          (1, 4096), (130, 4096), (5, 4104), (4, 8191), (3, 8192), (3, 8200), (2, 9001), (2, 20000), (20000, 64), (1500, 2048)]


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,h", SHAPES)
def test_forward(T, h, dt):
    dt = TYPES[dt]
    x, r, gain, _ = make(T, h, dt, seed=T + h)
    rstd = torch.full((T,), -1.0, device=DEV)
    out, s = binding.add_rmsnorm(x, r, gain, 1e-5, rstd=rstd)
    assert torch.equal(s, (x.float() + r.float()).to(dt))
    v, want = norm64(s, gain, 1e-5)
    assert_within(rstd, want, (CHAIN + 8) * U * want)
    assert_within(out, v, (half(dt) * 1.01 + (CHAIN + 8) * U) * v.abs() + torch.finfo(dt).smallest_normal * half(dt) * 2)
    # without a residual and without a gain, in place of neither: s is x
    o2, s2 = binding.add_rmsnorm(s, None, gain)
    assert s2 is s and torch.equal(o2, out)
    o3, _ = binding.add_rmsnorm(x, r)
    v3, _ = norm64(s, None, 1e-5)
    assert_within(o3, v3, (half(dt) * 1.01 + (CHAIN + 8) * U) * v3.abs() + torch.finfo(dt).smallest_normal * half(dt) * 2)


@gpu
@pytest.mark.parametrize("T,h", [(9, 120), (33, 1001), (130, 4096), (3, 8200)])
def test_forward_in_place(T, h):
    x, r, gain, _ = make(T, h, torch.bfloat16, seed=5)
    out, s = binding.add_rmsnorm(x, r, gain)
    for o, t in (("x", "r"), ("r", "x"), (None, "x"), ("x", None)):
        a, b = x.clone(), r.clone()
        named = {"x": a, "r": b, None: None}
        o1, s1 = binding.add_rmsnorm(a, b, gain, out=named[o], s=named[t])
        assert torch.equal(o1, out) and torch.equal(s1, s), (o, t)
    a = s.clone()
    o1, _ = binding.add_rmsnorm(a, None, gain, out=a)
    assert torch.equal(o1, out)


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,h,group", [(T, h, 0) for T, h in SHAPES] + [(1, 128, 128), (5, 256, 128), (70, 1024, 128),
                                                                       (9, 2176, 128), (130, 4096, 128), (3, 8320, 128),
                                                                       (2, 16384, 128), (12000, 128, 128)])
def test_e4m3(T, h, group, dt):
    dt = TYPES[dt]
    x, r, gain, _ = make(T, h, dt, seed=T + 3 * h)
    q, scales, s = binding.add_rmsnorm_e4m3(x, r, gain, 1e-5, group=group)
    assert torch.equal(s, (x.float() + r.float()).to(dt))
    v, _ = norm64(s, gain, 1e-5)
    parts = v.view(T, -1, group or h)
    want = parts.abs().amax(2) / 448
    assert scales.shape == want.shape
    assert_within(scales, want, (CHAIN + 12) * U * want)
    sc = scales.double().repeat_interleave(group or h, 1)
    got = q.float().double() * sc
    assert_within(got, v, (2.0 ** -4 + (CHAIN + 16) * U) * v.abs() + 2.0 ** -10 * 1.001 * sc)
    # the largest value of a group is 448, up to the sign
    assert bool((q.float().view(T, -1, group or h).abs().amax(2) == 448).all())
    q2, scales2, _ = binding.add_rmsnorm_e4m3(s, None, gain, 1e-5, group=group)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scales2, scales)


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,h", SHAPES)
@pytest.mark.parametrize("gained,along", [(True, True), (False, True), (True, False)])
def test_backward(T, h, dt, gained, along):
    dt = TYPES[dt]
    x, r, gain, g = make(T, h, dt, seed=2 * T + h)
    d_out = torch.randn((T, h), generator=g, device=DEV).to(dt)
    d_s = torch.randn((T, h), generator=g, device=DEV).to(dt) if along else None
    gain = gain if gained else None
    rstd = torch.empty(T, device=DEV)
    _, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
    dx, dgain = binding.add_rmsnorm_backward(d_out, s, rstd, gain, d_s=d_s)
    _, root = norm64(s, None, 1e-5)
    hat = s.double() * root[:, None]
    up = d_out.double() * (gain.double() if gained else 1.0)
    extra = d_s.double() if along else torch.zeros_like(hat)
    want = extra + root[:, None] * (up - hat * (up * hat).mean(1, keepdim=True))
    size = extra.abs() + root[:, None] * (up.abs() + hat.abs() * (up * hat).abs().mean(1, keepdim=True))
    tiny = torch.finfo(dt).smallest_normal * half(dt) * 2
    assert_within(dx, want, half(dt) * 1.01 * want.abs() + 2 * (CHAIN + 8) * U * size + tiny)
    if not gained:
        assert dgain is None
        return
    terms = d_out.double() * hat
    assert_within(dgain, terms.sum(0), half(dt) * 1.01 * terms.sum(0).abs() + (T + 2 * CHAIN) * U * terms.abs().sum(0) + tiny)
    again = binding.add_rmsnorm_backward(d_out, s, rstd, gain, d_s=d_s)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)  # a fixed order of the sums
    if along:  # d_s may become dx
        mine = d_s.clone()
        assert torch.equal(binding.add_rmsnorm_backward(d_out, s, rstd, gain, d_s=mine, dx=mine)[0], dx)


@gpu
def test_backward_is_the_slope_of_forward():
    # central differences of L = <d_out, out> + <d_s, s> in fp32; L is smooth, the step's error is O(step^2) and the
    # rounding of L about 64 * 37 * 2^-24 / step
    T, h, step = 5, 37, 2.0 ** -6
    x, r, gain, g = make(T, h, torch.float32, seed=1)
    d_out, d_s = (t.clone() for t in torch.randn((2, T, h), generator=g, device=DEV))  # each aligned by itself
    rstd = torch.empty(T, device=DEV)
    _, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
    dx, dgain = binding.add_rmsnorm_backward(d_out, s, rstd, gain, d_s=d_s)

    def loss(x, gain):
        out, s = binding.add_rmsnorm(x, r, gain)
        return float((out.double() * d_out.double()).sum() + (s.double() * d_s.double()).sum())

    for t, c in ((0, 0), (2, 17), (4, 36)):
        e = torch.zeros_like(x)
        e[t, c] = step
        slope = (loss(x + e, gain) - loss(x - e, gain)) / (2 * step)
        assert abs(slope - float(dx[t, c])) < 2e-3 * max(1.0, abs(slope)), (t, c, slope, float(dx[t, c]))
    for c in (0, 20, 36):
        e = torch.zeros_like(gain)
        e[c] = step
        slope = (loss(x, gain + e) - loss(x, gain - e)) / (2 * step)
        assert abs(slope - float(dgain[c])) < 2e-3 * max(1.0, abs(slope))


# ------------------------------------------------------------------------------- edges


@gpu
def test_no_rows():
    x = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    gain = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    out, s = binding.add_rmsnorm(x, x, gain)
    assert out.shape == (0, 64)
    q, scales, _ = binding.add_rmsnorm_e4m3(x, x, gain)
    assert q.shape == (0, 64) and scales.shape == (0, 1)
    dgain = torch.full((64,), 7.0, dtype=torch.bfloat16, device=DEV)
    dx, dgain = binding.add_rmsnorm_backward(x, x, torch.empty(0, device=DEV), gain, dgain=dgain)
    assert dx.shape == (0, 64) and not dgain.any()  # a sum of nothing, written all the same


@gpu
@pytest.mark.parametrize("h", [64, 1001, 4096, 8200])
def test_zeros_infinities_and_nan_stay_in_their_rows(h):
    x, r, gain, _ = make(6, h, torch.bfloat16, seed=3)
    x[1] = 0
    r[1] = 0
    x[2, 5] = float("nan")
    x[4, 0] = float("inf")
    out, s = binding.add_rmsnorm(x, r, gain)
    q, scales, _ = binding.add_rmsnorm_e4m3(x, r, gain)
    clean_x, clean_r = x.clone(), r.clone()
    clean_x[2], clean_x[4] = 1, 1
    ref, _ = binding.add_rmsnorm(clean_x, clean_r, gain)
    rq, rs, _ = binding.add_rmsnorm_e4m3(clean_x, clean_r, gain)
    for t in (0, 3, 5):
        assert torch.equal(out[t], ref[t]) and torch.equal(q[t].float(), rq[t].float()) and torch.equal(scales[t], rs[t])
    assert not out[1].any() and not q[1].float().any() and float(scales[1]) == 2.0 ** -126
    assert out[2].isnan().all() and q[2].float().isnan().all() and float(scales[2]) == 2.0 ** -126
    # rstd = 0: the infinity itself is NaN, the others 0
    assert out[4, 0].isnan() and not out[4, 1:].any() and q[4, 0].float().isnan() and not q[4, 1:].float().any()


@gpu
def test_rows_behind_the_last_are_left_alone():
    T, h = 37, 4096
    x, r, gain, _ = make(T, h, torch.bfloat16, seed=8)
    big = [torch.full((T + 3, h), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    rstd = torch.full((T + 3,), 5.0, device=DEV)
    out, s = binding.add_rmsnorm(x, r, gain, out=big[0][:T], s=big[1][:T], rstd=rstd[:T])
    assert all(bool((b[T:] == 5).all()) for b in (*big, rstd))
    dx = torch.full((T + 3, h), 5.0, dtype=torch.bfloat16, device=DEV)
    binding.add_rmsnorm_backward(x, s, rstd[:T], gain, dx=dx[:T])
    assert bool((dx[T:] == 5).all())


@gpu
def test_rows_beyond_32_bit_offsets():
    # 2^31 elements and more: the last rows of a tensor of 4.3 GB equal the same rows alone
    T, h = 33000, 65544
    assert T * h > 2 ** 31
    x = torch.zeros((T, h), dtype=torch.bfloat16, device=DEV)
    tail, _, gain, g = make(3, h, torch.bfloat16, seed=4)
    x[-3:] = tail
    rstd = torch.empty(T, device=DEV)
    out, _ = binding.add_rmsnorm(x, None, gain, rstd=rstd)
    want, _ = binding.add_rmsnorm(tail, None, gain)
    assert torch.equal(out[-3:], want) and not out[-4].any()
    dx, dgain = binding.add_rmsnorm_backward(x, x.clone(), rstd, gain, dx=out)
    dw, _ = binding.add_rmsnorm_backward(tail, tail.clone(), rstd[-3:].clone(), gain)
    assert torch.equal(dx[-3:], dw)


@gpu
def test_on_another_stream_and_in_a_graph():
    T, h = 300, 4096
    x, r, gain, g = make(T, h, torch.bfloat16, seed=6)
    d_out = torch.randn((T, h), generator=g, device=DEV).to(torch.bfloat16)
    rstd = torch.empty(T, device=DEV)
    out, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
    dx, dgain = binding.add_rmsnorm_backward(d_out, s, rstd, gain)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rstd2 = torch.zeros(T, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    o2, s2 = binding.add_rmsnorm(x, r, gain, rstd=rstd2, stream=side)
    dx2, dg2 = binding.add_rmsnorm_backward(d_out, s2, rstd2, gain, stream=side)
    side.synchronize()
    assert torch.equal(o2, out) and torch.equal(dx2, dx) and torch.equal(dg2, dgain)
    graph = torch.cuda.CUDAGraph()
    rstd3 = torch.zeros(T, device=DEV)
    with torch.cuda.graph(graph):
        o3, s3 = binding.add_rmsnorm(x, r, gain, rstd=rstd3)
        q3, c3, _ = binding.add_rmsnorm_e4m3(x, r, gain)
        dx3, dg3 = binding.add_rmsnorm_backward(d_out, s3, rstd3, gain)
    for k in range(3):
        x.copy_(torch.randn((T, h), generator=g, device=DEV))
        graph.replay()
        out, s = binding.add_rmsnorm(x, r, gain, rstd=rstd)
        q, c, _ = binding.add_rmsnorm_e4m3(x, r, gain)
        dx, dgain = binding.add_rmsnorm_backward(d_out, s, rstd, gain)
        assert torch.equal(o3, out) and torch.equal(dx3, dx) and torch.equal(dg3, dgain)
        assert torch.equal(q3.float(), q.float()) and torch.equal(c3, c)


@gpu
def test_unit_gain_without_addition_is_the_stack_norm():
    x, _, _, _ = make(50, 4096, torch.bfloat16, seed=9)
    out, _ = binding.add_rmsnorm(x)
    ref = binding.rmsnorm(x)
    # the two add up in different orders: rstd differs in its last bits, an output by one step at most
    assert bool(((out.float() - ref.float()).abs() <= torch.finfo(torch.bfloat16).eps * ref.float().abs()).all())
