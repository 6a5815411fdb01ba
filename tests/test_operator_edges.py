"""Calls of the norm and feed-forward operators that the sizes of test_norm_ops.py and test_ffn_ops.py pass by."""
import ctypes

import pytest
import torch

from paper_2402_14800_b200 import binding, build

DEV = "cuda:0"
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load_library()


# ------------------------------------------------------------------------------- no device


@pytest.mark.parametrize("h,f", [(8, 8), (64, 8), (128, 448), (72, 136), (520, 264), (520, 1032), (256, 512), (512, 1032),
                                 (1024, 2048), (2040, 5464), (4096, 14336)])
def test_gradients_launch_deals_each_item_once_and_reads_ahead_only_for_an_item(lib, h, f):
    most = 4096
    items, deal = (ctypes.c_int * most)(), (ctypes.c_int * 3)()
    for T in (1, 3, 20, 31, 33, 50, 64, 100, 128, 200, 256, 300, 611, 1025, 2048, 8000):
        for pairs in (74, 66, 5, 1):
            assert lib.moe_test_ffn_deal(T, h, f, pairs, 0, items, most, deal) == 0
            total, seen = deal[0], []
            for pair in range(min(total, pairs)):
                assert lib.moe_test_ffn_deal(T, h, f, pairs, pair, items, most, deal) == 0
                n, ahead = deal[1], deal[2]
                mine = list(items[:n])
                assert n <= most and ahead == (mine[0] if mine else -1), (T, pairs, pair, mine, ahead)
                seen += mine
            assert sorted(seen) == list(range(total)), (T, pairs)
    assert lib.moe_test_ffn_deal(1, 8, 8, 74, 4, items, most, deal) == -1  # four items: the launch has four pairs


def test_norm_gradients_refuse_every_overlap_with_an_output(lib):
    """Each output against each other tensor, at the same address and in part; dx may only be d_s itself."""
    T, h, e = 64, 256, 2
    n, g, r, w = T * h * e, h * e, T * 4, lib.moe_add_rmsnorm_backward_workspace(64, 256)
    names = ("d_out", "d_s", "s", "rstd", "gain", "dx", "dgain", "workspace")
    size = dict(zip(names, (n, n, n, r, g, n, g, w)))
    at = {k: (i + 1) << 28 for i, k in enumerate(names)}

    def call(**moved):
        a = {k: ctypes.c_void_p({**at, **moved}[k]) for k in names}
        return lib.moe_add_rmsnorm_backward(a["d_out"], a["d_s"], a["s"], a["rstd"], a["gain"], T, h, 0, a["dx"], a["dgain"],
                                            a["workspace"], w, None)

    for out in ("dx", "dgain", "workspace"):
        for other in names:
            if other == out:
                continue
            for place in (at[other], at[other] + size[other] - 16, at[other] - size[out] + 16):
                if (out, other) == ("dx", "d_s") and place == at[other]:
                    continue
                assert call(**{out: place}) == -1 and "overlap" in binding.last_error(), (out, other, place - at[other])


@pytest.mark.parametrize("off", [1, 2, 3])
def test_norm_refuses_fp32_buffers_between_two_values(lib, off):
    p = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(8)]
    astray = ctypes.c_void_p(0x800000 + off)
    assert lib.moe_add_rmsnorm(p[0], p[1], p[2], 4, 64, 1e-5, 0, p[3], p[4], astray, None) == -1
    assert "aligned" in binding.last_error()
    assert lib.moe_add_rmsnorm_e4m3(p[0], p[1], p[2], 4, 64, 1e-5, 0, 0, p[3], astray, p[4], None) == -1
    assert "aligned" in binding.last_error()
    assert lib.moe_add_rmsnorm_backward(p[0], p[1], p[2], astray, p[3], 4, 64, 0, p[4], p[5], p[6], 1 << 20, None) == -1
    assert "aligned" in binding.last_error()


LARGEST = """
import ctypes
from paper_2402_14800_b200 import binding
lib = binding.load_library()
out = (ctypes.c_int * 6)()
for T in ((1 << 24) - 5, 1 << 24):
    for h, f in ((8, 1 << 20), (1 << 20, 8), (1 << 20, 1 << 20), (4096, 1 << 20)):
        for pairs in (74, 1):
            for launch in range(4):
                assert lib.moe_test_ffn_plan(launch, T, h, f, pairs, out) == 0
                R, n_tile, S, mt, nt, kb = list(out)
                M, unit = f if launch in (0, 2) else h, 2 if launch == 0 else 4
                assert 8 <= R <= 128 and 16 <= n_tile <= 256 and 1 <= S <= 16
                assert (mt - 1) * unit * R < M <= mt * unit * R and (nt - 1) * n_tile < T <= nt * n_tile
                assert mt * nt * S <= 1 << 29
        assert lib.moe_ffn_forward_workspace(T, h, f) >= 2 * T * f and lib.moe_ffn_backward_workspace(T, h, f) >= 4 * T * f
        assert lib.moe_ffn_saved_bytes(T, f) >= 10 * T * f
print("planned")
"""


def test_the_largest_sizes_have_plans(lib):
    """Sizes that pass the argument check but no memory: what asks for a workspace or a plan still gets an answer."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", LARGEST], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "planned" in r.stdout, (r.returncode, r.stdout + r.stderr)


@pytest.mark.parametrize("value,early", [(None, 1), ("0", 1), ("1", 0)])
def test_plain_stream_order_is_read_for_calls_without_a_handle(lib, value, early):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = {k: v for k, v in os.environ.items() if k != "MOE_NO_PDL"}
    if value is not None:
        env["MOE_NO_PDL"] = value
    code = "from paper_2402_14800_b200 import binding; print(binding.load_library().moe_test_early_launches())"
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == str(early), r.stdout + r.stderr


WITHOUT_CUDA = """
import torch
assert hasattr(torch._C, "_cuda_getCurrentRawStream")
del torch._C._cuda_getCurrentRawStream  # as in a torch built without CUDA
import paper_2402_14800_b200
from paper_2402_14800_b200 import binding
assert binding.load_library().moe_num_subsets(8, 6) == 28
try:
    binding.add_rmsnorm(torch.zeros(4, 64))
except binding.MoeError:
    print("refused")
"""


def test_binding_loads_where_torch_has_no_cuda(lib):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", WITHOUT_CUDA], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "refused" in r.stdout, r.stdout + r.stderr


# ------------------------------------------------------------------------------- on the device


def block_inputs(T, h, f, dt, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)

    return (normal(T, h), normal(f, h, std=1.28 / h ** 0.5), normal(f, h, std=1.28 / h ** 0.5), normal(h, f, std=1.28 / f ** 0.5),
            normal(T, h, std=0.1))


@gpu
@pytest.mark.parametrize("T", [40, 300])
def test_a_long_launch_in_front_does_not_count_against_the_waits(lib, T):
    """The kernels' waits give up after 4 s; a launch in front that lets them start at once may take longer."""
    h, f = 520, 1032
    x, W1, W3, W2, dy = block_inputs(T, h, f, torch.bfloat16, seed=2)

    def step():
        saved = binding.ffn_saved(T, f, DEV)
        y = binding.ffn_forward(x, W1, W3, W2, saved=saved)
        return y, *binding.ffn_backward(dy, x, W1, W3, W2, saved)

    want = step()
    assert binding.operators_status(DEV) == 0
    assert lib.moe_test_hold(0, None) == -1 and lib.moe_test_hold(6001, None) == -1
    assert lib.moe_test_hold(4600, torch.cuda.current_stream().cuda_stream) == 0
    got = step()
    assert binding.operators_status(DEV) == 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))


FAILED_QUESTION = """
import torch
from paper_2402_14800_b200 import binding
lib = binding.load_library()
x, gain = torch.randn((700, 1024), device="cuda").bfloat16(), torch.ones(1024, device="cuda").bfloat16()
rstd = torch.empty(700, device="cuda")

def forward():
    return binding.add_rmsnorm(x, x, gain, rstd=rstd)

def e4m3():
    return binding.add_rmsnorm_e4m3(x, x, gain)

def backward():
    return binding.add_rmsnorm_backward(x, x, torch.ones(700, device="cuda"), gain)

for call in (forward, e4m3, backward):
    assert lib.moe_test_fail_occupancy(1) == 0
    try:
        call()
        raise SystemExit("%s went on after a failed question" % call.__name__)
    except binding.MoeError as e:
        assert "unknown error" in str(e), e
    assert lib.moe_test_fail_occupancy(0) == 0
    call()
torch.cuda.synchronize()
print("asked again")
"""


@gpu
def test_a_failed_question_for_residency_is_an_error_and_is_asked_again():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FAILED_QUESTION], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "asked again" in r.stdout, r.stdout + r.stderr


@gpu
@pytest.mark.parametrize("h", [256, 1024, 2048, 4096, 8320, 16384])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_e4m3_of_products_beyond_fp32(h, dt):
    """s * gain overflows in the second group of 128 columns and underflows in the last: v = (s * gain) * rstd there is
    infinite and 0, the other groups are as they would be alone."""
    T = 5
    g = torch.Generator(DEV).manual_seed(h)
    s = (torch.randn((T, h), generator=g, device=DEV) * 1e15).to(dt)
    s[:, 130] = 2e15
    gain = (1 + 0.3 * torch.rand(h, generator=g, device=DEV)).to(dt)
    plain_q, plain_scales, _ = binding.add_rmsnorm_e4m3(s, None, gain, group=128)
    s[:, -128:] = (torch.randn((T, 128), generator=g, device=DEV) * 1e-20).to(dt)
    gain[128:256], gain[-128:] = 1e25, 1e-30
    if h == 256:  # the second group is the last
        s[:, 130], gain[128:256] = 2e15, 1e25
    p = s.float() * gain.float()  # infinite or 0 in fp32 too
    q, scales, _ = binding.add_rmsnorm_e4m3(s, None, gain, group=128)
    assert bool(p[:, 130].isinf().all()) and bool(scales[:, 1].isinf().all())
    part, inf = q[:, 128:256].float(), p[:, 128:256].isinf()
    assert bool(part[inf].isnan().all()) and not part[~inf].any()
    if h > 256:
        assert not p[:, -128:].any() and not q[:, -128:].float().any() and bool((scales[:, -1] == 2.0 ** -126).all())
    # rstd of the whole row is another one now, but q and the ratio of two scales do not depend on it
    keep = [i for i in range(h // 128) if i not in (1, h // 128 - 1)]
    U = 2.0 ** -24
    for i in keep:
        a, b = (t[:, 128 * i:128 * (i + 1)].float() for t in (q, plain_q))
        assert torch.equal(a, b)
    if len(keep) > 1:
        now, then = scales[:, keep].double(), plain_scales[:, keep].double()
        ratio = (now / now[:, :1]) / (then / then[:, :1])
        assert bool(((ratio - 1).abs() <= 16 * U).all())  # four scales of two roundings each, taken double
    # a scale a row: infinite, NaN where the product is, 0 elsewhere
    q, scales, _ = binding.add_rmsnorm_e4m3(s, None, gain)
    assert bool(scales.isinf().all()) and bool(q.float()[p.isinf()].isnan().all()) and not q.float()[~p.isinf()].any()
    # the norm in the tensors' type takes s * rstd first
    out, _ = binding.add_rmsnorm(s, None, gain)
    assert bool(out.isfinite().all())


@gpu
@pytest.mark.parametrize("T", [3, 50, 300])
def test_the_documented_backward_is_the_gradient_of_the_documented_forward(T):
    """The README's lines from the forward calls to the gradients, run as they stand, against the 64-bit gradient of their y.

    Tolerance, in the 2-norm: a rounding is off by at most half a step, 2^-8 of a value in bf16; behind an output stand no
    more than eight (n, a, dg, du, dn, what they are multiplied with being given, and the output itself; p and q
    are fp32), and products of random operands keep the relative size of independent errors."""
    import os
    import re

    from paper_2402_14800_b200 import synth
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as file:
        blocks = re.findall(r"(?:^ {6}.*\n)+", file.read(), re.M)
    code = [b for b in blocks if "binding.ffn_backward" in b]
    assert len(code) == 1 and sum("binding.add_rmsnorm(" in b for b in blocks) == 2
    h, f, E = synth.TINY["h"], synth.TINY["f"], synth.TINY["E"]
    L = synth.make_layer_weights(h, f, E, seed=0)
    layer = binding.MoeLayer(*[t.to(DEV) for t in (L.W_gate, L.W1, L.W3, L.W2)])
    x, W1, W3, W2, dy = block_inputs(T, h, f, torch.bfloat16, seed=4)
    residual = block_inputs(T, h, 8, torch.bfloat16, seed=5)[0]
    gain = (1 + 0.1 * block_inputs(1, h, 8, torch.bfloat16, seed=6)[0][0].float()).bfloat16()
    names = dict(torch=torch, binding=binding, layer=layer, beta=0.0, T=T, f=f, device=DEV, x=x, residual=residual, gain=gain,
                 W1=W1, W3=W3, W2=W2, dy=dy)
    exec("\n".join(line[6:] for line in code[0].splitlines()), names)
    s, gn, w1, w3, w2 = leaves = [t.double().requires_grad_() for t in (names["s"], gain, W1, W3, W2)]
    n = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-5) * gn
    g = n @ w1.T
    y = (g * torch.sigmoid(g) * (n @ w3.T)) @ w2.T + s
    y.backward(dy.double())
    for k, want in [("y", y.detach()), *zip(("dx", "dgain", "dW1", "dW3", "dW2"), (t.grad for t in leaves))]:
        off = float((names[k].double() - want).norm() / want.norm())
        assert off < 8 * 2.0 ** -8, (k, off)
    layer.close()


@gpu
def test_sums_over_tokens_beyond_32_bit_offsets():
    """The weights' gradients where a, dg, du and the saved values pass 2^31 elements: with dy zero but for the last tokens
    they are those tokens' alone, and a range that is dropped, doubled or read elsewhere would show."""
    from tests.test_ffn_ops import check, reference
    T, h, f = 150100, 64, 14336
    assert T * f > 2 ** 31
    x, W1, W3, W2, dy = block_inputs(T, h, f, torch.bfloat16, seed=9)
    last = slice(T - 100, T)
    dy[:T - 100] = 0
    saved = binding.ffn_saved(T, f, DEV)
    binding.ffn_forward(x, W1, W3, W2, saved=saved)
    _, *grads = binding.ffn_backward(dy, x, W1, W3, W2, saved)
    want = reference(x[last].clone(), W1, W3, W2, dy[last].clone())
    for k, v in zip(("dW1", "dW3", "dW2"), grads):
        check(v, want[k], torch.bfloat16, k)


@gpu
def test_gradient_of_the_gain_beyond_32_bit_offsets():
    # rows of zeros add nothing, whatever their d_out: the sum is that of the last three rows
    T, h = 33000, 65544
    assert T * h > 2 ** 31
    g = torch.Generator(DEV).manual_seed(4)
    s = torch.zeros((T, h), dtype=torch.bfloat16, device=DEV)
    s[-3:] = torch.randn((3, h), generator=g, device=DEV)
    d_out = torch.ones((T, h), dtype=torch.bfloat16, device=DEV)
    d_out[-3:] = torch.randn((3, h), generator=g, device=DEV)
    gain = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    rstd = torch.rsqrt(s.new_zeros(T, dtype=torch.float32) + 1e-5)
    rstd[-3:] = torch.rsqrt(s[-3:].double().square().mean(1) + 1e-5).float()
    _, dgain = binding.add_rmsnorm_backward(d_out, s, rstd, gain)
    terms = d_out[-3:].double() * s[-3:].double() * rstd[-3:].double()[:, None]
    # a term is two roundings of 2^-24, the sum of three in any order two more; dgain one of 2^-8
    tol = 2.0 ** -8 * 1.01 * terms.sum(0).abs() + 4 * 2.0 ** -24 * terms.abs().sum(0) + torch.finfo(torch.bfloat16).smallest_normal
    assert bool(((dgain.double() - terms.sum(0)).abs() <= tol).all())
