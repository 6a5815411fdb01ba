"""What the operators beside the MoE layer are timed on: the residual addition with its RMS norm
(forward, backward, 8-bit output) and the dense gated feed-forward block (forward, training step).

A case names an operator (``kind``), the element type, the number of tokens and the layer's sizes.
h 4096 with f 14336 is the configured Mixtral layer of ``paper_2402_14800_b200.synth``, h 128 with
f 448 the tiny one; the other sizes are generic.

    add_rmsnorm        s = x + r, held in the type;  out = s * rstd * gain,  rstd = 1 / sqrt(mean(s^2) + eps)
    ... backward       g = d_out * gain;  dx = d_s + rstd * (g - s * rstd * mean(g * s * rstd));
                       dgain = sum over tokens of d_out * s * rstd
    add_rmsnorm_e4m3   scale = max |v| / 448 over a row or over 128 columns of it, q = e4m3(v / scale), v = s * rstd * gain
    ffn                a = silu(x W1^T) * (x W3^T);  y = a W2^T
    ... backward       da = dy W2;  dg = da * u * silu'(g);  du = da * silu(g);
                       dW2 = dy^T a;  dW1 = dg^T x;  dW3 = du^T x;  dx = dg W1 + du W3
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E4M3_MAX = 448.0

MOST_NORM = 32768 * 4096            # elements of the largest norm
MOST_FFN = 8192 * 4096 * 14336      # tokens * h * f of the largest forward pass; a training step has three times its work
MOST_TRAIN = 2048 * 4096 * 14336


def listed():
    return [
        # one token of one sequence between two layers: launch latency is everything
        dict(name="norm_1", kind="norm", type="bf16", tokens=1, h=4096),
        # the largest prompt batch of the benchmark, one norm of it
        dict(name="norm_32768", kind="norm", type="bf16", tokens=32768, h=4096),
        # a training step's norm at an ordinary batch, forward and backward
        dict(name="norm_train_8192", kind="norm_train", type="bf16", tokens=8192, h=4096),
        # a ragged batch in full precision, rows that no vector load divides
        dict(name="norm_train_777_fp32", kind="norm_train", type="fp32", tokens=777, h=1001),
        # a decode batch whose normalised rows go on in 8 bits, one scale a token
        dict(name="norm_e4m3_128", kind="norm_e4m3", type="bf16", tokens=128, h=4096, group=0),
        # a prompt in 8 bits, one scale for each 128 columns of a token
        dict(name="norm_e4m3_8000_fp16", kind="norm_e4m3", type="fp16", tokens=8000, h=2048, group=128),
        # batch-1 decoding of a dense block at the Mixtral sizes: nothing but weight streaming
        dict(name="ffn_1", kind="ffn", type="bf16", tokens=1, h=4096, f=14336),
        # a full decode batch
        dict(name="ffn_128", kind="ffn", type="bf16", tokens=128, h=4096, f=14336),
        # a chunk of a prompt, an odd number of tokens on odd sizes, in fp16
        dict(name="ffn_611_fp16", kind="ffn", type="fp16", tokens=611, h=2040, f=5464),
        # prompt processing
        dict(name="ffn_8192", kind="ffn", type="bf16", tokens=8192, h=4096, f=14336),
        # fine-tuning the tiny layer on a ragged batch
        dict(name="ffn_train_100", kind="ffn_train", type="bf16", tokens=100, h=128, f=448),
        # a fine-tuning step of one sequence of 2048 tokens
        dict(name="ffn_train_2048", kind="ffn_train", type="bf16", tokens=2048, h=4096, f=14336),
    ]


def _size(rng, lo, hi, step=1):
    """Spread over the logarithm of lo .. hi, a multiple of `step`."""
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random()) // step * step))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm_e4m3", "ffn", "ffn", "ffn_train", "ffn_train"])
    if kind.startswith("norm"):
        h = _size(rng, 64, 8192)
        group = 0
        if kind == "norm_e4m3" and rng.random() < 0.5:
            h, group = _size(rng, 128, 8192, 128), 128
        elif rng.random() < 0.6:
            h = h // 8 * 8
        tokens = _size(rng, 1, min(32768, MOST_NORM // h))
        case = dict(kind=kind, type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), tokens=tokens, h=h)
        if kind == "norm_e4m3":
            case["group"] = group
        return case
    h, f = _size(rng, 64, 4096, 8), _size(rng, 64, 14336, 8)
    most = MOST_FFN if kind == "ffn" else MOST_TRAIN
    tokens = _size(rng, 1, min(8192, most // (h * f)))
    return dict(kind=kind, type=rng.choice(["bf16", "bf16", "fp16"]), tokens=tokens, h=h, f=f)


# ------------------------------------------------------------------------------------ inputs


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(int(seed))
    T, h, dt = case["tokens"], case["h"], TYPES[case["type"]]

    def normal(*shape, std=1.0, to=dt):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(to)

    state = dict(case=dict(case))
    if case["kind"].startswith("norm"):
        # hidden states have a few channels of large values
        wide = torch.ones(h, device=DEV)
        wide[torch.randperm(h, generator=g, device=DEV)[: max(1, round(0.01 * h))]] = 20.0
        state.update(x=normal(T, h, std=0.5), r=(torch.randn((T, h), generator=g, device=DEV) * wide).to(dt),
                     gain=(1.0 + 0.2 * torch.randn(h, generator=g, device=DEV)).to(dt))
        if case["kind"] == "norm_train":
            state.update(d_out=normal(T, h), d_s=normal(T, h))
        return state
    f = case["f"]
    # weights whose projections of unit inputs have the spread of the Mixtral layer's (0.02 * sqrt(4096))
    state.update(x=normal(T, h), W1=normal(f, h, std=1.28 / h ** 0.5), W3=normal(f, h, std=1.28 / h ** 0.5),
                 W2=normal(h, f, std=1.28 / f ** 0.5))
    if case["kind"] == "ffn_train":
        state.update(d_y=normal(T, h, std=0.1))
    return state


# ------------------------------------------------------------------------------------ one pass


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_norm(s):
    from paper_2402_14800_b200 import binding
    out, total = binding.add_rmsnorm(s["x"], s["r"], s["gain"], EPS)
    return dict(out=out, s=total)


def _own_norm_train(s):
    from paper_2402_14800_b200 import binding
    rstd = torch.empty(s["x"].shape[0], dtype=torch.float32, device=s["x"].device)
    out, total = binding.add_rmsnorm(s["x"], s["r"], s["gain"], EPS, rstd=rstd)
    dx, dgain = binding.add_rmsnorm_backward(s["d_out"], total, rstd, s["gain"], d_s=s["d_s"])
    return dict(out=out, s=total, dx=dx, dgain=dgain)


def _own_norm_e4m3(s):
    from paper_2402_14800_b200 import binding
    q, scales, total = binding.add_rmsnorm_e4m3(s["x"], s["r"], s["gain"], EPS, group=s["case"]["group"])
    return dict(q=q, scales=scales, s=total)


def _own_ffn(s):
    from paper_2402_14800_b200 import binding
    return binding.ffn_forward(s["x"], s["W1"], s["W3"], s["W2"])


def _own_ffn_train(s):
    from paper_2402_14800_b200 import binding
    saved = binding.ffn_saved(s["x"].shape[0], s["W1"].shape[0], s["x"].device)
    y = binding.ffn_forward(s["x"], s["W1"], s["W3"], s["W2"], saved=saved)
    dx, dW1, dW3, dW2 = binding.ffn_backward(s["d_y"], s["x"], s["W1"], s["W3"], s["W2"], saved)
    return dict(y=y, dx=dx, dW1=dW1, dW3=dW3, dW2=dW2)


def _plain_sum(s):
    # the sum is what the residual stream holds, in its type; the norm is of what is held
    total = (s["x"].float() + s["r"].float()).to(s["x"].dtype)
    v = total.float()
    rstd = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return total, v, rstd


def _plain_norm(s):
    total, v, rstd = _plain_sum(s)
    return dict(out=(v * rstd * s["gain"].float()).to(total.dtype), s=total)


def _plain_norm_train(s):
    total, v, rstd = _plain_sum(s)
    hat = v * rstd
    d_out = s["d_out"].float()
    g = d_out * s["gain"].float()
    dx = s["d_s"].float() + rstd * (g - hat * (g * hat).mean(1, keepdim=True))
    return dict(out=(hat * s["gain"].float()).to(total.dtype), s=total, dx=dx.to(total.dtype),
                dgain=(d_out * hat).sum(0).to(total.dtype))


def _plain_norm_e4m3(s):
    total, v, rstd = _plain_sum(s)
    T, h = v.shape
    n = (v * rstd * s["gain"].float()).view(T, -1, s["case"]["group"] or h)
    scales = n.abs().amax(2) / E4M3_MAX
    q = (n / scales[:, :, None]).view(T, h).to(torch.float8_e4m3fn)
    return dict(q=q, scales=scales, s=total)


def _plain_ffn(s):
    x = s["x"].float()
    g, u = x @ s["W1"].float().T, x @ s["W3"].float().T
    return ((g * torch.sigmoid(g) * u) @ s["W2"].float().T).to(s["x"].dtype)


def _plain_ffn_train(s):
    dt = s["x"].dtype
    x, d_y = s["x"].float(), s["d_y"].float()
    W1, W3, W2 = s["W1"].float(), s["W3"].float(), s["W2"].float()
    g, u = x @ W1.T, x @ W3.T
    sig = torch.sigmoid(g)
    act = g * sig
    a = act * u
    y = a @ W2.T
    da = d_y @ W2
    dg = da * u * (sig * (1.0 + g * (1.0 - sig)))
    du = da * act
    return dict(y=y.to(dt), dx=(dg @ W1 + du @ W3).to(dt), dW1=(dg.T @ x).to(dt), dW3=(du.T @ x).to(dt),
                dW2=(d_y.T @ a).to(dt))


_OWN = dict(norm=_own_norm, norm_train=_own_norm_train, norm_e4m3=_own_norm_e4m3, ffn=_own_ffn, ffn_train=_own_ffn_train)
_PLAIN = dict(norm=_plain_norm, norm_train=_plain_norm_train, norm_e4m3=_plain_norm_e4m3, ffn=_plain_ffn,
              ffn_train=_plain_ffn_train)


# ------------------------------------------------------------------------------------ floors


def work(case):
    T, h, e = case["tokens"], case["h"], 4 if case["type"] == "fp32" else 2
    kind = case["kind"]
    if kind == "norm":      # x, r, gain in; out, s out
        return dict(bytes=(4 * T * h + h) * e, flops=5 * T * h)
    if kind == "norm_train":  # and d_out, d_s in; dx, dgain out; s and rstd are read again by the backward pass
        return dict(bytes=(8 * T * h + 3 * h) * e + 8 * T, flops=17 * T * h)
    if kind == "norm_e4m3":
        return dict(bytes=(3 * T * h + h) * e + T * h + 4 * T * (h // case["group"] if case["group"] else 1), flops=7 * T * h)
    f = case["f"]
    if kind == "ffn":       # three weight matrices and x in, y out
        return dict(bytes=(3 * h * f + 2 * T * h) * e, flops=6 * T * h * f)
    # weights read and their gradients written once; x, d_y in, y, dx out
    return dict(bytes=(6 * h * f + 4 * T * h) * e, flops=18 * T * h * f)


# ------------------------------------------------------------------------------------ the definition in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        held = (s["x"].double() + s["r"].double()).to(s["x"].dtype)  # what the residual stream holds
        t = held.double()
        root = t.square().sum(1).div(t.shape[1]).add(EPS).sqrt()
        hat = t / root[:, None]
        gain = s["gain"].double()
        out = hat * gain
        if kind == "norm":
            return dict(out=out, s=t)
        if kind == "norm_e4m3":
            parts = out.reshape(t.shape[0], -1, case["group"] or t.shape[1])
            scales = parts.abs().max(2).values / 448
            # nearest e4m3 value, ties to even: 3 bits behind the leading one, the smallest exponent is -6
            w = (parts / scales.unsqueeze(2)).reshape(out.shape)
            step = torch.exp2(torch.floor(torch.log2(w.abs().clamp_min(2.0 ** -6))) - 3)
            return dict(q=torch.round(w / step) * step, scales=scales, s=t)
        up = s["d_out"].double()
        inner = torch.einsum("th,th->t", up * gain, hat) / t.shape[1]
        dx = s["d_s"].double() + (up * gain - hat * inner[:, None]) / root[:, None]
        return dict(out=out, s=t, dx=dx, dgain=torch.einsum("th,th->h", up, hat))
    x, W1, W3, W2 = (s[k].double() for k in ("x", "W1", "W3", "W2"))
    gate, up = torch.mm(x, W1.t()), torch.mm(x, W3.t())
    swish = gate / (1 + torch.exp(-gate))
    y = torch.mm(swish * up, W2.t())
    if kind == "ffn":
        return y
    dy = s["d_y"].double()
    back = torch.mm(dy, W2)
    slope = 1 / (1 + torch.exp(-gate))
    d_gate = back * up * (slope + swish * (1 - slope))
    d_up = back * swish
    return dict(y=y, dx=torch.mm(d_gate, W1) + torch.mm(d_up, W3), dW1=torch.mm(d_gate.t(), x),
                dW3=torch.mm(d_up.t(), x), dW2=torch.mm(dy.t(), swish * up))
