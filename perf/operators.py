"""The operators of a transformer block's training step as cases that can be timed and compared.

A quantised transformer is fitted block by block on calibration rows before its outputs are corrected.  The block's
operators are layer norm, the product with bias, activation and residual in its epilogue, their gradients, and the
checkpoints in 8 bits that their backward passes read.  A case is one pass through one of them:

``norm``        layer norm forward: the rows, their means and reciprocal deviations
``norm_step``   layer norm forward with a checkpoint of its input, then the backward pass from that checkpoint; the
                gradient that arrives over the residual connection is added to the input's
``linear``      y = act(x W^T + b) + residual; ``pack``: also the pre-activation's checkpoint, returned as the values it
                stands for
``linear_grad`` the gradients of a product whose input is the activation of checkpointed rows (the second product of a
                block): the gradient of those rows, of the weight and of the bias
``checkpoint``  rows to 8 bits and back

Row counts and lengths are those of ``paper_2509_26277_amd/workloads.py`` (65536 calibration rows, 1000 and 1001
channels, 2048 bfloat16 channels, 256 .. 512 feature channels) or powers of two; the inner length of a block is four
times the outer one.
"""
import math

import torch

own = False

GROUP = 128  # channels that share a scale in a checkpoint
EPS = 1e-5


def listed():
    return [
        # one row at serving time: nothing but latency
        dict(name="norm_token", kind="norm", dtype="bf16", M=1, D=2048),
        # all rows of a calibration set through a norm
        dict(name="norm_rows", kind="norm", dtype="bf16", M=131072, D=2048),
        # a training step's norm, its input kept in 8 bits
        dict(name="norm_step", kind="norm_step", dtype="bf16", M=65536, D=1024),
        # the same in fp32 on rows that are not whole 16-byte groups
        dict(name="norm_step_ragged", kind="norm_step", dtype="f32", M=16411, D=1001),
        # one row through the first product of a block
        dict(name="linear_token", kind="linear", dtype="bf16", M=1, K=2048, N=8192, act="gelu", residual=False, pack=False),
        # a classifier's head in fp32
        dict(name="linear_head", kind="linear", dtype="f32", M=4096, K=512, N=1000, act="none", residual=False, pack=False),
        # the first product of a wide block
        dict(name="linear_rows", kind="linear", dtype="bf16", M=16384, K=2048, N=8192, act="gelu", residual=False, pack=False),
        # the first product of a block in training: its pre-activation is kept in 8 bits
        dict(name="linear_pack", kind="linear", dtype="bf16", M=16384, K=1024, N=4096, act="gelu", residual=False, pack=True),
        # odd lengths everywhere, and a residual
        dict(name="linear_ragged", kind="linear", dtype="bf16", M=5003, K=1030, N=1001, act="silu", residual=True, pack=False),
        # the second product's gradients in training
        dict(name="linear_grad", kind="linear_grad", dtype="bf16", M=16384, K=4096, N=1024, act="gelu"),
        # the same in fp32 on a feature map's channels
        dict(name="linear_grad_f32", kind="linear_grad", dtype="f32", M=8192, K=1024, N=256, act="gelu_tanh"),
        # calibration logits to 8 bits and back
        dict(name="checkpoint_rows", kind="checkpoint", dtype="f32", M=65536, D=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """Half of the lengths as they come, half in whole 16-byte groups."""
    D = _log_int(rng, lo, hi)
    return D if rng.random() < 0.5 else max(8, (D + 7) // 8 * 8)


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def draw(rng):
    """Any of the passes: 1 .. 131072 rows, lengths of 24 .. 8192, no more than 2^28 entries and, for products, 2.7e11
    multiplications in bfloat16 and 3.4e10 in fp32."""
    kind = rng.choice(["norm", "norm_step", "linear", "linear", "linear", "linear_grad", "linear_grad", "checkpoint"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    case = dict(kind=kind, dtype=dtype)
    if kind in ("norm", "norm_step", "checkpoint"):
        D = _length(rng, 24, 8192)
        most = (1 << (28 if kind == "norm" else 26)) // D
        return dict(case, M=_log_int(rng, 1 if kind == "norm" else 64, min(131072, most)), D=D)
    K, N = _length(rng, 64, 8192), _length(rng, 64, 8192)
    most = int((2.7e11 if dtype == "bf16" else 3.4e10) / (K * N * (2 if kind == "linear_grad" else 1)))
    M = _log_int(rng, 1 if kind == "linear" else 256, max(256, min(32768, most, (1 << 27) // max(K, N))))
    case.update(M=M, K=K, N=N, act=rng.choice(ACTS))
    if kind == "linear":
        case.update(residual=rng.random() < 0.5, pack=dtype == "bf16" and M >= 64 and rng.random() < 0.3)
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Draws:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 7919 + 4243)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape, scale=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda") * scale

    def rows(self, M, D, scale=1.0):
        """A residual stream's rows: channels with means of their own and a few of much larger deviation."""
        sd = torch.exp(self.normal(D, scale=0.5)) * scale
        return (self.normal(M, D) * sd + self.normal(D, scale=0.3 * scale)).to(self.dtype)

    def weight(self, N, K):
        return self.normal(N, K, scale=1.0 / math.sqrt(K)).to(self.dtype)


def prepare(case, seed):
    d = _Draws(seed, case["dtype"])
    M, s = case["M"], dict(case=case)
    if case["kind"] in ("norm", "norm_step", "checkpoint"):
        D = case["D"]
        s["x"] = d.rows(M, D)
        if case["kind"] != "checkpoint":
            s["w"], s["b"] = 1.0 + d.normal(D, scale=0.2), d.normal(D, scale=0.1)
        if case["kind"] == "norm_step":
            s["dy"], s["add"] = d.normal(M, D, scale=1e-2).to(d.dtype), d.normal(M, D, scale=1e-2).to(d.dtype)
        return s
    K, N = case["K"], case["N"]
    s["w"] = d.weight(N, K)
    if case["kind"] == "linear":
        s["x"], s["b"] = d.rows(M, K), d.normal(N, scale=0.1)
        s["res"] = d.rows(M, N) if case["residual"] else None
    else:
        s["dy"] = d.normal(M, N, scale=1e-2).to(d.dtype)
        s["codes"], s["scales"] = _pack(d.rows(M, K))  # as the forward pass left them
    return s


# ---------------------------------------------------------------------------
# the operators in their plain form: 32 bits, rounded once
# ---------------------------------------------------------------------------
def _groups(x):
    """Rows x groups x 128, zeros behind a row's end."""
    M, D = x.shape
    return torch.nn.functional.pad(x, (0, -D % GROUP)).view(M, -1, GROUP)


def _pack(x):
    """Codes of 8 bits and one scale a group: the largest magnitude a is 127 steps of a / 127."""
    v = _groups(x.float())
    a = v.abs().amax(2)
    k = torch.full_like(a, 127.0)
    held = a >= 2.0 ** -100
    q = torch.round(v * torch.where(held, k / a, torch.zeros_like(a))[:, :, None])
    return q.to(torch.int8).view(x.shape[0], -1)[:, :x.shape[1]].contiguous(), torch.where(held, a / k, torch.zeros_like(a))


def _unpack(codes, scales):
    return (_groups(codes.float()) * scales[:, :, None]).view(codes.shape[0], -1)[:, :codes.shape[1]]


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "checkpoint":
        return _unpack(*_pack(s["x"])).to(s["x"].dtype)
    if kind in ("norm", "norm_step"):
        x, t = s["x"].float(), s["x"].dtype
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + EPS)
        y = (x * rstd[:, None] * s["w"] + s["b"]).to(t)
        if kind == "norm":
            return dict(y=y, mean=mean, rstd=rstd)
        xh = (_unpack(*_pack(s["x"])) - mean[:, None]) * rstd[:, None]
        dy = s["dy"].float()
        g = dy * s["w"]
        dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) + s["add"].float()
        return dict(y=y, dx=dx.to(t), dw=(dy * xh).sum(0), db=dy.sum(0))
    w = s["w"].float()
    if kind == "linear":
        z = s["x"].float() @ w.t() + s["b"]
        y = _act(z, c["act"])
        y = (y if s["res"] is None else y + s["res"].float()).to(s["w"].dtype)
        return dict(y=y, z=_unpack(*_pack(z)).to(y.dtype)) if c["pack"] else y
    z, dy = _unpack(s["codes"], s["scales"]), s["dy"].float()
    dz = ((dy @ w) * _act_grad(z, c["act"])).to(s["w"].dtype)
    return dict(dz=dz, dw=(dy.t() @ _act(z, c["act"])).to(s["w"].dtype), db=dy.sum(0))


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _library(s):
    import paper_2509_26277_amd as cat

    c = s["case"]
    kind = c["kind"]
    if kind == "checkpoint":
        return cat.cat_unpack8(*cat.cat_pack8(s["x"]), dtype=s["x"].dtype)
    if kind == "norm":
        y, mean, rstd = cat.cat_layer_norm(s["x"], s["w"], s["b"], eps=EPS, want_stats=True)
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "norm_step":
        y, mean, rstd, packed = cat.cat_layer_norm(s["x"], s["w"], s["b"], eps=EPS, want_stats=True, pack=True)
        dx, dw, db = cat.cat_layer_norm_backward(s["dy"], mean, rstd, s["w"], packed=packed, residual_grad=s["add"])
        return dict(y=y, dx=dx, dw=dw, db=db)
    if kind == "linear":
        out = cat.cat_linear(s["x"], s["w"], s["b"], act=c["act"], residual=s["res"], pack=c["pack"])
        return dict(y=out[0], z=cat.cat_unpack8(*out[1], dtype=out[0].dtype)) if c["pack"] else out
    packed = (s["codes"], s["scales"])
    dz = cat.cat_linear_backward_input(s["dy"], s["w"], act=c["act"], packed=packed)
    dw, db = cat.cat_linear_backward_weight(s["dy"], packed=packed, act=c["act"])
    return dict(dz=dz, dw=dw, db=db)


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    M = case["M"]
    if case["kind"] in ("norm", "norm_step", "checkpoint"):
        D = case["D"]
        held = M * D + 4 * M * -(-D // GROUP)  # codes and scales
        if case["kind"] == "norm":
            return dict(bytes=2 * M * D * e + 8 * D + 8 * M, flops=8 * M * D)
        if case["kind"] == "norm_step":  # x, dy, add in, y, dx out; the checkpoint out and in
            return dict(bytes=5 * M * D * e + 2 * held + 16 * D + 16 * M, flops=25 * M * D)
        return dict(bytes=2 * M * D * e + 2 * held, flops=4 * M * D)
    K, N = case["K"], case["N"]
    if case["kind"] == "linear":
        held = M * N + 4 * M * -(-N // GROUP)
        return dict(bytes=(M * K + N * K + M * N * (2 if case["residual"] else 1)) * e + 4 * N
                    + (2 * held + M * N * e if case["pack"] else 0), flops=2 * M * N * K)
    return dict(bytes=(M * N + 2 * N * K + M * K) * e + M * K + 4 * M * -(-K // GROUP) + 4 * N, flops=4 * M * N * K)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _held64(x):
    """What a checkpoint of x stands for.  The format's own two roundings of a group's step to 32 bits are part of it."""
    M, D = x.shape
    out = torch.empty(M, D, dtype=torch.float64, device=x.device)
    for at in range(0, D, GROUP):
        v = x[:, at:at + GROUP].double()
        a = v.abs().max(dim=1, keepdim=True).values
        up, step = (127.0 / a).float().double(), (a / 127.0).float().double()
        out[:, at:at + GROUP] = torch.where(a < 2.0 ** -100, torch.zeros_like(v), (v * up).float().double().round() * step)
    return out


def _act64(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).to(z)
    if act == "gelu":  # z Phi(z)
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p + z * p * (1 - p)
    u = (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)  # 0.5 (1 + tanh u) is the logistic function at 2 u
    p = 1 / (1 + torch.exp(-2 * u))
    return z * p, p + z * p * (1 - p) * 2 * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * z ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "checkpoint":
        return _held64(s["x"])
    if kind in ("norm", "norm_step"):
        x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        sd = torch.sqrt(var + EPS)
        y = torch.addcmul(b, (x - mean) / sd, w)
        if kind == "norm":
            return dict(y=y, mean=mean[:, 0], rstd=1 / sd[:, 0])
        del x
        h = (_held64(s["x"]) - mean) / sd
        dy = s["dy"].double()
        g = dy * w
        D = g.shape[1]
        dx = s["add"].double() + (g - (g.sum(1, keepdim=True) + h * (g * h).sum(1, keepdim=True)) / D) / sd
        return dict(y=y, dx=dx, dw=torch.einsum("md,md->d", dy, h), db=torch.ones(len(dy), dtype=dy.dtype, device=dy.device) @ dy)
    if kind == "linear":
        z = torch.nn.functional.linear(s["x"].double(), s["w"].double(), s["b"].double())
        y = _act64(z, case["act"])[0]
        if s["res"] is not None:
            y += s["res"]
        return dict(y=y, z=_held64(z)) if case["pack"] else y
    scale = s["scales"].double().repeat_interleave(GROUP, 1)[:, :case["K"]]
    u, du = _act64(s["codes"].double() * scale, case["act"])
    dy = s["dy"].double()
    return dict(dz=torch.mm(dy, s["w"].double()) * du, dw=torch.mm(dy.t(), u), db=torch.ones(len(dy), dtype=dy.dtype, device=dy.device) @ dy)
