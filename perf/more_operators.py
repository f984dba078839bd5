"""Operators of quantised and of gated feed-forward blocks as cases that can be timed and compared.

The rows that are corrected come out of a quantised network.  Its products run on 8-bit integers, with a scale for every row
of the activations and one for every output channel of the weight; the feed-forward half of its blocks may be gated,
act(x Wg^T + bg) * (x Wu^T + bu), and is fitted in training before it is quantised.  A case is one pass:

``linear8``     rows to 8 bits, then y = act(x W^T + b) + residual as a product of 8-bit integers with a weight that was
                quantised once; ``norm``: the rows go through layer norm on the way to 8 bits
``gated8``      rows to 8 bits, then the gated product of 8-bit integers
``gated``       the gated product of float or bfloat16 rows; ``pack``: also the checkpoint in 8 bits of both projections,
                returned as the values it stands for
``gated_grad``  the gradients behind the gate, from the checkpoint and the gradient that arrives through the block's last
                product: of both projections, of their bias, of the last product's weight and of its bias

Row counts and lengths are those of ``paper_2509_26277_amd/workloads.py`` (65536 calibration rows, 1000 and 1001 channels,
2048 bfloat16 channels, 256 .. 512 feature channels) or powers of two; the inner length of a block is two to four times the
outer one.
"""
import math

import torch

own = False

GROUP = 128  # channels that share a scale in a checkpoint
EPS = 1e-5


def listed():
    return [
        # one row through the first product of a quantised block at serving time: latency
        dict(name="linear8_token", kind="linear8", dtype="bf16", M=1, K=2048, N=8192, act="gelu", residual=False, norm=False),
        # a small batch through the second one, added to the residual stream
        dict(name="linear8_batch", kind="linear8", dtype="bf16", M=48, K=8192, N=2048, act="none", residual=True, norm=False),
        # the first product of a wide quantised block over calibration rows
        dict(name="linear8_rows", kind="linear8", dtype="bf16", M=16384, K=2048, N=8192, act="gelu", residual=False, norm=False),
        # norm and first product of a narrow one over a whole calibration set
        dict(name="linear8_norm", kind="linear8", dtype="bf16", M=65536, K=512, N=2048, act="gelu", residual=False, norm=True),
        # a quantised classifier's head, whose logits stay float
        dict(name="linear8_head", kind="linear8", dtype="f32", M=65536, K=512, N=1000, act="none", residual=False, norm=False),
        # odd lengths everywhere
        dict(name="linear8_ragged", kind="linear8", dtype="bf16", M=5003, K=1030, N=1001, act="silu", residual=True, norm=False),
        # the gated product of a quantised block over calibration rows
        dict(name="gated8_rows", kind="gated8", dtype="bf16", M=16384, K=2048, F=4096, act="silu"),
        # the same for one row
        dict(name="gated8_token", kind="gated8", dtype="bf16", M=1, K=2048, F=8192, act="silu"),
        # the gated product in training: both projections are kept in 8 bits
        dict(name="gated_pack", kind="gated", dtype="bf16", M=16384, K=1024, F=4096, act="silu", pack=True),
        # in fp32 on a feature map's channels, odd lengths
        dict(name="gated_ragged", kind="gated", dtype="f32", M=4099, K=513, F=1001, act="gelu", pack=False),
        # the gradients behind the gate
        dict(name="gated_grad", kind="gated_grad", dtype="bf16", M=16384, N=1024, F=4096, act="silu"),
        # the same in fp32 on a feature map's channels
        dict(name="gated_grad_f32", kind="gated_grad", dtype="f32", M=8192, N=256, F=1000, act="gelu_tanh"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """Half of the lengths as they come, half in whole 16-byte groups."""
    D = _log_int(rng, lo, hi)
    return D if rng.random() < 0.5 else max(16, (D + 15) // 16 * 16)


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def draw(rng):
    """Any of the passes: 1 .. 65536 rows, lengths of 64 .. 8192, no more than 2^27 entries and 2.7e11 multiplications in 8
    bits or bfloat16, 3.4e10 in fp32."""
    kind = rng.choice(["linear8", "linear8", "linear8", "gated8", "gated", "gated", "gated_grad", "gated_grad"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    act = rng.choice(ACTS)
    a, b = _length(rng, 64, 8192), _length(rng, 64, 8192)
    macs = a * b * (1 if kind == "linear8" else 2)
    least = 256 if kind == "gated_grad" else 1
    most = int((3.4e10 if dtype == "f32" and kind in ("gated", "gated_grad") else 2.7e11) / macs)
    M = _log_int(rng, least, max(least, min(65536, most, (1 << 27) // max(a, 2 * b))))
    case = dict(kind=kind, dtype=dtype, act=act, M=M)
    if kind == "linear8":
        return dict(case, K=a, N=b, residual=rng.random() < 0.5, norm=dtype == "bf16" and rng.random() < 0.4)
    if kind == "gated8":
        return dict(case, K=a, F=b)
    if kind == "gated":
        return dict(case, K=a, F=b, pack=dtype == "bf16" and rng.random() < 0.5)
    return dict(case, N=a, F=b)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Draws:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 6271 + 977)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape, scale=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda") * scale

    def rows(self, M, D, scale=1.0):
        """A residual stream's rows: channels with means of their own and a few of much larger deviation."""
        sd = torch.exp(self.normal(D, scale=0.5)) * scale
        return (self.normal(M, D) * sd + self.normal(D, scale=0.3 * scale)).to(self.dtype)

    def weight(self, N, K):
        return self.normal(N, K, scale=1.0 / math.sqrt(K))


def prepare(case, seed):
    d = _Draws(seed, case["dtype"])
    M, s = case["M"], dict(case=case)
    if case["kind"] in ("linear8", "gated8"):
        K = case["K"]
        N = case["N"] if case["kind"] == "linear8" else 2 * case["F"]
        s["x"], s["b"] = d.rows(M, K), d.normal(N, scale=0.1)
        s["w8"], s["ws"] = _quantize(d.weight(N, K))  # as the network was quantised, once
        if case["kind"] == "linear8":
            s["res"] = d.rows(M, N) if case["residual"] else None
            if case["norm"]:
                s["nw"], s["nb"] = 1.0 + d.normal(K, scale=0.2), d.normal(K, scale=0.1)
        return s
    F = case["F"]
    if case["kind"] == "gated":
        s["x"], s["w"], s["b"] = d.rows(M, case["K"]), d.weight(2 * F, case["K"]).to(d.dtype), d.normal(2 * F, scale=0.1)
        return s
    N = case["N"]
    s["dy"], s["w"] = d.normal(M, N, scale=1e-2).to(d.dtype), d.weight(N, F).to(d.dtype)
    held = [_pack(d.rows(M, F)) for _ in range(2)]  # gate and value, as the forward pass left them
    s["codes"], s["scales"] = (torch.stack(t) for t in zip(*held))
    return s


# ---------------------------------------------------------------------------
# the operators in their plain form: 32 bits, rounded once
# ---------------------------------------------------------------------------
def _codes(v):
    """Codes of 8 bits along the last dimension and the scale of each: the largest magnitude a is 127 steps of a / 127."""
    a = v.abs().amax(-1)
    k = torch.full_like(a, 127.0)
    held = a >= 2.0 ** -100
    q = torch.round(v * torch.where(held, k / a, torch.zeros_like(a))[..., None])
    return q.to(torch.int8), torch.where(held, a / k, torch.zeros_like(a))


def _quantize(x):
    return _codes(x.float())


def _groups(x):
    """Rows x groups x 128, zeros behind a row's end."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % GROUP)).view(x.shape[0], -1, GROUP)


def _pack(x):
    q, s = _codes(_groups(x.float()))
    return q.view(x.shape[0], -1)[:, :x.shape[1]].contiguous(), s


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
    kind, act = c["kind"], c["act"]
    if kind in ("linear8", "gated8"):
        x, t = s["x"].float(), s["x"].dtype
        if c.get("norm"):
            x = x - x.mean(1, keepdim=True)
            x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["nw"] + s["nb"]
        q, qs = _quantize(x)
        z = (q.float() @ s["w8"].float().t()) * (qs[:, None] * s["ws"]) + s["b"]
        if kind == "gated8":
            return (_act(z[:, :c["F"]], act) * z[:, c["F"]:]).to(t)
        y = _act(z, act)
        return (y if s["res"] is None else y + s["res"].float()).to(t)
    F, t = c["F"], s["w"].dtype
    if kind == "gated":
        z = s["x"].float() @ s["w"].float().t() + s["b"]
        gate, value = z[:, :F], z[:, F:]
        h = (_act(gate, act) * value).to(t)
        return dict(h=h, gate=_unpack(*_pack(gate)).to(t), value=_unpack(*_pack(value)).to(t)) if c["pack"] else h
    dy = s["dy"].float()
    gate, value = _unpack(s["codes"][0], s["scales"][0]), _unpack(s["codes"][1], s["scales"][1])
    dh, u = dy @ s["w"].float(), _act(gate, act)
    dz = torch.cat((dh * value * _act_grad(gate, act), dh * u), 1)
    return dict(dz=dz.to(t), db=dz.sum(0), dw=(dy.t() @ (u * value)).to(t), dwb=dy.sum(0))


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _library(s):
    import paper_2509_26277_amd as cat

    c = s["case"]
    kind, act = c["kind"], c["act"]
    if kind in ("linear8", "gated8"):
        if c.get("norm"):
            q, qs = cat.cat_layer_norm_quantize(s["x"], s["nw"], s["nb"], eps=EPS)
        else:
            q, qs = cat.cat_quantize_rows(s["x"])
        if kind == "gated8":
            return cat.cat_gated_linear8(q, qs, s["w8"], s["ws"], s["b"], act=act, dtype=s["x"].dtype)
        return cat.cat_linear8(q, qs, s["w8"], s["ws"], s["b"], act=act, residual=s["res"], dtype=s["x"].dtype)
    if kind == "gated":
        out = cat.cat_gated_linear(s["x"], s["w"], s["b"], act=act, pack=c["pack"])
        if not c["pack"]:
            return out
        h, (codes, scales) = out
        return dict(h=h, gate=cat.cat_unpack8(codes[0], scales[0], dtype=h.dtype), value=cat.cat_unpack8(codes[1], scales[1], dtype=h.dtype))
    packed = (s["codes"], s["scales"])
    dz, db = cat.cat_gated_backward_input(s["dy"], s["w"], packed, act=act)
    dw, dwb = cat.cat_gated_backward_weight(s["dy"], packed, act=act)
    return dict(dz=dz, db=db, dw=dw, dwb=dwb)


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    M, kind = case["M"], case["kind"]
    if kind in ("linear8", "gated8"):
        # rows in, a weight of 8 bits with its scales and bias, rows out; the rows in 8 bits are between two launches
        K, wide = case["K"], case["N"] if kind == "linear8" else 2 * case["F"]
        out = (case["N"] * (2 if case["residual"] else 1)) if kind == "linear8" else case["F"]
        return dict(bytes=M * K * e + wide * (K + 8) + M * out * e, flops=2 * M * wide * K)
    F = case["F"]
    held = M * F + 4 * M * -(-F // GROUP)  # one projection's codes and scales
    if kind == "gated":
        # (the checkpoint is written, read again and returned as rows)
        return dict(bytes=(M * case["K"] + 2 * F * case["K"] + M * F) * e + 8 * F + (4 * held + 2 * M * F * e if case["pack"] else 0),
                    flops=4 * M * F * case["K"])
    N = case["N"]
    return dict(bytes=(M * N + 2 * N * F + 2 * M * F) * e + 2 * held + 8 * F + 4 * N, flops=4 * M * N * F)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _held64(x, group):
    """What x in 8 bits stands for, ``group`` channels to a scale.  The format's own roundings of a group's two quotients and
    of the product to 32 bits are part of it."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[1], group):
        v = x[:, at:at + group].double()
        a = v.abs().max(dim=1, keepdim=True).values
        up, step = (127.0 / a).float().double(), (a / 127.0).float().double()
        out[:, at:at + group] = torch.where(a < 2.0 ** -100, torch.zeros_like(v), (v * up).float().double().round() * step)
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
    kind, act = case["kind"], case["act"]
    if kind in ("linear8", "gated8"):
        x = s["x"].double()
        if case.get("norm"):
            var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
            x = torch.addcmul(s["nb"].double(), (x - mean) / torch.sqrt(var + EPS), s["nw"].double())
        z = torch.nn.functional.linear(_held64(x, x.shape[1]), s["w8"].double() * s["ws"].double()[:, None], s["b"].double())
        if kind == "gated8":
            gate, value = z.chunk(2, 1)
            return _act64(gate, act)[0] * value
        y = _act64(z, act)[0]
        return y if s["res"] is None else y + s["res"].double()
    if kind == "gated":
        wg, wv = s["w"].double().chunk(2)
        bg, bv = s["b"].double().chunk(2)
        x = s["x"].double()
        gate, value = torch.nn.functional.linear(x, wg, bg), torch.nn.functional.linear(x, wv, bv)
        h = _act64(gate, act)[0] * value
        return dict(h=h, gate=_held64(gate, GROUP), value=_held64(value, GROUP)) if case["pack"] else h
    gate, value = (c.double() * k.double().repeat_interleave(GROUP, 1)[:, :case["F"]] for c, k in zip(s["codes"], s["scales"]))
    u, du = _act64(gate, act)
    dy = s["dy"].double()
    dh, ones = torch.mm(dy, s["w"].double()), torch.ones(len(dy), dtype=torch.float64, device=dy.device)
    dz = torch.hstack((dh * value * du, dh * u))
    return dict(dz=dz, db=ones @ dz, dw=torch.mm(dy.t(), u * value), dwb=ones @ dy)
