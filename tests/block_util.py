"""Plain forms in 64 bits of the operators of a block's training step, and the bounds that the tests hold them to.

Half a step of a type is ``finfo(t).eps / 2`` of the value.  A sum of n products in fp32, in any order, is off by at most
n 2^-24 of the sum of their magnitudes."""
import math

import torch

U32 = 2.0 ** -24
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 128


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def pack_ref(x):
    """Codes and scales by the definition; its three roundings to 32 bits made from 64."""
    v = x.double().cpu()
    N, D = v.shape
    G = -(-D // GROUP)
    v = torch.nn.functional.pad(v, (0, G * GROUP - D)).view(N, G, GROUP)
    a = v.abs().amax(2)
    held = a >= 2.0 ** -100
    safe = torch.where(held, a, torch.ones_like(a))
    up, step = (127.0 / safe).float().double(), (safe / 127.0).float()
    code = torch.round((v * up[:, :, None]).float())
    code = torch.where(held[:, :, None], code, torch.zeros_like(code))
    return code.view(N, -1)[:, :D].to(torch.int8), torch.where(held, step, torch.zeros_like(step))


def unpack_ref(codes, scales):
    s = scales.double().cpu().repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return codes.double().cpu() * s


def act_ref(z, act):
    """act(z) and act'(z)."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if act == "gelu":
        p = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1.0 + z * (1.0 - p))
    u = math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)
    t = torch.tanh(u)
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)


# An activation and its derivative in fp32: a few roundings of numbers no larger than 1 + |z|; exp through the hardware's
# exponential is off by about |argument| half steps more, where |z| exp(-|z|) keeps |argument| times its result below 2.
ACT_ERR = 32 * U32
SLOPE = 1.2  # the steepest of the activations (gelu: 1.13); their second derivatives stay below it too


def norm_ref(x, w, b, eps):
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    return xh * w + b, mean[:, 0], rstd[:, 0]


def norm_backward_ref(dy, xh, rstd, w):
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def assert_close(got, want, bound, what):
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        b = bound[i] if torch.is_tensor(bound) and bound.shape == off.shape else bound
        where = [sorted(set(torch.nonzero(bad)[:, d].tolist())) for d in range(bad.dim())]
        where = "; ".join(f"{len(w)} from {w[0]} to {w[-1]}" for w in where)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} entries off ({where}), first at {i}: {got[i]} for {want[i]}, bound {b}")
