"""64-bit references and error bounds of the token-major operators (written from the formulas; no code of the library)."""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # rounding to nearest, p bits: 2^-p
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}   # absolute, where results go subnormal
F8 = torch.float8_e4m3fn
SCALE_MIN = 2.0 ** -126


def make_weight(M, C, Nb, p, seed):
    """fp32 weight with a seeded block mask: [M][C] and the mask (numpy)."""
    import ubp_synth
    L = ubp_synth.make_layer("linear", M, C, Nb, p, seed, Nc=1, make_x=False)
    return np.ascontiguousarray(L.W[:, :, 0] * L.mask).astype(np.float32), np.ascontiguousarray(L.mask)


def quantise(v):
    """[rows][n] float tensor -> (codes, scales) in fp32 arithmetic: s = max(max |v| / 448, 2^-126), code = e4m3(v / s)."""
    v = v.float()
    s = (v.abs().amax(1) / 448.0).clamp_min(SCALE_MIN)
    return (v / s[:, None]).to(F8), s


def typed_weight(W, dtype):
    """The weight as the plan holds it, in 64 bits: rounded to the type, or 8-bit codes times the row's scale."""
    w = torch.from_numpy(W)
    if dtype == F8:
        q, s = quantise(w)
        return q.double() * s.double()[:, None]
    return w.to(dtype).double()


def act64(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v / 2.0 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh((2.0 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def product64(x, W, bias, act, gated, residual):
    """x, W, bias, residual as 64-bit tensors (or None) -> (y, error bound per element without the output's rounding).
    Sum of n products in fp32 in any order, each addition rounding or truncating: |error| <= (n + 8) 2^-23 A with
    A = |x||W| + |b| (the 8 covers the scales' products, the bias and joining partial sums). The activations' slopes are
    below 1.13; their own evaluation is good to 2^-18 of the argument."""
    z = x @ W.t()
    A = x.abs() @ W.abs().t()
    n = (W != 0).sum(1).double() + 8
    if bias is not None:
        z, A = z + bias, A + bias.abs()
    dz = A * n * 2.0 ** -23
    if gated:
        F = W.shape[0] // 2
        g, u, dg, du = z[:, :F], z[:, F:], dz[:, :F], dz[:, F:]
        a = act64(g, act)
        da = 1.13 * dg + 2.0 ** -18 * g.abs()
        y = a * u
        d = da * u.abs() + (a.abs() + da) * du
    else:
        y = act64(z, act)
        d = 1.13 * dz + 2.0 ** -18 * (z.abs() if act != "none" else 0.0 * z)
    if residual is not None:
        y = y + residual
        d = d + 2.0 ** -23 * y.abs() + 2.0 ** -23 * residual.abs()
    return y, d


def e4m3_half_step(v):
    """Half the distance between neighbouring e4m3 numbers around |v| (64-bit tensor)."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))).clamp(-6, 8)
    return 0.5 * 2.0 ** (e - 3)
