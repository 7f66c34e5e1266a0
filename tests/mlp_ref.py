"""The MLP half of a block in 64 bits: its loss, the gradients that automatic differentiation gives of it, the same step with its tensors rounded to 8 bits as
the kernels round them, and the bounds that hold rounded gradients to the exact ones.  Plain torch on the CPU."""
import torch

from tests import q8_ref as R

EPS = 1e-6

# Rounding to E4M3 is off by 2^-4 of a value at the most: ROUND, 2^-4 / sqrt(3), of a tensor's 2-norm.  Roundings on the way to a gradient add up in
# quadrature: dY, Wdown, z or h, dz once; x and Wup twice, for both factors of the SwiGLU are off with them: sqrt(4 + 2 * 4) = 3.5 of them.  4.
ROUND = 2.0 ** -4 / 3 ** 0.5
BOUND = 4 * ROUND
# The part of dX along x, which the RMSNorm term takes away: what is left is the difference of two sums of the same products, one with z, dz and x as they were and
# one with them rounded.
BOUND_ALONG = 4 * ROUND


def loss(X, Wup, Wdown, dY):
    r = (X.square().mean(1, keepdim=True) + EPS).rsqrt()
    return ((R.swiglu((X * r) @ Wup.t()) @ Wdown.t() + X) * dY).sum()


def gradients(X, Wup, Wdown, dY):
    """dX, dWup, dWdown by automatic differentiation."""
    at = [t.clone().requires_grad_() for t in (X, Wup, Wdown)]
    return torch.autograd.grad(loss(*at, dY), at)


def rounded(x, square=False):
    if square:
        _, _, s = R.square(x)
        return R.round_e4m3(x / s) * s
    v, byte = R.quantized(x)
    return v * R.per_element(byte, *x.shape)


def step(X, Wup, Wdown, dY, eight=True, mistake=None):
    """dX, dWup, dWdown as the kernels compute them, with the roundings to 8 bits or without; `mistake`: a term left out."""
    q = rounded if eight else (lambda x, square=False: x)
    d = X.shape[1]
    r = (X.square().mean(1, keepdim=True) + EPS).rsqrt()
    x, up, down, dy = q(X), q(Wup, True), q(Wdown, True), q(dY)
    z = x @ up.t() * r
    zq, h = q(z), q(R.swiglu(z))
    g, u, dh = zq[:, 0::2], zq[:, 1::2], dy @ down
    sg = R.sigmoid(g)
    dz = torch.empty_like(z)
    dz[:, 0::2] = dh * u * (sg if mistake == "silu'" else sg + g * sg * (1 - sg))
    dz[:, 1::2] = dh * g * sg
    stat = (dz * zq).sum(1, keepdim=True) / d
    dzq, cn = q(dz), x * r
    if mistake == "gates":
        dzq = dzq.clone()
        dzq[:, 0::2] = 0
    v = dzq @ up
    if mistake == "no mlp":
        v, stat = v * 0, stat * 0
    dX = dY + (v - (0 if mistake == "rmsnorm" else cn * stat)) * r
    half = X.shape[0] // 2 if mistake == "half the tokens" else X.shape[0]
    return dX, dzq[:half].t() @ q(cn)[:half], dy[:half].t() @ h[:half]


def check(got, X, Wup, Wdown, dY):
    """The names of what is out of bounds, of (dX, dWup, dWdown) against automatic differentiation."""
    dX, dWup, dWdown = got
    tX, tWup, tWdown = gradients(X, Wup, Wdown, dY)
    bad = []

    def near(a, b, what):
        if not (a - b).norm() <= BOUND * b.norm():
            bad.append("%s: %.3f" % (what, (a - b).norm() / b.norm()))

    near(dX - dY, tX - dY, "dX")                             # the residual's part is dY itself
    near(dWup[0::2], tWup[0::2], "dWup, gates")
    near(dWup[1::2], tWup[1::2], "dWup, up")
    near(dWdown, tWdown, "dWdown")
    # the loss does not change with the size of a row of x but through the residual (and EPS), so its gradient's other part is at right angles to x
    r = (X.square().mean(1, keepdim=True) + EPS).rsqrt()
    z = (X * r) @ Wup.t()
    dz = R.swiglu_bwd(dY @ Wdown, z)
    along = ((dX - dY) * X).sum(1)
    whole = (dz @ Wup * r * X).sum(1)                        # without the RMSNorm term
    if not along.norm() <= BOUND_ALONG * whole.norm():
        bad.append("dX along x: %.3f" % (along.norm() / whole.norm()))
    return bad
