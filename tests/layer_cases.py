"""References and bounds of the tests of 4-bit weights and of the layer for few rows."""
import torch

from row_cases import ffn_reference, unit

U32 = 2.0 ** -24
SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def quantised(x):
    """The 4-bit form of rows [.., C] by its definition in 64 bits: codes and scales as integers, values in 64 bits."""
    C = x.shape[-1]
    w = torch.nn.functional.pad(x.double(), (0, -C % 32))
    w = w.reshape(*x.shape[:-1], -1, 32)
    bad = ~torch.isfinite(w).all(-1)
    w = torch.where(bad[..., None], torch.zeros_like(w), w)
    top = w.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, torch.full_like(top, -127).int()).clamp(min=-127)     # frexp: top in [2^(e - 1), 2^e)
    v = torch.ldexp(w, -e[..., None])
    size = v.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0)).double()
    size = (torch.round(size / step) * step).clamp(max=6.0)                 # halves to even
    code = (size[..., None] == torch.tensor(SIZES, dtype=torch.float64, device=x.device)).int().argmax(-1)
    code = code + 8 * torch.signbit(v).int()
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    values = torch.ldexp(torch.where(torch.signbit(v), -size, size), e[..., None])
    values = torch.where(bad[..., None], torch.full_like(values, float("nan")), values)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127)
    codes = code[..., 0::2] + 16 * code[..., 1::2]
    lead = x.shape[:-1]
    return codes.reshape(*lead, -1), scales, values.reshape(*lead, -1)[..., :C]


def values_of(w, C):
    """What codes and scales stand for, in 64 bits."""
    if not isinstance(w, dict):
        return w
    codes = torch.stack([w["codes"] & 15, w["codes"] >> 4], -1).long()
    size = torch.tensor(SIZES + tuple(-s for s in SIZES), dtype=torch.float64, device=codes.device)[codes]
    power = torch.where(w["scales"] == 255, float("nan"), torch.ldexp(torch.ones_like(w["scales"], dtype=torch.float64), w["scales"].int() - 127))
    size = size.reshape(*w["scales"].shape, 32) * power[..., None]
    return size.reshape(*w["codes"].shape[:-1], -1)[..., :C]


def layer(x, w_router, b_router, wg, wu, wd, k, act):
    """The layer in 64 bits: ids, weights and y with the bounds of their errors.  The bounds of the blocks are those of the feed-forward
    operator; a weight is off by a fast exponential of a difference rounded to fp32 and a quotient; the sum of k terms, each in parts, by a
    rounding per addition, the result by half a step."""
    n, C = x.shape
    H = wg.shape[1] if not isinstance(wg, dict) else wg["codes"].shape[1]
    logits = x.double() @ w_router.double().t()
    if b_router is not None:
        logits = logits + b_router.double()
    rank = torch.where(torch.isnan(logits), torch.full_like(logits, -torch.inf), logits)
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1]
    # NaN behind -inf.
    order = torch.gather(order, 1, torch.sort(torch.isnan(logits.gather(1, order)).int(), dim=-1, stable=True)[1])
    ids = order[:, :k]
    top = logits.gather(1, ids)
    d = top - top[:, :1]
    p = torch.exp(d)
    p = p / p.sum(-1, keepdim=True)
    err_p = p * (2.0 ** -20 + d.abs() * 2.0 ** -23)
    y, err, size = (torch.zeros((n, C), dtype=torch.float64, device=x.device) for _ in range(3))
    pick = lambda w, e: {i: t[e] for i, t in w.items()} if isinstance(w, dict) else w[e]        # noqa: E731
    for e in range(w_router.shape[0]):
        row, j = (ids == e).nonzero(as_tuple=True)
        if not len(row):
            continue
        g, u, v = values_of(pick(wg, e), C), values_of(pick(wu, e), C), values_of(pick(wd, e), H)
        z, bound = ffn_reference(x[row], g, u, v, act)["y"]
        q, eq = p[row, j][:, None], err_p[row, j][:, None]
        y.index_add_(0, row, q * z)
        err.index_add_(0, row, q * bound + eq * (z.abs() + bound))
        size.index_add_(0, row, q * (z.abs() + bound))
    err = err + (k + 12) * U32 * size
    return ids, (p, err_p * 1.05 + 1e-37), (y, err * 1.05 + unit(x.dtype) * 1.02 * y.abs() + torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps)
