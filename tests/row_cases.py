"""Inputs and references of the tests of the operators on dispatched rows."""
import types

import torch

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def unit(dtype):
    """Largest relative error of one rounding to `dtype`."""
    return torch.finfo(dtype).eps / 2


def handle(B, N, E=4, device=0):
    import paper_2507_04123_b200 as pkg
    grid = types.SimpleNamespace(min=(0.0, 0.0, 0.0), voxel=(1.0, 1.0, 1.0), dims=(8, 8, 1), max_points=0)
    return pkg.Bridge(pkg.make_config(device=device, max_batch=B, max_points=N, point_floats=4, grids=(grid, grid), num_cameras=1,
                                      img_h=8, img_w=8, feat_h=8, feat_w=8, feat_c=4, feat_stride=1, min_depth=0.1, thresholds=(),
                                      num_experts=E, lut=((0,), (0,))))


def ascending_offsets(B, N, E, seed, device=DEV):
    """Offsets with rows before the first and behind the last segment, and experts without rows."""
    g = torch.Generator()
    g.manual_seed(seed)
    cuts = torch.sort(torch.randint(0, N + 1, (B, E + 1), generator=g), 1).values
    if B > 1 and E > 2:
        cuts[1, 1] = cuts[1, 2]
    if B > 2:
        cuts[2] = N // 2                                      # a frame without rows of any expert
    cuts[0, 0], cuts[0, -1] = 0, N
    return cuts.to(torch.int32).to(device)


def expert_of_rows(offsets, N, E):
    """[B, N]: the expert of every row, E where none owns it."""
    j = torch.arange(N, device=offsets.device)[None, :, None]
    e = (j >= offsets[:, None, 1:]).sum(-1)
    return torch.where(j[..., 0] < offsets[:, :1], torch.full_like(e, E), e)


def norm_reference(x, e, E, w, b, eps):
    """The formulas of the layer norm in 64 bits; whatever rows of no expert hold comes out as it does."""
    x = x.double()
    at = e.clamp(max=E - 1)
    mean = x.mean(-1)
    var = (x - mean[..., None]).square().mean(-1)
    rstd = (var + eps) ** -0.5
    h = (x - mean[..., None]) * rstd[..., None]
    return {"mean": mean, "var": var, "rstd": rstd, "h": h, "y": h * w.double()[at] + b.double()[at]}


def activation(g, act):
    """act(g), its derivative, and the largest slopes of both, in 64 bits."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s)), 1.1, 0.5
    phi = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * phi, phi + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5, 1.13, 0.8


def ffn_reference(x, wg, wu, wd, act, dy=None):
    """One expert's rows [n, C] through the block and, with dy, its gradients: {name: (value, bound of the library's error)}.

    The bounds follow the roundings.  A sum of n products on the tensor cores is counted 4 u32 per term: it is added in fp32,
    whose adder may cut instead of round (2 u32 a term) and align terms to the largest (2 more).  The activations are off by
    2^-18 of themselves (fast exponential and reciprocal), but SiLU on bf16 rows, whose 1 / (1 + exp(-g)) is off by 2^-12.  Values between two products are rounded to the type, u of themselves
    and half a step of its smallest numbers; so are the results."""
    dtype = x.dtype
    u, tiny, s = unit(dtype), torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2, 4 * 2.0 ** -24
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    C, H = x.shape[1], wg.shape[0]

    def rounded(v, err):
        return err * (1 + u) + u * v.abs() + tiny

    g, up = x @ wg.t(), x @ wu.t()
    err_g, err_u = (C + 16) * s * (x.abs() @ wg.abs().t()), (C + 16) * s * (x.abs() @ wu.abs().t())
    a, da, slope, slope2 = activation(g, act)
    fast = 2.0 ** -18
    quick = 1.01 * 2.0 ** -12 if act == "silu" and dtype == torch.bfloat16 else 0.0
    err_a = slope * err_g + fast * (a.abs() + 2.0 ** -6 * g.abs()) + quick * g.abs()
    if act == "gelu":
        err_a = err_a + (0.75e-7 + 2.0 ** -22) * g.abs()      # of the formula used for the normal distribution, and its rounding
    h = a * up
    err_h = rounded(h, err_a * (up.abs() + err_u) + a.abs() * err_u + 2 * s * h.abs())
    y = h @ wd.t()
    out = {"y": (y, rounded(y, err_h @ wd.abs().t() + (H + 16) * s * ((h.abs() + err_h) @ wd.abs().t())))}
    if dy is None:
        return out
    dy = dy.double()
    n = x.shape[0]
    dh = dy @ wd
    err_dh = (C + 16) * s * (dy.abs() @ wd.abs())
    err_da = slope2 * err_g + 2 * fast * (1 + g.abs()) + quick * (1 + 2 * g.abs())       # s + g s (1 - s), s off by `quick`
    dg, du = dh * up * da, dh * a
    err_dg = rounded(dg, err_dh * ((up * da).abs()) + (dh.abs() + err_dh) * (err_u * (da.abs() + err_da) + up.abs() * err_da) + 3 * s * dg.abs())
    err_du = rounded(du, err_dh * a.abs() + (dh.abs() + err_dh) * err_a + 2 * s * du.abs())
    dx = dg @ wg + du @ wu
    size = (dg.abs() + err_dg) @ wg.abs() + (du.abs() + err_du) @ wu.abs()
    out["grad_x"] = (dx, rounded(dx, err_dg @ wg.abs() + err_du @ wu.abs() + (2 * H + 32) * s * size))
    for name, left, err, right in (("grad_gate", dg, err_dg, x), ("grad_up", du, err_du, x), ("grad_down", dy, None, h)):
        v = left.t() @ right
        if err is None:
            e = left.abs().t() @ err_h + (n + 700) * s * (left.abs().t() @ (right.abs() + err_h))
        else:
            e = err.t() @ right.abs() + (n + 700) * s * ((left.abs() + err).t() @ right.abs())
        out[name] = (v, rounded(v, e))
    return out
