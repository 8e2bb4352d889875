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
