"""References and bounds of the tests of dropout and of the residual operator."""
import numpy as np
import torch

from row_cases import expert_of_rows, unit

U32 = 2.0 ** -24
PARAMS = ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias")


def philox(counter, key):
    """Philox4x32 with 10 rounds on arrays of 32-bit words held in 64 bits: counter (4), key (2)."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c, k = [np.asarray(w, dtype=u) for w in counter], [int(w) for w in key]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def kept(seed, rows, C, p):
    """[rows, C] of truth values."""
    G = -(-C // 8)
    s, number = int(seed[0]) % 2 ** 64, int(seed[1]) % 2 ** 64
    row, group = np.repeat(np.arange(rows), G), np.tile(np.arange(G), rows)
    like = np.ones(rows * G, dtype=np.uint64)
    words = philox([row, group, like * np.uint64(number % 2 ** 32), like * np.uint64(number >> 32)], [s % 2 ** 32, s >> 32])
    bits = np.stack([(w >> np.uint64(16 * half)) & np.uint64(0xFFFF) for w in words for half in (0, 1)], -1)
    return torch.from_numpy(bits.reshape(rows, G * 8)[:, :C] >= threshold(p))


def factor(p):
    """What kept elements are multiplied with, and its relative error as a fp32 number."""
    t = threshold(p)
    return (65536.0 / (65536 - t) if t < 65536 else 0.0), (U32 if t else 0.0)


def tiny(dtype):
    """Half a step of the type's smallest numbers, and the same for fp32's."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def _norm(x, err, eps):
    """Layer norm without weights of rows x that are off by err: statistics, h and the errors of all.  As for the norm operator: a mean
    of C values in fp32 takes C additions and a product; a shift of the differences moves the variance by its product with
    them; rstd moves by half the relative change and takes an approximate root (2 ulp)."""
    C = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    err_mean = err.mean(-1, keepdim=True) + (C + 2) * U32 * (x.abs() + err).mean(-1, keepdim=True)
    d = x - mean
    err_d = err + err_mean + 2 * U32 * d.abs()
    var = d.square().mean(-1, keepdim=True)
    most = err_d.amax(-1, keepdim=True)
    rel = ((C + 4) * U32 * var + 2 * most * var.sqrt() + most ** 2) / (var + eps)
    rstd = (var + eps) ** -0.5
    err_rstd = (rel / 2 / (1 - rel).clamp(min=0.25) + 6 * U32) * rstd * 1.05
    h = d * rstd
    return mean, err_mean, rstd, err_rstd, h, err_d * rstd + (err_rstd / rstd) * (h.abs() + err_d * rstd) + U32 * h.abs()


def forward(x, f, offsets, E, gate, params, eps, keep, p):
    """{name: (value, bound)} of the forward call in 64 bits; keep: [B, N, C] or None."""
    B, N, C = x.shape
    e = expert_of_rows(offsets, N, E).clamp(max=E - 1) if offsets is not None else torch.zeros((B, N), dtype=torch.long, device=x.device)
    v = {k: (params[k].double()[e] if params.get(k) is not None else None) for k in PARAMS}
    xd, h = x.double(), f.double()
    zero, one = torch.zeros_like(h[..., :1]), torch.ones_like(h[..., :1])
    stats = [(zero, zero), (one, zero), (zero, zero), (one, zero)]
    err = torch.zeros_like(h)
    if v["post_weight"] is not None:
        m, em, r, er, h, err = _norm(h, err, eps)
        stats[:2] = [(m, em), (r, er)]
        h, err = h * v["post_weight"], err * v["post_weight"].abs() + U32 * (h * v["post_weight"]).abs()
        if v["post_bias"] is not None:
            h = h + v["post_bias"]
            err = err + U32 * (h.abs() + err)
    k, rel = factor(p)
    if keep is not None:
        h, err = torch.where(keep, h * k, torch.zeros_like(h)), torch.where(keep, err * k + 2 * rel * (h * k).abs(), torch.zeros_like(h))
    s = (v["scale"] if v["scale"] is not None else 1.0) * (gate.double()[..., None] if gate is not None else one)
    term = s * h
    o = xd + term
    err = s.abs() * err + 3 * U32 * term.abs() + U32 * o.abs()
    out = {"out": (o, err * 1.05 + unit(x.dtype) * 1.02 * o.abs() + tiny(x.dtype))}
    if v["pre_weight"] is not None:
        m, em, r, er, h, err = _norm(o, err, eps)
        stats[2:] = [(m, em), (r, er)]
        y = h * v["pre_weight"]
        err = err * v["pre_weight"].abs() + U32 * y.abs()
        if v["pre_bias"] is not None:
            y = y + v["pre_bias"]
            err = err + U32 * (y.abs() + err)
        out["y"] = (y, err * 1.05)
    out["stats"] = (torch.cat([a for a, _ in stats], -1), 1.05 * torch.cat([b.expand_as(a) for a, b in stats], -1))
    return out


def _norm_back(g, err_g, h, err_h, r):
    """r (g - mean(g) - h mean(g h)) and its error: the means add C terms."""
    C = g.shape[-1]
    a, c = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    err_a = err_g.mean(-1, keepdim=True) + (C + 3) * U32 * (g.abs() + err_g).mean(-1, keepdim=True)
    err_c = (err_g * h.abs() + g.abs() * err_h).mean(-1, keepdim=True) + (C + 6) * U32 * ((g.abs() + err_g) * h.abs()).mean(-1, keepdim=True)
    v = r * (g - a - h * c)
    return v, r * (err_g + err_a + err_h * (c.abs() + err_c) + h.abs() * err_c + 4 * U32 * (g.abs() + a.abs() + (h * c).abs())) * 1.05


def gradients(o, f, offsets, E, stats, grad_out, grad_y, gate, params, keep, p):
    """{name: (value, bound)} of the gradients in 64 bits, by the formulas, from the same statistics."""
    B, N, C = f.shape
    e = expert_of_rows(offsets, N, E) if offsets is not None else torch.zeros((B, N), dtype=torch.long, device=f.device)
    at, inside = e.clamp(max=E - 1), (e < E)[..., None]
    v = {k: (params[k].double()[at] if params.get(k) is not None else None) for k in PARAMS}
    # Rows of no expert may hold anything.
    clean = lambda t: None if t is None else torch.where(inside, t.double(), torch.zeros((), dtype=torch.float64, device=f.device))   # noqa: E731
    fd, do, dy = clean(f), clean(grad_out), clean(grad_y)
    st = clean(stats) if stats is not None else None
    if do is None:
        do = torch.zeros_like(fd)
    err_do = torch.zeros_like(fd)
    out = {}
    sums = {}
    if v["pre_weight"] is not None:
        h2 = (clean(o) - st[..., 2:3]) * st[..., 3:]
        err_h2 = 2.1 * U32 * h2.abs()
        g = dy * v["pre_weight"]
        back, err = _norm_back(g, U32 * g.abs(), h2, err_h2, st[..., 3:])
        do = do + back
        err_do = err + U32 * do.abs() + 2 * U32 * back.abs()
        sums["grad_pre_weight"] = (dy * h2, dy.abs() * err_h2 + U32 * (dy * h2).abs())
        sums["grad_pre_bias"] = (dy, torch.zeros_like(dy))
    out["grad_x"] = (do, err_do * 1.05 + unit(o.dtype) * 1.02 * do.abs() + tiny(o.dtype))
    k, rel = factor(p)
    t, err_t = do, err_do
    if keep is not None:
        zero = torch.zeros_like(do)
        t, err_t = torch.where(keep, do * k, zero), torch.where(keep, err_do * k + 2 * rel * (do * k).abs(), zero)
    gt = gate.double()[..., None] if gate is not None else 1.0
    gt = clean(gate[..., None]) if gate is not None else torch.ones_like(fd[..., :1])
    q = t * gt
    err_q = err_t * gt.abs() + U32 * q.abs()
    h, err_h, r = fd, torch.zeros_like(fd), None
    if v["post_weight"] is not None:
        r = st[..., 1:2]
        h = (fd - st[..., :1]) * r
        err_h = 2.1 * U32 * h.abs()
    w = v["post_weight"] if v["post_weight"] is not None else torch.ones_like(fd)
    b = v["post_bias"] if v["post_bias"] is not None else torch.zeros_like(fd)
    s = v["scale"] if v["scale"] is not None else torch.ones_like(fd)
    normed = h * w + b
    err_n = err_h * w.abs() + 2 * U32 * ((h * w).abs() + b.abs())
    term = s * t * normed
    err = s.abs() * (err_t * (normed.abs() + err_n) + t.abs() * err_n) + 3 * U32 * term.abs()
    out["grad_gate"] = (term.sum(-1), (err.sum(-1) + (C + 2) * U32 * (term.abs() + err).sum(-1)) * 1.05)
    g = q * s * w
    err_g = err_q * (s * w).abs() + 2 * U32 * g.abs()
    if r is not None:
        df, err = _norm_back(g, err_g, h, err_h, r)
    else:
        df, err = g, err_g
    out["grad_f"] = (df, err * 1.05 + unit(f.dtype) * 1.02 * df.abs() + tiny(f.dtype))
    one, two = (q, err_q), (q * h, err_q * h.abs() + q.abs() * err_h + U32 * (q * h).abs())
    per = {}
    for name, (x, ex) in [("one", one), ("two", two), *sums.items()]:
        value, bound, size = (torch.zeros((E, C), dtype=torch.float64, device=f.device) for _ in range(3))
        for i in range(E):
            rows = e == i
            n = int(rows.sum())
            value[i], size[i] = x[rows].sum(0), x[rows].abs().sum(0)
            # A fp32 sum of n terms in any order; their parts pass a few sums more.
            bound[i] = ex[rows].sum(0) + (n + 12) * U32 * (x[rows].abs() + ex[rows]).sum(0)
        per[name] = (value, bound * 1.05, size)
    P = {k: (params[k].double() if params.get(k) is not None else None) for k in PARAMS}
    S, W = (P[i] if P[i] is not None else torch.ones((E, C), dtype=torch.float64, device=f.device) for i in ("scale", "post_weight"))
    Bp = P["post_bias"] if P["post_bias"] is not None else torch.zeros_like(W)
    (v1, b1, z1), (v2, b2, z2) = per["one"], per["two"]
    out["grad_post_weight"] = (S * v2, S.abs() * (b2 + 2 * U32 * z2))
    out["grad_post_bias"] = (S * v1, S.abs() * (b1 + 2 * U32 * z1))
    out["grad_scale"] = (W * v2 + Bp * v1, W.abs() * (b2 + 4 * U32 * z2) + Bp.abs() * (b1 + 4 * U32 * z1))
    for name in sums:
        out[name] = per[name][:2]
    return out
