"""Plain 64-bit forms of the norm, dropout, rotary positions and 8-bit
projections, on the CPU, with bounds on what fp32 arithmetic may differ by."""
import numpy as np
import torch

U = 2.0 ** -24  # half a step of fp32, relative to the value


# ------------------------------------------------------------------ dropout --

def philox(counter, key):
    """Four words of Philox 4x32 with 10 rounds; counter and key lists of whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xffffffff, (a >> 32) ^ c[3] ^ k[1], a & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def words(first, n, seed, step, site):
    """Words of elements first .. first+n-1 as uint64 numpy array (each below 2^32)."""
    seed, step = int(seed) & (2 ** 64 - 1), int(step) & 0xffffffff
    j = np.arange(first // 4, (first + n + 3) // 4, dtype=np.uint64)
    m, s32 = np.uint64(0xffffffff), np.uint64(32)
    c = [j & m, j >> s32, np.full_like(j, step), np.full_like(j, site)]
    k = [seed & 0xffffffff, seed >> 32]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s32) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    w = np.stack(c, 1).reshape(-1)
    return w[first % 4:first % 4 + n]


def drop32(drop):
    return float(np.float32(drop))


def keep_mask(shape, rng, drop, site):
    """Truth values: which elements stay."""
    n = int(np.prod(shape))
    if drop == 0:
        return torch.ones(shape, dtype=torch.bool)
    thr = int(drop32(drop) * 2.0 ** 32)
    return torch.from_numpy(words(0, n, rng[0], rng[1], site) >= np.uint64(thr)).view(shape)


def dropout(x, rng, drop, site):
    x = x.double()
    if drop == 0:
        return x
    return torch.where(keep_mask(x.shape, rng, drop, site), x / (1 - drop32(drop)), torch.zeros_like(x))


# --------------------------------------------------------------------- norm --

def rows(x):
    """Features (..., C, H, W) or tokens (n, C) with the channels last."""
    return x if x.dim() == 2 else x.movedim(-3, -1)


def unrows(x, like):
    return x if like.dim() == 2 else x.movedim(-1, -3)


def norm(total, gamma, beta, eps):
    """(y, mean, rstd) of 64-bit features."""
    z = rows(total)
    mean = z.mean(-1)
    d = z - mean[..., None]
    rstd = 1 / torch.sqrt((d * d).mean(-1) + eps)
    y = d * rstd[..., None]
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return unrows(y, total), mean, rstd


def norm_bound(total, gamma, beta, eps, total_err):
    """Largest error of fp32's y, mean and rstd: a sum of C terms is off by C roundings of its terms' magnitudes."""
    z, e = rows(total), rows(total_err)
    C = z.shape[-1]
    y, mean, rstd = norm(total, gamma, beta, eps)
    g = torch.ones(C, dtype=torch.float64) if gamma is None else gamma.double().abs()
    dm = (C + 1) * U * z.abs().mean(-1) + e.mean(-1)
    d = (z - mean[..., None]).abs()
    dd = dm[..., None] + e + U * d  # of a difference from the mean
    var = (d * d).mean(-1)
    dvar = (2 * d * dd + dd * dd).mean(-1) + (C + 3) * U * var
    # 1 / sqrt(v) over the range that dvar leaves, and three roundings
    low = torch.clamp(var + eps - dvar, min=0)
    dr = 1 / torch.sqrt(low) - rstd + 4 * U / torch.sqrt(low)
    dy = g * ((d + dd) * dr[..., None] + dd * rstd[..., None]) + 4 * U * (g * d * rstd[..., None])
    dy = dy + 2 * U * rows(y).abs()
    return unrows(dy, total), dm, dr


def norm_backward(gy, total, stats, gamma, gtotal):
    """(gx, ggamma, gbeta) from statistics as given, in 64 bits, and bounds on fp32's errors of the same shapes.
    few: terms that are summed in fp32 before 64 bits take over."""
    few = 512
    gy, z = rows(gy.double()), rows(total.double())
    C = z.shape[-1]
    mean, rstd = stats[0].double()[..., None], stats[1].double()[..., None]
    xh = (z - mean) * rstd
    g = gy if gamma is None else gy * gamma.double()
    mg, mgx = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    gx = rstd * (g - mg - xh * mgx)
    add = 0 if gtotal is None else rows(gtotal.double())
    out = gx + add
    ag, agx, axh = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True), xh.abs()
    dxh = 2 * U * axh
    err = U * g.abs() + (C + 2) * U * ag + axh * (C + 6) * U * agx + dxh * mgx.abs()
    err = rstd * (err + 4 * U * (g.abs() + mg.abs() + (xh * mgx).abs())) + 2 * U * gx.abs() + U * out.abs()
    flat = lambda t: t.reshape(-1, C).sum(0)  # noqa: E731
    ggamma, gbeta = flat(gy * xh), flat(gy)
    return ((unrows(out, total), ggamma, gbeta),
            (unrows(err, total), (few + 4) * U * flat((gy * xh).abs()), (few + 1) * U * flat(gy.abs())))


# ------------------------------------------------------------------- rotary --

def pair_channels(rp):
    """(axis, first channel, second channel, frequency) of every pair of a head."""
    at, out = 0, []
    for a, n in enumerate(rp["pairs"]):
        theta = float(np.float32(rp["theta"][a]))
        for i in range(n):
            first, second = (at + 2 * i, at + 2 * i + 1) if rp.get("interleaved") else (at + i, at + n + i)
            out.append((a, first, second, theta ** (-i / n)))
        at += 2 * n
    return out


def rotate_video(x, times, rp, inverse=False):
    B, T, C, H, W, HD = (rp[n] for n in ("B", "T", "C", "H", "W", "HD"))
    z = x.double().reshape(B, T, HD, C // HD, H, W)
    if times is None:
        times = torch.arange(T).expand(B, T)
    pos = (times.double().view(B, T, 1, 1, 1), (rp.get("row0", 0) + torch.arange(H).double()).view(1, 1, 1, H, 1),
           (rp.get("col0", 0) + torch.arange(W).double()).view(1, 1, 1, 1, W))
    out = [z[:, :, :, c] for c in range(C // HD)]
    for axis, i, j, f in pair_channels(rp):
        ang = pos[axis] * f * (-1 if inverse else 1)
        out[i], out[j] = z[:, :, :, i] * torch.cos(ang) - z[:, :, :, j] * torch.sin(ang), \
            z[:, :, :, i] * torch.sin(ang) + z[:, :, :, j] * torch.cos(ang)
    return torch.stack(out, 3).reshape(x.shape)


def rotate_points(q, points, times, rp, inverse=False):
    n, HD = q.shape[0], rp["HD"]
    z = q.double().reshape(n, HD, -1)
    b, h, w = (points[:, j].long() for j in range(3))
    ok = (b >= 0) & (b < rp["B"]) & (h >= 0) & (h < rp["H"]) & (w >= 0) & (w < rp["W"])
    t = torch.zeros(n, dtype=torch.float64) if times is None else times[b.clamp(0, rp["B"] - 1)].double()
    pos = (t, rp.get("row0", 0) + h.double(), rp.get("col0", 0) + w.double())
    out = z.clone()
    for axis, i, j, f in pair_channels(rp):
        ang = (pos[axis] * f * (-1 if inverse else 1))[:, None]
        out[..., i] = z[..., i] * torch.cos(ang) - z[..., j] * torch.sin(ang)
        out[..., j] = z[..., i] * torch.sin(ang) + z[..., j] * torch.cos(ang)
    return torch.where(ok[:, None, None], out, torch.zeros_like(out)).reshape(q.shape)


def rotate_bound(x, rp, shape, far=0.0):
    """Per element 5 roundings of its pair's magnitudes: one of the angle, two of the sine or cosine, two of the
    products; far: the largest angle, whose own error is at most |angle| 2^-51."""
    Ch = rp["C"] // rp["HD"]
    z = x.double().abs()
    z = z.reshape(rp["B"], rp["T"], rp["HD"], Ch, rp["H"], rp["W"]).movedim(3, -1) if x.dim() > 2 else \
        z.reshape(x.shape[0], rp["HD"], Ch)
    out = torch.zeros_like(z)
    for _, i, j, _ in pair_channels(rp):
        out[..., i] = out[..., j] = (5 * U + far * 2.0 ** -51) * (z[..., i] + z[..., j])
    return (out.movedim(-1, 3) if x.dim() > 2 else out).reshape(shape)


# -------------------------------------------------------------- projections --

def quantise(v):
    """Codes (64 bits) and scales (fp32 values) along the last axis; scales NaN and codes 0 where not all is finite."""
    v = v.double()
    most = v.abs().amax(-1)
    ok = torch.isfinite(v).all(-1)
    s = (torch.where(ok, most, torch.ones_like(most)).clamp_min(2.0 ** -100) / 127).float().double()
    codes = torch.round(torch.where(ok[..., None], v, torch.zeros_like(v)) / s[..., None])  # halves to even
    return codes, torch.where(ok, s, torch.full_like(s, float("nan")))


def project(x, codes, scales, bias, parts):
    """(out, bound on fp32's error): a rounding each of the scaled sum's product and of the last addition."""
    q, s = quantise(rows(x))
    w = codes.double()
    acc = (q.reshape(-1, q.shape[-1]) @ w.t()).reshape(q.shape[:-1] + (w.shape[0],))
    prod = acc * s[..., None] * scales.double()
    out = prod if bias is None else prod + bias.double()
    err = 2 * U * prod.abs() + U * out.abs()

    def split(t):
        t = torch.stack(t.chunk(parts, -1))
        return t if x.dim() == 2 else t.movedim(-1, -3)

    return split(out), split(err)
