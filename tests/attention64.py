"""Plain 64-bit forms of the position bias and of the attention over 8-bit
frames, written from their definitions (include/snls.h), on the CPU."""
from __future__ import annotations

import math

import torch

F64 = torch.float64


def bucket(x32, edges):
    """Signed bucket of fp32 displacements."""
    j = torch.zeros(x32.shape, dtype=torch.long)
    for e in torch.tensor(list(edges), dtype=torch.float32):
        j += (x32.abs() >= e).long()
    return torch.where(x32 < 0, len(edges) - j, len(edges) + j)


def bias_entries(inds, p, bias):
    """(head, step, row, column) bucket indices of every neighbour and which neighbours contribute."""
    T, R = p["T"], bias["radius"]
    fr, dh, dw = inds[..., 0], inds[..., 1], inds[..., 2]
    ok = (fr >= 0) & (fr < T) & (fr == fr.floor()) & (dh.abs() < 1e6) & (dw.abs() < 1e6)
    t = torch.arange(T).view(1, 1, T, 1, 1, 1)
    step = (torch.where(ok, fr, torch.zeros_like(fr)).long() - t).clamp(-R, R) + R
    hd = torch.arange(p["HD"]).view(1, -1, 1, 1, 1, 1).expand(step.shape)
    return hd, step, bucket(dh, bias["edges"]), bucket(dw, bias["edges"]), ok


def biased(dists, inds, table, p, bias):
    """snls_bias in the precision of dists."""
    hd, st, bh, bw, ok = bias_entries(inds, p, bias)
    sign = 1.0 if p["dist_type"] == 0 else -1.0
    return torch.where(ok & dists.isfinite(), dists + sign * table.to(dists.dtype)[hd, st, bh, bw], dists)


def table_grad(grad, dists, inds, p, bias, heads):
    hd, st, bh, bw, ok = bias_entries(inds, p, bias)
    sign = 1.0 if p["dist_type"] == 0 else -1.0
    nb = 2 * len(bias["edges"]) + 1
    out = torch.zeros(heads, 2 * bias["radius"] + 1, nb, nb, dtype=F64)
    cnt, mag = torch.zeros_like(out), torch.zeros_like(out)
    use = ok & dists.isfinite()
    at = (hd[use], st[use], bh[use], bw[use])
    out.index_put_(at, sign * grad[use].to(F64), accumulate=True)
    cnt.index_put_(at, torch.ones(int(use.sum()), dtype=F64), accumulate=True)
    mag.index_put_(at, grad[use].to(F64).abs(), accumulate=True)
    return out, cnt, mag


def aggregate(v, dists, inds, p, scale):
    """snls_aggregate in 64 bits, differentiable in v and dists."""
    Bn, T, C, H, W, HD, P, s0 = (p[n] for n in ("B", "T", "C", "H", "W", "HD", "ps", "stride0"))
    Ch = C // HD
    nH, nW = (H - 1) // s0 + 1, (W - 1) // s0 + 1
    sign = 1.0 if p["dist_type"] == 0 else -1.0
    fr, dh, dw = (inds[..., j].to(F64) for j in range(3))
    ok = (fr >= 0) & (fr < T) & (fr == fr.floor()) & (dh.abs() < 1e6) & (dw.abs() < 1e6)
    dh, dw, fr = (torch.where(ok, x, torch.zeros_like(x)) for x in (dh, dw, fr))
    fin = dists.isfinite()
    lg = torch.where(fin, sign * scale * torch.where(fin, dists, torch.zeros_like(dists)),
                     torch.full_like(dists, -math.inf))
    top = lg.amax(-1, keepdim=True)
    e = torch.exp(lg - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    w = e / e.sum(-1, keepdim=True).clamp_min(1e-300)
    w = torch.where(ok, w, torch.zeros_like(w))
    vp = v.view(Bn, T, HD, Ch, H, W)
    ar = torch.arange
    b = ar(Bn).view(-1, 1, 1, 1, 1, 1)
    hd = ar(HD).view(1, -1, 1, 1, 1, 1)
    h = (ar(nH) * s0).view(1, 1, 1, -1, 1, 1)
    x = (ar(nW) * s0).view(1, 1, 1, 1, -1, 1)
    t = ar(T).view(1, 1, -1, 1, 1, 1)
    out = torch.zeros(Bn, T, HD, H, W, Ch, dtype=F64)
    cnt = torch.zeros(H, W, dtype=F64)
    for ph in range(-(P // 2), P - P // 2):
        for pw in range(-(P // 2), P - P // 2):
            y, xx = h + ph, x + pw
            inn = (y >= 0) & (y < H) & (xx >= 0) & (xx < W)
            read = 0
            for cy in (0, 1):
                for cx in (0, 1):
                    Y, X = y + dh.floor().long() + cy, xx + dw.floor().long() + cx
                    fy, fx = dh - dh.floor(), dw - dw.floor()
                    wt = (fy if cy else 1 - fy) * (fx if cx else 1 - fx)
                    on = inn & (Y >= 0) & (Y < H) & (X >= 0) & (X < W)
                    val = vp.permute(0, 1, 2, 4, 5, 3)[b, fr.long(), hd, Y.clamp(0, H - 1), X.clamp(0, W - 1)]
                    read = read + val * (wt * on)[..., None]
            add = (w[..., None] * read).sum(5)  # B HD T nH nW Ch
            yc, xc = y.clamp(0, H - 1), xx.clamp(0, W - 1)
            add = add * inn[..., 0, None]
            sh = add.shape[:5]
            out = out.index_put((b[..., 0].expand(sh), t[..., 0].expand(sh), hd[..., 0].expand(sh),
                                 yc[..., 0].expand(sh), xc[..., 0].expand(sh)), add, accumulate=True)
            i2 = inn[0, 0, 0, :, :, 0]
            cnt.index_put_((yc[0, 0, 0, :, :, 0].expand(nH, nW), xc[0, 0, 0, :, :, 0].expand(nH, nW)), i2.to(F64),
                           accumulate=True)
    out = out / cnt.clamp_min(1)[None, None, None, :, :, None]
    return out.permute(0, 1, 2, 5, 3, 4).reshape(Bn, T, C, H, W)


# ------------------------------------------------------------ 8-bit frames --

def e4m3(x, block):
    """(B, HD, Ch, H, W) values -> (values of the codes, scales): the smallest power of two per block, at least
    2^-126, quotients rounded to the nearest of e4m3's numbers, ties to even."""
    B, HD, Ch, H, W = x.shape
    x = x.to(F64)
    ny, nx = -(-H // block), -(-W // block)
    scales = torch.ones(B, HD, ny, nx, dtype=F64)
    codes = torch.zeros_like(x)
    for i in range(ny):
        for j in range(nx):
            blk = x[..., i * block:(i + 1) * block, j * block:(j + 1) * block]
            mag = torch.where(blk.isfinite(), blk.abs(), torch.zeros_like(blk)).amax((2, 3, 4))
            for b in range(B):
                for hd in range(HD):
                    m = float(mag[b, hd])
                    if m > 0:
                        e = max(math.frexp(m / 448.0)[1] - 1, -126)
                        while m > 448.0 * 2.0 ** e:
                            e += 1
                        scales[b, hd, i, j] = 2.0 ** e
            y = (blk / scales[:, :, i, j][:, :, None, None, None]).clamp(-448, 448)
            mant, ex = torch.frexp(y)  # |mant| in [0.5, 1): y = mant * 2^ex
            step = torch.ldexp(torch.ones_like(y), (ex - 4).clamp_min(-9))
            codes[..., i * block:(i + 1) * block, j * block:(j + 1) * block] = torch.round(y / step) * step
    return codes, scales


def decoded(codes, scales, cp):
    """A cache's codes and scales -> values (B, S, HD, H, W, Ch) in 64 bits."""
    Ch, g = cp["C"] // cp["HD"], cp["block"]
    s = scales.to(F64).repeat_interleave(g, 3)[:, :, :, :cp["H"]].repeat_interleave(g, 4)[..., :cp["W"]]
    return codes.cpu().view(torch.float8_e4m3fn).float().to(F64)[..., :Ch] * s.cpu()[..., None]


def attend(q, points, flows, ages, kv, vv, cp, ws, scale, table=None, bias=None):
    """q (n, C), points (n, 3), flows (n, S, 2) fp32 or None, kv / vv from decoded(): (out (n, C), largest |logit|)."""
    HD, H, W, S, C = (cp[n] for n in ("HD", "H", "W", "slots", "C"))
    n, Ch, r = q.shape[0], C // HD, ws // 2
    q = q.to(F64).view(n, HD, Ch)
    if flows is None:
        flows = torch.zeros(n, S, 2)
    out = torch.zeros(n, HD, Ch, dtype=F64)
    biggest = 0.0
    d = torch.arange(ws) - r
    hd = torch.arange(HD).view(-1, 1, 1)
    for i in range(n):
        b, h, w = (int(x) for x in points[i])
        if not (0 <= b < cp["B"] and 0 <= h < H and 0 <= w < W):
            continue
        lgs, vals = [], []
        for s in range(S):
            age = int(ages[b, s])
            Fh, Fw = flows[i, s, 0], flows[i, s, 1]
            if age < 0 or not (abs(float(Fh)) < 1e6 and abs(float(Fw)) < 1e6):
                continue
            ph, pw = h + float(Fh) + d.to(F64), w + float(Fw) + d.to(F64)
            # the centre's place is compared without adding: an offset of -1e-45 leaves row 0
            on = (((float(Fh) >= -(h + d)) & (float(Fh) <= H - 1 - h - d))[:, None]
                  & ((float(Fw) >= -(w + d)) & (float(Fw) <= W - 1 - w - d))[None])
            y, x = ph.floor().long(), pw.floor().long()
            fy, fx = ph - ph.floor(), pw - pw.floor()
            kt, vt = 0, 0
            for cy in (0, 1):
                for cx in (0, 1):
                    Y, X = (y + cy)[:, None], (x + cx)[None]
                    wgt = (fy if cy else 1 - fy)[:, None] * (fx if cx else 1 - fx)[None]
                    inn = (Y >= 0) & (Y < H) & (X >= 0) & (X < W)
                    Yc, Xc = Y.clamp(0, H - 1), X.clamp(0, W - 1)
                    k1 = torch.where(inn[None, ..., None], kv[b, s][hd, Yc, Xc], torch.zeros((), dtype=F64))
                    v1 = torch.where((inn & (wgt != 0))[None, ..., None], vv[b, s][hd, Yc, Xc],
                                     torch.zeros((), dtype=F64))
                    kt = kt + wgt[None, ..., None] * k1
                    vt = vt + wgt[None, ..., None] * v1
            lg = (kt * q[i][:, None, None]).sum(-1)
            if table is not None:
                bh, bw = bucket(Fh + d.float(), bias["edges"]), bucket(Fw + d.float(), bias["edges"])
                st = min(max(-age, -bias["radius"]), bias["radius"]) + bias["radius"]
                lg = lg + table.to(F64)[hd, st, bh[:, None], bw[None]]
            lg = scale * lg
            lg = torch.where(on[None] & lg.isfinite(), lg, torch.full_like(lg, -math.inf))
            lgs.append(lg.reshape(HD, -1))
            vals.append(vt.reshape(HD, ws * ws, Ch))
        if not lgs:
            continue
        lg, vt = torch.cat(lgs, 1), torch.cat(vals, 1)
        if lg.isfinite().any():
            biggest = max(biggest, float(lg[lg.isfinite()].abs().max()))
        top = lg.amax(1, keepdim=True)
        e = torch.exp(lg - torch.where(top.isfinite(), top, torch.zeros_like(top)))
        p = e / e.sum(1, keepdim=True).clamp_min(1e-300)
        vt = torch.where((p > 0)[..., None], vt, torch.zeros((), dtype=F64))
        out[i] = (p[..., None] * vt).sum(1)
    return out.view(n, C), biggest
