"""Windowed attention with sinks in 64 bits, straight from its definition: one sequence and one head at a time, dense."""
import math

import torch


def visible(lq, lk, window, sinks, device="cpu"):
    """[lq, lk] truth values; window 0: no window."""
    p = torch.arange(lk - lq, lk, device=device)[:, None]
    j = torch.arange(lk, device=device)[None]
    seen = j <= p
    return seen & ((j > p - window) | (j < sinks)) if window else seen


def attention(q, k, v, scale, seen, d_o=None):
    """q, d_o [lq, D], k, v [lk, D] (fp64), seen [lq, lk] -> dict: o, lse, and with d_o the gradients dq, dk, dv; and for tolerances the same
    sums over absolute values: o_abs = sum P |v|, score_abs = max sum |q k| scale, dq_abs, dk_abs, dv_abs, each with the terms' own sizes, and
    their parts from a unit error of delta (dq_delta, dk_delta) with delta_abs = sum |dO o|."""
    s = (q @ k.T) * scale
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.where(seen, torch.exp(s - top), 0.0)
    total = e.sum(1, keepdim=True)
    P = e / torch.where(total == 0, 1.0, total)
    vz, kz = torch.where(seen.any(0)[:, None], v, 0.0), torch.where(seen.any(0)[:, None], k, 0.0)
    r = dict(o=P @ vz, lse=(top + torch.log(total))[:, 0], o_abs=P @ vz.abs(), score_abs=float((q.abs() @ kz.abs().T).max()) * abs(scale))
    if d_o is not None:
        dP = d_o @ vz.T
        delta = (P * dP).sum(1, keepdim=True)
        dS = P * (dP - delta)
        r.update(dq=scale * dS @ kz, dk=scale * dS.T @ q, dv=P.T @ d_o)
        big = P * (dP.abs() + delta.abs())
        delta_abs = (d_o * r["o"]).abs().sum(1, keepdim=True)
        r.update(dq_abs=abs(scale) * big @ kz.abs(), dk_abs=abs(scale) * big.T @ q.abs(), dv_abs=P.T @ d_o.abs(),
                 dq_round=abs(scale) * dS.abs() @ kz.abs(), dk_round=abs(scale) * dS.abs().T @ q.abs(),
                 dq_delta=abs(scale) * (P * delta_abs) @ kz.abs(), dk_delta=abs(scale) * (P * delta_abs).T @ q.abs())
    return r


def chunk(q, k, v, scale, segs, window, sinks, d_o=None):
    """A chunk of segments (lq, prefix): q, d_o [T, Hq, D], k, v [Tk, Hkv, D] -> the dict of attention() in the layouts of the calls, in
    fp64 on q's device."""
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    f = lambda x: x.double()
    out = {}
    row = key = 0
    worst = 0.0
    for lq, prefix in segs:
        lk = lq + prefix
        seen = visible(lq, lk, window, sinks, q.device)
        for h in range(Hq):
            kh = h // (Hq // Hkv)
            r = attention(f(q[row:row + lq, h]), f(k[key:key + lk, kh]), f(v[key:key + lk, kh]), scale, seen,
                          None if d_o is None else f(d_o[row:row + lq, h]))
            worst = max(worst, r.pop("score_abs"))
            for name, x in r.items():
                if name not in out:
                    shape = (Hq, T) if name == "lse" else (k.shape if name[:2] in ("dk", "dv") else q.shape)
                    out[name] = torch.zeros(shape, dtype=torch.float64, device=q.device)
                if name == "lse":
                    out[name][h, row:row + lq] = x
                elif name[:2] in ("dk", "dv"):
                    out[name][key:key + lk, kh] += x
                else:
                    out[name][row:row + lq, h] = x
        row, key = row + lq, key + lk
    out["score_abs"] = worst
    out["keys"] = max(lq + p for lq, p in segs)
    out["rows"] = max(lq for lq, _ in segs) * (Hq // Hkv)
    return out


def tolerances(ref, dtype, D, rounded_products):
    """How far each result may be off, element by element, from what is rounded on the way (half a step, eps / 2 of the value):
      fp32 arithmetic   a sum of n terms: n 2^-24 of their absolute sum; a score: D 2^-24 of sum |q k|, which is a relative error of P
      results           half a step of their type (o, dq)
      delta = <dO, o>   from an o that is rounded to its type, where it is
      rounded_products  P and dS enter the second products with half a step of bf16"""
    bf16 = dtype == torch.bfloat16
    u, half = 2.0 ** -24, 2.0 ** -8 if bf16 else 2.0 ** -24
    c = u * (ref["keys"] + 2 * D * (1 + ref["score_abs"]))
    cr = u * (ref["rows"] + 2 * D * (1 + ref["score_abs"]))
    w = 2.0 ** -8 if rounded_products else 0.0
    tol = dict(o=half * ref["o"].abs() + (w + c) * ref["o_abs"], lse=c + 4 * u * ref["lse"].abs())
    if "dq" in ref:
        tol["dq"] = half * ref["dq"].abs() + w * ref["dq_round"] + half * ref["dq_delta"] + 2 * c * ref["dq_abs"]
        tol["dk"] = w * ref["dk_round"] + half * ref["dk_delta"] + 2 * (c + cr) * ref["dk_abs"]
        tol["dv"] = (w + 2 * (c + cr)) * ref["dv_abs"]
    return tol


def check(got, ref, tol, what):
    for name, t in tol.items():
        g, r = got[name].double(), ref[name]
        same = (g == r) | (torch.isnan(g) & torch.isnan(r))
        off = torch.where(same, 0.0, (g - r).abs())
        bad = ~(off <= t * 1.01 + 1e-37) & ~same
        assert not bad.any(), (what, name, int(bad.sum()), float((off - t)[bad].nan_to_num(nan=math.inf).max()), bad.nonzero()[:4].tolist())
