"""The gated residual with its norms, its gradient and the embedding's in 64 bits, from their formulas in plain torch operations, and how
large an fp32 kernel's error may be: sums of the sizes of the terms, which the tests multiply by fp32's half step."""
import torch

F32 = 2.0 ** -24                                   # half a step, relative


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def of_rows(v, rows, per):
    """A group's vector for every row; None stays None."""
    if v is None:
        return None
    v = v.double().reshape(-1, v.shape[-1])
    return v.expand(rows, -1) if per == 0 else v[torch.arange(rows, device=v.device) // per]


def there(rows, per, lens):
    if lens is None:
        return None
    row = torch.arange(rows, device=lens.device)
    return (row % per < lens.clamp(0, per)[row // per])[:, None]


def masked(v, keep):
    return v if keep is None else torch.where(keep, v, torch.zeros_like(v))


def moments(v, kind, eps):
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return mean, ((v - mean).square().mean(-1, keepdim=True) + eps).rsqrt()


def forward(x, h, gate, weight, bias, per=0, post="none", post_weight=None, norm="layer", plus=0.0, residual=1.0, eps=1e-6):
    """x_out, y, stats and the sizes of the terms of x_out and y; x, h 64-bit, of the rows that are there."""
    rows = x.shape[0]
    zero, one = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    pm, pi = zero, one
    if h is None:
        out, size = x, x.abs()
    else:
        t, tsize = h, h.abs()
        if post != "none":
            pm, pi = moments(h, post, eps)
            pw = 1.0 if post_weight is None else post_weight.double()
            t, tsize = (h - pm) * pi * pw, pi * (h.abs() + h.abs().amax(-1, keepdim=True)) * (pw if post_weight is None else pw.abs())
        g = of_rows(gate, rows, per)
        if g is not None:
            t, tsize = g * t, g.abs() * tsize
        out, size = residual * x + t, abs(residual) * x.abs() + tsize
    y = ysize = None
    m, i = zero, one
    if norm != "none":
        m, i = moments(out, norm, eps)
        gain, b = of_rows(weight, rows, per), of_rows(bias, rows, per)
        gain = torch.ones_like(out) if gain is None else plus + gain
        b = torch.zeros_like(out) if b is None else b
        y, ysize = (out - m) * i * gain + b, gain.abs() * i * (size + size.amax(-1, keepdim=True)) + b.abs()
    return out, y, torch.cat((m, i, pm, pi), 1), size, ysize


def centred(g, xh, kind):
    """g without its parts along xh and (a norm with a mean) along the row's ones; and the sizes of the terms."""
    along, mean = (g * xh).mean(-1, keepdim=True), g.mean(-1, keepdim=True)
    size = g.abs() + xh.abs() * (g * xh).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True)
    return (g - xh * along - mean if kind == "layer" else g - xh * along), size


def group_sum(v, per):
    rows = v.shape[0]
    if per == 0:
        return v.sum(0, keepdim=True)
    n = -(-rows // per)
    return torch.zeros((n, v.shape[1]), dtype=v.dtype, device=v.device).index_add_(0, torch.arange(rows, device=v.device) // per, v)


def backward(x_out, h, stats, gate, weight, dx_out, dy, per=0, lens=None, post="none", post_weight=None, norm="layer", plus=0.0, residual=1.0):
    """name -> (gradient, sizes of its terms), by the formula from the statistics as they are given (64 bits all of it)."""
    some = next(v for v in (x_out, dx_out, h) if v is not None)
    rows = some.shape[0]
    keep = there(rows, per, lens)
    m, i, pm, pi = (masked(s, keep) for s in stats.double().split(1, 1)) if stats is not None else (None,) * 4
    d = torch.zeros_like(some) if dx_out is None else masked(dx_out, keep)
    size, found = d.abs(), {}
    if norm != "none":
        x, g = masked(x_out, keep), masked(dy, keep)
        xh, xsize = (x - m) * i, i * (x.abs() + m.abs())
        gain = of_rows(weight, rows, per)
        gain = torch.ones_like(x) if gain is None else plus + gain
        found["dweight"] = group_sum(g * xh, per), group_sum(g.abs() * xsize, per)
        found["dbias"] = group_sum(g, per), group_sum(g.abs(), per)
        v, vsize = centred(g * gain, xh, norm)
        # xh's own rounding errors enter through its product with the mean
        vsize = vsize + xsize * (g * gain * xsize).abs().mean(-1, keepdim=True)
        d, size = d + i * v, size + i * vsize
    found["dx"] = residual * d, abs(residual) * size
    if h is not None:
        hv = masked(h, keep)
        g = of_rows(gate, rows, per)
        g = torch.ones_like(hv) if g is None else g
        u, usize = g * d, g.abs() * size
        if post == "none":
            found["dgate"] = group_sum(d * hv, per), group_sum(size * hv.abs(), per)
        else:
            pw = torch.ones_like(hv[0]) if post_weight is None else post_weight.double()
            hh, hsize = (hv - pm) * pi, pi * (hv.abs() + pm.abs())
            found["dgate"] = group_sum(d * hh, per) * pw, group_sum(size * hsize, per) * pw.abs()
            found["dpost_weight"] = (u * hh).sum(0), (usize * hsize).sum(0)
            u, usize = u * pw, usize * pw.abs()
            v, vsize = centred(u, hh, post)
            extra = usize + hsize * (usize * hsize).mean(-1, keepdim=True) + usize.mean(-1, keepdim=True)
            u, usize = pi * v, pi * (vsize + extra)
        found["dh"] = masked(u, keep), masked(usize, keep)
    found["dx"] = masked(found["dx"][0], keep), masked(found["dx"][1], keep)
    return found


def embedding_grad(ids, dout, classes, scale, base=None):
    """dtable and the sizes of its terms."""
    ids, d = ids.reshape(-1).long(), dout.double().reshape(ids.numel(), -1)
    ok = (ids >= 0) & (ids < classes)
    table = torch.zeros((classes, d.shape[1]), dtype=torch.float64, device=d.device)
    total, size = table.index_add(0, ids[ok], d[ok]) * scale, table.index_add(0, ids[ok], d[ok].abs()) * abs(scale)
    return (total, size) if base is None else (total + base.double(), size + base.double().abs())
