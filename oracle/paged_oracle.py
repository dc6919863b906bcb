"""Plain 64-bit implementation of the paged key/value cache, from the definitions (torch on the CPU).  Test
infrastructure only.  Batches are packed: sequence b has the rows q_start[b] .. q_start[b+1]-1, its last ones, and
kv_lens[b] keys."""
import torch

E4M3_MAX = 448.0


def e4m3_round(x):
    """float64 -> nearest e4m3 value (ties to even), saturating; subnormals are multiples of 2^-9."""
    x = x.double().clamp(-E4M3_MAX, E4M3_MAX)
    _, e = torch.frexp(x)                                       # |x| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def e4m3_scale(amax):
    """The least power of two s, 2^-100 at least, with amax <= 448 s (amax: float64 tensor without dimensions)."""
    e = -100
    while float(amax) > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def rotate(x, cos, sin):
    """Rows x [..., D] with table rows cos, sin [..., rot/2]: columns j and j + rot/2 are turned."""
    half = cos.shape[-1]
    a, b, rest = x[..., :half].double(), x[..., half:2 * half].double(), x[..., 2 * half:].double()
    c, s = cos.double(), sin.double()
    return torch.cat((a * c - b * s, b * c + a * s, rest), -1)


def sequences(q_start, kv_lens):
    """(b, first row, rows, keys) of each sequence."""
    q = [int(v) for v in q_start]
    return [(b, q[b], q[b + 1] - q[b], int(n)) for b, n in enumerate(kv_lens)]


def slots(table, b, n, page_size, pages):
    """(position, page, slot) of the first n positions of sequence b that lie in a page."""
    out = []
    for p in range(n):
        g = int(table[b][p // page_size])
        if 0 <= g < pages:
            out.append((p, g, p % page_size))
    return out


def append(k, v, k_cache, v_cache, table, q_start, kv_lens, cos=None, sin=None, q=None, k_scale=None, v_scale=None):
    """New (k_cache, v_cache, k_scale, v_scale, q_rot): float64 tensors of values that are not rounded for a 16-bit
    cache, of codes for an e4m3 one.  The caches come as float64 values (codes)."""
    kc, vc = k_cache.clone(), v_cache.clone()
    ks, vs = (k_scale.double().clone(), v_scale.double().clone()) if k_scale is not None else (None, None)
    q_rot = None if q is None else torch.full(q.shape, float("nan"), dtype=torch.float64)
    pages, P = kc.shape[0], kc.shape[2]
    for b, first, n, length in sequences(q_start, kv_lens):
        older = max(length - n, 0)
        place = {p: (g, i) for p, g, i in slots(table, b, length, P, pages)}
        new = {}
        for i in range(n):
            p = length - n + i
            if p < 0:
                continue
            turn = (lambda x: x.double()) if cos is None else (lambda x: rotate(x, cos[p], sin[p]))
            if q is not None:
                q_rot[first + i] = turn(q[first + i])
            if p in place:
                new[p] = (turn(k[first + i]), v[first + i].double())
        if ks is None:
            for p, (kr, vr) in new.items():
                g, i = place[p]
                kc[g, :, i], vc[g, :, i] = kr, vr
            continue
        for w in sorted({p // P for p in new}):
            mine = [p for p in new if p // P == w]
            g = place[mine[0]][0]
            kept = older - w * P  # older keys in the page
            for cache, scales, which in ((kc, ks, 0), (vc, vs, 1)):
                for h in range(cache.shape[1]):
                    s = e4m3_scale(max(new[p][which][h].abs().max() for p in mine))
                    if kept > 0:
                        before = float(scales[g, h])
                        s = max(s, before)
                        if s > before:
                            cache[g, h, :kept] = e4m3_round(cache[g, h, :kept] * (before / s))
                    for p in mine:
                        cache[g, h, p % P] = e4m3_round(new[p][which][h] / s)
                    scales[g, h] = s
    return kc, vc, ks, vs, q_rot


def attention(q, k_cache, v_cache, table, q_start, kv_lens, scale, causal, k_scale=None, v_scale=None):
    """o, lse and, for tolerances, sum_j p_j |v_j| and the largest sum_d |q_d k_jd| scale of each row, float64.  Rows
    behind the last sequence are NaN."""
    T, Hq, D = q.shape
    pages, Hkv, P, _ = k_cache.shape
    o = torch.full((T, Hq, D), float("nan"), dtype=torch.float64)
    lse, spread, size = o[..., 0].clone(), o.clone(), o[..., 0].clone()
    for b, first, n, length in sequences(q_start, kv_lens):
        where = slots(table, b, length, P, pages)
        g = torch.tensor([x[1] for x in where], dtype=torch.long)
        i = torch.tensor([x[2] for x in where], dtype=torch.long)
        pos = torch.tensor([x[0] for x in where], dtype=torch.long)
        row = torch.arange(n) + length - n
        seen = pos[None, :] <= row[:, None] if causal else torch.ones(n, len(where), dtype=torch.bool)
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            kk, vv = k_cache[g, hk, i].double(), v_cache[g, hk, i].double()
            if k_scale is not None:
                kk, vv = kk * k_scale[g, hk].double()[:, None], vv * v_scale[g, hk].double()[:, None]
            x = q[first:first + n, h].double()
            s = torch.where(seen, x @ kk.T * scale, -torch.inf)
            total = torch.logsumexp(s, -1)
            p = torch.where(total[:, None] > -torch.inf, torch.exp(s - total[:, None]), 0.0)
            o[first:first + n, h] = p @ vv
            spread[first:first + n, h] = p @ vv.abs()
            lse[first:first + n, h] = total
            if len(where):
                size[first:first + n, h] = torch.where(seen, x.abs() @ kk.abs().T * scale, 0.0).amax(-1)
            else:
                size[first:first + n, h] = 0.0
    return o, lse, spread, size
