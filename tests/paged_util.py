"""Plain 64-bit forms of rotary positions and of the paged cache's step, for the tests (CPU, torch)."""
import math

import torch


def inv_freq(r, theta=10000.0, scaling="none", factor=1.0, L=0, low=1.0, high=4.0):
    """Frequencies as the header defines them, one by one."""
    out = []
    for k in range(r // 2):
        base = theta * factor ** (r / (r - 2)) if scaling == "ntk" else theta
        f = base ** (-2 * k / r)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            wave = 2 * math.pi / f
            if wave > L / low:
                f /= factor
            elif wave >= L / high:
                t = (L / wave - low) / (high - low)
                f = (1 - t) * f / factor + t * f
        elif scaling == "ramp":
            at = lambda beta: r * math.log(L / (beta * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
            lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
            t = min(max((k - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = t * f / factor + (1 - t) * f
        out.append(f)
    return out


def rotate(x, pos, freqs, interleaved=False, magnitude=1.0, transpose=False):
    """x [..., n, d] (64-bit), pos [n]: pair by pair."""
    y = x.clone()
    h = len(freqs)
    for k, f in enumerate(freqs):
        a, b = (2 * k, 2 * k + 1) if interleaved else (k, k + h)
        ang = pos.double() * f
        c, s = torch.cos(ang) * magnitude, torch.sin(ang) * magnitude
        if transpose:
            s = -s
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def make_cache(a2sf, B, H, G, d, dtype, ps, past, room, seed, device="cuda", scale=0.0, garbage=float("nan")):
    """A PagedCache whose sequences hold ``past`` random tokens; everything else in the pool is ``garbage``."""
    g = torch.Generator().manual_seed(seed)
    mp = max(1, -(-(max(past) + room) // ps))
    pages = B * mp + 3
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = order[: B * mp].view(B, mp)
    k = torch.full((pages, H, ps, d), garbage, dtype=dtype)
    v, sc, pos = k.clone(), torch.full((pages, H, ps), garbage), torch.full((pages, H, ps), -7, dtype=torch.int32)
    for b in range(B):
        for s in range(past[b]):
            pg, o = int(table[b, s // ps]), s % ps
            k[pg, :, o] = torch.randn((H, d), generator=g).to(dtype) * (4 if s == 0 else 1)
            v[pg, :, o] = torch.randn((H, d), generator=g).to(dtype)
            sc[pg, :, o] = torch.rand((H,), generator=g)
            pos[pg, :, o] = s
    return a2sf.PagedCache(B, H, d, dtype, ps, pages, mp, group=G, scale=scale, device=device,
                           k_pages=k.to(device), v_pages=v.to(device), scores=sc.to(device), positions=pos.to(device),
                           page_table=table.contiguous().to(device), past=torch.tensor(past, dtype=torch.int32, device=device),
                           start=torch.tensor(past, dtype=torch.int32, device=device))


def slots(cache, x, b, n):
    """[H][n][...] of pool tensor ``x`` (on the CPU), slots 0..n-1 of sequence b."""
    t, ps = cache.page_table.cpu()[b].long(), cache.page_size
    j = torch.arange(n)
    return x[t[j // ps], :, j % ps].transpose(0, 1)


def attend_ref(K, V, q, scores, past, alpha, scale):
    """One sequence and K/V head in 64 bits: K, V [L][d], q [G][n][d], scores [L] -> out, lse, scores, sum P|V|, logit size."""
    G, n, d = q.shape
    L = past + n
    x = torch.einsum("gnd,ld->gnl", q, K) * scale
    hidden = torch.arange(L)[None, :] > past + torch.arange(n)[:, None]
    size = (torch.einsum("gnd,ld->gnl", q.abs(), K.abs()) * scale).max() if L else torch.zeros(())
    x = x.masked_fill(hidden, -math.inf)
    m = x.max(-1, keepdim=True).values
    e = torch.exp(x - m)
    s = e.sum(-1, keepdim=True)
    P = e / s
    w = torch.tensor([float(alpha) ** (n - 1 - i) for i in range(n)], dtype=torch.float64)
    new = scores * float(alpha) ** n + torch.einsum("n,gnl->l", w, P)
    return P @ V, (m + torch.log(s))[..., 0], new, P @ V.abs(), float(size)


def evict_ref(scores, positions, n, budget, recent_from):
    """Slots that stay, ascending, for one head: scores, positions [n] (numpy-like lists)."""
    order = sorted(range(n), key=lambda j: (positions[j] >= recent_from, scores[j], positions[j], j))
    return sorted(order[n - min(n, budget):])
