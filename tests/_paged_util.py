"""Paged caches for the tests: random tables, and the definitions of the operators in 64 bits on the CPU."""
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}       # a rounding is off by half a step at most


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def make_cache(lens, Hkv, page, C, R, dtype, phi_dtype, seed, junk=float("nan"), extra_blocks=1):
    """Pages in random order with `junk` wherever no token lies; table entries behind a request's pages are no pages."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    used = -(-lens // page)
    n_pages = int(used.sum()) + 3
    order = rng.permutation(n_pages)
    blocks = max(1, int(used.max()) + extra_blocks)
    table = np.full((len(lens), blocks), -1)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    held = torch.zeros((n_pages, page), dtype=torch.bool)
    for b, m in enumerate(lens):
        for t in range(0, int(m), page):
            held[table[b, t // page], :min(page, int(m) - t)] = True

    def pages(width, dt, scale=1.0):
        x = (torch.randn((n_pages, Hkv, page, width), generator=g) * scale).to(dt)
        x[~held[:, None, :, None].expand_as(x)] = junk
        return x.cuda()

    return {"k_pages": pages(C, dtype), "v_pages": pages(C, dtype),
            "phi_pages": pages(R, phi_dtype, R ** -0.25) if R else None, "table": i32(table), "lens": i32(lens)}


def gather(pages, table, b, m):
    """[Hkv, m, *] rows of request b in 64 bits."""
    page = pages.shape[2]
    rows = pages[table[b, :-(-m // page)].long()].transpose(0, 1).flatten(1, 2)[:, :m]
    return rows.double().cpu()


def attend64(q, c, starts=None, phi_q=None, slopes=None, causal=True, scale=0.0, hide=None):
    """out, lse and a bound of their errors, from the definition, request by request.  hide[b]: keys that are not seen."""
    B, H, N, C = q.shape
    scale = scale if scale > 0 else C ** -0.5
    Hkv = c["k_pages"].shape[1]
    out = torch.zeros((B, H, N, C), dtype=torch.float64)
    lse = torch.full((B, H, N), -math.inf, dtype=torch.float64)
    tol_o, tol_l = torch.full_like(out, 1e-30), torch.full_like(lse, 1e-30)
    low = q.dtype == torch.bfloat16
    for b, m in enumerate(c["lens"].tolist()):
        if m <= 0:
            continue
        k, v = (gather(c[n], c["table"], b, m).repeat_interleave(H // Hkv, 0) for n in ("k_pages", "v_pages"))
        f = gather(c["phi_pages"], c["table"], b, m).repeat_interleave(H // Hkv, 0) if phi_q is not None else None
        start = m - N if starts is None else int(starts[b])
        for n in range(N):
            pos = start + n
            if causal and not 0 <= pos < m:
                continue
            seen = torch.arange(m) < (pos + 1 if causal else m)
            if hide is not None:
                seen &= ~hide[b][:m]
            j = torch.arange(m)[seen].double()
            if not len(j):
                continue
            x = q[b, :, n].double().cpu()
            s = (k[:, seen] * x[:, None]).sum(-1) * scale
            size = (k[:, seen] * x[:, None]).abs().sum(-1) * scale
            if f is not None:
                pq = phi_q[0 if phi_q.shape[0] == 1 else b, :, n].double().cpu()
                s = s + (f[:, seen] * pq[:, None]).sum(-1)
                size = size + (f[:, seen] * pq[:, None]).abs().sum(-1)
            if slopes is not None:
                bias = -slopes.double().cpu()[:, None] * (pos - j)
                s, size = s + bias, size + bias.abs()
            lse[b, :, n] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            out[b, :, n] = (p[..., None] * v[:, seen]).sum(1)
            # Scores: C products and sums, the factors and the exponent's argument in fp32, each within 2^-24 of the sum of
            # magnitudes; rows and sums over the keys: one rounding a key at most; probabilities in bf16: two limbs, 2^-16.
            ds = (C + 80) * 2.0 ** -24 * size.amax(-1)
            dp = 2 * ds + (len(j) + 16) * 2.0 ** -23 + (2.0 ** -16 if low else 0)
            tol_o[b, :, n] = dp[:, None] * (p[..., None] * v[:, seen].abs()).sum(1) * 2
            tol_l[b, :, n] = dp + (lse[b, :, n].abs() + 1) * 2.0 ** -22
    tol_o += out.abs() * HALF[q.dtype]
    return out, lse, tol_o, tol_l


def check_attend(got, ref):
    """Every value within its bound; rows that see nothing are exactly out 0, lse -inf."""
    (o, l), (ro, rl, to, tl) = got, ref
    o, l = o.double().cpu(), l.double().cpu()
    empty = rl == -math.inf
    assert torch.equal(l == -math.inf, empty)
    assert (o[empty] == 0).all()
    over = ((o - ro).abs() / to).amax().item()
    over_l = ((l - rl).abs() / tl)[~empty].amax().item() if (~empty).any() else 0.0
    print(f"[paged] out at {over:.3f}, lse at {over_l:.3f} of the bound", flush=True)
    assert over <= 1 and over_l <= 1          # (a NaN fails both)


def plan_reference(lens, want, table, ring, state, N, page):
    """The pages' bookkeeping, request after request, on copies."""
    lens, want, table, ring = (np.array(x, dtype=np.int64) for x in (lens, want, table, ring))
    head, count = int(state[0]) % len(ring), int(state[1])
    n, cap = len(ring), table.shape[1] * page
    goal = []
    for o, w in zip(lens, want):
        o, w = max(int(o), 0), max(int(w), 0)
        goal.append(o if w > cap or w - o > N else w)
    for b, w in enumerate(goal):
        for j in range(-(-w // page), -(-max(int(lens[b]), 0) // page)):
            ring[(head + count) % n] = table[b, j]
            count += 1
    slots = np.full((len(lens), N), -1)
    pos = np.zeros((len(lens), N), np.int64)
    asked, avail, taken = 0, count, 0
    for b, w in enumerate(goal):
        o = max(int(lens[b]), 0)
        first, need = -(-o // page), -(-w // page) - -(-o // page)
        if need > 0:
            asked += need
            if asked > avail:
                goal[b] = w = o
            else:
                for j in range(need):
                    table[b, first + j] = ring[(head + taken + j) % n]
                taken += need
        for i in range(max(w - o, 0)):
            pos[b, i] = o + i
            slots[b, i] = table[b, (o + i) // page] * page + (o + i) % page
    return table, ring, np.array(goal), np.array([(head + taken) % n, avail - taken]), slots, pos
