"""Operators of a serving and training step around the attention kernels: rotary positions, the pages of a key-value
cache, and attention of new tokens over those pages.

A case is a dict of plain values; "op" says which operator it runs:

    "rotary"  turns channel pairs of q and k by position times frequency, one to three axes; step "train" runs the
              backward too
    "plan"    gives and takes cache pages as requests grow, shrink and end, and maps new tokens to cache slots
    "append"  stores the new tokens' keys, values and bias factors into their pages
    "attend"  softmax attention of a few new tokens per request over its pages, grouped heads, requests of their own
              lengths, bias by low-rank factors, ALiBi slopes or none

`own` chooses between the plain form of each operator (elementary torch operations) and the library's kernels.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


def _dt(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _rotary(step, B, N, H, Hkv, C, sections, far=1, dtype="bf16", interleaved=False, fused=True, shared=False):
    s = list(sections) + [0] * (3 - len(sections))
    return {"op": "rotary", "step": step, "B": B, "N": N, "H": H, "Hkv": Hkv, "C": C, "s0": s[0], "s1": s[1], "s2": s[2],
            "far": far, "dtype": dtype, "interleaved": interleaved, "fused": fused, "shared": shared}


def _plan(B, N, page, hi, spare):
    return {"op": "plan", "B": B, "N": N, "page": page, "hi": hi, "spare": spare}


def _append(B, N, Hkv, C, R, page, dtype="bf16", phi="f32", fused=True):
    return {"op": "append", "B": B, "N": N, "Hkv": Hkv, "C": C, "R": R, "page": page, "dtype": dtype, "phi": phi, "fused": fused}


def _attend(B, N, H, Hkv, C, page, lo, hi, bias="none", R=0, dtype="bf16", phi="f32", causal=True):
    return {"op": "attend", "B": B, "N": N, "H": H, "Hkv": Hkv, "C": C, "page": page, "lo": lo, "hi": hi, "bias": bias, "R": R,
            "dtype": dtype, "phi": phi, "causal": causal}


def listed():
    cases = {
        # the new tokens' queries and keys of a decoder in a long conversation: latency of one small call
        "rotary_token": _rotary("infer", 8, 1, 16, 4, 128, (64,), far=100000),
        # a vision model's training step, positions on a 32 x 32 grid
        "rotary_grid_train": _rotary("train", 8, 1024, 12, 12, 64, (16, 16), shared=True),
        # prompts of text, images and video (time, height, width) read at once, from the fused projection
        "rotary_video": _rotary("infer", 4, 16384, 16, 4, 128, (16, 24, 24), far=1000),
        # a decoder's step: each running request gets one more token, some end, some start
        "plan_token": _plan(64, 1, 16, 4096, 1.0),
        # a batch of prompts is admitted, more than there are pages for
        "plan_prompts": _plan(256, 4096, 16, 4096, 0.6),
        # one token of each request into the cache, with the rank-2 factors of its position
        "append_token": _append(64, 1, 8, 128, 2, 16),
        # prompts into the cache, read from the fused projection
        "append_prompts": _append(8, 4000, 16, 128, 0, 32),
        # one short request: latency
        "attend_one": _attend(1, 1, 16, 16, 128, 16, 300, 300, "alibi"),
        # the ALiBi decoder's next token for a batch of cached sequences about 4096 long
        "attend_alibi": _attend(8, 1, 16, 16, 128, 16, 2100, 8200, "alibi"),
        # grouped heads, a full batch of ragged conversations: the largest call
        "attend_grouped": _attend(32, 1, 32, 8, 128, 64, 500, 16384, "factors", 4),
        # a few drafted tokens are checked at once, in full precision
        "attend_draft_fp32": _attend(4, 5, 8, 4, 64, 32, 700, 5001, "factors", 8, "f32"),
        # decoder tokens look at the states of an encoder (no causal mask), one of odd length each
        "attend_encoder": _attend(48, 3, 12, 12, 64, 16, 1, 1500, "factors", 16, phi="bf16", causal=False),
    }
    return [dict(c, name=n) for n, c in cases.items()]


# ---- sizes ---------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _sections(rng, pairs):
    axes = rng.choice((1, 2, 3))
    if axes == 1 or pairs < 8:
        return (pairs if rng.random() < 0.7 else max(1, pairs // 2),)
    cuts = sorted(rng.sample(range(1, pairs), axes - 1))
    return tuple(b - a for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    op = rng.choice(("rotary", "rotary", "plan", "append", "attend", "attend", "attend", "attend"))
    H, G = rng.choice(((4, 1), (8, 1), (12, 1), (16, 1), (8, 2), (16, 4), (32, 4), (32, 8), (24, 3), (12, 6), (20, 5)))
    Hkv = H // G
    C = rng.choice((16, 32, 64, 64, 128, 128))
    page = rng.choice((16, 16, 32, 64, 128, 256))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "rotary":
        N = rng.choice((1, _log(rng, 2, 32768)))
        most = 4 * 16384 * 20 * 128 // (2 if dtype == "f32" else 1)
        B = _log(rng, 1, max(1, min(256, most // (N * (H + Hkv) * C * 3))))
        return _rotary(rng.choice(("infer", "infer", "train")), B, N, H, Hkv, C, _sections(rng, C // 2),
                       far=rng.choice((1, 1000, 100000)), dtype=dtype, interleaved=rng.random() < 0.3,
                       fused=rng.random() < 0.6, shared=rng.random() < 0.3)
    if op == "plan":
        N = rng.choice((1, 1, 4, _log(rng, 16, 4096)))
        B = _log(rng, 1, 1024)
        while B * N > 1 << 20:
            B //= 2
        return _plan(B, N, page, _log(rng, max(16, N), 8192), rng.choice((0.3, 0.9, 1.0, 1.5)))
    if op == "append":
        N = rng.choice((1, 1, _log(rng, 2, 4096)))
        B = _log(rng, 1, 256)
        while B * N * Hkv * C * (4 if dtype == "f32" else 2) > 8 * 4000 * 16 * 128 * 2:
            B = max(1, B // 2)
            N = N if B > 1 else N // 2
        return _append(B, N, Hkv, C, rng.choice((0, 2, 5, 16)), page, dtype, "f32" if dtype == "f32" else rng.choice(("f32", "bf16")),
                       fused=rng.random() < 0.6)
    bias = rng.choice(("none", "factors", "alibi"))
    phi = "f32" if dtype == "f32" else rng.choice(("f32", "bf16"))
    R = rng.choice((1, 2, 5, 8, 16)) if bias == "factors" else 0
    B, hi = _log(rng, 1, 128), _log(rng, 32, 32768)
    N, least, causal = rng.choice((1, 1, 1, 2, 3, 4, 5, 8, 16)), rng.choice((0, 1 / 8, 1)), rng.random() < 0.7
    while True:
        c = _attend(B, N, H, Hkv, C, page, int(hi * least), hi, bias, R, dtype, phi, causal)
        if _cost(c) <= _cost(next(x for x in listed() if x["name"] == "attend_grouped")):
            return c
        B, hi = (B // 2, hi) if B > 1 else (1, hi // 2)


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 16


# ---- inputs --------------------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n lengths from lo to hi, most of them short; the same ones for every seed."""
    i = (np.arange(n) + 0.5) / n if n > 1 else np.ones(1)
    return np.round(lo + (hi - lo) * i * i).astype(np.int64)


def _pairs(case):
    return [s for s in (case["s0"], case["s1"], case["s2"]) if s]


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _rand(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _prepare_rotary(c, g, rng):
    B, N, H, Hkv, C = c["B"], c["N"], c["H"], c["Hkv"], c["C"]
    dt, sections = _dt(c["dtype"]), _pairs(c)
    if c["fused"]:           # q, k and v as one projection leaves them: [B, N, H + 2 Hkv, C]
        x = _rand(g, (B, N, H + 2 * Hkv, C), dt)
        q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2)
    else:
        q, k = _rand(g, (B, H, N, C), dt), _rand(g, (B, Hkv, N, C), dt)
    bp = 1 if c["shared"] else B
    first = rng.integers(0, c["far"], (1, bp, 1))
    if len(sections) == 1:
        pos = first + np.arange(N)[None, None, :]
    else:                    # a grid: rows and columns (and frames) of the token's place
        w = max(1, int(math.isqrt(N)))
        t = np.broadcast_to(np.arange(N), (bp, N))
        pos = np.stack([first[0] + t // (w * w), t // w % w, t % w] if len(sections) == 3 else [first[0] + t // w, t % w])
    freqs = np.concatenate([10000.0 ** (-np.arange(s) / s) for s in sections]) if len(sections) == 2 else \
        10000.0 ** (-np.arange(sum(sections)) / sum(sections))
    s = {"q": q, "k": k, "pos": _i32(pos), "freqs": torch.from_numpy(freqs.astype(np.float32)).cuda(), "sections": sections}
    if c["step"] == "train":
        s["q"], s["k"] = q.detach().requires_grad_(), k.detach().requires_grad_()
        s["dq"], s["dk"] = _rand(g, (B, H, N, C), dt), _rand(g, (B, Hkv, N, C), dt)
    return s


def _prepare_plan(c, g, rng):
    B, N, page, hi = c["B"], c["N"], c["page"], c["hi"]
    max_blocks = -(-(hi + N) // page)
    lens = rng.permutation(_spread(1, hi, B))
    if N > 16:               # prompts: most places are empty before
        lens[rng.random(B) < 0.7] = 0
    want = lens + (1 if N == 1 else rng.integers(0, N + 1, B))
    kind = rng.random(B)
    want[kind < 0.1] = 0                                        # ended
    back = (kind >= 0.1) & (kind < 0.15)
    want[back] = np.maximum(lens[back] - rng.integers(0, 9, int(back.sum())), 0)      # drafted tokens that are not kept
    used = -(-lens // page)
    grow = np.maximum(-(-want // page) - used, 0).sum()
    n_pages = int((-(-_spread(1, hi, B) // page)).sum()) + int(c["spare"] * B * -(-N // page)) + 8
    n_free = min(int(grow * c["spare"]), n_pages - int(used.sum()))
    pages = rng.permutation(n_pages)
    table = np.full((B, max_blocks), -1)
    table[np.arange(max_blocks)[None, :] < used[:, None]] = pages[:used.sum()]
    head = int(rng.integers(0, n_pages))
    ring = np.zeros(n_pages)
    ring[(head + np.arange(n_free)) % n_pages] = pages[used.sum():used.sum() + n_free]
    return {"lens": _i32(lens), "want": _i32(want), "table": _i32(table), "ring": _i32(ring), "state": _i32([head, n_free])}


def _prepare_append(c, g, rng):
    B, N, Hkv, C, R, page = (c[n] for n in ("B", "N", "Hkv", "C", "R", "page"))
    dt, pdt = _dt(c["dtype"]), _dt(c["phi"])
    new = rng.permutation(np.maximum(N - (np.arange(B) % 4) * (N // 8), 0))       # ragged prompts
    if N == 1 and B > 8:
        new[:B // 16] = 0                                                        # requests that wait
    start = rng.integers(0, 4 * page, B)
    blocks = -(-(start + new) // page)
    n_pages = B * -(-(N + 4 * page) // page)
    pages = rng.permutation(n_pages)
    at = np.concatenate([[0], np.cumsum(blocks)])[:-1]
    p = start[:, None] + np.arange(N)[None, :]
    slots = np.where(np.arange(N)[None, :] < new[:, None], pages[np.minimum(at[:, None] + p // page, n_pages - 1)] * page + p % page, -1)
    if c["fused"]:
        x = _rand(g, (B, N, 2 * Hkv, C), dt)
        k, v = x[:, :, :Hkv].transpose(1, 2), x[:, :, Hkv:].transpose(1, 2)
    else:
        k, v = _rand(g, (B, Hkv, N, C), dt), _rand(g, (B, Hkv, N, C), dt)
    s = {"k": k, "v": v, "slots": _i32(slots), "phi_k": None, "phi_pages": None,
         "k_pages": _rand(g, (n_pages, Hkv, page, C), dt), "v_pages": _rand(g, (n_pages, Hkv, page, C), dt)}
    if R:
        s["phi_k"], s["phi_pages"] = _rand(g, (B, Hkv, N, R), pdt), _rand(g, (n_pages, Hkv, page, R), pdt)
    return s


def _prepare_attend(c, g, rng):
    B, N, H, Hkv, C, R, page = (c[n] for n in ("B", "N", "H", "Hkv", "C", "R", "page"))
    dt, pdt = _dt(c["dtype"]), _dt(c["phi"])
    lens = rng.permutation(_spread(c["lo"], c["hi"], B))
    used = -(-lens // page)
    n_pages = int(used.sum()) + 3
    table = np.full((B, max(1, int(used.max()))), -1)
    table[np.arange(table.shape[1])[None, :] < used[:, None]] = rng.permutation(n_pages)[:used.sum()]
    new = np.minimum(np.maximum(N - (np.arange(B) % 3 == 1), 1), lens)            # some requests have a token fewer
    s = {"q": _rand(g, (B, H, N, C), dt), "k_pages": _rand(g, (n_pages, Hkv, page, C), dt),
         "v_pages": _rand(g, (n_pages, Hkv, page, C), dt), "table": _i32(table), "lens": _i32(lens), "starts": _i32(lens - new),
         "phi_q": None, "phi_pages": None, "slopes": None, "causal": c["causal"]}
    if c["bias"] == "factors":
        s["phi_q"] = _rand(g, (B, H, N, R), pdt, R ** -0.25)
        s["phi_pages"] = _rand(g, (n_pages, Hkv, page, R), pdt, R ** -0.25)
    elif c["bias"] == "alibi":
        s["slopes"] = torch.from_numpy((2.0 ** (-8.0 * (np.arange(H) + 1.0) / H)).astype(np.float32)).cuda()
    return s


_PREPARE = {"rotary": _prepare_rotary, "plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    s = _PREPARE[case["op"]](case, g, np.random.default_rng([int(seed), 5]))
    s["case"] = dict(case)
    return s


# ---- plain forms ---------------------------------------------------------------------------------
def _turn(x, cos, sin, pairs, interleaved):
    x1 = x[..., 0:2 * pairs:2] if interleaved else x[..., :pairs]
    x2 = x[..., 1:2 * pairs:2] if interleaved else x[..., pairs:2 * pairs]
    x1, x2 = x1.float(), x2.float()
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack((y1, y2), -1).flatten(-2) if interleaved else torch.cat((y1, y2), -1)
    return torch.cat((y.to(x.dtype), x[..., 2 * pairs:]), -1)


def _rotary_plain(s):
    with torch.no_grad():
        c = s["case"]
        pairs = s["freqs"].numel()
        axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device="cuda"),
                                       torch.tensor(s["sections"], device="cuda"), output_size=pairs)
        angle = s["pos"].double()[axis].permute(1, 2, 0) * s["freqs"].double()       # far positions lose their angle in 32 bits
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        out = [_turn(s[n], cos, sin, pairs, c["interleaved"]) for n in ("q", "k")]
        if c["step"] == "train":
            out += [_turn(s[n], cos, -sin, pairs, c["interleaved"]) for n in ("dq", "dk")]
        return out


def _plan_plain(s):
    N, page, table, ring = s["case"]["N"], s["case"]["page"], s["table"], s["ring"]
    B, width = table.shape
    n = ring.numel()
    lens, want = s["lens"].long().clamp(min=0), s["want"].long().clamp(min=0)
    head, count = s["state"].long().unbind()
    want = torch.where((want > width * page) | (want - lens > N), lens, want)
    used, goal = (lens + page - 1) // page, (want + page - 1) // page
    freed, need = (used - goal).clamp(min=0), (goal - used).clamp(min=0)
    free_end, need_end = freed.cumsum(0), need.cumsum(0)
    avail = count + free_end[-1]
    granted = (need == 0) | (need_end <= avail)
    want = torch.where(granted, want, lens)
    need_at, taken = need_end - need, torch.where(granted, need, 0).sum()
    # freed pages go behind the ring's last one, request after request
    block = torch.arange(width, device="cuda")
    goes = (block >= goal[:, None]) & (block < used[:, None])
    place = (head + count + (free_end - freed)[:, None] + block - goal[:, None]) % n
    ring[place[goes]] = table[goes]
    # pages taken, in the order of the requests
    comes = (block >= used[:, None]) & (block < goal[:, None]) & granted[:, None]
    place = (head + need_at[:, None] + block - used[:, None]) % n
    table[comes] = ring[place[comes]]
    i = torch.arange(N, device="cuda")
    pos = lens[:, None] + i
    valid = i < (want - lens)[:, None]
    page_of = table.gather(1, torch.where(valid, pos // page, 0)).long()
    slots = torch.where(valid, page_of * page + pos % page, -1).int()
    state = torch.stack(((head + taken) % n, avail - taken)).int()
    return [table, ring, want.int(), state, slots, torch.where(valid, pos, 0).int()]


def _append_plain(s):
    slots, page = s["slots"].flatten().long(), s["case"]["page"]
    valid = slots >= 0
    to, row = slots[valid] // page, slots[valid] % page
    for new, pages in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"]), (s["phi_k"], s["phi_pages"])):
        if new is not None:
            pages[to, :, row] = new.permute(0, 2, 1, 3).flatten(0, 1)[valid]
    return [s["k_pages"], s["v_pages"], s["phi_pages"]]


def _attend_plain(s):
    c, table = s["case"], s["table"]
    B, H, N, C = s["q"].shape
    Hkv, page = s["k_pages"].shape[1:3]
    M, G = table.shape[1] * page, H // Hkv
    at = table.clamp(min=0).long()

    def rows(pages):         # [B, Hkv, M, *] of the pages in the order of the keys
        return pages[at].transpose(1, 2).flatten(2, 3).float()

    key = torch.arange(M, device="cuda")
    present = key < s["lens"][:, None]                                              # [B, M]
    pos = s["starts"][:, None] + torch.arange(N, device="cuda")                     # [B, N]
    seen = present[:, None].expand(B, N, M)
    if c["causal"]:
        seen = seen & (key <= pos[..., None]) & (pos < s["lens"][:, None])[..., None]
    score = torch.matmul(s["q"].float().reshape(B, Hkv, G * N, C), rows(s["k_pages"]).transpose(2, 3)) * C ** -0.5
    if s["phi_q"] is not None:
        R = s["phi_q"].shape[-1]
        score += torch.matmul(s["phi_q"].float().reshape(B, Hkv, G * N, R), rows(s["phi_pages"]).transpose(2, 3))
    score = score.reshape(B, H, N, M)
    if s["slopes"] is not None:
        score -= s["slopes"][:, None, None] * (pos[..., None] - key).float()[:, None]
    score = torch.where(seen[:, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(present[:, None, :, None], rows(s["v_pages"]), 0.0)             # rows behind the last key may hold anything
    out = torch.matmul(p.reshape(B, Hkv, G * N, M), v).reshape(B, H, N, C)
    out = torch.where(total > 0, out / total, 0.0).to(s["q"].dtype)
    return [out, (top + total.log())[..., 0]]


_PLAIN = {"rotary": _rotary_plain, "plan": _plan_plain, "append": _append_plain, "attend": _attend_plain}


# ---- the library's calls -------------------------------------------------------------------------
def _rotary_own(s):
    from paper_2505_12044_amd import api, autograd
    c = s["case"]
    if c["step"] == "infer":
        return list(api.fb_rotary_fwd(s["q"], s["k"], s["pos"], s["freqs"], s["sections"], interleaved=c["interleaved"]))
    yq, yk = autograd.rotary_positions(s["q"], s["k"], s["pos"], s["freqs"], s["sections"], interleaved=c["interleaved"])
    return [yq, yk, *torch.autograd.grad((yq, yk), (s["q"], s["k"]), (s["dq"], s["dk"]))]


def _plan_own(s):
    from paper_2505_12044_amd import api
    c = s["case"]
    return [s["table"], s["ring"], *api.fb_paged_plan(s["lens"], s["want"], s["table"], s["ring"], s["state"], c["N"], c["page"])]


def _append_own(s):
    from paper_2505_12044_amd import api
    api.fb_paged_append(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["phi_k"], s["phi_pages"])
    return [s["k_pages"], s["v_pages"], s["phi_pages"]]


def _attend_own(s):
    from paper_2505_12044_amd import api
    return list(api.fb_paged_attn_fwd(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["starts"], s["phi_q"],
                                      s["phi_pages"], s["slopes"], causal=s["causal"]))


_OWN = {"rotary": _rotary_own, "plan": _plan_own, "append": _append_own, "attend": _attend_own}


def run(state):
    op = state["case"]["op"]
    return _OWN[op](state) if own else _PLAIN[op](state)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    B, N = case["B"], case["N"]
    size = 4 if case.get("dtype") == "f32" else 2
    psize = 4 if case.get("phi") == "f32" else 2
    if case["op"] == "rotary":
        passes = 2 if case["step"] == "train" else 1
        elements = B * N * (case["H"] + case["Hkv"]) * case["C"]
        sections = _pairs(case)
        small = 4 * (len(sections) * (1 if case["shared"] else B) * N + sum(sections))
        return {"bytes": passes * (2 * elements * size + small),
                "flops": passes * 6 * B * N * (case["H"] + case["Hkv"]) * sum(sections)}
    if case["op"] == "plan":
        return {"bytes": 4 * (3 * B + 4) + 8 * B * N, "flops": 4 * B * N}
    if case["op"] == "append":
        tokens = int(np.maximum(N - (np.arange(B) % 4) * (N // 8), 0).sum()) - (B // 16 if N == 1 and B > 8 else 0)
        return {"bytes": 4 * B * N + 2 * tokens * case["Hkv"] * (2 * case["C"] * size + case["R"] * psize), "flops": 0}
    keys = int(_spread(case["lo"], case["hi"], B).sum())
    row = 2 * case["C"] * size + case["R"] * psize
    q = B * case["H"] * N * row + 4 * B * case["H"] * N
    return {"bytes": keys * case["Hkv"] * row + q + 4 * (-(-keys // case["page"]) + 2 * B),
            "flops": keys * case["H"] * N * (4 * case["C"] + 2 * case["R"] + 4)}


# ---- the definition in 64 bits -------------------------------------------------------------------
def _rotary_exact(c, s):
    pairs, start, out = sum(s["sections"]), 0, []
    turned = []
    for a, n in enumerate(s["sections"]):
        turned.append(s["pos"][a].double()[..., None] * s["freqs"][start:start + n].double())
        start += n
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.cat(turned, -1))[:, None]
    for name in ("q", "k", "dq", "dk"):
        if name in s:
            x = s[name].detach().double()
            first = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if c["interleaved"] else (slice(0, pairs), slice(pairs, 2 * pairs))
            z = torch.complex(x[..., first[0]], x[..., first[1]]) * (turn if name in ("q", "k") else turn.conj())
            y = x.clone(memory_format=torch.contiguous_format)
            y[..., first[0]], y[..., first[1]] = z.real, z.imag
            out.append(y)
    return out


def _plan_exact(c, s):
    N, page = c["N"], c["page"]
    table, ring, lens, want = (s[n].cpu().numpy().astype(np.int64) for n in ("table", "ring", "lens", "want"))
    head, count = s["state"].tolist()
    n, slots, pos = len(ring), np.full((len(lens), N), -1), np.zeros((len(lens), N), np.int64)
    goal = [int(o) if w > table.shape[1] * page or w - o > N else int(w) for o, w in zip(lens, want)]
    for b, (o, w) in enumerate(zip(lens, goal)):
        for j in range(-(-w // page), -(-int(o) // page)):
            ring[(head + count) % n] = table[b, j]
            count += 1
    full = False
    for b, (o, w) in enumerate(zip(lens, goal)):
        need = -(-w // page) - -(-int(o) // page)
        if need > 0:
            full = full or need > count
            if full:
                goal[b] = w = int(o)
            else:
                table[b, -(-int(o) // page):-(-w // page)] = ring[(head + np.arange(need)) % n]
                head, count = (head + need) % n, count - need
        if w > o:
            p = np.arange(int(o), w)
            slots[b, :w - o], pos[b, :w - o] = table[b, p // page] * page + p % page, p
    return [torch.from_numpy(np.asarray(x).astype(np.int32)) for x in (table, ring, goal, [head, count], slots, pos)]


def _append_exact(c, s):
    out = []
    place = s["slots"].cpu().numpy()
    for new, pages in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"]), (s["phi_k"], s["phi_pages"])):
        if new is None:
            out.append(None)
            continue
        y = pages.double().transpose(1, 2).flatten(0, 1).contiguous()          # [slots, Hkv, *]
        for b in range(len(place)):
            t = torch.from_numpy(np.flatnonzero(place[b] >= 0)).cuda()
            y.index_copy_(0, s["slots"][b].long()[t], new[b].double()[:, t].transpose(0, 1))
        out.append(y.unflatten(0, (pages.shape[0], pages.shape[2])).transpose(1, 2))
    return out


def _attend_exact(c, s):
    if _spread(c["lo"], c["hi"], c["B"]).sum() * c["H"] * c["N"] * c["C"] > 3e11:
        return None
    B, H, N, C = s["q"].shape
    Hkv, page = s["k_pages"].shape[1:3]
    out = torch.zeros((B, H, N, C), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, N), -math.inf, dtype=torch.float64, device="cuda")
    for b, (m, start) in enumerate(zip(s["lens"].tolist(), s["starts"].tolist())):
        pages = s["table"][b, :-(-m // page)].long()
        k, v, f = (None if s[n] is None else s[n][pages].transpose(0, 1).flatten(1, 2)[:, :m].double().repeat_interleave(H // Hkv, 0)
                   for n in ("k_pages", "v_pages", "phi_pages"))
        j = torch.arange(m, device="cuda", dtype=torch.float64)
        for i in range(N):
            last = min(m, start + i + 1) if c["causal"] else m
            if m == 0 or c["causal"] and start + i >= m:
                continue
            z = (k[:, :last] * s["q"][b, :, i, None].double()).sum(-1) / math.sqrt(C)
            if f is not None:
                z = z + (f[:, :last] * s["phi_q"][b, :, i, None].double()).sum(-1)
            if s["slopes"] is not None:
                z = z - s["slopes"].double()[:, None] * (start + i - j[:last])
            lse[b, :, i] = torch.logsumexp(z, -1)
            out[b, :, i] = (torch.softmax(z, -1)[..., None] * v[:, :last]).sum(1)
    return [out, lse]


_EXACT = {"rotary": _rotary_exact, "plan": _plan_exact, "append": _append_exact, "attend": _attend_exact}


def exact(case, seed):
    with torch.no_grad():
        return _EXACT[case["op"]](case, prepare(case, seed))
