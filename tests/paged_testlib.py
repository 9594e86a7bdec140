"""Plain implementations, in 64 bits or whole numbers, of the token-level cache's operators, and caches to try them on."""
from __future__ import annotations

import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


# ------------------------------------------------------------------------------------------------ page plan
def plan(lens, new, tables, ring, head, count, page, max_tokens):
    """One request after the other, as include/wk.h says it.  Lists in, a dict of lists out (tables and ring are copies)."""
    n_pages, max_pages = len(ring), len(tables[0])
    tables, ring, lens = [list(t) for t in tables], list(ring), list(lens)
    up = lambda v: -(-v // page) if v > 0 else 0  # noqa: E731
    slots, starts, rows, asked, taken, full, bad = [-1] * max_tokens, [], 0, 0, 0, False, False
    if not (0 <= head < n_pages and 0 <= count <= n_pages):
        head = count = 0
        bad = True
    ended = []
    for r, (have, n) in enumerate(zip(list(lens), new)):
        starts.append(rows)
        if n < 0:
            if have >= 0:
                ended.append((r, have))
                lens[r] = 0
            continue
        if n == 0:
            continue
        first, rows = rows, rows + n
        if have < 0 or up(have + n) > max_pages or rows > max_tokens:
            full = True
            continue
        need = up(have + n) - up(have)
        asked += need
        if need and asked > count:
            full = True
            continue
        for i in range(need):
            tables[r][up(have) + i] = ring[(head + taken + i) % n_pages]
        taken += need
        for j in range(n):
            pos = have + j
            ident = tables[r][pos // page]
            if 0 <= ident < n_pages:
                slots[first + j] = ident * page + pos % page
            else:
                bad = True
        lens[r] = have + n
    back = []
    for r, have in ended:
        for ident in tables[r][:min(up(have), max_pages)]:
            if 0 <= ident < n_pages:
                back.append(ident)
            elif ident != -1:
                bad = True
    if len(back) > n_pages - count:
        bad, back = True, back[:n_pages - count]
    for k, ident in enumerate(back):
        ring[(head + count + k) % n_pages] = ident
    return dict(slots=slots, starts=starts + [rows], lens=lens, tables=tables, ring=ring,
                state=[(head + taken) % n_pages, count - taken + len(back), 0, 0], full=full, bad=bad)


# ------------------------------------------------------------------------------------------------ rows in 8 bits
CODES = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()     # 0 .. 448, ascending


def quantise(x: torch.Tensor):
    """(codes as values in 64 bits, NaN where x is not finite; exponent bytes) of rows along the last axis."""
    x = x.double().cpu()
    fine = torch.isfinite(x)
    top = torch.where(fine, x, 0.0).abs().amax(-1)
    e = torch.zeros(top.shape, dtype=torch.int64)
    for i in range(top.numel()):
        t = top.view(-1)[i].item()
        if t:
            k = math.frexp(t)[1] - 12                       # surely too small an exponent, or the least
            while t > 448.0 * 2.0 ** max(k, -126):
                k += 1
            e.view(-1)[i] = min(max(k, -126), 127)
    y = torch.where(fine, x, 0.0) / torch.pow(2.0, e.double())[..., None]
    mag = y.abs()
    hi = torch.searchsorted(CODES, mag).clamp(max=126)      # first code that is at least as large
    lo = (hi - 1).clamp(min=0)
    up, down = CODES[hi] - mag, mag - CODES[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    value = torch.copysign(CODES[pick], y)
    return torch.where(fine, value, math.nan), (e + 127).to(torch.uint8)


# ------------------------------------------------------------------------------------------------ attention
def visible(n, window, sink):
    return [t for t in range(n) if not window or t < sink or t >= n - window]


def attend(Q, K, V, K_exp, V_exp, tables, lens, window=0, sink=0, scale=0.0):
    """O, lse in 64 bits and, beside them, a bound of what the kernel's O and lse may be off by.

    K, V [n_pages, page, kv_heads, d].  With u the half step of the type that weights are rounded to before they meet V, a
    weight's relative error is u + 2 * dlogit + 2^-22 (exponential) and a sum's over n values n * 2^-23; the weights below the normal numbers
    of fp16 (V in fp16 or 8 bits) are off by 2^-25 of the largest instead.  A logit's error is d products summed in 32 bits,
    each step off by 2^-23 of the sum of magnitudes, and its scaling.  O is rounded once more.
    """
    dev = Q.device
    B, H, d = Q.shape
    page, Hk = K.shape[1], K.shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    O = torch.zeros((B, H, d), dtype=torch.float64, device=dev)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=dev)
    O_tol, lse_tol = torch.zeros_like(O), torch.zeros_like(lse)
    e4m3 = K.dtype == torch.float8_e4m3fn
    half = K.dtype != torch.bfloat16
    u_w = 2.0 ** -11 if half else 2.0 ** -8
    for b in range(B):
        n = min(int(lens[b]), tables.shape[1] * page)
        if n <= 0:
            continue
        pos = torch.tensor(visible(n, window, sink), device=dev)
        ids = tables[b].long()[pos // page]
        there = (ids >= 0) & (ids < K.shape[0])
        ids, off = ids[there], (pos % page)[there]
        if ids.numel() == 0:
            continue
        k, v = K[ids, off].double(), V[ids, off].double()                         # [n, Hk, d]
        codes = v.abs().amax(0)                                                   # largest code of every column
        ve = torch.ones(v.shape[:2], dtype=torch.float64, device=dev)
        if e4m3:
            k = k * torch.pow(2.0, K_exp.transpose(1, 2)[ids, off].double() - 127)[..., None]
            ve = torch.pow(2.0, V_exp.transpose(1, 2)[ids, off].double() - 127)
            v = v * ve[..., None]
        q = Q[b].double().view(Hk, H // Hk, d)
        logits = torch.einsum("hgd,nhd->hgn", q, k) * scale
        mags = torch.einsum("hgd,nhd->hgn", q.abs(), k.abs()).amax(-1) * scale
        top = logits.amax(-1, keepdim=True)
        w = torch.where(top == -math.inf, 0.0, torch.exp(logits - top))
        total = w.sum(-1, keepdim=True)
        some = total.squeeze(-1) != 0
        p = torch.where(some[..., None], w / total, 0.0)
        o = torch.einsum("hgn,nhd->hgd", p, v)
        m = len(ids)
        dl = (d + 4) * 2.0 ** -23 * mags + 2.0 ** -22 * logits.abs().amax(-1)
        sums = (m + 16) * 2.0 ** -23
        size = torch.einsum("hgn,nhd->hgd", p, v.abs())
        tol = (u_w + 2 * dl[..., None] + 2.0 ** -22 + 2 * sums) * size
        if half:
            # lost below 2^-14 of the largest weight (with its row's power of two), times the largest code
            biggest = (p * ve.t()[:, None]).amax(-1)
            tol = tol + m * 2.0 ** -25 * biggest[..., None] * codes[:, None]
        tol = torch.where(some[..., None], tol, 0.0)               # a row without any weight is zero, exactly
        O[b] = o.reshape(H, d)
        O_tol[b] = (tol + HALF_STEP[Q.dtype] * (o.abs() + tol) + 2.0 ** -25).reshape(H, d)
        l = torch.where(some, top.squeeze(-1) + torch.log(total.squeeze(-1)), -math.inf)
        lse[b] = l.reshape(H)
        lse_tol[b] = (dl + sums + 2.0 ** -21 + l.abs().nan_to_num(0, 0, 0) * 2.0 ** -22).reshape(H)
    return O, lse, O_tol, lse_tol


def assert_attends(got, lse, ref):
    O, l, O_tol, l_tol = ref
    g = got.double()
    assert torch.equal(g.isnan(), O.isnan()) and torch.equal(lse.isnan(), l.isnan())
    fine = torch.isfinite(O)
    assert torch.equal(g[O.isinf()], O[O.isinf()])
    over = ((g - O).abs() - O_tol)[fine]
    assert over.numel() == 0 or over.max().item() <= 0, f"O is off by {((g - O).abs() / O_tol)[fine].max().item():.3g} of its bound"
    finite = torch.isfinite(l)
    assert torch.equal(torch.isfinite(lse), finite) and torch.equal(lse.double()[~finite & ~l.isnan()], l[~finite & ~l.isnan()])
    over = ((lse.double() - l).abs() - l_tol)[finite]
    assert over.numel() == 0 or over.max().item() <= 0, f"lse is off by {((lse.double() - l).abs() / l_tol)[finite].max().item():.3g} of its bound"


# ------------------------------------------------------------------------------------------------ caches
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


def cache(type_, n_pages, page, kv_heads, d, seed=0, layout="tokens", device="cuda"):
    """K, V, K_exp, V_exp filled with normals (rows of different size in 8 bits), in one of several layouts."""
    g = torch.Generator(device=device).manual_seed(seed)
    dt = TYPES[type_]
    shape = (n_pages, page, kv_heads, d)
    if layout == "tokens":
        pair = [torch.empty(shape, dtype=dt, device=device) for _ in range(2)]
    elif layout == "heads":                       # heads outside tokens
        pair = [torch.empty((n_pages, kv_heads, page, d), dtype=dt, device=device).transpose(1, 2) for _ in range(2)]
    elif layout == "paired":                      # K and V of a page side by side, rows wider than a head
        both = torch.empty((n_pages, 2, page, kv_heads, d + 32), dtype=dt, device=device)
        both.view(torch.uint8).fill_(0x7f)
        pair = [both[:, i, :, :, :d] for i in range(2)]
    exps = []
    for x in pair:
        val = torch.randn(shape, generator=g, device=device)
        if type_ == "e4m3":
            x.copy_((val * 100).to(dt))
            exps.append(torch.randint(115, 125, (n_pages, kv_heads, page), generator=g, device=device).to(torch.uint8))
        else:
            x.copy_(val.to(dt))
            exps.append(None)
    return pair[0], pair[1], exps[0], exps[1]


def tables_for(lens, page, n_pages, max_pages, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randperm(n_pages, generator=g).int()
    t = torch.full((len(lens), max_pages), 10 ** 9, dtype=torch.int32)      # places that must not be looked at
    at = 0
    for r, n in enumerate(lens):
        have = -(-n // page) if n > 0 else 0
        t[r, :have] = ids[at:at + have]
        at += have
    assert at <= n_pages
    return t.to(device)


def poison(K, V, K_exp, V_exp, tables, lens, window=0, sink=0):
    """Everything that no request may look at becomes NaN (exponents of 2^128)."""
    keep = torch.zeros(K.shape[:2], dtype=torch.bool)
    page = K.shape[1]
    for b, n in enumerate(lens):
        for t in visible(min(max(n, 0), tables.shape[1] * page), window, sink):
            ident = int(tables[b, t // page])
            if 0 <= ident < K.shape[0]:
                keep[ident, t % page] = True
    keep = keep.to(K.device)
    for x in (K, V):
        if x.dtype == torch.float8_e4m3fn:
            x.view(torch.uint8)[~keep] = 0x7f
        else:
            x[~keep] = math.nan
    for e in (K_exp, V_exp):
        if e is not None:
            e.transpose(1, 2)[~keep] = 255
