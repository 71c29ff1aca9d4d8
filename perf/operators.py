"""The 4-bit KV cache and its pages, as cases that can be timed.

A cache page holds 128 key rows of every kv head in 4 bits per element (one step and one lowest value per row and
head), so a decoding step reads about a quarter of the bytes.  Three operators, through the public entry points of
paper_2402_11809_b200.binding:

  attn    space_kvq_attn_step: the block of a step ((k+1)^2 rows; k = 0: one new token) attends over the 4-bit cache
          and, where they are given, its own bf16 rows
  append  space_kvq_append and space_kvq_read: new rows are put into the cache (a prompt's, a token's, or the accepted
          ones of a step), and read back as the bf16 values that they stand for
  pages   space_pages_copy: the row moves that forked sequences (copy-on-write) and a compacted pool need, over the
          pools of several layers at once

The plain forms below use elementary torch operations in 32 bits on the same inputs.
"""
import math

import numpy as np
import torch

own = False

PAGE = 128            # rows of a page
BLOCK = 32            # rows that are laid out together


def block_bytes(d):
    return BLOCK * d + 8 * BLOCK                 # K and V codes, then {step, lowest} in bf16 of every K and V row


# ------------------------------------------------------------------------------------------------ cases

def _attn(name, B, heads, d, L, k, block=True):
    return dict(name=name, kind="attn", B=B, H_q=heads[0], H_kv=heads[1], d=d, L_lo=L[0], L_hi=L[1], k=k, block=block)


def _append(name, B, H_kv, d, n, L, step=1):
    return dict(name=name, kind="append", B=B, H_kv=H_kv, d=d, n_lo=n[0], n_hi=n[1], L_lo=L[0], L_hi=L[1], step=step)


def _pages(name, cache, H_kv, d, layers, pages, moves, rows):
    return dict(name=name, kind="pages", cache=cache, H_kv=H_kv, d=d, layers=layers, pages=pages, moves=moves,
                r_lo=rows[0], r_hi=rows[1])


def listed():
    return [
        # one new token of a short chat on a small model: launches and latency are all there is
        _attn("attn_tiny_token", 1, (8, 8), 64, (128, 128), 0),
        # the step of one user of a 7B-shaped model, 2k tokens in
        _attn("attn_llama7b", 1, (32, 32), 128, (2048, 2048), 5),
        # a server's batch of users at ragged lengths, a step each
        _attn("attn_ragged16", 16, (32, 32), 128, (512, 4096), 5),
        # a 70B-shaped model with grouped queries at long context: the products are large
        _attn("attn_gqa70b", 8, (64, 8), 128, (8192, 8192), 6),
        # odd sizes: few ragged sequences that end inside pages, head size 64
        _attn("attn_odd5", 5, (16, 8), 64, (37, 1999), 3),
        # a full batch of users that decode token by token, lengths up to 16k: the cache's bytes are the cost
        _attn("attn_tokens64", 64, (32, 8), 128, (1024, 16384), 0),
        # one document of 131071 tokens, the token's own row already in the cache
        _attn("attn_long_token", 1, (32, 8), 128, (131071, 131071), 0, block=False),
        # the rows that the steps of a batch have accepted: root and up to k = 4 candidates out of 25 block rows
        _append("append_accepted", 64, 8, 128, (5, 5), (1024, 16384), step=5),
        # a few prompts of odd lengths behind what is cached, head size 64
        _append("append_prompts", 5, 8, 64, (37, 1999), (0, 300)),
        # a batch of long prompts at once
        _append("append_long", 16, 32, 128, (512, 4096), (0, 0)),
        # sixteen samples forked from prompts that end inside a page: their last pages become their own, 8 layers
        _pages("pages_fork", "kvq", 8, 128, 8, 512, 16, (1, 127)),
        # a pool that is made compact: whole pages of the bf16 cache of 4 layers move down
        _pages("pages_compact", "bf16", 8, 128, 4, 4096, 700, (128, 128)),
    ]


MAX_ATTN_BYTES = 6.0e8        # the largest listed step reads about this much
MAX_ATTN_FLOPS = 1.0e11
MAX_APPEND_ROWS = 16 * 32 * 2304
MAX_MOVE_BYTES = 1.4e9


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "pages"])
    d = rng.choice([64, 128, 128])
    if kind == "attn":
        k = rng.choice([0, 0, 1, 2, 3, 4, 5, 6, 7])
        H_kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 32])
        G = rng.choice([g for g in (1, 1, 2, 4, 4, 8, 16) if g * H_kv <= 64])
        B = _log(rng, 1, 64)
        most = min(MAX_ATTN_BYTES / (B * H_kv * (d + 8)), MAX_ATTN_FLOPS / (4 * d * B * H_kv * G * (k + 1) ** 2), 131071)
        hi = _log(rng, 64, max(65, int(most)))
        lo = max(0, int(hi * rng.choice([0.0, 0.1, 0.5, 0.5, 1.0])))
        return dict(kind=kind, B=B, H_q=G * H_kv, H_kv=H_kv, d=d, L_lo=lo, L_hi=hi, k=k,
                    block=True if k else rng.random() < 0.5)
    if kind == "append":
        H_kv = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
        B = _log(rng, 1, 64)
        if rng.random() < 0.4:
            k = rng.randint(0, 7)
            return dict(kind=kind, B=B, H_kv=H_kv, d=d, n_lo=k + 1, n_hi=k + 1, L_lo=0, L_hi=_log(rng, 16, 16384), step=k + 1)
        hi = _log(rng, 1, max(1, min(8192, MAX_APPEND_ROWS // (B * H_kv))))
        return dict(kind=kind, B=B, H_kv=H_kv, d=d, n_lo=(hi + 1) // 2, n_hi=hi, L_lo=0, L_hi=rng.randint(0, 1000), step=1)
    cache = rng.choice(["kvq", "bf16"])
    H_kv, layers = rng.choice([1, 2, 4, 8]), rng.randint(1, 8)
    page = H_kv * 4 * block_bytes(d) if cache == "kvq" else 2 * H_kv * PAGE * d * 2
    moves = _log(rng, 1, max(1, min(900, int(MAX_MOVE_BYTES / (2 * page * layers)))))
    lo, hi = rng.choice([(1, 127), (128, 128), (1, 128), (1, 20)])
    return dict(kind=kind, cache=cache, H_kv=H_kv, d=d, layers=layers, pages=moves * 2 + rng.randint(1, 300), moves=moves,
                r_lo=lo, r_hi=hi)


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case, lo, hi, seed, n):
    """Whole numbers of [lo, hi], known to work() as well."""
    return np.random.Generator(np.random.Philox(key=[seed, 77])).integers(lo, hi + 1, size=n).astype(np.int32)


def _seq(case, seed=0):
    """Lengths before the call, and rows per sequence that an append brings."""
    L = _lengths(case, case["L_lo"], case["L_hi"], seed, case["B"])
    if case["kind"] != "append":
        return L, None
    if case["step"] > 1 or case["n_lo"] == case["n_hi"] == 1:
        return L, _lengths(case, 1, case["n_hi"], seed + 1, case["B"])        # the root row, and the accepted ones
    return L, _lengths(case, case["n_lo"], case["n_hi"], seed + 1, case["B"])


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=g).to(torch.bfloat16)


def _quantise(x):
    """x [..., d] in 32 bits: codes 0..15, and the step and the lowest value (both bf16 values) of every row."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = torch.maximum((hi - lo) / 15, torch.maximum(lo.abs(), hi.abs()) / 4096).to(torch.bfloat16).float()
    code = ((x - lo) / torch.where(step > 0, step, torch.ones_like(step))).round().clamp(0, 15)
    return code, step, lo


def _pack(k, v):
    """Rows [pages, H, 128, d] as the bytes of pages [pages, H, 4 * block_bytes(d)]."""
    P, H, _, d = k.shape
    ck, sk, lk = _quantise(k.float())
    cv, sv, lv = _quantise(v.float())
    kb = ck.to(torch.uint8).view(P, H, 4, BLOCK, d // 2, 2)
    kb = (kb[..., 0] | (kb[..., 1] << 4)).view(P, H, 4, BLOCK * d // 2)
    # V: row 16a + 8e + 2t + h, channel 32w + 16(q/2) + 8(q%2) + n -> byte 512w + 64n + 16t + 8a + 4e + 2h + q/2
    vb = cv.to(torch.uint8).view(P, H, 4, 2, 2, 4, 2, d // 32, 2, 2, 8)       # block a e t h w q/2 q%2 n
    vb = vb[..., 0, :] | (vb[..., 1, :] << 4)                                 # block a e t h w q/2 n
    vb = vb.permute(0, 1, 2, 7, 9, 5, 3, 4, 6, 8).reshape(P, H, 4, BLOCK * d // 2)
    par = [torch.cat([s, z], -1).to(torch.bfloat16).view(P, H, 4, 2 * BLOCK).contiguous().view(torch.uint8) for s, z in ((sk, lk), (sv, lv))]
    return torch.cat([kb, vb] + par, -1).reshape(P, H, 4 * block_bytes(d)).contiguous()


def _pool(g, n_pages, H, d):
    pool = torch.empty(n_pages, H, 4 * block_bytes(d), dtype=torch.uint8, device="cuda")
    at = max(1, (1 << 26) // (H * PAGE * d))
    for p in range(0, n_pages, at):                        # (some pages at a time: the rows are larger than their codes)
        n = min(at, n_pages - p)
        pool[p:p + n] = _pack(_randn(g, n, H, PAGE, d), _randn(g, n, H, PAGE, d))
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    rng = np.random.Generator(np.random.Philox(key=[int(seed), 5]))
    d, H = case["d"], case["H_kv"]
    st = dict(case=case)
    if case["kind"] == "pages":
        n, m = case["pages"], case["moves"]
        if case["cache"] == "kvq":
            st["pools"] = [torch.randint(0, 256, (n, H, 4 * block_bytes(d)), dtype=torch.uint8, device="cuda", generator=g) for _ in range(case["layers"])]
        else:
            st["pools"] = [torch.empty(n, H, PAGE, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2 * case["layers"])]
        order = rng.permutation(n)[:2 * m]
        rows = _lengths(case, case["r_lo"], case["r_hi"], 0, m)
        st["moves"] = np.stack([order[:m], order[m:], rows], 1).astype(np.int32)
        return st
    L, count = _seq(case)
    B = case["B"]
    total = L + (count if count is not None else 0)
    pps = max(1, int((int(total.max()) + PAGE - 1) // PAGE))
    need = (total + PAGE - 1) // PAGE
    n_pages = int(need.sum()) + 3
    table = np.full((B, pps), -1, np.int32)
    free = rng.permutation(n_pages).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    for b in range(B):
        table[b, :need[b]] = free[at[b]:at[b + 1]]
    st["table"] = torch.from_numpy(table).cuda()
    st["kv_len"] = torch.from_numpy(L).cuda()
    if case["kind"] == "append":
        st["pool"] = torch.zeros(n_pages, H, 4 * block_bytes(d), dtype=torch.uint8, device="cuda")
        rows = max(1, (case["n_hi"] - 1) * case["step"] + 1) if case["step"] == 1 else case["step"] ** 2
        # K and V of a projection's output, one slice each
        st["kv_new"] = _randn(g, B, rows, 2, H, d)
        st["count"] = torch.from_numpy(count).cuda()
        st["k_out"], st["v_out"] = (torch.empty(B, case["n_hi"], H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st["len_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        return st
    n_q = (case["k"] + 1) ** 2
    st["pool"] = _pool(g, n_pages, H, d)
    st["q"] = (2 * torch.randn(B, n_q, case["H_q"], d, device="cuda", generator=g)).to(torch.bfloat16)
    st["new"] = (_randn(g, B, n_q, H, d), _randn(g, B, n_q, H, d)) if case["block"] else (None, None)
    st["out"] = torch.empty(B, n_q, case["H_q"], d, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(B, case["H_q"], n_q, dtype=torch.float32, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return _OWN[state["case"]["kind"]](state) if own else _PLAIN[state["case"]["kind"]](state)


def _context(state):
    """The handle and the argument structs that a user's program keeps from call to call."""
    if "call" not in state:
        from paper_2402_11809_b200 import binding as S
        c = state["case"]
        ctx = S.Context(max_batch=c["B"], n_q_heads=c.get("H_q", c["H_kv"]), n_kv_heads=c["H_kv"], head_dim=c["d"], k_max=7,
                        vocab=1, s_cap=max(128, state["table"].shape[1] * PAGE))
        if c["kind"] == "attn":
            kn, vn = state["new"]
            args = (ctx.kvq_attn_args(state["q"], state["pool"], state["table"], state["kv_len"], state["out"], c["k"],
                                      1 / math.sqrt(c["d"]), k_new=kn, v_new=vn, lse=state["lse"]),)
        else:
            kv = state["kv_new"]
            args = (ctx.kvq_append_args(kv[:, :, 0], kv[:, :, 1], state["pool"], state["table"], state["kv_len"],
                                        count=state["count"], row_step=c["step"], kv_len_out=state["len_out"]),
                    ctx.kvq_read_args(state["pool"], state["table"], state["len_out"], state["k_out"], state["v_out"],
                                      first=state["kv_len"]))
        state["call"] = (ctx, args)
    return state["call"]


def _own_attn(state):
    ctx, (args,) = _context(state)
    ctx.space_kvq_attn_step(args)
    return {"out": state["out"], "lse": state["lse"]}


def _own_append(state):
    ctx, (append, read) = _context(state)
    ctx.space_kvq_append(append)
    ctx.space_kvq_read(read)
    return {"k": state["k_out"], "v": state["v_out"], "kv_len": state["len_out"]}


def _own_pages(state):
    from paper_2402_11809_b200 import binding as S
    if "call" not in state:
        state["call"] = S.page_pools(state["pools"])
    S.space_pages_copy(state["call"], state["moves"])
    return state["pools"]


def _values(blocks, d):
    """Bytes of pages [..., 4 * block_bytes(d)] -> K and V rows [..., 128, d] in 32 bits."""
    lead = blocks.shape[:-1]
    x = blocks.reshape(*lead, 4, block_bytes(d))
    n = BLOCK * d // 2
    par = x[..., 2 * n:].contiguous().view(torch.bfloat16).reshape(*lead, 4, 2, BLOCK, 2).float()
    kb = x[..., :n].reshape(*lead, 4, BLOCK, d // 2)
    k = torch.stack([kb & 15, kb >> 4], -1).reshape(*lead, 4, BLOCK, d).float()
    k = k * par[..., 0, :, :1] + par[..., 0, :, 1:]
    vb = x[..., n:2 * n].reshape(*lead, 4, d // 32, 8, 4, 2, 2, 2, 2)             # w n t a e h q/2
    m = len(lead) + 1
    vb = vb.permute(*range(m), m + 3, m + 4, m + 2, m + 5, m, m + 6, m + 1)       # a e t h w q/2 n
    v = torch.stack([vb & 15, vb >> 4], -2).reshape(*lead, 4, BLOCK, d).float()
    v = v * par[..., 1, :, :1] + par[..., 1, :, 1:]
    return k.reshape(*lead, PAGE, d), v.reshape(*lead, PAGE, d)


def _visible(k, device):
    """Eq. 5, same-group reading: block row i = (g, o) sees earlier real tokens and its own group's masks."""
    i = torch.arange((k + 1) ** 2, device=device)
    g, o = i // (k + 1), i % (k + 1)
    earlier = i[:, None] >= i[None, :]
    return earlier & ((o[None, :] == 0) | ((o[:, None] != 0) & (g[:, None] == g[None, :])))


def _plain_attn(state):
    c = state["case"]
    B, H, d, k = c["B"], c["H_kv"], c["d"], c["k"]
    n_q, G = (k + 1) ** 2, c["H_q"] // H
    kc, vc = _values(state["pool"][state["table"].clamp(min=0).long()], d)       # [B, T, H, 128, d]
    S = kc.shape[1] * PAGE
    kc = kc.transpose(1, 2).reshape(B, H, S, d)
    vc = vc.transpose(1, 2).reshape(B, H, S, d)
    q = state["q"].float().reshape(B, n_q, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, n_q * G, d) / math.sqrt(d)
    s = q @ kc.transpose(-1, -2)
    there = torch.arange(S, device="cuda")[None] < state["kv_len"][:, None]
    s = s.masked_fill(~there[:, None, None], -math.inf)
    vc = vc.masked_fill(~there[:, None, :, None], 0.0)
    if c["block"]:
        kn, vn = (x.float().transpose(1, 2) for x in state["new"])               # [B, H, n_q, d]
        sn = (q @ kn.transpose(-1, -2)).reshape(B, H, n_q, G, n_q)
        sn = sn.masked_fill(~_visible(k, "cuda")[:, None], -math.inf).reshape(B, H, n_q * G, n_q)
        s, vc = torch.cat([s, sn], -1), torch.cat([vc, vn], 2)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = e.sum(-1, keepdim=True)
    o = (e @ vc) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (torch.log(total) + top).squeeze(-1)
    o = o.reshape(B, H, n_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, n_q, c["H_q"], d)
    lse = lse.reshape(B, H, n_q, G).permute(0, 1, 3, 2).reshape(B, c["H_q"], n_q)
    return {"out": o.to(torch.bfloat16), "lse": lse.contiguous()}


def _plain_append(state):
    c = state["case"]
    n, step = c["n_hi"], c["step"]
    there = torch.arange(n, device="cuda")[None] < state["count"][:, None]
    rows = []
    for which in (0, 1):
        x = state["kv_new"][:, :(n - 1) * step + 1:step, which].float()
        code, s, lo = _quantise(x)
        rows.append((code * s + lo).masked_fill(~there[:, :, None, None], 0.0).to(torch.bfloat16))
    return {"k": rows[0], "v": rows[1], "kv_len": state["kv_len"] + state["count"]}


def _plain_pages(state):
    moves = torch.from_numpy(state["moves"]).cuda().long()
    src, dst, rows = moves[:, 0], moves[:, 1], moves[:, 2]
    for pool in state["pools"]:
        if pool.dtype == torch.uint8:                      # 32 rows are laid out together
            n, H, size = pool.shape
            parts, kept = pool.view(n, H, 4, size // 4), torch.arange(4, device="cuda")[None] * BLOCK < rows[:, None]
        else:
            parts, kept = pool, torch.arange(PAGE, device="cuda")[None] < rows[:, None]
        parts[dst] = torch.where(kept[:, None, :, None], parts[src], parts[dst])
    return state["pools"]


_OWN = {"attn": _own_attn, "append": _own_append, "pages": _own_pages}
_PLAIN = {"attn": _plain_attn, "append": _plain_append, "pages": _plain_pages}


# ------------------------------------------------------------------------------------------------ bytes and products

def work(case):
    d, H = case["d"], case["H_kv"]
    if case["kind"] == "pages":
        rows = _lengths(case, case["r_lo"], case["r_hi"], 0, case["moves"]).astype(np.int64)
        if case["cache"] == "kvq":
            return {"bytes": 2 * int(((rows + BLOCK - 1) // BLOCK).sum()) * H * block_bytes(d) * case["layers"], "flops": 0}
        return {"bytes": 2 * int(rows.sum()) * H * d * 2 * 2 * case["layers"], "flops": 0}
    L, count = _seq(case)
    if case["kind"] == "append":
        rows = int(count.sum()) * H
        # bf16 rows in, codes and params out, and back (the rows past a count are written as zeros)
        return {"bytes": rows * (4 * d + 2 * (d + 8)) + case["B"] * case["n_hi"] * H * 4 * d, "flops": 0}
    n_q = (case["k"] + 1) ** 2
    new = n_q if case["block"] else 0
    keys = int(L.sum()) + case["B"] * new
    return {"bytes": int(L.sum()) * H * (d + 8) + case["B"] * new * H * 4 * d + case["B"] * n_q * case["H_q"] * (4 * d + 4),
            "flops": 4 * d * keys * case["H_q"] * n_q}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _rows64(pool, table_row, n, d):
    """Cache rows 0 .. n-1 of one sequence, [H, n, d] each, element by element from the format's definition."""
    r, c = torch.arange(n, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    pages = pool[table_row.long()[:(n + PAGE - 1) // PAGE]].transpose(0, 1)      # [H, T, bytes]
    flat = pages.reshape(pages.shape[0], -1)
    size, i = block_bytes(d), r % BLOCK
    base = (r // BLOCK) * size
    found = []
    for which in (0, 1):
        if which == 0:
            at, high = base + i * (d // 2) + c // 2, c % 2
        else:
            w, q, m = c // 32, c // 8 % 4, c % 8
            at = base + BLOCK * d // 2 + 512 * w + 16 * (4 * m + i // 2 % 4) + 8 * (i // 16) + 4 * (i // 8 % 2) + 2 * (i % 2) + q // 2
            high = q % 2
        code = (flat[:, at].int() >> (4 * high)) & 15
        p = base + BLOCK * d + which * 4 * BLOCK + 4 * i
        two = [(flat[:, p + o].int() | (flat[:, p + o + 1].int() << 8)) << 16 for o in (0, 2)]
        s, lo = (t.contiguous().view(torch.float32).double() for t in two)
        found.append(lo + s * code.double())
    return found


def exact(case, seed):
    if case["kind"] == "pages":
        return None
    st = prepare(case, seed)
    d, H, B = case["d"], case["H_kv"], case["B"]
    L, count = _seq(case)
    if case["kind"] == "append":
        out = {"kv_len": torch.from_numpy(L + count)}
        for which, name in ((0, "k"), (1, "v")):
            y = torch.zeros(B, case["n_hi"], H, d, dtype=torch.float64, device="cuda")
            for b in range(B):
                x = st["kv_new"][b, :(int(count[b]) - 1) * case["step"] + 1:case["step"], which].double()
                lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
                s = torch.max((hi - lo) / 15.0, torch.max(-lo, hi) * 2.0 ** -12)
                s = s.float().to(torch.bfloat16).double()          # held in bf16 by definition
                y[b, :x.shape[0]] = lo + s * torch.clamp(torch.round((x - lo) / s), 0, 15)
            out[name] = y
        return out
    k, G = case["k"], case["H_q"] // H
    n_q = (k + 1) ** 2
    if B * case["L_hi"] * H * n_q * G * d > 3e11:
        return None
    out = torch.zeros(B, n_q, case["H_q"], d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, case["H_q"], n_q), -math.inf, dtype=torch.float64, device="cuda")
    hidden = torch.ones(n_q, n_q, dtype=torch.bool, device="cuda")
    for i in range(n_q):
        for j in range(i + 1):
            gi, oi, gj, oj = i // (k + 1), i % (k + 1), j // (k + 1), j % (k + 1)
            hidden[i, j] = oj != 0 and (oi == 0 or gi != gj)
    for b in range(B):
        n = int(L[b])
        kc, vc = _rows64(st["pool"], st["table"][b], n, d)
        if case["block"]:
            kc, vc = (torch.cat([x, y[b].double().transpose(0, 1)], 1) for x, y in ((kc, st["new"][0]), (vc, st["new"][1])))
        if not kc.shape[1]:
            continue
        for h in range(case["H_q"]):
            s = st["q"][b, :, h].double() @ kc[h // G].T / math.sqrt(d)
            if case["block"]:
                s[:, n:].masked_fill_(hidden, -math.inf)
            lse[b, h] = torch.logsumexp(s, -1)
            out[b, :, h] = torch.softmax(s, -1) @ vc[h // G]
    return {"out": out, "lse": lse}
