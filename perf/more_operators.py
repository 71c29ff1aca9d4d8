"""What surrounds the attention of a decoding step, as cases that can be timed.

Four operators, through the public entry points of paper_2402_11809_b200.binding:

  attn    space_kvb_attn_step: the block of a step ((k+1)^2 rows; k = 0: one new token) attends over a cache in 8 bits
          (e4m3 codes with one power of two per 32 rows and head) and, where they are given, its own bf16 rows
  append  space_kvb_append and space_kvb_read: new rows are put into that cache, rotated by their position on the way
          where a table is given (and their queries with them), and read back as the values that they stand for
  rope    space_rope_append: queries and keys are rotated by position, keys and values put into the bf16 cache
  logits  space_logits_adjust (behind space_token_counts where a request starts): penalties for repeated tokens, biases
          and grammar masks on the logits of the block's rows, each of which has seen the candidates before it

The plain forms below use elementary torch operations in 32 bits on the same inputs.
"""
import math

import numpy as np
import torch

own = False

PAGE = 128            # rows of a page
BLOCK = 32            # rows that share a scale
PROMPT = 1 << 30      # counts: the token occurs in the prompt


def head_bytes(d):
    return 2 * PAGE * d + 2 * 4 * (PAGE // BLOCK)          # K and V codes of a page, then {K scale, V scale} of its blocks


# ------------------------------------------------------------------------------------------------ cases

def _attn(name, B, heads, d, L, k, block=True):
    return dict(name=name, kind="attn", B=B, H_q=heads[0], H_kv=heads[1], d=d, L_lo=L[0], L_hi=L[1], k=k, block=block)


def _append(name, B, heads, d, n, L, step=1, rot=0, interleaved=False):
    return dict(name=name, kind="append", B=B, H_q=heads[0], H_kv=heads[1], d=d, n_lo=n[0], n_hi=n[1], L_lo=L[0], L_hi=L[1],
                step=step, rot=rot, interleaved=interleaved)


def _rope(name, B, heads, d, n, L, rot, k=-1, interleaved=False, paged=True):
    return dict(name=name, kind="rope", B=B, H_q=heads[0], H_kv=heads[1], d=d, n_lo=n[0], n_hi=n[1], L_lo=L[0], L_hi=L[1],
                rot=rot, k=k, interleaved=interleaved, paged=paged)


def _logits(name, B, k, V, dtype, prompt=0, bias=0, masks=0, keep=0.5):
    return dict(name=name, kind="logits", B=B, k=k, V=V, dtype=dtype, prompt=prompt, bias=bias, masks=masks, keep=keep)


def listed():
    return [
        # one new token of a short chat on a small model: launches and latency are all there is
        _attn("attn_tiny_token", 1, (8, 8), 64, (128, 128), 0),
        # odd sizes: few ragged sequences that end inside pages, head size 64
        _attn("attn_odd5", 5, (16, 8), 64, (37, 1999), 3),
        # a server's batch of users at ragged lengths, a step of 36 rows each
        _attn("attn_ragged16", 16, (32, 32), 128, (512, 4096), 5),
        # a model with grouped queries at long context: 392 query rows to a kv head, the products are large
        _attn("attn_grouped", 8, (64, 8), 128, (8192, 8192), 6),
        # a full batch of users that decode token by token, lengths up to 16k: the cache's bytes are the cost
        _attn("attn_tokens64", 64, (32, 8), 128, (1024, 16384), 0),
        # one document of 131071 tokens, the token's own row already in the cache
        _attn("attn_long_token", 1, (32, 8), 128, (131071, 131071), 0, block=False),
        # the rows that the steps of a batch have accepted: root and up to k = 4 candidates out of 25 block rows
        _append("append_accepted", 64, (8, 8), 128, (5, 5), (1024, 16384), step=5),
        # a batch of prompts that come in pieces behind what is cached, rotated on the way
        _append("append_prompts", 16, (32, 8), 128, (512, 4096), (0, 300), rot=128),
        # the block of a step of sixteen users, into pages: positions of Eq. 4's rows
        _rope("rope_step16", 16, (32, 32), 128, (36, 36), (512, 4096), 128, k=5),
        # long prompts of odd lengths into a contiguous cache, neighbouring channels turned together, half of them
        _rope("rope_prompts", 4, (32, 8), 128, (3333, 8191), (0, 0), 64, interleaved=True, paged=False),
        # the first token of a batch of new requests: their prompts are counted, some tokens are favoured
        _logits("logits_prompt64", 64, 0, 128256, "f32", prompt=2048, bias=16),
        # a step of sixteen users under a grammar that leaves few tokens, an odd vocabulary
        _logits("logits_step16", 16, 5, 50257, "bf16", bias=3, masks=24, keep=0.02),
    ]


MAX_ATTN_BYTES = 1.1e9        # the largest listed step reads about this much
MAX_ATTN_FLOPS = 1.0e11
MAX_APPEND_ELEMENTS = 16 * 8 * 2304 * 128
MAX_ROPE_ELEMENTS = 4 * 48 * 5700 * 128
MAX_LOGITS_BYTES = 5.7e7


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "rope", "logits"])
    d = rng.choice([64, 128, 128])
    if kind == "logits":
        k = rng.choice([0, 0, 1, 2, 3, 5, 7])
        B = _log(rng, 1, 64)
        dtype = rng.choice(["f32", "bf16"])
        most = int(MAX_LOGITS_BYTES / (B * ((k + 1) ** 2 * (4 if dtype == "f32" else 2) + 4)))
        V = _log(rng, 500, max(501, min(200000, most)))
        return dict(kind=kind, B=B, k=k, V=V, dtype=dtype, prompt=rng.choice([0, 0, 7, 500, 3000]), bias=rng.choice([0, 1, 16, 300]),
                    masks=rng.choice([0, 0, 1, 5, 40]), keep=rng.choice([0.001, 0.1, 0.9]))
    k = rng.choice([0, 0, 1, 2, 3, 4, 5, 6, 7])
    H_kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 32])
    G = rng.choice([g for g in (1, 1, 2, 4, 4, 8, 16) if g * H_kv <= 64])
    B = _log(rng, 1, 64)
    if kind == "attn":
        most = min(MAX_ATTN_BYTES / (B * H_kv * 2 * d), MAX_ATTN_FLOPS / (4 * d * B * H_kv * G * (k + 1) ** 2), 131071)
        hi = _log(rng, 64, max(65, int(most)))
        lo = max(0, int(hi * rng.choice([0.0, 0.1, 0.5, 0.5, 1.0])))
        return dict(kind=kind, B=B, H_q=G * H_kv, H_kv=H_kv, d=d, L_lo=lo, L_hi=hi, k=k,
                    block=True if k else rng.random() < 0.5)
    rot = rng.choice([r for r in (16, 32, 64, 96, 128) if r <= d])
    inter = rng.random() < 0.4
    if kind == "append":
        if rng.random() < 0.4:
            return dict(kind=kind, B=B, H_q=H_kv, H_kv=H_kv, d=d, n_lo=k + 1, n_hi=k + 1, L_lo=0, L_hi=_log(rng, 16, 16384), step=k + 1,
                        rot=0, interleaved=False)
        hi = _log(rng, 1, max(1, min(8192, MAX_APPEND_ELEMENTS // (B * H_kv * d))))
        return dict(kind=kind, B=B, H_q=G * H_kv, H_kv=H_kv, d=d, n_lo=(hi + 1) // 2, n_hi=hi, L_lo=0, L_hi=rng.randint(0, 1000), step=1,
                    rot=rng.choice([0, rot]), interleaved=inter)
    step = rng.random() < 0.5
    hi = (k + 1) ** 2 if step else _log(rng, 1, max(1, min(8192, MAX_ROPE_ELEMENTS // (B * H_kv * (G + 2) * d))))
    return dict(kind=kind, B=B, H_q=G * H_kv, H_kv=H_kv, d=d, n_lo=hi if step else (hi + 1) // 2, n_hi=hi, L_lo=0,
                L_hi=rng.randint(0, 2000), rot=rot, k=k if step else -1, interleaved=inter, paged=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs

def _numbers(lo, hi, seed, n):
    """Whole numbers of [lo, hi], known to work() as well."""
    return np.random.Generator(np.random.Philox(key=[seed, 77])).integers(lo, hi + 1, size=n).astype(np.int32)


def _seq(case):
    """Lengths before the call, and the rows per sequence that come behind them."""
    L = _numbers(case["L_lo"], case["L_hi"], 0, case["B"])
    if case["kind"] == "attn":
        return L, None
    if case["kind"] == "append" and case["step"] > 1:
        return L, _numbers(1, case["n_hi"], 1, case["B"])                     # the root row, and the accepted ones
    return L, _numbers(case["n_lo"], case["n_hi"], 1, case["B"])


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=g).to(torch.bfloat16)


def _scale(top):
    """The least power of two of which 448 times is no less than top (32 bits), 2^-100 at least."""
    m, e = torch.frexp(top)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, e, torch.full_like(e, -100)).clamp(min=-100))


def _code(x, scale):
    """x / scale to the nearest e4m3 number, as 32-bit values: steps of 1/8 of its power of two, 2^-9 at least."""
    y = (x / scale).clamp(-448.0, 448.0)
    e = torch.frexp(y)[1].clamp(min=-5) - 4
    return torch.ldexp(torch.round(torch.ldexp(y, -e)), e)


def _pack(k, v):
    """Rows [pages, H, 128, d] as the bytes of pages [pages, H, head_bytes(d)]."""
    P, H, _, d = k.shape
    codes, scales = [], []
    for x in (k.float(), v.float()):
        s = _scale(x.abs().view(P, H, PAGE // BLOCK, BLOCK * d).amax(-1))
        c = _code(x.view(P, H, PAGE // BLOCK, BLOCK, d), s[..., None, None]).view(P, H, PAGE, d)
        codes.append(c.to(torch.float8_e4m3fn).view(torch.uint8))
        scales.append(s)
    kb = codes[0].view(P, H, PAGE, d // 16, 16).transpose(2, 3).reshape(P, H, PAGE * d)
    vb = codes[1].view(P, H, PAGE // 16, 16, d).transpose(3, 4).reshape(P, H, PAGE * d)
    sb = torch.stack(scales, -1).view(P, H, -1).contiguous().view(torch.uint8)
    return torch.cat([kb, vb, sb], -1).contiguous()


def _pool(g, n_pages, H, d):
    pool = torch.empty(n_pages, H, head_bytes(d), dtype=torch.uint8, device="cuda")
    at = max(1, (1 << 25) // (H * PAGE * d))
    for p in range(0, n_pages, at):                        # (some pages at a time: the rows are larger than their codes)
        n = min(at, n_pages - p)
        pool[p:p + n] = _pack(_randn(g, n, H, PAGE, d), _randn(g, n, H, PAGE, d))
    return pool


def _table(total, rng, extra=3):
    """Pages in any order for sequences of these lengths, and how many there are."""
    need = (total + PAGE - 1) // PAGE
    n_pages = int(need.sum()) + extra
    table = np.full((len(total), max(1, int(need.max()))), -1, np.int32)
    free = rng.permutation(n_pages).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    for b in range(len(total)):
        table[b, :need[b]] = free[at[b]:at[b + 1]]
    return table, n_pages


def _angles(n_pos, rot):
    """Cosines, then sines of every position's angles: what a model holds."""
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)[None]
    return torch.cat([a.cos(), a.sin()], 1).float().cuda()


def _block_positions(k, L):
    """Position of every block row (Sec. 3.2): what it sees of the block, its own row not counted, behind the cache."""
    i = np.arange((k + 1) ** 2)
    return (L[:, None] + (i // (k + 1) + i % (k + 1))[None]).astype(np.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    rng = np.random.Generator(np.random.Philox(key=[int(seed), 5]))
    st = dict(case=case)
    if case["kind"] == "logits":
        B, V, n = case["B"], case["V"], (case["k"] + 1) ** 2
        rand = lambda lo, hi, *s: torch.from_numpy(rng.integers(lo, hi, size=s).astype(np.int32)).cuda()
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        st["logits"] = (3 * torch.randn(B, n, V, device="cuda", generator=g)).to(dt)
        st["out"] = torch.empty_like(st["logits"])
        # tokens come back: the frequent ones of a language
        text = lambda m: torch.from_numpy((V * rng.random((B, m)) ** 3).astype(np.int32)).cuda()
        st["tokens"], st["n_tokens"] = text(max(1, case["prompt"])), torch.from_numpy(_numbers(case["prompt"] // 2, case["prompt"], 3, B)).cuda()
        st["counts"] = torch.zeros(B, V, dtype=torch.int32, device="cuda")
        history = text(400).long()
        st["counts"].scatter_add_(1, history, torch.ones_like(history, dtype=torch.int32))
        st["cand"] = text(max(1, case["k"]))[:, :case["k"]].contiguous()
        f = lambda lo, hi: torch.from_numpy(rng.uniform(lo, hi, B).astype(np.float32)).cuda()
        st["repetition"], st["presence"], st["frequency"] = f(1.0, 1.5), f(0.0, 1.0), f(0.0, 0.5)
        st["bias_tok"], st["bias_val"] = rand(0, V, B, max(1, case["bias"])), torch.randn(B, max(1, case["bias"]), device="cuda", generator=g)
        bits = torch.zeros(max(1, case["masks"]), (V + 31) // 32, dtype=torch.int32, device="cuda")
        for m in range(case["masks"]):
            kept = torch.zeros(bits.shape[1] * 32, dtype=torch.int32, device="cuda")
            kept[:V] = torch.rand(V, device="cuda", generator=g) < case["keep"]
            two = torch.tensor([1 << i if i < 31 else -(1 << 31) for i in range(32)], dtype=torch.int32, device="cuda")
            bits[m] = (kept.view(-1, 32) * two).sum(1).to(torch.int32)
        st["mask_bits"], st["mask_row"] = bits, rand(-1, max(1, case["masks"]), B, n)
        return st
    d, H, B = case["d"], case["H_kv"], case["B"]
    L, count = _seq(case)
    total = L + (count if count is not None else 0)
    table, n_pages = _table(total, rng)
    st["table"], st["kv_len"] = torch.from_numpy(table).cuda(), torch.from_numpy(L).cuda()
    if case["kind"] == "attn":
        n_q = (case["k"] + 1) ** 2
        st["pool"] = _pool(g, n_pages, H, d)
        st["q"] = (2 * torch.randn(B, n_q, case["H_q"], d, device="cuda", generator=g)).to(torch.bfloat16)
        st["new"] = (_randn(g, B, n_q, H, d), _randn(g, B, n_q, H, d)) if case["block"] else (None, None)
        st["out"] = torch.empty(B, n_q, case["H_q"], d, dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.empty(B, case["H_q"], n_q, dtype=torch.float32, device="cuda")
        return st
    st["count"], st["len_out"] = torch.from_numpy(count).cuda(), torch.zeros(B, dtype=torch.int32, device="cuda")
    rows = case["n_hi"] if case["kind"] == "rope" or case["step"] == 1 else case["step"] ** 2
    # q, k and v of a projection's output, one slice each
    st["qkv"] = _randn(g, B, rows, case["H_q"] + 2 * H, d)
    if case["rot"]:
        st["angles"] = _angles(int(total.max()) + 8, case["rot"])
        st["pos"] = torch.from_numpy(_block_positions(case["k"], L)).cuda() if case.get("k", -1) >= 0 else None
        st["q_out"] = torch.zeros(B, rows, case["H_q"], d, dtype=torch.bfloat16, device="cuda")
    if case["kind"] == "append":
        st["pool"] = _pool(g, n_pages, H, d)
        n = case["n_hi"] + BLOCK - 1                       # the rows of a block that has old rows are read back with the new ones
        st["first"] = torch.from_numpy(L // BLOCK * BLOCK).cuda()
        st["k_out"], st["v_out"] = (torch.empty(B, n, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return st
    if case["paged"]:
        st["cache"] = torch.zeros(2, n_pages, H, PAGE, d, dtype=torch.bfloat16, device="cuda")
    else:
        st["cache"] = torch.zeros(2, B, H, max(128, int(total.max()) + 1), d, dtype=torch.bfloat16, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return _OWN[state["case"]["kind"]](state) if own else _PLAIN[state["case"]["kind"]](state)


def _slices(state):
    c, x = state["case"], state["qkv"]
    return x[:, :, :c["H_q"]], x[:, :, c["H_q"]:c["H_q"] + c["H_kv"]], x[:, :, c["H_q"] + c["H_kv"]:]


def _context(state):
    """The handle and the argument structs that a user's program keeps from call to call."""
    if "call" not in state:
        from paper_2402_11809_b200 import binding as S
        c = state["case"]
        rows = state["table"].shape[1] * PAGE if "table" in state else 128
        if c["kind"] == "rope" and not c["paged"]:
            rows = state["cache"].shape[3]                 # (a contiguous cache has as many rows as the handle says)
        ctx = S.Context(max_batch=c["B"], n_q_heads=c.get("H_q", 1), n_kv_heads=c.get("H_kv", 1), head_dim=c.get("d", 64), k_max=7,
                        vocab=c.get("V", 1), s_cap=max(128, rows))
        if c["kind"] == "attn":
            kn, vn = state["new"]
            args = (ctx.kvb_attn_args(state["q"], state["pool"], state["table"], state["kv_len"], state["out"], c["k"],
                                      1 / math.sqrt(c["d"]), k_new=kn, v_new=vn, lse=state["lse"]),)
        elif c["kind"] == "append":
            q, k, v = _slices(state)
            turn = dict(rope=S.rope(state["angles"], interleaved=c["interleaved"]), q=q, q_out=state["q_out"]) if c["rot"] else {}
            args = (ctx.kvb_append_args(k, v, state["pool"], state["table"], state["kv_len"], count=state["count"],
                                        row_step=c["step"], kv_len_out=state["len_out"], **turn),
                    ctx.kvb_read_args(state["pool"], state["table"], state["len_out"], state["k_out"], state["v_out"],
                                      first=state["first"]))
        elif c["kind"] == "rope":
            q, k, v = _slices(state)
            args = (ctx.rope_append_args(S.rope(state["angles"], interleaved=c["interleaved"], pos=state["pos"]), q, state["q_out"], k,
                                         v=v, k_cache=state["cache"][0], v_cache=state["cache"][1], kv_len=state["kv_len"],
                                         count=state["count"], kv_len_out=state["len_out"],
                                         page_table=state["table"] if c["paged"] else None),)
        else:
            args = (ctx.logits_adjust_args(state["logits"], state["out"], c["k"], counts=state["counts"], cand=state["cand"] if c["k"] else None,
                                           repetition=state["repetition"], presence=state["presence"], frequency=state["frequency"],
                                           bias_tok=state["bias_tok"] if c["bias"] else None, bias_val=state["bias_val"] if c["bias"] else None,
                                           mask_bits=state["mask_bits"] if c["masks"] else None, mask_row=state["mask_row"] if c["masks"] else None),
                    ctx.token_counts_args(state["tokens"], state["counts"], n_tokens=state["n_tokens"], prompt=True, reset=True)
                    if c["prompt"] else None)
        state["call"] = (ctx, args)
    return state["call"]


def _own_attn(state):
    ctx, (args,) = _context(state)
    ctx.space_kvb_attn_step(args)
    return {"out": state["out"], "lse": state["lse"]}


def _own_append(state):
    ctx, (append, read) = _context(state)
    ctx.space_kvb_append(append)
    ctx.space_kvb_read(read)
    return {"k": state["k_out"], "v": state["v_out"], "kv_len": state["len_out"], "q": state.get("q_out")} if state["case"]["rot"] \
        else {"k": state["k_out"], "v": state["v_out"], "kv_len": state["len_out"]}


def _own_rope(state):
    ctx, (args,) = _context(state)
    ctx.space_rope_append(args)
    return {"q": state["q_out"], "cache": state["cache"], "kv_len": state["len_out"]}


def _own_logits(state):
    ctx, (adjust, count) = _context(state)
    if count is not None:
        ctx.space_token_counts(count)
    ctx.space_logits_adjust(adjust)
    return {"logits": state["out"], "counts": state["counts"]}


def _values(pages, d):
    """Bytes of pages [..., head_bytes(d)] -> K and V rows [..., 128, d] in 32 bits."""
    lead, n = pages.shape[:-1], PAGE * d
    s = pages[..., 2 * n:].contiguous().view(torch.float32).reshape(*lead, PAGE // BLOCK, 1, 2)
    k = pages[..., :n].reshape(*lead, d // 16, PAGE, 16).transpose(-2, -3).reshape(*lead, PAGE, d)
    v = pages[..., n:2 * n].reshape(*lead, PAGE // 16, d, 16).transpose(-1, -2).reshape(*lead, PAGE, d)
    return tuple((x.contiguous().view(torch.float8_e4m3fn).float().reshape(*lead, PAGE // BLOCK, BLOCK * d) * s[..., i])
                 .reshape(*lead, PAGE, d) for i, x in enumerate((k, v)))


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
    S = state["table"].shape[1] * PAGE
    out = torch.empty_like(state["out"])
    lse = torch.empty_like(state["lse"])
    there = torch.arange(S, device="cuda")[None] < state["kv_len"][:, None]
    at = max(1, int(2e9) // (H * S * (8 * d + 8 * n_q * G)))                     # sequences at a time: what memory holds
    for b in range(0, B, at):
        e = min(B, b + at)
        kc, vc = _values(state["pool"][state["table"][b:e].clamp(min=0).long()], d)       # [B, T, H, 128, d]
        kc, vc = (x.transpose(1, 2).reshape(e - b, H, S, d) for x in (kc, vc))
        q = state["q"][b:e].float().reshape(e - b, n_q, H, G, d).permute(0, 2, 1, 3, 4).reshape(e - b, H, n_q * G, d) / math.sqrt(d)
        s = (q @ kc.transpose(-1, -2)).masked_fill(~there[b:e, None, None], -math.inf)
        vc = vc.masked_fill(~there[b:e, None, :, None], 0.0)
        if c["block"]:
            kn, vn = (x[b:e].float().transpose(1, 2) for x in state["new"])      # [B, H, n_q, d]
            sn = (q @ kn.transpose(-1, -2)).reshape(e - b, H, n_q, G, n_q)
            sn = sn.masked_fill(~_visible(k, "cuda")[:, None], -math.inf).reshape(e - b, H, n_q * G, n_q)
            s, vc = torch.cat([s, sn], -1), torch.cat([vc, vn], 2)
        top = s.amax(-1, keepdim=True)
        w = torch.exp(s - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = w.sum(-1, keepdim=True)
        o = (w @ vc) / torch.where(total > 0, total, torch.ones_like(total))
        z = (torch.log(total) + top).squeeze(-1)
        out[b:e] = o.reshape(e - b, H, n_q, G, d).permute(0, 2, 1, 3, 4).reshape(e - b, n_q, c["H_q"], d).to(torch.bfloat16)
        lse[b:e] = z.reshape(e - b, H, n_q, G).permute(0, 1, 3, 2).reshape(e - b, c["H_q"], n_q)
    return {"out": out, "lse": lse}


def _rotate(x, rows, case):
    """x [B, n, H, d] in 32 bits, rows [B, n, rot] of the table."""
    rot = case["rot"]
    cos, sin = rows[:, :, None, :rot // 2], rows[:, :, None, rot // 2:]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _positions(state, n):
    if state["pos"] is not None:
        return state["pos"].long()
    return (state["kv_len"][:, None] + torch.arange(n, device="cuda")[None]).long().clamp(max=state["angles"].shape[0] - 1)


def _plain_append(state):
    c = state["case"]
    B, n, step, H, d = c["B"], c["n_hi"], c["step"], c["H_kv"], c["d"]
    q, k, v = (x[:, :(n - 1) * step + 1:step].float() for x in _slices(state))
    there = torch.arange(n, device="cuda")[None] < state["count"][:, None]
    got = {"kv_len": state["kv_len"] + state["count"]}
    if c["rot"]:
        rows = state["angles"][_positions(state, n)]
        k = _rotate(k, rows, c)
        got["q"] = _rotate(q, rows, c).masked_fill(~there[:, :, None, None], 0.0).to(torch.bfloat16)
    # the first block's old rows, then the new ones
    off = (state["kv_len"] % BLOCK).long()
    i = torch.arange(n + BLOCK - 1, device="cuda")[None]
    old, new = i < off[:, None], (i >= off[:, None]) & (i < (off + state["count"])[:, None])
    page = state["table"].gather(1, (state["kv_len"] // PAGE).long()[:, None].clamp(max=state["table"].shape[1] - 1))[:, 0].clamp(min=0).long()
    held = _values(state["pool"][page], d)                                       # [B, H, 128, d]
    from_held = ((state["first"] % PAGE).long()[:, None] + i).clamp(max=PAGE - 1)
    scales = state["pool"][page][..., 2 * PAGE * d:].contiguous().view(torch.float32).reshape(B, H, PAGE // BLOCK, 2)
    blocks = (n + 2 * BLOCK - 2) // BLOCK
    for which, (name, x) in enumerate((("k", k), ("v", v))):
        rows = x.gather(1, (i - off[:, None]).clamp(0, n - 1)[:, :, None, None].expand(B, -1, H, d))
        had = held[which].transpose(1, 2).gather(1, from_held[:, :, None, None].expand(B, -1, H, d))
        rows = torch.where(new[:, :, None, None], rows, torch.where(old[:, :, None, None], had, torch.zeros_like(rows)))
        top = torch.zeros(B, blocks * BLOCK, H, device="cuda")
        top[:, :n + BLOCK - 1] = rows.abs().amax(-1).masked_fill(~new[:, :, None], 0.0)
        s = _scale(top.view(B, blocks, BLOCK, H).amax(2))
        was = scales[..., which].gather(2, (state["first"] % PAGE // BLOCK).long()[:, None, None].expand(B, H, 1))[:, :, 0]
        s[:, 0] = torch.where((off > 0)[:, None], torch.maximum(s[:, 0], was), s[:, 0])
        s = s.repeat_interleave(BLOCK, 1)[:, :n + BLOCK - 1, :, None]
        got[name] = (_code(rows, s) * s).to(torch.bfloat16)
    return got


def _plain_rope(state):
    c = state["case"]
    q, k, v = _slices(state)
    n = q.shape[1]
    rows = state["angles"][_positions(state, n)]
    there = torch.arange(n, device="cuda")[None] < state["count"][:, None]
    q_out = torch.where(there[:, :, None, None], _rotate(q.float(), rows, c).to(torch.bfloat16), state["q_out"])
    k = _rotate(k.float(), rows, c).to(torch.bfloat16)
    b, r = there.nonzero(as_tuple=True)
    s = (state["kv_len"][b] + r).long()
    cache = state["cache"]
    if c["paged"]:
        cache[0][state["table"][b, s // PAGE].long(), :, s % PAGE] = k[b, r]
        cache[1][state["table"][b, s // PAGE].long(), :, s % PAGE] = v[b, r]
    else:
        cache[0][b, :, s], cache[1][b, :, s] = k[b, r], v[b, r]
    return {"q": q_out, "cache": cache, "kv_len": state["kv_len"] + state["count"]}


def _plain_logits(state):
    c = state["case"]
    B, V, k = c["B"], c["V"], c["k"]
    counts = state["counts"]
    if c["prompt"]:
        counts = torch.zeros_like(counts)
        there = torch.arange(state["tokens"].shape[1], device="cuda")[None] < state["n_tokens"][:, None]
        b, r = there.nonzero(as_tuple=True)
        counts[b, state["tokens"][b, r].long()] = PROMPT
    out = torch.empty_like(state["logits"])
    bias = torch.zeros(B, V, device="cuda")
    for j in range(c["bias"]):                             # (one entry after another: a token may be named twice)
        bias.scatter_add_(1, state["bias_tok"][:, j:j + 1].long(), state["bias_val"][:, j:j + 1])
    seen, many = counts != 0, (counts & (PROMPT - 1)).float()
    rep, pres, freq = (state[x][:, None, None] for x in ("repetition", "presence", "frequency"))
    for g in range(k + 1):
        if g:                                              # rows of sub-block g have candidate g behind them too
            tok = state["cand"][:, g - 1:g].long()
            many = many.scatter_add(1, tok, torch.ones_like(tok, dtype=torch.float32))
            seen = seen.scatter(1, tok, True)
        z = state["logits"][:, g * (k + 1):(g + 1) * (k + 1)].float()
        z = torch.where(seen[:, None], torch.where(z > 0, z / rep, z * rep), z)
        z = z - freq * many[:, None]
        z = torch.where((many > 0)[:, None], z - pres, z) + bias[:, None]
        if c["masks"]:
            which = state["mask_row"][:, g * (k + 1):(g + 1) * (k + 1)]
            bits = state["mask_bits"][which.clamp(min=0).long()]                 # [B, k + 1, words]
            kept = ((bits[..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(-2)[..., :V].bool()
            z = z.masked_fill(~(kept | (which < 0)[..., None]), -math.inf)
        out[:, g * (k + 1):(g + 1) * (k + 1)] = z.to(out.dtype)
    return {"logits": out, "counts": counts}


_OWN = {"attn": _own_attn, "append": _own_append, "rope": _own_rope, "logits": _own_logits}
_PLAIN = {"attn": _plain_attn, "append": _plain_append, "rope": _plain_rope, "logits": _plain_logits}


# ------------------------------------------------------------------------------------------------ bytes and products

def work(case):
    if case["kind"] == "logits":
        n, V, e = case["B"] * (case["k"] + 1) ** 2, case["V"], 4 if case["dtype"] == "f32" else 2
        counts = case["B"] * V * 4                         # read, or written anew
        return {"bytes": 2 * n * V * e + counts + case["masks"] * ((V + 31) // 32) * 4 + case["B"] * (case["prompt"] * 3 + case["bias"] * 8),
                "flops": 0}
    d, H = case["d"], case["H_kv"]
    L, count = _seq(case)
    if case["kind"] == "attn":
        n_q = (case["k"] + 1) ** 2
        new = n_q if case["block"] else 0
        keys = int(L.sum()) + case["B"] * new
        return {"bytes": int(L.sum()) * H * 2 * d + int(L.sum()) * H // 4 + case["B"] * new * H * 4 * d + case["B"] * n_q * case["H_q"] * (4 * d + 4),
                "flops": 4 * d * keys * case["H_q"] * n_q}
    rows = int(count.sum())
    table = min(rows, int((L + count).max())) * case["rot"] * 4
    if case["kind"] == "append":
        # bf16 rows in, codes out, and back (the rows past a count are written as zeros); queries in and out
        turned = 4 * d * rows * case["H_q"] + table if case["rot"] else 0
        return {"bytes": rows * H * (4 * d + 2 * 2 * d) + case["B"] * (case["n_hi"] + BLOCK - 1) * H * 4 * d + turned, "flops": 0}
    return {"bytes": rows * (case["H_q"] + 2 * H) * 4 * d + table, "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _rows64(pool, table_row, rows, d):
    """Cache rows `rows` of one sequence, [H, n, d] each, and their scales, element by element from the format's definition."""
    r, c = (rows % PAGE)[:, None], torch.arange(d, device="cuda")[None]
    flat = pool[table_row.long()[rows // PAGE]].transpose(0, 1)                  # [H, n, bytes]
    found = []
    for which in (0, 1):
        at = (c // 16) * (PAGE * 16) + r * 16 + c % 16 if which == 0 else PAGE * d + (r // 16) * (16 * d) + c * 16 + r % 16
        code = flat.gather(2, at[None].expand(flat.shape[0], -1, -1)).int()
        e, m = (code >> 3) & 15, (code & 7).double()
        x = torch.where(e > 0, (8 + m) * torch.ldexp(torch.ones_like(m), e - 10), m * 2.0 ** -9)
        p = 2 * PAGE * d + 8 * (r // BLOCK) + 4 * which + torch.arange(4, device="cuda")[None]
        word = (flat.gather(2, p[None].expand(flat.shape[0], -1, -1)).int() << torch.tensor([0, 8, 16, 24], device="cuda")).sum(-1).int()
        s = word.view(torch.float32).double()[..., None]
        found += [torch.where(code > 127, -x, x) * s, s]
    return found


def _turn64(x, rows, case):
    """Rows [m, H, d] in 64 bits; rows [m, 1, rot] of the table."""
    half, y = case["rot"] // 2, x.clone()
    c, s = rows[..., :half], rows[..., half:]
    i = torch.arange(half, device="cuda")
    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def _e4m3(y):
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    q = torch.exp2(e - 3)
    return torch.clamp(torch.round(y / q) * q, -448, 448)


def exact(case, seed):
    if case["kind"] == "attn" and case["B"] * case["L_hi"] * case["H_q"] * (case["k"] + 1) ** 2 * case["d"] > 3e11:
        return None
    st = prepare(case, seed)
    if case["kind"] == "logits":
        k, V = case["k"], case["V"]
        out = st["logits"].double()
        counts = torch.zeros_like(st["counts"]) if case["prompt"] else st["counts"]
        kept = ((st["mask_bits"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(1)[:, :V] == 1
        which = st["mask_row"].tolist()
        for b in range(case["B"]):
            if case["prompt"]:
                counts[b, st["tokens"][b, :int(st["n_tokens"][b])].unique().long()] = PROMPT
            extra = torch.zeros(V, dtype=torch.float64, device="cuda")
            if case["bias"]:
                extra.index_put_((st["bias_tok"][b].long(),), st["bias_val"][b].double(), accumulate=True)
            r, p, f = (st[x][b].double() for x in ("repetition", "presence", "frequency"))
            for i in range((k + 1) ** 2):
                n = (counts[b] % PROMPT).double()
                hit = counts[b] > 0
                for t in st["cand"][b, :i // (k + 1)].tolist():
                    n[t] += 1
                    hit[t] = True
                z = out[b, i]
                z = torch.where(hit, torch.where(z > 0, z / r, z * r), z) - f * n - p * (n > 0) + extra
                if case["masks"] and which[b][i] >= 0:
                    z[~kept[which[b][i]]] = -math.inf
                out[b, i] = z
        return {"logits": out, "counts": counts}
    d, H, B = case["d"], case["H_kv"], case["B"]
    L, count = _seq(case)
    if case["kind"] in ("append", "rope"):
        n = case["n_hi"]
        got = {"kv_len": torch.from_numpy(L + count)}
        q_all, k_all, v_all = _slices(st)
        turned = case["rot"] > 0
        if turned:
            at = st["pos"].cpu().numpy() if st["pos"] is not None else L[:, None] + np.arange(n)[None]
            got["q"] = torch.zeros(st["q_out"].shape, dtype=torch.float64, device="cuda")
        if case["kind"] == "append":
            step = case["step"]
            got["k"], got["v"] = (torch.zeros(B, n + BLOCK - 1, H, d, dtype=torch.float64, device="cuda") for _ in range(2))
        else:
            got["cache"] = st["cache"].double()
            step = 1
        for b in range(B):
            m, off = int(count[b]), int(L[b]) % BLOCK
            src = slice(0, (m - 1) * step + 1, step)
            x = [k_all[b, src].double(), v_all[b, src].double()]
            if turned:
                rows = st["angles"][torch.from_numpy(at[b, :m].astype(np.int64)).cuda()].double()[:, None]
                x[0] = _turn64(x[0], rows, case)
                got["q"][b, :m] = _turn64(q_all[b, src].double(), rows, case)
            if case["kind"] == "rope":
                s = int(L[b]) + torch.arange(m, device="cuda")
                for i in (0, 1):
                    if case["paged"]:
                        got["cache"][i][st["table"][b].long()[s // PAGE], :, s % PAGE] = x[i]
                    else:
                        got["cache"][i][b][:, s] = x[i].transpose(0, 1)
                continue
            old = _rows64(st["pool"], st["table"][b], int(L[b]) - off + torch.arange(off, device="cuda"), d) if off else None
            for i, name in ((0, "k"), (1, "v")):
                rows = x[i]
                if off:
                    rows = torch.cat([old[2 * i].transpose(0, 1), rows])
                for at0 in range(0, off + m, BLOCK):
                    part = rows[at0:at0 + BLOCK]
                    fresh = part[off:] if at0 == 0 else part
                    top = fresh.abs().amax(dim=(0, 2)).clamp(min=2.0 ** -90)
                    s = torch.exp2(torch.ceil(torch.log2(top / 448)))
                    s = torch.where(top > 448 * s, 2 * s, torch.where(top <= 224 * s, s / 2, s))
                    if at0 == 0 and off:
                        s = torch.maximum(s, old[2 * i + 1][:, 0, 0])
                    s = s[None, :, None]
                    got[name][b, at0:at0 + part.shape[0]] = _e4m3(part / s) * s
        return got
    k, G = case["k"], case["H_q"] // H
    n_q = (k + 1) ** 2
    out = torch.zeros(B, n_q, case["H_q"], d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, case["H_q"], n_q), -math.inf, dtype=torch.float64, device="cuda")
    hidden = torch.ones(n_q, n_q, dtype=torch.bool, device="cuda")
    for i in range(n_q):
        for j in range(i + 1):
            gi, oi, gj, oj = i // (k + 1), i % (k + 1), j // (k + 1), j % (k + 1)
            hidden[i, j] = oj != 0 and (oi == 0 or gi != gj)
    for b in range(B):
        n = int(L[b])
        kc, _, vc, _ = _rows64(st["pool"], st["table"][b], torch.arange(n, device="cuda"), d)
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
