"""Several samples of one prompt, decoded with auto-correction on a 4-bit or an 8-bit KV cache.

The library's part of such a server, around a small seeded model (two layers, its projections taken in torch):

  prompt      the prompt's rows go into the cache of every layer (space_kvq_append), once;
  fork        the samples share its pages (Pager.fork); the page in which it ends is copied for each of them before they
              write there (Pager.make_writable, space_pages_copy over all layers' pools);
  step        attention of the block's rows over cache and block (space_kvq_attn_step) in every layer, verification
              (space_verify), the accepted rows into the cache (space_kvq_append with their counts from the device), the
              loop's state (space_decode_advance): nothing waits for the host;
  end         rows past the end are given back (Pager.truncate), a finished sample's pages are released and the rest moved
              to the front of the pools (Pager.compact, space_pages_copy), and the others decode on.

With bits=8 the cache is the 8-bit one (space_kvb_append, space_kvb_attn_step).  A model with rotary=True has no table of
positions: queries and keys are turned (space_rope_append), the prompt's at 0, 1, .., a block's at its rows' positions.  With controls the
step's logits are changed before the verification (space_logits_adjust): penalties by what the prompt holds and the sample
has taken (space_token_counts, before the first step and after each), biases, and the tokens that are allowed.

Usage: python -m paper_2402_11809_b200.decode_kvq [samples] [k] [bits]      (default 4 3 4; needs a B200; 8 bits: with rotation and penalties)
"""
import math
import sys

PAGE = 128


class Model:
    """Two attention layers with shared heads between an embedding and a vocabulary head, all of it seeded."""

    def __init__(self, layers=2, h_q=8, h_kv=2, d=64, vocab=32, positions=4096, seed=0, rotary=False):
        import torch
        g = torch.Generator().manual_seed(seed)
        w = lambda *s, f=1.0: (torch.randn(*s, generator=g) * f).cuda()
        D = h_q * d
        self.layers, self.h_q, self.h_kv, self.d, self.vocab = layers, h_q, h_kv, d, vocab
        self.emb, self.pos = w(vocab + 1, D), w(positions, D, f=0.7)          # the last token is the mask token
        self.wq = [w(D, D, f=D ** -0.5) for _ in range(layers)]
        self.wkv = [w(D, 2 * h_kv * d, f=D ** -0.5) for _ in range(layers)]
        self.wo = [w(D, D, f=D ** -0.5) for _ in range(layers)]
        self.head = w(D, vocab, f=4 * D ** -0.5)
        self.angles = None
        if rotary:
            from . import binding as B
            self.angles = B.rope_table(positions, d)

    def embed(self, tokens, positions):                      # int [B, n] -> [B, n, D]
        return self.emb[tokens.long()] if self.angles is not None else self.emb[tokens.long()] + self.pos[positions.long()]

    def qkv(self, layer, x):                                 # bf16 [B, n, H_q, d]; K and V as slices of one tensor
        import torch
        b, n, _ = x.shape
        q = (x @ self.wq[layer]).to(torch.bfloat16).view(b, n, self.h_q, self.d)
        kv = (x @ self.wkv[layer]).to(torch.bfloat16).view(b, n, 2, self.h_kv, self.d)
        return q, kv[:, :, 0], kv[:, :, 1]

    def add(self, layer, x, attn):
        return x + attn.float().reshape(x.shape) @ self.wo[layer]

    def turn(self, ctx, q, k, kv_len, pos=None):
        """Queries and keys at their positions (in place), where the model turns them."""
        from . import binding as B
        if self.angles is not None:
            ctx.space_rope_append(ctx.rope_append_args(B.rope(self.angles, pos=pos), q, q, k, kv_len, k_out=k))

    def prompt(self, tokens, ctx):
        """K and V [1, n, H_kv, d] of every layer of a prompt [n]."""
        import torch
        x, out = self.embed(tokens[None], torch.arange(len(tokens), device="cuda")[None]), []
        for i in range(self.layers):
            q, k, v = self.qkv(i, x)
            self.turn(ctx, q, k, torch.zeros(1, dtype=torch.int32, device="cuda"))
            out.append((k, v))
            a = torch.nn.functional.scaled_dot_product_attention(q.float().transpose(1, 2), k.float().transpose(1, 2),
                                                                 v.float().transpose(1, 2), is_causal=True, enable_gqa=True)
            x = self.add(i, x, a.transpose(1, 2))
        return out


class Controls:
    """What changes a step's logits: penalties (1, 0, 0 change nothing), biases {token: number}, the tokens allowed (None: all)."""

    def __init__(self, repetition=1.0, presence=0.0, frequency=0.0, bias=None, allowed=None):
        self.repetition, self.presence, self.frequency, self.bias, self.allowed = repetition, presence, frequency, bias or {}, allowed

    def arguments(self, n, k, vocab):
        """The part of logits_adjust_args that they make up, for n samples."""
        import torch
        same = lambda x, dtype: torch.tensor([x] * n, dtype=dtype, device="cuda")
        a = {name: same(getattr(self, name), torch.float32) for name in ("repetition", "presence", "frequency")}
        if self.bias:
            a.update(bias_tok=same(list(self.bias), torch.int32), bias_val=same(list(self.bias.values()), torch.float32))
        if self.allowed is not None:
            words = [0] * ((vocab + 31) // 32)
            for t in self.allowed:
                words[t // 32] |= 1 << t % 32
            a.update(mask_bits=torch.tensor([[w - (w >> 31 << 32) for w in words]], dtype=torch.int32, device="cuda"),
                     mask_row=torch.zeros(n, (k + 1) ** 2, dtype=torch.int32, device="cuda"))
        return a


class Decoder:
    """samples continuations of one prompt; share=False gives every sample a copy of the prompt's rows of its own."""

    def __init__(self, model, prompt, samples, k, max_tokens, temperature=1.0, seed=0, share=True, bits=4, controls=None):
        import torch
        from . import binding as B
        self.B, self.m, self.k, self.n, self.max_tokens = B, model, k, samples, max_tokens
        self.bits, self.controls = bits, controls
        self.temperature, self.seed = temperature, seed
        self.prompt_rows = len(prompt) - 1                   # the last token opens the first block
        rows = self.prompt_rows + max_tokens + 2 * (k + 1)   # what a sample may ever write
        pps = (rows + PAGE - 1) // PAGE
        self.ctx = B.Context(max_batch=samples, n_q_heads=model.h_q, n_kv_heads=model.h_kv, head_dim=model.d, k_max=k,
                             vocab=model.vocab, s_cap=pps * PAGE)
        self.pools = [(B.kvq_pool if bits == 4 else B.kvb_pool)(samples * pps, model.h_kv, model.d) for _ in range(model.layers)]
        self.moves_to = B.page_pools(self.pools)
        self.pager = B.Pager(samples * pps, pps, samples)
        kv = model.prompt(torch.tensor(prompt[:-1], device="cuda"), self.ctx) if self.prompt_rows else []
        first = self.pager.admit()
        self.pager.reserve(first, self.prompt_rows)
        self._append([first], [x[0] for x in kv], [x[1] for x in kv], [0])
        self.slots, self.copied = [first], 0
        for _ in range(samples - 1):
            if share:
                s = self.pager.fork(first, self.prompt_rows)
            else:
                s = self.pager.admit()
                self.pager.reserve(s, self.prompt_rows)
                self._append([s], [x[0] for x in kv], [x[1] for x in kv], [0])
            self.slots.append(s)
        self.shared_pages = samples * self.pager.pages_per_seq - self.pager.free_pages
        for s in self.slots:
            self.pager.reserve(s, rows)
            self._move(self.pager.make_writable(s, self.prompt_rows, rows - self.prompt_rows))
        self.ids = torch.arange(samples, dtype=torch.int32, device="cuda")
        if controls:
            self.counts = torch.empty(samples, model.vocab, dtype=torch.int32, device="cuda")
            self.ctx.space_token_counts(self.ctx.token_counts_args(torch.tensor([prompt] * samples, dtype=torch.int32, device="cuda"), self.counts,
                                                                   prompt=True, reset=True))
        self._begin([prompt[-1]] * samples)

    def _move(self, moves):
        self.B.space_pages_copy(self.moves_to, moves)
        self.copied += len(moves)

    def _append(self, slots, ks, vs, lens, **more):
        import torch
        table, n = self._table(slots), torch.tensor(lens, dtype=torch.int32, device="cuda")
        for pool, k, v in zip(self.pools, ks, vs):
            self._rows(k, v, pool, table, n, **more)

    def _rows(self, *args, **more):
        ctx = self.ctx
        if self.bits == 4:
            ctx.space_kvq_append(ctx.kvq_append_args(*args, **more))
        else:
            ctx.space_kvb_append(ctx.kvb_append_args(*args, **more))

    def _attend(self, *args, **more):
        ctx = self.ctx
        if self.bits == 4:
            ctx.space_kvq_attn_step(ctx.kvq_attn_args(*args, **more))
        else:
            ctx.space_kvb_attn_step(ctx.kvb_attn_args(*args, **more))

    def _table(self, slots):
        import torch
        return torch.from_numpy(self.pager.batch_table(slots)).cuda()

    def _begin(self, last):
        import torch
        B, k, n = self.B, self.k, self.n
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.kv_len = torch.full((n,), self.prompt_rows, dtype=torch.int32, device="cuda")
        self.tokens, self.n_tokens, self.last, self.cand = i32(n, self.max_tokens), i32(n), i32(n), i32(n, k)
        self.cand_prob, self.finished = torch.zeros(n, k, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.block_tokens, self.block_pos = i32(n, (k + 1) ** 2), i32(n, (k + 1) ** 2)
        self.status = i32(n)
        self._state()
        self.ctx.space_decode_begin(self.state, torch.tensor(last, dtype=torch.int32, device="cuda"))

    def _state(self):
        """The loop's state, step outputs and table for the samples that are left."""
        import torch
        k, n = self.k, self.n
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.state = self.ctx.decode_state(self.tokens, self.n_tokens, self.last, self.cand, self.cand_prob, self.kv_len,
                                           self.finished, self.block_tokens, self.block_pos, k, mask_token_id=self.m.vocab)
        self.table = self._table(self.slots)
        self.out = torch.empty(n, (k + 1) ** 2, self.m.h_q, self.m.d, dtype=torch.bfloat16, device="cuda")
        self.n_accept, self.out_tokens, self.n_out, self.next_cand = i32(n), i32(n, k + 1), i32(n), i32(n, k)
        self.next_prob, self.done, self.next_len = torch.zeros(n, k, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), i32(n)
        if self.controls:
            self.adjust = self.controls.arguments(n, k, self.m.vocab)

    def step(self):
        ctx, k, m = self.ctx, self.k, self.m
        x, kv = m.embed(self.block_tokens, self.block_pos), []
        for i in range(m.layers):
            q, kn, vn = m.qkv(i, x)
            m.turn(ctx, q, kn, self.kv_len, self.block_pos)
            kv.append((kn, vn))
            self._attend(q, self.pools[i], self.table, self.kv_len, self.out, k, 1 / math.sqrt(m.d), k_new=kn, v_new=vn, status=self.status)
            x = m.add(i, x, self.out)
        logits = (x @ m.head).contiguous()
        if self.controls:
            ctx.space_logits_adjust(ctx.logits_adjust_args(logits, logits, k, counts=self.counts, cand=self.cand, status=self.status, **self.adjust))
        ctx.space_verify(ctx.verify_args(logits, self.cand, self.cand_prob, self.kv_len, self.n_accept, self.out_tokens,
                                         self.n_out, self.next_cand, self.next_prob, self.done, k,
                                         mode=self.B.MODE_GREEDY if self.temperature == 0 else self.B.MODE_SAMPLE,
                                         temperature=self.temperature or 1.0, seed=self.seed, seq_id=self.ids, status=self.status))
        for pool, (kn, vn) in zip(self.pools, kv):           # the last token's row and those of the accepted candidates
            self._rows(kn, vn, pool, self.table, self.kv_len, count=self.n_accept, count_bias=1, row_step=k + 1, kv_len_out=self.next_len,
                       status=self.status)
        if self.controls:
            ctx.space_token_counts(ctx.token_counts_args(self.out_tokens, self.counts, n_tokens=self.n_out))
        ctx.space_decode_advance(self.state, self.out_tokens, self.n_out, self.next_cand, self.next_prob, self.done, self.next_len)

    def drop(self, i):
        """Sample i leaves: its pages go back, the pools are packed, the others go on.  Returns its tokens."""
        import torch
        got = self.tokens[i, :int(self.n_tokens[i])].tolist()
        self.pager.truncate(self.slots[i], int(self.kv_len[i]))
        self.pager.release(self.slots[i])
        while len(moves := self.pager.compact()):
            self._move(moves)
        keep = [j for j in range(self.n) if j != i]
        sel = torch.tensor(keep, device="cuda")
        self.slots, self.n = [self.slots[j] for j in keep], self.n - 1
        for name in ("ids", "kv_len", "tokens", "n_tokens", "last", "cand", "cand_prob", "finished", "block_tokens", "block_pos", "status") + (("counts",) if self.controls else ()):
            setattr(self, name, getattr(self, name)[sel].contiguous())
        if self.n:
            self._state()
        return got


def main(argv):
    import torch
    from . import build
    build.build()
    samples = int(argv[1]) if len(argv) > 1 else 4
    k = int(argv[2]) if len(argv) > 2 else 3
    bits = int(argv[3]) if len(argv) > 3 else 4
    steps, m = 64, Model(rotary=bits == 8)
    prompt = torch.randint(0, m.vocab, (700,), generator=torch.Generator().manual_seed(1)).tolist()
    controls = Controls(repetition=1.1, presence=0.2, frequency=0.05) if bits == 8 else None
    dec = Decoder(m, prompt, samples, k, max_tokens=4 * steps, bits=bits, controls=controls)
    page_bytes = dec.pools[0][0].numel() * m.layers
    print(f"prompt of {len(prompt)} tokens, {samples} samples share {dec.shared_pages} pages of {page_bytes} bytes "
          f"(bf16: {2 * PAGE * m.h_kv * m.d * 2 * m.layers}), {dec.copied} copied at the fork")
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    dec.step()
    e0.record()
    for _ in range(steps):
        dec.step()
    e1.record()
    torch.cuda.synchronize()
    tok = dec.n_tokens.tolist()
    print(f"{steps} steps, {e0.elapsed_time(e1) / steps * 1e3:.0f} us each: {tok} tokens ({sum(tok) / (samples * (steps + 1)):.2f} a step and sample)")
    moved = dec.copied
    first = dec.drop(0)
    print(f"sample 0 leaves: {first[:16]} ...; {dec.copied - moved} pages moved, {dec.pager.free_pages} free")
    for _ in range(8 if dec.n else 0):
        dec.step()
    torch.cuda.synchronize()
    print(f"the others go on: {dec.n_tokens.tolist()} tokens, status {dec.status.tolist()}")


if __name__ == "__main__":
    main(sys.argv)
