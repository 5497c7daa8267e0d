"""Speculative decoding over long contexts on a paged cache of the program's own.

A small transformer with rotary positions, its products in torch; its cache, its attention and what is kept of the
drafts in the package's operators.  Every step a cheap drafter proposes tokens; the pages and rows of the new tokens
are planned, their queries and keys turned and appended, each chunk attends over what is cached, and every cached key's
weight is added up; the drafts that the model's distribution does not keep are rolled back, pages with them; contexts that
have grown past their budget keep the keys of largest weight.  Nothing waits for the host between steps.

    python examples/speculative_decoding.py
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2410_13839_gb300 import mtp  # noqa: E402


class Model:
    """Random weights of a pre-norm transformer with grouped key heads, and of a bigram drafter near it."""

    def __init__(self, seed=0, vocab=1025, layers=2, heads=8, kv_heads=2, dim=64, sharpness=4.0):
        gen = torch.Generator().manual_seed(seed)
        self.vocab, self.layers, self.heads, self.kv_heads, self.dim = vocab, layers, heads, kv_heads, dim
        d = heads * dim

        def w(*shape):
            return (torch.randn(*shape, generator=gen) * shape[-1] ** -0.5).cuda()
        self.embed = torch.randn(vocab, d, generator=gen).cuda()
        self.blocks = [dict(qkv=w((heads + 2 * kv_heads) * dim, d), out=w(d, d), up=w(2 * d, d), down=w(d, 2 * d))
                       for _ in range(layers)]
        self.head = w(vocab, d) * sharpness
        self.bigram = F.linear(F.layer_norm(self.embed, (d,)), self.head)  # what the model says of a token alone


class SpeculativeDecoder:
    def __init__(self, model, slots, drafts=4, budget=256, slack=64, sinks=4, recent=64, temperature=1.0, eos_id=-1,
                 page_size=16, max_prompt=512, seed=0):
        self.m, self.slots, self.drafts, self.budget, self.slack = model, slots, drafts, budget, slack
        self.sinks, self.recent, self.eos, self.page = sinks, recent, eos_id, page_size
        most = max(budget + slack, max_prompt) + 2 * (drafts + 1)
        self.stride = -(-most // page_size)
        self.n_pages = slots * self.stride
        i32 = dict(dtype=torch.int32, device="cuda")
        m = model
        self.pool = torch.zeros(self.n_pages, m.layers, 2, m.kv_heads, page_size, m.dim, dtype=torch.bfloat16, device="cuda")
        # a call's tables, lengths and weights, and the buffers that an eviction writes
        self.tables = [torch.full((slots, self.stride), -1, **i32) for _ in range(2)]
        self.lens = [torch.zeros(slots, **i32) for _ in range(2)]
        self.weights = [torch.zeros(slots, m.layers, m.kv_heads, self.stride * page_size, device="cuda") for _ in range(2)]
        self.refs, self.text = torch.zeros(self.n_pages, **i32), torch.zeros(slots, **i32)  # text: tokens behind the cache
        self.last, self.done = torch.zeros(slots, **i32), torch.zeros(slots, **i32)
        self.keep = torch.full((slots,), budget, **i32)
        self.temperature = torch.full((slots,), float(temperature), device="cuda")
        self.turns = mtp.mtp_rotary_turns(m.dim, mtp.MTP_ROTARY_BANDS, factor=8.0, context=8192.0)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.status, self.evicted, self.err = torch.zeros(4, **i32), torch.zeros(slots, **i32), torch.zeros(1, **i32)
        self.worst = torch.zeros((), **i32)
        self.history, self.workspaces = [], {}
        self.longest = 0  # a bound of the slots' lengths, known without asking the GPU

    def _workspace(self, name, nbytes):
        if name not in self.workspaces or self.workspaces[name].numel() < nbytes:
            self.workspaces[name] = torch.zeros(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        return self.workspaces[name], nbytes

    def _forward(self, tokens, new_lens, max_new):
        """Feeds every slot its first new_lens[s] of tokens [slots, max_new]; (hidden rows, row tokens, first rows)."""
        m, stream, rows = self.m, torch.cuda.current_stream(), tokens.numel()
        self.longest += max_new
        i32 = dict(dtype=torch.int32, device="cuda")
        before = self.lens[0].clone()
        cu, seq, pos = torch.empty(self.slots + 1, **i32), torch.empty(rows, **i32), torch.empty(rows, **i32)
        places = torch.empty(rows, dtype=torch.int64, device="cuda")
        plan = mtp.page_plan_args(
            kv_lens=self.lens[0], new_lens=new_lens, block_table=self.tables[0], page_refs=self.refs, out_kv_lens=self.lens[0],
            out_page_refs=self.refs, out_cu_rows=cu, out_slot_map=places, out_row_seq=seq, out_row_pos=pos,
            out_status=self.status, page_size=self.page)
        mtp.mtp_page_plan(plan, stream)
        self.worst = torch.minimum(self.worst, self.status[0])
        slot = seq.long().clamp(min=0)  # (rows past the last: anything)
        fed = tokens[slot, (pos - before[slot]).long().clamp(0, max_new - 1)].contiguous()
        # a token's position is its place in the text, whatever the cache still holds of it
        where = (self.text[slot] + pos - before[slot]).contiguous()
        x = m.embed[fed.long()]
        q16 = torch.zeros(rows, m.heads, m.dim, dtype=torch.bfloat16, device="cuda")
        att, lse = torch.zeros_like(q16), torch.zeros(rows, m.heads, device="cuda")
        for layer, w in enumerate(m.blocks):
            qkv = F.linear(F.layer_norm(x, x.shape[1:]), w["qkv"]).view(rows, -1, m.dim)
            q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
            turn = mtp.rotary_append_args(q=q, k=k, v=v, positions=where, slot_map=places, turns=self.turns,
                                          kv_pool=self.pool, layer=layer, out_q=q16)
            mtp.mtp_rotary_append(turn, stream)
            shared = dict(q=q16, kv_pool=self.pool, layer=layer, block_table=self.tables[0], cu_rows=cu, kv_lens=self.lens[0],
                          scale=m.dim ** -0.5, max_new=max_new, max_keys=self.longest, err_word=self.err)
            attend = mtp.chunk_attention_args(out=att, out_lse=lse, **shared)
            mtp.mtp_chunk_attention(attend, *self._workspace("attend", mtp.mtp_chunk_attention_workspace_bytes(attend)), stream)
            weigh = mtp.key_weights_args(lse=lse, weights=self.weights[0], **shared)
            mtp.mtp_key_weights(weigh, *self._workspace("weigh", mtp.mtp_key_weights_workspace_bytes(weigh)), stream)
            x = x + F.linear(att.float().flatten(1), w["out"])
            x = x + F.linear(F.gelu(F.linear(F.layer_norm(x, x.shape[1:]), w["up"])), w["down"])
        return x, fed, cu

    def prefill(self, prompts):
        """prompts: a list of token ids per slot, two at least each; the last one waits for the first step."""
        longest = max(len(p) for p in prompts)
        tokens = torch.tensor([list(p) + [0] * (longest - len(p)) for p in prompts], dtype=torch.int32)
        new = torch.tensor([len(p) - 1 for p in prompts], dtype=torch.int32)
        self.last.copy_(torch.tensor([p[-1] for p in prompts]))
        self._forward(tokens[:, :longest - 1].contiguous().cuda(), new.cuda(), longest - 1)
        self.text += new.cuda()
        self._evict()

    def step(self):
        """Drafts, verifies, rolls back; the step's tokens [slots, drafts + 1] (-1 past a slot's), their counts."""
        m, n, stream = self.m, self.drafts + 1, torch.cuda.current_stream()
        i32 = dict(dtype=torch.int32, device="cuda")
        # the drafter's tokens, one after another, and the distributions that they were drawn from
        tokens, guess = [self.last], []
        for _ in range(self.drafts):
            guess.append(m.bigram[tokens[-1].long()])
            noise = torch.rand(self.slots, m.vocab, device="cuda", generator=self.gen).clamp(1e-7, 1 - 1e-6).log().neg().log().neg()
            tokens.append((guess[-1] + self.temperature[:, None].clamp(min=0) * noise).argmax(-1).int())
        tokens, guess = torch.stack(tokens, 1), torch.stack(guess + guess[-1:], 1)
        new = torch.where(self.done == 0, n, 0).int()
        x, fed, cu = self._forward(tokens.contiguous(), new, n)
        self.logits = F.linear(F.layer_norm(x, x.shape[1:]), m.head)
        # a slot's rows are together, the finished slots' left out
        order = torch.argsort((self.done != 0).int(), stable=True)
        self.guess = guess[order].flatten(0, 1).contiguous()
        self.numbers = torch.rand(self.slots * n, 2, device="cuda", generator=self.gen)
        out, counts, done = torch.empty(self.slots, n, **i32), torch.empty(self.slots, **i32), torch.empty(self.slots, **i32)
        verify = mtp.draft_verify_args(
            logits=self.logits, draft_logits=self.guess, temperature=self.temperature, tokens=fed, uniforms=self.numbers,
            cu_rows=cu, kv_lens=self.lens[0], out_tokens=out, out_counts=counts, out_kv_lens=self.lens[0], out_done=done,
            max_new=n, eos_id=self.eos, block_table=self.tables[0], page_refs=self.refs, page_size=self.page,
            err_word=self.err)
        mtp.mtp_draft_verify(verify, stream)
        self.text += counts
        self.last = torch.where(counts > 0, out.gather(1, (counts - 1).clamp(min=0).long()[:, None])[:, 0], self.last)
        self.done = torch.maximum(self.done, done)
        self.history.append(out)
        self._evict()
        return out, counts

    def _evict(self):
        if self.longest <= self.budget + self.slack:
            return
        args = mtp.cache_evict_args(
            kv_lens=self.lens[0], keep=self.keep, block_table=self.tables[0], page_refs=self.refs, weights=self.weights[0],
            kv_pool=self.pool, out_kv_lens=self.lens[1], out_block_table=self.tables[1], out_page_refs=self.refs,
            out_weights=self.weights[1], out_status=self.evicted, sinks=self.sinks, recent=self.recent)
        mtp.mtp_cache_evict(args, *self._workspace("evict", mtp.mtp_cache_evict_workspace_bytes(args)),
                            torch.cuda.current_stream())
        self.worst = torch.minimum(self.worst, self.evicted.min())
        for pair in (self.tables, self.lens, self.weights):
            pair.reverse()
        self.longest = self.budget

    def texts(self):
        """Every slot's tokens; checks what the GPU reported."""
        if int(self.worst) or int(self.err):
            raise RuntimeError(f"a step failed with status {int(self.worst)}, device error word {int(self.err)}")
        out = torch.cat(self.history, 1).tolist()
        return [[t for t in row if t >= 0] for row in out]


def main():
    model = Model()
    dec = SpeculativeDecoder(model, slots=4, budget=96, slack=32, recent=32)
    dec.prefill([[(7 * s + 3 * i) % model.vocab for i in range(20 + 30 * s)] for s in range(4)])
    kept = 0
    for _ in range(24):
        _, counts = dec.step()
        kept = kept + counts.float().mean()
    for s, tokens in enumerate(dec.texts()):
        print(f"slot {s}: {len(tokens)} tokens, {int(dec.lens[0][s])} cached, {tokens[:12]} ...")
    print(f"tokens a step and slot: {float(kept) / 24:.2f}")


if __name__ == "__main__":
    main()
