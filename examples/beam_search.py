"""Beam search over codec tokens on a paged cache of the program's own.

The codec model of this repository, its blocks' products in torch, its cache and its search in
the package's paged operators: every step plans the pages and rows of the new tokens, appends
their keys and values, attends each chunk over what is cached, selects the best continuations of
every utterance's beams and reorders the cache.  A prompt is prefilled once, in the first beam; the
other beams share its pages from the first selection on.  Nothing waits for the host between steps.

    python examples/beam_search.py
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2410_13839_gb300 import mtp  # noqa: E402


class BeamSearch:
    """Beams of `batch` utterances; slots are utterance * beams + beam."""

    def __init__(self, model, weights, batch, beams, max_ctx, page_size=16, spare_pages=None):
        self.m, self.batch, self.beams, self.page = model, batch, beams, page_size
        self.w = {k: torch.tensor(v, dtype=torch.float32, device="cuda") for k, v in weights.items()}
        self.slots = slots = batch * beams
        self.stride = -(-max_ctx // page_size)
        self.n_pages = slots * self.stride + (slots if spare_pages is None else spare_pages)
        self.heads, self.dim = model.n_attn_heads, model.d_model // model.n_attn_heads
        i32 = dict(dtype=torch.int32, device="cuda")
        self.pool = torch.zeros(self.n_pages, model.layers, 2, self.heads, page_size, self.dim, dtype=torch.bfloat16,
                                device="cuda")
        self.tables = [torch.full((slots, self.stride), -1, **i32) for _ in range(2)]
        self.lens = [torch.zeros(slots, **i32) for _ in range(2)]
        self.refs = torch.zeros(self.n_pages, **i32)
        self.scores = torch.full((batch, beams), -float("inf"), device="cuda")
        self.scores[:, 0] = 0.0  # the search starts from one beam
        self.done = torch.zeros(batch, beams, **i32)
        self.parent, self.token = torch.zeros(batch, beams, **i32), torch.zeros(batch, beams, **i32)
        self.status, self.copied = torch.zeros(4, **i32), torch.zeros(4, **i32)
        self.worst, self.err = torch.zeros((), **i32), torch.zeros(1, **i32)
        self.workspaces = {}
        self.history = []
        self.longest = 0  # a bound of the slots' lengths, known without asking the GPU

    def _workspace(self, name, nbytes):
        """One that is kept, zeroed when it is made: the operators leave their counters zero."""
        if name not in self.workspaces or self.workspaces[name].numel() < nbytes:
            self.workspaces[name] = torch.zeros(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        return self.workspaces[name], nbytes

    def _position(self, pos):
        d = self.m.d_model
        freq = torch.pow(10000.0, -2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
        angle = pos.double()[:, None] * freq
        return torch.stack([angle.sin(), angle.cos()], -1).flatten(1).float()

    def _plan(self, new_lens, max_rows):
        i32 = dict(dtype=torch.int32, device="cuda")
        out = dict(out_cu_rows=torch.empty(self.slots + 1, **i32), out_row_seq=torch.empty(max_rows, **i32),
                   out_row_pos=torch.empty(max_rows, **i32),
                   out_slot_map=torch.empty(max_rows, dtype=torch.int64, device="cuda"))
        mtp.mtp_page_plan(mtp.page_plan_args(
            kv_lens=self.lens[0], new_lens=new_lens, block_table=self.tables[0], page_refs=self.refs,
            out_kv_lens=self.lens[0], out_page_refs=self.refs, out_status=self.status, page_size=self.page, **out),
            torch.cuda.current_stream())
        return out["out_cu_rows"], out["out_row_pos"], out["out_slot_map"]

    def _blocks(self, x, slot_map, cu_rows, max_new):
        """The block stack on rows x, whose keys and values go to slot_map."""
        stream, w, d = torch.cuda.current_stream(), self.w, self.m.d_model
        q16 = torch.empty(x.shape[0], self.heads, self.dim, dtype=torch.bfloat16, device="cuda")
        att = torch.zeros_like(q16)
        for layer in range(self.m.layers):
            p = f"layers.{layer}."
            h = F.layer_norm(x, (d,), w[p + "ln1_g"], w[p + "ln1_b"], self.m.ln_eps)
            qkv = F.linear(h, w[p + "wqkv"], w[p + "bqkv"]).view(-1, 3, self.heads, self.dim)
            mtp.mtp_cache_append(mtp.cache_append_args(k=qkv[:, 1], v=qkv[:, 2], slot_map=slot_map, kv_pool=self.pool,
                                                       layer=layer), stream)
            q16.copy_(qkv[:, 0])
            args = mtp.chunk_attention_args(q=q16, kv_pool=self.pool, layer=layer, block_table=self.tables[0],
                                            cu_rows=cu_rows, kv_lens=self.lens[0], out=att, scale=self.dim ** -0.5,
                                            max_new=max_new, max_keys=self.longest, err_word=self.err)
            mtp.mtp_chunk_attention(args, *self._workspace("attend", mtp.mtp_chunk_attention_workspace_bytes(args)), stream)
            x = x + F.linear(att.float().flatten(1), w[p + "wo"], w[p + "bo"])
            h = F.layer_norm(x, (d,), w[p + "ln2_g"], w[p + "ln2_b"], self.m.ln_eps)
            x = x + F.linear(F.gelu(F.linear(h, w[p + "w1"], w[p + "b1"])), w[p + "w2"], w[p + "b2"])
        return x

    def _advance(self, embedded, new_lens, max_new):
        """Feeds every slot its new rows; selects and reorders."""
        self.longest += max_new
        rows = embedded.shape[0]
        cu_rows, pos, slot_map = self._plan(new_lens, rows)
        x = self._blocks(embedded + self._position(pos.clamp(min=0)), slot_map, cu_rows, max_new)
        last = x[(cu_rows[1:].long() - 1).clamp(min=0)]  # (of a slot without rows: anything)
        z = F.layer_norm(last, (self.m.d_model,), self.w["lnf_g"], self.w["lnf_b"], self.m.ln_eps)
        self.logits = F.linear(z, self.w["w_heads"][0], self.w["b_heads"][0]).view(self.batch, self.beams, -1)
        stream, done, scores = torch.cuda.current_stream(), torch.empty_like(self.done), torch.empty_like(self.scores)
        args = mtp.beam_select_args(logits=self.logits, scores=self.scores, done=self.done, eos_id=self.m.eos_id,
                                    k=self.beams, out_scores=scores, out_parent=self.parent, out_token=self.token,
                                    out_done=done)
        mtp.mtp_beam_select(args, *self._workspace("select", mtp.mtp_beam_select_workspace_bytes(args)), stream)
        args = mtp.beam_reorder_args(parent=self.parent, block_table=self.tables[0], kv_lens=self.lens[0],
                                     page_refs=self.refs, kv_pool=self.pool, out_block_table=self.tables[1],
                                     out_kv_lens=self.lens[1], out_page_refs=self.refs, out_status=self.copied)
        mtp.mtp_beam_reorder(args, *self._workspace("reorder", mtp.mtp_beam_reorder_workspace_bytes(args)), stream)
        self.worst = torch.minimum(self.worst, torch.minimum(self.status[0], self.copied[0]))
        self.tables.reverse()
        self.lens.reverse()
        self.scores, self.done = scores, done
        at = self.parent.long()
        self.history = [h.gather(1, at) for h in self.history] + [self.token.clone()]

    def prefill(self, prompts):
        """prompts: (phonemes, acoustic codes) of every utterance."""
        rows, new = [], torch.zeros(self.slots, dtype=torch.int32)
        for b, (phones, codes) in enumerate(prompts):
            ids = lambda x: torch.as_tensor(x, dtype=torch.int64, device="cuda")  # noqa: E731
            rows += [self.w["tok_phone"][ids(phones)], self.w["tok_codec"][ids(codes)]]
            new[b * self.beams] = len(phones) + len(codes)
        self._advance(torch.cat(rows), new.cuda(), int(new.max()))

    def step(self):
        """Feeds the selected tokens; finished beams get none."""
        alive = self.done.flatten() == 0
        order = torch.argsort((~alive).int(), stable=True)  # the rows of the beams that go on, in the slots' order
        self._advance(self.w["tok_codec"][self.token.flatten().long()[order]], alive.int(), 1)

    def best(self):
        """(tokens, score) of every utterance's best beam; checks what the GPU reported."""
        if int(self.worst) or int(self.err):
            raise RuntimeError(f"a step failed with status {int(self.worst)}, device error word {int(self.err)}")
        tokens = torch.stack(self.history, -1).cpu()
        out = []
        for b in range(self.batch):
            seq = tokens[b, 0].tolist()
            out.append((seq[:seq.index(self.m.eos_id) + 1] if self.m.eos_id in seq else seq, float(self.scores[b, 0])))
        return out


def main():
    import synth
    model = synth.TINY
    search = BeamSearch(model, synth.make_weights(model), batch=2, beams=4, max_ctx=80)
    search.prefill([synth.make_prompt(i, 12 + i, 20, model.phone_vocab) for i in range(2)])
    for _ in range(20):
        search.step()
    for i, (tokens, score) in enumerate(search.best()):
        print(f"utterance {i}: log-probability {score:.3f}, codes {tokens}")


if __name__ == "__main__":
    main()
