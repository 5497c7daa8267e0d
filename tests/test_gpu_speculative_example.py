"""The speculative decoding example: every operator's step against its plain form on the step's own inputs, greedy decoding
against the model recomputed in 64 bits, and the cache's books after every step."""
import importlib.util
import os

import pytest

from gpu_util import lib_module
from test_gpu_cache_evict import _oracle as evicted
from test_gpu_draft_verify import _oracle as verified

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    lib_module()
    spec = importlib.util.spec_from_file_location("speculative_example", os.path.join(ROOT, "examples", "speculative_decoding.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _books(torch, dec):
    """Counts are the tables' holdings; no slot is longer than its table."""
    held = torch.zeros(dec.n_pages, dtype=torch.int64)
    for s, n in enumerate(dec.lens[0].tolist()):
        pages = dec.tables[0][s].tolist()
        used = -(-n // dec.page)
        assert all(p >= 0 for p in pages[:used]) and all(p == -1 for p in pages[used:]), (s, n, pages)
        for p in pages[:used]:
            held[p] += 1
    assert held.tolist() == dec.refs.tolist()


def _logits64(torch, F, m, tokens, turns):
    """The model's logits behind every token of a text, in 64 bits, positions from 0."""
    d = m.heads * m.dim
    x = m.embed[torch.tensor(tokens, device="cuda")].double()
    angle = torch.arange(len(tokens), device="cuda", dtype=torch.float64)[:, None] * (
        turns.double() % 2.0 ** 64 / 2.0 ** 64 * 2 * torch.pi)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turn(y):
        a, b = y[..., :m.dim // 2], y[..., m.dim // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    mask = torch.ones(len(tokens), len(tokens), dtype=torch.bool, device="cuda").tril()
    for w in m.blocks:
        qkv = F.linear(F.layer_norm(x, (d,)), w["qkv"].double()).view(len(tokens), -1, m.dim)
        q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
        g = m.heads // m.kv_heads
        k, v = turn(k).repeat_interleave(g, 1), v.repeat_interleave(g, 1)
        s = torch.einsum("nhd,thd->hnt", turn(q), k) * m.dim ** -0.5
        o = torch.einsum("hnt,thd->nhd", s.masked_fill(~mask, -torch.inf).softmax(-1), v)
        x = x + F.linear(o.flatten(1), w["out"].double())
        x = x + F.linear(F.gelu(F.linear(F.layer_norm(x, (d,)), w["up"].double())), w["down"].double())
    return F.linear(F.layer_norm(x, (d,)), m.head.double())


def test_greedy_decoding_is_the_models_own():
    """At temperature 0 the drafts change nothing but the number of steps: every token is the likeliest one, but for
    those within bf16's reach (keys, values and queries of a few hundred products are rounded to 2^-8)."""
    torch = pytest.importorskip("torch")
    import torch.nn.functional as F
    ex = _example()
    model = ex.Model(seed=3, vocab=300, heads=4, kv_heads=2)
    dec = ex.SpeculativeDecoder(model, slots=3, drafts=3, budget=400, temperature=0.0)
    prompts = [[(11 * s + 5 * i) % 300 for i in range(n)] for s, n in enumerate((2, 17, 40))]
    dec.prefill(prompts)
    several = 0
    for _ in range(12):
        _, counts = dec.step()
        several += int((counts > 1).sum())
        _books(torch, dec)
    assert several > 0  # some drafts were kept
    for p, text in zip(prompts, dec.texts()):
        logits = _logits64(torch, F, model, p + text[:-1], dec.turns)[len(p) - 1:]
        best = logits.max(-1).values
        got = logits.gather(1, torch.tensor(text, device="cuda")[:, None])[:, 0]
        assert float((best - got).max()) <= 0.25  # (logits have a spread of 4; a mistaken token is off by several)


@pytest.mark.parametrize("temperature,eos", [(1.0, 7), (0.6, -1)])
def test_every_step_follows_the_rules(temperature, eos):
    torch = pytest.importorskip("torch")
    ex = _example()
    model = ex.Model(seed=5, vocab=200, heads=8, kv_heads=2, sharpness=3.0)
    dec = ex.SpeculativeDecoder(model, slots=4, drafts=4, budget=64, slack=16, sinks=4, recent=20, temperature=temperature, eos_id=eos, max_prompt=200)
    evictions = []
    plain_evict = dec._evict

    def watched():
        if dec.longest <= dec.budget + dec.slack:
            return plain_evict()
        st = dict(table=dec.tables[0].cpu(), refs=dec.refs.tolist(), lens=dec.lens[0].tolist(), weights=dec.weights[0].clone(),
                  pool=dec.pool.clone(), page=dec.page)
        want = evicted(torch, st, [dec.budget] * dec.slots, dec.sinks, dec.recent)
        plain_evict()
        lens, table, refs, w, pool = want
        assert dec.lens[0].tolist() == lens and dec.tables[0].tolist() == table and dec.refs.tolist() == refs
        assert torch.equal(dec.pool.view(torch.int16), pool.view(torch.int16))
        for s, n in enumerate(lens):
            assert torch.equal(dec.weights[0][s, ..., :n], w[s, ..., :n])
        evictions.append(1)
    dec._evict = watched
    dec.prefill([[(13 * s + 3 * i) % 200 for i in range(n)] for s, n in enumerate((2, 30, 90, 150))])
    given = dec.weights[0].sum(-1)
    for _ in range(14):
        before = (dec.lens[0].tolist(), dec.done.tolist(), dec.text.tolist())
        seen = {}
        plain_verify = ex.mtp.mtp_draft_verify

        def verify(args, stream):
            seen.update(lens=dec.lens[0].tolist(), table=dec.tables[0].tolist(), refs=dec.refs.tolist())
            plain_verify(args, stream)
        ex.mtp.mtp_draft_verify = verify
        evict, dec._evict = dec._evict, lambda: None
        fed = {}
        forward = dec._forward

        def watch(*a):
            fed["out"] = forward(*a)
            return fed["out"]
        dec._forward = watch
        try:
            out, counts = dec.step()
        finally:
            ex.mtp.mtp_draft_verify, dec._evict, dec._forward = plain_verify, evict, forward
        new = [0 if d else 5 for d in before[1]]
        rows = sum(new)
        assert seen["lens"] == [n + a for n, a in zip(before[0], new)]
        case = dict(new=new, logits=dec.logits[:rows].double().cpu().numpy(), draft=dec.guess[:rows].double().cpu().numpy(),
                    temperature=[float(t) for t in dec.temperature.tolist()], tokens=fed["out"][1][:rows].tolist(),
                    uniforms=dec.numbers.tolist(), lens=seen["lens"], table=seen["table"], refs=seen["refs"], page=dec.page,
                    max_new=5, eos=eos)
        tokens, n, lens, done, table, refs = verified(case)
        assert out.tolist() == tokens and counts.tolist() == n and dec.lens[0].tolist() == lens
        assert dec.tables[0].tolist() == table and dec.refs.tolist() == refs
        assert dec.done.tolist() == [max(a, b) for a, b in zip(before[1], done)]
        _books(torch, dec)
        dec._evict()
        _books(torch, dec)
        assert all(m <= dec.budget + dec.slack + 5 for m in dec.lens[0].tolist())
    assert len(evictions) >= 2 and bool((given > 0).all())
    dec.texts()
