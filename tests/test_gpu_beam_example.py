"""The beam-search example against the oracle: whole sequences recomputed in 64 bits, beam by beam.

The oracle follows the GPU's choices (which beams, which tokens), so that a near-tie changes nothing: after every step
each live beam's logits are compared, and the selected scores with the best of the oracle's."""
import importlib.util
import os

import numpy as np
import pytest

import synth
from gpu_util import LOGIT_ATOL, lib_module
from oracle.model import ARDecoder
from oracle.select import head_logits

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    lib_module()
    spec = importlib.util.spec_from_file_location("beam_search_example", os.path.join(ROOT, "examples", "beam_search.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _logits(o, model, phones, codes):
    """Head 1's logits behind a sequence of phonemes and codes."""
    tokens = np.concatenate([phones, codes])
    hidden = o.forward(tokens, np.arange(len(tokens)) < len(phones), o.new_cache())[-1]
    return head_logits(hidden, o.w, 1, model.ln_eps)[0]


@pytest.mark.parametrize("beams,page,eos_bias", [(4, 16, 1.0), (3, 32, -4.0), (1, 16, -4.0)])
def test_beam_search_follows_the_oracle(beams, page, eos_bias):
    model, batch, steps = synth.TINY, 2, 10
    weights = synth.make_weights(model, eos_bias=eos_bias)
    search = _example().BeamSearch(model, weights, batch, beams, max_ctx=64, page_size=page)
    prompts = [synth.make_prompt(i, 9 + 7 * i, 14 + 5 * i, model.phone_vocab) for i in range(batch)]
    o = ARDecoder(model, weights)
    seqs = [[list(codes)] + [None] * (beams - 1) for _, codes in prompts]
    scores = np.full((batch, beams), -np.inf)
    scores[:, 0] = 0.0
    done = np.zeros((batch, beams), bool)
    ended = False
    for step in range(steps):
        search.prefill(prompts) if step == 0 else search.step()
        logits = search.logits.double().cpu().numpy()
        parent, token, got = search.parent.cpu().numpy(), search.token.cpu().numpy(), search.scores.double().cpu().numpy()
        for b, (phones, _) in enumerate(prompts):
            total = np.full((beams, model.codec_vocab), -np.inf)
            for w in range(beams):
                if not np.isfinite(scores[b, w]):
                    continue
                if done[b, w]:
                    total[w, model.eos_id] = scores[b, w]
                    continue
                ref = _logits(o, model, phones, np.array(seqs[b][w]))
                assert np.abs(logits[b, w] - ref).max() <= LOGIT_ATOL, (step, b, w)
                total[w] = scores[b, w] + ref - np.logaddexp.reduce(ref)
            best = np.sort(total.ravel())[::-1][:beams]
            # a step's log-probability errs by two logits' error at most; errors of the steps add up
            assert np.abs(got[b] - best).max() <= 2 * LOGIT_ATOL * (step + 1), (step, b)
            chosen = total[parent[b], token[b]]
            assert np.abs(got[b] - chosen).max() <= 2 * LOGIT_ATOL * (step + 1), (step, b)
            old, was = seqs[b], done[b].copy()
            seqs[b] = [list(old[p]) if was[p] else list(old[p]) + [int(t)] for p, t in zip(parent[b], token[b])]
            done[b] = [was[p] or t == model.eos_id for p, t in zip(parent[b], token[b])]
            scores[b] = chosen
        assert np.array_equal(search.done.cpu().numpy() != 0, done)
        ended |= bool(done.any())
        lens = search.lens[0].cpu().numpy().reshape(batch, beams)
        # every token but the one selected last is cached
        assert all(lens[b, w] == len(prompts[b][0]) + len(seqs[b][w]) - 1 for b in range(batch) for w in range(beams))
        held = np.zeros(search.n_pages, int)
        table = search.tables[0].cpu().numpy()
        np.add.at(held, table[table >= 0], 1)
        assert np.array_equal(held, search.refs.cpu().numpy())
    assert ended == (eos_bias > 0)
    for b, (tokens, score) in enumerate(search.best()):
        assert abs(score - scores[b, 0]) <= 2 * LOGIT_ATOL * steps and tokens == seqs[b][0][len(prompts[b][1]):]
