"""The example that learns from its own answers scores them as they were drawn, as far as a score can."""
import os
import sys

import pytest

import paper_2401_15207_amd as H

pytestmark = pytest.mark.gpu


def test_answers_are_scored_at_the_temperature_they_are_drawn_at(monkeypatch):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import learn_from_own_answers as E
    drawn, scored = [], []
    logprob, score = H.kernel_token_logprob, H.HiftModel.score

    def look(logits, vocab, targets, scale, *more, **named):
        drawn.append(scale)
        return logprob(logits, vocab, targets, scale, *more, **named)

    def at(self, tokens, targets, group_id=-1, temperature=1.0, top=0):
        scored.append(1.0 / temperature)
        return score(self, tokens, targets, group_id, temperature, top)

    monkeypatch.setattr(H, "kernel_token_logprob", look)
    monkeypatch.setattr(H.HiftModel, "score", at)
    E.run(workload="C1", batch=2, sweeps=1, prompt=4, answer=3, say=lambda *a, **k: None)
    assert len(scored) == 4 and len(drawn) == 12 and set(scored) == set(drawn)
