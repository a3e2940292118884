"""Contexts with prompts in 8 bits and more (sequence, kv head) pairs than CUs."""
import dataclasses

import numpy as np
import pytest

import workloads as W
from tests import _support as S
from tests.test_gpu_kv8_context import _oracle, _session

pytestmark = pytest.mark.gpu


def _workload():
    w = W.get("C1")
    prompts = [700 + 50 * b for b in range(9)]
    return w.with_(target=dataclasses.replace(w.target, q_heads=32, kv_heads=32), draft=None,
                   seqs=tuple(W.SeqLayout(p) for p in prompts), p_accept=(0.8,) * 9)


def test_verify_against_the_oracle_and_the_same_for_every_K():
    """288 pairs, 16 pages a group: a prompt's 10 to 17 pages in one or two groups.  Passes of 9 and 27 rows, whose
    products are the packed GEMV's (past 32 rows another form sums in another order, whatever the cache)."""
    w = _workload()
    T, _ = S.oracle_decoders(w, W.HostWeights(w))
    drafts = np.random.default_rng(1).integers(0, w.vocab, (9, 2)).astype(np.int32)
    first = []
    for K in (2, 0):
        s = _session(w, K=K, with_draft=False)
        s.verify(drafts if K else None, logits=True)
        first.append(s.logits[:, 0].clone())
        if K:
            gl = s.logits.float().cpu().numpy()
            for b in (0, 8):
                r = _oracle(w.with_(K=2), b, T, None, s, with_draft=False).verify(drafts[b])
                for j in range(3):
                    assert S.normwise_err(gl[b, j], r.logits[j]) <= S.LOGIT_RTOL, (b, j)
        s.sync()
        s.close()
    assert first[0].equal(first[1])
