"""Limits of the context-free operators and of contexts whose prompts are held in 8 bits, checked on the host."""
import dataclasses

import pytest

import workloads as W
from paper_2606_31160_amd import binding as B
from tests.test_abi_host import _cfg, _seqs


def _many_heads(scenes, kv_heads, prompt, K=8):
    w = W.get("C1")
    w = w.with_(target=dataclasses.replace(w.target, q_heads=kv_heads, kv_heads=kv_heads))
    cfg = _cfg(w, K=K, batch=scenes)
    cfg.flags = B.SPEC_FLAG_KV8
    return (cfg, *_seqs(w, cfg, prefix=prompt, blocks=[]))


@pytest.mark.parametrize("scenes,kv_heads,prompt,pages", [(16, 32, 8192, 16), (9, 32, 600, 12), (9, 32, 200, 4)])
def test_pages_of_a_group_grow_with_long_prompts_of_many_heads(scenes, kv_heads, prompt, pages):
    """More sequences times kv heads than the 256 CUs: groups of 4 pages would be several a CU."""
    for K in (0, 8):
        cfg, seqs, keep = _many_heads(scenes, kv_heads, prompt, K)
        assert B.spec_debug_attn_pages(cfg, seqs) == pages
