"""Limits of the context-free operators and of contexts whose prompts are held in 8 bits, checked on the host."""
import dataclasses

import pytest

import workloads as W
from paper_2606_31160_amd import binding as B
from tests.test_abi_host import _cfg, _seqs
from tests.test_operators_host import attn, cache, refused


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


@pytest.mark.parametrize("draft", [True, False])
def test_contexts_with_prompts_in_8_bits_hold_no_partials_that_nothing_writes(draft):
    """Sixteen scenes of 8192 tokens at the 7B target's heads.  Of the 8-bit context: half the prompts' bytes and their
    scales (8 bytes a page, layer and kv head); no bf16 attention's partials of the target (bf16 rows, two words, four
    of the readout, for each page, sequence, query head and row), but its own (a row block of 16 fp32 rows, their
    maxima and sums and a word, for each group)."""
    w = W.get("C5")
    if not draft:
        w = w.with_(draft=None)
    n, pages = {}, {}
    for flags in (0, B.SPEC_FLAG_KV8):
        cfg = _cfg(w.with_(draft=W.get("C5").draft), K=8, batch=16)
        if not draft:
            cfg.draft = B.dims(None)
        cfg.flags = flags
        seqs, keep = _seqs(w, cfg, prefix=8192, blocks=[])
        n[flags] = B.spec_workspace_bytes(cfg, seqs)
        pages[flags] = B.spec_debug_attn_pages(cfg, seqs)
        each = B.spec_seq_pages(cfg, seqs[0])
    t = w.target
    slots = 16 * 8192 * t.kv_heads * t.head_dim * t.layers * 2
    saved = slots - 16 * 128 * t.kv_heads * t.layers * 8
    rows = each * 16 * 9
    heads = t.q_heads - (w.draft.q_heads if draft else 0)
    saved += rows * heads * (2 * t.head_dim + 8 + 16)
    groups = 16 * t.kv_heads * -(-each // pages[B.SPEC_FLAG_KV8])
    blocks = 4                                    # of 9 x 7 rows
    own = groups * blocks * (16 * t.head_dim * 4 + 16 * 8 + 8)
    assert t.q_heads // t.kv_heads == 7
    assert abs(n[0] - n[B.SPEC_FLAG_KV8] - (saved - own)) <= 64 << 10     # page tables, alignment


@pytest.mark.parametrize("scale,fine", [(2.0 ** 127, True), (1e-45, True), (1.0001 * 2.0 ** 127, False), (3.4e38, False)])
def test_attention_scales_whose_product_with_log2_e_is_no_number_are_refused(scale, fine):
    """(A call that is fine otherwise ends at its workspace.)"""
    status, text = (3, "workspace") if fine else (1, "scale must be positive and at most 2^127")
    refused(lambda: attn(cache(), scale=scale), status, text)


def test_attention_takes_what_its_limits_say():
    """Each limit of a pass, and one more."""
    n = lambda c, *a: B.spec_kv8_attn_workspace_bytes(c, *a)  # noqa: E731
    one = cache(kv_heads=1)
    assert n(one, 1, 80, 13107, 1) > 0                                            # 80 x 13107 = 1048560 rows of a kv head
    refused(lambda: n(one, 1, 70, 14980, 1), 1, "rows*q_heads/kv_heads")          # 1048600
    assert n(cache(kv_heads=16384), 1, 1, 16384, 1) > 0                           # q_heads*head_dim = 2^20
    refused(lambda: n(cache(kv_heads=16385), 1, 1, 16385, 1), 1, "q_heads*head_dim")
    assert n(one, 4, 1, 1, 2 ** 25 - 1) > 0                                       # table_stride, and 2^27 pages less four
    refused(lambda: n(one, 1, 1, 1, 2 ** 25), 1, "table_stride")
    refused(lambda: n(one, 5, 1, 1, 2 ** 25 - 1), 1, "batch*kv_heads*table_stride")
