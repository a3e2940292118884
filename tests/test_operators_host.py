"""Refusals of the context-free operators: checked on the host before anything touches a GPU."""
import ctypes

import pytest

from paper_2606_31160_amd import binding as B

P = 1 << 20   # stands for a device pointer; never read


def cache(**kw):
    d = dict(kv_heads=2, head_dim=64, pages8=3, k8=P, v8=P, k_scale=P, v_scale=P, pages16=2, k16=P, v16=P)
    d.update(kw)
    return B.kv8(**d)


def attn(c, **kw):
    d = dict(batch=2, rows=3, q_heads=4, d_table=P, table_stride=5, d_packed=P, d_visible=P, q=P, q_stride=256, scale=0.125,
             out=P, out_stride=256, d_lse=0, d_err=0, workspace=P, workspace_bytes=0, stream=0)
    d.update(kw)
    B.spec_kv8_attn(c, *(d[k] for k in ("batch", "rows", "q_heads", "d_table", "table_stride", "d_packed", "d_visible", "q",
                                        "q_stride", "scale", "out", "out_stride", "d_lse", "d_err", "workspace",
                                        "workspace_bytes", "stream")))


def refused(f, status, text):
    with pytest.raises(B.SpecError) as e:
        f()
    assert e.value.status == status and text in str(e.value), str(e.value)


INVAL, CAPACITY = 1, 3


@pytest.mark.parametrize("kw,text", [
    (dict(head_dim=96), "head_dim"), (dict(kv_heads=0), "kv_heads"), (dict(kv_heads=3), "q_heads"),
    (dict(pages8=-1), "page count"), (dict(pages16=-1), "page count"), (dict(k8=0), "8-bit pages"),
    (dict(v8=P + 8), "8-bit pages"), (dict(k_scale=0), "8-bit pages"), (dict(v_scale=P + 2), "8-bit pages"),
    (dict(k16=0), "bf16 pages"), (dict(v16=P + 4), "bf16 pages")])
def test_attention_refuses_a_bad_cache(kw, text):
    refused(lambda: attn(cache(**kw)), INVAL, text)
    refused(lambda: B.spec_kv8_attn_workspace_bytes(cache(**kw), 2, 3, 4, 5), INVAL, text)


@pytest.mark.parametrize("kw,text", [
    (dict(batch=0), "batch"), (dict(rows=0), "batch"), (dict(batch=20, rows=9), "SPEC_MAX_ROWS"),
    (dict(batch=2 ** 30, rows=2 ** 30), "SPEC_MAX_ROWS"), (dict(q_heads=0), "q_heads"), (dict(q_heads=5), "q_heads"),
    (dict(table_stride=0), "table_stride"), (dict(table_stride=2 ** 30), "table_stride"), (dict(q_stride=248), "q_stride"),
    (dict(q_stride=260), "q_stride"), (dict(out_stride=255), "q_stride"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(scale=0.0), "scale"), (dict(scale=-0.1), "scale"), (dict(q=P + 2), "misaligned"), (dict(q=0), "null"), (dict(out=P + 8), "misaligned"),
    (dict(d_table=0), "null"), (dict(d_packed=P + 1), "misaligned"), (dict(d_visible=0), "null"), (dict(d_lse=P + 2), "misaligned"),
    (dict(d_err=P + 2), "misaligned"), (dict(workspace=0), "workspace"), (dict(workspace=P + 16), "workspace")])
def test_attention_refuses_bad_arguments(kw, text):
    refused(lambda: attn(cache(), **kw), INVAL, text)


@pytest.mark.parametrize("cache_kw,kw,text", [
    (dict(kv_heads=1), dict(batch=1, rows=70, q_heads=16384), "rows*q_heads/kv_heads"),
    (dict(kv_heads=64), dict(batch=2, rows=1, q_heads=64, table_stride=2 ** 20 + 1), "batch*kv_heads*table_stride")])
def test_attention_refuses_what_no_grid_holds(cache_kw, kw, text):
    refused(lambda: attn(cache(**cache_kw), q_stride=1 << 20, out_stride=1 << 20, **kw), INVAL, text)


def test_attention_refuses_a_small_workspace():
    n = B.spec_kv8_attn_workspace_bytes(cache(), 2, 3, 4, 5)
    assert n > 0
    refused(lambda: attn(cache(), workspace_bytes=n - 1), CAPACITY, "spec_kv8_attn_workspace_bytes")
    refused(lambda: attn(None), INVAL, "null cache")


def test_attention_workspace_grows_with_the_pass_only():
    """The groups of a call are bounded by what the chip runs at once, not by the cache's length."""
    c = cache(kv_heads=4, head_dim=128)
    short, long = (B.spec_kv8_attn_workspace_bytes(c, 1, 9, 28, n) for n in (64, 2048))
    assert short <= long <= 32 << 20
    assert B.spec_kv8_attn_workspace_bytes(c, 1, 9, 28, 1) < short


@pytest.mark.parametrize("kw,text", [
    (dict(k=0), "null"), (dict(v=P + 8), "misaligned"), (dict(row_stride=120), "row_stride"), (dict(row_stride=132), "row_stride"),
    (dict(rows=0), "rows"), (dict(rows=-5), "rows"), (dict(rows=2 ** 28 + 1), "rows"), (dict(d_pages=0), "null"), (dict(d_err=P + 1), "misaligned")])
def test_pack_refuses_bad_arguments(kw, text):
    d = dict(k=P, v=P, row_stride=128, rows=64, d_pages=P, d_err=0, stream=0)
    d.update(kw)
    refused(lambda: B.spec_kv8_pack(cache(), *d.values()), INVAL, text)


@pytest.mark.parametrize("kw,text", [(dict(head_dim=32), "head_dim"), (dict(pages8=0, k8=0), "no 8-bit pages"), (dict(kv_heads=0), "kv_heads"),
                                     (dict(kv_heads=70000), "kv heads"), (dict(v8=0), "8-bit pages")])
def test_pack_refuses_a_bad_cache(kw, text):
    refused(lambda: B.spec_kv8_pack(cache(**kw), P, P, 1 << 24, 64, P), INVAL, text)


def scores(**kw):
    d = dict(logits=P, dtype=B.SPEC_BF16, rows=2, vocab=1000, row_stride=1000, d_tokens=P, n_tokens=1, top=5, d_logprob=P,
             d_entropy=P, d_top_token=P, d_top_logprob=P, workspace=P, workspace_bytes=1 << 20, stream=0)
    d.update(kw)
    B.spec_logprobs(*d.values())


@pytest.mark.parametrize("kw,text", [
    (dict(logits=0), "null"), (dict(logits=P + 1), "misaligned"), (dict(logits=P + 2, dtype=B.SPEC_F32), "misaligned"),
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=0), "rows"), (dict(rows=65536), "rows"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), "vocab"), (dict(row_stride=999), "row_stride"),
    (dict(n_tokens=-1), "n_tokens"), (dict(d_tokens=0), "null"), (dict(d_logprob=0), "null"), (dict(top=33), "top"),
    (dict(top=-1), "top"), (dict(vocab=4, row_stride=4), "top"), (dict(d_top_token=0), "null"), (dict(d_top_logprob=P + 2), "misaligned"),
    (dict(d_entropy=P + 2), "misaligned"), (dict(workspace=0), "workspace"), (dict(workspace=P + 128), "workspace")])
def test_logprobs_refuses_bad_arguments(kw, text):
    refused(lambda: scores(**kw), INVAL, text)


def test_logprobs_refuses_a_small_workspace():
    n = B.spec_logprobs_workspace_bytes(2, 1000, 5)
    refused(lambda: scores(workspace_bytes=n - 1), CAPACITY, "spec_logprobs_workspace_bytes")
    for bad in ((0, 10, 1), (1, 0, 0), (1, 10, 11), (1, 100, 33)):
        refused(lambda: B.spec_logprobs_workspace_bytes(*bad), INVAL, "spec_logprobs_workspace_bytes")
    assert B.lib().spec_logprobs_workspace_bytes(1, 10, 1, None) == INVAL
    assert B.lib().spec_kv8_attn_workspace_bytes(ctypes.byref(cache()), 1, 1, 4, 1, None) == INVAL


def test_contexts_with_prompts_in_8_bits_take_less_workspace():
    import workloads as W
    from tests.test_abi_host import _blocks, _cfg, _seqs
    w = W.get("C1")
    n = []
    for flags in (0, B.SPEC_FLAG_KV8):
        cfg = _cfg(w)
        cfg.flags = flags
        seqs, keep = _seqs(w, cfg, blocks=_blocks(w))
        n.append(B.spec_workspace_bytes(cfg, seqs))
        assert B.spec_debug_attn_pages(cfg, seqs) >= 1
    assert n[1] < n[0]
