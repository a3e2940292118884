"""Refusals of the operators of a tree's pass: checked on the host before anything touches a GPU."""
import ctypes

import pytest

from paper_2606_31160_amd import binding as B

P = 1 << 24   # stands for a device pointer; never read
INVAL, CAPACITY = 1, 3


def cache(**kw):
    d = dict(kv_heads=2, head_dim=64, pages=3, k=P, v=P, layers=2, layer_stride=3 * 2 * 64 * 64)
    d.update(kw)
    return B.kv(**d)


def rows(**kw):
    d = dict(batch=2, rows=9, d_first=P, d_len=2 * P, d_table=3 * P, table_stride=5, d_parent=4 * P, d_err=5 * P)
    d.update(kw)
    return B.rows(**d)


def rope(**kw):
    d = dict(base=10000.0, section=(8, 12, 12), interleaved=0)
    d.update(kw)
    return B.rope(**d)


def append(c=None, r=None, o=None, **kw):
    d = dict(layer=0, d_pos=P, q_heads=4, q=P, q_stride=256, k=P, v=P, kv_stride=128, q_out=2 * P, q_out_stride=256, stream=0)
    d.update(kw)
    layer = d.pop("layer")
    B.spec_kv_append(c or cache(), layer, r or rows(), o or rope(), *d.values())


def attn(c=None, r=None, **kw):
    d = dict(layer=0, q_heads=4, q=P, q_stride=256, scale=0.125, out=P, out_stride=256, d_lse=0, workspace=P, workspace_bytes=0,
             stream=0)
    d.update(kw)
    layer = d.pop("layer")
    B.spec_tree_attn(c or cache(), layer, r or rows(), *d.values())


def commit(c=None, r=None, **kw):
    d = dict(d_tokens=6 * P, d_greedy=7 * P, stop_token=-1, d_budget=0, d_path=8 * P, d_committed=9 * P, d_n=10 * P,
             d_new_len=11 * P, stream=0)
    d.update(kw)
    B.spec_tree_commit(c or cache(), r or rows(), *d.values())


def refused(f, status, text):
    with pytest.raises(B.SpecError) as e:
        f()
    assert e.value.status == status and text in str(e.value), str(e.value)


@pytest.mark.parametrize("kw,text", [
    (dict(head_dim=96), "head_dim"), (dict(kv_heads=0), "kv_heads"), (dict(kv_heads=65536), "kv_heads"), (dict(pages=0), "pages"),
    (dict(layers=0), "layers"), (dict(layers=257), "layers"), (dict(layer_stride=3 * 2 * 64 * 64 - 8), "layer_stride"),
    (dict(layer_stride=3 * 2 * 64 * 64 + 4), "layer_stride"), (dict(layer_stride=-8), "layer_stride"),
    (dict(layer_stride=(1 << 63) - 8), "layer_stride"), (dict(k=0), "null"), (dict(v=P + 8), "misaligned")])
def test_a_bad_cache_is_refused(kw, text):
    for f in (append, attn, commit):
        refused(lambda: f(cache(**kw)), INVAL, text)
    refused(lambda: B.spec_tree_attn_workspace_bytes(cache(**kw), rows(), 4), INVAL, text)


def test_one_layer_needs_no_stride():
    assert B.spec_tree_attn_workspace_bytes(cache(layers=1, layer_stride=0), rows(), 4) > 0


@pytest.mark.parametrize("kw,text", [
    (dict(batch=0), "batch"), (dict(batch=161), "batch"), (dict(rows=0), "rows"), (dict(rows=161), "rows"),
    (dict(table_stride=0), "table_stride"), (dict(table_stride=(1 << 25) - 15), "table_stride"), (dict(d_first=0), "null"),
    (dict(d_len=P + 2), "misaligned"), (dict(d_table=0), "null"), (dict(d_parent=P + 1), "misaligned"), (dict(d_err=P + 2), "misaligned")])
def test_bad_rows_are_refused(kw, text):
    for f in (lambda r: append(r=r, d_pos=0), lambda r: attn(r=r), lambda r: commit(r=r)):
        refused(lambda: f(rows(**kw)), INVAL, text)
    refused(lambda: B.spec_tree_attn_workspace_bytes(cache(), rows(**kw), 4), INVAL, text)


def test_null_descriptions_are_refused():
    L = B.lib()
    c, r, o = cache(), rows(), rope()
    assert L.spec_kv_append(None, 0, r, o, P, 0, 0, 0, P, P, 128, 0, 0, 0) == INVAL
    assert L.spec_kv_append(c, 0, None, o, P, 0, 0, 0, P, P, 128, 0, 0, 0) == INVAL
    assert L.spec_kv_append(c, 0, r, None, P, 0, 0, 0, P, P, 128, 0, 0, 0) == INVAL
    assert L.spec_tree_attn(None, 0, r, 4, P, 256, 1.0, P, 256, 0, P, 1 << 30, 0) == INVAL
    assert L.spec_tree_attn(c, 0, None, 4, P, 256, 1.0, P, 256, 0, P, 1 << 30, 0) == INVAL
    assert L.spec_tree_commit(None, r, P, P, -1, 0, 0, 0, 0, 0, 0) == INVAL
    assert L.spec_tree_commit(c, None, P, P, -1, 0, 0, 0, 0, 0, 0) == INVAL
    assert L.spec_tree_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 4, None) == INVAL


@pytest.mark.parametrize("kw,text", [
    (dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(q_heads=-1), "q_heads"), (dict(q_heads=16385, q_stride=1 << 22), "q_heads"),
    (dict(q_stride=248), "q_stride"), (dict(q_stride=260), "q_stride"), (dict(q_out_stride=252), "q_out_stride"), (dict(kv_stride=120), "kv_stride"),
    (dict(kv_stride=132), "kv_stride"), (dict(q=0), "null"), (dict(k=0), "null"), (dict(v=P + 8), "misaligned"), (dict(q_out=P + 4), "misaligned"),
    (dict(d_pos=P + 2), "misaligned"), (dict(q_out=P, q_out_stride=264), "same stride")])
def test_append_refuses_bad_arguments(kw, text):
    refused(lambda: append(**kw), INVAL, text)


@pytest.mark.parametrize("kw", [dict(section=(8, 12, 11)), dict(section=(-1, 21, 12)), dict(base=1.0), dict(base=float("nan")),
                                dict(base=float("inf")), dict(interleaved=2), dict(section=(2 ** 31 - 1, 2 ** 31 - 1, 34))])
def test_append_refuses_a_bad_rotation(kw):
    refused(lambda: append(o=rope(**kw)), INVAL, next(k for k in kw))


def test_append_takes_many_rows_only_where_no_tree_says_their_positions():
    refused(lambda: append(r=rows(rows=161), d_pos=0), INVAL, "rows")
    refused(lambda: append(r=rows(rows=2 ** 28 + 1, d_parent=0)), INVAL, "rows")


@pytest.mark.parametrize("kw,text", [
    (dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(q_heads=0), "q_heads"), (dict(q_heads=3), "q_heads"), (dict(q_stride=248), "q_stride"),
    (dict(q_stride=260), "q_stride"), (dict(out_stride=255), "q_stride"), (dict(q_heads=16386, q_stride=1 << 22, out_stride=1 << 22), "too large"),
    (dict(scale=float("nan")), "scale"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(q=0), "null"), (dict(out=P + 8), "misaligned"), (dict(d_lse=P + 2), "misaligned"), (dict(workspace=0), "workspace"),
    (dict(workspace=P + 16), "workspace")])
def test_attention_refuses_bad_arguments(kw, text):
    refused(lambda: attn(**kw), INVAL, text)


def test_attention_refuses_what_no_grid_holds():
    r = rows(batch=3, table_stride=(1 << 25) - 16)
    refused(lambda: attn(r=r), INVAL, "batch*kv_heads*table_stride")


def test_attention_refuses_a_small_workspace():
    n = B.spec_tree_attn_workspace_bytes(cache(), rows(), 4)
    refused(lambda: attn(workspace_bytes=n - 1), CAPACITY, "spec_tree_attn_workspace_bytes")


@pytest.mark.parametrize("kw,text", [
    (dict(d_tokens=0), "null"), (dict(d_greedy=P + 2), "misaligned"), (dict(d_budget=P + 1), "misaligned"), (dict(d_path=P + 2), "misaligned"),
    (dict(d_n=P + 1), "misaligned"), (dict(stop_token=-2), "stop_token"), (dict(d_new_len=2 * P), "overlaps an input"),
    (dict(d_new_len=2 * P + 4), "overlaps an input"), (dict(d_committed=7 * P), "overlaps an input"), (dict(d_path=4 * P + 32), "overlaps an input"),
    (dict(d_n=3 * P + 36), "overlaps an input"), (dict(d_n=11 * P), "outputs overlap"), (dict(d_path=9 * P - 32), "outputs overlap")])
def test_commit_refuses_bad_arguments(kw, text):
    refused(lambda: commit(**kw), INVAL, text)


def test_append_refuses_more_heads_than_a_grid_holds():
    refused(lambda: append(cache(kv_heads=32768, layers=1), kv_stride=1 << 24), INVAL, "too many heads")
