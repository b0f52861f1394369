"""What the calls around a paged cache refuse, through the C ABI with addresses that are never dereferenced, and through the binding with tensors
that are on no GPU: nothing is enqueued (there is no GPU here)."""
import ctypes as C
import os

import pytest
import torch

import paper_2503_01840_amd as E
from paper_2503_01840_amd import binding as Bd

AT = 1 << 20                                                 # an address


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(E.LIB_PATH):
        from paper_2503_01840_amd.build import build_library
        build_library()
    return E.lib()


def _kv(**over):
    v = dict(k=AT, v=AT, k_exp=None, v_exp=None, page_table=AT, dtype=1, n_pages=10, page_size=16, max_pages=4, n_kv_heads=2, head_dim=128)
    v.update(over)
    return Bd.PagedKV(*[v[n] for n, _ in Bd.PagedKV._fields_])


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(page_table=None), -1), (dict(dtype=2), -1), (dict(dtype=2, k_exp=AT), -1), (dict(dtype=3), -2),
              (dict(dtype=-1), -2), (dict(n_pages=0), -2), (dict(page_size=0), -2), (dict(max_pages=0), -2), (dict(n_kv_heads=0), -2), (dict(head_dim=96), -2),
              (dict(head_dim=0), -2), (dict(n_pages=1 << 20, page_size=1 << 11), -2), (dict(max_pages=1 << 20, page_size=1 << 11), -2), (dict(k=AT + 8), -2),
              (dict(v=AT + 2), -2)]


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_caches_that_cannot_be(L, over, code):
    kv = _kv(**over)
    assert L.eagle3_paged_append(kv, 1, 1, AT, None, None, AT, AT, 1, 256, None) == code
    assert L.eagle3_paged_read(kv, 1, 1, AT, None, None, AT, AT, 1, 256, None) == code
    assert L.eagle3_paged_attention(kv, 1, 2, AT, 256, AT, 10, 1.0, AT, None, AT, 1 << 40, None) == code
    n = C.c_size_t(5)
    assert L.eagle3_paged_attention_workspace(kv, 1, 2, 10, n) == code and n.value == 5


def _rows(**over):
    v = dict(kv=_kv(), B=2, rows=3, start=AT, n=None, row_start=None, k=AT, v=AT, n_rows=6, stride=256)
    v.update(over)
    return list(v.values()) + [None]


@pytest.mark.parametrize("over,code", [(dict(kv=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(B=0), -2), (dict(B=-1), -2), (dict(rows=0), -2),
                                       (dict(n_rows=0), -2), (dict(n_rows=1 << 31), -2), (dict(stride=255), -2), (dict(stride=260), -2), (dict(stride=1 << 62), -2),
                                       (dict(k=AT + 8), -2), (dict(v=AT + 4), -2), (dict(B=1 << 20, rows=1 << 10), -2)])
def test_rows_that_cannot_be(L, over, code):
    assert L.eagle3_paged_append(*_rows(**over)) == code
    assert L.eagle3_paged_read(*_rows(**over)) == code


def test_append_needs_a_start(L):
    assert L.eagle3_paged_append(*_rows(start=None)) == -1


def _attention(**over):
    v = dict(kv=_kv(), B=2, H=8, q=AT, stride=1024, kv_len=AT, max_len=64, scale=1.0, out=AT, lse=None, ws=AT, ws_bytes=1 << 40)
    v.update(over)
    return list(v.values()) + [None]


@pytest.mark.parametrize("over,code", [(dict(kv=None), -1), (dict(q=None), -1), (dict(kv_len=None), -1), (dict(out=None), -1), (dict(B=0), -2), (dict(B=65536), -2),
                                       (dict(H=0), -2), (dict(H=7), -2), (dict(H=65536), -2), (dict(max_len=0), -2), (dict(max_len=65), -2), (dict(stride=1023), -2),
                                       (dict(stride=1026), -2), (dict(stride=1 << 62), -2), (dict(q=AT + 8), -2), (dict(out=AT + 2), -2)])
def test_attention_that_cannot_be(L, over, code):
    assert L.eagle3_paged_attention(*_attention(**over)) == code


def test_attention_wants_the_workspace_that_it_tells(L):
    kv = _kv(n_pages=100000, max_pages=8192)
    n = C.c_size_t()
    assert L.eagle3_paged_attention_workspace(kv, 1, 8, 131072, None) == -1
    assert L.eagle3_paged_attention_workspace(kv, 1, 8, 131072, n) == 0
    if n.value:                                              # a long context is worked on in parts
        for ws, size in ((None, n.value), (AT, n.value - 1), (AT + 128, n.value)):
            assert L.eagle3_paged_attention(*_attention(kv=kv, B=1, max_len=131072, ws=ws, ws_bytes=size)) == -3


def _rope(**over):
    spec = dict(turns=AT, rot_dim=64, interleaved=0, amplitude=1.0)
    v = dict(dtype=1, rows=2, d=64, spec=None, positions=AT, H=4, q=AT, qs=256, qo=AT, qos=256, Hkv=2, k=AT, ks=128, ko=AT, kos=128)
    for n in list(over):
        if n in spec:
            spec[n] = over.pop(n)
    v["spec"] = Bd.RopeSpec(*spec.values())
    v.update(over)
    return list(v.values()) + [None]


@pytest.mark.parametrize("over,code", [(dict(spec=None), -1), (dict(turns=None), -1), (dict(positions=None), -1), (dict(q=None), -1), (dict(qo=None), -1),
                                       (dict(ko=None), -1), (dict(dtype=2), -2), (dict(dtype=-1), -2), (dict(rows=0), -2), (dict(d=63), -2), (dict(d=0), -2),
                                       (dict(d=1026), -2), (dict(rot_dim=0), -2), (dict(rot_dim=66), -2), (dict(rot_dim=31), -2), (dict(H=0), -2), (dict(Hkv=0), -2),
                                       (dict(qs=255), -2), (dict(qos=255), -2), (dict(ks=127), -2), (dict(kos=0), -2), (dict(qs=512, qos=256), -2),
                                       (dict(rows=1 << 24, d=2, rot_dim=2, H=1, Hkv=1), -2),
                                       (dict(H=1 << 24, qs=1 << 30, qos=1 << 30), -2), (dict(rows=(1 << 24) - 1, d=1024, H=64, Hkv=8, qs=1 << 16, qos=1 << 16, ks=1 << 13, kos=1 << 13), -2)])
def test_rotations_that_cannot_be(L, over, code):
    assert L.eagle3_rope(*_rope(**over)) == code
    assert L.eagle3_rope_grad(*_rope(**over)) == code


def test_the_binding_wants_tensors_on_a_gpu(L):
    pool, table = torch.zeros(4, 16, 2, 64), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        E.PagedKVCache(pool, pool, table)
    with pytest.raises(ValueError):
        E.eagle3_rope(None, table, pool[0])


@pytest.mark.parametrize("call", ["append", "read"])
@pytest.mark.parametrize("rows", [1, 2])
def test_values_lie_as_the_keys_do(L, monkeypatch, call, rows):
    """The heads of a value row one behind the other, as those of a key row: of one row too.  (Tensors on the CPU, the launch replaced by a list.)"""
    from types import SimpleNamespace
    sent = []
    monkeypatch.setattr(Bd, "_on", lambda gpu, call, *args: sent.append(args))
    cache = SimpleNamespace(gpu=-1, B=1, row_dtype=torch.bfloat16, heads=8, d=128, c=None)
    z = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)
    start = torch.zeros(1, dtype=torch.int32)
    go = (lambda k, v: E.eagle3_paged_append(cache, k, v, start)) if call == "append" else (lambda k, v: E.eagle3_paged_read(cache, start, out=(k, v)))
    k = z(rows, 8, 128)
    bad = [z(rows, 24, 128)[:, ::3], z(rows, 128, 8).transpose(1, 2), z(1, 1, 128).expand(rows, 8, 128), z(1, 1, 1).expand(rows, 8, 128), z(rows, 8, 256)[..., ::2],
           z(rows, 4, 128), z(rows + 1, 8, 128), z(rows, 8, 64), z(rows, 8, 128).float(), z(rows * 8, 128)]
    for v in bad:
        for pair in ((k, v), (v, k)):
            with pytest.raises(ValueError):
                go(*pair)
    if rows > 1:                                              # one distance from row to row for both
        with pytest.raises(ValueError):
            go(k, z(rows, 16, 128)[:, :8])
    assert not sent
    # any distance for a single row, and for a single head's strides
    packed = z(rows, 24, 128)
    good = [(k, z(rows, 8, 128)), (packed[:, :8], packed[:, 16:])] + ([(k, packed[:, 8:16])] if rows == 1 else [])
    for i, (k, v) in enumerate(good):
        go(k, v)
        assert sent[-1][6:8] == (k.data_ptr(), v.data_ptr()) and sent[-1][8:] == (rows, k.stride(0) if rows > 1 else 8 * 128)
    cache.heads = 1
    go(z(rows, 1, 128), z(rows, 128, 1).transpose(1, 2))
