"""What the entry points of attention and of caches held in 4 bits refuse, and what their workspaces are (no GPU is touched: every call ends before a launch)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from paper_2504_08009_amd import binding
from paper_2504_08009_amd.binding import _Kv4

P = 1 << 20  # an address that nobody reads
F32, BF16, F16 = oz.OZ2_F32, oz.OZ2_BF16, oz.OZ2_F16
INT64 = 2 ** 63 - 1



class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld_token", ctypes.c_int64), ("ld_head", ctypes.c_int64), ("type", ctypes.c_int)]


class _Sequences(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("table", ctypes.c_void_p), ("ld_table", ctypes.c_int64), ("lengths", ctypes.c_void_p),
                ("tokens", ctypes.c_int64), ("cu", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_sequence", ctypes.c_int64),
                ("positions_head", ctypes.c_int64), ("weights", ctypes.c_void_p), ("weights_sequence", ctypes.c_int64), ("weights_head", ctypes.c_int64)]


class _Kept(ctypes.Structure):
    _fields_ = [("lengths", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_sequence", ctypes.c_int64), ("positions_head", ctypes.c_int64),
                ("weights", ctypes.c_void_p), ("weights_sequence", ctypes.c_int64), ("weights_head", ctypes.c_int64)]


def ref(s):
    return None if s is None else ctypes.byref(s)


def rows(at=P, token=1024, head=128, kind=BF16):
    return _Rows(at, token, head, kind)


def attention(tokens=0, sequences=1, cu=P, heads=8, kv_heads=2, dim=128, scale=0.1, q=None, k=None, v=None, out=None):
    q, k, v, out = q or rows(), k or rows(P << 1, 256), v or rows(P << 2, 256), out or rows(P << 3)
    return oz.lib().oz2_attention(tokens, sequences, cu, heads, kv_heads, dim, scale, 1, ref(q), ref(k), ref(v), ref(out), None)


def test_attention_refuses():
    assert attention() == 0  # no tokens: nothing to do
    assert attention(tokens=5, sequences=0) == 0
    assert attention(tokens=-1) == -1 and attention(tokens=INT64) == -1
    assert attention(sequences=-1) == -2 and attention(sequences=INT64) == -2
    assert attention(tokens=5, cu=None) == -3
    assert attention(heads=0) == -4 and attention(heads=1 << 20, kv_heads=1) == -4
    assert attention(kv_heads=0) == -5 and attention(kv_heads=3) == -5 and attention(kv_heads=16) == -5
    assert attention(dim=0) == -6 and attention(dim=257) == -6
    for scale in (0.0, -0.1, float("nan"), float("inf")):
        assert attention(scale=scale) == -7
    for bad in (rows(kind=3), rows(kind=-1), rows(None), rows(token=1023), rows(head=127), rows(token=0), rows(token=-1024), rows(token=INT64), rows(head=INT64)):
        assert attention(tokens=5, q=bad) == -9
        assert attention(tokens=5, out=bad) == -12
    assert attention(tokens=5, k=rows(kind=F16)) == -10 and attention(tokens=5, v=rows(kind=F32)) == -11
    assert attention(tokens=5, k=rows(token=255)) == -10 and attention(tokens=5, v=rows(None)) == -11


def test_results_over_inputs_are_refused():
    # 5 tokens of 8 heads of 128 bf16: 2048 bytes a token, 10240 in all
    for at in (P, P + 16, P + 10238, P - 10238):
        assert attention(tokens=5, out=rows(at)) == -12
    for at in ((P << 1), (P << 1) + 5 * 512 - 2, (P << 2) - 10238):
        assert attention(tokens=5, out=rows(at)) == -12
    # heads of one packed tensor q, k, v, out: no byte in common, yet one after the other
    packed = dict(q=rows(P, 2560), k=rows(P + 2048, 2560), v=rows(P + 2560, 2560))
    assert attention(tokens=0, out=rows(P + 2560 + 512, 2560), **packed) == 0
    assert attention(tokens=5, out=rows(P + 2560 + 510, 2560), **packed) == -12  # (the last of a token's values is the next one's first)


def cache(**more):
    f = dict(pages=4, page_size=32, heads=2, dim=64, k_codes=P, v_codes=P << 1, codes_page=2048, codes_head=1024, k_scales=P << 2, v_scales=P << 3, scales_page=64, scales_head=32)
    f.update(more)
    return _Kv4(*(f[name] for name, _ in _Kv4._fields_))


def sequences(**more):
    f = dict(sequences=3, max_pages=4, table=P, ld_table=4, lengths=P, tokens=3, cu=P, positions=P << 4, positions_sequence=256, positions_head=128, weights=P << 5,
             weights_sequence=256, weights_head=128)
    f.update(more)
    return _Sequences(*(f[name] for name, _ in _Sequences._fields_))


BAD_CACHES = [dict(pages=0), dict(pages=1 << 31), dict(page_size=0), dict(page_size=8), dict(page_size=24), dict(heads=0), dict(heads=1 << 16), dict(dim=0), dict(dim=12),
              dict(dim=264), dict(k_codes=None), dict(v_codes=P + 2), dict(k_scales=P + 8), dict(v_scales=None), dict(codes_head=1023), dict(codes_head=1026),
              dict(codes_page=1024), dict(codes_page=INT64), dict(scales_head=31), dict(scales_page=66), dict(scales_page=32), dict(codes_page=0)]
BAD_SEQUENCES = [dict(sequences=-1), dict(sequences=1 << 16), dict(max_pages=-1), dict(max_pages=1 << 26), dict(table=None), dict(ld_table=3), dict(lengths=None),
                 dict(positions_head=127), dict(weights_sequence=255), dict(weights_head=INT64), dict(positions_sequence=-256)]


def calls(c, on, **more):
    kept = more.get("to")
    L, ctx = oz.lib(), oz.Context()
    yield L.oz2_kv4_append(ref(c), ref(on), more.get("at"), ref(rows(P, 128, 64)), ref(rows(P << 1, 128, 64)), None, None, None), 0
    yield L.oz2_kv4_attention(ref(c), ref(on), 8, 0.1, ref(rows(P, 512, 64)), ref(rows(P << 1, 512, 64)), None), 0
    yield L.oz2_context_kv4_attention(ctx.handle, ref(c), ref(on), 8, 0.1, ref(rows(P, 512, 64)), ref(rows(P << 1, 512, 64)), None), 1
    yield L.oz2_kv4_evict(ref(c), ref(on), 4, 0, ref(kept), None), 0
    yield L.oz2_context_kv4_evict(ctx.handle, ref(c), ref(on), 4, 0, ref(kept), None), 1


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(bad):
    for rc, shift in calls(cache(**bad), sequences()):
        assert rc == -1 - shift
    assert oz.lib().oz2_kv4_attention_workspace_bytes(ref(cache(**bad)), 3, 4, 3, 8, 0) == 0
    assert oz.lib().oz2_kv4_evict_workspace_bytes(ref(cache(**bad)), 3, 4, 4) == 0


@pytest.mark.parametrize("bad", BAD_SEQUENCES, ids=str)
def test_bad_sequences_are_refused(bad):
    for rc, shift in calls(cache(), sequences(**bad)):
        assert rc == -2 - shift


def test_strides_of_single_pages_heads_and_sequences_say_nothing():
    one = cache(pages=1, heads=1, codes_page=0, codes_head=0, scales_page=1, scales_head=3)
    on = sequences(sequences=1, ld_table=0, tokens=0, positions_sequence=0, positions_head=0, weights_sequence=0, weights_head=0)
    q, out = rows(P, 512, 64), rows(P << 1, 512, 64)
    assert oz.lib().oz2_kv4_attention(ref(one), ref(on), 8, 0.1, ref(q), ref(out), None) == 0


def test_appends_are_refused():
    L, c = oz.lib(), cache()
    k, v, held = rows(P, 128, 64), rows(P << 1, 128, 64), rows(P << 2, 128, 64)

    def append(on=None, at=None, k=k, v=v, held_k=None, held_v=None):
        return L.oz2_kv4_append(ref(c), ref(on or sequences()), at, ref(k), ref(v), ref(held_k), ref(held_v), None)

    assert append(sequences(tokens=0)) == 0 and append(sequences(sequences=0, tokens=0, table=None, lengths=None)) == 0
    assert append(sequences(tokens=-1)) == -2 and append(sequences(tokens=1 << 26)) == -2 and append(sequences(cu=None)) == -2
    assert append(sequences(positions=None), at=P) == -3
    assert append(k=rows(None, 128, 64)) == -4 and append(k=rows(P, 127, 64)) == -4 and append(v=rows(P, 128, 64, F16)) == -5
    assert append(held_k=rows(P << 2, 128, 64, F32)) == -6 and append(held_v=rows(P << 2, 128, 60)) == -7
    assert append(held_k=rows(P + 2, 128, 64)) == -6 and append(held_k=v) == -6 and append(held_v=k) == -7
    assert append(held_k=held, held_v=held) == -7


def test_attention_over_a_cache_is_refused():
    L, c = oz.lib(), cache()

    def step(on=None, heads=8, scale=0.1, q=rows(P, 512, 64), out=rows(P << 1, 512, 64)):
        return L.oz2_kv4_attention(ref(c), ref(on or sequences()), heads, scale, ref(q), ref(out), None)

    assert step(sequences(tokens=0)) == 0
    assert step(heads=7) == -3 and step(heads=0) == -3 and step(sequences(tokens=1 << 22)) == -3
    assert step(scale=-1.0) == -4
    assert step(q=rows(None, 512, 64)) == -5 and step(out=rows(P << 1, 511, 64)) == -6 and step(out=rows(P + 1024, 512, 64)) == -6
    oz.set_workspace(None, 0)
    assert step() == 1  # no workspace


def test_evictions_are_refused():
    L, c, ctx = oz.lib(), cache(), oz.Context()
    to = lambda **more: _Kept(*(dict(dict(lengths=P << 6, positions=P << 7, positions_sequence=256, positions_head=128, weights=P << 8, weights_sequence=256,
                                          weights_head=128), **more)[name] for name, _ in _Kept._fields_))

    def evict(on=None, keep=4, recent=0, to=None):
        return L.oz2_context_kv4_evict(ctx.handle, ref(c), ref(on or sequences()), keep, recent, ref(to), None)

    assert evict(sequences(sequences=0, table=None, lengths=None, positions=None, weights=None)) == 0
    assert evict(sequences(positions=None)) == -3 and evict(sequences(weights=None)) == -3
    assert evict(keep=-1) == -4 and evict(recent=-1) == -5 and evict(recent=5) == -5
    assert evict(to=to(lengths=None)) == -6 and evict(to=to(positions_head=100)) == -6
    assert evict(to=to(weights=P << 5, weights_sequence=512)) == -6
    assert evict() == 1 and evict(to=to()) == 1  # no workspace


def test_workspaces_grow_with_what_is_asked():
    L, c = oz.lib(), cache(pages=1000, page_size=64)
    c = cache(pages=1000, page_size=64, codes_head=2048, codes_page=4096, scales_head=64, scales_page=128)
    size = lambda s, p, t, h, w: L.oz2_kv4_attention_workspace_bytes(ref(c), s, p, t, h, w)
    assert 0 < size(1, 1, 1, 8, 0) < size(1, 500, 1, 8, 0) < size(1, 500, 4, 8, 0) < size(1, 500, 4, 8, 1)
    assert size(1, 0, 0, 8, 0) > 0
    assert size(1, 1, 1, 7, 0) == 0 and size(1, 1, 1, 0, 0) == 0 and size(-1, 1, 1, 8, 0) == 0 and size(1, 1, 1 << 24, 8, 0) == 0 and size(1, 1 << 40, 1, 8, 0) == 0
    evict = lambda s, p, keep: L.oz2_kv4_evict_workspace_bytes(ref(c), s, p, keep)
    assert 0 < evict(1, 10, 0) <= evict(1, 10, 640) < evict(1, 10, 320) and evict(1, 10, 10 ** 12) > 0
    assert evict(1, 1, -1) == 0


def test_bytes_are_laid_out_like_the_structures():
    kinds = ((_Rows, binding._pack_rows, (P, 5, 6, 2)), (_Sequences, binding._pack_sequences, tuple(range(1, 14))), (_Kept, binding._pack_kept, tuple(range(1, 8))))
    for kind, pack, values in kinds:
        assert bytes(kind(*values)) == pack(*values) and len(pack(*values)) == ctypes.sizeof(kind)
