"""What the calls on a 4-bit cache, on attention weights and on eviction refuse, before anything is launched (addresses that are never
read); no device is needed."""
import ctypes

import pytest

NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 5, 6
G = dict(n_seq=1, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=64, max_blocks=64, n_draft=4)
APPEND = dict(pool=0x1000, n_pages=4, table=0x2000, lens=0x3000, q=0x4000, k=0x5000, v=0x6000, qs=1024, ks=256, vs=256, start=0x7000, n=8, rope=0x8000,
              rows=16, rot=128, pairs=0, q_out=0x9000, lens_out=0xa000, reps=0xb000, status=None)
COMMIT = dict(pool=0x1000, n_pages=4, table=0x2000, lens=0x3000, dk=0x4000, dv=0x5000, idx=0x6000, cnt=0x7000, most=4, lens_out=0x8000, reps=0x9000)
VERIFY = dict(q=0x1000, kv=(0x1000, 0x2000, 0x3000, 4), dk=0x4000, dv=0x5000, parent=None, idx=0x6000, cnt=0x7000, most=4, scale=0.0, out=0x8000, lse=None,
              ws=0x9000, bytes=1 << 30, status=None)
CHUNK = dict(q=0x1000, kv=(0x1000, 0x2000, 0x3000, 4), start=0x4000, n=8, scale=0.0, out=0x8000, lse=None, ws=0x9000, bytes=1 << 30, status=None)
READ = dict(kv=(0x1000, 0x2000, 0x3000, 4), first=0x4000, start=0x5000, n=8, k=0x6000, v=0x7000, status=None)
WEIGHTS = dict(q=0x1000, kv=(0x1000, 0x2000, 0x3000, 0x4000, 4), lse=0x5000, idx=0x6000, cnt=0x7000, most=4, path=0x8000, n_path=0x9000, scale=0.0, w=0xa000,
               w_out=0xb000, status=None)
EVICT = dict(k=0x1000, v=0x2000, n_pages=4, table=0x3000, lens=0x4000, w=0x5000, budget=0x6000, sink=4, recent=64, lens_out=0x7000, w_out=0x8000, reps=0x9000,
             status=None)


def _call(name, args, geom={}, **over):
    import paper_2512_21911_b200.binding as b
    g = b.make_geom(**{**G, **geom})
    a = []
    for k, v in {**args, **over}.items():
        if k == "kv" and v is not None:
            v = ctypes.byref((b.sv_kv if len(v) == 5 else b.sv_kv_q4)(*v))
        a.append(v)
    return getattr(b._lib, name)(ctypes.byref(g), *a, None)


@pytest.mark.parametrize("over,code", [
    (dict(pool=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(q=None), NULL),
    (dict(q_out=None), NULL), (dict(start=None), NULL), (dict(lens_out=None), NULL), (dict(n=-1), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 30), SHAPE),
    (dict(lens_out=0x3000), SHAPE), (dict(rot=0), SHAPE), (dict(rot=24), SHAPE), (dict(rot=144), SHAPE), (dict(rows=0), SHAPE), (dict(ks=128), SHAPE),
    (dict(vs=128), SHAPE), (dict(qs=512), SHAPE), (dict(q_out=0x4000, qs=2048), SHAPE), (dict(ks=260), ALIGN), (dict(pool=0x1040), ALIGN), (dict(k=0x5004), ALIGN),
    (dict(rope=0x8004), ALIGN), (dict(reps=0xb004), ALIGN)])
def test_append(over, code):
    assert _call("sv_rope_append_q4", APPEND, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(pool=None), NULL), (dict(dk=None), NULL), (dict(idx=None), NULL), (dict(cnt=None), NULL), (dict(lens_out=None), NULL), (dict(most=0), SHAPE),
    (dict(most=5), SHAPE), (dict(lens_out=0x3000), SHAPE), (dict(n_pages=0), SHAPE), (dict(pool=0x1010), ALIGN), (dict(dv=0x5008), ALIGN)])
def test_commit(over, code):
    assert _call("sv_kv_append_q4", COMMIT, **over) == code


@pytest.mark.parametrize("name,args,over,code", [
    ("sv_verify_attn_q4", VERIFY, dict(q=None), NULL), ("sv_verify_attn_q4", VERIFY, dict(kv=None), NULL), ("sv_verify_attn_q4", VERIFY, dict(dk=None), NULL),
    ("sv_verify_attn_q4", VERIFY, dict(out=None), NULL), ("sv_verify_attn_q4", VERIFY, dict(cnt=None), NULL), ("sv_verify_attn_q4", VERIFY, dict(ws=None), NULL),
    ("sv_verify_attn_q4", VERIFY, dict(most=0), SHAPE), ("sv_verify_attn_q4", VERIFY, dict(scale=-1.0), SHAPE),
    ("sv_verify_attn_q4", VERIFY, dict(scale=float("nan")), SHAPE), ("sv_verify_attn_q4", VERIFY, dict(kv=(0x1000, 0x2000, 0x3000, 0)), SHAPE),
    ("sv_verify_attn_q4", VERIFY, dict(kv=(0x1010, 0x2000, 0x3000, 4)), ALIGN), ("sv_verify_attn_q4", VERIFY, dict(dv=0x5008), ALIGN),
    ("sv_verify_attn_q4", VERIFY, dict(ws=0x9008), ALIGN), ("sv_verify_attn_q4", VERIFY, dict(bytes=64), WORKSPACE),
    ("sv_chunk_attn_q4", CHUNK, dict(q=None), NULL), ("sv_chunk_attn_q4", CHUNK, dict(start=None), NULL), ("sv_chunk_attn_q4", CHUNK, dict(n=-1), SHAPE),
    ("sv_chunk_attn_q4", CHUNK, dict(out=0x8008), ALIGN), ("sv_chunk_attn_q4", CHUNK, dict(bytes=64), WORKSPACE), ("sv_chunk_attn_q4", CHUNK, dict(scale=-0.5), SHAPE),
    ("sv_kv_read_q4", READ, dict(first=None), NULL), ("sv_kv_read_q4", READ, dict(v=None), NULL), ("sv_kv_read_q4", READ, dict(k=0x6008), ALIGN),
    ("sv_kv_read_q4", READ, dict(n=-2), SHAPE)])
def test_attention_and_reading(name, args, over, code):
    assert _call(name, args, **over) == code


@pytest.mark.parametrize("name,args", [("sv_rope_append_q4", APPEND), ("sv_kv_append_q4", COMMIT), ("sv_verify_attn_q4", VERIFY), ("sv_chunk_attn_q4", CHUNK),
                                       ("sv_kv_read_q4", READ), ("sv_attn_weights", WEIGHTS), ("sv_kv_evict", EVICT)])
def test_geometries(name, args):
    for geom, code in ((dict(n_q_heads=7), SHAPE), (dict(head_dim=64), UNSUPPORTED), (dict(block_size=32), UNSUPPORTED), (dict(n_seq=0), SHAPE),
                       (dict(max_blocks=0), SHAPE), (dict(n_q_heads=260, n_draft=1), UNSUPPORTED)):
        assert _call(name, args, geom) == code, geom


@pytest.mark.parametrize("over,code", [
    (dict(q=None), NULL), (dict(lse=None), NULL), (dict(w=None), NULL), (dict(w_out=None), NULL), (dict(cnt=None), NULL), (dict(path=None), NULL),
    (dict(n_path=None), NULL), (dict(most=0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(q=0x1008), ALIGN), (dict(w=0xa004), ALIGN)])
def test_weights(over, code):
    assert _call("sv_attn_weights", WEIGHTS, **over) == code


@pytest.mark.parametrize("over,geom,code", [
    (dict(k=None), {}, NULL), (dict(w=None), {}, NULL), (dict(budget=None), {}, NULL), (dict(w_out=None), {}, NULL), (dict(sink=-1), {}, SHAPE),
    (dict(recent=-1), {}, SHAPE), (dict(lens_out=0x4000), {}, SHAPE), (dict(n_pages=0), {}, SHAPE), (dict(k=0x1040), {}, ALIGN), (dict(reps=0x9004), {}, ALIGN),
    ({}, dict(max_blocks=6145), UNSUPPORTED)])
def test_evict(over, geom, code):
    assert _call("sv_kv_evict", EVICT, geom, **over) == code


def test_tensors_are_checked():
    torch = pytest.importorskip("torch")
    import paper_2512_21911_b200 as sv
    t = torch.zeros(16, dtype=torch.uint8)
    with pytest.raises(TypeError):
        sv.make_kv_q4(t, t, t)
    with pytest.raises(TypeError):
        sv.sv_kv_evict(sv.make_geom(**G), t, t, t, t, t, t, 0, 0, t, t)
