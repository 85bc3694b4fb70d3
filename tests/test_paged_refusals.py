"""What the calls on rotary positions and on the paged cache refuse, before anything is launched (no GPU work)."""
import ctypes

import pytest


def lib():
    from paper_2404_08856_amd import spd
    return spd, ctypes.CDLL(spd.LIB_PATH)


i32, u32, f32, sz = ctypes.c_int32, ctypes.c_uint32, ctypes.c_float, ctypes.c_size_t
null, some, odd = ctypes.c_void_p(None), ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 8)      # never read: the call ends before


def expect(code, name, *args):
    spd, l = lib()
    l.spd_last_error.restype = ctypes.c_char_p
    fn = getattr(l, name)
    fn.restype = i32
    assert fn(*args) == code and l.spd_last_error()


def config(**kw):
    spd, _ = lib()
    c = spd.spd_rope_config(64, 0, 10000.0, 1.0, 1.0, 2.0, 4096.0, 1.0, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def by(s):
    return ctypes.byref(s) if s is not None else null


@pytest.mark.parametrize("R", [0, -2, 3, 258, 1 << 30])
def test_rotary_dims(R):
    spd, _ = lib()
    n = sz()
    expect(spd.SPD_ERR_SHAPE, "spd_rope_table_bytes", i32(R), ctypes.byref(n))
    expect(spd.SPD_ERR_SHAPE, "spd_rope_table", by(config(rotary_dim=R)), some, sz(1 << 20), null)


@pytest.mark.parametrize("bad", [{"theta": 0.0}, {"theta": -1.0}, {"theta": float("inf")}, {"theta": float("nan")}, {"magnitude": float("nan")}, {"scaling": 4}, {"scaling": -1},
                                 {"scaling": 1, "factor": 0.0}, {"scaling": 2, "factor": float("nan")}, {"scaling": 2, "low": 2.0}, {"scaling": 3, "low": 0.0},
                                 {"scaling": 3, "original_positions": 0.0}, {"scaling": 2, "high": float("inf")}])
def test_rope_configs(bad):
    spd, _ = lib()
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table", by(config(**bad)), some, sz(1 << 20), null)


def test_rope_tables():
    spd, _ = lib()
    n = sz()
    assert spd._lib.spd_rope_table_bytes(64, ctypes.byref(n)) == 0 and n.value == 16 + 32 * 8
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table_bytes", i32(64), null)
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table", null, some, sz(1 << 20), null)
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table", by(config()), null, sz(1 << 20), null)
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table", by(config()), odd, sz(1 << 20), null)
    expect(spd.SPD_ERR_CAPACITY, "spd_rope_table", by(config()), some, sz(n.value - 1), null)
    factors = (ctypes.c_float * 32)(*([1.0] * 31 + [0.0]))
    expect(spd.SPD_ERR_INVALID_ARG, "spd_rope_table", by(config(h_factors=factors)), some, sz(1 << 20), null)


def apply(code, rope=(4096, 64, 0), x=(4096, 640, 64), out=(8192, 640, 64), positions=some, rows=3, heads=10, dim=64, flags=0):
    spd, _ = lib()
    r = None if rope is None else spd.spd_rope(*rope)
    a, b = (None if t is None else spd.spd_heads(*t) for t in (x, out))
    expect(code, "spd_rope_apply", by(r), by(a), by(b), positions, i32(rows), i32(heads), i32(dim), u32(flags), null)


def test_rope_apply():
    spd, _ = lib()
    bad, shape = spd.SPD_ERR_INVALID_ARG, spd.SPD_ERR_SHAPE
    apply(bad, rope=None); apply(bad, x=None); apply(bad, out=None); apply(bad, positions=null)
    apply(bad, rope=(None, 64, 0)); apply(bad, rope=(4104, 64, 0)); apply(bad, rope=(4096, 64, 2))
    apply(shape, rope=(4096, 66, 0)); apply(shape, rope=(4096, 7, 0)); apply(shape, rope=(4096, 0, 0))
    apply(bad, x=(None, 640, 64)); apply(bad, x=(4097, 640, 64)); apply(bad, out=(4098, 640, 64))
    apply(bad, x=(4096, 639, 64)); apply(bad, x=(4096, 640, 63)); apply(bad, out=(8192, 0, 64)); apply(bad, x=(4096, 1 << 41, 64))
    apply(bad, x=(4096, 64, 191)); apply(bad, out=(4096, 641, 64))
    apply(bad, flags=4); apply(bad, flags=8)
    for rows in (0, -1, (1 << 20) + 1):
        apply(shape, rows=rows)
    for heads in (0, 1025):
        apply(shape, heads=heads)
    for dim in (1, 0, 257):
        apply(shape, dim=dim)


CACHE = dict(k=4096, v=8192, k_scale=None, v_scale=None, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, e4m3=0)
BATCH = dict(n_seqs=2, n_rows=4, max_pages=5, table_stride=5, page_table=4096, lens=4096, row_start=None)


def structs(cache, batch):
    spd, _ = lib()
    c = None if cache is None else spd.spd_paged_cache(*{**CACHE, **cache}.values())
    b = None if batch is None else spd.spd_paged_batch(*{**BATCH, **batch}.values())
    return c, b


def both(code, cache={}, batch={}):
    """Refused alike by append, attention and its workspace's size."""
    spd, _ = lib()
    c, b = structs(cache, batch)
    dim = 64 if c is None else max(1, c.head_dim)
    h, n = spd.spd_heads(4096, 1 << 20, 256), sz()
    expect(code, "spd_paged_append", by(c), by(b), by(h), by(h), null, null, i32(0), null, null, u32(0), null)
    expect(code, "spd_paged_attention", by(c), by(b), by(h), by(h), i32(2), f32(1.0), i32(0), null, null, u32(0), some, sz(1 << 40), null)
    expect(code, "spd_paged_attention_workspace_bytes", by(c), by(b), i32(2), ctypes.byref(n))


def test_caches_and_batches():
    spd, _ = lib()
    bad, shape = spd.SPD_ERR_INVALID_ARG, spd.SPD_ERR_SHAPE
    both(bad, cache=None); both(bad, batch=None)
    for at in ("k", "v"):
        both(bad, cache={at: None}); both(bad, cache={at: 4104})
    for at in ("page_table", "lens"):
        both(bad, batch={at: None})
    for dim in (0, 32, 96, 256, -64):
        both(shape, cache={"head_dim": dim})
    for size in (0, 8, 24, 512, -16):
        both(shape, cache={"page_size": size})
    for n in (0, -1):
        both(shape, cache={"n_pages": n}); both(shape, cache={"n_kv_heads": n}); both(shape, batch={"n_seqs": n}); both(shape, batch={"n_rows": n}); both(shape, batch={"max_pages": n})
    both(shape, cache={"n_kv_heads": 1025}); both(shape, batch={"n_seqs": 4097}); both(shape, batch={"n_rows": (1 << 20) + 1}); both(shape, batch={"max_pages": (1 << 26) + 1, "table_stride": 1 << 27})
    both(bad, cache={"e4m3": 2}); both(bad, cache={"e4m3": 1}); both(bad, cache={"e4m3": 1, "k_scale": 4096}); both(bad, cache={"k_scale": 4096, "v_scale": 4096})
    both(bad, batch={"table_stride": 4}); both(bad, batch={"table_stride": 1 << 41}); both(shape, batch={"n_rows": 5})


def append(code, k=(4096, 128, 64), v=(4096, 128, 64), q=None, q_out=None, heads=0, rope=None, positions=null, flags=0):
    spd, _ = lib()
    c, b = structs({}, {})
    ks, vs, qs, qo = (None if t is None else spd.spd_heads(*t) for t in (k, v, q, q_out))
    r = None if rope is None else spd.spd_rope(*rope)
    expect(code, "spd_paged_append", by(c), by(b), by(ks), by(vs), by(qs), by(qo), i32(heads), by(r), positions, u32(flags), null)


def test_appends():
    spd, _ = lib()
    bad, shape = spd.SPD_ERR_INVALID_ARG, spd.SPD_ERR_SHAPE
    rope, q = (4096, 64, 0), (4096, 128, 64)
    append(bad, k=None); append(bad, v=None); append(bad, q=q, heads=2, rope=rope); append(bad, q_out=q, heads=2, rope=rope)
    append(bad, k=(None, 128, 64)); append(bad, v=(4096, 127, 64)); append(bad, k=(4096, 128, 0)); append(bad, v=(4097, 128, 64))
    append(bad, q=q, q_out=q, heads=2); append(bad, positions=some)
    append(shape, q=q, q_out=q, heads=0, rope=rope); append(shape, q=q, q_out=q, heads=1025, rope=rope)
    append(bad, q=q, q_out=(4096, 256, 64), heads=2, rope=rope); append(bad, q=q, q_out=(4096, 64, 64), heads=2, rope=rope)
    append(shape, rope=(4096, 66, 0)); append(bad, rope=(4098, 64, 0)); append(bad, flags=2)


def test_appends_of_too_many_rows_and_heads():
    spd, _ = lib()
    c, b = structs({"n_kv_heads": 1024}, {"n_seqs": 1, "n_rows": 1 << 20})
    h = spd.spd_heads(4096, 1 << 20, 64)
    expect(spd.SPD_ERR_SHAPE, "spd_paged_append", by(c), by(b), by(h), by(h), null, null, i32(0), null, null, u32(0), null)


def attention(code, q=(4096, 128, 64), out=(8192, 128, 64), heads=2, scale=1.0, window=0, seen=null, flags=0, ws=some, size=1 << 40):
    spd, _ = lib()
    c, b = structs({}, {})
    a, o = (None if t is None else spd.spd_heads(*t) for t in (q, out))
    expect(code, "spd_paged_attention", by(c), by(b), by(a), by(o), i32(heads), f32(scale), i32(window), seen, null, u32(flags), ws, sz(size), null)


def test_attention_in_the_place_of_its_queries():
    attention(lib()[0].SPD_ERR_INVALID_ARG, out=(4096, 128, 64))


def test_attentions():
    spd, _ = lib()
    bad, shape = spd.SPD_ERR_INVALID_ARG, spd.SPD_ERR_SHAPE
    attention(bad, q=None); attention(bad, out=None); attention(bad, q=(None, 128, 64)); attention(bad, out=(8192, 100, 64)); attention(bad, q=(4098, 128, 64))
    for heads in (0, 1, 3, 1026, -2):
        attention(shape, heads=heads)
    for scale in (float("nan"), float("inf"), -float("inf")):
        attention(bad, scale=scale)
    attention(bad, window=-1); attention(bad, window=4, seen=some); attention(bad, flags=2); attention(bad, ws=odd)
    attention(spd.SPD_ERR_CAPACITY, ws=null); attention(spd.SPD_ERR_CAPACITY, size=0)
    n = sz()
    c, b = structs({}, {})
    expect(bad, "spd_paged_attention_workspace_bytes", by(c), by(b), i32(2), null)
    expect(shape, "spd_paged_attention_workspace_bytes", by(c), by(b), i32(3), ctypes.byref(n))


def test_forwards_without_a_model():
    spd, _ = lib()
    c, b = structs({}, {})
    r, n = spd.spd_rope(4096, 64, 0), sz()
    expect(spd.SPD_ERR_INVALID_ARG, "spd_verify_forward_paged", null, some, by(c), by(b), by(r), null, null, some, some, sz(1 << 40), null)
    expect(spd.SPD_ERR_INVALID_ARG, "spd_verify_paged_workspace_bytes", null, by(c), by(b), ctypes.byref(n))
    expect(spd.SPD_ERR_INVALID_ARG, "spd_verify_paged_workspace_bytes", some, by(c), by(b), null)
