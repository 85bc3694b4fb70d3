"""What the calls on 4-bit weights and on log probabilities refuse, before anything is launched (no GPU work)."""
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


@pytest.mark.parametrize("at", range(3))
def test_null_pointers(at):
    spd, _ = lib()
    three = [null if i == at else some for i in range(3)]
    bad = spd.SPD_ERR_INVALID_ARG
    expect(bad, "spd_q4_quantize", three[0], sz(64), u32(0), i32(16), i32(64), i32(32), three[1], three[2], null)
    expect(bad, "spd_q4_dequantize", three[0], three[1], i32(16), i32(64), i32(32), three[2], sz(64), u32(0), null)
    expect(bad, "spd_q4_pack", three[0], three[1], i32(16), i32(64), i32(32), three[2], sz(1 << 30), null)
    expect(bad, "spd_q4_matmul", three[0], i32(16), i32(64), i32(32), three[1], sz(64), u32(0), i32(1), three[2], sz(16), some, sz(1 << 30), null)
    expect(bad, "spd_model_create_q4", three[0], three[1], three[2], sz(0), some, sz(0), null, sz(0), null, null)
    expect(bad, "spd_model_bytes_q4", null, i32(32), null, null, null)
    expect(bad, "spd_q4_bytes", i32(16), i32(16), i32(32), null)
    expect(bad, "spd_q4_matmul_workspace_bytes", i32(1), i32(16), i32(16), null)
    expect(bad, "spd_logprobs_workspace_bytes", i32(1), i32(16), i32(0), null)


@pytest.mark.parametrize("N,K,group", [(0, 64, 32), (16, 0, 32), (-1, 64, 32), (16, 64, 16), (16, 64, 0), (16, 64, 256), (16, 64, -32),
                                       (1, 2**24 + 1, 32), (2**26 + 1, 64, 128), (2**25 + 1, 1024, 64), (2**31 - 1, 2**31 - 1, 32)])
def test_shapes(N, K, group):
    spd, _ = lib()
    n = ctypes.c_size_t()
    bad = spd.SPD_ERR_SHAPE
    expect(bad, "spd_q4_bytes", i32(N), i32(K), i32(group), ctypes.byref(n))
    expect(bad, "spd_q4_quantize", some, sz(max(K, 64)), u32(0), i32(N), i32(K), i32(group), some, some, null)
    expect(bad, "spd_q4_dequantize", some, some, i32(N), i32(K), i32(group), some, sz(64), u32(0), null)
    expect(bad, "spd_q4_pack", some, some, i32(N), i32(K), i32(group), some, sz(1 << 30), null)
    expect(bad, "spd_q4_matmul", some, i32(N), i32(K), i32(group), some, sz(64), u32(0), i32(1), some, sz(16), some, sz(1 << 30), null)


@pytest.mark.parametrize("rows", [0, -1, 65])
def test_rows_of_a_product(rows):
    spd, _ = lib()
    n = ctypes.c_size_t()
    expect(spd.SPD_ERR_SHAPE, "spd_q4_matmul", some, i32(16), i32(64), i32(32), some, sz(64), u32(0), i32(rows), some, sz(16), some, sz(1 << 30), null)
    expect(spd.SPD_ERR_SHAPE, "spd_q4_matmul_workspace_bytes", i32(rows), i32(16), i32(64), ctypes.byref(n))


def test_strides_flags_alignment_and_capacity():
    spd, _ = lib()
    bad, full = spd.SPD_ERR_INVALID_ARG, spd.SPD_ERR_CAPACITY
    mm = lambda code, packed=some, xs=64, flags=0, ys=16, ws=some, rows=1: expect(code, "spd_q4_matmul", packed, i32(16), i32(64), i32(32), some, sz(xs), u32(flags), i32(rows), some, sz(ys), ws, sz(0), null)
    mm(bad, xs=63)
    mm(bad, ys=15)
    mm(bad, flags=2)
    mm(bad, packed=odd)
    mm(bad, ws=odd)
    n = ctypes.c_size_t()
    for rows in (1, 64):
        l = lib()[1]
        assert l.spd_q4_matmul_workspace_bytes(i32(rows), i32(16), i32(64), ctypes.byref(n)) == 0
        if n.value:
            mm(full, rows=rows)
            mm(full, ws=null, rows=rows)
    expect(bad, "spd_q4_quantize", some, sz(63), u32(0), i32(16), i32(64), i32(32), some, some, null)
    expect(bad, "spd_q4_quantize", some, sz(64), u32(2), i32(16), i32(64), i32(32), some, some, null)
    expect(bad, "spd_q4_dequantize", some, some, i32(16), i32(64), i32(32), some, sz(63), u32(0), null)
    expect(bad, "spd_q4_dequantize", some, some, i32(16), i32(64), i32(32), some, sz(64), u32(4), null)
    expect(bad, "spd_q4_pack", some, some, i32(16), i32(64), i32(32), odd, sz(1 << 30), null)
    expect(full, "spd_q4_pack", some, some, i32(16), i32(64), i32(32), some, sz(1023), null)
    expect(spd.SPD_ERR_SHAPE, "spd_q4_bytes", i32(2**31 - 1), i32(2**31 - 1), i32(32), ctypes.byref(n))


def test_log_probability_arguments():
    spd, l = lib()
    bad = spd.SPD_ERR_INVALID_ARG

    def lp(code, rows=some, stride=100, tokens=some, n=2, vocab=100, temperature=1.0, flags=0, out=some, rank=some, top=2, ids=some, ilp=some, ws=some):
        expect(code, "spd_token_logprobs", rows, sz(stride), tokens, i32(n), i32(vocab), f32(temperature), u32(flags), out, null, rank, i32(top), ids, ilp, ws, sz(0), null)
    lp(bad, rows=null)
    lp(bad, tokens=null)
    lp(bad, tokens=null, out=null)
    lp(bad, ids=null)
    lp(bad, ilp=null)
    lp(bad, n=0)
    lp(bad, vocab=0)
    lp(bad, top=-1)
    lp(bad, top=33)
    lp(bad, stride=99)
    lp(bad, flags=2)
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        lp(bad, temperature=t)
    lp(bad, ws=odd)
    lp(spd.SPD_ERR_SHAPE, vocab=2**24 + 1, stride=2**25)
    lp(spd.SPD_ERR_SHAPE, n=2**22 + 1)
    lp(spd.SPD_ERR_SHAPE, n=2**21 + 1, vocab=32769, stride=32769)
    n = ctypes.c_size_t()
    for rows, vocab, top in ((0, 10, 1), (1, 0, 1), (1, 10, -1), (1, 10, 33)):
        expect(bad, "spd_logprobs_workspace_bytes", i32(rows), i32(vocab), i32(top), ctypes.byref(n))
    assert l.spd_logprobs_workspace_bytes(i32(1), i32(1 << 20), i32(5), ctypes.byref(n)) == 0
    if n.value:
        lp(spd.SPD_ERR_CAPACITY, n=1, vocab=1 << 20, stride=1 << 20, ws=null)


@pytest.mark.parametrize("n,vocab", [(2**22, 5000), (2**22, 32768), (2**21, 32769)])
def test_log_probabilities_of_as_many_rows_as_a_launch_has_no_threads_for(n, vocab):
    spd, _ = lib()                                         # 2^22 workgroups of 1024: 2^32 threads
    expect(spd.SPD_ERR_SHAPE, "spd_token_logprobs", some, sz(vocab), some, i32(n), i32(vocab), f32(1.0), u32(0), some, null, null, i32(0), null, null, some, sz(1 << 40), null)


@pytest.mark.parametrize("N,K", [(2**26, 64), (2**26 - 3, 512), (2**11, 2**24)])
def test_matrices_that_a_launch_has_no_threads_for(N, K):
    spd, _ = lib()                                         # 2^24 workgroups of 256: 2^32 threads
    n = ctypes.c_size_t()
    expect(spd.SPD_ERR_SHAPE, "spd_q4_bytes", i32(N), i32(K), i32(128), ctypes.byref(n))
    expect(spd.SPD_ERR_SHAPE, "spd_q4_quantize", some, sz(K), u32(0), i32(N), i32(K), i32(128), some, some, null)


def test_what_the_binding_refuses():
    torch = pytest.importorskip("torch")
    spd, _ = lib()
    host = -1                                              # the device number of a tensor in host memory
    good = torch.zeros((4, 8))
    assert spd._matrix(good, host) == (good.data_ptr(), 8, 0)
    assert spd._matrix(good[:, 2:7].to(torch.bfloat16), host)[1:] == (5, 1)
    assert spd._matrix(good[:, 2:7], host)[1] == 8 and spd._matrix(good[2:3, ::8], host)[1] == 1
    for bad in (good.double(), good.t(), good[:, ::2], good[0:1].expand(4, 8)):
        with pytest.raises(AssertionError):
            spd._matrix(bad, host)
    with pytest.raises(AssertionError):
        spd._matrix(good, 0)
    assert spd._own(None, host, torch.float32, (4, 8)) is None and spd._own(good, host, torch.float32, (4, 8)) == good.data_ptr()
    for t, d, dtype, shape in ((good, 0, torch.float32, (4, 8)), (good, host, torch.int32, (4, 8)), (good, host, torch.float32, (8, 4)), (good[:, :4], host, torch.float32, (4, 4))):
        with pytest.raises(AssertionError):
            spd._own(t, d, dtype, shape)
    for t, d in ((good, host), (good.to(torch.uint8), 0), (good.to(torch.uint8)[:, :4], host)):
        with pytest.raises(AssertionError):
            spd._scratch(t, d)


def test_model_bytes_in_4_bits():
    from paper_2404_08856_amd import spd, synth
    s = synth.SHAPES["llama7b"]
    cfg = spd.make_config(s, 1, 1024)
    p16, kv16, _ = spd.spd_model_bytes(cfg)
    embed = s.vocab * s.d_model * 2
    for group in (32, 64, 128):
        p4, kv4, ws = spd.spd_model_bytes_q4(cfg, group)
        assert kv4 == kv16 and ws > 0
        weights = s.streamed_weight_bytes() / 2                # 4 bits each and 16 a group
        assert weights * (0.5 + 2 / group) + embed <= p4 < 1.01 * (weights * (0.5 + 2 / group) + embed)
    with pytest.raises(spd.SpdError) as e:
        spd.spd_model_bytes_q4(cfg, 48)
    assert e.value.code == spd.SPD_ERR_SHAPE
