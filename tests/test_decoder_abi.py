"""A decoder's operators at the boundary, without a GPU: what is refused before anything is launched, what does nothing, the rotation table, and the oracle
against closed forms and the encoder's own attention."""
import ctypes as C
import os
import shutil
import subprocess
import sys

import numpy as np
import pytest

import paper_2604_28175_amd as S
from oracle import decoder as D
from oracle import ops

A = 4096                                  # an address that nothing looks at: every call here ends before a launch
OK, INVALID, SHAPE, NOMEM = S.OK, S.E_INVALID, S.E_SHAPE, S.E_NOMEM


def cache(**over):
    d = dict(k=A, v=A, k_scale=A, v_scale=A, type=S.KV_I8, pages=10, page_tokens=64, kv_heads=2, head_dim=128)
    d.update(over)
    return S.KvCacheDesc(*[d[n] for n, _ in S.KvCacheDesc._fields_])


def batch(**over):
    d = dict(q_start=A, kv_len=A, page_table=A, seqs=3, tokens=9, max_q=4, max_kv=300, table_pitch=5)
    d.update(over)
    return S.KvBatchDesc(*[d[n] for n, _ in S.KvBatchDesc._fields_])


def quantize(x=A, M=4, K=64, pitch=64, q=A, scale=A):
    return S.lib.strait_k_quantize_rows(None, x, M, K, pitch, q, scale, 0)


@pytest.mark.parametrize("over,status", [(dict(M=-1), INVALID), (dict(K=0), INVALID), (dict(K=72), SHAPE), (dict(x=None), INVALID), (dict(x=A + 8), INVALID), (dict(pitch=56), INVALID),
                                         (dict(pitch=68), INVALID), (dict(q=None), INVALID), (dict(q=A + 4), INVALID), (dict(scale=None), INVALID), (dict(scale=A + 2), INVALID),
                                         (dict(M=0, x=None), OK)])
def test_quantize_rows_refuses(over, status):
    assert quantize(**over) == status
    assert status == OK or "quantize_rows" in S.last_error()


def gemm(x=A, xs=A, w=A, ws=A, bias=A, M=4, N=8, K=64, act=0, res=None, y=A, out_f32=0):
    return S.lib.strait_k_gemm_i8(None, x, xs, w, ws, bias, M, N, K, act, res, y, out_f32, 0)


@pytest.mark.parametrize("over,status", [(dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(K=8), SHAPE), (dict(K=131072), SHAPE), (dict(act=4), INVALID), (dict(act=-1), INVALID),
                                         (dict(x=None), INVALID), (dict(xs=None), INVALID), (dict(w=None), INVALID), (dict(ws=None), INVALID), (dict(y=None), INVALID), (dict(x=A + 8), INVALID),
                                         (dict(w=A + 1), INVALID), (dict(y=A + 1), INVALID), (dict(y=A + 2, out_f32=1), INVALID), (dict(res=A + 1), INVALID), (dict(bias=A + 2), INVALID),
                                         (dict(M=0, x=None, y=None), OK)])
def test_gemm_i8_refuses(over, status):
    assert gemm(**over) == status
    assert status == OK or "gemm_i8" in S.last_error()


BAD_CACHE = [dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 1), dict(k_scale=None), dict(v_scale=None), dict(type=2), dict(pages=0), dict(kv_heads=0)]
BAD_CACHE_SHAPE = [dict(page_tokens=16), dict(page_tokens=48), dict(page_tokens=512), dict(head_dim=96), dict(head_dim=256), dict(pages=1 << 30, kv_heads=2)]
BAD_BATCH = [dict(q_start=None), dict(kv_len=None), dict(page_table=None), dict(seqs=-1), dict(tokens=-1), dict(max_q=0), dict(max_q=10), dict(max_kv=0), dict(table_pitch=4),
             dict(max_kv=0x7fffffff)]


def append(c, b, q=A, k=A, v=A, pq=512, pk=256, pv=256, heads=4, rope=A, rows=300, dim=128, q_out=A):
    return S.lib.strait_k_kv_append(None, c and C.byref(c), b and C.byref(b), q, k, v, pq, pk, pv, heads, rope, rows, dim, 0, q_out, 0)


def attend(c, b, q=A, pq=512, heads=4, scale=0.1, window=0, sinks=0, out=A, ws=A, ws_bytes=1 << 40):
    return S.lib.strait_k_attention_paged(None, c and C.byref(c), b and C.byref(b), q, pq, heads, scale, window, sinks, out, ws, ws_bytes, 0)


@pytest.mark.parametrize("call,name", [(append, "kv_append"), (attend, "attention_paged")])
def test_caches_and_batches_that_do_not_fit_are_refused(call, name):
    assert call(None, batch()) == INVALID and call(cache(), None) == INVALID
    for over in BAD_CACHE:
        assert call(cache(**over), batch()) == INVALID, over
        assert S.last_error().startswith(name)
    for over in BAD_CACHE_SHAPE:
        assert call(cache(**over), batch()) == SHAPE, over
    for over in BAD_BATCH:
        assert call(cache(), batch(**over)) == INVALID, over
    for over in (dict(tokens=0), dict(seqs=0)):
        assert call(cache(), batch(**over)) == OK, over
    assert call(cache(), batch(), heads=3) == INVALID and call(cache(), batch(), heads=0) == INVALID
    assert call(cache(), batch(), heads=1 << 17) == SHAPE


@pytest.mark.parametrize("over,status", [(dict(k=None), INVALID), (dict(v=A + 2), INVALID), (dict(pk=248), INVALID), (dict(pv=260), INVALID), (dict(q=A, q_out=None), INVALID),
                                         (dict(q=None), INVALID), (dict(pq=504), INVALID), (dict(q_out=A + 8), INVALID), (dict(pq=1024), INVALID),
                                         (dict(dim=8), SHAPE), (dict(dim=24), SHAPE), (dict(dim=144), SHAPE), (dict(rows=299), INVALID), (dict(rope=A + 4), INVALID), (dict(rope=None), INVALID)])
def test_kv_append_refuses(over, status):
    assert append(cache(), batch(), **over) == status and S.last_error().startswith("kv_append")


@pytest.mark.parametrize("over,status", [(dict(q=None), INVALID), (dict(q=A + 2), INVALID), (dict(pq=510), INVALID), (dict(pq=504), INVALID), (dict(out=None), INVALID), (dict(out=A + 8), INVALID),
                                         (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
                                         (dict(window=-1), INVALID), (dict(sinks=-1), INVALID)])
def test_attention_paged_refuses(over, status):
    assert attend(cache(), batch(), **over) == status and S.last_error().startswith("attention_paged")


def test_attention_paged_says_what_workspace_it_needs():
    need = C.c_size_t(1)
    ask = lambda c, b, heads=4, window=0, sinks=0: S.lib.strait_k_attention_paged_workspace(C.byref(c), C.byref(b), heads, window, sinks, C.byref(need))
    assert ask(cache(), batch(tokens=0)) == OK and need.value == 0
    assert ask(cache(), batch(), heads=3) == INVALID and need.value == 0
    assert S.lib.strait_k_attention_paged_workspace(C.byref(cache()), C.byref(batch()), 4, 0, 0, None) == INVALID
    long = batch(seqs=1, tokens=1, max_q=1, max_kv=100000, table_pitch=4000)
    assert ask(cache(), long) == OK
    if need.value:
        assert attend(cache(), long, ws=None) == NOMEM and attend(cache(), long, ws_bytes=need.value - 1) == NOMEM and "workspace" in S.last_error()
        assert attend(cache(), long, ws=A + 4) == INVALID


def test_what_a_launch_cannot_hold_is_refused():
    assert quantize(M=1 << 24) == SHAPE and quantize(M=1 << 24, K=4096, pitch=4096) == SHAPE
    big = 0x7fffffff
    for m, n in ((1, big), (20, big), (big, 1), (big, 64), (1 << 24, 1 << 24), (big, big)):
        assert gemm(M=m, N=n, K=16) == SHAPE, (m, n)
    for call in (append, attend):
        assert call(cache(), batch(max_kv=(1 << 29) + 1, table_pitch=1 << 24)) == SHAPE and "max_kv" in S.last_error()
    assert append(cache(kv_heads=4), batch(seqs=1 << 23, tokens=1 << 23, max_q=1), pk=512, pv=512) == SHAPE
    assert attend(cache(), batch(seqs=1 << 24, max_q=1), heads=2, ws_bytes=1 << 62) == SHAPE


def test_a_product_goes_into_its_residual_in_fp16_only():
    assert gemm(res=A, y=A, out_f32=1) == INVALID and "y may be res" in S.last_error()


def test_parts_take_room_only_for_what_is_joined():
    """A long prompt beside single tokens: room for the parts of a few tokens of each sequence, not of the prompt's."""
    need = C.c_size_t(0)
    b = batch(seqs=8, tokens=8192 + 7, max_q=8192, max_kv=131072, table_pitch=2048)
    assert S.lib.strait_k_attention_paged_workspace(C.byref(cache()), C.byref(b), 8, 0, 0, C.byref(need)) == OK
    rows = 8 * 4 * 8                                      # sequences, tokens of 16 rows, heads
    assert 0 < need.value <= rows * 131072 // 32 // 8 * (128 + 2) * 4 + 16


@pytest.mark.parametrize("positions,dim,base", [(1, 2, 10000.0), (70001, 64, 10000.0), (500, 128, 500000.0)])
def test_rope_table(positions, dim, base):
    t = S.rope_table(positions, dim, base)
    angle = np.arange(positions, dtype=np.longdouble)[:, None] * np.longdouble(base) ** (-2 * np.arange(dim // 2, dtype=np.longdouble) / dim)
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float64)
    # half a step of fp32, and the angle's own rounding in 64 bits (position * 2^-52)
    assert t.shape == (positions, dim) and np.abs(t - want).max() <= 2.0 ** -25 + positions * 2.0 ** -51


def test_rope_table_refuses():
    for args in ((-1, 4, 1e4), (4, 3, 1e4), (4, 0, 1e4), (4, 4, 0.0), (4, 4, float("nan")), (4, 4, float("inf"))):
        with pytest.raises(S.StraitError) as e:
            S.rope_table(*args)
        assert e.value.status == INVALID
    assert S.rope_table(0, 4).shape == (0, 4)


def test_the_binding_refuses_what_is_not_on_a_gpu_or_of_another_type():
    import torch
    x = torch.zeros(4, 64, dtype=torch.float16)
    for call in (lambda: S.k_quantize_rows(x), lambda: S.k_gemm_i8(x, x, x, x), lambda: S.KvCache(x, x), lambda: S.KvCache(x.int(), x), lambda: S.KvBatch(x, x, x, 1, 1)):
        with pytest.raises(S.StraitError) as e:
            call()
        assert e.value.status == INVALID


# ---- the oracle's own pins

def test_oracle_quantize_rows_and_product():
    r = np.random.default_rng(5)
    x = r.standard_normal((6, 48)).astype(np.float16)
    x[2], x[3, 5], x[4, 1] = 0, np.inf, np.nan
    q, s = D.quantize_rows(x)
    assert np.isnan(s[[3, 4]]).all() and not q[[2, 3, 4]].any() and s[2] == 0 and (np.abs(q[[0, 1, 5]]).max(1) == 127).all()
    assert (np.abs(q[:2] * s[:2, None].astype(np.float64) - x[:2]) <= 0.5 * s[:2, None] * (1 + 1e-6)).all()
    w, ws = r.integers(-128, 128, (5, 48)).astype(np.int8), np.ones(5, np.float32)
    assert np.array_equal(D.gemm_i8(q[:2], np.ones(2, np.float32), w, ws), (q[:2].astype(int) @ w.T.astype(int)).astype(float))


def test_oracle_rotation():
    r = np.random.default_rng(6)
    x = r.standard_normal((3, 64))
    for inter in (False, True):
        y = D.rotate(x, 1234, 32, 10000.0, inter)
        a, b = D.pair(32, inter)
        assert np.allclose(y[:, a] ** 2 + y[:, b] ** 2, x[:, a] ** 2 + x[:, b] ** 2) and np.array_equal(y[:, 32:], x[:, 32:])
        # a product of two rotated vectors depends on the distance of their positions alone
        z = r.standard_normal((3, 64))
        dots = [(D.rotate(x, p, 64, 10000.0, inter) * D.rotate(z, p + 7, 64, 10000.0, inter)).sum(1) for p in (0, 900)]
        assert np.allclose(*dots)
        table = S.rope_table(1235, 32)
        assert np.allclose(D.rotate32(x.astype(np.float32), table[1234], inter), y, atol=1e-6)


def test_oracle_attention_is_the_encoders_where_nothing_is_masked():
    r = np.random.default_rng(7)
    qkv = r.standard_normal((1, 9, 3 * 64)).astype(np.float16)
    want = ops.attention(qkv[..., :64], qkv[..., 64:128], qkv[..., 128:], np.array([9]), 1)[0]
    q, k, v = (qkv[0, :, 64 * i:64 * i + 64].astype(np.float64) for i in range(3))
    got, _ = D.attention(q, k, v, np.full(9, 8), 0.125, 0, 0)
    assert np.allclose(got, want, atol=1e-12)
    # window and sinks by hand: position 5 of 9 keys, window 2, 1 sink sees 0, 4, 5
    one, _ = D.attention(q[:1], k, v, np.array([5]), 0.125, 2, 1)
    few, _ = D.attention(q[:1], k[[0, 4, 5]], v[[0, 4, 5]], np.array([2]), 0.125, 0, 0)
    assert np.allclose(one, few, atol=1e-12)
    assert not D.attention(q[:1], k, v, np.array([-1]), 0.125, 0, 0)[0].any()


def test_oracle_append_in_pieces():
    """What the codes stand for stays within half a step of each scale that a page has had."""
    r = np.random.default_rng(8)
    codes, scale = np.zeros((3, 2, 32, 64), np.int8), np.full((3, 2), np.nan, np.float32)
    table, x = np.array([[2, 0]]), r.standard_normal((50, 2, 64)).astype(np.float16)
    steps = np.zeros((3, 2))
    for lo, hi in ((0, 1), (1, 20), (20, 21), (21, 50)):
        where = list(D.places([0, hi - lo], [hi], table, 32, 3, 50, 64, hi - lo))
        before = scale.copy()
        D.append_int8(codes, scale, x[lo:hi], where, None, False)
        steps += np.where(scale != before, np.nan_to_num(scale), 0)
        for t in range(hi):
            g, row = table[0][t // 32], t % 32
            assert (np.abs(codes[g, :, row] * scale[g][:, None].astype(np.float64) - x[t]) <= 0.5001 * np.maximum(steps[g], scale[g])[:, None]).all()
    assert np.isnan(scale[1]).all()


def test_attention_over_more_sequences_than_a_launch_holds_is_refused():
    """Also where the number of tiles that are found by counting, or a product of sizes, would leave its type."""
    big = 0x7fffffff
    need = C.c_size_t(1)
    for seqs, heads, tokens, max_q, max_kv in ((big, 1, 1000, 1000, 1), (big, 1, 1000, 1000, 1 << 29), (big, 1 << 16, 1, 1, 1 << 29), (big, 1 << 15, 100, 100, 1 << 20), (1 << 30, 1 << 10, 8, 8, 1 << 28),
                                               (big - 100, 2, 5000, 300, 64)):
        for kind in (S.KV_F16, S.KV_I8):
            c, b = cache(type=kind, pages=1, kv_heads=heads), batch(seqs=seqs, tokens=tokens, max_q=max_q, max_kv=max_kv, table_pitch=1 << 24)
            assert attend(c, b, pq=heads * 128, heads=heads, ws_bytes=1 << 62) == SHAPE, (seqs, heads, tokens, max_q, max_kv)
            assert S.lib.strait_k_attention_paged_workspace(C.byref(c), C.byref(b), heads, 0, 0, C.byref(need)) == SHAPE and need.value == 0


def test_a_workspace_that_is_missing_or_too_small_or_misaligned_is_refused():
    """One token over a long cache is shared out over parts, so it needs room."""
    need = C.c_size_t(0)
    long = batch(seqs=1, tokens=1, max_q=1, max_kv=100000, table_pitch=4000)
    for kind in (S.KV_F16, S.KV_I8):
        assert S.lib.strait_k_attention_paged_workspace(C.byref(cache(type=kind)), C.byref(long), 4, 0, 0, C.byref(need)) == OK and need.value > 0
        assert attend(cache(type=kind), long, ws=None) == NOMEM and "workspace" in S.last_error()
        assert attend(cache(type=kind), long, ws_bytes=need.value - 1) == NOMEM and attend(cache(type=kind), long, ws_bytes=0) == NOMEM
        assert attend(cache(type=kind), long, ws=A + 4, ws_bytes=need.value) == INVALID and "workspace" in S.last_error()


DEVICES = """
import ctypes, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)          # ahead of the runtime that the library brings along
sys.path.insert(0, sys.argv[2])
from paper_2604_28175_amd.binding import lib
A = 4096
recorded = lambda what: ctypes.c_int.in_dll(recorder, "recorded_" + what)
counts = []
for device in (0, 1, 0, 7, 63, 64, 100, 1, 64):
    recorded("device").value = device
    for m, n, k in ((1, 64, 64), (40, 8192, 4096), (128, 4096, 4096), (509, 5003, 2064), (512, 4096, 4096), (512, 5120, 2048), (2048, 4096, 4096), (8192, 16384, 4096)):
        for res, f32 in ((None, 0), (A, 0), (None, 1)):
            assert lib.strait_k_gemm_i8(None, A, A, A, A, None, m, n, k, 0, res, A, f32, 0) == 0, lib.strait_last_error()
    counts.append(recorded("asked").value)
print(counts, recorded("wide").value, recorded("unasked").value)
sys.exit(0 if recorded("wide").value > 100 and recorded("unasked").value == 0 and counts[1] == 2 * counts[0] and counts[2] == counts[1] else 1)
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_lds_beyond_the_default_is_asked_for_on_every_device(tmp_path):
    """The attribute belongs to a device's copy of a kernel; tests/native/devices_recorder.c stands in for the runtime."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    recorder = str(tmp_path / "recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", recorder, os.path.join(root, "tests", "native", "devices_recorder.c")], check=True)
    r = subprocess.run([sys.executable, "-c", DEVICES, recorder, root], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-1500:] + r.stderr[-1500:]
