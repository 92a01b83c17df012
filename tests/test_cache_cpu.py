"""Host side of the growing cache, on the CPU: the index rules that keep every access in
its buffer, and the refusals of the C ABI and of the binding (all before any device work,
so the pointers here are never followed)."""
import ctypes
import gc
import os
import shutil
import subprocess
import weakref

import numpy as np
import pytest
import torch

import oracle
import paper_2607_17715_amd as c2kv
from oracle import cache_oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_index_rules_hold_for_any_device_array(tmp_path):
    exe = str(tmp_path / "cache_index")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I",
                    os.path.join(ROOT, "paper_2607_17715_amd", "csrc"),
                    os.path.join(ROOT, "tests", "cache_index.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe, "4000", "5"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:]
    assert int(r.stdout.split()[1]) > 10000, r.stdout


P = 1 << 20                      # an aligned address that no call may follow


def _args(**kw):
    a = dict(hq=8, hkv=2, d=128, act=c2kv.C2KV_BF16, base=1e4, scale=0.0, store=c2kv.C2KV_BF16,
             k=P, v=P, ks=None, vs=None, n_pages=4, page=64, batch=2, n_tokens=5, tok_off=P,
             kv_len=P, table=P, max_pages=3, max_chunk=0, max_kv=0, rows=P, rows2=P, stride=0)
    a.update(kw)
    cfg = c2kv.AttnCfg(a["hq"], a["hkv"], a["d"], a["act"], a["base"], a["scale"])
    cache = c2kv.CacheDesc(a["store"], a["k"], a["v"], a["ks"], a["vs"], a["n_pages"], a["page"])
    ch = c2kv.ChunksDesc(a["batch"], a["n_tokens"], a["tok_off"], a["kv_len"], a["table"],
                         a["max_pages"], a["max_chunk"], a["max_kv"])
    return a, cfg, cache, ch


def _calls(a, cfg, cache, ch):
    r, lib = ctypes.byref, c2kv.lib()
    nbytes = ctypes.c_size_t()
    pool = c2kv.PoolDesc(a["store"], a["k"], a["v"], a["ks"], a["vs"], 10)
    return {
        "write": lambda: lib.c2kv_cache_write(r(cfg), r(cache), r(ch), a["rows"], a["stride"],
                                              a["rows2"], a["stride"], None, None),
        "read": lambda: lib.c2kv_cache_read(r(cfg), r(cache), r(ch), None, a["rows"], a["rows2"],
                                            None),
        "attend": lambda: lib.c2kv_cache_attend(r(cfg), r(cache), r(ch), a["rows"], a["stride"],
                                                None, a["rows2"], None, P, 1 << 40, None),
        "workspace": lambda: lib.c2kv_cache_attend_workspace(r(cfg), r(cache), r(ch), r(nbytes)),
        "pool": lambda: lib.c2kv_pool_write(r(cfg), r(pool), a["n_tokens"], P, a["rows"],
                                            a["stride"], a["rows2"], a["stride"], None, None),
    }


INVAL, UNSUP = c2kv.C2KV_E_INVAL, c2kv.C2KV_E_UNSUPPORTED
ALL = ("write", "read", "attend", "workspace", "pool")
CACHE = ALL[:4]
ROWS = ("write", "read", "attend", "pool")


@pytest.mark.parametrize("kw,calls,status,text", [
    (dict(hq=7), ALL, INVAL, "multiple"),
    (dict(hkv=0), ALL, INVAL, "multiple"),
    (dict(d=96), ALL, UNSUP, "96"),
    (dict(act=c2kv.C2KV_I8), ALL, INVAL, "act_dtype"),
    (dict(base=0.0), ALL, INVAL, "rope_base"),
    (dict(base=float("nan")), ALL, INVAL, "rope_base"),
    (dict(scale=float("inf")), ALL, INVAL, "softmax_scale"),
    (dict(hq=1 << 17, hkv=1 << 16), ALL, UNSUP, "query heads"),
    (dict(k=None), ALL, INVAL, "NULL"),
    (dict(v=None), ALL, INVAL, "NULL"),
    (dict(store=7), ALL, INVAL, "dtype"),
    (dict(store=c2kv.C2KV_F32), ALL, UNSUP, "combination"),
    (dict(store=c2kv.C2KV_I8, act=c2kv.C2KV_F32), ALL, UNSUP, "combination"),
    (dict(store=c2kv.C2KV_I8, ks=P), ALL, INVAL, "scale"),
    (dict(store=c2kv.C2KV_I8, ks=P, vs=P + 4), ALL, INVAL, "16 bytes"),
    (dict(k=P + 2), ALL, INVAL, "16 bytes"),
    (dict(n_pages=-1), CACHE, INVAL, "n_pages"),
    (dict(page=0), CACHE, INVAL, "page_size"),
    (dict(page=96), CACHE, INVAL, "page_size"),
    (dict(page=1 << 17), CACHE, UNSUP, "65536"),
    (dict(batch=0), CACHE, INVAL, "batch"),
    (dict(n_tokens=-1), CACHE, INVAL, "n_tokens"),
    (dict(n_tokens=-1), ("pool",), INVAL, "n and n_rows"),
    (dict(max_chunk=-1), CACHE, INVAL, "max_chunk"),
    (dict(max_kv=-2), CACHE, INVAL, "max_kv"),
    (dict(max_pages=0), CACHE, INVAL, "max_pages"),
    (dict(tok_off=None), CACHE, INVAL, "NULL"),
    (dict(kv_len=None), CACHE, INVAL, "NULL"),
    (dict(table=None), CACHE, INVAL, "NULL"),
    (dict(max_pages=1 << 25), CACHE, UNSUP, "2^30"),
    (dict(n_tokens=1 << 30), CACHE, UNSUP, "2^31"),
    (dict(rows=None), ROWS, INVAL, "NULL"),
    (dict(rows2=None), ROWS, INVAL, "NULL"),
    (dict(rows=P + 8), ROWS, INVAL, "16 bytes"),
    (dict(rows2=P + 8), ROWS, INVAL, "16 bytes"),
    (dict(stride=128), ("write", "attend", "pool"), INVAL, "stride"),
    (dict(stride=-2048), ("write", "attend", "pool"), INVAL, "stride"),
    (dict(stride=1028), ("write", "attend", "pool"), INVAL, "16 bytes"),
])
def test_refusals(kw, calls, status, text):
    built = _args(**kw)
    for name in calls:
        st = _calls(*built)[name]()
        msg = c2kv.lib().c2kv_last_error().decode()
        assert st == status and text in msg, (name, st, msg)


def test_attention_workspace_is_checked():
    a, cfg, cache, ch = _args()
    r, lib = ctypes.byref, c2kv.lib()
    n = ctypes.c_size_t()
    assert lib.c2kv_cache_attend_workspace(r(cfg), r(cache), r(ch), r(n)) == c2kv.C2KV_OK
    assert n.value > 0
    call = lambda ws, size: lib.c2kv_cache_attend(r(cfg), r(cache), r(ch), P, 0, None, P, None, ws,
                                                  size, None)
    for ws, size, text in ((None, n.value, "NULL"), (P + 128, n.value, "aligned"),
                           (P, n.value - 1, "bytes")):
        assert call(ws, size) == c2kv.C2KV_E_WORKSPACE
        assert text in lib.c2kv_last_error().decode()
    # more key tiles than the work line counts
    a, cfg, cache, ch = _args(batch=1 << 20, n_tokens=1 << 20, max_pages=1 << 24, max_chunk=1)
    for st in (lib.c2kv_cache_attend_workspace(r(cfg), r(cache), r(ch), r(n)), call(P, 1 << 40)):
        assert st == UNSUP and "2^31" in lib.c2kv_last_error().decode()


def _workspace(**kw):
    n = ctypes.c_size_t()
    a, cfg, cache, ch = _args(ks=P, vs=P, **kw)
    assert c2kv.lib().c2kv_cache_attend_workspace(*map(ctypes.byref, (cfg, cache, ch, n))) == 0
    return n.value


def _holds(groups, rows, d):
    """Two partials of `rows` rows a workgroup, and its join of 32 bytes."""
    up = lambda x: -(-x // 256) * 256
    return up(2 * groups * rows * d * 4) + up(2 * groups * rows * 8) + up(32 * groups)


@pytest.mark.parametrize("store", [c2kv.C2KV_BF16, c2kv.C2KV_I8])
@pytest.mark.parametrize("heads,d,groups,rows", [
    (1, 128, 512, 16), (16, 128, 512, 16), (16, 64, 512, 16),
    # two workgroups a CU where they fit: not with 85 KB of LDS
    (17, 128, 256, 32), (32, 128, 256, 32), (32, 64, 512, 32),
    # no two parts: blocks, which read the cache once for all heads
    (33, 128, 256, 128), (37, 64, 256, 128), (66, 128, 256, 128), (129, 128, 256, 256),
])
def test_workgroups_of_single_tokens(heads, d, groups, rows, store):
    got = _workspace(hq=heads, hkv=1, d=d, store=store, n_tokens=2, max_chunk=1, max_pages=1 << 12)
    assert got == _holds(groups, rows, d)


def test_workgroups_of_two_parts():
    """34 to 64 heads a kv-head: int8 in two parts, bf16 in blocks."""
    for d, groups in ((128, 256), (64, 512)):
        kw = dict(hq=40, hkv=1, d=d, n_tokens=2, max_chunk=1, max_pages=1 << 12)
        assert _workspace(store=c2kv.C2KV_I8, **kw) == _holds(groups, 32, d)
        assert _workspace(store=c2kv.C2KV_BF16, **kw) == _holds(256, 128, d)


@pytest.mark.parametrize("kw,calls,text", [
    (dict(hq=1, hkv=1, n_tokens=(1 << 29) + 1), CACHE, "2^29 tokens"),
    (dict(batch=(1 << 22) + 1), CACHE, "2^22 requests"),
    (dict(n_tokens=(1 << 28) + 1, hq=1, hkv=1), ("pool",), "2^28 rows"),
    # products of bounds that pass 64 bits
    (dict(hq=65535, hkv=65535, batch=1 << 22, n_tokens=1 << 15, max_pages=1 << 24),
     ("attend", "workspace"), "2^31 key tiles"),
    (dict(hq=1, hkv=1, batch=1 << 22, n_tokens=1 << 29, max_pages=1 << 24),
     ("attend", "workspace"), "2^31 key tiles"),
])
def test_what_a_launch_cannot_count_is_refused(kw, calls, text):
    built = _args(**kw)
    for name in calls:
        st = _calls(*built)[name]()
        msg = c2kv.lib().c2kv_last_error().decode()
        assert st == UNSUP and text in msg, (name, st, msg)


def test_tiles_that_a_launch_cannot_count_are_refused():
    """Each bound alone is accepted, but the tiles of both together are 2^24 workgroups."""
    built = _args(hq=1, hkv=1, batch=1 << 22, n_tokens=1 << 29)
    for name in ("write", "read"):
        st = _calls(*built)[name]()
        msg = c2kv.lib().c2kv_last_error().decode()
        assert st == UNSUP and "2^24 tiles" in msg, (name, st, msg)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_accepted_calls_have_grids_that_a_launch_counts(tmp_path):
    exe = str(tmp_path / "cache_launch")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I",
                    os.path.join(ROOT, "paper_2607_17715_amd", "csrc"),
                    os.path.join(ROOT, "tests", "cache_launch.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:]
    assert int(r.stdout.split()[1]) > 1000, r.stdout


def test_null_descriptors_are_refused():
    a, cfg, cache, ch = _args()
    lib, r = c2kv.lib(), ctypes.byref
    for c, d, e in ((None, r(cache), r(ch)), (r(cfg), None, r(ch)), (r(cfg), r(cache), None)):
        assert lib.c2kv_cache_write(c, d, e, P, 0, P, 0, None, None) == INVAL
        assert lib.c2kv_cache_read(c, d, e, None, P, P, None) == INVAL
        assert lib.c2kv_cache_attend(c, d, e, P, 0, None, P, None, P, 0, None) == INVAL
    assert lib.c2kv_cache_attend_workspace(r(cfg), r(cache), r(ch), None) == INVAL
    pool = c2kv.PoolDesc(c2kv.C2KV_BF16, P, P, None, None, 10)
    assert lib.c2kv_pool_write(r(cfg), None, 1, P, P, 0, P, 0, None, None) == INVAL
    assert lib.c2kv_pool_write(None, r(pool), 1, P, P, 0, P, 0, None, None) == INVAL
    assert lib.c2kv_pool_write(r(cfg), r(pool), 1, None, P, 0, P, 0, None, None) == INVAL


def test_calls_without_tokens_do_nothing():
    """No row: every call succeeds without a device, null rows included."""
    a, cfg, cache, ch = _args(n_tokens=0, rows=None, rows2=None)
    for name, call in _calls(a, cfg, cache, ch).items():
        assert call() == c2kv.C2KV_OK, name


def test_binding_refuses_shapes_and_types():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    with pytest.raises(ValueError):                      # v not transposed
        c2kv.Cache(z(2, 2, 64, 128), z(2, 2, 64, 128))
    with pytest.raises(ValueError):                      # scales of another shape
        c2kv.Cache(z(2, 2, 64, 128, dtype=torch.int8), z(2, 2, 128, 64, dtype=torch.int8),
                   z(2, 2, 128, dtype=torch.float32), z(2, 2, 64, dtype=torch.float32))
    with pytest.raises(ValueError):                      # not on a device
        c2kv.Cache(z(2, 2, 64, 128), z(2, 2, 128, 64))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError):                      # int64 lengths
        c2kv.Chunks(i(3), i(2).long(), i(2, 4), 5)
    with pytest.raises(ValueError):                      # one offset missing
        c2kv.Chunks(i(2), i(2), i(2, 4), 5)


@pytest.mark.parametrize("what", ["k_scale", "v_scale"])
@pytest.mark.parametrize("scale", [
    torch.ones(7, 2, dtype=torch.float16),               # half the bytes that are written
    torch.ones(7),                                       # one scale a row
    torch.ones(6, 2),                                    # a row short
    torch.ones(2, 7),
])
def test_binding_refuses_pool_scales(monkeypatch, scale, what):
    """c2kv_pool_write stores a float32 at row * H_kv + head of the scales."""
    monkeypatch.setattr(c2kv, "_dev_ptr", lambda t: None if t is None else t.data_ptr())
    k, good = torch.zeros(7, 2, 64, dtype=torch.int8), torch.ones(7, 2)
    assert c2kv.pool_desc(k, k.clone(), good, good.clone()).k_scale == good.data_ptr()
    with pytest.raises(ValueError, match="scales"):
        c2kv.pool_desc(k, k.clone(), **{"k_scale": good, "v_scale": good, what: scale})


@pytest.mark.parametrize("i", [1, 2, 3])
def test_binding_refuses_pools_over_two_devices(monkeypatch, i):
    monkeypatch.setattr(c2kv, "_dev_ptr", lambda t: None)
    t = [torch.zeros(7, 2, 64, dtype=torch.int8), torch.zeros(7, 2, 64, dtype=torch.int8),
         torch.ones(7, 2), torch.ones(7, 2)]
    c2kv.pool_desc(*t)
    t[i] = t[i].to("meta")
    with pytest.raises(ValueError, match="different devices"):
        c2kv.pool_desc(*t)


def test_host_pool_knows_its_rows(monkeypatch):
    """c2kv_pool_write writes into a host pool as into one on the device."""
    monkeypatch.setattr(c2kv.HostPool, "_put", lambda self, a: P)
    k, sc = np.zeros((7, 2, 64), np.int8), np.ones((7, 2), np.float32)
    assert c2kv.HostPool(k, k, "i8", sc, sc).desc.row_shape == (2, 64)
    for bad in (sc.astype(np.float16), sc[:6], sc[:, 0]):
        with pytest.raises(ValueError, match="scales"):
            c2kv.HostPool(k, k, "i8", sc, bad)
    for dtype in ("f32", "bf16"):
        with pytest.raises(ValueError, match="bytes an element"):
            c2kv.HostPool(k, k, dtype)


def test_pool_descriptor_keeps_its_tensors(monkeypatch):
    """Its pointers must not outlive what they point to."""
    monkeypatch.setattr(c2kv, "_dev_ptr", lambda t: t.data_ptr())
    t = [torch.zeros(7, 2, 64, dtype=torch.int8), torch.zeros(7, 2, 64, dtype=torch.int8),
         torch.ones(7, 2), torch.ones(7, 2)]
    refs = [weakref.ref(x) for x in t]
    pool = c2kv.pool_desc(*t)
    del t
    gc.collect()
    assert all(r() is not None for r in refs)
    del pool
    gc.collect()
    assert all(r() is None for r in refs)


def test_binding_refuses_rows_that_overlap():
    """A token stride of 0 (an expanded row) means dense rows to the library."""
    cfg = c2kv.attn_cfg(2, 2, 64, "bf16", 1e4)
    rows = lambda t: c2kv._rows(t, cfg, 2, 3, t.get_device(), "k")
    base = torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    c2kv._torch()
    assert rows(base) == (base.data_ptr(), 128)
    assert rows(base[::2]) == (base.data_ptr(), 256)
    for t in (base[:1].expand(4, 2, 64), base.flatten().as_strided((4, 2, 64), (64, 64, 1))):
        with pytest.raises(ValueError, match="overlap"):
            rows(t)


def test_binding_refuses_a_stream_of_another_device(monkeypatch):
    class Stream:
        device_index, cuda_stream = 1, 0
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="stream of device 1"):
        c2kv._run(lambda *a: pytest.fail("launched"), 0, Stream())


def test_cache_oracle_equals_composed_attention():
    """A cache that holds a causal sequence gives the oracle's composed attention over an
    empty composition, and the same with its pages in another order."""
    r = np.random.default_rng(4)
    n, H, D, PS = 70, 2, 64, 64
    q, k, v = (r.standard_normal((n, h, D)) for h in (4, H, H))
    ref, lse = oracle.attend(np.zeros((0, H, D)), np.zeros((0, H, D)), q, k, v, 0, 1e4)[:2]
    pos = np.arange(n)
    for table in (np.array([[0, 1]]), np.array([[2, 0]])):
        kp, vp = np.zeros((3, H, PS, D)), np.zeros((3, H, D, PS))
        where = cache_oracle.places([0, n], [n], table, PS, 3, n)
        for i, (b, j, p, o) in where.items():
            kp[p, :, o], vp[p, :, :, o] = cache_oracle.turned(k, pos, 1e4)[i], v[i]
        out, lse2, has = cache_oracle.attend(q, pos, kp, vp, [0, n], [n], table, 1e4)
        assert has.all()
        np.testing.assert_allclose(out, ref, atol=1e-12)
        np.testing.assert_allclose(lse2.T, lse, atol=1e-12)
