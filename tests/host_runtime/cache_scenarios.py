"""Scenarios of tests/test_cache_host.py: each runs in a process of its own, as ``python -m tests.host_runtime.cache_scenarios NAME
FAKE_LIBRARY``, with the library's HIP calls going to fake_hip.cpp (whose kernels do nothing)."""
import ctypes
import sys

import numpy as np

import paper_2512_15550_amd as ck
from paper_2512_15550_amd.binding import _CCacheParams

OK, EINVAL, EHIP, EUNSUPPORTED = 0, -1, -3, -4
PTR = 4096          # a device pointer on a 16-byte boundary
INF, NAN = float("inf"), float("nan")


class Host:
    def __init__(self, fake_path):
        self.fake = ctypes.CDLL(fake_path, mode=ctypes.RTLD_GLOBAL)
        self.fake.fake_live_bytes.restype = ctypes.c_size_t
        self.lib = ck.load_library()

    def create(self, expect=OK, freq=None, axis=None, **over):
        p = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, dtype=ck.BF16, num_pages=100, max_pages=50, max_new=64, sm_scale=0.0,
                 softcap=0.0, rope_base=10000.0)
        p.update(over)
        cp = _CCacheParams(rope_freq=None if freq is None else freq.ctypes.data, rope_axis=None if axis is None else axis.ctypes.data, **p)
        out = ctypes.c_void_p(1)
        rc = self.lib.ctkvr_cache_create(ctypes.byref(cp), None, ctypes.byref(out))
        assert rc == expect, (over, rc, ck.ctkvr_last_error())
        assert (out.value is not None) == (rc == OK) and (rc == OK or ck.ctkvr_last_error())
        return out.value

    def append(self, c, expect=OK, **over):
        a = dict(q=PTR, qs=1024, k=PTR, ks=256, v=PTR, vs=256, pos=None, cu=PTR, cur=PTR, table=PTR, total=10, q_out=PTR, kp=PTR, vp=PTR)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_append, expect, over, c, *a.values(), None)

    def attn(self, c, expect=OK, **over):
        a = dict(q=PTR, qs=1024, kp=PTR, vp=PTR, cu=PTR, cur=PTR, table=PTR, total=10, slopes=None, prefix=None, first=None, out=PTR, lse=None)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_attn, expect, over, c, *a.values(), None)

    def weights(self, c, expect=OK, **over):
        a = dict(q=PTR, qs=1024, lse=PTR, kp=PTR, cu=PTR, cur=PTR, table=PTR, total=10, slopes=None, prefix=None, first=None, decay=1.0, w_in=None,
                 w_out=PTR, stride=800)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_weights, expect, over, c, *a.values(), None)

    def evict(self, c, expect=OK, **over):
        a = dict(w_in=PTR, stride=800, cur=PTR, table=PTR, budget=100, n_init=4, n_local=10, kp=PTR, vp=PTR, w_out=None, ids=PTR, lens=None)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_evict, expect, over, c, *a.values(), None)

    def called(self, fn, expect, over, *args):
        n = self.fake.fake_launches()
        rc = fn(*args)
        assert rc == expect, (fn.__name__, over, rc, ck.ctkvr_last_error())
        done = self.fake.fake_launches() - n
        assert done == 0 or rc == OK, "launched although refused"
        return done


def parameters(x):
    for code, changes in ((EINVAL, (dict(batch=0), dict(n_q_heads=7), dict(n_kv_heads=0), dict(dtype=2), dict(num_pages=0), dict(max_pages=0),
                                    dict(max_new=0), dict(sm_scale=-1.0), dict(sm_scale=NAN), dict(sm_scale=INF), dict(softcap=-0.5), dict(softcap=NAN),
                                    dict(softcap=INF), dict(softcap=1e-7), dict(softcap=1e16), dict(sm_scale=1e16), dict(rope_base=0.0), dict(rope_base=NAN), dict(rope_base=INF))),
                          (EUNSUPPORTED, (dict(head_dim=64), dict(n_q_heads=6), dict(n_q_heads=32), dict(page_size=12), dict(page_size=512), dict(page_size=0),
                                          dict(max_pages=(1 << 16) + 1), dict(max_new=(1 << 20) + 1), dict(batch=(1 << 16) + 1)))):
        for over in changes:
            x.create(expect=code, **over)
    freq = np.ones(64)
    freq[9] = NAN
    x.create(expect=EINVAL, freq=freq)
    axis = np.zeros(64, np.uint8)
    axis[5] = 3
    x.create(expect=EINVAL, axis=axis)
    assert x.lib.ctkvr_cache_create(None, None, ctypes.byref(ctypes.c_void_p())) == EINVAL and x.lib.ctkvr_cache_create(None, None, None) == EINVAL
    x.lib.ctkvr_cache_free(None)
    for fn in (x.append, x.attn, x.weights, x.evict):
        fn(None, expect=EINVAL)
    assert "NULL" in ck.ctkvr_last_error()


def arguments(x):
    c = x.create()
    f = x.create(dtype=ck.F32)
    assert x.append(c) > 0 and x.attn(c) > 0 and x.weights(c) > 0 and x.evict(c) > 0
    for fn in (x.append, x.attn, x.weights):
        fn(c, expect=EINVAL, total=-1)
        fn(c, expect=EINVAL, total=65)
        for name in ("cu", "cur", "table"):
            fn(c, expect=EINVAL, **{name: None})
        fn(c, expect=EINVAL, q=PTR + 8)
        fn(c, expect=EINVAL, qs=1023)
        fn(c, expect=EINVAL, qs=1028)
        assert fn(f, qs=1028) > 0               # 16 bytes are four elements there
        fn(f, expect=EINVAL, qs=1026)
    # no tokens: nothing to do, but the weights decay
    assert x.append(c, total=0, q=None, k=None, v=None, q_out=None) == 0 and x.attn(c, total=0, q=None, out=None) == 0
    assert x.weights(c, total=0, q=None, lse=None) > 0
    for over in (dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(kp=None), dict(vp=None), dict(q=None, q_out=None, k=None, v=None),
                 dict(ks=255), dict(ks=260), dict(vs=128), dict(k=PTR + 2), dict(v=PTR + 4), dict(q_out=PTR + 8), dict(kp=PTR + 8), dict(vp=PTR + 8)):
        x.append(c, expect=EINVAL, **over)
    assert x.append(c, q=None, q_out=None) > 0 and x.append(c, k=None, v=None, kp=None, vp=None) > 0
    for over in (dict(q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(out=PTR + 2), dict(kp=PTR + 4), dict(vp=PTR + 4)):
        x.attn(c, expect=EINVAL, **over)
    for over in (dict(q=None), dict(lse=None), dict(kp=None), dict(w_out=None), dict(stride=799), dict(decay=NAN), dict(decay=INF), dict(kp=PTR + 4)):
        x.weights(c, expect=EINVAL, **over)
    for over in (dict(w_in=None), dict(stride=799), dict(cur=None), dict(table=None), dict(kp=None), dict(vp=None), dict(ids=None), dict(budget=0),
                 dict(budget=13), dict(n_init=-1), dict(n_local=-1), dict(n_init=2 ** 31 - 1, n_local=2 ** 31 - 1), dict(kp=PTR + 4),
                 dict(budget=(1 << 20) + 1)):
        x.evict(c, expect=EINVAL, **over)
    x.lib.ctkvr_cache_free(c)
    x.lib.ctkvr_cache_free(f)


def other_device(x):
    """A handle's calls run on its device, whichever is current, and leave the current one; so does giving it back."""
    x.fake.hipSetDevice(1)
    c = x.create()
    assert x.fake.fake_live_bytes(1) > 0 and x.fake.fake_live_bytes(0) == 0
    x.fake.hipSetDevice(0)
    for fn in (x.append, x.attn, x.weights, x.evict):
        assert fn(c) > 0
        d = ctypes.c_int(-1)
        x.fake.hipGetDevice(ctypes.byref(d))
        assert d.value == 0
    n0, n1 = x.fake.fake_syncs(0), x.fake.fake_syncs(1)
    x.lib.ctkvr_cache_free(c)
    assert x.fake.fake_syncs(0) == n0 and x.fake.fake_syncs(1) > n1
    x.fake.hipSetDevice(1)
    assert x.lib.ctkvr_release_scratch() == OK and x.fake.fake_live_bytes(1) == 0


def refused_wait(x):
    """A handle given back while its device cannot be waited for: its memory serves nothing else until it can."""
    c = x.create()
    held, n = x.fake.fake_live_bytes(0), x.fake.fake_mallocs()
    x.fake.fake_refuse_syncs(1, 0)
    x.lib.ctkvr_cache_free(c)
    d = x.create()
    assert x.fake.fake_mallocs() == n + 1 and x.fake.fake_live_bytes(0) == 2 * held
    x.fake.fake_refuse_syncs(0, 0)
    x.lib.ctkvr_cache_free(d)
    assert x.lib.ctkvr_release_scratch() == OK and x.fake.fake_live_bytes(0) == 0


def lengths_in_place(x):
    """Eviction may write the lengths over those that it read, which takes a launch behind all that read them; arrays that overlap otherwise are
    refused."""
    c = x.create(batch=5)
    apart = x.evict(c, lens=PTR + 20)
    assert x.evict(c, cur=PTR + 20, lens=PTR) == apart and x.evict(c) == apart
    assert x.evict(c, lens=PTR) == apart + 1
    for off in (4, 8, 16, -4, -16):
        x.evict(c, expect=EINVAL, lens=PTR + off)
        assert "overlaps" in ck.ctkvr_last_error()
    x.lib.ctkvr_cache_free(c)


def largest_batches(x):
    """What creation admits can be launched (fewer than 2^32 threads a dimension of a grid); what cannot is refused there."""
    for geometry in (dict(batch=1024, n_q_heads=8, n_kv_heads=8, page_size=256, max_pages=512, num_pages=2),
                     dict(batch=8, n_q_heads=64, n_kv_heads=8, page_size=256, max_pages=4096, num_pages=2),
                     dict(batch=(1 << 16) - 1, n_q_heads=64, n_kv_heads=64, page_size=1, max_pages=1, num_pages=2),
                     dict(batch=(1 << 13) - 1, n_q_heads=1 << 10, n_kv_heads=1 << 9, page_size=16, max_pages=2, num_pages=2)):
        for dtype in (ck.BF16, ck.F32):
            h, g = geometry["n_q_heads"], geometry["n_kv_heads"]
            c = x.create(dtype=dtype, max_new=1 << 20, **geometry)
            for total in (1, 64, 1024, 1 << 14, 1 << 16, 1 << 18, 1 << 20):
                rows = dict(total=total, qs=h * 128)
                assert x.append(c, ks=g * 128, vs=g * 128, **rows) > 0 and x.attn(c, **rows) > 0 and x.weights(c, stride=1 << 20, **rows) > 0
            assert x.evict(c, stride=1 << 20) > 0
            x.lib.ctkvr_cache_free(c)
    for batch, g in ((1 << 16, 64), (1 << 12, 1 << 10)):
        x.create(expect=EUNSUPPORTED, batch=batch, n_q_heads=g, n_kv_heads=g, max_pages=1)


SCENARIOS = {f.__name__: f for f in (parameters, arguments, other_device, refused_wait, lengths_in_place, largest_batches)}

if __name__ == "__main__":
    SCENARIOS[sys.argv[1]](Host(sys.argv[2]))
    print("ok")
