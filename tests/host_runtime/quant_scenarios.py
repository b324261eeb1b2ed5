"""Scenarios of tests/test_quant_host.py: each runs in a process of its own, as ``python -m tests.host_runtime.quant_scenarios NAME
FAKE_LIBRARY``, with the library's HIP calls going to fake_hip.cpp (whose kernels do nothing)."""
import ctypes
import sys

import paper_2512_15550_amd as ck
from tests.host_runtime.cache_scenarios import EINVAL, OK, PTR
from tests.host_runtime.cache_scenarios import Host as CacheHost

CODES = dict(format=ck.KV_INT8, k=PTR, ks=PTR, v=PTR, vs=PTR)


class Host(CacheHost):
    def quant_append(self, c, expect=OK, **over):
        a = dict(q=PTR, q_stride=1024, kn=PTR, k_stride=256, vn=PTR, v_stride=256, pos=None, cu=PTR, cur=PTR, table=PTR, total=10, q_out=PTR, **CODES)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_quant_append, expect, over, c, *a.values(), None)

    def read(self, c, expect=OK, **over):
        a = dict(**CODES, first=None, cur=PTR, table=PTR, out_table=PTR, cols=50, pool=100, kp=PTR, vp=PTR)
        a.update(over)
        return self.called(self.lib.ctkvr_cache_quant_read, expect, over, c, *a.values(), None)

    def attending(self, fn, c, expect, over, **more):
        a = dict(q=PTR, q_stride=1024, **CODES, cu=PTR, cur=PTR, table=PTR, total=10, **more, out=PTR, lse=None)
        a.update(over)
        return self.called(fn, expect, over, c, *a.values(), None)

    def quant_attn(self, c, expect=OK, **over):
        return self.attending(self.lib.ctkvr_cache_quant_attn, c, expect, over, slopes=None, prefix=None, first=None)

    def window(self, c, expect=OK, **over):
        return self.attending(self.lib.ctkvr_cache_window_attn, c, expect, over, window=100, sinks=4, slopes=None)

    def tree(self, c, expect=OK, **over):
        return self.attending(self.lib.ctkvr_cache_tree_attn, c, expect, over, mask=PTR, words=2, first=None)


PLAIN = dict(format=ck.KV_PLAIN, ks=None, vs=None)


def arguments(x):
    for dtype in (ck.BF16, ck.F32):
        c = x.create(dtype=dtype)
        takes_tokens, attends = (x.quant_append, x.quant_attn, x.window, x.tree), (x.quant_attn, x.window, x.tree)
        for fn in takes_tokens + (x.read,):
            fn(None, expect=EINVAL)
            for format in (ck.KV_INT8, ck.KV_FP8):
                assert fn(c, format=format) > 0
            for format in (-1, 3):
                fn(c, expect=EINVAL, format=format)
            for over in (dict(ks=None), dict(vs=None), dict(k=PTR + 8), dict(v=PTR + 4), dict(ks=PTR + 2), dict(vs=PTR + 1), dict(k=None), dict(v=None),
                         dict(cur=None), dict(table=None)):
                fn(c, expect=EINVAL, **over)
        for fn in (x.quant_append, x.read, x.quant_attn):       # they are of 8-bit rows
            fn(c, expect=EINVAL, **PLAIN)
        for fn in (x.window, x.tree):
            assert fn(c, **PLAIN) > 0
            fn(c, expect=EINVAL, format=ck.KV_PLAIN)            # plain rows have no scales
        for fn in takes_tokens:
            fn(c, expect=EINVAL, total=-1)
            fn(c, expect=EINVAL, total=65)
            assert fn(c, total=0) == 0
            for over in (dict(cu=None), dict(q=PTR + 8), dict(q_stride=1023), dict(q_stride=1020)):
                fn(c, expect=EINVAL, **over)
        for fn in attends:
            for over in (dict(q=None), dict(out=None), dict(out=PTR + 8)):
                fn(c, expect=EINVAL, **over)
        for over in (dict(q=None), dict(q_out=None), dict(kn=None), dict(vn=None), dict(k_stride=255), dict(v_stride=128), dict(kn=PTR + 2), dict(vn=PTR + 4),
                     dict(q_out=PTR + 8)):
            x.quant_append(c, expect=EINVAL, **over)
        assert x.quant_append(c, q=None, q_out=None) > 0
        for over in (dict(kp=None, vp=None), dict(kp=PTR + 8), dict(vp=PTR + 8), dict(out_table=None), dict(cols=0), dict(pool=0), dict(cols=(1 << 16) + 1),
                     dict(cols=2 ** 31 - 1)):
            x.read(c, expect=EINVAL, **over)
        assert x.read(c, kp=None, k=None, ks=None) > 0 and x.read(c, vp=None, v=None, vs=None) > 0 and x.read(c, cols=1 << 16) > 0
        for over in (dict(window=0), dict(window=-1), dict(window=-2 ** 31), dict(sinks=-1)):
            x.window(c, expect=EINVAL, **over)
        assert x.window(c, window=2 ** 31 - 1, sinks=2 ** 31 - 1) > 0
        for over in (dict(mask=None), dict(mask=PTR + 2), dict(words=0), dict(words=-1), dict(words=(1 << 15) + 1)):
            x.tree(c, expect=EINVAL, **over)
        x.lib.ctkvr_cache_free(c)


def other_device(x):
    """A handle's calls run on its device, whichever is current, and leave the current one."""
    x.fake.hipSetDevice(1)
    c = x.create()
    x.fake.hipSetDevice(0)
    for fn in (x.quant_append, x.read, x.quant_attn, x.window, x.tree):
        assert fn(c) > 0
        d = ctypes.c_int(-1)
        x.fake.hipGetDevice(ctypes.byref(d))
        assert d.value == 0
    x.lib.ctkvr_cache_free(c)
    x.fake.hipSetDevice(1)
    assert x.lib.ctkvr_release_scratch() == OK and x.fake.fake_live_bytes(1) == 0


def largest_batches(x):
    """What creation admits can be launched (fewer than 2^32 threads a dimension of a grid, fewer than 2^16 blocks in the second)."""
    for geometry in (dict(batch=1024, n_q_heads=8, n_kv_heads=8, page_size=256, max_pages=512, num_pages=2),
                     dict(batch=1, n_q_heads=1, n_kv_heads=1, page_size=1, max_pages=1 << 20, num_pages=2),
                     dict(batch=8, n_q_heads=64, n_kv_heads=8, page_size=256, max_pages=4096, num_pages=2),
                     dict(batch=(1 << 16) - 1, n_q_heads=64, n_kv_heads=64, page_size=1, max_pages=1, num_pages=2),
                     dict(batch=(1 << 13) - 1, n_q_heads=1 << 10, n_kv_heads=1 << 9, page_size=16, max_pages=2, num_pages=2)):
        for dtype in (ck.BF16, ck.F32):
            h, g = geometry["n_q_heads"], geometry["n_kv_heads"]
            c = x.create(dtype=dtype, max_new=1 << 20, **geometry)
            for total in (1, 64, 1024, 1 << 14, 1 << 16, 1 << 18, 1 << 20):
                rows = dict(total=total, q_stride=h * 128)
                assert x.quant_append(c, k_stride=g * 128, v_stride=g * 128, **rows) > 0
                for fn in (x.quant_attn, x.window, x.tree):
                    assert fn(c, **rows) > 0
                for fn in (x.window, x.tree):
                    assert fn(c, **rows, **PLAIN) > 0
            assert x.read(c, cols=(1 << 20) // geometry["page_size"]) > 0
            x.lib.ctkvr_cache_free(c)


SCENARIOS = {f.__name__: f for f in (arguments, other_device, largest_batches)}

if __name__ == "__main__":
    SCENARIOS[sys.argv[1]](Host(sys.argv[2]))
    print("ok")
