"""The operators on a paged cache without a GPU: arguments that are refused before anything is launched (the pointers are made up:
nothing reads them), and calls with nothing to do."""
import ctypes as C

import pytest

from paper_2603_09215_amd import binding as sb

EINVAL, ENOMEM = -1, -3
P = 1 << 20   # an aligned address that nothing follows


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


def cache(**kw):
    v = dict(dtype=1, n_pages=10, n_layers=2, n_kv_heads=2, page_tokens=16, head_dim=64, layer=1, pool=P, size=C.sizeof(sb.SparkCache))
    return sb.SparkCache(**{**v, **kw})


def batch(**kw):
    v = dict(m=3, n=2, max_pages=4, starts=P, lengths=P, table=P, size=C.sizeof(sb.SparkCacheBatch))
    return sb.SparkCacheBatch(**{**v, **kw})


def rotation(**kw):
    v = dict(rotary=64, interleaved=0, amplitude=1.0, freqs=P, positions=None, q_gain=None, k_gain=None, eps=1e-6, size=C.sizeof(sb.SparkRotation))
    return sb.SparkRotation(**{**v, **kw})


def append(lib, c=None, b=None, r=None, **kw):
    v = dict(heads=4, src=1, q=P, qs=256, k=P, ks=128, v=P, vs=128, out=2 * P, os=256)
    v.update(kw)
    return lib.spark_cache_append(c or cache(), b or batch(), r or rotation(), v["heads"], v["src"], v["q"], v["qs"], v["k"], v["ks"], v["v"], v["vs"], v["out"],
                                  v["os"], None)


def attend(lib, c=None, b=None, **kw):
    v = dict(heads=4, q=P, qs=256, scale=0.1, causal=1, out=2 * P, os=256, lse=None, ws=None, bytes=0)
    v.update(kw)
    return lib.spark_cache_attend(c or cache(), b or batch(), v["heads"], v["q"], v["qs"], v["scale"], v["causal"], v["out"], v["os"], v["lse"], v["ws"],
                                  v["bytes"], None)


def weigh(lib, c=None, b=None, **kw):
    v = dict(heads=4, q=P, qs=256, scale=0.1, causal=1, lse=P, before=None, decay=1.0, out=P)
    v.update(kw)
    return lib.spark_cache_weigh(c or cache(), b or batch(), v["heads"], v["q"], v["qs"], v["scale"], v["causal"], v["lse"], v["before"], v["decay"], v["out"], None)


def evict(lib, c=None, b=None, **kw):
    v = dict(w=P, keep=20, first=2, recent=3, table=None, pages=0, wo=P, kept=P, lengths=2 * P)
    v.update(kw)
    return lib.spark_cache_evict(c or cache(), b or batch(), v["w"], v["keep"], v["first"], v["recent"], v["table"], v["pages"], v["wo"], v["kept"], v["lengths"], None)


BAD_CACHES = [dict(size=4), dict(dtype=2), dict(dtype=-1), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(n_layers=0), dict(n_layers=(1 << 16) + 1),
              dict(n_kv_heads=0), dict(n_kv_heads=(1 << 12) + 1), dict(page_tokens=0), dict(page_tokens=24), dict(page_tokens=1 << 17), dict(head_dim=96),
              dict(head_dim=256), dict(layer=-1), dict(layer=2), dict(pool=None), dict(pool=P + 8)]
BAD_BATCHES = [dict(size=4), dict(m=-1), dict(m=(1 << 22) + 1), dict(n=-1), dict(n=(1 << 16) + 1), dict(max_pages=0), dict(max_pages=-4),
               dict(max_pages=(1 << 20) + 1), dict(lengths=None), dict(lengths=P + 2), dict(table=None), dict(table=P + 1)]


def test_caches_and_batches(lib):
    for call in (append, attend, weigh, evict):
        for kw in BAD_CACHES:
            assert call(lib, c=cache(**kw)) == EINVAL, (call, kw)
        for kw in BAD_BATCHES:
            assert call(lib, b=batch(**kw)) == EINVAL, (call, kw)
        assert call(lib, c=cache(n_kv_heads=1 << 12), b=batch(n=1 << 9), **({} if call is evict else dict(heads=1 << 12))) == EINVAL
    for call in (append, attend, weigh):
        for kw in (dict(starts=None), dict(starts=P + 2)):
            assert call(lib, b=batch(**kw)) == EINVAL, (call, kw)
        for heads in (0, -2, 3, (1 << 12) + 2):
            assert call(lib, heads=heads) == EINVAL, (call, heads)
        wide = dict(qs=4096, os=4096) if call is not weigh else dict(qs=4096)
        assert call(lib, b=batch(m=1 << 22), heads=32, **wide) == EINVAL


def test_append_arguments(lib):
    for kw in (dict(src=2), dict(src=-1), dict(q=None), dict(q=P + 1), dict(qs=255), dict(qs=-256), dict(qs=(1 << 40) + 1), dict(k=None), dict(k=P + 1), dict(ks=127),
               dict(v=None), dict(v=P + 1), dict(vs=127), dict(out=None), dict(out=2 * P + 1), dict(os=255), dict(out=P, os=264), dict(out=P, src=0)):
        assert append(lib, **kw) == EINVAL, kw
    for kw in (dict(size=4), dict(rotary=-2), dict(rotary=3), dict(rotary=66), dict(amplitude=float("nan")), dict(amplitude=float("inf")), dict(freqs=None),
               dict(freqs=P + 4), dict(positions=P + 2), dict(q_gain=P + 1), dict(k_gain=P + 2), dict(eps=-1.0), dict(eps=float("nan"))):
        assert append(lib, r=rotation(**kw)) == EINVAL, kw
    assert lib.spark_cache_append(cache(), batch(), None, 4, 1, P, 256, P, 128, P, 128, P, 256, None) == EINVAL
    assert append(lib, b=batch(m=0)) == 0
    assert append(lib, b=batch(n=0)) == 0
    assert append(lib, b=batch(m=0), r=rotation(rotary=0, freqs=None)) == 0
    assert append(lib, b=batch(m=0), out=P) == 0   # in place


def test_attend_arguments(lib):
    for kw in (dict(q=None), dict(q=P + 8), dict(qs=255), dict(qs=260), dict(out=None), dict(out=P + 8), dict(os=248), dict(os=260), dict(lse=P + 1), dict(scale=0.0),
               dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(lib, **kw) == EINVAL, kw
    assert attend(lib, b=batch(m=0)) == 0
    assert attend(lib, b=batch(n=0)) == 0
    size = C.c_size_t()
    assert lib.spark_cache_workspace_bytes(cache(), batch(), 4, None) == EINVAL
    assert lib.spark_cache_workspace_bytes(cache(), batch(), 5, C.byref(size)) == EINVAL
    assert lib.spark_cache_workspace_bytes(None, batch(), 4, C.byref(size)) == EINVAL
    assert lib.spark_cache_workspace_bytes(cache(), None, 4, C.byref(size)) == EINVAL
    for kw in BAD_CACHES[:-2]:
        assert lib.spark_cache_workspace_bytes(cache(**kw), batch(), 4, C.byref(size)) == EINVAL, kw


def test_weigh_arguments(lib):
    for kw in (dict(q=None), dict(q=P + 8), dict(qs=255), dict(qs=260), dict(lse=None), dict(lse=P + 2), dict(before=P + 2), dict(out=None), dict(out=P + 2),
               dict(scale=0.0), dict(scale=float("inf")), dict(decay=float("nan")), dict(decay=float("inf"))):
        assert weigh(lib, **kw) == EINVAL, kw
    assert weigh(lib, b=batch(n=0)) == 0


def test_evict_arguments(lib):
    for kw in (dict(w=None), dict(w=P + 2), dict(wo=None), dict(wo=P + 2), dict(kept=None), dict(kept=P + 2), dict(lengths=None), dict(lengths=P),
               dict(lengths=P + 2), dict(keep=0), dict(keep=-1), dict(keep=65), dict(first=-1), dict(recent=-1), dict(first=18), dict(first=1 << 30, recent=1 << 30),
               dict(table=P, pages=1), dict(table=P, pages=0), dict(table=P, pages=-5), dict(table=P + 2, pages=4), dict(table=P, pages=(1 << 24) + 1)):
        assert evict(lib, **kw) == EINVAL, kw
    assert evict(lib, table=P, pages=3) == EINVAL   # the batch's own table in other rows
    assert evict(lib, b=batch(n=0)) == 0


def test_scales(lib):
    for call in (attend, weigh):
        for scale in (2.0 ** 127 * 1.01, -2.0 ** 127 * 1.01, 0.0, -0.0, 1e-46, float("inf"), float("nan")):
            assert call(lib, scale=scale) == EINVAL, (call, scale)
        for scale in (2.0 ** 127, -2.0 ** 127, 1e-45):
            assert call(lib, scale=scale, b=batch(n=0)) == 0
