"""CPU-side checks of the page pool's C ABI: configurations, sizes, plans and what is refused before a device is touched."""
import ctypes
import struct

import pytest

from paper_2604_16734_b200 import binding
from paper_2604_16734_b200.binding import (KVC_BF16, KVC_EINVAL, KVC_ESTATE, KVC_F32, KVC_OK, KVC_PAGES_INT8, KVC_PAGES_PLAIN,
                                           KvcPoolConfig, KvcPromptPlan)


def create(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=KVC_BF16, page_format=KVC_PAGES_PLAIN, page_size=64, n_pages=10,
                max_seqs=4, softmax_scale=0.0, device=0, flags=0)
    base.update(kw)
    h = ctypes.c_void_p()
    return binding.lib().kvc_pool_create(ctypes.byref(KvcPoolConfig(**base)), ctypes.byref(h)), h


def test_create_validates_configuration():
    lib = binding.lib()
    rc, h = create()
    assert rc == KVC_OK and h.value and lib.kvc_pool_launch_count(h) == 0 and isinstance(lib.kvc_pool_last_error(h), bytes)
    assert lib.kvc_pool_destroy(h) == KVC_OK
    for bad in (dict(n_q_heads=7), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=258), dict(head_dim=96), dict(dtype=2), dict(page_format=2),
                dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(n_pages=0), dict(max_seqs=0), dict(max_seqs=1 << 16), dict(max_seqs=1025),
                dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(device=-1), dict(device=64),
                dict(flags=1), dict(n_pages=2 ** 31 - 1, n_kv_heads=64, n_q_heads=64)):
        rc, h = create(**bad)
        assert rc == KVC_EINVAL and not h.value, bad
    assert lib.kvc_pool_create(None, ctypes.byref(ctypes.c_void_p())) == KVC_EINVAL
    assert lib.kvc_pool_destroy(None) == KVC_ESTATE and lib.kvc_pool_launch_count(None) == -1


@pytest.mark.parametrize("dtype,fmt,row", [(KVC_BF16, KVC_PAGES_PLAIN, 2 * 128), (KVC_F32, KVC_PAGES_PLAIN, 4 * 128), (KVC_BF16, KVC_PAGES_INT8, 128 + 4),
                                           (KVC_F32, KVC_PAGES_INT8, 128 + 4)])
def test_sizes(dtype, fmt, row):
    rc, h = create(dtype=dtype, page_format=fmt, n_pages=3, page_size=32)
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert rc == KVC_OK and binding.lib().kvc_pool_nbytes(h, ctypes.byref(a), ctypes.byref(b)) == KVC_OK
    assert a.value == 2 * 3 * 2 * 32 * row and b.value >= 256
    assert binding.lib().kvc_pool_destroy(h) == KVC_OK


def test_refusals_before_a_device_is_touched():
    lib = binding.lib()
    rc, h = create()
    assert rc == KVC_OK
    P = 4096                                                    # an aligned address that is never used
    write = dict(k=P, v=P, ts=256, hs=128, slots=P, n=5, blob=P, ws=P)
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(blob=None), dict(ws=None), dict(k=P + 8), dict(v=P + 2), dict(blob=P + 4),
                dict(slots=P + 4), dict(ts=127), dict(hs=64), dict(hs=132), dict(ts=-256), dict(n=-1), dict(n=1 << 31)):
        a = {**write, **bad}
        assert lib.kvc_pool_write(h, a["k"], a["v"], a["ts"], a["hs"], a["slots"], a["n"], a["blob"], a["ws"], None) == KVC_EINVAL, bad
        assert lib.kvc_pool_read(h, a["blob"], a["slots"], a["n"], a["k"], a["v"], a["ts"], a["hs"], a["ws"], None) == KVC_EINVAL, bad
        assert lib.kvc_pool_last_error(h)
    dec = dict(q=P, qs=1024, k=P, v=P, ks=256, table=P, tst=2, lens=P, n=3, blob=P, ws=P, out=P, lse=P)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(out=None), dict(blob=None), dict(ws=None), dict(q=P + 2),
                dict(k=P + 8), dict(out=P + 4), dict(table=P + 2), dict(lens=P + 1), dict(lse=P + 2), dict(qs=1023), dict(qs=1028), dict(ks=128),
                dict(tst=0), dict(tst=-1), dict(tst=1 << 26), dict(n=5), dict(n=-1)):
        a = {**dec, **bad}
        assert lib.kvc_pool_decode(h, a["q"], a["qs"], a["k"], a["v"], a["ks"], a["table"], a["tst"], a["lens"], a["n"], a["blob"], a["ws"], a["out"],
                                   a["lse"], None) == KVC_EINVAL, bad
    plan = KvcPromptPlan()
    for lens in ([3, -1], [2 ** 31 - 1, 2 ** 31 - 1]):
        assert lib.kvc_pool_plan(h, (ctypes.c_int * 2)(*lens), 2, ctypes.byref(plan), None) == KVC_EINVAL
    assert lib.kvc_pool_plan(h, None, 1, ctypes.byref(plan), None) == KVC_EINVAL and lib.kvc_pool_plan(h, None, 0, None, None) == KVC_EINVAL
    assert lib.kvc_pool_plan(h, (ctypes.c_int * 2)(3, 4), 2, ctypes.byref(plan), None) == KVC_OK
    pro = dict(q=P, qs=1024, k=P, v=P, ks=256, items=P, ws=P, out=P, lse=P)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(items=None), dict(ws=None), dict(out=None), dict(q=P + 2), dict(items=P + 8), dict(lse=P + 2),
                dict(qs=1016), dict(qs=1025), dict(ks=255)):
        a = {**pro, **bad}
        assert lib.kvc_pool_prompt(h, a["q"], a["qs"], a["k"], a["v"], a["ks"], ctypes.byref(plan), a["items"], a["ws"], a["out"], a["lse"], None) == KVC_EINVAL, bad
    for field, value in (("n_tokens", -1), ("n_items", -1), ("row_tiles", 3), ("item_bytes", 0), ("n_tokens", 2 ** 31), ("n_q_heads", 4),
                         ("n_kv_heads", 1)):
        other = KvcPromptPlan.from_buffer_copy(plan)
        setattr(other, field, value)
        assert lib.kvc_pool_prompt(h, P, 1024, P, P, 256, ctypes.byref(other), P, P, P, P, None) == KVC_EINVAL, field
    assert lib.kvc_pool_launch_count(h) == 0
    assert lib.kvc_pool_destroy(h) == KVC_OK


@pytest.mark.parametrize("dtype,hq,hkv", [(KVC_BF16, 8, 2), (KVC_BF16, 7, 1), (KVC_BF16, 128, 1), (KVC_BF16, 32, 32), (KVC_F32, 8, 2), (KVC_F32, 7, 1)])
@pytest.mark.parametrize("lens", [[], [0, 0], [1], [0, 1, 33, 0, 128, 129, 4000], [5] * 300, [20000, 3, 700]])
def test_a_plan_covers_every_row_once_longest_first(dtype, hq, hkv, lens):
    lib = binding.lib()
    rc, h = create(dtype=dtype, n_q_heads=hq, n_kv_heads=hkv)
    assert rc == KVC_OK
    plan = KvcPromptPlan()
    arr = (ctypes.c_int * len(lens))(*lens)
    assert lib.kvc_pool_plan(h, arr, len(lens), ctypes.byref(plan), None) == KVC_OK
    units = plan.n_items * (1 if dtype == KVC_F32 else hkv)
    ctas = min(units, 148)
    held = 16 * units + (0 if dtype == KVC_F32 else -(-ctas // 4) * 16)
    assert (plan.n_seqs, plan.n_tokens, plan.item_bytes) == (len(lens), sum(lens), held)
    buf = ctypes.create_string_buffer(plan.item_bytes + 16)
    assert lib.kvc_pool_plan(h, arr, len(lens), ctypes.byref(plan), buf) == KVC_OK
    assert buf.raw[plan.item_bytes:] == bytes(16)
    G = hq // hkv
    starts, first = {}, 0
    for n in lens:
        if n:
            starts[first] = n
        first += n
    entries = list(struct.iter_unpack("4i", buf.raw[:16 * units]))
    per, step = (plan.row_tiles / G, 1) if dtype == KVC_F32 else (128 // G, 2)
    tiles_of = {a: -(-n * G // plan.row_tiles) if dtype == KVC_F32 else -(-n // per) for a, n in starts.items()}
    keys = lambda e: min(e[1], (e[2] + step) * per)  # noqa: E731
    if dtype == KVC_F32:                                     # pieces for all kv-heads, those with the most keys first
        want = {(a, t) for a in starts for t in range(tiles_of[a])}
        work = [-(-min(e[1], -(-(e[2] + 1) * plan.row_tiles // G)) // 128) for e in entries]
        assert work == sorted(work, reverse=True)
        lists = [[(e[0], e[1], e[2])] for e in entries]
    else:                                                    # a list per CTA, its first units in front, its last unit marked
        others = list(struct.unpack(f"{ctas}i", buf.raw[16 * units:16 * units + 4 * ctas]))
        assert others == sorted(others) and all(ctas <= x <= units for x in others)
        want = {(a, t, g) for a in starts for t in range(0, tiles_of[a], step) for g in range(hkv)}
        lists = [[entries[i]] + entries[others[i]:(others + [units])[i + 1]] for i in range(ctas)]
        for x in lists:
            assert [e[3] < 0 for e in x] == [False] * (len(x) - 1) + [True]
        lists = [[(e[0], e[1], e[2], e[3] if e[3] >= 0 else ~e[3]) for e in x] for x in lists]
        load = [sum(-(-keys(e) // 128) + 1 for e in x) for x in lists]
        if load:                                             # nobody has more than one unit above the least
            assert max(load) - min(load) <= max(-(-keys(e) // 128) + 1 for e in entries)
    flat = [e for x in lists for e in x]
    assert all(starts[e[0]] == e[1] for e in flat) and all(0 <= e[2] * per < e[1] for e in flat)
    seen = [(e[0], e[2], *e[3:]) for e in flat]
    assert len(seen) == len(set(seen)) and set(seen) == want
    assert lib.kvc_pool_destroy(h) == KVC_OK


def test_pool_refuses_to_run_without_a_gpu():
    import torch

    from paper_2604_16734_b200.pool import Pool
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(RuntimeError):
        Pool(8, 2, 128, torch.bfloat16, 4)
