"""Host side of the paged key-value cache: refusals that need no GPU.  Addresses are made up; a refused call touches none."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
from paper_1712_01084_b200 import binding as pb

INVALID, UNSUPPORTED = 1, 6
AT = 1 << 40            # an address


def _cache(**kw):
    f = dict(k=AT, v=AT + (1 << 30), k_scales=None, v_scales=None, k_page=16 * 2 * 64, k_token=2 * 64, k_head=64, v_page=16 * 2 * 64, v_token=2 * 64, v_head=64,
             pages=10, page_size=16, kv_heads=2, head_dim=64, dtype=pb.PP_BF16)
    f.update(kw)
    return pb._PagedCacheC(*(f[n] for n, _ in pb._PagedCacheC._fields_))


def _space(cache, q_type=pb.PP_BF16, batch=0, heads=4, width=5, window=0):
    out = ctypes.c_int64(-1)
    st = pb.lib().pp_paged_attention_workspace(None if cache is None else ctypes.addressof(cache), q_type, batch, heads, width, window, ctypes.byref(out))
    return st, out.value


Q8 = dict(dtype=pb.PP_E4M3, k_scales=AT + (2 << 30), v_scales=AT + (3 << 30))
BAD_CACHES = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(v=AT), INVALID), (dict(pages=0), INVALID), (dict(page_size=0), INVALID), (dict(kv_heads=0), INVALID),
              (dict(head_dim=0), INVALID), (dict(dtype=9), UNSUPPORTED), (dict(head_dim=257, k_head=257, k_token=514, k_page=1 << 20, v_head=257, v_token=514, v_page=1 << 20), UNSUPPORTED),
              (dict(page_size=(1 << 20) + 1), UNSUPPORTED), (dict(pages=2 ** 31 - 1, page_size=1024), UNSUPPORTED), (dict(k_scales=AT), INVALID), (dict(dtype=pb.PP_I8), INVALID),
              (dict(Q8, v_scales=None), INVALID), (dict(Q8, v_scales=Q8["k_scales"]), INVALID), (dict(k=AT + 1), INVALID), (dict(Q8, k_scales=AT + 2), INVALID),
              (dict(k_page=-1), INVALID), (dict(v_token=1 << 60), INVALID), (dict(k_head=63), INVALID), (dict(k_token=127), INVALID), (dict(v_page=0), INVALID),
              (dict(k_page=2047), INVALID), (dict(k_token=64, k_head=64), INVALID)]


@pytest.mark.parametrize("case", range(len(BAD_CACHES)))
def test_descriptions_of_a_cache(case):
    change, want = BAD_CACHES[case]
    assert _space(_cache(**change))[0] == want
    assert pb.lib().pp_kv_append(ctypes.addressof(_cache(**change)), None, 0, 0, 0, None, 0, 0, AT, 128, 64, AT, 128, 64, pb.PP_BF16, 1, AT, None, None, 0, 0, None) == want


def test_good_descriptions_of_a_cache():
    assert _space(None)[0] == INVALID
    assert _space(_cache()) == (0, 0)
    assert _space(_cache(**Q8), pb.PP_F32) == (0, 0)
    assert _space(_cache(k_token=64, k_head=16 * 64)) == (0, 0)                              # head by head
    assert _space(_cache(k_page=1 << 40, k_token=200, k_head=70)) == (0, 0)                  # rows with gaps
    assert _space(_cache(pages=1, k_page=0)) == (0, 0)                                       # an axis of one entry has no distance
    assert _space(_cache(page_size=1, kv_heads=1, k_token=0, k_head=0, v_token=0, v_head=0)) == (0, 0)


def test_calls_that_the_workspace_refuses():
    c = _cache()
    assert pb.lib().pp_paged_attention_workspace(ctypes.addressof(c), pb.PP_BF16, 0, 4, 5, 0, None) == INVALID
    for kw, want in ((dict(q_type=pb.PP_F16), UNSUPPORTED), (dict(q_type=pb.PP_E4M3), UNSUPPORTED), (dict(batch=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID),
                     (dict(width=0), INVALID), (dict(window=-1), INVALID), (dict(width=2 ** 31 // 16), UNSUPPORTED), (dict(heads=1 << 21), UNSUPPORTED),
                     (dict(batch=1 << 20, heads=1 << 14), UNSUPPORTED)):
        assert _space(c, **kw)[0] == want, kw


def _attend(c, **kw):
    f = dict(q=AT, q_row=256, q_head=64, q_type=pb.PP_BF16, table=AT, ld_table=5, width=5, lengths=AT, batch=2, heads=4, scale=0.125, window=0, out=AT + 4096, lse=None,
             workspace=None, workspace_bytes=0)
    f.update(kw)
    return pb.lib().pp_paged_attention(ctypes.addressof(c), *f.values(), None)


def test_attention_calls_that_are_refused():
    c = _cache()
    for kw in (dict(q=None), dict(table=None), dict(lengths=None), dict(out=None), dict(q_row=-1), dict(q_head=-1), dict(q_row=1 << 60), dict(ld_table=4), dict(scale=math.inf),
               dict(scale=math.nan), dict(q=AT + 1), dict(out=AT + 1), dict(table=AT + 2), dict(lengths=AT + 1), dict(lse=AT + 2), dict(workspace=AT + 8), dict(out=AT),
               dict(out=AT + 1022), dict(out=AT - 1022)):
        assert _attend(c, **kw) == INVALID, kw
    assert _attend(c, batch=0, q=None, out=None, table=None, lengths=None) == 0


def _plan(**kw):
    f = dict(lengths=AT, added=AT + 4096, table=AT + 8192, ld_table=4, width=4, free_pages=AT + 12288, n_free=10, taken=AT + 16384, requests=3, page_size=16, rows=8,
             slots=AT + 20480, positions=AT + 24576, starts=AT + 28672, lengths_out=AT + 32768, taken_out=AT + 36864)
    f.update(kw)
    return pb.lib().pp_paged_plan(*f.values(), None)


def test_plan_calls_that_are_refused():
    for kw in (dict(requests=-1), dict(width=0), dict(page_size=0), dict(rows=-1), dict(n_free=-1), dict(taken=None), dict(starts=None), dict(taken_out=None), dict(lengths=None),
               dict(added=None), dict(table=None), dict(lengths_out=None), dict(ld_table=3), dict(slots=None), dict(positions=None), dict(free_pages=None), dict(lengths=AT + 2),
               dict(slots=AT + 20484), dict(lengths_out=AT + 4), dict(lengths_out=AT + 4096), dict(taken_out=AT), dict(starts=AT + 24576), dict(table=AT + 12288 - 40),
               dict(positions=AT + 20480 + 60), dict(taken_out=AT + 28672 + 12)):
        assert _plan(**kw) == INVALID, kw
    for kw in (dict(requests=8193), dict(width=2 ** 27, ld_table=2 ** 27), dict(page_size=2 ** 31 - 1)):
        assert _plan(**kw) == UNSUPPORTED, kw


def _append(c, **kw):
    f = dict(q=AT, q_token=512, q_head=64, heads=4, q_out=AT + (1 << 20), o_token=256, o_head=64, k=AT + 512, k_token=512, k_head=64, v=AT + 768, v_token=512, v_head=64,
             dtype=pb.PP_BF16, tokens=3, slots=AT, positions=AT, inv_freq=AT, pairs=32, interleaved=0)
    f.update(kw)
    return pb.lib().pp_kv_append(ctypes.addressof(c), *f.values(), None)


def test_append_calls_that_are_refused():
    c = _cache()
    for kw in (dict(tokens=-1), dict(heads=-1), dict(heads=0), dict(q=None), dict(q_out=None), dict(pairs=33), dict(pairs=-1), dict(pairs=0), dict(positions=None), dict(inv_freq=None),
               dict(k=None), dict(v=None), dict(slots=None), dict(q=AT + 1), dict(k=AT + 1), dict(slots=AT + 4), dict(positions=AT + 2), dict(inv_freq=AT + 1), dict(q_token=-1),
               dict(k_head=-2), dict(v_token=1 << 60), dict(o_head=63), dict(o_token=255), dict(q_out=AT), dict(q_out=AT, o_token=512, o_head=65),
               dict(q_out=AT + 512, o_token=512)):
        assert _append(c, **kw) == INVALID, kw
    for kw in (dict(dtype=pb.PP_F32), dict(dtype=pb.PP_F16), dict(dtype=pb.PP_I8)):
        assert _append(c, **kw) == UNSUPPORTED, kw
    assert _append(_cache(**Q8), dtype=pb.PP_E4M3) == UNSUPPORTED
    assert _append(c, tokens=0, k=None, v=None, slots=None) == 0


def test_entries_refuse_host_tensors():
    with pytest.raises(ValueError, match="on device"):
        pb.pp_paged_plan(*(torch.zeros(2, dtype=torch.int32) for _ in range(2)), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
                         torch.zeros(1, dtype=torch.int32), 16, out=_Plan)
    with pytest.raises(TypeError, match="lengths must be a tensor"):
        pb.pp_paged_plan([1], None, None, None, None, 16, out=_Plan)
    with pytest.raises(ValueError, match="rows or out"):
        pb.pp_paged_plan(torch.zeros(1), None, None, None, None, 16)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        pb.PagedCache(torch.zeros(1, 2, 2, 64), torch.zeros(1, 2, 2, 64))
    with pytest.raises(ValueError, match="k must be a CUDA tensor"):
        pb.pp_kv_append(_Cache, x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        pb.pp_paged_attention(_Cache, x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    for f in (pb._fast.paged_plan, pb._fast.kv_append, pb._fast.paged_attention):
        with pytest.raises(TypeError, match="arguments"):
            f(1, 2)


class _Plan:
    slots, positions, starts, lengths, taken = (torch.zeros(2, dtype=torch.int64),) + tuple(torch.zeros(n, dtype=torch.int32) for n in (2, 3, 2, 1))


class _Cache:
    _at, head_dim, kv_heads, device = 0, 64, 2, 0
