"""Arrays of a paged cache's calls that lie on one another are refused, and those between rows are not.  Addresses are made up on the CPU,
where only calls that are refused, or that have no requests, are made; what is accepted runs on the GPU with real tensors."""
import ctypes
import itertools
import random

import pytest

torch = pytest.importorskip("torch")
from paper_1712_01084_b200 import binding as pb
from test_paged_entry import AT, INVALID, _append, _attend, _cache, _space

Q8 = dict(dtype=pb.PP_I8, k_scales=AT + (2 << 30), v_scales=AT + (3 << 30))


def _bytes(at, strides, counts, dim, size):
    out = set()
    for place in itertools.product(*(range(n) for n in counts)):
        first = at + sum(s * i for s, i in zip(strides, place)) * size
        out.update(range(first, first + dim * size))
    return out


def _apart(strides, counts, dim):
    span = dim
    for s, n in sorted(zip(strides, counts)):
        if n > 1:
            if s < span:
                return False
            span += s * (n - 1)
    return True


def test_keys_on_values():
    """Every distance of small caches of one layout, token by token, head by head, with gaps: against sets of bytes."""
    rng = random.Random(1)
    met = {True: 0, False: 0}
    for _ in range(60):
        counts, dim = [rng.randint(1, 3) for _ in range(3)], rng.randint(1, 4)
        strides, span = [0, 0, 0], dim
        for axis in rng.sample(range(3), 3):                 # from the innermost axis out, any order
            strides[axis] = span + rng.choice((0, 0, 1, 5, 9))
            span = strides[axis] * (counts[axis] - 1) + span if counts[axis] > 1 else span
        assert _apart(strides, counts, dim)
        keys = _bytes(AT, strides, counts, dim, 1)
        for d in range(-span - 2, span + 3):
            meet = bool(keys & _bytes(AT + d, strides, counts, dim, 1))
            c = _cache(**dict(Q8, v=AT + d, k_page=strides[0], k_token=strides[1], k_head=strides[2], v_page=strides[0], v_token=strides[1], v_head=strides[2], pages=counts[0],
                              page_size=counts[1], kv_heads=counts[2], head_dim=dim))
            assert (_space(c, pb.PP_F16, heads=counts[2])[0] == INVALID) == meet, (counts, strides, dim, d)
            met[meet] += 1
    assert min(met.values()) > 500


def test_interleaved_caches():
    """Keys and values of a page side by side, of a token, of a head: fine; a row too near: not."""
    f = dict(k_page=2 * 16 * 128, k_token=128, k_head=64, v_page=2 * 16 * 128, v_token=128, v_head=64)
    assert _space(_cache(v=AT + 16 * 128 * 2, **f))[0] == 0
    assert _space(_cache(v=AT + 16 * 128 * 2 - 2, **f))[0] == INVALID
    f = dict(k_page=16 * 256, k_token=256, k_head=64, v_page=16 * 256, v_token=256, v_head=64)
    assert _space(_cache(v=AT + 256, **f))[0] == 0 and _space(_cache(v=AT + 254, **f))[0] == INVALID
    f = dict(k_page=16 * 256, k_token=256, k_head=128, v_page=16 * 256, v_token=256, v_head=128)
    assert _space(_cache(v=AT + 128, **f))[0] == 0 and _space(_cache(v=AT + 130, **f))[0] == INVALID


def test_scales_on_rows_and_on_one_another():
    size, scales = 10 * 16 * 2 * 64, 10 * 16 * 2 * 4
    for k_scales, v_scales, want in ((AT - scales, AT + size, 0), (AT - scales + 4, AT + size, INVALID), (AT + size - 4, AT + (1 << 29), INVALID), (AT + (1 << 29), AT + 64, INVALID),
                                     (AT + (1 << 29), AT + (1 << 29) + scales, 0), (AT + (1 << 29), AT + (1 << 29) + scales - 4, INVALID),
                                     (AT + (1 << 30) + 128, AT + (1 << 29), INVALID)):
        assert _space(_cache(**dict(Q8, k_scales=k_scales, v_scales=v_scales)), pb.PP_F32)[0] == want
    # in the gap behind each page
    gap = dict(k_page=2 * 16 * 128, v_page=2 * 16 * 128, pages=2)
    assert _space(_cache(**dict(Q8, k_scales=AT + 16 * 128, **gap)), pb.PP_F32)[0] == 0
    assert _space(_cache(**dict(Q8, k_scales=AT + 16 * 128 - 4, **gap)), pb.PP_F32)[0] == INVALID


FAR = dict(q=AT + (8 << 30), table=AT + (9 << 30), lengths=AT + (10 << 30), out=AT + (11 << 30), lse=AT + (12 << 30), workspace=AT + (13 << 30), workspace_bytes=1 << 20)
CACHE, OUT, LSE = 10 * 16 * 2 * 64 * 2, 2 * 4 * 64 * 2, 2 * 4 * 4


@pytest.mark.parametrize("change", [
    dict(out=AT), dict(out=AT + CACHE - 2), dict(out=AT - OUT + 2), dict(out=AT + (1 << 30) + 64), dict(lse=AT + 256), dict(lse=AT + (1 << 30) + CACHE - 4), dict(workspace=AT + 4096),
    dict(workspace=AT - (1 << 20) + 16), dict(out=FAR["table"]), dict(out=FAR["table"] + 36), dict(out=FAR["lengths"] + 4), dict(lse=FAR["table"] - LSE + 4), dict(lse=FAR["lengths"]),
    dict(workspace=FAR["table"] - 16), dict(workspace=FAR["lengths"] - 256), dict(lse=FAR["q"] + 256), dict(workspace=FAR["q"] - 16), dict(lse=FAR["out"] + OUT - 4),
    dict(out=FAR["lse"] + LSE - 2), dict(workspace=FAR["out"] - 4096), dict(workspace=FAR["lse"] - (1 << 20) + 16)])
def test_attention_that_writes_on_what_it_reads(change):
    assert _attend(_cache(), **dict(FAR, **change)) == INVALID


def test_attention_that_writes_on_scales():
    for at in (Q8["k_scales"], Q8["v_scales"] + 10 * 16 * 2 * 4 - 4):
        for name in ("out", "lse", "workspace"):
            assert _attend(_cache(**Q8), **dict(FAR, q_type=pb.PP_F32, **{name: at // 16 * 16})) == INVALID


APART = dict(q=AT + (8 << 30), q_out=AT + (9 << 30), k=AT + (10 << 30), v=AT + (11 << 30), slots=AT + (12 << 30), positions=AT + (13 << 30), inv_freq=AT + (14 << 30))


@pytest.mark.parametrize("change", [
    dict(q_out=AT), dict(q_out=AT + CACHE - 2), dict(q_out=AT + (1 << 30)), dict(slots=AT + 16), dict(slots=AT - 16), dict(positions=AT + (1 << 30)), dict(inv_freq=AT + CACHE - 4),
    dict(slots=APART["q_out"]), dict(slots=APART["q_out"] - 16), dict(positions=APART["q_out"] + 3 * 256 * 2 - 4), dict(inv_freq=APART["q_out"] + 512), dict(q_out=APART["inv_freq"] + 124),
    dict(q=AT + 512, q_out=AT + 512, o_token=512)])
def test_append_that_writes_on_what_it_reads(change):
    assert _append(_cache(), **dict(APART, **change)) == INVALID


def test_append_that_writes_on_scales():
    for change in (dict(q_out=Q8["k_scales"]), dict(slots=Q8["v_scales"] + 8), dict(positions=Q8["k_scales"] + 4), dict(inv_freq=Q8["v_scales"] + 64)):
        assert _append(_cache(**Q8), **dict(APART, **change)) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_between_rows(dtype):
    """out, slots and the turned q in the gap behind a page's rows, k and v from rows of the cache that are not written: as elsewhere."""
    pages, page, g, d, gap = 6, 4, 2, 64, 2048
    store = torch.randn(pages, 2 * page * g * d + gap, device="cuda").to(dtype)
    half = page * g * d
    k, v = (store[:, i * half:(i + 1) * half].view(pages, page, g, d) for i in range(2))
    c = pb.PagedCache(k, v)
    q = torch.randn(2, 4, d, device="cuda").to(dtype)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([7, 5], dtype=torch.int32, device="cuda")
    want = pb.pp_paged_attention(c, q, table, lengths)
    out = store[1, 2 * half:2 * half + 2 * 4 * d].view(2, 4, d)
    assert pb.pp_paged_attention(c, q, table, lengths, out=out) is out and torch.equal(out, want)
    # the last rows of page 4 copied to page 5, turned by nothing
    slots = torch.tensor([5 * page, 5 * page + 1], device="cuda")
    turned = store[2, 2 * half:2 * half + 2 * 4 * d].view(2, 4, d)
    pb.pp_kv_append(c, k[4, 2:], v[4, 2:], slots, q=q, out=turned)
    assert torch.equal(turned, q) and torch.equal(k[5, :2], k[4, 2:]) and torch.equal(v[5, :2], v[4, 2:])
    for bad in (store[1, 2 * half - 1:2 * half - 1 + 2 * 4 * d], store[3, :2 * 4 * d], store.view(-1)[half - 2 * 4 * d + 1:half + 1]):
        if bad.data_ptr() % 4 and dtype == torch.float32:
            continue
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            pb.pp_paged_attention(c, q, table, lengths, out=bad.view(2, 4, d))
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            pb.pp_kv_append(c, k[4, 2:], v[4, 2:], slots, q=q, out=bad.view(2, 4, d))
    for other in (table.view(-1), lengths):
        o = other.view(torch.float32) if dtype == torch.float32 else other.view(dtype)
        small = pb.PagedCache(k[..., :1], v[..., :1])
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            pb.pp_paged_attention(small, q[:1, :2, :1], table[:1], lengths[:1], out=o[:2].view(1, 2, 1))
