"""The host side of the pages of an 8-bit cache, of attention over shared prefixes and of log-probabilities, without a GPU: sizes and every call's refusals, which
come before any launch."""
import ctypes as C

import pytest
import torch

import test_kv8_host as base
from paper_2411_05894_amd import binding as sv
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_ECAPACITY, SSSD_EINVAL, SSSD_OK

L, FAKE = kv8._lib(), base.FAKE
PAGES_AT = 1 << 21


def cache(**change):
    return base.cache(**{"block_table": PAGES_AT, **change})


def size_of(**change):
    n = C.c_size_t()
    assert L.sssd_kv8_pages_sizes(C.byref(base.config(**change)), C.byref(n)) == SSSD_OK
    return n.value


def pages(table=PAGES_AT, refs=FAKE, workspace=FAKE, ws_bytes=None):
    return kv8.Kv8PagesArgs(table, refs, workspace, size_of() if ws_bytes is None else ws_bytes)


def ref(s):
    return None if s is None else s if isinstance(s, bytes) else C.byref(s)


def fork(kv=None, book=None, origins=FAKE, lens=FAKE, **_):
    return L.sssd_kv8_fork(ref(kv), ref(book), origins, lens, None)


def reserve(kv=None, book=None, first=0, B=2, n=3, lens=FAKE, counts=None, **_):
    return L.sssd_kv8_reserve(ref(kv), ref(book), first, B, n, lens, counts, None)


def compact(kv=None, book=None, to=None, to_book=None, **_):
    return L.sssd_kv8_compact(ref(kv), ref(book), ref(to), ref(to_book), None, None, None)


def test_page_sizes():
    assert size_of(max_batch=3000) > size_of() and size_of(n_pages=1000) > size_of(n_pages=10) and size_of() % 256 == 0
    n = C.c_size_t()
    for bad in (dict(format=2), dict(max_seq=0), dict(head_dim=96)):
        assert L.sssd_kv8_pages_sizes(C.byref(base.config(**bad)), C.byref(n)) == SSSD_EINVAL
    assert L.sssd_kv8_pages_sizes(None, C.byref(n)) == L.sssd_kv8_pages_sizes(C.byref(base.config()), None) == SSSD_EINVAL


@pytest.mark.parametrize("call", [fork, reserve, compact])
def test_page_calls_refuse(call):
    ok = dict(kv=cache(), book=pages())
    for bad in (dict(kv=None), dict(book=None), dict(book=pages(table=None)), dict(book=pages(refs=None)), dict(book=pages(workspace=None)), dict(book=pages(workspace=FAKE + 64)),
                dict(kv=cache(block_table=None)), dict(kv=cache(block_table=PAGES_AT + 4)), dict(kv=cache(cache=None)), dict(kv=cache(cache=FAKE + 16)), dict(kv=cache(status=None)),
                dict(kv=cache(flags=1))):
        assert call(**{**ok, **bad}) == SSSD_EINVAL, bad
    many = dict(n_pages=2 ** 30 + 1)
    for bad in (dict(kv=cache(cache_bytes=1)), dict(book=pages(ws_bytes=size_of() - 1)), dict(kv=cache(**many), book=pages(ws_bytes=size_of(**many)))):
        assert call(**{**ok, **bad}) == SSSD_ECAPACITY, bad


def test_fork_and_reserve_refuse():
    ok = dict(kv=cache(), book=pages())
    assert fork(**ok, origins=None) == fork(**ok, lens=None) == SSSD_EINVAL
    many = dict(max_batch=65536, max_seq=32)
    assert fork(kv=cache(**many), book=pages(ws_bytes=size_of(**many))) == SSSD_ECAPACITY
    for bad in (dict(lens=None), dict(first=-1), dict(B=0), dict(B=-3), dict(n=0)):
        assert reserve(**ok, **bad) == SSSD_EINVAL, bad
    for bad in (dict(B=4), dict(first=2), dict(first=2 ** 31 - 1), dict(n=101)):
        assert reserve(**ok, **bad) == SSSD_ECAPACITY, bad
    far = dict(max_batch=1 << 16, max_seq=1 << 20, n_pages=100)
    assert reserve(kv=cache(**far), book=pages(ws_bytes=size_of(**far)), B=1 << 16, n=1 << 20) == SSSD_ECAPACITY


def test_compact_refuses_other_pools():
    ok = dict(kv=cache(), book=pages())
    there = lambda **c: dict(to=cache(cache=FAKE * 4, block_table=PAGES_AT + 256, **c), to_book=pages(table=PAGES_AT + 256, refs=FAKE + 256, ws_bytes=1 << 30))  # noqa: E731
    assert compact(**ok, to=cache()) == compact(**ok, to_book=pages()) == SSSD_EINVAL
    for change in (dict(format=1), dict(n_layers=1), dict(n_kv_heads=4), dict(head_dim=128), dict(max_batch=2), dict(max_seq=200)):
        assert compact(**ok, **there(**change)) == SSSD_EINVAL, change
    same = there()
    for to in (dict(to=cache(block_table=PAGES_AT + 256)), dict(to_book=pages(table=PAGES_AT + 256, ws_bytes=1 << 30))):       # the same cache, the same counts
        assert compact(**ok, **{**same, **to}) == SSSD_EINVAL
    assert compact(**ok, to=same["to"], to_book=pages(table=PAGES_AT + 512)) == SSSD_EINVAL


def shared(kv=None, layer=0, B=2, n=3, q=base.rows(), out=base.rows(), lens=FAKE, groups=1, starts=FAKE, shares=FAKE, workspace=FAKE, ws_bytes=1 << 40, **_):
    return L.sssd_kv8_attention_shared(ref(kv), layer, B, n, ref(q), ref(out), lens, None, None, groups, starts, shares, workspace, ws_bytes, None)


def test_shared_attention_refuses():
    ok = dict(kv=base.cache())
    for bad in (dict(kv=None), dict(B=0), dict(n=0), dict(lens=None), dict(groups=-1), dict(starts=None), dict(shares=None), dict(workspace=None), dict(workspace=FAKE + 16),
                dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(out=base.rows(type=1)), dict(q=base.rows(data=FAKE + 2)), dict(kv=base.cache(cache=None)),
                dict(kv=base.cache(status=None)), dict(kv=base.cache(n_pages=11))):
        assert shared(**{**ok, **bad}) == SSSD_EINVAL, bad
    for bad in (dict(B=4), dict(n=33), dict(groups=3), dict(ws_bytes=1000), dict(kv=base.cache(cache_bytes=5))):
        assert shared(**{**ok, **bad}) == SSSD_ECAPACITY, bad
    n = C.c_size_t()
    sizes = lambda B, n_, **c: L.sssd_kv8_shared_sizes(C.byref(base.config(**c)), B, n_, C.byref(n))  # noqa: E731
    assert sizes(1, 1) == SSSD_OK
    small = n.value
    assert sizes(3, 32) == SSSD_OK and n.value > small
    assert sizes(0, 1) == sizes(1, 0) == sizes(1, 1, head_dim=7) == SSSD_EINVAL
    assert sizes(4, 1) == sizes(1, 33) == sizes(1 << 20, 32, max_batch=1 << 20, max_seq=64) == SSSD_ECAPACITY
    assert L.sssd_kv8_shared_sizes(C.byref(base.config()), 1, 1, None) == SSSD_EINVAL


def logprobs(logits=FAKE, type=0, rows=2, vocab=100, stride=100, temperature=1.0, tokens=FAKE, m=1, lp=FAKE, ranks=None, entropy=None, top=2, ids=FAKE, top_lp=FAKE,
             scratch=FAKE, scratch_bytes=1 << 40):
    return sv.lib().sssd_op_logprobs(logits, type, rows, vocab, stride, temperature, tokens, m, lp, ranks, entropy, top, ids, top_lp, scratch, scratch_bytes, None)


def test_logprobs_refuse():
    for bad in (dict(logits=None), dict(type=2), dict(rows=0), dict(vocab=0), dict(stride=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(temperature=1e-39), dict(temperature=2e36), dict(temperature=9e-39), dict(tokens=None), dict(lp=None), dict(m=-1), dict(top=-1), dict(top=101), dict(ids=None), dict(top_lp=None),
                dict(vocab=5000, scratch=None), dict(vocab=5000, scratch=FAKE + 8), dict(logits=FAKE + 2), dict(logits=FAKE + 1, type=1)):
        assert logprobs(**bad) == SSSD_EINVAL, bad
    for bad in (dict(m=33), dict(top=65), dict(vocab=5000, scratch_bytes=16), dict(vocab=2 ** 30 + 1), dict(rows=2 ** 31 - 1, vocab=128256, stride=128256)):
        assert logprobs(**bad) == SSSD_ECAPACITY, bad
    size = sv.lib().sssd_op_logprobs_scratch_bytes
    assert 0 < size(0, 1, 9000, 0, 0) < size(0, 100, 9000, 1, 0) < size(0, 100, 9000, 1, 50)
    assert size(2, 1, 1, 0, 0) == size(0, 0, 1, 0, 0) == size(0, 1, 0, 0, 0) == size(0, 1, 9, 33, 0) == size(0, 1, 99, 0, 65) == size(0, 1, 9, 0, 10) == 0


def test_the_binding_checks_tensors():
    z = torch.zeros(2, 9)
    with pytest.raises(AssertionError):
        sv.sssd_op_logprobs(z)                       # not on a GPU
    with pytest.raises(AssertionError):
        sv.sssd_op_logprobs(z.half())
