"""The host side of include/sssd_kv8.h without a GPU: sizes, frequencies, and every call's refusals, which come before any launch."""
import ctypes as C
import math

import pytest
import torch

from kv8_reference import frequencies
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_ECAPACITY, SSSD_EINVAL, SSSD_OK, SssdError

L = kv8._lib()
FAKE = 1 << 20      # never read: the calls that get it are refused


def config(**change):
    c = dict(format=0, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_batch=3, max_seq=100, n_pages=0)
    c.update(change)
    return kv8.Kv8Config(*c.values())


def cache(**change):
    cfg = config(**{k: v for k, v in change.items() if k in [f[0] for f in kv8.Kv8Config._fields_]})
    size, ws, _, _ = kv8.sssd_kv8_sizes(cfg)
    a = dict(cfg=cfg, cache=FAKE, cache_bytes=size, workspace=FAKE, ws_bytes=ws, block_table=None, status=FAKE, flags=0)
    a.update({k: v for k, v in change.items() if k in a})
    return kv8.Kv8(*a.values())


def rows(data=FAKE, type=0, b=6400, r=640, h=64):
    return kv8.ROWS(data or 0, type, b, r, h)


def rope(turns=FAKE, rotary=64, pairs=0):
    return kv8.RopeArgs(turns, rotary, pairs, 1.0)


def test_sizes():
    size, ws, per_seq, pages = kv8.sssd_kv8_sizes(config())
    assert per_seq == 4 and pages == 12
    assert size == 2 * ((12 * 2 * (64 * 64 + 8) + 255) // 256 * 256) and ws > 0     # two layers of whole 256 bytes
    assert kv8.sssd_kv8_sizes(config(n_pages=5))[3] == 5
    assert kv8.sssd_kv8_sizes(config(format=1, head_dim=128, max_seq=1, max_batch=1))[2] == 1
    for bad in (dict(format=2), dict(format=-1), dict(n_layers=0), dict(n_kv_heads=3), dict(n_q_heads=0), dict(head_dim=96), dict(max_batch=0), dict(max_seq=0),
                dict(max_seq=2**31 - 1), dict(n_pages=-1), dict(n_q_heads=130), dict(max_batch=2**30, max_seq=2**20),
                dict(n_pages=2**31 - 1, n_kv_heads=2**30, n_q_heads=2**30, n_layers=2**30)):
        assert L.sssd_kv8_sizes(C.byref(config(**bad)), None, None, None, None) == SSSD_EINVAL, bad
    assert L.sssd_kv8_sizes(None, None, None, None, None) == SSSD_EINVAL
    assert L.sssd_kv8_sizes(C.byref(config()), None, None, None, None) == SSSD_OK


@pytest.mark.parametrize("rotary", [2, 6, 64, 128, 1024])
@pytest.mark.parametrize("scaling", [{}, dict(scaling="linear", factor=4.0), dict(scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192),
                                     dict(scaling="bands", factor=32.0, low=0.0, high=32.0, original=4096)])
def test_frequencies(rotary, scaling):
    for base in (10000.0, 500000.0):
        got = kv8.sssd_rope_frequencies(rotary, base, **scaling)
        want = frequencies(rotary, base, **scaling) / (2 * math.pi)
        assert ((got - want).abs() <= 8 * 2.0 ** -53 * want + 1e-300).all()     # a power, two products and a quotient, in 64 bits


def test_frequencies_refuse():
    turns = (C.c_double * 600)()
    call = lambda *a: L.sssd_rope_frequencies(C.byref(kv8.RopeConfig(*a)), turns)  # noqa: E731
    assert call(64, 10000.0, 0, 0.0, 0.0, 0.0, 0) == SSSD_OK
    for bad in ((0, 1e4, 0, 1, 1, 4, 1), (63, 1e4, 0, 1, 1, 4, 1), (1026, 1e4, 0, 1, 1, 4, 1), (64, 1.0, 0, 1, 1, 4, 1), (64, float("nan"), 0, 1, 1, 4, 1),
                (64, 1e4, 3, 1, 1, 4, 1), (64, 1e4, 1, 0.0, 1, 4, 1), (64, 1e4, 2, 8, 4, 4, 1), (64, 1e4, 2, 8, -1, 4, 1), (64, 1e4, 2, 8, 1, 4, 0)):
        assert call(*bad) == SSSD_EINVAL, bad
    assert L.sssd_rope_frequencies(None, turns) == L.sssd_rope_frequencies(C.byref(kv8.RopeConfig(64, 1e4, 0, 1, 1, 4, 1)), None) == SSSD_EINVAL
    with pytest.raises(SssdError):
        kv8.sssd_rope_frequencies(64, 0.5)


def test_rope_refuses():
    ok = dict(x=rows(), out=rows(), B=1, n=1, heads=2, d=64, positions=FAKE, rope=rope())
    def call(**change):
        a = {**ok, **change}
        ref = lambda s: s if s is None or isinstance(s, bytes) else C.byref(s)  # noqa: E731
        return L.sssd_op_rope(ref(a["x"]), ref(a["out"]), a["B"], a["n"], a["heads"], a["d"], a["positions"], ref(a["rope"]), None)
    for bad in (dict(x=None), dict(out=None), dict(x=rows(data=None)), dict(out=rows(type=1)), dict(x=rows(type=2)), dict(x=rows(data=FAKE + 2)), dict(B=0), dict(n=0),
                dict(heads=0), dict(heads=65536), dict(d=0), dict(d=8193), dict(d=2048, rope=rope(rotary=1026)), dict(positions=None), dict(rope=None), dict(rope=rope(turns=None)), dict(rope=rope(rotary=66)),
                dict(rope=rope(rotary=3)), dict(rope=rope(rotary=0)), dict(rope=rope(pairs=2)), dict(n=2, out=rows(r=1280))):
        assert call(**bad) == SSSD_EINVAL, bad
    assert call(B=1 << 20, n=1 << 10, out=rows()) == SSSD_ECAPACITY


def calls():
    ref = lambda s: s if s is None or isinstance(s, bytes) else C.byref(s)  # noqa: E731
    def append(kv=None, layer=0, first=0, B=2, n=3, k=None, v=None, lens=FAKE, rope=None, parents=None, q=None, q_out=None, **_):
        return L.sssd_kv8_append(ref(kv), layer, first, B, n, ref(k), ref(v), lens, None, ref(rope), parents, ref(q), ref(q_out), None)
    def read(kv=None, layer=0, first=0, B=2, n=3, k=None, v=None, **_):
        return L.sssd_kv8_read(ref(kv), layer, first, B, n, None, None, ref(k), ref(v), None)
    def attention(kv=None, layer=0, B=2, n=3, q=None, out=None, lens=FAKE, window=0, sinks=0, **_):
        return L.sssd_kv8_attention(ref(kv), layer, B, n, ref(q), ref(out), lens, None, None, window, sinks, None)
    def commit(kv=None, B=2, n=3, lens=FAKE, accepted=FAKE, **_):
        return L.sssd_kv8_commit_tree(ref(kv), B, n, lens, accepted, None, None)
    return append, read, attention, commit


BASE = dict(k=rows(), v=rows(), q=None, out=rows())


def refused(call, code, **change):
    a = {**BASE, "kv": cache(), **change}
    if call.__name__ == "attention":
        a["q"] = change.get("q", rows())
    assert call(**a) == code, (call.__name__, change)


def test_cache_calls_refuse():
    append, read, attention, commit = calls()
    for call in (append, read, attention, commit):
        for bad in (dict(kv=None), dict(B=0), dict(B=-1), dict(n=0), dict(kv=cache(cache=None)), dict(kv=cache(cache=FAKE + 16)), dict(kv=cache(status=None)), dict(kv=cache(flags=1)),
                    dict(kv=cache(n_pages=11))):       # too few pages without a table
            refused(call, SSSD_EINVAL, **bad)
        for bad in (dict(B=4), dict(n=101), dict(kv=cache(cache_bytes=1))):
            refused(call, SSSD_ECAPACITY, **bad)
        if call is not commit:
            for layer in (-1, 2):
                refused(call, SSSD_EINVAL, layer=layer)
        if call in (append, attention, commit):
            refused(call, SSSD_EINVAL, lens=None)
    for call in (append, read):
        for bad in (dict(first=-1), dict(k=None), dict(v=None), dict(v=rows(type=1)), dict(k=rows(type=5)), dict(k=rows(data=FAKE + 1))):
            refused(call, SSSD_EINVAL, **bad)
        refused(call, SSSD_ECAPACITY, first=2)
    for bad in (dict(n=33, parents=FAKE), dict(q=rows()), dict(q_out=rows(), rope=rope()), dict(q=rows(), q_out=rows()), dict(rope=rope(rotary=66)),
                dict(q=rows(), q_out=rows(type=1), rope=rope()), dict(q=rows(), q_out=rows(r=1280), rope=rope()), dict(rope=rope(turns=None))):
        refused(append, SSSD_EINVAL, **bad)
    for bad in (dict(window=-1), dict(sinks=-1), dict(q=rows(type=1)), dict(q=None), dict(out=rows(data=None)), dict(kv=cache(workspace=None)),
                dict(kv=cache(workspace=FAKE + 64))):
        refused(attention, SSSD_EINVAL, **bad)
    refused(attention, SSSD_ECAPACITY, n=33)
    refused(attention, SSSD_ECAPACITY, kv=cache(ws_bytes=1))
    refused(commit, SSSD_ECAPACITY, n=33)
    refused(commit, SSSD_EINVAL, accepted=None)
    assert L.sssd_kv8_sync(None, None) == SSSD_EINVAL and L.sssd_kv8_sync(C.byref(cache(status=None)), None) == SSSD_EINVAL


def test_calls_past_what_a_launch_holds_are_refused():
    append, read, attention, commit = calls()
    big = lambda **c: cache(max_batch=1 << 20, max_seq=1 << 9, n_kv_heads=8, n_q_heads=64, block_table=FAKE, n_pages=1, **c)  # noqa: E731
    for call in (append, read):
        refused(call, SSSD_ECAPACITY, kv=big(), B=1 << 20, n=512)
    refused(attention, SSSD_ECAPACITY, kv=big(), B=1 << 20, n=1)
    refused(commit, SSSD_ECAPACITY, kv=big(n_layers=8), B=1 << 20, n=1)


def test_the_binding_checks_tensors():
    x = torch.zeros(2, 3, 2, 64)
    with pytest.raises(AssertionError):
        kv8._rows(x, 0)                  # another device
    with pytest.raises(AssertionError):
        kv8._rows(x.half(), -1)
    with pytest.raises(AssertionError):
        kv8._rows(x[0, 0], -1)
    with pytest.raises(AssertionError):
        kv8._rows(x.transpose(2, 3), -1)     # channels not in a row
    with pytest.raises(AssertionError):
        kv8._ints(torch.zeros(2, dtype=torch.int64), (2,), -1)
    with pytest.raises(AssertionError):
        kv8._ints(torch.zeros(3, dtype=torch.int32), (2,), -1)
    assert kv8._rows(x[:, :, 1:], -1) == kv8.ROWS(x.data_ptr() + 256, 0, 384, 128, 64) and len(kv8.ROWS(0, 0, 0, 0, 0)) == 40   # sssd_rows


def test_queries_come_with_a_place_for_them():
    c = kv8.Kv8Cache.__new__(kv8.Kv8Cache)      # without device buffers: the check comes first
    c.n_q_heads, c.n_kv_heads, c.head_dim, c.device = 2, 2, 64, -1
    x, lens = torch.zeros(1, 3, 2, 64), torch.zeros(1, dtype=torch.int32)
    for more in (dict(q=x), dict(q_out=x)):
        with pytest.raises(AssertionError, match="together"):
            c.sssd_kv8_append(0, x, x, lens, **more)
