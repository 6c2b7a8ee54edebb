"""The paged cache's entry points refuse what they cannot take before any launch, and the call module what is no such tensor: no GPU
needed."""
import ctypes as C

import pytest
import torch

from paper_2605_13915_b200 import binding
from paged_reference import evicted

OK, NULL, SHAPE, ALIGN, UNSUPPORTED, ROOM, CUDA = 0, 1, 2, 3, 4, 5, 6
P = 4096                                    # an address that is never read: every call below fails in the host's checks


def _cache(int8=False, **changes):
    D, Hkv, page = 64, 2, 16
    c = binding.PagedCache(P, P, P if int8 else None, P if int8 else None, 1 if int8 else 0, 8, page, Hkv, D, D)
    c.k_stride[:] = c.v_stride[:] = [page * Hkv * D, Hkv * D, D]
    c.k_scale_stride[:] = c.v_scale_stride[:] = [page * Hkv, Hkv, 1]
    for name, value in changes.items():
        if isinstance(value, dict):
            for i, v in value.items():
                getattr(c, name)[i] = v
        else:
            setattr(c, name, value)
    return c


def _append(c, k_new=P, v_new=P, n=4, k_ld=128, v_ld=128, table=P, max_blocks=4, seqlens=P, cu=P, B=2, weights=None, ld=0):
    return binding.lib().msd_kv_append_paged(k_new, v_new, n, k_ld, v_ld, C.byref(c) if c else None, table, max_blocks, seqlens, cu, B, weights, ld, None)


def _attend(c, q=P, q_ld=256, table=P, max_blocks=4, seqlens=P, B=2, Hq=4, out=P, lse=None, weights=None, ld=0, ws=P, room=1 << 40):
    return binding.lib().msd_attn_decode_paged(q, q_ld, C.byref(c) if c else None, table, max_blocks, seqlens, B, Hq, 0.1, out, lse, weights, ld, ws,
                                               room, None)


def _evict(c, table=P, max_blocks=4, seqlens=P, weights=P, ld=64, B=2, budget=32, recent=4, sinks=2, dst=2 * P, dst_blocks=2, new_seqlens=3 * P,
           new_weights=4 * P, new_ld=32, kept=P):
    return binding.lib().msd_kv_evict_paged(C.byref(c) if c else None, table, max_blocks, seqlens, weights, ld, B, budget, recent, sinks, dst,
                                            dst_blocks, new_seqlens, new_weights, new_ld, kept, None)


@pytest.mark.parametrize("call", [_append, _attend, _evict])
def test_caches_that_are_refused(call):
    assert call(None) == NULL
    assert call(_cache(k=None)) == NULL
    assert call(_cache(True, k_scale=None)) == NULL
    assert call(_cache(True, v_scale=None)) == NULL
    assert call(_cache(type=2)) == UNSUPPORTED
    assert call(_cache(D=264)) == UNSUPPORTED
    assert call(_cache(Dv=512)) == UNSUPPORTED
    for name, value in (("num_blocks", 0), ("num_blocks", 1 << 31), ("page_size", 0), ("page_size", 65537), ("Hkv", 0), ("D", 0), ("D", 60), ("Dv", -8)):
        assert call(_cache(**{name: value})) == SHAPE, name
    assert call(_cache(True, D=72)) == SHAPE                                   # INT8: rows of whole 16 bytes
    assert call(_cache(v=P + 8)) == ALIGN
    assert call(_cache(True, k_scale=P + 2)) == ALIGN
    assert call(_cache(k_stride={1: 68})) == ALIGN
    assert call(_cache(True, v_stride={2: 72})) == ALIGN
    assert call(_cache(v_stride={0: -2048})) == SHAPE
    assert call(_cache(True, k_scale_stride={2: -1})) == SHAPE


def test_append_refuses():
    c = _cache()
    assert _append(c, B=0) == OK and _append(c, n=0) == OK                      # nothing to do
    for name in ("k_new", "v_new", "table", "seqlens", "cu"):
        assert _append(c, **{name: None}) == NULL, name
    for changes in ({"B": -1}, {"n": -1}, {"max_blocks": 0}, {"k_ld": 120}, {"v_ld": 0}, {"weights": P, "ld": 0}):
        assert _append(c, **changes) == SHAPE, changes
    for changes in ({"k_new": P + 2}, {"v_new": P + 8}, {"k_ld": 129}, {"table": P + 1}, {"weights": P + 2, "ld": 9}):
        assert _append(c, **changes) == ALIGN, changes


def test_attention_refuses():
    c = _cache()
    assert _attend(c, B=0) == OK
    for name in ("q", "table", "seqlens", "out", "ws"):
        assert _attend(c, **{name: None}) == NULL, name
    for changes in ({"Hq": 3}, {"Hq": 0}, {"B": -1}, {"max_blocks": 0}, {"q_ld": 255}, {"weights": P, "ld": 0}, {"weights": P, "ld": 1 << 31}):
        assert _attend(c, **changes) == SHAPE, changes
    for changes in ({"q": P + 2}, {"q_ld": 260}, {"out": P + 8}, {"ws": P + 512}, {"lse": P + 2}, {"weights": P + 1, "ld": 8}):
        assert _attend(c, **changes) == ALIGN, changes
    assert _attend(c, room=1024) == ROOM
    assert _attend(_cache(num_blocks=1 << 30, k_stride={0: 2048}), room=1 << 60) == UNSUPPORTED       # rows more than 64 GiB apart
    need = binding.attn_decode_paged_workspace_bytes
    assert need(2, 4, 2, 64) <= need(2, 4, 2, 64, 100) <= need(2, 4, 2, 64, 5000) <= need(64, 4, 2, 64, 5000)
    assert need(64, 32, 8, 128, 8192) >= 64 * 32 * 8192 * 4                       # a score for each head and position
    assert need(2, 5, 2, 64) == 0 and need(2, 4, 2, 512) == 0
    # sizes that would not fit a launch or an address are refused, not wrapped
    assert need(1 << 20, 8192, 32, 64) == 0 and need(1 << 20, 8192, 1, 64, (1 << 31) - 1) == 0 and need(1 << 20, 8192, 1, 64, 1 << 31) == 0
    assert _attend(c, B=1 << 21) == UNSUPPORTED and _attend(c, B=1 << 20, Hq=8192, q_ld=8192 * 64, weights=P, ld=(1 << 31) - 1) == UNSUPPORTED
    assert _attend(c, B=1 << 16, max_blocks=1 << 27, room=1 << 40) == UNSUPPORTED and _attend(c, B=1 << 16, max_blocks=1 << 27, room=0) == ROOM


def test_eviction_refuses():
    c = _cache()
    assert _evict(c, B=0) == OK
    for name in ("table", "seqlens", "weights", "dst", "new_seqlens", "new_weights", "kept"):
        assert _evict(c, **{name: None}) == NULL, name
    for changes in ({"budget": 0}, {"recent": 31, "sinks": 2}, {"recent": -1}, {"sinks": -1}, {"new_ld": 31}, {"ld": 0}, {"B": -1}, {"max_blocks": 0},
                    {"dst_blocks": 0}):
        assert _evict(c, **changes) == SHAPE, changes
    # the kept tokens go to pages, weights and lengths of their own
    for changes in ({"dst": P}, {"new_weights": P}, {"new_seqlens": P}):
        assert _evict(c, **changes) == UNSUPPORTED, changes
    assert _evict(c, weights=P + 2) == ALIGN and _evict(c, kept=P + 2) == ALIGN


def test_results_over_inputs_are_refused():
    """Each range that a call writes against each that it reads, from the first common byte to the last."""
    c = _cache()
    row, out = 4 * 64 * 2, 2 * 4 * 64 * 2                                       # bytes of a query row and of the results of two sequences
    far = 1 << 20
    for at in (P, P + 16, P + row - 16, P - out + 16, P + far, P + far + row - 16, P + far - out + 16, P + far - row):
        assert _attend(c, q=P, q_ld=far // 2, out=at, ws=far * far) == UNSUPPORTED, at
    base = dict(table=1 << 20, seqlens=2 << 20, weights=3 << 20, dst=4 << 20, new_seqlens=5 << 20, new_weights=6 << 20, kept=7 << 20)
    size = dict(table=2 * 4 * 4, seqlens=8, weights=2 * 2 * 64 * 4, dst=2 * 2 * 4, new_seqlens=8, new_weights=2 * 2 * 32 * 4, kept=2 * 2 * 32 * 4)
    written = ("new_seqlens", "new_weights", "kept")
    for w in written:
        for r in size:
            if r == w:
                continue
            for at in (base[r], base[r] + size[r] - 4, base[r] - size[w] + 4):
                assert _evict(c, **dict(base, **{w: at})) == UNSUPPORTED, (w, r, at)


def test_call_module_takes_cuda_tensors_only():
    calls = binding._calls()
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    k, table, n = t(4, 16, 2, 64), t(2, 4, dtype=torch.int32), t(2, dtype=torch.int32)
    w, ws = t(2, 2, 64, dtype=torch.float32), t(4096, dtype=torch.uint8)
    for name, args in (("kv_append_paged", (k[0], k[0], k, k, None, None, table, n, t(3, dtype=torch.int32), None)),
                       ("attn_decode_paged", (t(2, 4, 64), k, k, None, None, table, n, 0.1, None, ws, t(2, 4, 64), None)),
                       ("kv_evict_paged", (k, k, None, None, table, n, w, 8, 1, 1, table, n, w, t(2, 2, 8, dtype=torch.int32)))):
        with pytest.raises(ValueError, match="CUDA tensors"):
            getattr(calls, name)(*args)
        with pytest.raises(TypeError):
            getattr(calls, name)("no tensor", *args[1:])
        with pytest.raises(TypeError):
            getattr(calls, name)()


def test_division_by_the_page_size():
    """The device divides positions by the page size with a multiplication: for every kind of page, at the quotients' borders."""
    for d in (1, 2, 3, 5, 7, 8, 16, 20, 48, 64, 100, 127, 128, 255, 4097, 65535, 65536):
        s = 0
        while 1 << s < d:
            s += 1
        mul = ((1 << 32) * ((1 << s) - d)) // d + 1
        assert mul < 1 << 32
        top = 0x7FFFF000 // d
        for q in (0, 1, 2, 3, 1000, 65537, top // 2, top - 1, top):
            for n in (q * d - 1, q * d, q * d + 1, q * d + d - 1):
                if 0 <= n < 1 << 31:
                    high = (n * mul) >> 32
                    assert high + n < 1 << 32 and (high + n) >> s == n // d, (n, d)


def test_the_reference_keeps_what_the_definition_says():
    nan, inf = float("nan"), float("inf")
    assert evicted([1.0, 2.0, 3.0], 3, 3, 0, 0) == [0, 1, 2]
    assert evicted([5.0, 1.0, 1.0, 1.0, 0.0], 5, 3, 1, 0) == [0, 1, 4]          # a tie: the lower ones
    assert evicted([0.0, 9.0, nan, inf, -inf, 2.0], 6, 3, 0, 1) == [0, 2, 3]    # NaN above infinity
    assert evicted([-0.0, 0.0, 0.0], 3, 2, 0, 0) == [0, 1]
