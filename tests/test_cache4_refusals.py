"""What the calls on a 4-bit cache refuse, without a launch: by the C library's own checks, through fake addresses on the host."""
import ctypes as C

import pytest
import torch

import paper_2602_01345_b200.binding as nv

FAKE = 1 << 20                         # an address that is never dereferenced: every call here is refused before any launch


@pytest.fixture()
def ctx():
    """A context's checks come before its device: a zeroed block stands in for it, large enough for its error text."""
    if torch.cuda.is_available():
        h = nv.Context(0)
        yield h.handle
    else:
        yield C.cast(C.create_string_buffer(4096), C.c_void_p)


def _cache(**kw):
    f = dict(k_codes=FAKE, v_codes=2 * FAKE, k_scales=3 * FAKE, v_scales=4 * FAKE, kv_len=5 * FAKE, B=2, Lmax=64, C=128, n_heads=2)
    f.update(kw)
    return nv._Cache4(*[f[n] for n, _ in nv._Cache4._fields_])


OTHER = dict(k_codes=11 * FAKE, v_codes=12 * FAKE, k_scales=13 * FAKE, v_scales=14 * FAKE, kv_len=15 * FAKE)

BAD_CACHES = [
    (dict(B=-1), 1), (dict(Lmax=-1), 1), (dict(C=96), 2), (dict(C=0), 2), (dict(n_heads=0), 2), (dict(n_heads=3), 2), (dict(n_heads=4), 2),
    (dict(C=512, n_heads=2), 2), (dict(k_codes=None), 1), (dict(v_scales=None), 1), (dict(v_codes=FAKE + 4), 3), (dict(k_scales=FAKE + 8), 3),
    (dict(kv_len=None), 1), (dict(kv_len=FAKE + 2), 1),
]


def _calls(ctx, cache):
    c = C.byref(cache)
    w = 20 * FAKE
    other = nv._Cache4(*[dict(OTHER, B=cache.B, Lmax=64, C=cache.C, n_heads=cache.n_heads)[n] for n, _ in nv._Cache4._fields_])
    return [nv._lib.nova_cache4_append(ctx, c, FAKE, FAKE, 1024, FAKE, 4, 1, None),
            nv._lib.nova_cache4_read(ctx, c, None, FAKE, 4, FAKE, FAKE, 1024, None),
            nv._lib.nova_cache4_attention(ctx, c, FAKE, 1024, FAKE, 4, FAKE, None, None),
            nv._lib.nova_cache4_weights(ctx, c, FAKE, 1024, FAKE, FAKE, 4, None, FAKE, None),
            nv._lib.nova_cache4_evict(ctx, c, w, 8, 2, C.byref(other), None, 21 * FAKE, None)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches(ctx, change, status):
    assert _calls(ctx, _cache(**change)) == [status] * 5


def test_null_context_and_cache(ctx):
    c = C.byref(_cache())
    assert nv._lib.nova_cache4_append(None, c, FAKE, FAKE, 128, FAKE, 4, 1, None) == 1
    assert nv._lib.nova_cache4_read(None, c, None, FAKE, 4, FAKE, FAKE, 128, None) == 1
    assert nv._lib.nova_cache4_attention(None, c, FAKE, 128, FAKE, 4, FAKE, None, None) == 1
    assert nv._lib.nova_cache4_weights(None, c, FAKE, 128, FAKE, FAKE, 4, None, FAKE, None) == 1
    assert nv._lib.nova_cache4_evict(None, c, FAKE, 8, 2, c, None, FAKE, None) == 1
    assert nv._lib.nova_cache4_append(ctx, None, FAKE, FAKE, 128, FAKE, 4, 1, None) == 1
    assert nv._lib.nova_cache4_evict(ctx, c, FAKE, 8, 2, None, None, FAKE, None) == 1
    assert nv._lib.nova_cache4_workspace_bytes(None, c, 4) == 0


@pytest.mark.parametrize("k,cu,m,ld,status", [(None, FAKE, 4, 128, 1), (FAKE, None, 4, 128, 1), (FAKE, FAKE, -1, 128, 1), (FAKE, FAKE, 4, 120, 1),
                                              (FAKE, FAKE, 4, 132, 3), (FAKE + 2, FAKE, 4, 128, 3)])
def test_bad_rows(ctx, k, cu, m, ld, status):
    c = C.byref(_cache())
    assert nv._lib.nova_cache4_append(ctx, c, k, FAKE, ld, cu, m, 1, None) == status
    assert nv._lib.nova_cache4_append(ctx, c, FAKE, k, ld, cu, m, 1, None) == status
    assert nv._lib.nova_cache4_read(ctx, c, None, cu, m, k, FAKE, ld, None) == status
    assert nv._lib.nova_cache4_attention(ctx, c, k, ld, cu, m, FAKE, None, None) == status
    assert nv._lib.nova_cache4_attention(ctx, c, FAKE, ld, cu, m, k, None, None) == status
    assert nv._lib.nova_cache4_weights(ctx, c, k, ld, FAKE, cu, m, None, FAKE, None) == status


def test_bad_vectors(ctx):
    c = C.byref(_cache())
    assert nv._lib.nova_cache4_attention(ctx, c, FAKE, 128, FAKE, 4, 2 * FAKE, FAKE + 2, None) == 3
    assert nv._lib.nova_cache4_attention(ctx, c, FAKE, 128, FAKE, 4, FAKE, None, None) == 1      # in place
    assert nv._lib.nova_cache4_weights(ctx, c, FAKE, 128, None, FAKE, 4, None, FAKE, None) == 1
    assert nv._lib.nova_cache4_weights(ctx, c, FAKE, 128, FAKE, FAKE, 4, None, None, None) == 1
    assert nv._lib.nova_cache4_weights(ctx, c, FAKE, 128, FAKE, None, 0, None, FAKE, None) == 1
    assert nv._lib.nova_cache4_weights(ctx, c, FAKE, 128, FAKE, FAKE, 4, FAKE + 1, FAKE, None) == 3


def test_bad_evictions(ctx):
    def evict(src=None, dst=None, weight=20 * FAKE, budget=8, recent=2, w_out=None, rows=21 * FAKE):
        return nv._lib.nova_cache4_evict(ctx, C.byref(_cache(**(src or {}))), weight, budget, recent, C.byref(_cache(**dict(OTHER, **(dst or {})))),
                                         w_out, rows, None)
    assert evict(budget=-1, recent=0) == 1 and evict(recent=-1) == 1 and evict(recent=9) == 1
    assert evict(budget=65) == 2
    assert evict(src=dict(Lmax=(1 << 30) + 1)) == 2
    assert evict(dst=dict(B=3)) == 1 and evict(dst=dict(C=192)) == 2 and evict(dst=dict(C=256)) == 1 and evict(dst=dict(n_heads=1)) == 1
    assert evict(weight=None) == 1 and evict(w_out=20 * FAKE) == 1
    assert evict(weight=20 * FAKE + 2) == 3 and evict(w_out=22 * FAKE + 1) == 3 and evict(rows=21 * FAKE + 2) == 3
    # memory that overlaps without starting at the same place: 2 * 64 rows of 64 bytes of codes, of 8 of scales, 512 bytes of weights
    assert evict(dst=dict(k_codes=FAKE + 2 * 64 * 64 - 16)) == 1 and evict(dst=dict(v_scales=4 * FAKE - 2 * 64 * 8 + 16)) == 1
    assert evict(w_out=20 * FAKE + 2 * 64 * 4 - 4) == 1 and evict(rows=11 * FAKE + 64) == 1 and evict(rows=15 * FAKE) == 1
    for shared in ("k_codes", "v_codes", "k_scales", "v_scales", "kv_len"):
        assert evict(dst={shared: getattr(_cache(), shared)}) == 1
    if not torch.cuda.is_available():
        assert evict(rows=None) == 4                   # no workspace for the list


def test_binding_refuses_wrong_tensors():
    def cache(**kw):
        f = dict(k_codes=torch.zeros((1, 4, 64), dtype=torch.uint8), v_codes=torch.zeros((1, 4, 64), dtype=torch.uint8),
                 k_scales=torch.zeros((1, 4, 4), dtype=torch.bfloat16), v_scales=torch.zeros((1, 4, 4), dtype=torch.bfloat16),
                 kv_len=torch.zeros(1, dtype=torch.int32), n_heads=1)
        f.update(kw)
        return nv.Cache4(**f)
    c = cache()
    for kw in (dict(k_codes=torch.zeros((1, 4, 64), dtype=torch.int8)), dict(v_codes=torch.zeros((1, 5, 64), dtype=torch.uint8)),
               dict(k_scales=torch.zeros((1, 4, 2), dtype=torch.bfloat16)), dict(v_scales=torch.zeros((1, 4, 4))), dict(kv_len=torch.zeros(2, dtype=torch.int32)),
               dict(v_codes=torch.zeros((1, 4, 128), dtype=torch.uint8)[..., ::2])):
        with pytest.raises(AssertionError):
            cache(**kw)
    rows = torch.zeros((3, 128), dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    for bad in (rows.float(), rows[:, :64], torch.zeros((3, 256), dtype=torch.bfloat16)[:, ::2], rows[0]):
        with pytest.raises(AssertionError):
            nv._rows4(c, bad)
    assert nv._rows4(c, torch.zeros((3, 384), dtype=torch.bfloat16)[:, 128:256]) == (3, 384)
    with pytest.raises(AssertionError):
        nv._cu4(c, cu.long())
    with pytest.raises(AssertionError):
        nv._cu4(c, torch.zeros(3, dtype=torch.int32))
