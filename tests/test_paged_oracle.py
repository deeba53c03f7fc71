"""Pins of the paged-cache oracle by hand, and the refusals of the entry points (no GPU)."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2608_03682_b200 import binding, build


def test_heads_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])                 # mean square 25 / 4
    y, _ = P.heads(x, np.array([0.0, 1.0, 0.0, 0.0]), 0.0, None, None)
    assert np.allclose(y[0, 0], [1.2, 3.2, 0.0, 0.0])
    table = np.array([[[1.0, 0.0], [1.0, 0.0]], [[0.0, 1.0], [1.0, 0.0]]])   # position 1 turns the first pair by 90 degrees
    y, size = P.heads(np.array([[[1.0, 2.0, 3.0, 4.0]]]), None, 0.0, table, [1])
    assert np.allclose(y[0, 0], [-3.0, 2.0, 1.0, 4.0]) and np.allclose(size[0, 0], [3.0, 2.0, 1.0, 4.0])


def test_slots_append_and_pack_by_hand():
    table = [[2, 0], [1, -1]]
    assert list(P.slots(table[0], 2, 3)) == [4, 5, 0]
    k = np.arange(4.0).reshape(4, 1, 1) + 1
    pk, pv = P.append(np.zeros((6, 1, 1)), np.zeros((6, 1, 1)), k, -k, [0, 2, 4], [3, 2], table, 2)
    assert list(pk.ravel()) == [2.0, 0.0, 3.0, 4.0, 0.0, 1.0] and list(pv.ravel()) == [-2.0, 0.0, -3.0, -4.0, 0.0, -1.0]
    packed, cu = P.pack(np.stack([pk, pv])[None], [3, 2], table, 2)
    assert list(cu) == [0, 3, 5] and list(packed[0, 0].ravel()) == [0.0, 1.0, 2.0, 3.0, 4.0]


def test_attention_by_hand():
    assert list(P.limits(3, 5, True, 0)) == [3, 4, 5] and list(P.limits(3, 5, True, 4)) == [4, 4, 5]
    assert list(P.limits(4, 2, True, 0)) == [0, 0, 1, 2] and list(P.limits(2, 3, False, 0)) == [3, 3]
    k = np.zeros((4, 1, 2))
    v = np.array([[[1.0, 0.0]], [[3.0, 0.0]], [[5.0, 0.0]], [[np.nan, 0.0]]])
    out, _, _ = P.attend(np.ones((3, 1, 2)), k, v, [0, 3], [2], [[0, 1]], 2, True)
    assert np.array_equal(out[:, 0, 0], [0.0, 1.0, 2.0])   # equal logits: means of the first 0, 1 and 2 values
    k[1, 0, 0] = 1.0                                        # one logit larger by log 3
    out, _, _ = P.attend(np.array([[[np.log(3.0), 0.0]]]), k, v, [0, 1], [2], [[0]], 2, False, scale=1.0)
    assert np.isclose(out[0, 0, 0], (1.0 + 3.0 * 3.0) / 4.0)


# ---- refusals: checked before the device is touched
@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


ADDRESS = 1 << 20         # an aligned address that nothing reads


def _cache(**kw):
    d = binding.PagedCacheDesc(C.sizeof(binding.PagedCacheDesc), 2, 1, 64, 16, binding.DTYPES["bf16"], 4, ADDRESS)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def _heads(**kw):
    d = binding.HeadsDesc(C.sizeof(binding.HeadsDesc), 4, 1, 64, binding.DTYPES["bf16"], binding.DTYPES["bf16"], 1e-6)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def _attend(lib, cache, **kw):
    a = dict(layer=0, hq=4, tokens=2, q=ADDRESS, q_stride=256, batch=1, cu=ADDRESS, lens=ADDRESS, table=ADDRESS, most=2, causal=1, prefix=None,
             scale=0.0, out=2 * ADDRESS, work=None, size=0, status=ADDRESS)
    a.update(kw)
    return lib.phyai_paged_attention(C.byref(cache) if cache is not None else None, *list(a.values())[:-1], a["status"], None)


BAD, NO = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED


@pytest.mark.parametrize("cache,status", [
    (dict(struct_size=4), BAD), (dict(pages=None), BAD), (dict(pages=ADDRESS + 8), BAD), (dict(n_layers=0), BAD), (dict(n_pages=0), BAD),
    (dict(n_kv_heads=0), BAD), (dict(head_dim=96), NO), (dict(page_size=0), NO), (dict(page_size=8), NO), (dict(page_size=48), NO),
    (dict(page_size=512), NO), (dict(dtype=binding.DTYPES["w8e4m3"]), NO), (dict(n_pages=1 << 31), BAD),
])
def test_caches_that_are_refused(lib, cache, status):
    assert _attend(lib, _cache(**cache)) == status
    assert lib.phyai_paged_last_error()
    assert lib.phyai_pack_paged_kv(C.byref(_cache(**cache)), 1, ADDRESS, ADDRESS, 2, ADDRESS, 8, ADDRESS, ADDRESS, None) == status


@pytest.mark.parametrize("call", [
    dict(layer=2), dict(hq=0), dict(q=None), dict(q=ADDRESS + 2), dict(q_stride=255), dict(q_stride=260), dict(q_stride=192), dict(batch=0), dict(batch=1025),
    dict(cu=None), dict(lens=None), dict(table=None), dict(most=0), dict(causal=0, prefix=ADDRESS), dict(scale=-1.0), dict(scale=float("nan")),
    dict(out=None), dict(out=2 * ADDRESS + 4), dict(out=ADDRESS), dict(q=2 * ADDRESS - 1008), dict(out=ADDRESS + 32768 - 16), dict(status=None), dict(most=1 << 28), dict(cu=ADDRESS + 2), dict(lens=ADDRESS + 1),
    dict(table=ADDRESS + 3), dict(status=ADDRESS + 2), dict(prefix=ADDRESS + 2), dict(tokens=1 << 31),
])
def test_attention_calls_that_are_refused(lib, call):
    assert _attend(lib, _cache(), **call) == BAD
    assert lib.phyai_paged_last_error()


def test_attention_heads_that_do_not_divide_are_refused(lib):
    assert _attend(lib, _cache(n_kv_heads=3)) == BAD
    assert _attend(lib, None) == BAD


@pytest.mark.parametrize("desc,call,status", [
    (dict(struct_size=1), {}, BAD), (dict(n_kv_heads=0), {}, BAD), (dict(n_q_heads=0), {}, BAD), (dict(head_dim=80), {}, NO),
    (dict(out_dtype=binding.DTYPES["f32"]), {}, NO), (dict(in_dtype=binding.DTYPES["w4a16"]), {}, NO), ({}, dict(k=None), BAD),
    ({}, dict(q_out=None), BAD), ({}, dict(k_out=None), BAD), ({}, dict(status=None), BAD), ({}, dict(positions=None), BAD),
    ({}, dict(q_stride=128), BAD), ({}, dict(k_stride=32), BAD), ({}, dict(k_stride=68), BAD), ({}, dict(rope=ADDRESS + 4), BAD),
    ({}, dict(n_positions=0), BAD), ({}, dict(q_gain=ADDRESS + 4), BAD), ({}, dict(positions=ADDRESS + 2), BAD), ({}, dict(status=ADDRESS + 1), BAD),
])
def test_head_calls_that_are_refused(lib, desc, call, status):
    a = dict(tokens=3, q=ADDRESS, q_stride=256, k=ADDRESS, k_stride=64, positions=ADDRESS, rope=ADDRESS, n_positions=10, q_gain=None, k_gain=None,
             q_out=ADDRESS, k_out=ADDRESS, status=ADDRESS)
    a.update(call)
    assert lib.phyai_norm_rope_heads(C.byref(_heads(**desc)), *a.values(), None) == status
    assert lib.phyai_paged_last_error()


@pytest.mark.parametrize("desc,call,status", [
    (dict(n_kv_heads=2), dict(k_stride=128, v_stride=128), BAD), (dict(head_dim=128), dict(q_stride=512, k_stride=128, v_stride=128), BAD),
    (dict(in_dtype=0, out_dtype=0), {}, BAD), ({}, dict(v=None), BAD), ({}, dict(v=ADDRESS + 8), BAD), ({}, dict(v_stride=60), BAD),
    ({}, dict(layer=7), BAD), ({}, dict(batch=2000), BAD), ({}, dict(cu=None), BAD), ({}, dict(status=None), BAD),
])
def test_append_calls_that_are_refused(lib, desc, call, status):
    a = dict(layer=0, tokens=3, q=ADDRESS, q_stride=256, k=ADDRESS, k_stride=64, v=ADDRESS, v_stride=64, batch=1, cu=ADDRESS, lens=ADDRESS,
             table=ADDRESS, most=2, positions=None, rope=ADDRESS, n_positions=10, q_gain=None, k_gain=None, q_out=ADDRESS, status=ADDRESS)
    a.update(call)
    assert lib.phyai_append_paged_kv(C.byref(_cache()), C.byref(_heads(**desc)), *a.values(), None) == status


def test_pack_calls_that_are_refused(lib):
    c = _cache()
    ok = [1, ADDRESS, ADDRESS, 2, ADDRESS, 8, ADDRESS, ADDRESS]
    for i, v in ((0, 0), (0, 1025), (1, None), (2, None), (3, 0), (4, None), (4, ADDRESS + 4), (6, None), (7, None), (5, 1 << 31)):
        a = list(ok)
        a[i] = v
        assert lib.phyai_pack_paged_kv(C.byref(c), *a, None) == BAD, (i, v)


def test_calls_without_tokens_do_nothing(lib):
    assert _attend(lib, _cache(), tokens=0, q=None, out=None) == binding.OK
    assert lib.phyai_paged_attention_workspace_bytes(C.byref(_cache()), 4, 0, 1, 2) == 0


def test_no_workspace_for_calls_that_are_refused(lib):
    for c, *a in ((_cache(), 4, 0xffffffff, 1, 2), (_cache(), 4, 0xffffffff, 0xffffffff, 2), (_cache(n_kv_heads=3), 4, 8, 1, 2), (_cache(n_kv_heads=8), 4, 8, 1, 2),
                  (_cache(), 4, 8, 1025, 2), (_cache(page_size=0), 4, 8, 1, 0), (_cache(), 4, 8, 1, 0xffffffff), (_cache(n_kv_heads=0), 4, 8, 1, 2)):
        assert lib.phyai_paged_attention_workspace_bytes(C.byref(c), *a) == 0


def test_a_stream_of_another_device_is_refused():
    with pytest.raises(ValueError):
        binding._Elsewhere(torch.device("cuda", 0), types.SimpleNamespace(device=torch.device("cuda", 1)))


def test_options(lib):
    for key, value in ((b"wait_limit", 0), (b"wait_limit", -1), (b"wait_limit", 1 << 31), (b"other", 1), (None, 1)):
        assert lib.phyai_paged_set_option(key, value) == BAD and lib.phyai_paged_last_error()
    assert lib.phyai_paged_set_option(b"wait_limit", 1 << 22) == binding.OK
    with pytest.raises(binding.PhyaiError):
        binding.set_paged_option("wait_limit", 0)


@pytest.mark.parametrize("dtype,bytes_of_a_row", [("bf16", 128), ("f32", 256)])
def test_packing_into_the_pages_is_refused(lib, dtype, bytes_of_a_row):
    pool, packed = 2 * 2 * 64 * bytes_of_a_row, 2 * 2 * 8 * bytes_of_a_row           # 2 layers of 4 pages of 16 rows; 8 rows
    c = _cache(dtype=binding.DTYPES[dtype])
    for at in (ADDRESS, ADDRESS + pool - 16, ADDRESS - packed + 16):
        lib.phyai_pack_paged_kv(None, 0, None, None, 0, None, 0, None, None, None)
        assert lib.phyai_pack_paged_kv(C.byref(c), 1, ADDRESS, ADDRESS, 2, at, 8, ADDRESS, ADDRESS, None) == BAD
        assert b"overlaps" in lib.phyai_paged_last_error()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_tables_for_more_keys_than_the_kernels_count(lib, page):
    """Lengths are rounded up to tiles of 128 keys in 32 bits."""
    most = ((1 << 31) - 1) // page
    while most * page > (1 << 31) - 256:
        assert _attend(lib, _cache(page_size=page), most=most) == BAD
        assert lib.phyai_paged_attention_workspace_bytes(C.byref(_cache(page_size=page)), 4, 2, 1, most) == 0
        assert lib.phyai_pack_paged_kv(C.byref(_cache(page_size=page)), 1, ADDRESS, ADDRESS, most, 2 * ADDRESS, 8, ADDRESS, ADDRESS, None) == BAD
        most -= 1
