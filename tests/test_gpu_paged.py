"""The operators around a paged cache against the float64 oracle, through the public entry points.

Tolerances.  u = 2^-24 (fp32), h = half a step of the output type relative to the value (bf16 2^-8, fp32 2^-24).
* A head: the sum of dh squares is off by at most (dh + 2) u, its root, the products with the gain and the rotation add at most 10 u of
  the terms' size |a cos| + |b sin|: (dh + 12) u of it, and the store's rounding h |y|.
* Attention: a logit is off by (dh + 4) u of its sum |q k| scale (log2 units included), which is the relative error of its weight, in the
  numerator and in the denominator; the two sums over n keys add n u each, exponentials and merges of key ranges fewer than 64 u; the bf16
  path rounds each weight to bf16, 2^-8.  Of the size sum w |v| of a result, and the store's rounding of h (|o| + the error before it)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import expert_oracle as O
from oracle import paged_oracle as P
from paper_2608_03682_b200 import binding, synth

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
EPS = 1e-6


def rope_table(positions, dh, theta=10000.0):
    ang = np.arange(positions, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(dh // 2) / dh)[None, :]
    return torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], axis=-1).astype(np.float32))


def normal(rng, shape, dtype="bf16", std=1.0):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(std)).to(TYPES[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def check_heads(got, x, gain, table, positions, dtype):
    y, size = P.heads(f64(x), None if gain is None else f64(gain), EPS, None if table is None else f64(table), positions)
    tol = (x.shape[-1] + 12) * U * size
    tol = tol + HALF[dtype] * (np.abs(y) + tol)
    err = np.abs(f64(got) - y)
    assert (err <= tol).all(), (err - tol).max()


def check_attention(got, ref, dtype, dh, n_keys):
    out, size, big = ref
    rel = 2 * (dh + 4) * U * big + (2 * n_keys + 64) * U + (2.0 ** -8 if dtype == "bf16" else 0.0)
    tol = rel * size
    tol = tol + HALF[dtype] * (np.abs(out) + tol)
    err = np.abs(got - out)
    assert (err <= tol).all(), (np.nanmax(err - tol), np.argwhere(~(err <= tol))[:5])


class Paged:
    """A pool with requests in pages drawn without order; rows that hold no cached token are NaN."""

    def __init__(self, seed, q_lens, kv_lens, Hkv, dh, page, dtype="bf16", layers=2, layer=1, first_row=0, last_rows=0, spare_pages=3):
        self.rng = rng = np.random.default_rng(seed)
        self.q_lens, self.kv_lens, self.page, self.layer, self.dtype, self.Hkv, self.dh = q_lens, kv_lens, page, layer, dtype, Hkv, dh
        need = [-(-n // page) for n in kv_lens]
        n_pages = sum(need) + spare_pages
        ids = rng.permutation(n_pages)
        self.table = np.full((len(kv_lens), max(max(need), 1) + 1), -7, dtype=np.int32)      # (entries past the last page name no page)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.pages = torch.full((layers, 2, n_pages * page, Hkv, dh), float("nan"), dtype=TYPES[dtype])
        for b, n in enumerate(kv_lens):
            rows = P.slots(self.table[b], page, n)
            for l in range(layers):
                for p in range(2):
                    self.pages[l, p, rows] = normal(rng, (n, Hkv, dh), dtype)
        self.cu = first_row + np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.T = int(self.cu[-1]) + last_rows
        self.cache = binding.PagedCache(self.pages.cuda(), page)

    def device_args(self):
        return ints(self.cu), ints(self.kv_lens), ints(self.table)


# ------------------------------------------------------------------------------------------------------------------
# norm and rotation of heads
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq,Hkv,dh", [(8, 1, 256), (8, 2, 128), (4, 1, 64), (3, 3, 64), (5, 1, 128), (7, 7, 256)])
@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("T", [1, 5, 1203])
def test_heads_match_the_oracle(Hq, Hkv, dh, src, dst, T):
    rng = np.random.default_rng(T + dh)
    qkv = normal(rng, (T, (Hq + 2 * Hkv) * dh + 8), src, 3.0)          # (8: the rows' stride is not the heads' width)
    table, positions = rope_table(700, dh), rng.integers(0, 700, T)
    gq, gk = normal(rng, (dh,), "f32", 0.3), normal(rng, (dh,), "f32", 0.3)
    dev = qkv.cuda()
    q, k = dev[:, :Hq * dh].view(T, Hq, dh), dev[:, Hq * dh:(Hq + Hkv) * dh].view(T, Hkv, dh)
    status = ints([0])
    yq, yk = binding.norm_rope_heads(q, k, ints(positions), table.cuda(), gq.cuda(), gk.cuda(), eps=EPS, dtype=TYPES[dst], status=status)
    check_heads(yq, q, gq, table, positions, dst)
    check_heads(yk, k, gk, table, positions, dst)
    yq, yk = binding.norm_rope_heads(q, k, None, None, None, gk.cuda(), eps=EPS, dtype=TYPES[dst], status=status)     # q as it is, k normed
    check_heads(yq, q, None, None, None, dst)
    check_heads(yk, k, gk, None, None, dst)
    none, yk = binding.norm_rope_heads(None, k, ints(positions), table.cuda(), dtype=TYPES[dst], status=status)        # k, rotated only
    assert none is None and int(status.item()) == 0
    check_heads(yk, k, None, table, positions, dst)


def test_heads_in_place_and_zero_rows():
    rng = np.random.default_rng(3)
    T, Hq, Hkv, dh = 40, 4, 2, 128
    q, k = normal(rng, (T, Hq, dh)), normal(rng, (T, Hkv, dh))
    q[7] = 0                                                            # the norm of a zero head is zero
    table, positions, g = rope_table(50, dh), rng.integers(0, 50, T), normal(rng, (dh,), "f32", 0.3)
    qd, kd, status, lib = q.cuda(), k.cuda(), ints([0]), binding.load_library()
    pos, rope, gd = ints(positions), table.cuda(), g.cuda()
    desc = binding.HeadsDesc(C.sizeof(binding.HeadsDesc), Hq, Hkv, dh, 1, 1, EPS)
    st = lib.phyai_norm_rope_heads(C.byref(desc), T, qd.data_ptr(), Hq * dh, kd.data_ptr(), Hkv * dh, pos.data_ptr(), rope.data_ptr(), 50, gd.data_ptr(),
                                   gd.data_ptr(), qd.data_ptr(), kd.data_ptr(), status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == binding.OK
    check_heads(qd, q, g, table, positions, "bf16")
    check_heads(kd, k, g, table, positions, "bf16")
    assert not qd[7].any() and int(status.item()) == 0


def test_heads_with_a_position_outside_the_table():
    rng = np.random.default_rng(4)
    k, table, status = normal(rng, (6, 1, 64)).cuda(), rope_table(10, 64).cuda(), ints([0])
    _, y = binding.norm_rope_heads(None, k, ints([0, 9, 3, 10, 2, 1]), table, status=status)
    assert int(status.item()) == binding.ERR_INVALID_ARG
    status.zero_()
    binding.norm_rope_heads(None, k, ints([0, 9, -1, 5, 2, 1]), table, status=status)
    assert int(status.item()) == binding.ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq,Hkv,dh,page,src,dst,q_lens,kv_lens", [
    (8, 1, 256, 64, "bf16", "bf16", [1], [1]),
    (8, 1, 256, 64, "bf16", "bf16", [1] * 5, [64, 65, 1, 900, 128]),
    (8, 2, 128, 16, "f32", "bf16", [3, 0, 40, 1], [3, 0, 57, 17]),
    (4, 1, 64, 32, "f32", "f32", [17, 33, 5], [17, 50, 5]),
    (6, 2, 128, 128, "bf16", "bf16", [300, 0, 211], [300, 40, 513]),
    (3, 3, 64, 256, "bf16", "bf16", [2] * 70, [2 + 3 * i for i in range(70)]),
    (8, 1, 256, 16, "f32", "bf16", [968, 600], [968, 600]),
])
def test_append_matches_the_oracle(Hq, Hkv, dh, page, src, dst, q_lens, kv_lens):
    p = Paged(11, q_lens, kv_lens, Hkv, dh, page, dst, first_row=2, last_rows=3)
    qkv = normal(p.rng, (p.T, (Hq + 2 * Hkv) * dh), src)
    dev = qkv.cuda()
    q, k, v = (dev[:, a * dh:b * dh].view(p.T, b - a, dh) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    gq, gk, table = normal(p.rng, (dh,), "f32", 0.3), normal(p.rng, (dh,), "f32", 0.3), rope_table(1200, dh)
    before = p.cache.pages.clone()
    places = np.concatenate([np.arange(kv - n, kv) for n, kv in zip(q_lens, kv_lens)]).astype(np.int64)
    live = np.arange(p.cu[0], p.cu[-1])
    for positions in (None, p.rng.integers(0, 1200, p.T)):
        at = places if positions is None else positions[live]
        p.cache.pages.copy_(before)
        out = p.cache.append(1, k, v, *p.device_args(), table.cuda(), gk.cuda(), q=q, q_gain=gq.cuda(), eps=EPS,
                             positions=None if positions is None else ints(positions))
        assert p.cache.poll_status() == 0
        check_heads(out[2:2 + len(live)], q[2:2 + len(live)], gq, table, at, dst)
        rows = np.concatenate([P.slots(p.table[b], page, kv)[kv - n:] for b, (n, kv) in enumerate(zip(q_lens, kv_lens))])
        after = p.cache.pages
        check_heads(after[1, 0][rows], k[2:2 + len(live)], gk, table, at, dst)
        assert torch.equal(after[1, 1][rows], v[2:2 + len(live)].to(TYPES[dst]))
        rest = np.setdiff1d(np.arange(after.shape[2]), rows)
        assert torch.equal(after[0].view(torch.uint8), before[0].view(torch.uint8))                         # the other layer
        assert torch.equal(after[1][:, rest].contiguous().view(torch.uint8), before[1][:, rest].contiguous().view(torch.uint8))
    p.cache.pages.copy_(before)                                                               # keys and values as they are, no q
    assert p.cache.append(1, k, v, *p.device_args(), None) is None
    assert torch.equal(p.cache.pages[1, 0][rows], k[2:2 + len(live)].to(TYPES[dst]))


@pytest.mark.parametrize("what", ["backwards", "past", "negative", "long", "more new than cached", "lens negative"])
def test_append_with_lengths_out_of_order_writes_nothing(what):
    p = Paged(12, [3, 4], [10, 20], 1, 64, 16)
    cu, lens = p.cu.copy(), list(p.kv_lens)
    if what == "backwards": cu[1] = 9
    if what == "past": cu[2] = p.T + 1
    if what == "negative": cu[0] = -1
    if what == "long": lens[1] = p.table.shape[1] * 16 + 1
    if what == "more new than cached": lens[0] = 2
    if what == "lens negative": lens[1] = -1
    before = p.cache.pages.clone()
    k = normal(p.rng, (p.T, 1, 64)).cuda()
    p.cache.append(0, k, k, ints(cu), ints(lens), ints(p.table), None)
    assert p.cache.status.item() == binding.ERR_INVALID_ARG
    assert torch.equal(before.view(torch.uint8), p.cache.pages.view(torch.uint8))
    p.cache.append(0, k, k, *p.device_args(), None)                    # the word is up: nothing is written
    assert torch.equal(before.view(torch.uint8), p.cache.pages.view(torch.uint8))
    assert p.cache.poll_status() == binding.ERR_INVALID_ARG and p.cache.poll_status() == 0
    p.cache.append(0, k, k, *p.device_args(), None)
    assert not torch.equal(before.view(torch.uint8), p.cache.pages.view(torch.uint8))


def test_append_to_a_page_that_does_not_exist():
    p = Paged(13, [5, 5], [30, 20], 1, 64, 16)
    before, k = p.cache.pages.clone(), normal(p.rng, (p.T, 1, 64)).cuda()
    table = p.table.copy()
    table[0, 1] = p.cache.n_pages
    p.cache.append(0, k, k, ints(p.cu), ints(p.kv_lens), ints(table), None)
    assert p.cache.poll_status() == binding.ERR_INVALID_ARG
    rows = P.slots(p.table[1], 16, 20)[15:]
    rest = np.setdiff1d(np.arange(before.shape[2]), rows)              # only the other request's places may have changed
    assert torch.equal(before[:, :, rest].contiguous().view(torch.uint8), p.cache.pages[:, :, rest].contiguous().view(torch.uint8))


# ------------------------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------------------------
HEADS = [(8, 1, 256), (8, 2, 128), (4, 1, 64), (4, 4, 128), (6, 2, 256), (5, 1, 128), (32, 2, 64)]
LENS = {
    "tokens": ([1] * 9, [1, 15, 16, 17, 64, 129, 300, 33, 2]),
    "none": ([1, 0, 2, 1], [0, 5, 40, 70]),                             # no cached token; no new token
    "few": ([2, 5, 1, 3], [2, 70, 128, 257]),
    "more new than cached": ([6, 3], [4, 0]),                           # rows that see no key
    "chunks": ([33, 70, 16], [33, 200, 130]),
    "one chunk": ([130], [400]),
}


def run_attention(p, Hq, causal, prefix=None, scale=None, stride=0, layer=1):
    q = normal(p.rng, (p.T, Hq * p.dh + stride), p.dtype)
    qd = q.cuda()[:, :Hq * p.dh].view(p.T, Hq, p.dh)
    out = torch.full((p.T, Hq, p.dh), 777.0, dtype=TYPES[p.dtype], device="cuda")
    got = p.cache.attend(layer, qd, *p.device_args(), causal=causal, prefix_lens=None if prefix is None else ints(prefix), scale=scale, out=out)
    assert got is out and p.cache.poll_status() == 0
    live = slice(int(p.cu[0]), int(p.cu[-1]))
    dead = np.setdiff1d(np.arange(p.T), np.arange(live.start, live.stop))
    assert (out[dead] == 777.0).all()                                   # rows of no request stay as they were
    planes = f64(p.cache.pages[layer])
    ref = P.attend(f64(q[:, :Hq * p.dh].reshape(p.T, Hq, p.dh)), planes[0], planes[1], p.cu, p.kv_lens, p.table, p.page, causal, prefix, scale)
    check_attention(f64(out)[live], [r[live] for r in ref], p.dtype, p.dh, max(p.kv_lens) if p.kv_lens else 0)
    return qd, out


@pytest.mark.parametrize("Hq,Hkv,dh", HEADS)
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("mask", ["causal", "full", "prefix"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_matches_the_oracle(Hq, Hkv, dh, lens, mask, dtype):
    q_lens, kv_lens = LENS[lens]
    page = [16, 32, 64, 128, 256][(dh // 64 + len(lens) + len(mask)) % 5]
    p = Paged(21, q_lens, kv_lens, Hkv, dh, page, dtype, first_row=1, last_rows=2)
    prefix = None if mask != "prefix" else [n * 2 // 3 for n in kv_lens]
    run_attention(p, Hq, mask != "full", prefix, stride=8)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,dh", [(8, 1, 256), (4, 2, 128), (2, 1, 64)])
def test_attention_over_every_page_size(page, Hq, Hkv, dh):
    for q_lens, kv_lens in (([1, 1], [517, 255]), ([40, 17], [300, 17])):
        p = Paged(22, q_lens, kv_lens, Hkv, dh, page)
        run_attention(p, Hq, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.02, 3.0])
def test_attention_with_a_scale_and_large_logits(dtype, scale):
    p = Paged(23, [1, 30, 2], [700, 90, 2], 1, 128, 32, dtype)
    run_attention(p, 4, True, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (8, 1, 256, [1], [5000]), (8, 2, 128, [1, 1], [9001, 30]), (4, 1, 64, [2], [4100]), (8, 2, 128, [9], [3333]), (8, 1, 256, [40], [2500]),
])
def test_attention_over_long_histories(dtype, Hq, Hkv, dh, q_lens, kv_lens):
    p = Paged(24, q_lens, kv_lens, Hkv, dh, 64, dtype)
    run_attention(p, Hq, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [(8, 1, 256, [2, 1], [2, 40]), (4, 2, 128, [40, 3], [150, 20]), (2, 1, 64, [20], [33])])
def test_keys_that_a_row_does_not_see_have_no_part_in_it(dtype, value, Hq, Hkv, dh, q_lens, kv_lens):
    """The last token of every request has infinite or NaN keys and values: only its own row sees them."""
    p = Paged(25, q_lens, kv_lens, Hkv, dh, 16, dtype)
    q = normal(p.rng, (p.T, Hq, dh), dtype).cuda()
    clean = p.cache.attend(1, q, *p.device_args()).clone()
    last = [P.slots(p.table[b], 16, kv)[-1] for b, kv in enumerate(kv_lens)]
    p.cache.pages[1, :, last] = value
    got = p.cache.attend(1, q, *p.device_args())
    assert p.cache.poll_status() == 0
    rows = np.setdiff1d(np.arange(p.T), p.cu[1:] - 1)
    planes = f64(p.cache.pages[1])
    ref = P.attend(f64(q), planes[0], planes[1], p.cu, kv_lens, p.table, 16, True)
    check_attention(f64(got)[rows], [r[rows] for r in ref], dtype, dh, max(kv_lens))
    seen = p.cu[1:] - 1
    assert not torch.isfinite(got[seen]).all()
    assert torch.isfinite(clean).all()


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (8, 2, 128, [40] * 6, [6000, 300, 40, 2000, 100, 77]), (8, 1, 256, [64, 33], [5000, 33]), (4, 4, 64, [90, 1, 0, 17], [3000, 4000, 10, 17]),
    (8, 1, 256, [300], [2100]), (8, 1, 128, [400, 3], [400, 5000]), (6, 2, 128, [0, 0, 100, 0], [50, 20000, 3000, 0]),
])
@pytest.mark.parametrize("mask", ["causal", "full", "prefix"])
def test_attention_of_few_units_over_keys_of_any_lengths(Hq, Hkv, dh, q_lens, kv_lens, mask):
    """All tiles in a row, an equal part for each pair of blocks: parts that begin and end inside a unit, that hold several, units of one part."""
    prefix = [min(n, 70 * (i + 1)) for i, n in enumerate(kv_lens)] if mask == "prefix" else None
    run_attention(Paged(37, q_lens, kv_lens, Hkv, dh, 64, first_row=2, last_rows=3), Hq, mask != "full", prefix)


@pytest.mark.parametrize("seed", range(10))
def test_attention_of_few_units_at_random_lengths(seed):
    rng = np.random.default_rng(1000 + seed)
    Hq, Hkv, dh = [(8, 1, 256), (8, 2, 128), (4, 2, 64), (32, 8, 128)][seed % 4]
    kv = [int(2 ** rng.uniform(0, 12.5)) for _ in range(int(rng.integers(1, 7)))]
    q = [int(rng.integers(0, min(n, 150) + 1)) for n in kv]
    q[0] = max(q[0], 1)
    run_attention(Paged(38 + seed, q, kv, Hkv, dh, [16, 32, 64, 128, 256][seed % 5]), Hq, seed % 3 != 0)


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [(8, 1, 256, [150, 20], [4000, 900]), (8, 2, 128, [90], [7000])])
def test_keys_that_a_row_does_not_see_in_a_part_of_a_long_history(value, Hq, Hkv, dh, q_lens, kv_lens):
    """The newer half of the new tokens' keys and values, in whole tiles and inside one, hidden from the older half's rows."""
    p = Paged(39, q_lens, kv_lens, Hkv, dh, 32)
    q = normal(p.rng, (p.T, Hq, dh)).cuda()
    rows = []
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        p.cache.pages[1, :, P.slots(p.table[b], 32, kv)[kv - n // 2:]] = value
        rows += range(int(p.cu[b]), int(p.cu[b]) + n - n // 2)
    got = p.cache.attend(1, q, *p.device_args())
    assert p.cache.poll_status() == 0
    planes = f64(p.cache.pages[1])
    ref = P.attend(f64(q), planes[0], planes[1], p.cu, kv_lens, p.table, 32, True)
    check_attention(f64(got)[rows], [r[rows] for r in ref], "bf16", dh, max(kv_lens))


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (256, 1, 64, [1, 3], [40, 3]), (128, 1, 128, [2, 1], [200, 130]), (96, 1, 64, [5], [70]), (40, 4, 256, [30, 2], [131, 64]),
])
def test_attention_of_wide_groups_of_heads(Hq, Hkv, dh, q_lens, kv_lens):
    run_attention(Paged(30, q_lens, kv_lens, Hkv, dh, 32), Hq, True)


@pytest.mark.parametrize("dtype,q_len", [("bf16", 1), ("bf16", 5), ("f32", 1)])
def test_attention_of_1024_requests(dtype, q_len):
    rng = np.random.default_rng(33)
    kv = [int(x) for x in rng.integers(0, 40, 1024)]
    q = [min(q_len, n) if i % 7 else 0 for i, n in enumerate(kv)]
    run_attention(Paged(34, q, kv, 1, 64, 16, dtype), 4, True)


@pytest.mark.parametrize("dtype,q_lens,kv_lens", [("bf16", [1, 1, 1], [300, 2, 77]), ("bf16", [40, 9, 1], [300, 9, 77]), ("f32", [3, 1, 1], [300, 2, 77])])
def test_attention_with_a_table_far_wider_than_the_requests(dtype, q_lens, kv_lens):
    p = Paged(35, q_lens, kv_lens, 2, 128, 16, dtype)
    p.table = np.concatenate([p.table, np.full((3, 5000), 2 ** 31 - 1, dtype=np.int32)], axis=1)
    run_attention(p, 8, True)
    got, cu = p.cache.pack(ints(p.table), ints(kv_lens), sum(kv_lens) + 100)
    ref, _ = P.pack(p.pages.view(torch.int16 if dtype == "bf16" else torch.int32).numpy(), kv_lens, p.table, 16)
    assert np.array_equal(got[:, :, :sum(kv_lens)].contiguous().view(torch.int16 if dtype == "bf16" else torch.int32).cpu().numpy(), ref)


def test_attention_writes_nothing_while_the_status_word_is_up():
    for q_lens, kv_lens, dtype in (([1, 1], [50, 40], "bf16"), ([1], [3000], "bf16"), ([30, 60], [300, 200], "bf16"), ([3, 4], [10, 20], "f32")):
        p = Paged(36, q_lens, kv_lens, 1, 128, 16, dtype)
        q = normal(p.rng, (p.T, 4, 128), dtype).cuda()
        out = torch.full_like(q, 5.0)
        p.cache.status.fill_(binding.ERR_TIMEOUT)
        p.cache.attend(1, q, *p.device_args(), out=out)
        packed, _ = p.cache.pack(ints(p.table), ints(kv_lens), sum(kv_lens), out=torch.full((2, 2, sum(kv_lens), 1, 128), 5.0, dtype=TYPES[dtype], device="cuda"))
        assert (out == 5.0).all() and (packed == 5.0).all() and p.cache.poll_status() == binding.ERR_TIMEOUT
        p.cache.attend(1, q, *p.device_args(), out=out)
        assert p.cache.poll_status() == 0 and not (out == 5.0).any()


def test_attention_with_pages_shared_by_requests():
    p = Paged(26, [1, 4, 40], [100, 90, 97], 1, 256, 16)
    p.table[1, :5], p.table[2, :4] = p.table[0, :5], p.table[0, :4]     # a common beginning
    run_attention(p, 8, True)


def test_attention_is_the_same_every_time():
    for q_lens, kv_lens in (([1] * 4, [3000, 77, 900, 12]), ([50, 200], [1800, 200])):
        p = Paged(27, q_lens, kv_lens, 2, 128, 64)
        q = normal(p.rng, (p.T, 8, 128)).cuda()
        first = p.cache.attend(1, q, *p.device_args()).clone()
        for _ in range(5):
            assert torch.equal(first, p.cache.attend(1, q, *p.device_args()))


@pytest.mark.parametrize("what", ["backwards", "past", "long", "lens negative"])
@pytest.mark.parametrize("q_lens,kv_lens,dtype", [([1, 1], [50, 40], "bf16"), ([30, 60], [300, 200], "bf16"), ([3, 4], [10, 20], "f32")])
def test_attention_with_lengths_out_of_order_writes_nothing(what, q_lens, kv_lens, dtype):
    p = Paged(28, q_lens, kv_lens, 1, 128, 16, dtype)
    cu, lens = p.cu.copy(), list(kv_lens)
    if what == "backwards": cu[1] = cu[2] + 1
    if what == "past": cu[2] = p.T + 1
    if what == "long": lens[1] = p.table.shape[1] * 16 + 1
    if what == "lens negative": lens[0] = -3
    q = normal(p.rng, (p.T, 4, 128), dtype).cuda()
    out = torch.full_like(q, 5.0)
    p.cache.attend(1, q, ints(cu), ints(lens), ints(p.table), out=out)
    assert p.cache.poll_status() == binding.ERR_INVALID_ARG and (out == 5.0).all()


@pytest.mark.parametrize("q_lens,kv_lens,dtype", [([1, 1], [50, 40], "bf16"), ([30, 60], [300, 200], "bf16"), ([3, 4], [10, 20], "f32")])
def test_attention_over_a_page_that_does_not_exist(q_lens, kv_lens, dtype):
    p = Paged(29, q_lens, kv_lens, 1, 128, 16, dtype)
    for entry in (-1, p.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = p.table.copy()
        table[1, 0] = entry
        p.cache.attend(1, normal(p.rng, (p.T, 4, 128), dtype).cuda(), ints(p.cu), ints(p.kv_lens), ints(table))
        assert p.cache.poll_status() == binding.ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------------------------
# pack, and the operators as they are used together
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,Hkv,dh,page,lens", [("bf16", 1, 256, 64, [816]), ("bf16", 3, 64, 16, [0, 1, 16, 17, 300]), ("f32", 2, 128, 32, [33, 0, 64]),
                                                    ("bf16", 1, 64, 256, [0]), ("f32", 1, 64, 16, [5] * 300)])
def test_pack_matches_the_oracle(dtype, Hkv, dh, page, lens):
    p = Paged(31, [0] * len(lens), lens, Hkv, dh, page, dtype, layers=3)
    total = sum(lens)
    out = torch.full((3, 2, total + 5, Hkv, dh), 9.0, dtype=TYPES[dtype], device="cuda")
    got, cu = p.cache.pack(ints(p.table), ints(lens), total + 5, out=out)
    assert p.cache.poll_status() == 0
    ref, ref_cu = P.pack(p.pages.view(torch.int16 if dtype == "bf16" else torch.int32).numpy(), lens, p.table, page)
    assert np.array_equal(cu.cpu().numpy(), ref_cu)
    assert np.array_equal(got[:, :, :total].contiguous().view(torch.int16 if dtype == "bf16" else torch.int32).cpu().numpy(), ref)
    assert (got[:, :, total:] == 9.0).all()
    if total > 1:
        out.fill_(9.0)
        p.cache.pack(ints(p.table), ints(lens), total - 1, out=out[:, :, :total - 1].contiguous())
        assert p.cache.poll_status() == binding.ERR_INVALID_ARG


def test_pack_of_a_page_that_does_not_exist():
    p = Paged(32, [0, 0], [40, 50], 1, 64, 16)
    p.table[1, 2] = -1
    p.cache.pack(ints(p.table), ints([40, 50]), 90)
    assert p.cache.poll_status() == binding.ERR_INVALID_ARG


def prefill(cache, table, lens, chunks, layers, weights, rope, Hq, seed):
    """A backbone's layers in little: rows of q | k | v made from the token numbers and the layer's input, appended and attended over."""
    L, Hkv, dh = layers, cache.n_kv_heads, cache.head_dim
    x = [torch.randn(n, 64, generator=torch.Generator().manual_seed(seed + b)).cuda() for b, n in enumerate(lens)]
    done, outs = [0] * len(lens), [[] for _ in lens]
    for step in range(max(len(c) for c in chunks)):
        n = [c[step] if step < len(c) else 0 for c in chunks]
        rows = torch.cat([x[b][done[b]:done[b] + n[b]] for b in range(len(lens))])
        done = [d + m for d, m in zip(done, n)]
        cu, kv, tab = ints(np.concatenate([[0], np.cumsum(n)])), ints(done), ints(table)
        h = rows
        for l in range(L):
            qkv = (h @ weights[l][0]).to(torch.bfloat16)
            T = qkv.shape[0]
            q, k, v = qkv[:, :Hq * dh].view(T, Hq, dh), qkv[:, Hq * dh:(Hq + Hkv) * dh].view(T, Hkv, dh), qkv[:, (Hq + Hkv) * dh:].view(T, Hkv, dh)
            qr = cache.append(l, k, v, cu, kv, tab, rope, weights[l][2], q=q, q_gain=weights[l][3])
            h = h + cache.attend(l, qr, cu, kv, tab).view(T, Hq * dh).float() @ weights[l][1]
        for b, part in enumerate(h.split(n)):
            outs[b].append(part)
    return [torch.cat(o) for o in outs]


def test_prefix_prefilled_in_chunks_feeds_the_denoising_loop():
    """Chunks of any size give the cache of one chunk (to the rounding of the differently split sums), and the packed cache gives the
    actions of the same cache packed by phyai_pack_prefix_kv, bit for bit."""
    cfg = synth.ExpertConfig(n_layers=2, width=256, mlp_dim=512, n_q_heads=2, n_kv_heads=1, head_dim=128, state_dim=6, action_dim=5, horizon=13,
                             has_state_token=True, max_prefix_len=200, max_batch=3)
    Hq, Hkv, dh, lens, page = 4, 1, 128, [150, 37, 64], 16
    rng = np.random.default_rng(41)
    weights = [(normal(rng, (64, (Hq + 2 * Hkv) * dh), "f32", 0.125).cuda(), normal(rng, (Hq * dh, 64), "f32", 0.04).cuda(),
                normal(rng, (dh,), "f32", 0.1).cuda(), normal(rng, (dh,), "f32", 0.1).cuda()) for _ in range(cfg.n_layers)]
    rope = rope_table(256, dh).cuda()
    caches, results = [], []
    for chunks in ([[150], [37], [64]], [[100, 1, 49], [1, 35, 1], [16, 48]], [[7] * 21 + [3], [37], [1] * 64]):
        p = Paged(42, [0, 0, 0], lens, Hkv, dh, page, layers=cfg.n_layers)
        results.append(prefill(p.cache, p.table, lens, chunks, cfg.n_layers, weights, rope, Hq, 5))
        assert p.cache.poll_status() == 0
        caches.append(p)
    for other, res in zip(caches[1:], results[1:]):
        for b in range(3):
            assert O.max_rel_err(f64(res[b]), f64(results[0][b])) < 2e-2      # bf16 rows, weights rounded at other maxima
    p = caches[0]
    packed, cu = p.cache.pack(ints(p.table), ints(lens), sum(lens))
    k, v = (torch.zeros(cfg.n_layers, 3, 160, Hkv, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b, n in enumerate(lens):
        rows = P.slots(p.table[b], page, n)
        k[:, b, :n], v[:, b, :n] = p.cache.pages[:, 0][:, rows], p.cache.pages[:, 1][:, rows]
    dense, cu2, status = binding.pack_prefix_kv(k, v, ints(lens), sum(lens))
    assert torch.equal(packed, dense) and torch.equal(cu, cu2)
    W = synth.make_weights(cfg, 1, std=0.05)
    with binding.Expert(cfg, binding.weights_to_device(W)) as ex:
        states, noise = torch.randn(3, 6).cuda(), torch.randn(3, 13, 5).cuda()
        a = ex.denoise_batched(packed, cu, states, noise, 3).clone()
        b = ex.denoise_batched(dense, cu2, states, noise, 3)
        assert ex.poll_status() == 0 and torch.equal(a, b) and torch.isfinite(a).all()


# ------------------------------------------------------------------------------------------------------------------
# streams, graphs, large caches
# ------------------------------------------------------------------------------------------------------------------
def test_operators_on_a_stream_of_their_own():
    p = Paged(51, [1, 40], [700, 130], 1, 256, 64)
    q = normal(p.rng, (p.T, 8, 256)).cuda()
    k = normal(p.rng, (p.T, 1, 256)).cuda()
    args = p.device_args()
    rope = rope_table(1000, 256).cuda()
    qr = p.cache.append(1, k, k, *args, rope, q=q)
    want = p.cache.attend(1, qr, *args)
    packed, cu = p.cache.pack(args[2], args[1], 830)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(torch.cuda.Stream()):
        q2 = p.cache.append(1, k, k, *args, rope, q=q, stream=side)
        got = p.cache.attend(1, q2, *args, stream=side)
        packed2, cu2 = p.cache.pack(args[2], args[1], 830, stream=side)
        hq, hk = binding.norm_rope_heads(q, k, ints(np.arange(p.T)), rope, stream=side)
    side.synchronize()
    assert torch.equal(want, got) and torch.equal(packed, packed2) and torch.equal(cu, cu2) and torch.equal(qr, q2)
    want = binding.norm_rope_heads(q, k, ints(np.arange(p.T)), rope)
    assert torch.equal(want[0], hq) and torch.equal(want[1], hk)


def test_calls_on_two_streams_at_a_time():
    """Each of them alone fills the device; results as one after the other."""
    cases = []
    for seed, Hq, Hkv, dh, q_lens, kv_lens in ((54, 8, 1, 256, [300] * 6, [300] * 6), (55, 8, 2, 128, [200, 77], [3000, 900]), (56, 4, 1, 64, [500, 600], [600, 600]), (57, 8, 1, 256, [1] * 30, [700] * 30)):
        p = Paged(seed, q_lens, kv_lens, Hkv, dh, 64)
        q = normal(p.rng, (p.T, Hq, dh)).cuda()
        args = p.device_args()
        cases.append((p, q, args, p.cache.attend(1, q, *args).clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = [p.cache.attend(1, q, *args, stream=st) for (p, q, args, _), st in zip(cases, streams)]
        torch.cuda.synchronize()
        for (p, _, _, want), g in zip(cases, got):
            assert p.cache.poll_status() == 0 and torch.equal(want, g)


def test_captured_calls_follow_the_lengths_of_a_replay():
    """One graph of append and attend, replayed while the requests grow token by token; two graphs side by side keep apart."""
    graphs = []
    for seed in (52, 53):
        p = Paged(seed, [1, 1], [400, 30], 2, 128, 16)
        k, v, q = (normal(p.rng, (2, h, 128)).cuda() for h in (2, 2, 8))
        cu, lens, table = p.device_args()
        rope = rope_table(500, 128).cuda()
        p.cache.attend(1, p.cache.append(1, k, v, cu, lens, table, rope, q=q), cu, lens, table)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            qr = p.cache.append(1, k, v, cu, lens, table, rope, q=q)
            out = p.cache.attend(1, qr, cu, lens, table)
        graphs.append((p, graph, k, v, q, lens, out, rope, qr, cu, table))      # (a graph reads them at their addresses)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for n in ((350, 30), (351, 1), (7, 29), (400, 17)):
        for p, graph, k, v, q, lens, *_ in graphs:
            lens.copy_(torch.tensor(n, dtype=torch.int32))
            k.normal_()
            q.normal_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g[1].replay()
        torch.cuda.synchronize()
        for p, graph, k, v, q, lens, out, rope, qr, *_ in graphs:
            assert p.cache.poll_status() == 0
            planes = f64(p.cache.pages[1])
            ref = P.attend(f64(qr), planes[0], planes[1], p.cu, n, p.table, 16, True)
            check_attention(f64(out), ref, "bf16", 128, max(n))
            rows = [P.slots(p.table[b], 16, n[b])[-1] for b in range(2)]
            check_heads(p.cache.pages[1, 0][rows], k, None, rope, [m - 1 for m in n], "bf16")


def test_rows_past_32_bits_of_a_large_pool():
    """Pages whose rows lie more than 2^32 elements into the pool."""
    dh, page, n_pages = 256, 256, 36000                                  # 9.2 M rows of 256: 2.36 G elements a plane, 9.4 GB
    pages = torch.zeros(1, 2, n_pages * page, 1, dh, dtype=torch.bfloat16, device="cuda")
    cache = binding.PagedCache(pages, page)
    rng = np.random.default_rng(61)
    table = np.array([[n_pages - 1, 5, n_pages - 3], [n_pages - 2, n_pages - 9, 17]], dtype=np.int32)
    rope = rope_table(800, dh).cuda()
    for q_lens, lens in (([600, 500], [600, 500]), ([1, 1], [601, 501])):
        cu = np.concatenate([[0], np.cumsum(q_lens)])
        T = int(cu[-1])
        q, k, v = normal(rng, (T, 8, dh)).cuda(), normal(rng, (T, 1, dh)).cuda(), normal(rng, (T, 1, dh)).cuda()
        cache.append(0, k, v, ints(cu), ints(lens), ints(table), rope)
        for b in range(2):
            rows = P.slots(table[b], page, lens[b])[lens[b] - q_lens[b]:]
            assert torch.equal(pages[0, 1][torch.from_numpy(rows).cuda()], v[cu[b]:cu[b + 1]])
        out = cache.attend(0, q, ints(cu), ints(lens), ints(table))
        assert cache.poll_status() == 0
        pick = np.array([0, 1, T // 2, T - 1]) if T > 4 else np.arange(T)
        used = np.concatenate([P.slots(table[b], page, lens[b]) for b in range(2)])
        small = pages[0][:, torch.from_numpy(used).cuda()]               # the oracle's pool: the used rows alone
        planes = f64(small)
        for t in pick:
            b = int(np.searchsorted(cu, t, side="right") - 1)
            at = lens[b] - q_lens[b] + t - cu[b] + 1
            first = 0 if b == 0 else lens[0]
            fake = np.arange(at)[None, :] + first
            ref = P.attend(f64(q[t:t + 1]), planes[0], planes[1], [0, 1], [int(at)], fake, 1, True)
            check_attention(f64(out[t:t + 1]), ref, "bf16", dh, 700)
    packed, _ = cache.pack(ints(table), ints([601, 501]), 1102)
    assert cache.poll_status() == 0 and torch.equal(packed[0], pages[0][:, torch.from_numpy(used).cuda()])


def test_arguments_that_the_binding_refuses():
    p = Paged(71, [2], [20], 2, 64, 16)
    q, k = normal(p.rng, (2, 4, 64)).cuda(), normal(p.rng, (2, 2, 64)).cuda()
    cu, lens, table = p.device_args()
    for bad in (lambda: p.cache.attend(1, q.float(), cu, lens, table), lambda: p.cache.attend(1, q.transpose(0, 1), cu, lens, table),
                lambda: p.cache.attend(1, q, cu.long(), lens, table), lambda: p.cache.attend(1, q, cu[:1], lens, table),
                lambda: p.cache.attend(1, q, cu, lens.cpu(), table), lambda: p.cache.attend(1, q, cu, lens, table, out=torch.empty(2, 4, 32).cuda()),
                lambda: p.cache.attend(1, q, cu, lens, table, scale=0.0), lambda: p.cache.append(1, k, k[:1], cu, lens, table, None),
                lambda: p.cache.append(1, k, k.float(), cu, lens, table, None), lambda: p.cache.append(1, k, k, cu, lens, table, rope_table(30, 32).cuda()),
                lambda: p.cache.pack(table, lens, 20, out=torch.empty(2, 2, 19, 2, 64).cuda()), lambda: binding.PagedCache(p.cache.pages, 24),
                lambda: binding.PagedCache(p.cache.pages.half(), 16), lambda: binding.norm_rope_heads(q, k, torch.zeros(3).int().cuda(), None)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: p.cache.attend(2, q, cu, lens, table), lambda: p.cache.attend(1, q[:, :3].contiguous(), cu, lens, table),
                lambda: p.cache.attend(1, q, cu, lens, table, causal=False, prefix_lens=lens), lambda: p.cache.append(5, k, k, cu, lens, table, None)):
        with pytest.raises(binding.PhyaiError) as e:
            bad()
        assert e.value.status == binding.ERR_INVALID_ARG
    assert p.cache.poll_status() == 0
