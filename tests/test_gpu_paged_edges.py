"""The operators around a paged cache where calls go wrong or run long: bad entries and words that are up, waits that run out, other streams,
and the kernels' forms for many units, many rows and long ranges, against the float64 oracle.  Tolerances: see test_gpu_paged.py."""
import os
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2608_03682_b200 import binding
from tests.test_gpu_paged import EPS, TYPES, Paged, check_attention, check_heads, f64, ints, normal, rope_table

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------------
# what a call finds wrong on the device
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("q_len", [1, 3])
def test_fp32_blocks_that_begin_while_others_raise_the_word(q_len):
    """Every request of several waves of blocks has a bad entry, so that blocks begin before, while and after the word goes up: all threads of
    a block go by one value of it."""
    batch, kv = 600, 48
    p = Paged(81, [q_len] * batch, [kv] * batch, 2, 128, 16, "f32", layers=1, layer=0)
    q, args = normal(p.rng, (p.T, 4, 128), "f32").cuda(), p.device_args()
    want = p.cache.attend(0, q, *args)
    assert p.cache.poll_status() == 0
    table = p.table.copy()
    table[:, 1] = p.cache.n_pages
    bad = ints(table)
    for _ in range(50):
        p.cache.attend(0, q, *args[:2], bad)
        assert p.cache.poll_status() == binding.ERR_INVALID_ARG
    assert torch.equal(want, p.cache.attend(0, q, *args)) and p.cache.poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens,dtype", [(8, 2, 128, [1, 1], [9001, 3000], "bf16"), (8, 1, 256, [40], [2500], "bf16"),
                                                            (8, 2, 128, [1, 2], [900, 300], "f32")])
def test_the_word_changes_under_calls_that_run(Hq, Hkv, dh, q_lens, kv_lens, dtype):
    """The second kernel of split calls reads the word, too; whatever it finds while another stream writes it, the call ends, reads nothing outside
    its workspace (filled here with what would be 2^30 key ranges) and later ones are right."""
    p = Paged(82, q_lens, kv_lens, Hkv, dh, 64, dtype)
    q, args, side = normal(p.rng, (p.T, Hq, dh), dtype).cuda(), p.device_args(), torch.cuda.Stream()
    want = p.cache.attend(1, q, *args)
    torch.cuda.synchronize()
    for _ in range(20):
        for _ in range(20):
            torch.full((1 << 22,), float(1 << 30), device="cuda")       # (freed: the next call's workspace)
            p.cache.attend(1, q, *args)
            with torch.cuda.stream(side):
                p.cache.status.fill_(binding.ERR_INVALID_ARG)
                p.cache.status.zero_()
        torch.cuda.synchronize()
    assert torch.equal(want, p.cache.attend(1, q, *args)) and p.cache.poll_status() == 0


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("T,Hq,Hkv,dh", [(6, 3, 1, 64), (5000, 8, 1, 256), (3000, 8, 2, 128)])
def test_rows_of_positions_outside_the_table_are_nan_and_no_others(src, dst, T, Hq, Hkv, dh):
    """With a word, with one that is up, and without."""
    rng = np.random.default_rng(T + dh)
    table, positions, g = rope_table(100, dh), rng.integers(0, 100, T), normal(rng, (dh,), "f32", 0.3)
    q, k = normal(rng, (T, Hq, dh), src).cuda(), normal(rng, (T, Hkv, dh), src).cuda()
    bad = rng.permutation(T)[:max(2, T // 50)]
    positions[bad] = rng.choice([-1, 100, 2 ** 31 - 1, -2 ** 31], len(bad))
    good = np.setdiff1d(np.arange(T), bad)
    for status in (ints([0]), ints([binding.ERR_TIMEOUT]), None):
        yq, yk = binding.norm_rope_heads(q, k, ints(positions), table.cuda(), g.cuda(), None, eps=EPS, dtype=TYPES[dst], status=status)
        assert status is None or status.item() == binding.ERR_INVALID_ARG
        assert torch.isnan(yq[bad]).all() and torch.isnan(yk[bad]).all()
        check_heads(yq[good], q[good], g, table, positions[good], dst)
        check_heads(yk[good], k[good], None, table, positions[good], dst)


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def some_bad(p, share=0.1):
    """The table with an entry of some requests that names no page; their numbers."""
    table, bad = p.table.copy(), []
    for b, n in enumerate(p.kv_lens):
        pages = -(-n // p.page)
        if pages and p.rng.random() < share or not bad and b + 1 == len(p.kv_lens):
            table[b, p.rng.integers(0, pages)] = p.rng.choice([-1, p.cache.n_pages, 2 ** 31 - 1, -2 ** 31])
            bad.append(b)
    return table, bad


def rows_of(p, requests):
    return np.concatenate([np.arange(p.cu[b], p.cu[b + 1]) for b in requests]).astype(np.int64)


WAVES = [(8, 1, 256, [1] * 700, [20, 300] * 350, "bf16"), (16, 1, 64, [1] * 300, [40, 700, 90] * 100, "bf16"), (8, 2, 128, [1, 1, 2], [9001, 30, 3000], "bf16"),
         (8, 1, 256, [2, 2], [3000, 2000], "bf16"), (8, 1, 256, [70, 150, 90] * 40, [70, 150, 300] * 40, "bf16"), (8, 2, 128, [40, 60, 1], [2500, 90, 700], "bf16"),
         (4, 2, 128, [1] * 600, [48] * 600, "f32"), (8, 2, 128, [1, 2], [5000, 300], "f32"), (4, 1, 64, [30, 50], [300, 50], "f32")]


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens,dtype", WAVES)
def test_attention_of_requests_beside_bad_entries(Hq, Hkv, dh, q_lens, kv_lens, dtype):
    """In several waves of blocks, in key ranges, in units of pairs: their rows are what they are without, call after call; later calls write nothing."""
    p = Paged(89, q_lens, kv_lens, Hkv, dh, 16, dtype, layers=1)
    q, args = normal(p.rng, (p.T, Hq, dh), dtype).cuda(), p.device_args()
    want = p.cache.attend(0, q, *args)
    assert p.cache.poll_status() == 0
    for _ in range(10):
        table, bad = some_bad(p)
        good = rows_of(p, np.setdiff1d(np.arange(len(q_lens)), bad))
        out = torch.full_like(q, 5.0)
        p.cache.attend(0, q, *args[:2], ints(table), out=out)
        assert same(want[good], out[good])
        out.fill_(5.0)
        p.cache.attend(0, q, *args, out=out)
        assert (out == 5.0).all() and p.cache.poll_status() == binding.ERR_INVALID_ARG
    assert same(want, p.cache.attend(0, q, *args)) and p.cache.poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,dh,src,dst,q_lens,kv_lens", [
    (8, 1, 256, "bf16", "bf16", [1] * 700, [20, 300] * 350), (8, 2, 128, "f32", "bf16", [30, 90, 61] * 40, [30, 100, 200] * 40), (4, 1, 64, "f32", "f32", [17, 1], [17, 40])])
def test_append_of_requests_beside_bad_entries(Hq, Hkv, dh, src, dst, q_lens, kv_lens):
    p = Paged(90, q_lens, kv_lens, Hkv, dh, 16, dst, layers=1)
    q, k, v = (normal(p.rng, (p.T, h, dh), src).cuda() for h in (Hq, Hkv, Hkv))
    args, rope, before = p.device_args(), rope_table(400, dh).cuda(), p.cache.pages.clone()
    want = p.cache.append(0, k, v, *args, rope, q=q)
    after = p.cache.pages.clone()
    for _ in range(10):
        table, bad = some_bad(p)
        keep = np.setdiff1d(np.arange(len(q_lens)), bad)
        written = np.concatenate([P.slots(p.table[b], 16, kv_lens[b])[kv_lens[b] - q_lens[b]:] for b in keep])
        theirs = np.concatenate([P.slots(p.table[b], 16, kv_lens[b])[kv_lens[b] - q_lens[b]:] for b in bad])
        rest = np.setdiff1d(np.arange(before.shape[2]), np.concatenate([written, theirs]))
        p.cache.pages.copy_(before)
        got = p.cache.append(0, k, v, *args[:2], ints(table), rope, q=q)
        st = p.cache.status.item()                                      # (0: the bad entry is of a page without new tokens)
        assert st in (binding.OK, binding.ERR_INVALID_ARG)
        good = rows_of(p, keep)
        assert same(got[good], want[good]) and same(p.cache.pages[:, :, written].contiguous(), after[:, :, written].contiguous())
        assert same(p.cache.pages[:, :, rest].contiguous(), before[:, :, rest].contiguous())
        if st:
            now = p.cache.pages.clone()
            p.cache.append(0, v, k, *args, rope)
            assert same(now, p.cache.pages) and p.cache.poll_status() == st


@pytest.mark.parametrize("Hkv,dh,dtype,lens", [(1, 256, "bf16", [300, 20, 700] * 40), (2, 64, "f32", [40] * 300), (1, 64, "bf16", [40, 50])])
def test_pack_of_requests_beside_bad_entries(Hkv, dh, dtype, lens):
    p = Paged(91, [0] * len(lens), lens, Hkv, dh, 16, dtype, layers=3)
    kv, total = ints(lens), sum(lens)
    want, cu = p.cache.pack(ints(p.table), kv, total)
    assert p.cache.poll_status() == 0
    for _ in range(10):
        table, bad = some_bad(p)
        got, cu2 = p.cache.pack(ints(table), kv, total)
        assert torch.equal(cu, cu2)
        for b in np.setdiff1d(np.arange(len(lens)), bad):
            assert same(got[:, :, cu[b]:cu[b + 1]].contiguous(), want[:, :, cu[b]:cu[b + 1]].contiguous())
        out = torch.full_like(got, 5.0)
        p.cache.pack(ints(p.table), kv, total, out=out)                 # the word is up
        assert (out == 5.0).all() and p.cache.poll_status() == binding.ERR_INVALID_ARG


def test_words_raised_by_entries_and_captured_calls():
    """A replay goes by the word as any call does: raised by lengths or by another call it stops it, whatever the replay before met."""
    p = Paged(92, [1, 1], [60, 40], 1, 64, 16)
    q, (cu, lens, table) = normal(p.rng, (2, 4, 64)).cuda(), p.device_args()
    out = p.cache.attend(1, q, cu, lens, table)
    want, good = out.clone(), table.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.attend(1, q, cu, lens, table, out=out)
    table[1, 0] = -1
    graph.replay()
    assert torch.equal(out[0], want[0]) and p.cache.poll_status() == binding.ERR_INVALID_ARG
    table.copy_(good)
    for spoil in (lambda: p.cache.attend(1, q, cu, ints([60, -1]), table), lambda: p.cache.attend(1, q, cu, lens, torch.full_like(table, -1)),
                  lambda: p.cache.status.fill_(binding.ERR_TIMEOUT),
                  lambda: binding.norm_rope_heads(None, q, ints([0, 9]), rope_table(5, 64).cuda(), status=p.cache.status)):
        spoil()
        out.fill_(5.0)
        graph.replay()
        assert (out == 5.0).all() and p.cache.poll_status() != 0
        graph.replay()
        assert torch.equal(out, want) and p.cache.poll_status() == 0


@pytest.mark.parametrize("lens,room", [([40, -1], 90), ([40, 16 * 5], 200), ([40, 50], 89), ([2 ** 31 - 1, 50], 90), ([-2 ** 31, 50], 90)])
def test_pack_with_lengths_out_of_order_writes_nothing(lens, room):
    p = Paged(86, [0, 0], [40, 50], 1, 64, 16)                          # (a table of four pages and one entry more)
    p.table = p.table[:, :4]
    out, cu = torch.full((2, 2, room, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda"), ints([7, 7, 7])
    kv, table = ints(lens), ints(p.table)
    st = p.cache.lib.phyai_pack_paged_kv(p.cache._desc_ptr, 2, kv.data_ptr(), table.data_ptr(), 4, out.data_ptr(), room, cu.data_ptr(),
                                         p.cache.status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == binding.OK and p.cache.poll_status() == binding.ERR_INVALID_ARG
    assert (out == 9.0).all() and cu.tolist() == [7, 7, 7]


def test_poll_status_waits_for_calls_on_other_streams():
    p = Paged(85, [1, 2], [50, 40], 1, 64, 16)
    q, k, args = normal(p.rng, (p.T, 4, 64)).cuda(), normal(p.rng, (p.T, 1, 64)).cuda(), p.device_args()
    table = p.table.copy()
    table[:, :4] = -1
    bad, side = ints(table), torch.cuda.Stream()
    want = p.cache.attend(1, q, *args)
    for call in (lambda: p.cache.attend(1, q, *args[:2], bad, stream=side), lambda: p.cache.append(0, k, k, *args[:2], bad, None, stream=side),
                 lambda: p.cache.pack(bad, args[1], 90, stream=side)):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                               # about 10 ms ahead of the call
        call()
        assert p.cache.poll_status() == binding.ERR_INVALID_ARG
        got = p.cache.attend(1, q, *args, stream=side)                  # the word is down for any stream
        assert p.cache.poll_status() == 0 and torch.equal(want, got)


def test_poll_status_of_one_stream_does_not_wait_for_others():
    p = Paged(97, [1, 2], [50, 40], 1, 64, 16)
    q, args = normal(p.rng, (p.T, 4, 64)).cuda(), p.device_args()
    bad, side, other, done = torch.full_like(args[2], -1), torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Event()
    want = p.cache.attend(1, q, *args)
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        torch.cuda._sleep(1_000_000_000)                                # half a second
        done.record()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    p.cache.attend(1, q, *args[:2], bad, stream=side)
    assert p.cache.poll_status(side) == binding.ERR_INVALID_ARG and not done.query()
    got = p.cache.attend(1, q, *args)                                   # the word is down for any stream
    assert p.cache.poll_status() == 0 and done.query() and torch.equal(want, got)
    with pytest.raises(ValueError):
        p.cache.poll_status(types.SimpleNamespace(device=torch.device("cuda", 1)))


# ------------------------------------------------------------------------------------------------------------------
# waits that run out (the data that they wait for does arrive: nothing hangs)
# ------------------------------------------------------------------------------------------------------------------
def expired(p, q, args, want, sure=True):
    """``sure``: a wait does expire (with a tile or two for each warp all copies may have come by the second poll: the call is good then)."""
    out = torch.full_like(q, 5.0)
    torch.full((1 << 28,), 0, dtype=torch.uint8, device="cuda")         # keys and values come from memory
    binding.set_paged_option("wait_limit", 1)
    try:
        p.cache.attend(1, q, *args, out=out)
        torch.cuda.synchronize()
    finally:
        binding.set_paged_option("wait_limit", 1 << 22)
    status = p.cache.status.item()
    assert status == binding.ERR_TIMEOUT or not sure and status == binding.OK and same(want, out)
    p.cache.status.fill_(binding.ERR_TIMEOUT)
    out.fill_(5.0)
    p.cache.attend(1, q, *args, out=out)                                # the word is up: nothing is written
    assert (out == 5.0).all() and p.cache.poll_status() == binding.ERR_TIMEOUT and p.cache.poll_status() == 0
    assert same(want, p.cache.attend(1, q, *args)) and p.cache.poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (8, 1, 256, [1], [969]), (8, 1, 256, [1] * 300, [200] * 300),       # a cluster of eight; blocks of their own
    (8, 2, 128, [1, 1], [9001, 3000]), (4, 1, 64, [2] * 3, [4100, 17, 300]),       # key ranges
    (8, 1, 256, [2], [3000]), (16, 1, 128, [1] * 80, [500] * 80),       # 16 rows
    (4, 1, 64, [1] * 300, [2000] * 300),                                # thirty tiles a warp
])
def test_expired_waits_of_few_rows(Hq, Hkv, dh, q_lens, kv_lens):
    p = Paged(83, q_lens, kv_lens, Hkv, dh, 64)
    q, args = normal(p.rng, (p.T, Hq, dh)).cuda(), p.device_args()
    want = p.cache.attend(1, q, *args)
    assert p.cache.poll_status() == 0
    expired(p, q, args, want, sure=sum(kv_lens) > 500000)


@pytest.mark.parametrize("hidden", [False, True])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (8, 1, 256, [64, 33], [5000, 33]), (8, 2, 128, [40] * 6, [6000, 300, 40, 2000, 100, 77]), (4, 4, 64, [90, 1, 0, 17], [3000, 4000, 10, 17]),   # split units
    (8, 1, 256, [300] * 9, [300] * 9), (8, 1, 128, [600] * 5, [600] * 5), (4, 1, 64, [700, 90], [700, 1000]),                                    # whole ones
])
def test_expired_waits_of_many_rows(Hq, Hkv, dh, q_lens, kv_lens, hidden):
    """``hidden``: with values that some rows do not see and that make these look once more, behind the last unit."""
    p = Paged(84, q_lens, kv_lens, Hkv, dh, 32)
    if hidden:
        for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
            if n:
                p.cache.pages[1, 1, P.slots(p.table[b], 32, kv)[-(n // 2 + 1):]] = float("inf")
    q, args = normal(p.rng, (p.T, Hq, dh)).cuda(), p.device_args()
    want = p.cache.attend(1, q, *args)
    assert p.cache.poll_status() == 0
    expired(p, q, args, want)


# ------------------------------------------------------------------------------------------------------------------
# infinities and NaN among the keys that a row does see
# ------------------------------------------------------------------------------------------------------------------
FORMS = [(8, 1, 256, [1], [40], "bf16"), (8, 1, 256, [1] * 300, [20] * 300, "bf16"), (8, 2, 128, [1, 2], [9001, 30], "bf16"), (8, 1, 256, [2], [3000], "bf16"),
         (8, 1, 128, [64, 3], [64, 200], "bf16"), (8, 1, 256, [40], [2500], "bf16"), (4, 1, 64, [700], [700], "bf16"),
         (4, 1, 64, [1, 3], [50, 20], "f32"), (8, 2, 128, [1], [5000], "f32"), (4, 1, 64, [40], [300], "f32")]


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens,dtype", FORMS)
def test_rows_all_of_whose_logits_are_minus_infinity(Hq, Hkv, dh, q_lens, kv_lens, dtype):
    """0 / 0 is NaN, as in the formula; zero is the result of a row that sees no key.  The queries' first channel is 1, and the keys' -infinity in all keys of
    the last request but its last one: rows that see that key have a finite logit."""
    p = Paged(87, q_lens, kv_lens, Hkv, dh, 16, dtype)
    b = len(kv_lens) - 1
    p.cache.pages[1, 0, P.slots(p.table[b], 16, kv_lens[b])[:-1], :, 0] = -float("inf")
    q = normal(p.rng, (p.T, Hq, dh), dtype).cuda()
    q[:, :, 0] = 1.0
    args = p.device_args()
    got = p.cache.attend(1, q, *args)
    assert p.cache.poll_status() == 0
    planes = f64(p.cache.pages[1])
    ref = P.attend(f64(q), planes[0], planes[1], p.cu, kv_lens, p.table, 16, True)
    blind = np.arange(int(p.cu[b]), int(p.cu[b + 1]) - 1)               # rows of the last request that do not see its last key
    rest = np.setdiff1d(np.arange(p.T), blind)
    assert torch.isnan(got[blind]).all() and np.isnan(ref[0][blind]).all()
    ref[2][rest] = np.nan_to_num(ref[2][rest], posinf=float(dh))        # (the sums |q k| of finite logits are below that)
    check_attention(f64(got)[rest], [r[rest] for r in ref], dtype, dh, max(kv_lens))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens,dtype", FORMS)
def test_every_row_that_sees_nan_or_infinite_logits_is_nan(value, Hq, Hkv, dh, q_lens, kv_lens, dtype):
    p = Paged(88, q_lens, kv_lens, Hkv, dh, 16, dtype)
    b = len(kv_lens) - 1
    first = kv_lens[b] - (q_lens[b] + 1) // 2                           # a key that the newer rows of the last request see
    p.cache.pages[1, 0, P.slots(p.table[b], 16, kv_lens[b])[first]] = value
    q = normal(p.rng, (p.T, Hq, dh), dtype).abs().cuda() + 0.25         # (positive: the logits are +infinity, not of either sign)
    got = p.cache.attend(1, q, *p.device_args())
    assert p.cache.poll_status() == 0
    sees = np.arange(int(p.cu[b + 1]) - (q_lens[b] + 1) // 2, int(p.cu[b + 1]))
    assert torch.isnan(got[sees]).all() and torch.isfinite(got[np.setdiff1d(np.arange(p.T), sees)]).all()


# ------------------------------------------------------------------------------------------------------------------
# the kernels' forms for many units, many rows and long ranges, on picked rows
# ------------------------------------------------------------------------------------------------------------------
def run_picked(p, Hq, mask, every):
    """Against the oracle on every ``every``-th token of a request, and its first and last: each as a request of one token over the keys that it sees."""
    prefix = [n * 2 // 3 for n in p.kv_lens] if mask == "prefix" else None
    q, args = normal(p.rng, (p.T, Hq, p.dh), p.dtype).cuda(), p.device_args()
    out = torch.full_like(q, 777.0)
    p.cache.attend(1, q, *args, causal=mask != "full", prefix_lens=None if prefix is None else ints(prefix), out=out)
    assert p.cache.poll_status() == 0
    live = np.arange(int(p.cu[0]), int(p.cu[-1]))
    assert (out[np.setdiff1d(np.arange(p.T), live)] == 777.0).all()
    tokens, seen, table = [], [], []
    for b, (n, kv) in enumerate(zip(p.q_lens, p.kv_lens)):
        lim = P.limits(n, kv, mask != "full", 0 if prefix is None else prefix[b])
        for i in sorted((set(range(b % every, n, every)) | {0, n - 1}) & set(range(n))):
            tokens.append(int(p.cu[b]) + i), seen.append(int(lim[i])), table.append(p.table[b])
    planes = f64(p.cache.pages[1])
    ref = P.attend(f64(q[tokens]), planes[0], planes[1], np.arange(len(tokens) + 1), seen, table, p.page, False)
    check_attention(f64(out)[tokens], ref, p.dtype, p.dh, max(p.kv_lens))


@pytest.mark.parametrize("mask", ["causal", "full", "prefix"])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,past,page", [
    (8, 1, 256, [968, 900, 701, 611, 968, 33, 850, 777], 0, 64),        # 187 units of 32 tokens: three rounds of 74 pairs
    (8, 1, 256, [1500, 40, 1, 900], 333, 16),
    (8, 2, 128, [700, 650, 512, 801, 90, 700, 333, 700], 0, 32),        # 146 units of 64 tokens and a kv head
    (32, 8, 128, [300, 411, 65], 200, 128),
    (16, 1, 64, [400, 390, 411, 17, 400, 512, 300, 399], 50, 256),      # 179 units of 16 tokens
])
def test_attention_of_more_units_than_pairs(Hq, Hkv, dh, q_lens, past, page, mask):
    p = Paged(93, q_lens, [n + past * (i % 3) for i, n in enumerate(q_lens)], Hkv, dh, page, first_row=3, last_rows=2)
    run_picked(p, Hq, mask, 29)


@pytest.mark.parametrize("mask", ["causal", "full", "prefix"])
@pytest.mark.parametrize("Hq,Hkv,dh", [(8, 8, 64), (12, 4, 64), (8, 8, 128), (8, 8, 256), (16, 2, 256)])
def test_attention_fp32_of_many_rows(Hq, Hkv, dh, mask):
    """Tiles of 64 rows: as many of them as there are SMs."""
    q_lens = [700, 1, 0, 556]
    assert sum(q_lens) * (Hq // Hkv) // 64 * Hkv >= 148
    run_picked(Paged(94, q_lens, [900, 300, 5, 556], Hkv, dh, 32, "f32", first_row=1, last_rows=1), Hq, mask, 23)


@pytest.mark.parametrize("mask", ["causal", "full", "prefix"])
@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens", [
    (8, 1, 256, [2], [9000]), (8, 1, 256, [2, 1], [5000, 7777]), (16, 1, 128, [1], [6001]), (8, 1, 64, [2, 2, 1], [8192, 17, 5000]),     # clusters of eight, ranges
    (8, 2, 128, [4, 3], [5003, 9000]), (8, 1, 256, [2] * 20, [1100 + 37 * i for i in range(20)]), (16, 1, 64, [1] * 12, [4096] * 12),    # of eight, of one range
    (8, 1, 256, [2] * 50, [700 + i for i in range(50)]), (16, 2, 128, [2] * 60, [600] * 60), (8, 1, 64, [2, 1] * 160, [300, 290] * 160),   # of four, two, one
])
def test_attention_of_nine_to_sixteen_rows(Hq, Hkv, dh, q_lens, kv_lens, mask):
    run_picked(Paged(95, q_lens, kv_lens, Hkv, dh, 64, first_row=1, last_rows=2), Hq, mask, 1)


@pytest.mark.parametrize("Hq,Hkv,dh,q_lens,kv_lens,dtype", [
    (8, 1, 256, [1] * 64, [32768] + [600 + 5 * i for i in range(63)], "bf16"), (8, 2, 128, [1] * 63 + [65], [900] * 63 + [2000], "bf16"),
    (8, 1, 256, [1] * 30 + [300], [700] * 30 + [900], "bf16"), (4, 1, 128, [1] * 20 + [100], [300] * 20 + [400], "f32"),
])
def test_attention_of_requests_of_very_different_lengths(Hq, Hkv, dh, q_lens, kv_lens, dtype):
    """One long history among short ones; a chunk among single tokens."""
    run_picked(Paged(96, q_lens, kv_lens, Hkv, dh, 64, dtype), Hq, "causal", 13)


# ------------------------------------------------------------------------------------------------------------------
# captured calls
# ------------------------------------------------------------------------------------------------------------------
FIRST = """
import sys, torch
from paper_2608_03682_b200 import binding
ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
pages, k, q = (torch.ones(s, device="cuda").bfloat16() for s in ((1, 2, 64, 1, 64), (4, 1, 64), (4, 4, 64)))
cu, lens, table, pos, status, cache = ints([0, 4]), ints([20]), ints([[0, 1]]), ints([0, 1, 2, 3]), ints([0]), binding.PagedCache(pages, 16)
rope = torch.zeros(10, 32, 2, device="cuda")
calls = dict(heads=lambda: binding.norm_rope_heads(q, k, pos, rope, status=status)[1], append=lambda: cache.append(0, k, k, cu, lens, table, None, q=q),
             attend=lambda: cache.attend(0, q, cu, lens, table), pack=lambda: cache.pack(table, lens, 20)[0])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = calls[sys.argv[1]]()
graph.replay()
assert cache.poll_status() == 0 and int(status) == 0 and bool((out == (sys.argv[1] != "heads")).all())
"""


@pytest.mark.parametrize("call", ["heads", "append", "attend", "pack"])
def test_the_first_call_of_a_process_may_be_captured(call):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST, call], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_heads_without_a_word_in_a_graph_and_out_of_it():
    """The first such call of a device in a capture, replayed, and calls out of it, with positions outside the table."""
    binding._unread_words.clear()
    rng = np.random.default_rng(98)
    k, table = normal(rng, (40, 2, 64)).cuda(), rope_table(50, 64)
    positions, rope = rng.integers(0, 50, 40), table.cuda()
    positions[7] = 50
    pos, good = ints(positions), np.setdiff1d(np.arange(40), [7])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first, second = (binding.norm_rope_heads(None, k, pos, rope)[1] for _ in range(2))
    for _ in range(3):
        graph.replay()
        third = binding.norm_rope_heads(None, k, pos, rope)[1]
        for y in (first, second, third):
            assert torch.isnan(y[7]).all()
            check_heads(y[good], k[good], None, table, positions[good], "bf16")
