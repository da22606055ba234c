"""The serving calls on the GPU against their fp64 oracle.

Tolerances (a bf16 rounding is off by at most 2^-8 of the value).
Norm and rotation: one rounding of the result, 2^-8 |r|; in front of it some twenty fp32 roundings of the two products a result
is the difference of, 32 * 2^-24 of their sizes.
Decode: the result's rounding, 2^-8 |o|; the probabilities, 2^-16 sum(p |v|); fp32 scores of at most |q||k| scale ~ 40 summed
over 128 products are off by about 1e-5 and their exponentials by as much, 1e-4 of sum(p |v|) covers both and the fp32 sums.  lse: 1e-4 for the same reason."""
import os
import subprocess
import sys
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2609_20971_b200 import (PagedCache, PagedStep, RbsError, alloc_step, paged_decode_workspace_bytes, rbs_device_status, rbs_paged_decode,
                                   rbs_paged_extend, rbs_qk_norm_rope, rbs_qk_norm_rope_paged, rope_frequencies)
from paper_2609_20971_b200.binding import rbs_prefill_varlen

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _randn(seed, *shape, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ extend


def _extend_case(seed, seqs, page, most, old, new, n_free, n_pages, tokens, used):
    g = np.random.default_rng(seed)
    lens = g.integers(old[0], old[1] + 1, seqs)
    table = g.integers(-2, n_pages + 1, (seqs, most))
    return lens, g.integers(new[0], new[1] + 1, seqs), table, g.permutation(max(n_free, n_pages))[:n_free], used, page, n_pages, tokens


EXTENDS = [
    (1, 1, 16, 4, (0, 0), (1, 1), 8, 50, 1, None),              # the first token of a sequence
    (2, 64, 64, 20, (0, 1000), (1, 1), 200, 2000, 64, 3),       # a decode step
    (3, 7, 1, 40, (0, 9), (0, 25), 300, 400, 200, 0),           # pages of one token
    (4, 33, 24, 9, (0, 200), (0, 60), 30, 500, 700, 11),        # pool and rows run out, tokens behind the end of the table
    (5, 1500, 16, 6, (0, 90), (0, 40), 3000, 4000, 40000, 7),   # more sequences than threads
    (6, 8192, 256, 3, (-5, 700), (-3, 2), 9000, 9000, 9000, 1),  # the most there may be, negative lengths
    (7, 3, 128, 300, (0, 0), (20000, 38400), 900, 901, 100000, None),
    (8, 5, 16, 4, (0, 60), (0, 0), 0, 10, 0, None),             # nothing new
    (9, 5, 16, 4, (0, 60), (0, 9), 0, 10, 37, None),            # no free page at all
]


@pytest.mark.parametrize("seed, seqs, page, most, old, new, n_free, n_pages, tokens, used", EXTENDS)
@pytest.mark.parametrize("wide", [0, 5])
def test_extend_equals_the_oracle(seed, seqs, page, most, old, new, n_free, n_pages, tokens, used, wide):
    lens, add, table, free, used, page, n_pages, tokens = _extend_case(seed, seqs, page, most, old, new, n_free, n_pages, tokens, used)
    want = so.extend(lens, add, table, free, page, n_pages, tokens, used or 0)
    whole = torch.full((seqs, most + wide), 77, dtype=torch.int32, device="cuda")
    rows = whole[:, :most]
    rows.copy_(_ints(table))
    out = alloc_step(seqs, tokens, "cuda")
    for t in (out.lens, out.cu, out.positions, out.slots, out.used):
        t.fill_(-99)
    args = (_ints(lens), _ints(add), rows, _ints(free), page, n_pages, tokens)
    for _ in range(2):      # the same again when repeated
        rbs_paged_extend(*args, free_used=None if used is None else _ints([used]), out=out)
        got = [x.cpu().numpy() for x in (rows, out.lens, out.cu, out.positions, out.slots)]
        for name, x, y in zip(("table", "lens", "cu", "positions", "slots"), got, want):
            assert np.array_equal(x, y), name
        assert out.used.item() == want[5]
    assert bool((whole[:, most:] == 77).all())


def _many_rows(seed, page, rows, pool):
    """Zeros and lengths of 1 to 3 beside long ones, 200,000 to 260,000 tokens; `rows` more rows than tokens, `pool` more pages than needed."""
    g = np.random.default_rng(seed)
    seqs = 700
    add = np.where(g.random(seqs) < 0.03, g.integers(8000, 13000, seqs), g.integers(0, 4, seqs))
    add[:5], add[100:110], add[-3:] = 0, 0, 0
    add[300] += 210000 - add.sum() if add.sum() < 210000 else 0
    lens = g.integers(0, 3 * page + 2, seqs)
    most = int((-(-(lens + add) // page)).max()) + 1
    need = int((-(-(lens + add) // page) + -lens // page).sum())
    n_pages = int((-(-lens // page)).sum()) + need + 10
    return lens, add, g.integers(0, n_pages, (seqs, most)), g.permutation(n_pages)[:need + pool], 0, page, n_pages, int(add.sum()) + rows


MANY_ROWS = [(1, 1, 0, 5), (2, 16, 1, 5), (3, 24, 6, 5), (4, 16, -20000, 5), (5, 24, 3, -700), (6, 1, -3333, -100000)]


@pytest.mark.parametrize("seed, page, rows, pool", MANY_ROWS)
@pytest.mark.parametrize("offset", [0, 1])      # outputs that take 16-byte stores, and that do not
def test_extend_of_many_rows_equals_the_oracle(seed, page, rows, pool, offset):
    lens, add, table, free, used, page, n_pages, tokens = _many_rows(seed, page, rows, pool)
    assert tokens > 1024 * torch.cuda.get_device_properties(0).multi_processor_count
    want = so.extend(lens, add, table, free, page, n_pages, tokens, used)
    whole = [torch.full((n + 9,), -99, dtype=torch.int32, device="cuda") for n in (len(lens), len(lens) + 1, tokens, tokens, 1)]
    out = PagedStep(*(t[offset:t.shape[0] - 9 + offset] for t in whole))
    rows = _ints(table)
    rbs_paged_extend(_ints(lens), _ints(add), rows, _ints(free), page, n_pages, tokens, free_used=_ints([used]), out=out)
    for x, y in zip((rows, out.lens, out.cu, out.positions, out.slots), want):
        assert np.array_equal(x.cpu().numpy(), y)
    assert out.used.item() == want[5]
    assert all(bool((t[:offset] == -99).all() and (t[t.shape[0] - 9 + offset:] == -99).all()) for t in whole)


@pytest.mark.parametrize("lens, add, page, most", [
    ([2147482640, 0], [10, 1], 1000, 2147483),                            # a length within a page of 2^31
    ([1000000000, 0, 1499999998], [5, 3, 4], 1500000000, 1),              # pages of more than 2^30 tokens
    ([(1 << 30) + 3, 1 << 30, 0, 5], [4, 1, 0, 2], (1 << 30) + 1, 1)])
def test_extend_of_lengths_and_page_sizes_near_31_bits(lens, add, page, most):
    tokens, n_pages = sum(add) + 2, 0x7fffffff // page
    table = np.full((len(lens), most), -1)
    for s, n in enumerate(lens):
        table[s, :-(-n // page)] = n_pages - 1
    free = [0] * 3
    want = so.extend(lens, add, table, free, page, n_pages, tokens)
    whole = torch.full((3 * len(lens), most), 77, dtype=torch.int32, device="cuda")      # the table, and as much in front of it and behind
    rows = whole[len(lens):2 * len(lens)]
    rows.copy_(_ints(table))
    out = rbs_paged_extend(_ints(lens), _ints(add), rows, _ints(free), page, n_pages, tokens)
    for x, y in zip((rows, out.lens, out.cu, out.positions, out.slots), want):
        assert np.array_equal(x.cpu().numpy(), y)
    assert out.used.item() == want[5]
    assert bool((whole[:len(lens)] == 77).all() and (whole[2 * len(lens):] == 77).all())


def test_extend_into_the_most_rows_there_may_be():
    """2^31 - 3 rows: the four of the last 16-byte store would end at row 2^31.  Rows behind the last are watched."""
    n = (1 << 31) - 3
    step = alloc_step(1, 0, "cuda")
    step.positions, step.slots = (torch.full((n + 3,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    whole = step.positions, step.slots
    step.positions, step.slots = (t[:n] for t in whole)
    rbs_paged_extend(_ints([0]), _ints([1]), _ints([[-1]]), _ints([0]), 1, 1, n, out=step)
    assert step.lens.item() == 1 and step.cu.tolist() == [0, 1] and step.slots[0].item() == 0
    assert whole[0][n:].tolist() == [7] * 3 and whole[1][n:].tolist() == [7] * 3
    for part in range(0, n, 1 << 28):
        assert not bool(step.positions[part:part + (1 << 28)].any()) and bool((step.slots[max(part, 1):part + (1 << 28)] == -1).all())


def test_extend_step_after_step_hands_out_every_page_once():
    page, n_pages, seqs = 16, 61, 6
    g = np.random.default_rng(3)
    table = torch.full((seqs, 30), -1, dtype=torch.int32, device="cuda")
    free = _ints(g.permutation(n_pages))
    lens, used, seen = _ints([0] * seqs), _ints([0]), []
    for _ in range(12):
        new = g.integers(0, 19, seqs)
        step = rbs_paged_extend(lens, _ints(new), table, free, page, n_pages, int(new.sum()) + 2, free_used=used)
        lens, used = step.lens, step.used
        seen += step.slots[:int(new.sum())].tolist()
    assert min(seen) >= 0 and len(set(seen)) == len(seen) == int(lens.sum())


# ------------------------------------------------------------------------------------------------ norm and rotation


def _frequencies(rot, base=1e6):
    return torch.tensor(base ** (-np.arange(0, rot, 2) / max(rot, 1)), dtype=torch.float32, device="cuda")


def _check_turn(got, x, positions, freq, weight, **more):
    want, size = so.norm_rope(_f64(x), positions.cpu().numpy(), [] if freq is None else _f64(freq), None if weight is None else _f64(weight), **more)
    err = np.abs(_f64(got) - want)
    assert (err <= STEP * np.abs(want) + 32 * 2.0 ** -24 * size).all(), float((err / (np.abs(want) + 1e-30)).max())


# of the many tokens each with another number of warps to a token, and a last thread block with fewer tokens than the others
@pytest.mark.parametrize("tokens, hq, hkv", [(1, 1, 1), (1, 32, 4), (3, 3, 1), (61, 40, 8), (257, 16, 16), (1003, 8, 2), (1501, 5, 1), (5003, 3, 2)])
@pytest.mark.parametrize("rot, interleaved, norm", [(128, False, True), (128, True, True), (64, False, False), (64, True, True), (96, False, True),
                                                    (8, True, False), (8, False, True), (0, False, True)])
def test_norm_rope_equals_the_oracle(tokens, hq, hkv, rot, interleaved, norm):
    x = _randn(tokens + rot, tokens, hq + 2 * hkv, 128, scale=3.0)      # slices of a fused projection
    q, k, _ = x.split((hq, hkv, hkv), dim=1)
    g = torch.Generator(device="cuda").manual_seed(rot)
    pos = torch.randint(-50, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    freq = None if rot == 0 else _frequencies(rot)
    wq, wk = (torch.randn(128, generator=g, device="cuda") for _ in range(2)) if norm else (None, None)
    before = x.clone()
    oq, ok = rbs_qk_norm_rope(q, k, pos, freq, q_norm=wq, k_norm=wk, eps=1e-5, interleaved=interleaved, magnitude=1.25)
    more = {"eps": 1e-5, "interleaved": interleaved, "magnitude": 1.25}
    _check_turn(oq, q, pos, freq, wq, **more)
    _check_turn(ok, k, pos, freq, wk, **more)
    assert torch.equal(x, before)


def test_norm_rope_of_a_batch_in_place_and_with_one_norm_only():
    q, k = _randn(1, 3, 77, 6, 128), _randn(2, 3, 77, 2, 128)
    pos, freq, w = torch.arange(77, dtype=torch.int32, device="cuda"), _frequencies(128), torch.randn(128, device="cuda")
    q0, k0 = q.clone(), k.clone()
    apart = rbs_qk_norm_rope(q, k, pos, freq, k_norm=w)
    oq, ok = rbs_qk_norm_rope(q, k, pos, freq, k_norm=w, out_q=q, out_k=k)
    assert oq is q and ok is k and torch.equal(apart[0], q) and torch.equal(apart[1], k)
    _check_turn(q, q0, pos, freq, None)
    _check_turn(k, k0, pos, freq, w)


# 2, 4 and 8 tokens to a thread block, blocks that begin in one entry of the batch and end in another one or in the fourth
@pytest.mark.parametrize("batch, tokens, hq, hkv", [(3, 301, 3, 1), (5, 401, 2, 1), (7, 701, 4, 2), (1000, 3, 2, 1), (2600, 1, 1, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_of_large_batches_equals_the_oracle(batch, tokens, hq, hkv, interleaved):
    x = _randn(batch, tokens, batch, hq + hkv, 128, scale=2.0).transpose(0, 1)      # the batch is not the slowest dimension
    q, k = x.split((hq, hkv), dim=2)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    pos = torch.randint(0, 1 << 18, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    freq, w = _frequencies(96), torch.randn(128, generator=g, device="cuda")
    oq, ok = rbs_qk_norm_rope(q, k, pos, freq, q_norm=w, eps=1e-5, interleaved=interleaved)
    _check_turn(oq, q, pos, freq, w, eps=1e-5, interleaved=interleaved)
    _check_turn(ok, k, pos, freq, None, interleaved=interleaved)


def test_angles_of_far_positions_are_exact():
    """At position 2^31 - 1 an angle rounded to fp32 would be off by tens of radians."""
    q = _randn(5, 6, 2, 128)
    pos = _ints([0, 1, (1 << 24) + 1, 123456789, (1 << 31) - 1, -(1 << 31)])
    freq = _frequencies(128, 10000.0)
    oq, _ = rbs_qk_norm_rope(q, q, pos, freq)
    # the oracle's own angle, rounded to fp64, is off by up to 2^31 * 2^-53 = 2.4e-7: added to the 32 roundings of 6e-8
    want, size = so.norm_rope(_f64(q), pos.cpu().numpy(), _f64(freq))
    assert (np.abs(_f64(oq) - want) <= STEP * np.abs(want) + 40 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_any_frequency_and_position(interleaved):
    """Frequencies from 1e-6 to 2^40 of either sign, the angle in exact fractions with 60 digits of pi.  One element of each pair cancels to
    less than 2^-12 of its two products, so that the result's rounding, 2^-20 of them, leaves the angle's error in sight.
    Of their size, in 2^-24: angle 2^-25.9 revolutions 1.7, sine and cosine 2, magnitude 1, two products 2."""
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494")
    freq = torch.tensor(np.geomspace(1e-6, 2.0 ** 40, 64) * (-1) ** (np.arange(64) // 5), dtype=torch.float32)
    pos = [1, -1000, (1 << 24) + 1, 123456789, (1 << 31) - 1, -(1 << 31)]
    turn = np.array([[float((p * Fraction(f) / (2 * pi)) % 1) for f in freq.tolist()] for p in pos])
    cos, sin = np.cos(2 * np.pi * turn), np.sin(2 * np.pi * turn)
    other = np.arange(128, 256)[:, None, None] / 128.0                     # every bf16 number of [1, 2) for v, and u beside it
    u = torch.tensor(other * sin / cos).to(torch.bfloat16).double().numpy()
    best = np.abs(u * cos / (other * sin) - 1).argmin(0)[None]
    u, v = np.take_along_axis(u, best, 0)[0], other[best[0], 0, 0]
    x = np.stack((u, v), -1 if interleaved else -2).reshape(len(pos), 1, 128)
    q = torch.tensor(x, device="cuda").to(torch.bfloat16)
    got = _f64(rbs_qk_norm_rope(q, q, _ints(pos), freq.cuda(), interleaved=interleaved)[0])
    pairs = got.reshape(len(pos), 64, 2).transpose(2, 0, 1) if interleaved else got.reshape(len(pos), 2, 64).transpose(1, 0, 2)
    for y, want in zip(pairs, (u * cos - v * sin, v * cos + u * sin)):
        size = np.abs(u) + np.abs(v)
        assert (np.abs(y - want) <= STEP * np.abs(want) + 8 * 2.0 ** -24 * size).all()
    assert (np.abs(u * cos - v * sin) < 2.0 ** -12 * (np.abs(u) + np.abs(v))).all()


def test_frequencies_that_are_no_numbers_give_no_numbers():
    q, pos, freq = _randn(8, 5, 2, 128), torch.arange(5, dtype=torch.int32, device="cuda"), _frequencies(128)
    clean, _ = rbs_qk_norm_rope(q, q, pos, freq)
    freq[3], freq[10], freq[40] = float("inf"), float("nan"), -float("inf")
    got, _ = rbs_qk_norm_rope(q, q, pos, freq)
    bad = torch.tensor([i + 64 * j for i in (3, 10, 40) for j in (0, 1)], device="cuda")
    assert bool(got[..., bad].isnan().all())
    got[..., bad] = clean[..., bad]
    assert torch.equal(got, clean)


def test_norm_of_zeros_and_of_small_and_large_rows():
    q = _randn(7, 6, 2, 128)
    for row, scale in enumerate((0.0, 1e-12, 1e-18, 1e12, 3e17)):
        q[row] *= scale
    pos, w = torch.arange(6, dtype=torch.int32, device="cuda"), torch.rand(128, device="cuda") + 0.5
    for eps in (1e-6, 0.0):
        oq, _ = rbs_qk_norm_rope(q, q, pos, _frequencies(128), q_norm=w, k_norm=w, eps=eps)
        # the smallest normal number in place of a zero eps: the mean square of the smallest row here is 1e-36
        _check_turn(oq, q, pos, _frequencies(128), w, eps=max(eps, 2.0 ** -126))


def test_norm_rope_keeps_nan_and_infinity_in_their_rows():
    q = _randn(6, 5, 3, 128)
    q[1, 2, 7], q[3, 0, 100] = float("nan"), float("inf")
    pos, w = torch.arange(5, dtype=torch.int32, device="cuda"), torch.ones(128, device="cuda")
    clean = q.clone()
    clean[1, 2], clean[3, 0] = 1.0, 1.0
    a, b = (rbs_qk_norm_rope(x, x, pos, _frequencies(128), q_norm=w, k_norm=w)[0] for x in (q, clean))
    assert a[1, 2].isnan().all() and not a[3, 0].isfinite().all()
    a[1, 2], a[3, 0] = b[1, 2], b[3, 0]
    assert torch.equal(a, b)


def _cache(seed, pages, page, hkv, order):
    shape = (pages, page, hkv, 128) if order == "token" else (pages, hkv, page, 128)
    k, v = _randn(seed, *shape), _randn(seed + 1, *shape)
    return (k, v) if order == "token" else (k.transpose(1, 2), v.transpose(1, 2))


@pytest.mark.parametrize("tokens, hq, hkv, page, order", [(1, 32, 4, 64, "token"), (48, 32, 4, 16, "head"), (3, 3, 1, 1, "token"), (129, 40, 8, 24, "token"),
                                                          (700, 16, 16, 256, "head"), (1501, 6, 3, 64, "token"), (5003, 8, 2, 16, "head")])
@pytest.mark.parametrize("keep_k", [False, True])
def test_norm_rope_paged_writes_its_slots_and_nothing_else(tokens, hq, hkv, page, order, keep_k):
    pages = tokens // page + 3
    x = _randn(tokens, tokens, hq + 2 * hkv, 128, scale=2.0)
    q, k, v = x.split((hq, hkv, hkv), dim=1)
    kc, vc = _cache(7, pages, page, hkv, order)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].int()
    slots[1::5] = -1                      # rows of a padded batch
    slots[2::7] = pages * page + 5        # and of a cache that is smaller than its user thinks
    pos = torch.randint(0, 40000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    freq, w = _frequencies(128), torch.randn(128, generator=g, device="cuda")
    k_before, v_before = kc.clone(), vc.clone()
    out_k = torch.empty(tokens, hkv, 128, dtype=torch.bfloat16, device="cuda") if keep_k else None
    oq = rbs_qk_norm_rope_paged(q, k, v, pos, slots, freq, kc, vc, q_norm=w, k_norm=w, out_k=out_k)
    want_q, want_k = rbs_qk_norm_rope(q, k, pos, freq, q_norm=w, k_norm=w)      # its own test compares it with the oracle
    assert torch.equal(oq, want_q) and (out_k is None or torch.equal(out_k, want_k))
    good = ((slots >= 0) & (slots < pages * page)).nonzero()[:, 0]
    at = slots[good].long()
    k_before[at // page, at % page], v_before[at // page, at % page] = want_k[good], v[good]
    assert torch.equal(kc, k_before) and torch.equal(vc, v_before)


def test_norm_rope_paged_of_a_padded_batch_with_fewer_slots_than_tokens():
    q, k, v, kc = _randn(1, 9, 8, 128), _randn(2, 9, 2, 128), _randn(3, 9, 2, 128), torch.zeros(2, 8, 2, 128, dtype=torch.bfloat16, device="cuda")
    vc, pos, freq = torch.zeros_like(kc), torch.arange(9, dtype=torch.int32, device="cuda"), _frequencies(128)
    for slots in (_ints([5, 9, 2]), _ints([])):
        kc.zero_(), vc.zero_()
        oq = rbs_qk_norm_rope_paged(q, k, v, pos, slots, freq, kc, vc)
        want_q, want_k = rbs_qk_norm_rope(q, k, pos, freq)
        n, at = slots.numel(), slots.long()
        want_kc, want_vc = torch.zeros_like(kc), torch.zeros_like(vc)
        want_kc[at // 8, at % 8], want_vc[at // 8, at % 8] = want_k[:n], v[:n]
        assert torch.equal(oq, want_q) and torch.equal(kc, want_kc) and torch.equal(vc, want_vc)


# ------------------------------------------------------------------------------------------------ decode


def _sequences(seed, lens, page, hkv, order="token", spare=2):
    """A cache in which every element that belongs to no sequence is NaN, and the table: entries behind a sequence are far out of range."""
    g = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    perm = g.permutation(pages)
    table = np.full((len(lens), max(max(need), 1) + 1), 1 << 30)
    k, v = _cache(seed, pages, page, hkv, order)
    mine = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    at = 0
    for s, n in enumerate(lens):
        table[s, :need[s]] = perm[at:at + need[s]]
        at += need[s]
        t = np.arange(n)
        mine[torch.tensor(table[s, t // page], device="cuda").long(), torch.tensor(t % page, device="cuda").long()] = True
    k[~mine], v[~mine] = float("nan"), float("nan")
    return k, v, _ints(table), _ints(lens)


def _check_decode(out, lse, q, k, v, table, lens, scale=None):
    o, l, size = so.decode(_f64(q), _f64(k), _f64(v), table.cpu().numpy(), lens.cpu().numpy(), scale)
    err = np.abs(_f64(out) - o)
    assert (err <= STEP * np.abs(o) + (2.0 ** -16 + 1e-4) * size).all(), float((err - STEP * np.abs(o)).max())
    got = _f64(lse)
    assert np.array_equal(np.isinf(got), np.isinf(l))
    fine = np.isfinite(l)
    assert np.abs(got[fine] - l[fine]).max(initial=0.0) <= 1e-4


LENS = [1, 0, 15, 16, 17, 63, 64, 65, 127, 129, 400, 0, 1000, 2, 255, 257]


@pytest.mark.parametrize("hq, hkv", [(1, 1), (4, 2), (32, 4), (40, 8), (9, 1), (16, 1), (17, 1), (40, 1), (16, 16)])
@pytest.mark.parametrize("page, order", [(16, "token"), (64, "head"), (1, "token"), (24, "token"), (100, "head"), (256, "token")])
def test_decode_equals_the_oracle(hq, hkv, page, order):
    k, v, table, lens = _sequences(hq + page, LENS, page, hkv, order)
    q = _randn(hq, len(LENS), hq, 128, scale=1.5)
    out, lse = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    _check_decode(out, lse, q, k, v, table, lens)
    again, _ = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    assert torch.equal(out, again)


@pytest.mark.parametrize("lens, hq, hkv, page", [
    ([20011], 32, 4, 64), ([9000, 1], 8, 2, 128), ([1, 9000], 16, 16, 16), ([0, 5000, 0], 5, 1, 24), ([0] * 5, 8, 2, 16), ([1], 3, 1, 16),
    ([33, 1] * 150, 4, 2, 16), ([700] * 40 + [30000], 8, 1, 256)])
def test_decode_of_long_and_uneven_batches(lens, hq, hkv, page):
    k, v, table, n = _sequences(len(lens), lens, page, hkv)
    q = _randn(3, len(lens), hq, 128, scale=1.5)
    out, lse = rbs_paged_decode(q, k, v, table, n, return_lse=True)
    _check_decode(out, lse, q, k, v, table, n)


def test_decode_scale_strides_and_a_narrow_table():
    k, v, table, lens = _sequences(9, [77, 500, 3], 16, 2)
    x = _randn(9, 3, 8 + 4, 128)
    q = x[:, :8]                                                        # a slice of the fused projection
    whole = torch.full((3, 10, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:, 1:9, 128:]
    wide = torch.full((3, table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    for scale in (0.3, -0.05):
        o, lse = rbs_paged_decode(q, k, v, wide[:, :table.shape[1]], lens, out=out, return_lse=True, softmax_scale=scale)
        _check_decode(o, lse, q, k, v, table, lens, scale)
    assert bool((whole[:, 0] == 7).all() and (whole[:, 9] == 7).all() and (whole[..., :128] == 7).all())
    lens[1] = 1 << 30                                                   # longer than its table: as long as the table
    cut = lens.clone()
    cut[1] = 20 * 16
    a, b = (rbs_paged_decode(q, k, v, table[:, :20].contiguous(), n) for n in (lens, cut))
    assert torch.equal(a, b)


@pytest.mark.parametrize("hq, hkv", [(32, 4), (40, 1)])
def test_decode_into_its_own_queries(hq, hkv):
    k, v, table, lens = _sequences(21, [5000, 0, 17, 300, 1, 900], 32, hkv)
    q = _randn(22, 6, hq, 128)
    want = rbs_paged_decode(q, k, v, table, lens)
    got = rbs_paged_decode(q, k, v, table, lens, out=q)
    assert got is q and torch.equal(q, want)


def test_decode_of_more_sequences_than_one_chunk_of_the_search():
    g = np.random.default_rng(4)
    lens = [int(n) for n in g.integers(0, 40, 1500)]
    lens[700], lens[1499] = 3000, 77
    k, v, table, n = _sequences(23, lens, 16, 1)
    q = _randn(24, 1500, 2, 128)
    out, lse = rbs_paged_decode(q, k, v, table, n, return_lse=True)
    _check_decode(out, lse, q, k, v, table, n)


def test_decode_of_sequences_that_share_their_pages():
    """A common prompt: 330 block tables name the same pages, 58 thousand tiles of work over 0.7 MB of keys.  That much work goes to
    two waves of thread blocks."""
    k, v, table, _ = _sequences(25, [2900], 16, 1)
    lens = [2900 - 3 * (i % 50) for i in range(330)]
    table = table.expand(330, -1).contiguous()
    q = _randn(26, 330, 3, 128, scale=1.5)
    assert sum(-(-n // 16) + 2 for n in lens) > 444 * 4 * 32
    out, lse = rbs_paged_decode(q, k, v, table, _ints(lens), return_lse=True)
    _check_decode(out, lse, q, k, v, table, _ints(lens))


def _shared(seed, seqs, hq, hkv, page, longest):
    """Block tables that all name the same pages, and lengths with work for two waves of thread blocks."""
    k, v, table, _ = _sequences(seed, [longest], page, hkv)
    lens = [longest - 7 * (i % 40) for i in range(seqs)]
    items = hkv * (-(-(hq // hkv) // 16))
    assert sum(-(-n // 16) + 2 for n in lens) * items > 444 * 4 * 32
    return _randn(seed + 1, seqs, hq, 128, scale=1.5), k, v, table.expand(seqs, -1).contiguous(), _ints(lens)


SHARED = [(31, 330, 3, 1, 24, 2900), (32, 330, 9, 1, 16, 2900), (33, 330, 16, 1, 24, 2900), (34, 110, 40, 1, 16, 3000), (35, 100, 16, 4, 16, 2600),
          (36, 100, 64, 4, 24, 2600)]


@pytest.mark.parametrize("seed, seqs, hq, hkv, page, longest", SHARED)
def test_decode_in_two_waves(seed, seqs, hq, hkv, page, longest):
    q, k, v, table, lens = _shared(seed, seqs, hq, hkv, page, longest)
    out, lse = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    t = torch.arange(longest, device="cuda")
    kd, vd = (x[table[0, t // page].long(), t % page].double().transpose(0, 1) for x in (k, v))      # [hkv, tokens, 128]
    score = q.double().view(seqs, hkv, hq // hkv, 128).transpose(0, 1) @ kd.transpose(1, 2)[:, None] / 128 ** 0.5
    score.masked_fill_(t >= lens[:, None, None], -torch.inf)
    p = score.softmax(-1)
    ref, size = ((p @ x[:, None]).transpose(0, 1).reshape(seqs, hq, 128) for x in (vd, vd.abs()))
    assert bool(((out.double() - ref).abs() <= STEP * ref.abs() + (2.0 ** -16 + 1e-4) * size).all())
    assert float((lse.double() - score.logsumexp(-1).transpose(0, 1).reshape(seqs, hq)).abs().max()) <= 1e-4
    assert torch.equal(out, rbs_paged_decode(q, k, v, table, lens))


def test_decode_leaves_out_tokens_whose_page_does_not_exist():
    k, v, table, lens = _sequences(11, [300, 40, 64], 16, 2)
    q = _randn(12, 3, 8, 128)
    for s, at, page in ((0, 0, -1), (0, 7, k.shape[0]), (0, 18, -(1 << 31)), (1, 1, (1 << 31) - 1), (2, 0, -1), (2, 1, -1), (2, 2, -1), (2, 3, -1)):
        table[s, at] = page
    out, lse = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    _check_decode(out, lse, q, k, v, table, lens)
    assert bool((out[2] == 0).all() and (lse[2] == -np.inf).all())


def test_decode_of_one_dominant_key_and_of_scores_far_apart():
    k, v, table, lens = _sequences(13, [2000, 90], 64, 1)
    q = _randn(14, 2, 4, 128)
    p, o = int(table[0, 30]), 50
    k[p, o, 0] = (q[0, 0] * 20).to(torch.bfloat16)                      # a score of some 200
    k[int(table[1, 1]), 10:20, 0] = -(q[1, 1] * 30).to(torch.bfloat16)
    out, lse = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    ref, l, size = so.decode(_f64(q), _f64(k), _f64(v), table.cpu().numpy(), lens.cpu().numpy())
    # scores of up to 350: fp32 rounding of a sum of that size, 350 * 2^-24 per addition over 8 steps of the product
    assert (np.abs(_f64(out) - ref) <= STEP * np.abs(ref) + (2.0 ** -16 + 1e-3) * size).all()
    assert np.abs(_f64(lse) - l).max() <= 1e-3


@pytest.mark.parametrize("hq, hkv", [(8, 8), (16, 1)])
def test_decode_keeps_probabilities_in_32_bits(hq, hkv):
    """Values that cancel: two keys of score 0 hold the negative of what the third key's probability makes of its value, to 2^-17 of
    it, so that the output's own rounding leaves the probability's in sight.
    The score is one product, |x| <= 2 in log2 units: its scale is rounded three times, 3 * 2^-24 |x|, and the exponential is off by 2^-22:
    together below 2^-21 of a probability that makes up half of `size`.  Three terms in fp32 with up to three products each leave
    9 * 2^-24 of it, so 2^-20 covers all.  Two bf16 numbers in place of a probability are off by up to 2^-18."""
    g = np.random.default_rng(5)
    seqs = 64
    bf16 = lambda x: torch.tensor(x).to(torch.bfloat16).double().numpy()  # noqa: E731
    x, w = bf16(g.uniform(0.25, 15.0, (seqs, hkv))), bf16(g.uniform(1.0, 2.0, (seqs, hkv, 128)))
    want = -np.exp(-x / np.sqrt(128.0))[..., None] * w
    q = np.zeros((seqs, hkv, hq // hkv, 128))
    q[..., 0] = x[..., None]
    k, v = np.zeros((seqs, 16, hkv, 128)), np.zeros((seqs, 16, hkv, 128))
    k[:, 2, :, 0], v[:, 2] = -1.0, w
    v[:, 0] = bf16(want)
    v[:, 1] = bf16(want - v[:, 0])
    q, k, v = (torch.tensor(t, device="cuda").to(torch.bfloat16) for t in (q.reshape(seqs, hq, 128), k, v))
    table, lens = torch.arange(seqs, dtype=torch.int32, device="cuda")[:, None], _ints([3] * seqs)
    out = rbs_paged_decode(q, k, v, table, lens)
    ref, _, size = so.decode(_f64(q), _f64(k), _f64(v), table.cpu().numpy(), lens.cpu().numpy())
    assert np.abs(ref).max() < 2.0 ** -16 * size.max()
    assert (np.abs(_f64(out) - ref) <= STEP * np.abs(ref) + 2.0 ** -20 * size).all()


@pytest.mark.parametrize("hq, page", [(8, 16), (8, 24), (32, 16)])
def test_decode_passes_infinite_values_on(hq, page):
    """Values of infinity, in keys of any weight: alone in its sequence, the maximum, somewhere in a sequence that many warps share."""
    where = [(0, 0), (1, 0), (1, 1), (1, 2), (2, 50), (3, 0), (3, 2999), (3, 5999)]
    k, v, table, lens = _sequences(17, [1, 3, 100, 6000], page, 2)
    q = _randn(18, 4, hq, 128)
    clean = rbs_paged_decode(q, k, v, table, lens)
    inf, half = float("inf"), hq // 2      # heads of the second KV head
    for s, t in where + [(2, None)]:       # None: in the key of largest weight of the first of those heads
        if t is None:
            t = np.argmax(_f64(k)[table[s, :-(-100 // page)].long().cpu().numpy(), :, 1].reshape(-1, 128)[:100] @ _f64(q)[s, half])
        at = (int(table[s, int(t) // page]), int(t) % page, 1)
        other = (int(table[s, 0]), 0, 1)
        kept, kept_other = v[at].clone(), v[other].clone()
        v[at][60], v[at][61], v[at][62] = inf, -inf, inf
        if at != other:
            v[other][62] = -inf            # the sum of both is no number
        out = rbs_paged_decode(q, k, v, table, lens)
        v[other], v[at] = kept_other, kept
        assert bool((out[s, half:, 60] == inf).all() and (out[s, half:, 61] == -inf).all()), (s, t)
        assert bool((out[s, half:, 62] == inf).all() if at == other else out[s, half:, 62].isnan().all())
        out[s, half:, 60:63] = clean[s, half:, 60:63]
        assert torch.equal(out, clean)


def test_decode_passes_nan_of_a_key_on_to_the_heads_that_read_it():
    k, v, table, lens = _sequences(15, [100, 100], 16, 2)
    q = _randn(16, 2, 8, 128)
    clean = rbs_paged_decode(q, k, v, table, lens)
    k[int(table[0, 2]), 3, 1, 60] = float("nan")
    out = rbs_paged_decode(q, k, v, table, lens)
    assert out[0, 4:].isnan().all()
    assert torch.equal(out[0, :4], clean[0, :4]) and torch.equal(out[1], clean[1])


def test_offsets_beyond_32_bits():
    """Pages 5 GB apart: byte offsets and element offsets pass 2^32 and 2^31."""
    far = 5 * (1 << 30) // 2 // 1024 * 1024
    room = torch.zeros(far + (1 << 20), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.as_strided(room, (2, 16, 4, 128), (far, 512, 128, 1), at) for at in (0, 1 << 19))
    k.copy_(_randn(1, 2, 16, 4, 128)), v.copy_(_randn(2, 2, 16, 4, 128))
    table, lens, q = _ints([[1, 0], [1, -1]]), _ints([29, 16]), _randn(3, 2, 32, 128)
    out, lse = rbs_paged_decode(q, k, v, table, lens, return_lse=True)
    _check_decode(out, lse, q, k, v, table, lens)
    x, pos, slots = _randn(4, 2, 4, 128), _ints([5, 6]), _ints([31, 3])
    rbs_qk_norm_rope_paged(_randn(5, 2, 8, 128), x, x, pos, slots, None, k, v)
    assert torch.equal(k[1, 15], x[0]) and torch.equal(v[0, 3], x[1])


# ------------------------------------------------------------------------------------------------ calls together


def test_calls_on_another_stream_and_in_a_replayed_graph():
    """A decode step (pages and slots, norm + rotation + write, attention) captured once and replayed while lengths, inputs and
    the cache change in place, against plain calls."""
    page, n_pages, hq, hkv = 16, 400, 8, 2
    start = [0, 100, 31, 700, 5]
    S = len(start)
    freq, w = _frequencies(64), torch.rand(128, device="cuda") + 0.5
    free = torch.randperm(n_pages, device="cuda").int()

    class State:
        def __init__(self):
            self.k, self.v = (torch.zeros(n_pages, page, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.table = torch.full((S, 60), -1, dtype=torch.int32, device="cuda")
            self.lens, self.used, self.one = _ints([0] * S), _ints([0]), _ints([1] * S)
            self.x = torch.empty(S, hq + 2 * hkv, 128, dtype=torch.bfloat16, device="cuda")
            self.ws = torch.empty(paged_decode_workspace_bytes(S, hq, hkv, page, n_pages, 60), dtype=torch.uint8, device="cuda")
            x = _randn(1, sum(start), hq + 2 * hkv, 128)
            first = rbs_paged_extend(self.lens, _ints(start), self.table, free, page, n_pages, sum(start))
            rbs_qk_norm_rope_paged(*x.split((hq, hkv, hkv), 1), first.positions, first.slots, freq, self.k, self.v, k_norm=w)
            self.lens.copy_(first.lens), self.used.copy_(first.used)

        def step(self):
            st = rbs_paged_extend(self.lens, self.one, self.table, free, page, n_pages, S, free_used=self.used)
            q = rbs_qk_norm_rope_paged(*self.x.split((hq, hkv, hkv), 1), st.positions, st.slots, freq, self.k, self.v, q_norm=w, k_norm=w)
            out, lse = rbs_paged_decode(q, self.k, self.v, self.table, st.lens, return_lse=True, workspace=self.ws)
            self.lens.copy_(st.lens), self.used.copy_(st.used)
            return q, out, lse
    a, b, side = State(), State(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.x.copy_(_randn(2, *b.x.shape))
        b.step()
    torch.cuda.current_stream().wait_stream(side)
    a.x.copy_(_randn(2, *a.x.shape))
    a.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.step()
    for seed in range(3, 30):      # some sequences begin new pages on the way
        for s in (a, b):
            s.x.copy_(_randn(seed, *s.x.shape))
        want = a.step()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert torch.equal(a.k, b.k) and torch.equal(a.table, b.table) and torch.equal(a.lens, b.lens)
    assert b.lens.tolist() == [n + 28 for n in start]
    _check_decode(got[1], got[2], got[0], b.k, b.v, b.table, b.lens)
    assert rbs_device_status() == 0


def test_prompts_and_generated_tokens_of_a_paged_cache():
    """Packed prompts through the cache and the prefill call, then tokens one by one, sequences that end and others that take their
    pages.  A prompt's last row of dense prefill attention is what decode attention of that token gives; everything the
    decode steps read is followed by the oracle's own norm, rotation and attention in 64 bits."""
    hq, hkv, layers, page = 8, 2, 2, 16
    lens = [130, 1, 300]
    cache = PagedCache(layers, 60, page, hkv, len(lens), 50, "cuda")
    freq, magnitude = rope_frequencies(128, 1e4, scaling="yarn", factor=4.0, trained_len=64)
    w = torch.rand(2, 128, device="cuda") + 0.5
    turn = {"q_norm": w[0], "k_norm": w[1], "magnitude": magnitude}
    kept = [[[] for _ in lens] for _ in range(layers)]      # (key, value) rows of every sequence, in bf16

    def tokens(seed, step, new, layer, out_k=None):
        n = step.slots.shape[0]
        x = _randn(seed + layer, n, hq + 2 * hkv, 128, scale=2.0)
        q, k, v = x.split((hq, hkv, hkv), dim=1)
        got = cache.write(layer, q, k, v, step, freq, out_k=out_k, **turn)
        _check_turn(got, q, step.positions, freq, w[0], magnitude=magnitude)
        keys, _ = rbs_qk_norm_rope(k, k, step.positions, freq, q_norm=w[1], k_norm=w[1], magnitude=magnitude)
        _check_turn(keys, k, step.positions, freq, w[1], magnitude=magnitude)
        row = 0
        for s, m in enumerate(new):
            kept[layer][s] += [(keys[i], v[i]) for i in range(row, row + m)]
            row += m
        return got, v

    def check(layer, q, out, lse):
        for s, rows in enumerate(kept[layer]):
            assert int(cache.lens[s]) == len(rows)
            if not rows:
                assert bool((out[s] == 0).all() and (lse[s] == -np.inf).all())
                continue
            k, v = (_f64(torch.stack([r[i] for r in rows])[None]) for i in (0, 1))
            o, l, size = so.decode(_f64(q[s:s + 1]), k, v, np.zeros((1, 1), int), [len(rows)])
            assert (np.abs(_f64(out[s]) - o[0]) <= STEP * np.abs(o[0]) + (2.0 ** -16 + 1e-4) * size[0]).all()
            assert np.abs(_f64(lse[s]) - l[0]).max() <= 1e-4

    step = cache.extend(_ints(lens), sum(lens))
    cu = np.concatenate(([0], np.cumsum(lens)))
    for layer in range(layers):
        k = torch.empty(sum(lens), hkv, 128, dtype=torch.bfloat16, device="cuda")
        q, v = tokens(100, step, lens, layer, out_k=k)
        prompt_out, _ = rbs_prefill_varlen(q, k, v.contiguous(), cu.tolist(), 64, alpha_base=1e-30, alpha_rescue=1e-30)      # every block
        last = torch.tensor(cu[1:] - 1, device="cuda")
        out, lse = cache.attend(layer, q[last].contiguous(), return_lse=True)
        check(layer, q[last], out, lse)
        # prefill attention is within 2e-2 (max) and 2e-3 (mean) of the exact value, decode attention nearer
        gap = (prompt_out[last].float() - out.float()).abs()
        assert gap.max() <= 3e-2 and gap.mean() <= 3e-3
    seed = 200
    for new in ([1, 1, 1], [1, 0, 1], [5, 1, 1], [1, 1, 1]):
        step = cache.extend(_ints(new), sum(new) + 1)
        pad = step.slots[sum(new):]
        assert bool((pad == -1).all())
        for layer in range(layers):
            q, _ = tokens(seed, step, new, layer)
            ends = (step.cu[1:] - 1).clamp(min=0).long()
            out, lse = cache.attend(layer, q[ends].contiguous(), return_lse=True)
            check(layer, q[ends], out, lse)
        seed += 10
    assert int(cache.used) == sum(-(-len(rows) // page) for rows in kept[0])
    held = -(-len(kept[0][1]) // page)
    cache.release([2, 0, 2])
    for layer in range(layers):
        kept[layer][0], kept[layer][2] = [], []
    assert int((cache.free_pages >= 0).sum()) == 60 - held and int(cache.used) == 0
    new = [700, 1, 150]      # the pages of the sequences that ended are needed
    step = cache.extend(_ints(new), sum(new))
    assert int(step.slots.min()) >= 0 and len(set(step.slots.tolist())) == sum(new)
    for layer in range(layers):
        q, _ = tokens(seed, step, new, layer)
        ends = (step.cu[1:] - 1).long()
        out, lse = cache.attend(layer, q[ends].contiguous(), return_lse=True)
        check(layer, q[ends], out, lse)
    n = len(kept[0][1])
    left = 60 - sum(-(-len(rows) // page) for rows in kept[0])
    fit = -(-n // page) * page - n + left * page      # what the begun page and the pages that are left can hold
    step = cache.extend(_ints([0, 200, 0]), 200)      # more than that
    assert 0 < fit < 200 and int(cache.used) > 60
    assert bool((step.slots[:fit] >= 0).all()) and bool((step.slots[fit:] == -1).all())
    cache.release([])
    with pytest.raises(RbsError):
        cache.release([3])


def test_a_sequence_that_ran_out_of_pages_is_named_until_it_ends():
    cache = PagedCache(1, 3, 16, 1, 2, 8, "cuda")
    cache.extend(_ints([20, 10]), 30)
    assert cache.short() == []
    cache.extend(_ints([1, 9]), 10)                # the second one's 17th to 19th tokens find no page
    assert cache.short() == [1] and cache.release([0]) == [1] and int(cache.used) == 0
    step = cache.extend(_ints([0, 14]), 14)        # the page that is begun stays missing, the next one is there
    assert (step.slots < 0).tolist() == [True] * 13 + [False] and cache.short() == [1]
    assert cache.release([1]) == [] and int((cache.free_pages >= 0).sum()) == 3


def test_calls_on_two_streams_at_once():
    """Two streams issue decode steps side by side, each with its own sequences; nothing is shared but the library."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    cases = []
    for i, (lens, hq, hkv, page) in enumerate((([3000, 20, 700], 32, 4, 64), ([100] * 50 + [5000], 16, 2, 24))):
        k, v, table, n = _sequences(30 + i, lens, page, hkv)
        q = _randn(40 + i, len(lens), hq, 128)
        cases.append((q, k, v, table, n, rbs_paged_decode(q, k, v, table, n)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(40):
        for side, (q, k, v, table, n, _) in zip(range(2), cases):
            with torch.cuda.stream(streams[side]):
                got[side].append(rbs_paged_decode(q, k, v, table, n))
    torch.cuda.synchronize()
    for side in range(2):
        assert all(torch.equal(out, cases[side][5]) for out in got[side])


def test_calls_refuse_what_does_not_fit_together():
    q, cache, table, lens = _randn(1, 2, 8, 128), _randn(2, 3, 16, 2, 128), _ints([[0], [1]]), _ints([3, 4])
    pos, freq = _ints([0, 1]), _frequencies(128)
    k = q[:, :2].contiguous()
    bad_decodes = [(q.float(), cache, cache, table, lens), (q, cache[..., :64], cache[..., :64], table, lens), (q, cache, cache[:2], table, lens),
                   (q, cache, cache, table[:1], lens), (q, cache, cache, table, lens[:1]), (q, cache, cache, table, lens.long()),
                   (q, cache, cache, table.long(), lens), (q, cache, cache, table[0], lens), (q, cache.cpu(), cache, table, lens),
                   (q[:, :7], cache, cache, table, lens), (q[..., ::2], cache, cache, table, lens), (q[0], cache, cache, table, lens)]
    for args in bad_decodes:
        with pytest.raises(RbsError):
            rbs_paged_decode(*args)
    with pytest.raises(RbsError):
        rbs_paged_decode(q, cache, cache, table, lens, out=torch.empty_like(q[:1]))
    for args in [(q, k, pos[:1], freq), (q, k, pos.long(), freq), (q, k, pos, freq.double()), (q, k[:1], pos, freq), (q.half(), k, pos, freq),
                 (q, k, pos, freq[:3]), (q, k, pos, torch.cat((freq, freq))), (q, k.cpu(), pos, freq), (q[None], k, pos, freq)]:
        with pytest.raises(RbsError):
            rbs_qk_norm_rope(*args)
    with pytest.raises(RbsError):
        rbs_qk_norm_rope(q, k, pos, freq, q_norm=torch.ones(64, device="cuda"))
    for args in [(q, k, k[:1], pos, pos, freq, cache, cache), (q, k, k, pos, torch.cat((pos, pos)), freq, cache, cache), (q, k, k, pos, pos, freq, cache, cache[:, :, :1]),
                 (q, q, q, pos, pos, freq, cache, cache)]:
        with pytest.raises(RbsError):
            rbs_qk_norm_rope_paged(*args)
    for args in [(lens, lens[:1], table, pos, 16, 3, 2), (lens.long(), lens, table, pos, 16, 3, 2), (lens, lens, table[:1], pos, 16, 3, 2),
                 (lens, lens, table, pos, 0, 3, 2), (lens, lens, table, pos, 16, 3, 1 << 31)]:
        with pytest.raises((RbsError, RuntimeError)):
            rbs_paged_extend(*args)
    step = alloc_step(2, 2, "cuda")
    step.lens = lens
    with pytest.raises(RbsError):
        rbs_paged_extend(lens, lens, table, pos, 16, 3, 2, out=step)


DEBUG_CHILD = r"""
import sys, torch
sys.path.insert(0, "tests")
import test_gpu_serving as t
from paper_2609_20971_b200 import rbs_device_status
from paper_2609_20971_b200.binding import rbs_version
assert "debug checks" in rbs_version()
torch.save(t.debug_outputs(), sys.argv[1])
assert rbs_device_status(clear=True) == 0, "a device-side check failed"
print("debug child ok")
"""


def debug_outputs():
    got = []
    for seed, lens, hq, hkv, page in ((1, LENS, 40, 8, 24), (2, [20011], 32, 4, 64), (3, [33, 1] * 150, 16, 1, 16), (4, [700] * 40 + [30000], 8, 1, 256)):
        k, v, table, n = _sequences(seed, lens, page, hkv)
        got += rbs_paged_decode(_randn(seed, len(lens), hq, 128), k, v, table, n, return_lse=True)
    for case in EXTENDS:
        lens, add, table, free, used, page, n_pages, tokens = _extend_case(*case)
        table = _ints(table)
        out = rbs_paged_extend(_ints(lens), _ints(add), table, _ints(free), page, n_pages, tokens, free_used=None if used is None else _ints([used]))
        got += [table, out.lens, out.cu, out.positions, out.slots, out.used]
    return [x.cpu() for x in got]


def test_debug_library_runs_the_calls_clean_and_bit_identical(tmp_path):
    from paper_2609_20971_b200.build import build_library
    build_library(debug=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, RBS_DEBUG="1", PYTHONPATH=root + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, "-c", DEBUG_CHILD, str(tmp_path / "out.pt")], env=env, cwd=root, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "debug child ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
    assert all(torch.equal(x, y) for x, y in zip(torch.load(tmp_path / "out.pt"), debug_outputs(), strict=True))


def debug_outputs_of_large_calls():
    got = []
    for case in SHARED:
        got += rbs_paged_decode(*_shared(*case), return_lse=True)
    for case in MANY_ROWS:
        lens, add, table, free, used, page, n_pages, tokens = _many_rows(*case)
        table = _ints(table)
        out = rbs_paged_extend(_ints(lens), _ints(add), table, _ints(free), page, n_pages, tokens, free_used=_ints([used]))
        got += [table, out.lens, out.cu, out.positions, out.slots, out.used]
    return [x.cpu() for x in got]


def test_debug_library_runs_large_calls_clean_and_bit_identical(tmp_path):
    from paper_2609_20971_b200.build import build_library
    build_library(debug=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, RBS_DEBUG="1", PYTHONPATH=root + os.pathsep + os.environ.get("PYTHONPATH", ""))
    child = DEBUG_CHILD.replace("debug_outputs()", "debug_outputs_of_large_calls()")
    r = subprocess.run([sys.executable, "-c", child, str(tmp_path / "out.pt")], env=env, cwd=root, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "debug child ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
    assert all(torch.equal(x, y) for x, y in zip(torch.load(tmp_path / "out.pt"), debug_outputs_of_large_calls(), strict=True))
