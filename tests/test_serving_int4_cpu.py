"""The cache in 4 bits without a GPU: what its calls refuse before they launch anything, and pins of their fp64 oracle."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2609_20971_b200 import PagedCache, RbsError, binding, rbs_paged_decode_int4, rbs_paged_read_int4, rbs_paged_write_int4
from paper_2609_20971_b200.binding import RbsCacheInt4, RbsPagedShape, RbsTensor

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x1000
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    from paper_2609_20971_b200.build import build_library
    build_library()
    return binding.load_library()


def _t(ptr=P, sb=0, st=128, sh=128):
    return RbsTensor(ptr, sb, st, sh)


def _cache(codes=None, scales=None):
    return RbsCacheInt4(codes or _t(st=64, sh=64), scales or _t(st=8, sh=8))


def _shape(**change):
    v = dict(n_seqs=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=50, max_pages=7, table_stride=8)
    v.update(change)
    return RbsPagedShape(**v)


def _write(lib, shape=None, n=5, k=None, v=None, slots=P, kc=None, vc=None):
    return lib.rbs_paged_write_int4(shape or _shape(), n, k or _t(), v or _t(), slots, kc or _cache(), vc or _cache(), None)


def _read(lib, shape=None, kc=None, vc=None, table=P, starts=None, cu=P, n=5, k=None, v=None):
    return lib.rbs_paged_read_int4(shape or _shape(), kc or _cache(), vc or _cache(), table, starts, cu, n, k or _t(), v or _t(), None)


def _decode(lib, shape=None, q=None, kc=None, vc=None, table=P, lens=P, o=None, scale=0.0, ws=0x100000, n=1 << 40):
    return lib.rbs_paged_decode_int4(shape or _shape(), q or _t(), kc or _cache(), vc or _cache(), table, lens, o or _t(), None, scale, ws, n, None)


BAD_PAGES = [(dict(page_size=0), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=1 << 20, page_size=1 << 11), UNSUPPORTED)]
BAD_TABLES = [(dict(n_seqs=0), INVALID), (dict(max_pages=0), INVALID), (dict(table_stride=6), INVALID),
              (dict(max_pages=1 << 20, table_stride=1 << 20, page_size=1 << 11), UNSUPPORTED)]
BAD_HEADS = [(dict(n_q_heads=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(n_q_heads=9), UNSUPPORTED)]
BAD_ROWS = [_t(None), _t(P + 8), _t(st=130), _t(sh=0), _t(st=-128), _t(sh=4)]
BAD_CACHES = [_cache(codes=_t(None, st=64, sh=64)), _cache(scales=_t(None, st=8, sh=8)), _cache(codes=_t(P + 8, st=64, sh=64)),
              _cache(scales=_t(P + 4, st=8, sh=8)), _cache(codes=_t(st=72, sh=64)), _cache(codes=_t(st=64, sh=8)), _cache(codes=_t(sb=24, st=64, sh=64)),
              _cache(scales=_t(st=12, sh=8)), _cache(scales=_t(st=8, sh=4)), _cache(scales=_t(sb=4, st=8, sh=8)), _cache(codes=_t(st=0, sh=64)),
              _cache(scales=_t(st=8, sh=0)), _cache(codes=_t(sb=-64, st=64, sh=64)), _cache(scales=_t(st=-8, sh=8))]


@pytest.mark.parametrize("change, want", BAD_PAGES + BAD_HEADS + [(dict(n_q_heads=40000, n_kv_heads=40000), UNSUPPORTED)])
def test_write_and_read_refuse_shapes(lib, change, want):
    assert _write(lib, _shape(**change)) == want
    assert _read(lib, _shape(**change)) == want


@pytest.mark.parametrize("change, want", BAD_TABLES)
def test_read_refuses_tables(lib, change, want):
    assert _read(lib, _shape(**change)) == want


@pytest.mark.parametrize("change, want", BAD_PAGES + BAD_TABLES + BAD_HEADS)
def test_decode_refuses_shapes(lib, change, want):
    assert _decode(lib, _shape(**change)) == want
    assert lib.rbs_paged_decode_int4_workspace_bytes(_shape(**change)) == 0


@pytest.mark.parametrize("bad", BAD_CACHES)
@pytest.mark.parametrize("which", ["kc", "vc"])
def test_calls_refuse_caches(lib, bad, which):
    assert _write(lib, **{which: bad}) == INVALID
    assert _read(lib, **{which: bad}) == INVALID
    assert _decode(lib, **{which: bad}) == INVALID


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_calls_refuse_tensors(lib, bad):
    for which in ("k", "v"):
        assert _write(lib, **{which: bad}) == INVALID
        assert _read(lib, **{which: bad}) == INVALID
    for which in ("q", "o"):
        assert _decode(lib, **{which: bad}) == INVALID


def test_calls_refuse_arguments(lib):
    assert _write(lib, slots=None) == INVALID and _write(lib, n=-1) == INVALID
    assert lib.rbs_paged_write_int4(None, 5, _t(), _t(), P, _cache(), _cache(), None) == INVALID
    for args in (dict(table=None), dict(cu=None), dict(n=-1)):
        assert _read(lib, **args) == INVALID
    for args in (dict(table=None), dict(lens=None), dict(scale=NAN), dict(scale=INF), dict(scale=3e38)):
        assert _decode(lib, **args) == INVALID
    assert lib.rbs_paged_decode_int4_workspace_bytes(None) == 0


def test_calls_without_rows_do_nothing(lib):
    assert _write(lib, n=0, slots=None, k=_t(None), v=_t(None)) == OK
    assert _read(lib, n=0, k=_t(None), v=_t(None)) == OK


def test_decode_refuses_tables_of_too_many_tiles_and_workspaces(lib):
    big = dict(n_seqs=1 << 13, n_q_heads=128, n_kv_heads=128, max_pages=1 << 17, table_stride=1 << 17)
    assert _decode(lib, _shape(**big)) == UNSUPPORTED
    need = lib.rbs_paged_decode_int4_workspace_bytes(_shape())
    assert need > 0
    for args in (dict(ws=None), dict(ws=0x100080), dict(n=0), dict(n=need - 1)):
        assert _decode(lib, **args) == WORKSPACE


@pytest.mark.parametrize("keys", [16, 32])
def test_decode_takes_tables_up_to_the_border_of_31_bits(lib, keys):
    """A call that is taken goes on to the workspace, which is refused here."""
    def call(**change):
        s = _shape(n_seqs=1, table_stride=1 << 20, **change)
        if keys == 32:
            return _decode(lib, s, ws=None)
        return lib.rbs_paged_decode(s, _t(), _t(), _t(), P, P, _t(), None, 0.0, None, 0, None)
    heads = 1 << 16
    for hq, hkv in ((heads, heads), (heads * 16, heads), (heads // 2 * 17, heads // 2), (heads // 2 * 32, heads // 2)):
        for units, want in ((32767, WORKSPACE), (32768, UNSUPPORTED)):      # 2^16 of them, of which 3 are not for tokens
            assert call(n_q_heads=hq, n_kv_heads=hkv, page_size=keys, max_pages=units - 3) == want
    assert call(n_q_heads=15 << 20, n_kv_heads=1 << 20, max_pages=1) == WORKSPACE
    assert call(n_q_heads=1 << 24, n_kv_heads=1 << 20, max_pages=1) == UNSUPPORTED


def test_calls_refuse_host_tensors_and_caches_of_other_bits():
    x, ints = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache = torch.zeros(3, 16, 4, 64, dtype=torch.uint8), torch.zeros(3, 16, 4, 8, dtype=torch.uint8)
    table = torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_paged_write_int4(x, x, ints, cache, cache)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_paged_read_int4(cache, cache, table, torch.zeros(3, dtype=torch.int32), 4)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_paged_decode_int4(x, cache, cache, table, ints)
    with pytest.raises(RbsError, match="bits"):
        PagedCache(1, 3, 16, 2, 1, 3, "cpu", bits=8)
    with pytest.raises(RbsError, match="16 bits"):
        PagedCache(1, 3, 16, 2, 1, 3, "cpu").read(0, 5)


def test_a_cache_in_4_bits_takes_9_bytes_where_bf16_takes_32():
    a, b = (PagedCache(2, 3, 16, 2, 1, 3, "cpu", bits=bits) for bits in (4, 16))
    size = sum(t.numel() for c in (a.k, a.v) for t in c)
    assert 32 * size == 9 * (2 * b.k.numel() * b.k.element_size())
    (kc, ks), (vc, vs) = a._layer(1)
    assert kc.shape == vc.shape == (3, 16, 2, 64) and ks.shape == vs.shape == (3, 16, 2, 8)
    assert kc.stride() == (2 * 16 * 64, 64, 16 * 64, 1)


# ------------------------------------------------------------------------------------------------ pins of the oracle


def test_oracle_scales_are_the_numbers_of_5_exponent_and_3_mantissa_bits():
    v = so.scale_int4(np.arange(168))
    assert v[0] == 0 and v[1] == 2.0 ** -14 and v[8] == 2.0 ** -11 and v[167] == 480 and v[96] == 1 and v[100] == 1.5
    assert (np.diff(v) > 0).all() and np.isnan(so.scale_int4([255])[0])
    # an eighth of them are the fp16 numbers whose bits are the byte and seven zeros
    assert np.array_equal(v / 8, (np.arange(168, dtype=np.uint16) << 7).view(np.float16).astype(np.float64))


def test_oracle_quantisation_by_hand():
    x = np.zeros((1, 128))
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = 7.0, 2.5, -2.5, -0.5       # scale 1: ties go away from zero
    x[0, 16:19] = -8.0, 7.5, -7.6                                    # 7.5 / 7 = 1.07 is nearer to 1 + 1/8 than to 1
    x[0, 32] = 7.0 * (1 + 1 / 16)                                    # half way between the scales 1 and 1 + 1/8: the even byte
    x[0, 48] = 7.0 * (1 + 3 / 16)                                    # half way between 1 + 1/8 and 1 + 2/8
    x[0, 64], x[0, 65] = 1e30, -5.0                                  # saturated
    x[0, 80] = 2.0 ** -13                                            # a scale of less than half of the smallest
    x[0, 96], x[0, 112] = np.inf, np.nan
    code, byte = so.quantise_int4(x)
    assert byte.tolist() == [[96, 97, 96, 98, 167, 0, 255, 255]]
    assert code[0, :4].tolist() == [15, 11, 5, 7] and code[0, 16:19].tolist() == [1, 15, 1]
    assert code[0, 32] == 15 and code[0, 48] == 15 and code[0, 64:66].tolist() == [15, 8] and (code[0, 80:] == 8).all()
    assert np.array_equal(so.unpack_int4([[0x21, 0xf0] + [0x88] * 62])[0, :5], [1, 2, 0, 15, 8])


def test_oracle_quantisation_is_within_half_a_scale():
    g = np.random.default_rng(1)
    x = g.standard_normal((400, 128)) * 2.0 ** g.integers(-12, 8, (400, 1))
    code, byte = so.quantise_int4(x)
    assert code.min() == 0 and code.max() == 15
    bound = np.maximum(np.repeat(so.scale_int4(byte), 16, -1) / 2, 2.0 ** -12)
    assert (np.abs(so.dequantise_int4(code, byte) - x) <= bound).all()


def test_oracle_range_ends_at_7_and_minus_8_times_the_largest_scale():
    x = np.zeros((8, 128))
    x[:, ::16] = np.linspace(-3840, 3360, 64).reshape(8, 8)              # one large element per scale, all within half a scale
    x[:, 1::16] = g = np.linspace(-3840, 3360, 64)[::-1].reshape(8, 8)   # and another beside it
    code, byte = so.quantise_int4(x)
    back = so.dequantise_int4(code, byte)
    assert (np.abs(back - x) <= np.repeat(so.scale_int4(byte), 16, -1) / 2).all() and np.abs(g).max() == 3840
    x[:] = 3840.0                                                        # 8 scales of 480, of which there are codes for 7
    assert (so.dequantise_int4(*so.quantise_int4(x)) == 3360).all()
    assert (so.dequantise_int4(*so.quantise_int4(-2 * x)) == -3840).all()


def test_oracle_ties_by_fractions():
    """bf16 numbers of few bits: scales and codes against exact fractions."""
    g = np.random.default_rng(2)
    x = g.integers(-127, 128, (60, 128)) * 2.0 ** g.integers(-9, 3, (60, 1))
    code, byte = so.quantise_int4(x)
    values = [Fraction(v) for v in so.scale_int4(np.arange(168))]
    for r in range(60):
        for j in range(8):
            part = [Fraction(v) for v in x[r, 16 * j:16 * j + 16]]
            want = max(max(part) / 7, min(part) / -8)
            near = min(abs(v - want) for v in values)
            best = [b for b, v in enumerate(values) if abs(v - want) == near]
            assert byte[r, j] == (best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])
            s = values[byte[r, j]]
            for v, c in zip(part, code[r, 16 * j:16 * j + 16]):
                n = 0 if s == 0 else int(abs(v) / s + Fraction(1, 2)) * (1 if v > 0 else -1)
                assert c - 8 == min(max(n, -8), 7)


def test_division_of_slots_by_the_page_size_is_exact():
    """slot / page as a product and a shift, as the kernels take it: every page size near a power of two, slots at every border."""
    g = np.random.default_rng(3)
    sizes = {1, 2, 3, 24, 100, (1 << 31) - 1} | {(1 << b) + d for b in range(1, 31) for d in (-1, 0, 1)} | set(g.integers(1, 1 << 31, 500).tolist())
    for d in sizes - {0}:
        shift = (d - 1).bit_length()
        factor = ((1 << (31 + shift)) + d - 1) // d
        assert factor < 1 << 32
        most = ((1 << 31) - 1) // d
        for q in {0, 1, most, most // 2, most - 1, int(g.integers(0, most + 1))} - {-1}:
            for n in (q * d - 1, q * d, q * d + d - 1, (1 << 31) - 1):
                if 0 <= n < 1 << 31:
                    assert n * factor >> (31 + shift) == n // d


def test_the_structure_has_the_size_of_the_header():
    assert ctypes.sizeof(RbsCacheInt4) == 2 * ctypes.sizeof(RbsTensor) == 64
