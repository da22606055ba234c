"""The serving calls without a GPU: what the library refuses before it launches anything, and pins of their fp64 oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2609_20971_b200 import PagedCache, RbsError, binding, rbs_paged_decode, rbs_paged_extend, rbs_qk_norm_rope, rope_frequencies
from paper_2609_20971_b200.binding import RbsPagedShape, RbsRope, RbsTensor

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


def _shape(**change):
    v = dict(n_seqs=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=50, max_pages=7, table_stride=8)
    v.update(change)
    return RbsPagedShape(**v)


BAD_TABLES = [(dict(n_seqs=0), INVALID), (dict(page_size=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
              (dict(table_stride=6), INVALID), (dict(n_pages=1 << 20, page_size=1 << 11), UNSUPPORTED),
              (dict(max_pages=1 << 20, table_stride=1 << 20, page_size=1 << 11), UNSUPPORTED)]
BAD_HEADS = [(dict(n_q_heads=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(n_q_heads=9), UNSUPPORTED)]


def _extend(lib, shape, seq_lens=P, new_lens=2 * P, free=3 * P, n_free=4, used=None, tokens=5, table=4 * P, out=5 * P, cu=6 * P,
            positions=7 * P, slots=8 * P, used_out=9 * P):
    return lib.rbs_paged_extend(shape, seq_lens, new_lens, free, n_free, used, tokens, table, out, cu, positions, slots, used_out, None)


@pytest.mark.parametrize("change, want", BAD_TABLES + [(dict(n_seqs=8193), UNSUPPORTED)])
def test_extend_refuses_shapes(lib, change, want):
    assert _extend(lib, _shape(**change)) == want


@pytest.mark.parametrize("args, want", [
    (dict(seq_lens=None), INVALID), (dict(new_lens=None), INVALID), (dict(table=None), INVALID), (dict(out=None), INVALID),
    (dict(cu=None), INVALID), (dict(used_out=None), INVALID), (dict(free=None), INVALID), (dict(positions=None), INVALID),
    (dict(slots=None), INVALID), (dict(n_free=-1), INVALID), (dict(tokens=-1), INVALID),
    (dict(out=P), INVALID), (dict(out=2 * P), INVALID), (dict(used=9 * P), INVALID),      # outputs that are inputs
    (dict(tokens=0x7fffffff - 7 * 16), UNSUPPORTED)])
def test_extend_refuses_arguments(lib, args, want):
    assert _extend(lib, _shape(), **args) == want


def test_extend_refuses_no_shape(lib):
    assert _extend(lib, None) == INVALID


def _turn(**change):
    v = dict(positions=P, inv_freq=P, q_norm=P, k_norm=P, eps=1e-6, magnitude=1.0, rot_dim=128, interleaved=0)
    v.update(change)
    return RbsRope(**v)


BAD_TURNS = [(dict(positions=None), INVALID), (dict(inv_freq=None), INVALID), (dict(q_norm=P + 4), INVALID), (dict(k_norm=P + 8), INVALID),
             (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(magnitude=NAN), INVALID),
             (dict(magnitude=INF), INVALID), (dict(rot_dim=-8), INVALID), (dict(interleaved=2), INVALID), (dict(rot_dim=136), UNSUPPORTED),
             (dict(rot_dim=20), UNSUPPORTED)]
BAD_ROWS = [_t(None), _t(P + 8), _t(st=130), _t(sh=0), _t(st=-128), _t(sh=4)]


@pytest.mark.parametrize("change, want", BAD_TURNS)
def test_norm_rope_refuses_rotations(lib, change, want):
    assert lib.rbs_qk_norm_rope(1, 5, 8, 2, 128, _t(), _t(), _turn(**change), _t(), _t(), None) == want
    assert lib.rbs_qk_norm_rope_paged(_shape(), 5, _t(), _t(), _t(), _turn(**change), P, 5, _t(), _t(None), _t(), _t(), None) == want


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("bad", BAD_ROWS)
def test_norm_rope_refuses_tensors(lib, which, bad):
    rows = [_t() for _ in range(4)]
    rows[which] = bad
    assert lib.rbs_qk_norm_rope(1, 5, 8, 2, 128, rows[0], rows[1], _turn(), rows[2], rows[3], None) == INVALID


def test_norm_rope_refuses_sizes(lib):
    for batch, tokens, hq, hkv, d, want in [(0, 5, 8, 2, 128, INVALID), (1, 0, 8, 2, 128, INVALID), (1, 5, 0, 2, 128, INVALID),
                                            (1, 5, 8, 0, 128, INVALID), (1, 5, 8, 2, 64, UNSUPPORTED)]:
        assert lib.rbs_qk_norm_rope(batch, tokens, hq, hkv, d, _t(), _t(), _turn(), _t(), _t(), None) == want
    assert lib.rbs_qk_norm_rope(1, 5, 8, 2, 128, _t(), _t(), None, _t(), _t(), None) == INVALID
    for outs in ((_t(sb=0), _t(sb=640)), (_t(sb=640), _t(sb=0))):      # a batch that would be written over itself
        assert lib.rbs_qk_norm_rope(2, 5, 8, 2, 128, _t(), _t(), _turn(), *outs, None) == INVALID


@pytest.mark.parametrize("which", range(6))
@pytest.mark.parametrize("bad", BAD_ROWS)
def test_norm_rope_paged_refuses_tensors(lib, which, bad):
    rows = [_t() for _ in range(6)]      # Q, K, V, Q', caches
    rows[which] = bad
    q, k, v, o, kc, vc = rows
    assert lib.rbs_qk_norm_rope_paged(_shape(), 5, q, k, v, _turn(), P, 5, o, _t(None), kc, vc, None) == INVALID


def test_norm_rope_paged_refuses_shapes(lib):
    for change, want in BAD_HEADS + [(dict(page_size=0), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=1 << 20, page_size=1 << 11), UNSUPPORTED)]:
        assert lib.rbs_qk_norm_rope_paged(_shape(**change), 5, _t(), _t(), _t(), _turn(), P, 5, _t(), _t(None), _t(), _t(), None) == want
    assert lib.rbs_qk_norm_rope_paged(_shape(), 0, _t(), _t(), _t(), _turn(), P, 5, _t(), _t(None), _t(), _t(), None) == INVALID
    assert lib.rbs_qk_norm_rope_paged(_shape(), 5, _t(), _t(), _t(), _turn(), None, 5, _t(), _t(None), _t(), _t(), None) == INVALID
    assert lib.rbs_qk_norm_rope_paged(_shape(), 5, _t(), _t(), _t(), _turn(), P, 5, _t(), _t(st=4), _t(), _t(), None) == INVALID


@pytest.mark.parametrize("n_slots", [-1, 6])
def test_norm_rope_paged_refuses_more_slots_than_tokens(lib, n_slots):
    assert lib.rbs_qk_norm_rope_paged(_shape(), 5, _t(), _t(), _t(), _turn(), P, n_slots, _t(), _t(None), _t(), _t(), None) == INVALID


def _decode(lib, shape, q=None, k=None, v=None, table=P, lens=P, o=None, scale=0.0, ws=0x100000, n=1 << 40):
    return lib.rbs_paged_decode(shape, q or _t(), k or _t(), v or _t(), table, lens, o or _t(), None, scale, ws, n, None)


@pytest.mark.parametrize("change, want", BAD_TABLES + BAD_HEADS)
def test_decode_refuses_shapes(lib, change, want):
    assert _decode(lib, _shape(**change)) == want
    assert lib.rbs_paged_decode_workspace_bytes(_shape(**change)) == 0


@pytest.mark.parametrize("name", ["q", "k", "v", "o"])
@pytest.mark.parametrize("bad", BAD_ROWS)
def test_decode_refuses_tensors(lib, name, bad):
    assert _decode(lib, _shape(), **{name: bad}) == INVALID


@pytest.mark.parametrize("args", [dict(table=None), dict(lens=None), dict(scale=NAN), dict(scale=INF)])
def test_decode_refuses_arguments(lib, args):
    assert _decode(lib, _shape(), **args) == INVALID


@pytest.mark.parametrize("scale", [3e38, -2.4e38])
def test_decode_refuses_scales_that_are_infinite_in_units_of_log_2(lib, scale):
    assert _decode(lib, _shape(), scale=scale) == INVALID


def test_decode_refuses_tables_of_too_many_tiles(lib):
    big = dict(n_seqs=1 << 13, n_q_heads=64, n_kv_heads=64, max_pages=1 << 17, table_stride=1 << 17)
    assert _decode(lib, _shape(**big)) == UNSUPPORTED


@pytest.mark.parametrize("args", [dict(ws=None), dict(ws=0x100080), dict(n=0), dict(n=-1)])
def test_decode_refuses_workspaces(lib, args):
    if args.get("n") == -1:
        args = dict(n=lib.rbs_paged_decode_workspace_bytes(_shape()) - 1)
    assert _decode(lib, _shape(), **args) == WORKSPACE


def test_calls_refuse_host_tensors():
    x, ints = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache = torch.zeros(3, 16, 4, 128, dtype=torch.bfloat16)
    table = torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_qk_norm_rope(x, x, ints, None)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_paged_decode(x, cache, cache, table, ints, workspace=ints)
    with pytest.raises(RbsError, match="CUDA"):
        rbs_paged_extend(ints, ints, table, ints, 16, 3, 4)


# ------------------------------------------------------------------------------------------------ pins of the oracle


def test_oracle_rotation_keeps_lengths_and_depends_on_distances_only():
    g = np.random.default_rng(1)
    q, k = g.standard_normal((2, 1, 1, 128))
    f = 1e4 ** (-np.arange(64) / 64)
    for interleaved in (False, True):
        turned = lambda x, p: so.norm_rope(x[None], np.array([p]), f, interleaved=interleaved)[0].ravel()  # noqa: E731
        assert np.allclose(np.linalg.norm(turned(q, 777)), np.linalg.norm(q), rtol=1e-12)
        assert np.allclose(turned(q, 1000) @ turned(k, 900), turned(q, 107) @ turned(k, 7), rtol=1e-9)
        assert np.array_equal(turned(q, 0), q.ravel())


def test_oracle_norm_has_unit_mean_square_and_leaves_the_rest_of_the_head():
    x = np.random.default_rng(2).standard_normal((3, 2, 128)) * 7
    y, _ = so.norm_rope(x, np.arange(3), np.array([0.5, 0.1]), np.ones(128), eps=0.0)
    assert np.allclose((y * y).mean(-1), 1.0)
    assert np.allclose(y[..., 4:], x[..., 4:] / np.sqrt((x * x).mean(-1, keepdims=True)))


def test_oracle_decode_of_one_token_is_its_value_and_of_equal_keys_the_mean():
    g = np.random.default_rng(3)
    q, k, v = g.standard_normal((2, 2, 128)), np.zeros((2, 4, 1, 128)), g.standard_normal((2, 4, 1, 128))
    out, lse, _ = so.decode(q, k, v, np.array([[1, 0], [0, -1]]), [1, 3])
    assert np.allclose(out[0, 0], v[1, 0, 0]) and np.allclose(out[1, 1], v[0, :3, 0].mean(0))
    assert np.allclose(lse, np.log([[1, 1], [3, 3]]))
    assert np.all(so.decode(q, k, v, np.array([[1, 0], [0, -1]]), [0, 8])[1][0] == -np.inf)


def test_oracle_extend_gives_every_token_a_place_of_its_own():
    table, lens, cu, pos, slots, used = so.extend([3, 0, 4], [6, 0, 1], np.array([[9, -1, -1], [-1] * 3, [8, -1, -1]]), [0, 1, 2, 3], 4, 10, 9)
    assert table.tolist() == [[9, 0, 1], [-1] * 3, [8, 2, -1]] and used == 3
    assert lens.tolist() == [9, 0, 5] and cu.tolist() == [0, 6, 6, 7]
    assert pos.tolist() == [3, 4, 5, 6, 7, 8, 4, 0, 0]
    assert slots.tolist() == [39, 0, 1, 2, 3, 4, 8, -1, -1]


def test_rope_frequencies():
    f, m = rope_frequencies(64, 1e4, device="cpu")
    want = 1e4 ** (-np.arange(32) / 32)
    assert m == 1.0 and f.dtype == torch.float32 and np.allclose(f.numpy(), want, rtol=1e-7)
    assert np.allclose(rope_frequencies(64, 1e4, scaling="linear", factor=4.0, device="cpu")[0].numpy(), want / 4, rtol=1e-7)
    ntk = rope_frequencies(64, 1e4, scaling="ntk", factor=4.0, device="cpu")[0].numpy()
    assert np.isclose(ntk[0], want[0]) and np.isclose(ntk[-1], want[-1] / 4, rtol=1e-6)
    yarn, m = rope_frequencies(64, 1e4, scaling="yarn", factor=4.0, trained_len=4096, device="cpu")
    turns = 4096 * want / (2 * np.pi)
    ratio = yarn.numpy() / want
    assert np.isclose(m, 0.1 * np.log(4.0) + 1.0)
    assert np.allclose(ratio[turns > 45], 1.0, rtol=1e-6) and np.allclose(ratio[turns < 0.7], 0.25, rtol=1e-6)
    assert (np.diff(ratio) <= 1e-7).all()
    for args in ((60, 1e4), (0, 1e4), (136, 1e4), (64, 1.0)):
        with pytest.raises(RbsError):
            rope_frequencies(*args, device="cpu")
    for more in ({"scaling": "other"}, {"scaling": "yarn", "factor": 2.0}, {"factor": 0.5}):
        with pytest.raises(RbsError):
            rope_frequencies(64, 1e4, device="cpu", **more)


def test_a_shortage_of_pages_can_be_seen_until_its_sequences_end():
    """Three sequences on a pool of six pages: the second one's third page and the last one's only page were not there."""
    cache = PagedCache(1, 6, 4, 1, 4, 5, "cpu")
    cache.block_table[0, :2], cache.block_table[1, :2], cache.block_table[2, :2] = (torch.tensor(p, dtype=torch.int32) for p in ([4, 1], [0, 2], [5, 3]))
    cache.lens.copy_(torch.tensor([8, 9, 5, 1]))
    cache.used.fill_(8)
    assert cache.short() == [1, 3]
    assert cache.release([0]) == [1, 3] and int(cache.used) == 0      # pages are free again, tokens are still missing
    assert cache.short() == [1, 3] and cache.release([]) == [1, 3]
    assert cache.release([3]) == [1] and cache.release([1]) == []
    assert sorted(cache.free_pages[cache.free_pages >= 0].tolist()) == [0, 1, 2, 4] and cache.lens.tolist() == [0, 0, 5, 0]


def test_the_library_builds_without_a_pytorch_with_cuda(lib, tmp_path, monkeypatch):
    """Only the marshalling module needs one."""
    from paper_2609_20971_b200 import build
    monkeypatch.setattr(build, "NATIVE", str(tmp_path / "_native.so"))
    monkeypatch.setattr(build, "NATIVE_STAMP", str(tmp_path / "_native.stamp"))
    monkeypatch.setattr(torch.version, "cuda", None)
    assert build.build_library() == build.LIB and not (tmp_path / "_native.so").exists()
    with pytest.raises(RuntimeError):
        build.build_native()


def test_the_marshalling_module_is_rebuilt_for_another_pytorch(lib, tmp_path, monkeypatch):
    from paper_2609_20971_b200 import build
    assert not build.needs_native()
    stamp = tmp_path / "_native.stamp"
    monkeypatch.setattr(build, "NATIVE_STAMP", str(stamp))
    assert build.needs_native()
    stamp.write_text(build.native_stamp())
    assert not build.needs_native()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.needs_native()
