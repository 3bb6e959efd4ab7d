"""Pins of the paged-cache oracle: closed forms of the format, a block's places, the pages' invariants, and the library's
host-side refusals, none of which needs a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2502_11101_b200 as cf
from oracle import paged_oracle as P
from paper_2502_11101_b200 import build as cf_build


def test_numbers_that_the_format_has_come_back():
    for scale in (1.0, 2.0 ** -40, 1.5, 0.0078125 * 251):
        x = np.array([s * l * scale for l in P.LEVELS for s in (1, -1)] * 2)
        codes, got = P.quantise_group(x)
        assert got == P.round_to_bf16(scale) and np.array_equal(P.numbers(np.array(codes)[None], np.array([[got]]))[0], x * got / scale)


def test_ties_go_to_the_even_code():
    halves = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4)
    codes, scale = P.quantise_group(halves)
    assert scale == 1.0 and codes[:8] == [0, 2, 2, 4, 4, 6, 6, 7]
    codes, _ = P.quantise_group(-halves)
    assert codes[:8] == [8, 10, 10, 12, 12, 14, 14, 15]


def test_groups_that_are_not_kept_as_numbers():
    x = np.ones(32)
    x[5] = np.inf
    codes, scale = P.quantise_group(x)
    assert np.isnan(scale) and not any(codes)
    assert P.quantise_group(np.zeros(32)) == ([0] * 32, 0.0)
    assert P.quantise_group(np.full(32, 1e-38 * 6)) == ([0] * 32, 0.0)
    x = np.zeros(32)
    x[0] = 2.0 ** -126 * 6
    assert P.quantise_group(x)[1] == 2.0 ** -126


def test_many_groups_are_kept_as_one_by_one():
    rng = np.random.default_rng(3)
    x = np.round(rng.standard_normal((200, 32)) * 8) / 8 * np.exp2(rng.integers(-100, 100, (200, 1)))
    x[7, 3], x[8, 0], x[9] = np.nan, np.inf, 0.0
    codes, scales = P.quantise(x)
    for i, group in enumerate(x):
        one = P.quantise_group(group)
        assert one[0] == codes[i].tolist() and (one[1] == scales[i, 0] or np.isnan(one[1]) and np.isnan(scales[i, 0]))


def test_a_rounding_is_at_most_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp(rng.uniform(-20, 20, (50, 1)))
    codes, scales = P.quantise(x)
    off = np.abs(P.numbers(codes, scales) - x) / np.repeat(scales, 32, -1)
    # steps are 0.5, 1 and 2 scales wide; a scale rounded down by 2^-9 leaves the largest 6 * 2^-9 above 6
    assert off.max() <= 1.0 + 6 * 2.0 ** -9


@pytest.mark.parametrize("dim", [64, 128])
def test_a_block_has_one_place_for_everything(dim):
    k, v, ks, vs = P.places(dim)
    taken = np.concatenate([k.ravel(), v.ravel()] + [2 * (s.ravel() + i) + h for s in (ks, vs) for i in (0, 1) for h in (0, 1)])
    assert sorted(taken) == list(range(36 * dim))


def test_growing_and_shrinking_back_leaves_the_stack():
    rng = np.random.default_rng(1)
    pool = P.Pool(9, 16, 60, 12)
    pool.resize(rng.integers(0, 70, 9), 0, None)
    before = (list(pool.free), [list(t) for t in pool.table])
    rows = list(pool.rows)
    pool.resize([r + int(g) for r, g in zip(rows, rng.integers(0, 40, 9))], 0, None)
    pool.resize(rows, 0, None)
    assert before == (pool.free, pool.table) and not pool.status


def test_pages_are_had_once():
    rng = np.random.default_rng(2)
    pool = P.Pool(7, 32, 25, 6)
    for _ in range(50):
        pool.resize(rng.integers(-1, 200, 7), 0, None)
        held = [p for t in pool.table for p in t] + pool.free
        assert sorted(held) == list(range(25))
        assert all(len(t) == -(-r // 32) for t, r in zip(pool.table, pool.rows))


# ------------------------------------------------------------------------------------------------ host-side refusals

FAKE = 4096                                          # any aligned non-null address: refused calls dereference nothing


def _pages(**kw):
    sizes = dict(n_requests=3, page_rows=32, n_pages=10, table_cols=4, table=FAKE, rows=FAKE, free_pages=FAKE, free_count=FAKE, status=FAKE)
    sizes.update(kw)
    return cf.cf_pages(*[sizes[n] for n, _ in cf.cf_pages._fields_])


@pytest.fixture(scope="module")
def lib():
    cf_build.build()
    return cf.load_library()


BAD_PAGES = [dict(n_requests=0), dict(n_requests=-1), dict(n_requests=(1 << 20) + 1), dict(page_rows=0), dict(page_rows=24), dict(page_rows=8),
             dict(n_pages=0), dict(table_cols=0), dict(table_cols=1 << 27), dict(n_requests=1 << 20, table_cols=1 << 12), dict(table=None),
             dict(rows=None), dict(free_pages=None), dict(free_count=None), dict(status=None)]


@pytest.mark.parametrize("bad", BAD_PAGES, ids=[str(b) for b in BAD_PAGES])
def test_descriptors_that_make_no_sense_are_refused(lib, bad):
    pages, geom, ref = _pages(**bad), cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), ctypes.byref
    assert lib.cf_pages_init(ref(pages), None) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_pages_resize(ref(pages), FAKE, 0, 1, FAKE, None) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_pages_status(ref(pages), None) == cf.CF_ERR_INVALID_ARG
    assert cf.cf_kv4_layer_bytes(geom, pages) == 0 and cf.cf_kv4_attn_workspace_bytes(geom, pages, 1, 1) == 0
    assert lib.cf_kv4_write(ref(geom), ref(pages), 1, 1, FAKE, FAKE, FAKE, 128, 128, FAKE, 0, None) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_kv4_read(ref(geom), ref(pages), 1, 1, FAKE, FAKE, 0, FAKE, FAKE, 128, 128, None) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_kv4_attn(ref(geom), ref(pages), 1, 1, FAKE, 0, FAKE, 0, 0.0, FAKE, 0, None, FAKE, 1 << 40, None) == cf.CF_ERR_INVALID_ARG


def test_pool_and_workspace_sizes(lib):
    assert ctypes.sizeof(cf.cf_pages) == 56
    geom = cf.make_geom(12, 2, 128, cf.CF_BF16, 32768, 1e6)
    assert cf.cf_kv4_layer_bytes(geom, _pages()) == 10 * 2 * 2 * 18 * 128
    assert cf.cf_kv4_layer_bytes(geom, _pages(n_pages=1 << 24, page_rows=64)) == (1 << 24) * 2 * 4 * 18 * 128      # beyond 32 bits
    assert cf.cf_kv4_attn_workspace_bytes(geom, _pages(), 1, 1) > 0
    for q_len, layers in ((0, 1), (-1, 1), (1, 0), (1, 65536), (1 << 23, 1)):
        assert cf.cf_kv4_attn_workspace_bytes(geom, _pages(), q_len, layers) == 0
    assert cf.cf_kv4_layer_bytes(cf.make_geom(12, 2, 96, cf.CF_BF16, 32768, 1e6), _pages()) == 0


def test_calls_that_make_no_sense_are_refused(lib):
    pages, geom, ref = _pages(), cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), ctypes.byref
    bad = cf.CF_ERR_INVALID_ARG
    assert lib.cf_pages_resize(ref(pages), None, 0, 1, FAKE, None) == bad
    assert lib.cf_pages_resize(ref(pages), FAKE, 0, -1, FAKE, None) == bad
    assert lib.cf_pages_resize(ref(pages), FAKE, 0, 0, FAKE, None) == bad            # slots without room
    assert lib.cf_pages_resize(ref(pages), FAKE, 0, 1, None, None) == bad            # room without slots
    layer = cf.cf_kv4_layer_bytes(geom, pages)

    def write(layers=1, n=5, slots=FAKE, k=FAKE, v=FAKE, kv_stride=5 * 128, row_stride=128, kv4=FAKE, kv4_stride=layer):
        return lib.cf_kv4_write(ref(geom), ref(pages), layers, n, slots, k, v, kv_stride, row_stride, kv4, kv4_stride, None)

    def read(layers=1, n=5, slots=FAKE, k=FAKE, v=FAKE, kv_stride=5 * 128, row_stride=128, kv4=FAKE, kv4_stride=layer):
        return lib.cf_kv4_read(ref(geom), ref(pages), layers, n, slots, kv4, kv4_stride, k, v, kv_stride, row_stride, None)

    for call in (write, read):
        assert call(n=0) == cf.CF_OK                                                  # nothing to do
        for kw in (dict(layers=0), dict(n=-1), dict(slots=None), dict(k=None), dict(v=None), dict(kv4=None), dict(k=FAKE + 8), dict(v=FAKE + 2),
                   dict(kv4=FAKE + 8), dict(row_stride=127), dict(row_stride=132), dict(kv4_stride=layer + 8), dict(kv_stride=5 * 128 + 4),
                   dict(layers=2, kv_stride=4 * 128), dict(layers=2, kv4_stride=layer - 16)):
            assert call(**kw) == bad, kw

    need = cf.cf_kv4_attn_workspace_bytes(geom, pages, 2, 1)

    def attn(layers=1, q_len=2, q=FAKE, q_stride=3 * 2 * 4 * 64, kv4=FAKE, kv4_stride=layer, out=FAKE, out_stride=3 * 2 * 4 * 64, ws=FAKE, ws_bytes=need):
        return lib.cf_kv4_attn(ref(geom), ref(pages), layers, q_len, q, q_stride, kv4, kv4_stride, 0.0, out, out_stride, None, ws, ws_bytes, None)

    for kw in (dict(layers=0), dict(q_len=0), dict(q=None), dict(kv4=None), dict(out=None), dict(ws=None), dict(q=FAKE + 8), dict(out=FAKE + 8),
               dict(kv4=FAKE + 8), dict(q_stride=12), dict(out_stride=12), dict(kv4_stride=8), dict(layers=2, q_stride=128),
               dict(layers=2, out_stride=128), dict(layers=2, kv4_stride=layer - 16)):
        assert attn(**kw) == bad, kw
    assert attn(ws=FAKE + 64) == cf.CF_ERR_WORKSPACE and attn(ws_bytes=need - 1) == cf.CF_ERR_WORKSPACE
    for odd in (cf.make_geom(4, 2, 96, cf.CF_BF16, 4096, 1e4), cf.cf_geom(4, 2, 64, 7, 0, 4096, 1e4)):
        assert lib.cf_kv4_write(ref(odd), ref(pages), 1, 1, FAKE, FAKE, FAKE, 256, 256, FAKE, 0, None) == cf.CF_ERR_UNSUPPORTED
        assert lib.cf_kv4_attn(ref(odd), ref(pages), 1, 1, FAKE, 0, FAKE, 0, 0.0, FAKE, 0, None, FAKE, 1 << 40, None) == cf.CF_ERR_UNSUPPORTED


def test_the_binding_refuses_other_shapes_types_and_devices():
    """Before anything reaches the library; tensors of the host are among what is refused."""
    from paper_2502_11101_b200 import marshal_ctypes as M
    geom, pages = cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), _pages()
    rows, slots = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 5), dtype=torch.int64)
    pool = torch.zeros((2, cf.cf_kv4_layer_bytes(geom, pages)), dtype=torch.uint8)
    k = torch.zeros((2, 3, 5, 2, 64), dtype=torch.bfloat16)
    q, work = torch.zeros((2, 3, 1, 4, 64), dtype=torch.bfloat16), torch.zeros(1 << 20, dtype=torch.uint8)
    lse = torch.zeros((2, 3, 4, 1))
    bad = [lambda: M.pages_resize(pages, rows, 0, slots, None), lambda: M.pages_resize(pages, rows.long(), 0, slots, None),
           lambda: M.pages_resize(pages, rows[:2], 0, slots, None), lambda: M.pages_resize(pages, rows, 0, slots.int(), None),
           lambda: M.pages_resize(pages, rows, 0, slots.flatten()[:14], None), lambda: M.pages_resize(pages, rows, 0, slots.T, None)]
    for call in (M.kv4_write, M.kv4_read):
        bad += [lambda c=call: c(geom, pages, pool, slots, k, k, None), lambda c=call: c(geom, pages, pool, slots, k.float(), k.float(), None),
                lambda c=call: c(geom, pages, pool, slots, k, k[:, :, :4], None), lambda c=call: c(geom, pages, pool, slots[:2], k, k, None),
                lambda c=call: c(geom, pages, pool[:1], slots, k, k, None), lambda c=call: c(geom, pages, pool.float(), slots, k, k, None),
                lambda c=call: c(geom, pages, pool, slots, k.transpose(1, 2), k.transpose(1, 2), None),
                lambda c=call: c(geom, pages, pool, slots, k[..., :32], k[..., :32], None), lambda c=call: c(geom, pages, pool, slots.int(), k, k, None)]
    bad += [lambda: M.kv4_attn(geom, pages, pool, q, q.clone(), work, lse, 0.0, None), lambda: M.kv4_attn(geom, pages, pool, q[0], q[0], work, lse, 0.0, None),
            lambda: M.kv4_attn(geom, pages, pool, q, q.float(), work, lse, 0.0, None), lambda: M.kv4_attn(geom, pages, pool, q[:, :2], q[:, :2], work, None, 0.0, None),
            lambda: M.kv4_attn(geom, pages, pool[:1], q, q, work, lse, 0.0, None), lambda: M.kv4_attn(geom, pages, pool, q, q, work, lse[:1], 0.0, None),
            lambda: M.kv4_attn(geom, pages, pool, q, q, work, lse.double(), 0.0, None)]
    for i, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
            pytest.fail("call %d was not refused" % i)


def test_the_binding_refuses_small_pools_other_types_and_no_requests():
    """Each before the device of the tensors is looked at: the message says so."""
    from paper_2502_11101_b200 import marshal_ctypes as M
    geom, pages = cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), _pages()
    slots, layer = torch.zeros((3, 5), dtype=torch.int64), cf.cf_kv4_layer_bytes(geom, pages)
    pool, small = torch.zeros((2, layer), dtype=torch.uint8), torch.zeros((2, layer - 16), dtype=torch.uint8)
    k, q = torch.zeros((2, 3, 5, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 3, 1, 4, 64), dtype=torch.bfloat16)
    work = torch.zeros(1 << 20, dtype=torch.uint8)
    for call in (M.kv4_write, M.kv4_read):
        with pytest.raises(AssertionError, match="fewer bytes"):
            call(geom, pages, small, slots, k, k, None)
        with pytest.raises(AssertionError, match="storage type"):
            call(geom, pages, pool, slots, k.half(), k.half(), None)
    with pytest.raises(AssertionError, match="fewer bytes"):
        M.kv4_attn(geom, pages, small, q, q, work, None, 0.0, None)
    with pytest.raises(AssertionError, match="storage type"):
        M.kv4_attn(geom, pages, pool, q.half(), q.half(), work, None, 0.0, None)
    none = _pages(n_requests=0)
    with pytest.raises(AssertionError, match="one per request"):
        M.pages_resize(none, torch.zeros(0, dtype=torch.int32), 0, torch.zeros((0, 1), dtype=torch.int64), None)
    host = [torch.zeros(n, dtype=torch.int32) for n in ((3, 4), 3, 10, 1, 1)]
    with pytest.raises(AssertionError):
        cf.make_pages(*host, 16)
