"""What the calls on the 4-bit pages take and refuse before a GPU is asked: layouts that torch gives to keys and values of one token,
one layer, one head; limits.  Tensors of the host pass the checks of layout and are refused for their device, or reach a library
that only notes what it is given."""
import ctypes

import pytest
import torch

import paper_2502_11101_b200 as cf
from paper_2502_11101_b200 import binding
from paper_2502_11101_b200 import build as cf_build
from paper_2502_11101_b200 import marshal_ctypes as M

FAKE = 4096


@pytest.fixture(scope="module")
def lib():
    cf_build.build()
    return cf.load_library()


def _pages(n_pages=10, page_rows=32):
    return cf.cf_pages(3, page_rows, n_pages, 4, FAKE, FAKE, FAKE, FAKE, FAKE)


def _cut(layers, requests, tokens, heads, dim, pad, dtype=torch.bfloat16):
    """Keys and values cut out of a fused projection [layers, requests, tokens, K | V | rest]."""
    n = heads * dim
    wide = torch.zeros((layers, requests, tokens, 2 * n + pad), dtype=dtype)
    return wide[..., :n].unflatten(-1, (heads, dim)), wide[..., n:2 * n].unflatten(-1, (heads, dim))


class Noting:
    """In place of the library: what a call is given."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        if name == "cf_kv4_layer_bytes":
            return lambda g, p: 0
        return lambda *a: self.seen.append((name, a)) or 0


# layers, requests, tokens, heads, dim, padding
SHAPES = [(1, 8, 1, 4, 128, 8), (1, 1, 1, 4, 128, 8), (3, 8, 1, 4, 128, 64), (3, 1, 1, 2, 64, 8), (1, 1, 5, 2, 64, 16), (2, 7, 3, 1, 64, 8),
          (2, 1, 4, 1, 128, 0), (1, 5, 1, 1, 64, 40)]


@pytest.mark.parametrize("layers,requests,tokens,heads,dim,pad", SHAPES)
def test_rows_cut_out_of_a_fused_projection(lib, monkeypatch, layers, requests, tokens, heads, dim, pad):
    geom, pages = cf.make_geom(heads, heads, dim, torch.bfloat16, 4096, 1e4), _pages()
    k, v = _cut(layers, requests, tokens, heads, dim, pad)
    pool = torch.zeros((layers, cf.cf_kv4_layer_bytes(geom, pages)), dtype=torch.uint8)
    slots = torch.zeros((requests, tokens), dtype=torch.int64)
    row = 2 * heads * dim + pad
    native = binding._load_native(cf_build.NATIVE_PATH)
    for module in (M, native):
        for call in (module.kv4_write, module.kv4_read):
            with pytest.raises(AssertionError, match="current device"):      # the layout is taken, the host's tensors are not
                call(geom, pages, pool, slots, k, v, 0)
    note = Noting()
    monkeypatch.setattr(M, "_require_here", lambda *t: None)
    monkeypatch.setattr(binding, "load_library", lambda: note)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    for call in (M.kv4_write, M.kv4_read):
        call(geom, pages, pool, slots, k, v, None)
    (_, w), (_, r) = note.seen
    n = requests * tokens
    apart = row if n > 1 else heads * dim
    between = n * row if layers > 1 else 0
    assert w[2:9] == (layers, n, slots.data_ptr(), k.data_ptr(), v.data_ptr(), between, apart)
    assert r[2:5] == (layers, n, slots.data_ptr()) and r[9:11] == (between, apart)


@pytest.mark.parametrize("module", ["native", "ctypes"])
def test_a_dimension_of_one_may_have_any_stride(lib, module):
    """Layers, rows and heads of which there is one."""
    module = binding._load_native(cf_build.NATIVE_PATH) if module == "native" else M
    geom, pages = cf.make_geom(1, 1, 64, torch.bfloat16, 4096, 1e4), _pages()
    base = torch.zeros(4096, dtype=torch.bfloat16)
    pool = torch.zeros(1 << 20, dtype=torch.uint8).as_strided((1, cf.cf_kv4_layer_bytes(geom, pages)), (3, 1))
    slots = torch.zeros(6, dtype=torch.int64)
    k = base.as_strided((1, 6, 1, 1, 64), (7, 72, 5, 3, 1))
    v = base.as_strided((1, 6, 1, 1, 64), (9, 72, 1, 4096, 1))
    for call in (module.kv4_write, module.kv4_read):
        with pytest.raises(AssertionError, match="current device"):
            call(geom, pages, pool, slots, k, v, 0)
        with pytest.raises(AssertionError, match="one shape and stride"):
            call(geom, pages, pool, slots, k, base.as_strided((1, 6, 1, 1, 64), (7, 80, 5, 3, 1)), 0)
        with pytest.raises(AssertionError, match="one behind the other"):
            call(geom, pages, pool, slots, *[base.as_strided((1, 2, 3, 1, 64), (7, 256, 64, 64, 1))] * 2, 0)
    q = base.as_strided((1, 3, 1, 1, 64), (3, 64, 5, 9, 1))
    with pytest.raises(AssertionError, match="current device"):
        module.kv4_attn(geom, pages, pool, q, q, torch.zeros(1 << 20, dtype=torch.uint8), None, 0.0, 0)


def test_one_layer_has_no_distance_to_the_next(lib, monkeypatch):
    geom, pages, note = cf.make_geom(1, 1, 64, torch.bfloat16, 4096, 1e4), _pages(), Noting()
    pool = torch.zeros(1 << 20, dtype=torch.uint8).as_strided((1, cf.cf_kv4_layer_bytes(geom, pages)), (3, 1))
    q = torch.zeros(4096, dtype=torch.bfloat16).as_strided((1, 3, 1, 1, 64), (3, 64, 5, 9, 1))
    monkeypatch.setattr(M, "_require_here", lambda *t: None)
    monkeypatch.setattr(binding, "load_library", lambda: note)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    M.kv4_attn(geom, pages, pool, q, q, torch.zeros(1 << 20, dtype=torch.uint8), None, 0.0, None)
    (_, a), = note.seen
    assert (a[5], a[7], a[10]) == (0, 0, 0)


@pytest.mark.parametrize("module", ["native", "ctypes"])
@pytest.mark.parametrize("shape", [(2, 0, 3, 2, 64), (2, 3, 0, 2, 64), (1, 0, 2, 64)])
def test_no_rows_pass_the_checks_of_layout(lib, module, shape):
    module = binding._load_native(cf_build.NATIVE_PATH) if module == "native" else M
    geom, pages = cf.make_geom(2, 2, 64, torch.bfloat16, 4096, 1e4), _pages()
    pool = torch.zeros((shape[0], cf.cf_kv4_layer_bytes(geom, pages)), dtype=torch.uint8)
    k = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(AssertionError, match="current device"):
        module.kv4_write(geom, pages, pool, torch.zeros(0, dtype=torch.int64), k, k, 0)


def test_limits_of_waits_that_make_no_sense_are_refused(lib):
    pages, geom, ref = _pages(), cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), ctypes.byref
    layer = cf.cf_kv4_layer_bytes(geom, pages)

    def call(limit, ws_bytes):
        return lib.cf_debug_kv4_attn(ref(geom), ref(pages), 1, 1, FAKE, 0, FAKE, layer, 0.0, FAKE, 0, None, FAKE, ws_bytes, limit, 1, None)

    for limit in (0, -1, 2000000001):
        assert call(limit, 1 << 40) == cf.CF_ERR_INVALID_ARG
    assert call(1000, 0) == cf.CF_ERR_WORKSPACE


def _way(hq, hkv, dim, dtype, requests, page_rows, cols, q_len, layers=1):
    pages = cf.cf_pages(requests, page_rows, 4 * requests * cols, cols, FAKE, FAKE, FAKE, FAKE, FAKE)
    return cf.cf_debug_kv4_attn_kernel(cf.make_geom(hq, hkv, dim, dtype, 32768, 1e6), pages, q_len, layers)


WARPS, CTAS, CLUSTERS, TCGEN05 = 0, 1, 2, 3


@pytest.mark.parametrize("want,call", [
    # the tensor cores from 57 query columns of a kv head and eight units of 128 on, bf16 and head_dim 128
    (TCGEN05, (28, 4, 128, torch.bfloat16, 4, 64, 252, 24)), (TCGEN05, (8, 1, 128, torch.bfloat16, 8, 16, 30, 8)),
    (TCGEN05, (57, 1, 128, torch.bfloat16, 8, 16, 3000, 1)), (CTAS, (56, 1, 128, torch.bfloat16, 8, 16, 3000, 1)),
    (CTAS, (8, 1, 128, torch.bfloat16, 7, 16, 3000, 8)), (TCGEN05, (8, 1, 128, torch.bfloat16, 4, 16, 3000, 17)),
    (CTAS, (28, 4, 64, torch.bfloat16, 4, 64, 252, 24)), (CTAS, (28, 4, 128, torch.float32, 4, 64, 252, 24)),
    # clusters by the room of the table, fewer than six steps of 32 rows to a warp (nine with few columns), 8 CTAs of 4 (8) warps
    (CLUSTERS, (12, 2, 128, torch.bfloat16, 1, 64, 95, 1)), (CTAS, (12, 2, 128, torch.bfloat16, 1, 64, 96, 1)),
    (CLUSTERS, (2, 2, 128, torch.bfloat16, 1, 64, 287, 1)), (CTAS, (2, 2, 128, torch.bfloat16, 1, 64, 288, 1)),
    (CTAS, (12, 2, 128, torch.bfloat16, 1, 64, 512, 1)),
    # shares of single warps where units are many
    (CTAS, (28, 4, 128, torch.bfloat16, 88, 32, 190, 1)), (WARPS, (28, 4, 128, torch.bfloat16, 89, 32, 190, 1)),
    (WARPS, (4, 4, 128, torch.bfloat16, 700, 16, 5, 1)), (CTAS, (32, 32, 128, torch.bfloat16, 8, 64, 340, 1))])
def test_how_a_call_is_done(lib, want, call):
    """On both sides of the lines of the dispatch, for 148 multiprocessors."""
    assert _way(*call) == want


def test_how_a_call_is_done_is_asked_properly(lib):
    pages, geom, ref = _pages(), cf.make_geom(4, 2, 64, cf.CF_BF16, 4096, 1e4), ctypes.byref
    assert lib.cf_debug_kv4_attn_kernel(ref(geom), ref(pages), 0, 1, FAKE) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_debug_kv4_attn_kernel(ref(geom), ref(pages), 1, 1, None) == cf.CF_ERR_INVALID_ARG


def test_pages_of_another_device_are_refused(lib, monkeypatch):
    """Their arrays would be read and written from a device that they are not on."""
    geom, pages = cf.make_geom(1, 1, 64, torch.bfloat16, 4096, 1e4), _pages()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    pages.device = 1
    rows, slots, pool = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros((1, cf.cf_kv4_layer_bytes(geom, pages)), dtype=torch.uint8)
    k, q, work = torch.zeros((1, 3, 1, 64), dtype=torch.bfloat16), torch.zeros((1, 3, 1, 1, 64), dtype=torch.bfloat16), torch.zeros(1 << 20, dtype=torch.uint8)
    for call in (lambda: cf.cf_pages_init(pages), lambda: cf.cf_pages_status(pages), lambda: M.pages_resize(pages, rows, 0, slots, None),
                 lambda: M.kv4_write(geom, pages, pool, slots, k, k, None), lambda: M.kv4_read(geom, pages, pool, slots, k, k, None),
                 lambda: M.kv4_attn(geom, pages, pool, q, q, work, None, 0.0, None), lambda: cf.cf_debug_kv4_attn(geom, pages, pool, q, q, work, 1000)):
        with pytest.raises(AssertionError, match="pages on the current device"):
            call()


@pytest.mark.parametrize("n_rows", [(1 << 31) - 1, (1 << 31) - 3])
def test_rows_that_are_too_many_are_refused(lib, n_rows):
    """Their number is rounded up to fours, beyond 32 bits."""
    geom, pages, ref = cf.make_geom(8, 8, 64, cf.CF_BF16, 4096, 1e4), _pages(), ctypes.byref
    layer, stride = cf.cf_kv4_layer_bytes(geom, pages), n_rows * 512
    assert lib.cf_kv4_write(ref(geom), ref(pages), 4, n_rows, FAKE, FAKE, FAKE, stride, 512, FAKE, layer, None) == cf.CF_ERR_INVALID_ARG
    assert lib.cf_kv4_read(ref(geom), ref(pages), 4, n_rows, FAKE, FAKE, layer, FAKE, FAKE, stride, 512, None) == cf.CF_ERR_INVALID_ARG


def test_pages_and_table_entries_fit_32_bits_together(lib):
    """The stack's height while pages come back: what it holds and what all requests release, whatever the lengths say."""
    geom, ref = cf.make_geom(1, 1, 64, cf.CF_BF16, 4096, 1e4), ctypes.byref
    for n_requests, cols, n_pages, fine in ((1 << 10, 1 << 20, (1 << 30) - 1, True), (1 << 10, 1 << 20, 1 << 30, False), (1, 1, (1 << 31) - 1, False),
                                            (1, 1, (1 << 31) - 2, True), (1 << 10, (1 << 21) - 1, 1024, False), (1 << 10, (1 << 21) - 1, 1023, True)):
        pages = cf.cf_pages(n_requests, 16, n_pages, cols, FAKE, FAKE, FAKE, FAKE, FAKE)
        assert (cf.cf_kv4_layer_bytes(geom, pages) != 0) == fine, (n_requests, cols, n_pages)
        if not fine:
            assert lib.cf_pages_resize(ref(pages), FAKE, 0, 0, None, None) == cf.CF_ERR_INVALID_ARG
            assert lib.cf_pages_init(ref(pages), None) == cf.CF_ERR_INVALID_ARG


@pytest.mark.parametrize("module", ["native", "ctypes"])
def test_a_workspace_has_the_bytes_that_it_counts(lib, module):
    """A view with gaps, or of the same byte many times, has fewer behind its address."""
    module = binding._load_native(cf_build.NATIVE_PATH) if module == "native" else M
    geom, pages = cf.make_geom(1, 1, 64, torch.bfloat16, 4096, 1e4), _pages()
    pool = torch.zeros((1, cf.cf_kv4_layer_bytes(geom, pages)), dtype=torch.uint8)
    q = torch.zeros((1, 3, 1, 1, 64), dtype=torch.bfloat16)
    need = cf.cf_kv4_attn_workspace_bytes(geom, pages, 1, 1)
    for work in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros((need // 64, 128), dtype=torch.uint8)[:, :64]):
        with pytest.raises(AssertionError, match="workspace"):
            module.kv4_attn(geom, pages, pool, q, q, work, None, 0.0, 0)
