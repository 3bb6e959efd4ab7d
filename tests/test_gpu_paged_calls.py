"""Calls on the 4-bit pages that a program makes and that the tests of the operators by themselves do not."""
import numpy as np
import pytest
import torch

import paper_2502_11101_b200 as cf
from oracle import paged_oracle as P
from paper_2502_11101_b200 import marshal_ctypes
from tests.test_gpu_paged import DTYPES, Pages, _attend, _check_attention, _filled, _same_pages

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "ctypes"])
def marshal(request, monkeypatch):
    if request.param == "ctypes":
        monkeypatch.setattr(cf.binding, "_NATIVE", marshal_ctypes)
    return request.param


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("requests,tokens", [(1, 1), (8, 1), (1, 5), (8, 2)])
def test_rows_out_of_a_fused_projection(marshal, dtype, dim, layers, requests, tokens):
    """A step's keys and values as a projection leaves them, [layers, requests, tokens, K | V | Q]: in, and back into such a buffer."""
    heads, extra, page_rows, n_pages = 4, 24, 32, 5
    n = heads * dim
    geom, pages = cf.make_geom(2 * heads, heads, dim, DTYPES[dtype], 4096, 1e4), Pages(requests, page_rows, n_pages, 2)
    gen = torch.Generator().manual_seed(requests + tokens)
    wide = torch.randn((layers, requests, tokens, 2 * n + extra), generator=gen).to(DTYPES[dtype])
    fused, back = wide.cuda(), torch.full_like(wide, 55.0).cuda()
    k, v, kb, vb = [t[..., i * n:(i + 1) * n].unflatten(-1, (heads, dim)) for t in (fused, back) for i in (0, 1)]
    slots = torch.from_numpy(np.random.default_rng(layers).permutation(n_pages * page_rows)[:requests * tokens].reshape(requests, tokens)).cuda()
    pool = torch.zeros((layers, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8, device="cuda")
    dense = torch.zeros_like(pool)
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k, v)
    cf.cf_kv4_read(geom, pages.desc, pool, slots, kb, vb)
    cf.cf_kv4_write(geom, pages.desc, dense, slots.flatten(), k.flatten(1, 2).contiguous(), v.flatten(1, 2).contiguous())
    torch.cuda.synchronize()
    assert cf.cf_pages_status(pages.desc) == 0 and torch.equal(pool, dense) and pool.any()
    for x, got in ((k, kb), (v, vb)):
        assert torch.equal(got.cpu(), torch.from_numpy(P.numbers(*P.quantise(x.double().cpu().numpy()))).to(DTYPES[dtype]))
    assert (back[..., 2 * n:] == 55.0).all()


# hq, hkv, q_len, columns of the table: short caches by clusters, shares of the line, few columns and many, the tensor-core kernel
FORMS = [(4, 4, 1, 0), (4, 4, 1, 3000), (1, 1, 1, 0), (1, 1, 1, 3000), (8, 1, 1, 0), (8, 1, 1, 3000), (28, 4, 1, 0), (28, 4, 1, 3000), (12, 1, 6, 0),
         (12, 4, 24, 0)]


@pytest.mark.parametrize("pattern", ["one", "pairs"])
@pytest.mark.parametrize("hq,hkv,q_len,cols", FORMS)
def test_a_table_may_name_a_page_twice_in_a_row(hq, hkv, q_len, cols, pattern):
    """Pages of 16 rows: a step's second block is its first one.  As a table of zeros has it (a warm-up, a capture), or a passage
    that is repeated."""
    dim, columns = 128, 20
    geom = cf.make_geom(hq, hkv, dim, torch.bfloat16, 32768, 1e6)
    lengths = [320, 23, 175]
    pages, pool, kept = _filled(geom, hkv, dim, [96, 90, 80], 16, 1, seed=hq, cols=cols or columns)
    _attend(geom, pages, pool, torch.randn((1, 3, q_len, hq, dim), device="cuda").bfloat16())     # leaves other rows in shared memory
    repeated = []
    for b, n in enumerate(lengths):
        at = [0 if pattern == "one" else i // 2 % 5 for i in range(columns)]
        k, v = [np.concatenate([x[16 * i:16 * i + 16] for i in at])[:n] for x in kept[0][b]]
        pages.table[b, :columns] = pages.table[b, torch.tensor(at, device="cuda")].clone()
        repeated.append((k, v))
    pages.rows.copy_(torch.tensor(lengths, dtype=torch.int32))
    q = torch.randn((1, 3, q_len, hq, dim), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, [repeated], dim ** -0.5)


def _marks(work, units):
    """What the attention kernel leaves for the join: a mark of four numbers for each unit, or for each share (an SM's) where those are
    fewer, at the end of the workspace."""
    n = min(units, torch.cuda.get_device_properties(0).multi_processor_count)
    return work[work.numel() - -(-16 * n // 256) * 256:][:16 * n].view(torch.int32).view(n, 4)


@pytest.mark.parametrize("hq,hkv,q_len,requests", [(28, 4, 24, 3), (12, 1, 20, 9), (32, 8, 20, 30)])
def test_waits_of_the_tensor_core_kernel_that_run_out(hq, hkv, q_len, requests):
    """The call ends with an error that the host reads, and without marks that were not written: the join would take anything for
    one, and read and write where it says.  (Here the workspace is all -1, which the join passes over.)"""
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, 128, [700 + 31 * i % 400 for i in range(requests)], 16, 1, seed=hq)
    q = torch.randn((1, requests, q_len, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    right, right_lse = _attend(geom, pages, pool, q)
    units = requests * hkv * -(-hq // hkv * q_len // 128)
    work = torch.empty(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, q_len, 1), dtype=torch.uint8, device="cuda")
    for limit, copies in ((2000000, False), (1, False), (1, True), (20000, True), (2000000, True)):
        work.fill_(255)
        out, lse = torch.full_like(q, 99.0), torch.full_like(right_lse, 99.0)
        pages.status.zero_()
        cf.cf_debug_kv4_attn(geom, pages.desc, pool, q, out, work, limit, copies, lse=lse)
        status, marks = cf.cf_pages_status(pages.desc), _marks(work, units)
        if not copies:
            assert status == cf.CF_ERR_TIMEOUT and (marks == 0).all() and (out == 99.0).all() and (lse == 99.0).all()
        elif status == 0:
            assert torch.equal(out, right) and torch.equal(lse, right_lse)
        else:
            assert status == cf.CF_ERR_TIMEOUT
        assert (marks >= 0).all()
    pages.status.zero_()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0 and torch.equal(out, right) and torch.equal(lse, right_lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,q_len,cols", [(4, 4, 1, 0), (4, 4, 1, 3000), (28, 4, 1, 0), (28, 4, 1, 3000), (12, 1, 2, 0), (12, 1, 2, 3000)])
def test_waits_that_run_out(dtype, hq, hkv, q_len, cols):
    geom = cf.make_geom(hq, hkv, 128, DTYPES[dtype], 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, 128, [700, 40, 333], 32, 1, seed=hq, cols=cols or None)
    q = torch.randn((1, 3, q_len, hq, 128), generator=torch.Generator().manual_seed(4)).to(DTYPES[dtype]).cuda()
    right, right_lse = _attend(geom, pages, pool, q)
    work = torch.full((cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, q_len, 1),), 255, dtype=torch.uint8, device="cuda")
    for limit, copies in ((2000000, False), (1, False), (1, True), (2000000, True)):
        out, lse = torch.full_like(q, 99.0), torch.full_like(right_lse, 99.0)
        pages.status.zero_()
        cf.cf_debug_kv4_attn(geom, pages.desc, pool, q, out, work, limit, copies, lse=lse)
        status = cf.cf_pages_status(pages.desc)
        assert status == cf.CF_ERR_TIMEOUT if not copies else status in (0, cf.CF_ERR_TIMEOUT)
        assert status != 0 or torch.equal(out, right) and torch.equal(lse, right_lse)
    pages.status.zero_()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0 and torch.equal(out, right) and torch.equal(lse, right_lse)


@pytest.mark.parametrize("dtype,dim,heads,page_rows,n_rows,layers,pad", [
    ("bf16", 64, 9, 48, 140001, 1, 0), ("bf16", 128, 7, 16, 100003, 1, 8), ("f32", 128, 5, 64, 63001, 3, 0), ("f32", 64, 13, 32, 90002, 2, 16)])
def test_many_rows_of_several_heads(dtype, dim, heads, page_rows, n_rows, layers, pad):
    """Calls of so many rows that a warp takes several heads of its own, the last of them fewer: as the same rows a few at a time, in
    and out, and as the format says."""
    gen = torch.Generator(device="cuda").manual_seed(n_rows)
    n_pages = n_rows // page_rows + 3
    slots = torch.randperm(n_pages * page_rows, generator=gen, device="cuda")[:n_rows]
    at = torch.randperm(n_rows, generator=gen, device="cuda")
    slots[at[:500]], slots[at[500:510]] = -1, n_pages * page_rows + 3
    slots[-3:] = slots[-3:].abs() % (n_pages * page_rows)
    geom = cf.make_geom(heads, heads, dim, DTYPES[dtype], 4096, 1e4)
    pages = Pages(2, page_rows, n_pages, 4)
    k, v = [(torch.randn((layers, n_rows, heads * dim + pad), generator=gen, device="cuda") * 3).to(DTYPES[dtype])[..., :heads * dim].unflatten(-1, (heads, dim))
            for _ in range(2)]
    k[0, 5, 1, 7], v[-1, -1, -1, 33] = float("inf"), float("nan")
    start = torch.randint(0, 256, (layers, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8, generator=gen, device="cuda")
    pools, backs = [start.clone(), start.clone()], [[torch.full((layers, n_rows, heads, dim), 55.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2)] for _ in range(2)]
    for pool, back, step in zip(pools, backs, (n_rows, 5000)):
        for i in range(0, n_rows, step):
            rows = slice(i, i + step)
            cf.cf_kv4_write(geom, pages.desc, pool, slots[rows], k[:, rows], v[:, rows])
            assert cf.cf_pages_status(pages.desc) in (0, cf.CF_ERR_RANGE)
        for i in range(0, n_rows, step):
            rows = slice(i, i + step)
            cf.cf_kv4_read(geom, pages.desc, pool, slots[rows], back[0][:, rows], back[1][:, rows])
    assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE
    assert torch.equal(pools[0], pools[1]) and not torch.equal(pools[0], start)
    sample = torch.cat([at[500:900], torch.arange(n_rows - 3, n_rows, device="cuda"), torch.arange(8, device="cuda")])
    kept = (slots[sample] >= 0) & (slots[sample] < n_pages * page_rows)
    for x, one, few in zip((k, v), *backs):
        assert torch.equal(one.nan_to_num(nan=1e30), few.nan_to_num(nan=1e30))
        assert (one[:, slots < 0] == 55.0).all() and (one[:, slots >= n_pages * page_rows] == 55.0).all()
        want = torch.from_numpy(P.numbers(*P.quantise(x[:, sample].double().cpu().numpy()))).to(DTYPES[dtype])
        want[:, ~kept.cpu()] = 55.0
        assert torch.equal(one[:, sample].cpu().nan_to_num(nan=1e30), want.nan_to_num(nan=1e30))


@pytest.mark.parametrize("n_requests,page_rows,cols", [(8, 16, 9), (1000, 32, 5), (1024, 16, 6), (2500, 16, 5)])
@pytest.mark.parametrize("max_new", [None, 1, 70])
def test_the_lengths_may_be_the_pages_own_for_any_number_of_requests(n_requests, page_rows, cols, max_new):
    """Eight blocks read the lengths that one of them overwrites, in one round and in several."""
    rng = np.random.default_rng(n_requests)
    n_pages = n_requests * cols * 2 // 3
    got, want = Pages(n_requests, page_rows, n_pages, cols), P.Pool(n_requests, page_rows, n_pages, cols)
    rows = [int(r) for r in rng.integers(0, cols * page_rows // 2, n_requests)]
    got.resize(rows)
    want.resize(rows, 0, None)
    for extra in (1, page_rows + 1, -7, 0, 1, -page_rows, 3):
        extra = min(extra, 1) if max_new == 1 else extra
        slots = None if max_new is None else torch.full((n_requests, max_new), 777, dtype=torch.int64, device="cuda")
        expect = want.resize(list(want.rows), extra, max_new)
        cf.cf_pages_resize(got.desc, got.rows, extra, slots)
        torch.cuda.synchronize()
        _same_pages(got, want)
        assert max_new is None or np.array_equal(slots.cpu().numpy(), np.array(expect))
        assert cf.cf_pages_status(got.desc) in (want.status or {0})
        want.status.clear()
        got.status.zero_()


@pytest.mark.parametrize("hq,hkv,lengths,page_rows,q_len,layers", [
    (28, 4, [130, 24, 10, 0], 32, 24, 1), (6, 2, [333, 50, 200, 65], 32, 20, 1), (4, 1, [300, 17, 64, 63, 65, 128, 1, 0], 16, 15, 1),
    (57, 1, [190, 4, 64], 48, 1, 3), (16, 2, [9000, 3], 64, 100, 1)],
    ids=lambda x: str(x) if isinstance(x, int) else "%dx%d" % (len(x), max(x)))
def test_calls_that_the_tensor_core_kernel_takes(hq, hkv, lengths, page_rows, q_len, layers):
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, 128, lengths, page_rows, layers, seed=q_len)
    assert cf.cf_debug_kv4_attn_kernel(geom, pages.desc, q_len, layers) == 3
    q = torch.randn((layers, len(lengths), q_len, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)
    again, lse2 = _attend(geom, pages, pool, q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("way,hq,hkv,q_len,cols,requests", [(2, 28, 4, 1, 0, 96), (0, 28, 4, 1, 3000, 96), (0, 4, 4, 1, 0, 200), (0, 12, 1, 3, 0, 300), (1, 28, 4, 1, 3000, 3), (1, 4, 4, 1, 3000, 3),
                                                            (1, 12, 1, 3, 3000, 3), (2, 28, 4, 1, 0, 3), (2, 4, 4, 1, 0, 3), (2, 12, 1, 3, 0, 3), (3, 28, 4, 24, 0, 3)])
def test_every_way_of_doing_a_call(way, hq, hkv, q_len, cols, requests):
    """Shares of warps and of CTAs, clusters, the tensor cores: each is what the call takes."""
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, 128, [(37 * i + 290) % 321 for i in range(requests)], 32, 1, seed=hq + q_len, cols=cols or None)
    assert cf.cf_debug_kv4_attn_kernel(geom, pages.desc, q_len, 1) == way
    q = torch.randn((1, requests, q_len, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)


def test_pages_of_another_device_are_refused(marshal):
    geom, pages = cf.make_geom(1, 1, 64, torch.bfloat16, 4096, 1e4), Pages(3, 16, 10, 4)
    assert pages.desc.device == torch.cuda.current_device()
    slots, pool = torch.full((3, 1), -1, dtype=torch.int64, device="cuda"), torch.zeros((1, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8, device="cuda")
    k, q = torch.zeros((1, 3, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 3, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    work = torch.zeros(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, 1, 1), dtype=torch.uint8, device="cuda")
    calls = (lambda: cf.cf_pages_init(pages.desc), lambda: cf.cf_pages_status(pages.desc), lambda: cf.cf_pages_resize(pages.desc, pages.rows, 0, slots),
             lambda: cf.cf_kv4_write(geom, pages.desc, pool, slots, k, k), lambda: cf.cf_kv4_read(geom, pages.desc, pool, slots, k, k),
             lambda: cf.cf_kv4_attn(geom, pages.desc, pool, q, q.clone(), work))
    for call in calls:
        call()
    pages.desc.device = pages.desc.device + 1          # as if they had been made on the next one
    for call in calls:
        with pytest.raises(AssertionError, match="pages on the current device"):
            call()
