"""Calls on the 4-bit pages that a program makes and that the tests of the operators by themselves do not."""
import numpy as np
import pytest
import torch

import paper_2502_11101_b200 as cf
from oracle import paged_oracle as P
from paper_2502_11101_b200 import marshal_ctypes
from tests.test_gpu_paged import DTYPES, Pages, _attend, _check_attention, _filled

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
