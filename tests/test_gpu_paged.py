"""The paged cache held in 4 bits (cf_pages_*, cf_kv4_*) against the oracle: pages and slots exactly, codes and scales bit for bit,
attention within the bounds of its roundings."""
import numpy as np
import pytest
import torch

import oracle
import paper_2502_11101_b200 as cf
from oracle import paged_oracle as P
from paper_2502_11101_b200 import marshal_ctypes
from paper_2502_11101_b200 import workloads as W
from paper_2502_11101_b200.session import Session

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Pages:
    """Device arrays and descriptor of a pool's pages."""

    def __init__(self, n_requests, page_rows, n_pages, cols):
        def ints(*shape):
            return torch.full(shape, 12345, dtype=torch.int32, device="cuda")
        self.table, self.rows, self.free, self.count, self.status = ints(n_requests, cols), ints(n_requests), ints(n_pages), ints(1), ints(1)
        self.page_rows = page_rows
        self.desc = cf.make_pages(self.table, self.rows, self.free, self.count, self.status, page_rows)
        cf.cf_pages_init(self.desc)

    def resize(self, rows, extra=0, max_new=None):
        slots = None if max_new is None else torch.full((len(rows), max_new), 777, dtype=torch.int64, device="cuda")
        cf.cf_pages_resize(self.desc, torch.tensor(rows, dtype=torch.int32, device="cuda"), extra, slots)
        return slots


def _same_pages(got: Pages, want: P.Pool):
    table, count = got.table.cpu().numpy(), int(got.count.item())
    assert got.rows.tolist() == want.rows
    assert count == len(want.free) and got.free[:count].tolist() == want.free
    for b, pages in enumerate(want.table):
        assert table[b, :len(pages)].tolist() == pages and (table[b, len(pages):] == -1).all()


# ------------------------------------------------------------------------------------------------------------- pages

@pytest.mark.parametrize("n_requests,page_rows,n_pages,cols,max_new,steps", [
    (1, 16, 5, 4, 1, 12), (3, 48, 9, 3, 7, 12), (40, 16, 300, 16, 256, 8), (33, 32, 40, 20, 64, 10), (700, 64, 2000, 9, 3, 8),
    (1024, 16, 3000, 6, 96, 5), (1025, 16, 3000, 6, 96, 5), (2500, 32, 4000, 5, 160, 4), (5, 16, 4000, 600, 9600, 4)])
def test_pages_and_slots(n_requests, page_rows, n_pages, cols, max_new, steps):
    rng = np.random.default_rng(n_requests + page_rows)
    got, want = Pages(n_requests, page_rows, n_pages, cols), P.Pool(n_requests, page_rows, n_pages, cols)
    torch.cuda.synchronize()
    _same_pages(got, want)
    for step in range(steps):
        kind = step % 4
        most = min(cols * page_rows, 2 * n_pages * page_rows // n_requests + 1)
        if kind == 0:                                # new lengths for everyone, some of them gone
            rows, extra = rng.integers(-2, most + 1, n_requests), 0
        elif kind == 1:                              # a step each
            rows, extra = np.array(want.rows), 1
        elif kind == 2:                              # a few grow, some shrink, most stay
            rows, extra = np.array(want.rows) + rng.choice([0, 0, 0, max_new // 2, -5, max_new], n_requests), 0
        else:                                        # further than the table or the slots go
            rows, extra = np.array(want.rows) + rng.choice([0, 1, cols * page_rows, max_new + 1], n_requests), 0
        room = None if step == steps - 1 else max_new
        slots = got.resize([int(r) for r in rows], extra, room)
        expect = want.resize(rows, extra, room)
        torch.cuda.synchronize()
        _same_pages(got, want)
        if room is not None:
            assert np.array_equal(slots.cpu().numpy(), np.array(expect))
        assert cf.cf_pages_status(got.desc) in (want.status or {0})
        if want.status:
            want.status.clear()
            got.status.zero_()


def test_a_pool_that_runs_out_serves_those_before():
    got = Pages(4, 16, 3, 8)
    slots = got.resize([16, 33, 10, 0], 0, 40)
    assert cf.cf_pages_status(got.desc) == cf.CF_ERR_WORKSPACE
    assert got.rows.tolist() == [16, 0, 0, 0] and int(got.count.item()) == 2
    assert slots[0, :16].tolist() == list(range(16)) and (slots[1:] == -1).all()
    got.status.zero_()
    got.resize([20, 0, 0, 16], 0, 40)
    assert cf.cf_pages_status(got.desc) == 0 and got.rows.tolist() == [20, 0, 0, 16] and int(got.count.item()) == 0


def test_lengths_may_be_the_pages_own():
    got = Pages(3, 16, 9, 3)
    got.resize([15, 16, 0])
    slots = torch.zeros((3, 1), dtype=torch.int64, device="cuda")
    cf.cf_pages_resize(got.desc, got.rows, 1, slots)
    assert got.rows.tolist() == [16, 17, 1] and cf.cf_pages_status(got.desc) == 0
    assert slots.flatten().tolist() == [15, int(got.table[1, 1]) * 16, int(got.table[2, 0]) * 16]


# -------------------------------------------------------------------------------------------------------------- rows

def _values(shape, dtype, seed):
    """Normal numbers with groups of zeros, ties, tiny, huge and broken ones among them."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=gen)
    groups = x.view(-1, 32)
    n = len(groups)
    groups[0 % n] = 0.0
    groups[1 % n] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0] * 2)
    groups[2 % n] *= 1e-30
    groups[3 % n] *= 3e36
    groups[4 % n] *= 1e-38
    groups[5 % n] = torch.tensor([3.0e38, -1.0] * 16)
    if n > 12:
        groups[9, 3], groups[10, 31], groups[11, 0] = float("inf"), float("-inf"), float("nan")
    return x.to(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,heads,page_rows,n_rows,layers,pad", [(64, 1, 16, 1, 1, 0), (128, 2, 16, 37, 2, 8), (64, 5, 48, 50, 1, 64),
                                                                  (128, 8, 32, 6, 3, 0), (128, 1, 64, 203, 1, 16)])
def test_rows_are_kept_as_the_format_says(dtype, dim, heads, page_rows, n_rows, layers, pad):
    n_pages = (n_rows + 20) // page_rows + 2
    rng = np.random.default_rng(n_rows + dim)
    slots = rng.permutation(n_pages * page_rows)[:n_rows].astype(np.int64)
    if n_rows > 5:
        slots[rng.permutation(n_rows)[:3]] = -1
        first = int(np.argmax(slots >= 0))
        slots[first:first + 1] = slots[first]
    geom = cf.make_geom(heads, heads, dim, DTYPES[dtype], 4096, 1e4)
    pages = Pages(2, page_rows, n_pages, 4)
    layer = cf.cf_kv4_layer_bytes(geom, pages.desc)
    pool = torch.randint(0, 256, (layers, layer + 32), dtype=torch.uint8, generator=torch.Generator().manual_seed(3)).cuda()
    before = pool.cpu().numpy()
    wide = [torch.zeros((layers, n_rows, heads * dim + pad), dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    k, v = [w[..., :heads * dim].unflatten(-1, (heads, dim)) for w in wide]
    kh, vh = _values((layers, n_rows, heads, dim), DTYPES[dtype], 1), _values((layers, n_rows, heads, dim), DTYPES[dtype], 2)
    k.copy_(kh), v.copy_(vh)
    sg = torch.from_numpy(slots).cuda()
    cf.cf_kv4_write(geom, pages.desc, pool[:, :layer], sg, k, v)
    back = [torch.full((layers, n_rows, heads * dim + pad), 55.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    kb, vb = [w[..., :heads * dim].unflatten(-1, (heads, dim)) for w in back]
    cf.cf_kv4_read(geom, pages.desc, pool[:, :layer], sg, kb, vb)
    torch.cuda.synchronize()
    assert cf.cf_pages_status(pages.desc) == 0
    after = pool.cpu().numpy()
    assert np.array_equal(after[:, layer:], before[:, layer:])
    want = before[:, :layer].reshape(layers, n_pages, heads, page_rows // 16, 18 * dim).copy()
    kp, vp, ksp, vsp = P.places(dim)
    for name, (x, code_at, scale_at, got) in {"k": (kh, kp, ksp, kb), "v": (vh, vp, vsp, vb)}.items():
        codes, scales = P.quantise(x.double().numpy())
        read = got.cpu()
        for i, slot in enumerate(slots):
            if slot < 0:
                assert (read[:, i] == 55.0).all()
                continue
            page, rest = divmod(int(slot), page_rows)
            block, row = divmod(rest, 16)
            for l in range(layers):
                for h in range(heads):
                    cell = want[l, page, h, block]
                    for d in range(dim):
                        byte, half = divmod(int(code_at[row, d]), 2)
                        cell[byte] = (cell[byte] & (0xf0 >> (4 * half))) | (int(codes[l, i, h, d]) << (4 * half))
                    for j in range(dim // 32):
                        s = scales[l, i, h, j]
                        bits = 0x7fff if np.isnan(s) else int(np.float32(s).view(np.uint32)) >> 16
                        cell[scale_at[row, j]], cell[scale_at[row, j] + 1] = bits & 255, bits >> 8
            value = torch.from_numpy(P.numbers(codes[:, i], scales[:, i])).to(DTYPES[dtype])
            assert torch.equal(torch.nan_to_num(read[:, i].double(), nan=1e300), torch.nan_to_num(value.double(), nan=1e300)), name
    assert np.array_equal(after[:, :layer], want.reshape(layers, -1))
    for w in back:
        assert pad == 0 or (w[..., heads * dim:] == 55.0).all()


def test_slots_beyond_the_pool_are_skipped_and_reported():
    geom, pages = cf.make_geom(2, 2, 64, torch.bfloat16, 4096, 1e4), Pages(1, 16, 2, 2)
    pool = torch.full((1, cf.cf_kv4_layer_bytes(geom, pages.desc)), 9, dtype=torch.uint8, device="cuda")
    k = torch.ones((1, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([32, 1 << 40, 0x7fffffffffffffff], device="cuda")
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k, k)
    assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE and (pool == 9).all()
    pages.status.zero_()
    cf.cf_kv4_read(geom, pages.desc, pool, slots, k, k)
    assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE and (k == 1).all()


# --------------------------------------------------------------------------------------------------------- attention

def _filled(geom, heads, dim, lengths, page_rows, layers, seed, cols=None, stale=True):
    """Pages, a pool whose rows in use hold known numbers (the others are random bytes, NaN scales among them), and those
    numbers in 64 bits [layers][request] -> (k, v)."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page_rows) for n in lengths]
    n_pages = max(1, sum(need)) + 2
    pages = Pages(len(lengths), page_rows, n_pages, cols or max(need + [1]) + 1)
    # pages handed out in a random order
    pages.free.copy_(torch.from_numpy(rng.permutation(n_pages).astype(np.int32)))
    longest = max(list(lengths) + [1])
    slots = pages.resize([int(n) for n in lengths], 0, longest)
    pool = torch.randint(0, 256, (layers, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8,
                         generator=torch.Generator().manual_seed(seed)).cuda()
    if not stale:
        pool.zero_()
    gen = torch.Generator().manual_seed(seed + 1)
    k = torch.randn((layers, len(lengths), longest, heads, dim), generator=gen) * torch.where(torch.rand((heads, dim), generator=gen) < 0.05, 3.0, 1.0)
    v = torch.randn((layers, len(lengths), longest, heads, dim), generator=gen)
    dt = torch.bfloat16 if geom.dtype == cf.CF_BF16 else torch.float32
    k, v = k.to(dt), v.to(dt)
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k.cuda(), v.cuda())
    kept = [[[P.numbers(*P.quantise(x[l, b, :n].double().numpy())) for x in (k, v)] for b, n in enumerate(lengths)] for l in range(layers)]
    return pages, pool, kept


def _attend(geom, pages, pool, q, softmax_scale=0.0, stream=None):
    layers, b, n, hq, d = q.shape
    out, lse = torch.full_like(q, 99.0), torch.full((layers, b, hq, n), 99.0, device="cuda")
    work = torch.full((cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, n, layers),), 255, dtype=torch.uint8, device="cuda")
    cf.cf_kv4_attn(geom, pages.desc, pool, q, out, work, lse=lse, softmax_scale=softmax_scale, stream=stream)
    return out, lse


def _check_attention(geom, out, lse, q, kept, scale):
    """Roundings that are counted: the result to its type; a probability to 11 bits (fp32 storage: 22) twice, as product with a
    scale and in the running sum's units; a logit, fp32 sums of D exact products of which each is at most `reach` off by a rounding of the
    sum (fp32 storage: the queries' 22 bits too); exp2 by 2^-21; the sums over the keys, fp32.
    And where probabilities vanish: the product of a probability and a value's scale is held as fp16 in units of 2^(c - 7), 2^c at most
    twice the largest scale of the request, so below fp16's normal numbers it is off by up to 2^-25 such units, half the last
    place.  A code is at most 6, six scales are the largest value, and the sum of the probabilities is at least 1 in these
    units (the key that set the maximum): each key adds at most 2^-25 * 2^-7 * 2 = 2^-31 of the request's largest value, and
    2^-8 of that for the scale's own rounding."""
    f32 = geom.dtype == cf.CF_F32
    out, lse, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    for l in range(len(kept)):
        for b in range(len(kept[l])):
            k, v = kept[l][b]
            o, e, spread, reach = P.attention(q[l, b], k, v, scale)
            keys = k.shape[0]
            logit = reach * (q.shape[-1] * 2.0 ** -24 + (2.0 ** -21 if f32 else 0.0)) + 2.0 ** -21
            total = logit + (keys + 32) * 2.0 ** -24
            tol = np.abs(o) * (2.0 ** -24 if f32 else 2.0 ** -8) + spread * ((2.0 ** -21 if f32 else 2.0 ** -11) + 2 * total)[..., None]
            tol = tol + keys * 2.0 ** -31 * (1 + 2.0 ** -8) * (np.abs(v).max() if keys else 0.0)
            off = np.abs(out[l, b] - o)
            assert (off <= tol).all(), (l, b, float((off / tol).max()))
            hidden = np.isinf(e)
            assert np.array_equal(np.isneginf(lse[l, b]), hidden)
            bound = total.T + 2.0 ** -23 * np.abs(np.where(hidden, 0.0, e)) + 2.0 ** -22
            assert (np.abs(np.where(hidden, 0.0, lse[l, b]) - np.where(hidden, 0.0, e)) <= bound).all(), (l, b)


CASES = [
    # dtype, q heads, kv heads, head_dim, lengths, page_rows, q_len, layers
    ("bf16", 1, 1, 128, [1], 16, 1, 1),
    ("bf16", 4, 4, 64, [0, 1, 15, 16, 17, 33, 0], 16, 1, 1),
    ("bf16", 12, 2, 128, [1011], 64, 1, 1),
    ("bf16", 28, 4, 128, [5, 700, 64, 65, 0, 129], 32, 1, 2),
    ("bf16", 32, 32, 128, [300, 17], 48, 1, 1),
    ("bf16", 64, 4, 128, [77, 400], 64, 1, 1),
    ("bf16", 9, 1, 64, [250, 3], 16, 1, 3),
    ("bf16", 12, 2, 128, [40, 3, 0, 200], 16, 5, 1),
    ("bf16", 28, 4, 128, [130, 24, 10], 32, 24, 1),
    ("bf16", 8, 2, 64, [33, 7, 64], 16, 3, 2),
    ("f32", 4, 4, 64, [0, 83, 16, 1], 16, 1, 1),
    ("f32", 8, 2, 128, [500, 31], 80, 1, 1),
    ("f32", 16, 1, 128, [90, 5], 16, 4, 2),
    ("f32", 8, 2, 64, [70, 2, 0], 32, 7, 1),
    ("bf16", 2, 1, 128, [17000], 256, 1, 1),
    ("bf16", 4, 2, 64, [40 + i % 90 for i in range(300)], 16, 1, 2),
    ("bf16", 4, 4, 128, [1 + 7 * i % 50 for i in range(700)], 16, 1, 1),
    ("f32", 2, 2, 64, [i % 40 for i in range(1500)], 16, 1, 1),
]


@pytest.mark.parametrize("dtype,hq,hkv,dim,lengths,page_rows,q_len,layers", CASES, ids=["%s-%d/%d-%d-%dx%d-q%d-l%d" % (c[0], c[1], c[2], c[3], len(c[4]), max(c[4]), c[6], c[7]) for c in CASES])
def test_attention_over_pages(dtype, hq, hkv, dim, lengths, page_rows, q_len, layers):
    geom = cf.make_geom(hq, hkv, dim, DTYPES[dtype], 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, dim, lengths, page_rows, layers, seed=len(lengths) + dim)
    q = torch.randn((layers, len(lengths), q_len, hq, dim), generator=torch.Generator().manual_seed(4)).to(DTYPES[dtype]).cuda()
    out, lse = _attend(geom, pages, pool, q)
    torch.cuda.synchronize()
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, kept, dim ** -0.5)
    again, lse2 = _attend(geom, pages, pool, q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_scale,softmax_scale", [(1e-20, 1e19), (3e4, 3e-5), (60.0, 0.0), (1e30, 1e-31), (0.0, 0.0), (5.0, -0.2)])
def test_queries_of_any_size(dtype, q_scale, softmax_scale):
    """Logits that climb far above the first keys', that are all alike, and queries outside fp16's range."""
    geom = cf.make_geom(6, 2, 128, DTYPES[dtype], 32768, 1e6)
    pages, pool, kept = _filled(geom, 2, 128, [333, 50], 32, 1, seed=9)
    q = (torch.randn((1, 2, 2, 6, 128), generator=torch.Generator().manual_seed(4)) * q_scale).to(DTYPES[dtype]).cuda()
    out, lse = _attend(geom, pages, pool, q, softmax_scale)
    _check_attention(geom, out, lse, q, kept, softmax_scale or 128 ** -0.5)


def test_values_of_any_size():
    """Scales of the values that grow by 2^40 along a request, and shrink along another."""
    geom = cf.make_geom(4, 2, 64, torch.float32, 32768, 1e6)
    lengths = [160, 160, 40]
    pages, pool, _ = _filled(geom, 2, 64, lengths, 16, 1, seed=2)
    slots = torch.zeros((3, 160), dtype=torch.int64, device="cuda")
    for b, n in enumerate(lengths):
        rows = torch.arange(160, device="cuda")
        slots[b] = torch.where(rows < n, pages.table[b, torch.clamp(rows // 16, max=pages.table.shape[1] - 1)].long() * 16 + rows % 16, -1)
    gen = torch.Generator().manual_seed(1)
    k, v = torch.randn((1, 3, 160, 2, 64), generator=gen), torch.randn((1, 3, 160, 2, 64), generator=gen)
    v[0, 0] *= 2.0 ** torch.linspace(-30, 10, 160)[:, None, None]
    v[0, 1] *= 2.0 ** torch.linspace(10, -30, 160)[:, None, None]
    v[0, 2] *= 1e-33
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k.cuda(), v.cuda())
    kept = [[[P.numbers(*P.quantise(x[0, b, :n].double().numpy())) for x in (k, v)] for b, n in enumerate(lengths)]]
    q = torch.randn((1, 3, 1, 4, 64), generator=gen).cuda()
    out, lse = _attend(geom, pages, pool, q)
    # what lies 2^-29 below the largest scale of its request loses bits of its probability: that much of the largest is allowed
    o, want = out.double().cpu().numpy(), [P.attention(q[0, b].double().cpu().numpy(), *kept[0][b], 64 ** -0.5) for b in range(3)]
    for b in range(3):
        top = np.abs(kept[0][b][1]).max()
        assert (np.abs(o[0, b] - want[b][0]) <= want[b][2] * 2.0 ** -17 + top * 2.0 ** -28).all()


def test_numbers_that_are_not_finite_stay_with_the_queries_that_see_them():
    geom = cf.make_geom(2, 1, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 1, 128, [40, 40], 16, 1, seed=5)
    k, v = torch.randn((1, 1, 1, 128)).bfloat16(), torch.randn((1, 1, 1, 128)).bfloat16()
    v[..., 70] = float("inf")
    slot = int(pages.table[0, 38 // 16]) * 16 + 38 % 16
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), v.cuda())
    q = torch.randn((1, 2, 4, 2, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    nan = torch.isnan(out[0]).cpu()
    want = torch.zeros_like(nan)
    want[0, 2:, :, 64:96] = True                    # row 38 is seen by the last two of four queries; a group of 32 dims
    assert torch.equal(nan, want) and torch.isfinite(lse).all()
    k[..., 3] = float("nan")
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), torch.zeros_like(v).cuda())
    out, lse = _attend(geom, pages, pool, q)
    want[0, 2:] = True
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.equal(torch.isnan(lse[0, 0]).cpu(), want[0, :, :, 0].T)


def test_strided_layers_and_a_stream_of_its_own():
    geom = cf.make_geom(4, 2, 64, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 2, 64, [100, 30], 16, 3, seed=6)
    q = torch.randn((6, 2, 1, 4, 64), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    wide = torch.full((6, 2, 1, 4, 64), 99.0, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, 1, 3), dtype=torch.uint8, device="cuda")
    lse = torch.zeros((3, 2, 4, 1), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    cf.cf_kv4_attn(geom, pages.desc, pool, q[::2], wide[::2], work, lse=lse, stream=stream)
    stream.synchronize()
    assert (wide[1::2] == 99.0).all()
    _check_attention(geom, wide[::2], lse, q[::2], kept, 0.125)


def test_a_table_that_points_outside_is_reported():
    """Reads stay inside the pool; the status says that the results mean nothing."""
    geom = cf.make_geom(4, 2, 64, torch.bfloat16, 32768, 1e6)
    pages, pool, _ = _filled(geom, 2, 64, [100, 30], 16, 1, seed=6)
    pages.table[0, 2] = 1 << 30
    q = torch.zeros((1, 2, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE
    pages.status.zero_()
    pages.table[0, 2] = 0
    pages.rows[1] = 1 << 30
    _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE


@pytest.mark.parametrize("marshal", ["native", "ctypes"])
def test_a_decoding_loop_over_the_caches_that_pruning_left(marshal, monkeypatch):
    """Stack, final caches, pages, rows in 4 bits and four steps, captured as one graph and replayed; against the oracle's attention
    over what the format keeps."""
    if marshal == "ctypes":
        monkeypatch.setattr(cf.binding, "_NATIVE", marshal_ctypes)
    cfg = W.WorkloadConfig("decode", 2, 8, 2, 128, "bf16", 1e4, 4096, 7, 20, 150, 5, 2, 2, ((1, 3),))
    meta = W.make_meta(cfg, 0)
    q, (k, v), (k_self, v_self) = W.make_q(meta), W.make_kv(meta), W.make_kv_self(meta)
    sess = Session(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.torch_dtype, cfg.pos_range, cfg.rope_theta, cfg.q_len,
                   meta.doc_len, meta.req_doc_begin, meta.doc_src_start, tail_reserve=cfg.q_len)
    qg, kg, vg, ksg, vsg = [t.cuda() for t in (q, k, v, k_self, v_self)]
    sess.run_stack(qg, kg, vg, cfg.schedule, oracle.ALLOC_ALIGN, torch.empty_like(qg))
    L, B, hq, hkv, d, room, steps = cfg.n_layers, cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, 3 * 150 + cfg.q_len, 4
    k_fin = torch.zeros((L, B, room, hkv, d), dtype=torch.bfloat16, device="cuda")
    v_fin = torch.zeros_like(k_fin)
    final_rows = torch.zeros(B, dtype=torch.int32, device="cuda")
    sess.assemble(kg, vg, ksg, vsg, k_fin, v_fin, final_rows)
    pages = Pages(B, 32, 2 * B * (room // 32 + 2), room // 32 + 2)
    pool = torch.zeros((L, cf.cf_kv4_layer_bytes(sess.geom, pages.desc)), dtype=torch.uint8, device="cuda")
    slots = torch.zeros((B, room), dtype=torch.int64, device="cuda")
    one = torch.zeros((B, 1), dtype=torch.int64, device="cuda")
    gen = torch.Generator().manual_seed(7)
    q_new, k_new, v_new = [torch.randn((steps, L, B, 1, h, d), generator=gen).bfloat16().cuda() for h in (hq, hkv, hkv)]
    out, lse = torch.zeros_like(q_new), torch.zeros((steps, L, B, hq, 1), device="cuda")
    work = torch.empty(cf.cf_kv4_attn_workspace_bytes(sess.geom, pages.desc, 1, L), dtype=torch.uint8, device="cuda")

    def loop():
        cf.cf_pages_init(pages.desc)
        cf.cf_pages_resize(pages.desc, final_rows, 0, slots)
        cf.cf_kv4_write(sess.geom, pages.desc, pool, slots, k_fin, v_fin)
        for t in range(steps):
            cf.cf_pages_resize(pages.desc, final_rows, t + 1, one)
            for l in range(L):
                cf.cf_kv4_write(sess.geom, pages.desc, pool[l:l + 1], one, k_new[t, l:l + 1], v_new[t, l:l + 1])
                cf.cf_kv4_attn(sess.geom, pages.desc, pool[l:l + 1], q_new[t, l:l + 1], out[t, l:l + 1], work, lse=lse[t, l:l + 1])

    loop()
    torch.cuda.synchronize()
    first = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop()
    out.zero_(), lse.zero_(), pool.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert cf.cf_pages_status(pages.desc) == 0 and torch.equal(out, first[0]) and torch.equal(lse, first[1])
    for t in range(steps):
        kept = []
        for l in range(L):
            kept.append([])
            for b in range(B):
                n = int(final_rows[b])
                whole = [torch.cat([c[l, b, :n], x[:t + 1, l, b, 0]]).double().cpu().numpy() for c, x in ((k_fin, k_new), (v_fin, v_new))]
                kept[-1].append([P.numbers(*P.quantise(x)) for x in whole])
        _check_attention(sess.geom, out[t], lse[t], q_new[t], kept, d ** -0.5)


@pytest.mark.parametrize("hq,hkv,lengths,page_rows,q_len,layers", [
    (12, 2, [64], 64, 16, 1), (28, 4, [130, 24, 10, 0], 32, 24, 1), (4, 4, [500, 33], 48, 40, 2), (64, 4, [300, 5], 16, 9, 1),
    (8, 1, [1500], 80, 33, 1), (7, 1, [63, 64, 65, 127, 128, 129], 16, 19, 1), (28, 4, [40 * i % 333 for i in range(40)], 16, 5, 1),
    (16, 2, [9000, 3], 64, 100, 1)],
    ids=lambda x: str(x) if isinstance(x, int) else "%dx%d" % (len(x), max(x)))
def test_attention_of_many_query_columns(hq, hkv, lengths, page_rows, q_len, layers):
    """The tensor-core kernel: one and several tiles of columns, the last one with columns that are none, ends of requests inside and
    between tiles and pages, queries that see nothing."""
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, hkv, 128, lengths, page_rows, layers, seed=q_len)
    q = torch.randn((layers, len(lengths), q_len, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    torch.cuda.synchronize()
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)
    again, lse2 = _attend(geom, pages, pool, q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("q_scale,softmax_scale", [(1e-20, 1e19), (3e4, 3e-5), (60.0, 0.0), (1e30, 1e-31), (0.0, 0.0), (5.0, -0.2)])
def test_many_queries_of_any_size(q_scale, softmax_scale):
    geom = cf.make_geom(6, 2, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 2, 128, [333, 50], 32, 1, seed=9)
    q = (torch.randn((1, 2, 20, 6, 128), generator=torch.Generator().manual_seed(4)) * q_scale).to(torch.bfloat16).cuda()
    out, lse = _attend(geom, pages, pool, q, softmax_scale)
    _check_attention(geom, out, lse, q, kept, softmax_scale or 128 ** -0.5)


def test_many_queries_over_keys_and_values_of_any_size():
    """Scales that grow and shrink along a request, tile by tile and inside tiles."""
    geom = cf.make_geom(4, 1, 128, torch.bfloat16, 32768, 1e6)
    lengths = [300, 300, 300]
    pages, pool, _ = _filled(geom, 1, 128, lengths, 16, 1, seed=2)
    rows = torch.arange(300, device="cuda")
    slots = torch.stack([pages.table[b, rows // 16].long() * 16 + rows % 16 for b in range(3)])
    gen = torch.Generator().manual_seed(1)
    k, v = torch.randn((1, 3, 300, 1, 128), generator=gen), torch.randn((1, 3, 300, 1, 128), generator=gen)
    v[0, 0] *= 2.0 ** torch.linspace(-30, 10, 300)[:, None, None]
    v[0, 1] *= 2.0 ** torch.linspace(10, -30, 300)[:, None, None]
    v[0, 2] *= 1e-30
    k[0, 1] *= 2.0 ** torch.linspace(-12, 2, 300)[:, None, None]
    k[0, 2, 100:116] *= 2.0 ** torch.linspace(-10, 3, 16)[:, None, None]
    k, v = k.bfloat16(), v.bfloat16()
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k.cuda(), v.cuda())
    kept = [[[P.numbers(*P.quantise(x[0, b].double().numpy())) for x in (k, v)] for b in range(3)]]
    q = torch.randn((1, 3, 12, 4, 128), generator=gen).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)


def test_many_queries_and_numbers_that_are_not_finite():
    geom = cf.make_geom(2, 1, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 1, 128, [140, 40], 16, 1, seed=5)
    k, v = torch.randn((1, 1, 1, 128)).bfloat16(), torch.randn((1, 1, 1, 128)).bfloat16()
    v[..., 70] = float("inf")
    slot = int(pages.table[0, 130 // 16]) * 16 + 130 % 16
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), v.cuda())
    q = torch.randn((1, 2, 20, 2, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    want = torch.zeros((2, 20, 2, 128), dtype=torch.bool)
    want[0, 10:, :, 64:96] = True                   # row 130 of 140 is seen by the last ten of twenty queries
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.isfinite(lse).all()
    k[..., 3] = float("nan")
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), torch.zeros_like(v).cuda())
    out, lse = _attend(geom, pages, pool, q)
    want[0, 10:] = True
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.equal(torch.isnan(lse[0, 0]).cpu(), want[0, :, :, 0].T)


@pytest.mark.parametrize("hq,hkv,lengths,page_rows,q_len,layers", [
    (12, 2, [64, 1, 200, 63], 64, 16, 1), (4, 4, [500, 33], 48, 57, 2), (8, 1, [1500, 0, 17], 80, 47, 1), (28, 4, [40 * i % 333 for i in range(40)], 16, 9, 1)],
    ids=lambda x: str(x) if isinstance(x, int) else "%dx%d" % (len(x), max(x)))
def test_attention_of_many_query_columns_in_eight_units(hq, hkv, lengths, page_rows, q_len, layers):
    """Enough columns and units for the tensor-core kernel."""
    test_attention_of_many_query_columns(hq, hkv, lengths, page_rows, q_len, layers)


@pytest.mark.parametrize("q_scale,softmax_scale", [(1e-20, 1e19), (3e4, 3e-5), (60.0, 0.0), (1e30, 1e-31), (0.0, 0.0), (5.0, -0.2)])
def test_many_columns_of_any_size(q_scale, softmax_scale):
    geom = cf.make_geom(12, 2, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 2, 128, [333, 50, 128, 7], 32, 1, seed=9)
    q = (torch.randn((1, 4, 20, 12, 128), generator=torch.Generator().manual_seed(4)) * q_scale).to(torch.bfloat16).cuda()
    out, lse = _attend(geom, pages, pool, q, softmax_scale)
    _check_attention(geom, out, lse, q, kept, softmax_scale or 128 ** -0.5)


def test_many_columns_over_keys_and_values_of_any_size():
    """Scales that grow and shrink along a request, tile by tile and inside tiles: the units of blocks and of O, and their limits."""
    geom = cf.make_geom(16, 4, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, _ = _filled(geom, 4, 128, [300, 300, 300], 16, 1, seed=2)
    rows = torch.arange(300, device="cuda")
    slots = torch.stack([pages.table[b, rows // 16].long() * 16 + rows % 16 for b in range(3)])
    gen = torch.Generator().manual_seed(1)
    k, v = torch.randn((1, 3, 300, 4, 128), generator=gen), torch.randn((1, 3, 300, 4, 128), generator=gen)
    v[0, 0] *= 2.0 ** torch.linspace(-30, 10, 300)[:, None, None]
    v[0, 1] *= 2.0 ** torch.linspace(10, -30, 300)[:, None, None]
    v[0, 1, 150:] *= 2.0 ** -60
    v[0, 2] *= 1e-30
    k[0, 1] *= 2.0 ** torch.linspace(-12, 2, 300)[:, None, None]
    k[0, 2, 100:116] *= 2.0 ** torch.linspace(-10, 3, 16)[:, None, None]
    k, v = k.bfloat16(), v.bfloat16()
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k.cuda(), v.cuda())
    kept = [[[P.numbers(*P.quantise(x[0, b].double().numpy())) for x in (k, v)] for b in range(3)]]
    q = torch.randn((1, 3, 20, 16, 128), generator=gen).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)


def test_many_columns_and_numbers_that_are_not_finite():
    geom = cf.make_geom(8, 4, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 4, 128, [140, 40], 16, 1, seed=5)
    k, v = torch.randn((1, 1, 4, 128)).bfloat16(), torch.randn((1, 1, 4, 128)).bfloat16()
    v[..., 2, 70] = float("inf")
    slot = int(pages.table[0, 130 // 16]) * 16 + 130 % 16
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), v.cuda())
    q = torch.randn((1, 2, 30, 8, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    want = torch.zeros((2, 30, 8, 128), dtype=torch.bool)
    want[0, 20:, 4:6, 64:96] = True                 # row 130 of 140 is seen by the last ten of thirty queries; kv head 2, a group of dims
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.isfinite(lse).all()
    k[..., 2, 3] = float("nan")
    cf.cf_kv4_write(geom, pages.desc, pool, torch.tensor([slot], device="cuda"), k.cuda(), torch.zeros_like(v).cuda())
    out, lse = _attend(geom, pages, pool, q)
    want[0, 20:, 4:6] = True
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.equal(torch.isnan(lse[0, 0]).cpu(), want[0, :, :, 0].T)


def test_many_columns_captured_and_on_a_stream_of_its_own():
    geom = cf.make_geom(32, 8, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 8, 128, [700, 90], 16, 3, seed=6)
    q = torch.randn((6, 2, 20, 32, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    wide = torch.full_like(q, 99.0)
    work = torch.empty(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, 20, 3), dtype=torch.uint8, device="cuda")
    lse = torch.zeros((3, 2, 32, 20), device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cf.cf_kv4_attn(geom, pages.desc, pool, q[::2], wide[::2], work, lse=lse)
        cf.cf_kv4_attn(geom, pages.desc, pool, q[::2], wide[::2], work, lse=lse)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert (wide[1::2] == 99.0).all()
    _check_attention(geom, wide[::2], lse, q[::2], kept, 128 ** -0.5)


def test_tensors_of_the_host_are_refused():
    geom = cf.make_geom(2, 1, 64, torch.bfloat16, 4096, 1e4)
    pages = Pages(1, 16, 2, 2)
    rows, slots = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int64)
    pool = torch.zeros((1, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8, device="cuda")
    k = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, 1, 1, 2, 64), dtype=torch.bfloat16)
    work = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    for call in (lambda: cf.cf_pages_resize(pages.desc, rows, 0, slots.cuda()), lambda: cf.cf_pages_resize(pages.desc, rows.cuda(), 0, slots),
                 lambda: cf.cf_kv4_write(geom, pages.desc, pool, slots.cuda(), k, k), lambda: cf.cf_kv4_read(geom, pages.desc, pool, slots, k.cuda(), k.cuda()),
                 lambda: cf.cf_kv4_write(geom, pages.desc, pool.cpu(), slots.cuda(), k.cuda(), k.cuda()),
                 lambda: cf.cf_kv4_attn(geom, pages.desc, pool, q, q.cuda(), work), lambda: cf.cf_kv4_attn(geom, pages.desc, pool, q.cuda(), q.cuda(), work.cpu())):
        with pytest.raises(AssertionError):
            call()


@pytest.mark.parametrize("dtype,hq,hkv,dim,lengths,page_rows,q_len,layers", [CASES[i] for i in (0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11, 12, 13)],
                         ids=lambda x: str(x) if not isinstance(x, list) else "%dx%d" % (len(x), max(x)))
@pytest.mark.parametrize("cols", [3000, 0])
def test_attention_with_room_for_long_requests(dtype, hq, hkv, dim, lengths, page_rows, q_len, layers, cols):
    """A table with room for long requests has shares of the line where its columns only hold the rows there are has clusters."""
    geom = cf.make_geom(hq, hkv, dim, DTYPES[dtype], 32768, 1e6)
    need = max(1, -(-max(lengths) // page_rows))
    pages, pool, kept = _filled(geom, hkv, dim, lengths, page_rows, layers, seed=len(lengths) + dim, cols=cols or need)
    q = torch.randn((layers, len(lengths), q_len, hq, dim), generator=torch.Generator().manual_seed(4)).to(DTYPES[dtype]).cuda()
    out, lse = _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0
    _check_attention(geom, out, lse, q, kept, dim ** -0.5)


@pytest.mark.parametrize("hq,hkv,rows,requests", [(4, 4, 60, 3), (4, 4, 500, 2), (12, 2, 250, 1), (12, 2, 5000, 1), (28, 4, 1000, 8), (28, 4, 90, 30)])
def test_attention_by_clusters_of_every_size(hq, hkv, rows, requests):
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    lengths = [rows - i * rows // requests for i in range(requests)]
    pages, pool, kept = _filled(geom, hkv, 128, lengths, 16, 1, seed=rows, cols=-(-rows // 16))
    q = torch.randn((1, requests, 1, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    _check_attention(geom, out, lse, q, kept, 128 ** -0.5)
    graph = torch.cuda.CUDAGraph()
    work = torch.empty(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, 1, 1), dtype=torch.uint8, device="cuda")
    again = torch.zeros_like(out)
    with torch.cuda.graph(graph):
        for _ in range(3):
            cf.cf_kv4_attn(geom, pages.desc, pool, q, again, work)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_scale,softmax_scale", [(3e4, 3e-5), (60.0, 0.0), (5.0, -0.2)])
def test_queries_of_any_size_with_room_for_long_requests(dtype, q_scale, softmax_scale):
    geom = cf.make_geom(6, 2, 128, DTYPES[dtype], 32768, 1e6)
    pages, pool, kept = _filled(geom, 2, 128, [333, 50, 1900], 32, 1, seed=9, cols=3000)
    q = (torch.randn((1, 3, 2, 6, 128), generator=torch.Generator().manual_seed(4)) * q_scale).to(DTYPES[dtype]).cuda()
    out, lse = _attend(geom, pages, pool, q, softmax_scale)
    _check_attention(geom, out, lse, q, kept, softmax_scale or 128 ** -0.5)


@pytest.mark.parametrize("hq,cols", [(1, 3000), (1, 40), (12, 3000), (12, 40)])
def test_numbers_that_are_not_finite_over_several_parts(hq, cols):
    """A request that several warps, shares or CTAs have: a NaN goes through the joins."""
    geom = cf.make_geom(hq, 1, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, kept = _filled(geom, 1, 128, [640, 500], 16, 1, seed=5, cols=cols)
    k, v = torch.randn((1, 1, 1, 128)).bfloat16(), torch.randn((1, 1, 1, 128)).bfloat16()
    v[..., 70] = float("inf")
    row = 638
    slot = torch.tensor([int(pages.table[0, row // 16]) * 16 + row % 16], device="cuda")
    cf.cf_kv4_write(geom, pages.desc, pool, slot, k.cuda(), v.cuda())
    q = torch.randn((1, 2, 3, hq, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, lse = _attend(geom, pages, pool, q)
    want = torch.zeros(out[0].shape, dtype=torch.bool)
    want[0, 1:, :, 64:96] = True                    # row 638 of 640 is seen by the last two of three queries
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.isfinite(lse).all()
    k[..., 3] = float("nan")
    cf.cf_kv4_write(geom, pages.desc, pool, slot, k.cuda(), torch.zeros_like(v).cuda())
    out, lse = _attend(geom, pages, pool, q)
    want[0, 1:] = True
    assert torch.equal(torch.isnan(out[0]).cpu(), want) and torch.equal(torch.isnan(lse[0, 0]).cpu(), want[0, :, :, 0].T)


@pytest.mark.parametrize("hq,hkv,q_len,cols", [(4, 2, 1, 0), (4, 2, 1, 3000), (32, 4, 9, 0)])
def test_a_table_that_points_outside_is_reported_by_every_kernel(hq, hkv, q_len, cols):
    geom = cf.make_geom(hq, hkv, 128, torch.bfloat16, 32768, 1e6)
    pages, pool, _ = _filled(geom, hkv, 128, [100, 30, 80], 16, 1, seed=6, cols=cols or None)
    q = torch.zeros((1, 3, q_len, hq, 128), dtype=torch.bfloat16, device="cuda")
    for bad in (1 << 30, -1, pages.free.shape[0]):
        right, pages.table[0, 2] = int(pages.table[0, 2]), bad
        _attend(geom, pages, pool, q)
        assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE
        pages.status.zero_()
        pages.table[0, 2] = right
    for bad in (1 << 30, -5):
        right, pages.rows[1] = int(pages.rows[1]), bad
        _attend(geom, pages, pool, q)
        assert cf.cf_pages_status(pages.desc) == cf.CF_ERR_RANGE
        pages.status.zero_()
        pages.rows[1] = right
    _attend(geom, pages, pool, q)
    assert cf.cf_pages_status(pages.desc) == 0


def test_calls_on_two_streams_at_once():
    """Over one pool, each with its own queries, results and workspace: as by themselves."""
    cases = []
    for hq, q_len, cols in ((28, 1, 3000), (28, 1, None), (28, 24, 3000), (28, 3, 3000)):
        geom = cf.make_geom(hq, 4, 128, torch.bfloat16, 32768, 1e6)
        pages, pool, _ = _filled(geom, 4, 128, [900, 40, 333, 0], 32, 1, seed=8, cols=cols)
        q = torch.randn((1, 4, q_len, hq, 128), generator=torch.Generator().manual_seed(q_len)).bfloat16().cuda()
        cases.append((geom, pages, pool, q, _attend(geom, pages, pool, q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    work = [torch.empty(cf.cf_kv4_attn_workspace_bytes(c[0], c[1].desc, c[3].shape[2], 1), dtype=torch.uint8, device="cuda") for c in cases]
    outs, lses = [torch.full_like(c[3], 99.0) for c in cases], [torch.full_like(c[4][1], 99.0) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (geom, pages, pool, q, _) in enumerate(cases):
            cf.cf_kv4_attn(geom, pages.desc, pool, q, outs[i], work[i], lse=lses[i], stream=streams[i])
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert torch.equal(outs[i], c[4][0]) and torch.equal(lses[i], c[4][1])


def test_pages_beyond_four_gigabytes():
    """The last pages of a pool of 4.7 GB against the same rows in a small pool."""
    heads, dim, page_rows, lengths = 32, 128, 64, [150, 64, 1]
    geom = cf.make_geom(heads, heads, dim, torch.bfloat16, 32768, 1e6)
    gen = torch.Generator().manual_seed(1)
    k, v = [torch.randn((1, 3, 150, heads, dim), generator=gen).bfloat16().cuda() for _ in range(2)]
    q = torch.randn((1, 3, 1, heads, dim), generator=gen).bfloat16().cuda()
    many = torch.randn((1, 3, 72, heads, dim), generator=gen).bfloat16().cuda()
    results = []
    for n_pages in (8, 16000):
        pages = Pages(3, page_rows, n_pages, 3)
        pages.free.copy_(torch.arange(n_pages, dtype=torch.int32))
        slots = pages.resize(lengths, 0, 150)
        assert int(pages.table.max()) == n_pages - 1
        pool = torch.zeros((1, cf.cf_kv4_layer_bytes(geom, pages.desc)), dtype=torch.uint8, device="cuda")
        assert n_pages == 8 or pool.numel() > 1 << 32
        cf.cf_kv4_write(geom, pages.desc, pool, slots, k, v)
        back = [torch.zeros_like(k) for _ in range(2)]
        cf.cf_kv4_read(geom, pages.desc, pool, slots, back[0], back[1])
        results.append(back + list(_attend(geom, pages, pool, q)) + list(_attend(geom, pages, pool, many)))
        assert cf.cf_pages_status(pages.desc) == 0
        del pool
    assert results[0][0].abs().max() > 0
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("marshal", ["native", "ctypes"])
def test_small_pools_other_types_and_no_requests_are_refused(marshal, monkeypatch):
    if marshal == "ctypes":
        monkeypatch.setattr(cf.binding, "_NATIVE", marshal_ctypes)
    geom, pages = cf.make_geom(4, 2, 64, torch.bfloat16, 4096, 1e4), Pages(3, 16, 10, 4)
    slots = torch.full((3, 5), -1, dtype=torch.int64, device="cuda")
    layer = cf.cf_kv4_layer_bytes(geom, pages.desc)
    pool, small = torch.zeros((2, layer), dtype=torch.uint8, device="cuda"), torch.zeros((2, layer - 16), dtype=torch.uint8, device="cuda")
    k = torch.zeros((2, 3, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 3, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    work = torch.zeros(cf.cf_kv4_attn_workspace_bytes(geom, pages.desc, 1, 2), dtype=torch.uint8, device="cuda")
    none = cf.make_pages(torch.zeros((0, 4), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), pages.free, pages.count,
                         pages.status, 16)
    for call in (lambda: cf.cf_kv4_write(geom, pages.desc, small, slots, k, k), lambda: cf.cf_kv4_read(geom, pages.desc, small, slots, k, k),
                 lambda: cf.cf_kv4_write(geom, pages.desc, pool, slots, k.half(), k.half()), lambda: cf.cf_kv4_read(geom, pages.desc, pool, slots, k.half(), k.half()),
                 lambda: cf.cf_kv4_attn(geom, pages.desc, small, q, q.clone(), work), lambda: cf.cf_kv4_attn(geom, pages.desc, pool, q.half(), q.half(), work),
                 lambda: cf.cf_pages_resize(none, torch.zeros(0, dtype=torch.int32, device="cuda"), 0, torch.zeros((0, 1), dtype=torch.int64, device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    cf.cf_kv4_write(geom, pages.desc, pool, slots, k, k)
    cf.cf_kv4_attn(geom, pages.desc, pool, q, q.clone(), work)
    assert cf.cf_pages_status(pages.desc) == 0
