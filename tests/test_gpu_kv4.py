"""The 4-bit key/value cache on the GPU against its definition in 64 bits (kv4_util): bytes
written and values read exactly, pages chosen exactly, attention within bounds that the
types and the float32 sums give."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests import kv4_util as ref
from tests.kv4_util import DTYPES, PAGE, Batch

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


# ---- writing and reading

def special(rng, shape, dtype):
    """Values that quantise in every way: ties, zeros of both signs, subnormals, huge ones."""
    x = rng.standard_normal(shape)
    x = x * np.exp2(rng.integers(-20, 12, shape[:-1] + (1,)))
    kind = rng.integers(0, 12, shape)
    grid = rng.integers(-28, 29, shape) / 4.0           # every tie and every code
    x = np.where(kind < 4, grid, x)
    x = np.where(kind == 4, 0.0, x)
    x = np.where(kind == 5, -0.0, x)
    rows = rng.integers(0, 8, shape[:-1] + (1,))
    x = np.where(rows == 0, 0.0 * x, x)                 # whole rows of signed zeros
    small = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    large = {"f16": 2.0 ** 15, "bf16": 2.0 ** 127, "f32": 2.0 ** 127}[dtype]
    x = np.where(rows == 1, grid * 4 * small, x)        # subnormal
    x = np.where(rows == 2, rng.uniform(-1.99, 1.99, shape) * large, x)
    x = np.where(rows == 3, rng.uniform(-1, 1, shape) * small * 2.0 ** 11, x)
    return torch.from_numpy(x).to(DTYPES[dtype])


def expected_bytes(pages, heads, dim, slots, k, v):
    c = ref.Cache(pages, heads, dim, fill=0xA5)
    for s, a, b in zip(slots, k.double().numpy(), v.double().numpy()):
        if 0 <= s < pages * PAGE:
            c.write(s, a, b)
    return c


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (7, 3), (150, 2)])
def test_append_writes_the_layout_and_read_returns_it(dim, dtype, tokens, heads):
    rng = np.random.default_rng(tokens * dim)
    pages = tokens // PAGE + 3
    k, v = special(rng, (tokens, heads, dim), dtype), special(rng, (tokens, heads, dim), dtype)
    slots = rng.permutation(pages * PAGE)[:tokens]
    want = expected_bytes(pages, heads, dim, slots, k, v)
    data = torch.full((pages, heads, 76 * dim), 0xA5, dtype=torch.uint8, device="cuda")
    cache = lce.KV4Cache(heads, dim, data=data)
    at = torch.from_numpy(slots).cuda()
    lce.kv4_append(cache, k.cuda(), v.cuda(), at)
    assert np.array_equal(data.cpu().numpy(), want.data)
    for out in ("f32", "bf16", "f16"):
        got = lce.kv4_read(cache, at, dtype=DTYPES[out])
        for i in range(2):
            exact = torch.from_numpy(np.stack([want.read(s)[i] for s in slots]))
            assert torch.equal(got[i].cpu(), exact.to(DTYPES[out])), (out, i)


def test_long_append_and_read_take_four_tokens_a_thread():
    """Enough tokens for the variant with four in flight, a last workgroup partly filled."""
    rng = np.random.default_rng(1)
    tokens, heads, dim = 8192 + 11, 8, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    k, v = (torch.randn(tokens, heads, dim, device="cuda", generator=g).bfloat16()
            for _ in range(2))
    pages = tokens // PAGE + 2
    slots = rng.permutation(pages * PAGE)[:tokens]
    at = torch.from_numpy(slots).cuda()
    cache = lce.KV4Cache(heads, dim, pages=pages)
    lce.kv4_append(cache, k, v, at)
    got = lce.kv4_read(cache, at, dtype=torch.float32)
    for x, y in ((k, got[0]), (v, got[1])):
        codes, byte, _ = ref.quantise(x.cpu().double().numpy())
        assert np.array_equal(ref.values(codes, byte), y.cpu().double().numpy())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_reads_of_more_than_the_caches_hold(dtype):
    """The same values as in smaller pieces."""
    heads, dim, pages = 8, 256, 205
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    data = torch.randint(0, 256, (pages, heads, 76 * dim), dtype=torch.uint8, device="cuda",
                         generator=g)
    data[:, :, 64 * dim:68 * dim] = data[:, :, 64 * dim:68 * dim] % 16 + 120
    cache = lce.KV4Cache(heads, dim, data=data)
    slots = torch.randperm(pages * PAGE, device="cuda", generator=g)
    k, v = lce.kv4_read(cache, slots, dtype=DTYPES[dtype])
    assert k.numel() * k.element_size() * 2 > 100 << 20
    for at in range(0, len(slots), 1500):
        a, b = lce.kv4_read(cache, slots[at:at + 1500], dtype=DTYPES[dtype])
        assert torch.equal(k[at:at + 1500], a) and torch.equal(v[at:at + 1500], b)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_append_takes_strided_rows_and_drops_slots_outside(dtype):
    rng = np.random.default_rng(5)
    heads, dim, tokens, pages = 2, 64, 33, 2
    rows = special(rng, (tokens, 5 * heads, dim), dtype).cuda()
    k, v = rows[:, 3 * heads:4 * heads], rows[:, 4 * heads:].transpose(0, 1).contiguous()
    v = v.transpose(0, 1)                               # heads outermost in memory
    slots = rng.permutation(pages * PAGE)[:tokens]
    slots[4], slots[9], slots[10] = -1, pages * PAGE, 2 ** 40
    data = torch.full((pages, heads, 76 * dim), 0xA5, dtype=torch.uint8, device="cuda")
    cache = lce.KV4Cache(heads, dim, data=data)
    at = torch.from_numpy(slots).cuda()
    lce.kv4_append(cache, k, v, at)
    want = expected_bytes(pages, heads, dim, slots, k.cpu(), v.cpu())
    assert np.array_equal(data.cpu().numpy(), want.data)
    got = lce.kv4_read(cache, at, dtype=torch.float32)
    for i in (4, 9, 10):
        assert not got[0][i].any() and not got[1][i].any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_append_of_values_that_are_not_finite(dim, dtype):
    rng = np.random.default_rng(6)
    heads, tokens = 2, 12
    k, v = (torch.from_numpy(rng.standard_normal((tokens, heads, dim))).to(DTYPES[dtype])
            for _ in range(2))
    k[1, 0, 3], k[2, 1, dim - 1], v[4, 0, 33], v[5, 1, 0], v[6, 0, 5] = NAN, INF, -INF, NAN, NAN
    k[6, 0, 40] = -INF
    slots = np.arange(tokens) * 5
    want = expected_bytes(1, heads, dim, slots, k, v)
    data = torch.full((1, heads, 76 * dim), 0xA5, dtype=torch.uint8, device="cuda")
    cache = lce.KV4Cache(heads, dim, data=data)
    lce.kv4_append(cache, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
    assert np.array_equal(data.cpu().numpy(), want.data)
    rk, rv = lce.kv4_read(cache, torch.from_numpy(slots).cuda(), dtype=torch.float32)
    assert rk[1, 0].isnan().all() and rk[4, 0].isnan().all()
    assert rv[4, 0, 32:64].isnan().all() and rv[4, 0, :32].isfinite().all()
    assert rk[1, 1].isfinite().all() and rv[1].isfinite().all()


def test_no_tokens_is_no_work():
    cache = lce.KV4Cache(2, 64, pages=1)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    x = torch.empty(0, 2, 64, device="cuda")
    lce.kv4_append(cache, x, x, none)
    k, v = lce.kv4_read(cache, none)
    assert k.shape == v.shape == (0, 2, 64)


def test_cache_of_more_than_four_gib():
    """Records past 2^32 bytes: written, read, attended to and scored at their own place."""
    heads, dim, pages = 8, 256, 28000                   # 4.36e9 bytes
    cache = lce.KV4Cache(heads, dim, pages=pages)
    b = Batch(11, [130], [1], 16, heads, dim, "bf16")
    far = [pages - 1, 3, pages - 2]
    table = torch.tensor([far], dtype=torch.int32, device="cuda")
    for i, page in enumerate(far):
        cache.data[page] = torch.from_numpy(b.cache.data[b.table[0, i]]).cuda()
    _, q, _, start, lengths = b.device(lce)
    out, lse = lce.kv4_attention(cache, q, table, start, lengths, return_lse=True)
    check_attention(b, out, lse, 1 / 16)
    got = lce.kv4_select(cache, q, table, start, lengths, 2)
    assert np.array_equal(got.cpu().numpy(), b.select(2))
    slots = torch.tensor([far[0] * PAGE + 7, far[2] * PAGE + 1], device="cuda")
    k, v = lce.kv4_read(cache, slots, dtype=torch.float32)
    assert np.array_equal(k.cpu().double().numpy(), b.k[0][[7, 129]])
    assert np.array_equal(v.cpu().double().numpy(), b.v[0][[7, 129]])
    lce.kv4_append(cache, v, k, slots)
    k2, v2 = lce.kv4_read(cache, slots, dtype=torch.float32)
    assert torch.equal(k2, v) and torch.equal(v2, k)


# ---- attention

def check_attention(b, out, lse, scale, causal=True, window=0, pages=None):
    want, want_lse, bound, lse_bound = b.attention(scale, causal, window, pages)
    near = np.abs(out.cpu().double().numpy() - want) <= bound
    assert near.all(), np.argwhere(~near)[:5]
    got = lse.cpu().double().numpy()
    empty = np.isinf(want_lse)
    assert np.array_equal(np.isneginf(got), empty)
    near = np.abs(got[~empty] - want_lse[~empty]) <= lse_bound[~empty]
    assert near.all()


def attend(b, causal=True, window=0, pages=None, scale=None, **kw):
    scale = b.dim ** -0.5 if scale is None else scale
    dev = None if pages is None else torch.from_numpy(pages).cuda()
    out, lse = lce.kv4_attention(*b.device(lce), scale=scale, causal=causal, window=window,
                                 pages=dev, return_lse=True, **kw)
    check_attention(b, out, lse, scale, causal, window, pages)
    return out, lse


LENGTHS = [200, 0, 1, 63, 64, 65, 130, 2, 321]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 2), (5, 1), (24, 1)])
@pytest.mark.parametrize("chunk", [0, 1, 3])
def test_single_tokens(dim, dtype, q_heads, kv_heads, chunk):
    queries = [min(1, n) for n in LENGTHS]
    b = Batch(dim + q_heads, LENGTHS, queries, q_heads, kv_heads, dim, dtype)
    with lce.tuning(kv4_chunk=chunk):
        attend(b, max_q=1, max_len=321)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 40), (False, 70), (True, 1)])
@pytest.mark.parametrize("chunk", [0, 2])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_several_tokens(dim, dtype, causal, window, chunk, rows):
    lengths, queries = [150, 3, 64, 0, 90, 129], [5, 3, 1, 0, 90, 17]
    b = Batch(dim, lengths, queries, 6, 2, dim, dtype)
    with lce.tuning(kv4_chunk=chunk, kv4_rows=rows):
        attend(b, causal, window)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_prompts(dim, dtype):
    """Tiles of 32 and 128 rows that are full, that several pages are whole for, and whose last
    waves have no rows; sequences shorter than their tile."""
    b = Batch(25, [260, 33, 500, 1], [260, 33, 111, 1], 5, 1, dim, dtype)
    out, lse = attend(b, max_q=260)
    again = lce.kv4_attention(*b.device(lce), max_q=260)
    assert torch.equal(out, again)
    for rows in (32, 128):
        with lce.tuning(kv4_rows=rows, kv4_chunk=1):
            attend(b, window=77)


@pytest.mark.parametrize("rows", [16, 32, 128])
def test_more_queries_than_tokens_leave_rows_that_see_nothing(rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(3, [4, 70], [7, 2], 4, 2, 64, "bf16")
    for causal in (True, False):
        out, lse = attend(b, causal)
        if causal:
            assert not out[:3].any() and torch.isneginf(lse[:3]).all()


@pytest.mark.parametrize("rows", [16, 32, 128])
def test_no_sequence_has_tokens(rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(3, [0, 0], [2, 1], 4, 2, 128, "f16")
    for causal in (True, False):
        out, lse = attend(b, causal)
        assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_many_sequences_and_long_ones(dtype, rows):
    """More sequences than lanes; one long enough that a wave takes several of its pages."""
    lce.set_tuning(kv4_rows=rows)
    rng = np.random.default_rng(2)
    lengths = [int(n) for n in rng.integers(0, 90, 150)]
    lengths[77] = 1900
    queries = [min(n, int(x)) for n, x in zip(lengths, rng.integers(0, 4, 150))]
    b = Batch(8, lengths, queries, 4, 1, 64, dtype)
    attend(b)
    lce.set_tuning(kv4_chunk=1000)
    attend(b, max_len=1900)


@pytest.mark.parametrize("kv_heads,lengths", [
    (1, [700, 64, 1, 3000, 65, 128, 900, 2]),
    (1, [5000] + [7] * 6 + [64] * 8 + [400]),
    (2, [2100, 30, 1, 640]),
    (4, [1900, 3000])])
@pytest.mark.parametrize("q_len", [1, 3])
@pytest.mark.parametrize("chunk", [0, 1, 5])
def test_splits_of_a_few_heads_of_ragged_sequences(kv_heads, lengths, q_len, chunk):
    q_lens = [min(q_len, n) for n in lengths]
    b = Batch(71, lengths, q_lens, 4 * kv_heads, kv_heads, 128, "bf16")
    with lce.tuning(kv4_chunk=chunk):
        attend(b)


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "bf16"), (128, "f16")])
def test_many_short_prompts_and_ones_on_a_past(dim, dtype):
    rng = np.random.default_rng(72)
    lengths = [int(x) for x in rng.integers(60, 400, 10)]
    attend(Batch(73, lengths, [min(n, 128) for n in lengths], 32, 8, dim, dtype))
    attend(Batch(74, [700, 3, 1000, 64], [700, 3, 900, 64], 32, 4, dim, dtype))


def test_hints_that_are_wrong_cost_no_result():
    b = Batch(9, [700, 20], [3, 20], 8, 2, 128, "bf16")
    for max_q, max_len in ((1, 1), (1, 64), (4000, 10 ** 6), (None, None)):
        attend(b, max_q=max_q, max_len=max_len)


@pytest.mark.parametrize("window", [0, 30])
def test_hints_at_the_ends_of_their_range(window):
    b = Batch(75, [900, 64, 1, 200], [1, 2, 1, 3], 8, 2, 128, "bf16")
    for max_q in (1, 2 ** 31 - 1):
        for max_len in (1, 2 ** 31 - 1):
            attend(b, window=window, max_q=max_q, max_len=max_len)


def test_strided_queries_and_scale():
    b = Batch(10, [100, 50], [3, 50], 6, 3, 64, "bf16")
    cache, q, table, start, lengths = b.device(lce)
    rows = torch.empty(q.shape[0], 12, 64, dtype=q.dtype, device="cuda").fill_(NAN)
    rows[:, 2:8] = q
    out, lse = lce.kv4_attention(cache, rows[:, 2:8], table, start, lengths, scale=0.3,
                                 return_lse=True)
    check_attention(b, out, lse, 0.3)
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)
    again, _ = lce.kv4_attention(cache, turned, table, start, lengths, scale=0.3, return_lse=True)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("spread", [1e-3, 30.0])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_flat_and_sharp_scores(dtype, spread, rows):
    """Scores that are all alike, and rows that one token takes nearly whole (large maxima that
    rise from page to page)."""
    lce.set_tuning(kv4_rows=rows)
    b = Batch(12, [500], [2], 4, 1, 128, dtype)
    attend(b, scale=spread / 11.3)


@pytest.mark.parametrize("dtype,tiny,huge", [("bf16", 2.0 ** -70, 2.0 ** 60), ("f16", 2.0 ** -22, 2.0 ** 14)])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_queries_of_any_size(dtype, tiny, huge, rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(13, [90], [6], 2, 1, 64, dtype)
    rng = np.random.default_rng(0)
    q = b.q.double().numpy()
    q[0] *= tiny
    q[1] = 0
    q[2] = np.sign(q[2]) * huge * rng.uniform(0.5, 1, q[2].shape)
    q[3, :, ::7] *= 2.0 ** -9                            # one row of very different channels
    b.q = torch.from_numpy(q).to(DTYPES[dtype])
    attend(b, scale=1.0 / huge)
    attend(b, scale=0.125 if dtype == "f16" else 2.0 ** -40)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_tokens_without_a_number_reach_only_rows_that_see_them(dtype, rows):
    with lce.tuning(kv4_rows=rows):
        tokens_without_a_number(dtype)


def tokens_without_a_number(dtype):
    odd = [(0, 70, 0, 5, "k", NAN), (0, 95, 1, 3, "v", INF), (1, 0, 0, 60, "v", NAN)]
    b = Batch(14, [100, 80], [40, 3], 4, 2, 64, dtype, odd=odd)
    out, lse = lce.kv4_attention(*b.device(lce), return_lse=True)
    want, want_lse, bound, _ = b.attention(0.125)
    bad = np.isnan(want_lse)
    assert bad.any() and not bad.all()
    got = out.cpu().double().numpy()
    assert np.array_equal(np.isnan(lse.cpu().numpy()), bad)
    assert np.isnan(got[bad]).all()
    assert np.all(np.abs(got - want)[~bad] <= bound[~bad])
    # a window that has left token 70 behind
    out, lse = lce.kv4_attention(*b.device(lce), window=4, return_lse=True)
    want, want_lse, bound, _ = b.attention(0.125, window=4)
    bad = np.isnan(want_lse)
    assert np.array_equal(np.isnan(lse.cpu().numpy()), bad)
    assert np.all(np.abs(out.cpu().double().numpy() - want)[~bad] <= bound[~bad])


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_query_rows_without_a_number(value, rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(15, [70, 9], [2, 1], 4, 2, 128, "bf16")
    clean = attend(b)[0]
    b.q[1, 2, 77] = value
    out, lse = lce.kv4_attention(*b.device(lce), return_lse=True)
    assert out[1, 2].isnan().all() and lse[1, 2].isnan()
    out[1, 2] = clean[1, 2]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("rows", [16, 32, 128])
def test_pages_outside_the_cache_are_hidden(rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(16, [200], [2], 4, 2, 64, "bf16")
    cache, q, table, start, lengths = b.device(lce)
    for bad in (-1, b.cache.pages, 2 ** 31 - 1, -2 ** 31):
        table[0, 1] = bad
        out, lse = lce.kv4_attention(cache, q, table, start, lengths, return_lse=True)
        only = np.broadcast_to(np.array([0, 2, 3], np.int32), (2, 2, 3))
        check_attention(b, out, lse, 0.125, pages=only)
        assert not (lce.kv4_select(cache, q, table, start, lengths, 4) == 1).any()


@pytest.mark.parametrize("rows", [16, 32, 128])
def test_array_values_outside_their_range(rows):
    """q_start and lengths are forced into range on the device; other rows stay as they are."""
    lce.set_tuning(kv4_rows=rows)
    b = Batch(17, [100, 64], [2, 1], 4, 2, 64, "f16")
    cache, q, table, start, lengths = b.device(lce)
    want = lce.kv4_attention(cache, q, table, start, lengths)
    out = torch.full_like(q, 7.0)
    start[-1] = 2 ** 31 - 1                            # rows end with q
    lce.kv4_attention(cache, q, table, start, lengths, out=out)
    assert torch.equal(out, want)
    start.copy_(torch.tensor([0, 2, 2]))               # the last row is nobody's
    out.fill_(7.0)
    lce.kv4_attention(cache, q, table, start, lengths, out=out)
    assert torch.equal(out[:2], want[:2]) and (out[2] == 7.0).all()
    lengths[0] = 2 ** 31 - 1                           # table of 2 pages: 128 tokens
    out, lse = lce.kv4_attention(cache, q, table, torch.tensor([0, 2, 3], dtype=torch.int32).cuda(),
                                 lengths, return_lse=True)
    assert torch.equal(out[2], want[2])
    lengths[0] = -5
    out, lse = lce.kv4_attention(cache, q, table, start, lengths, return_lse=True)
    assert not out[:2].any() and torch.isneginf(lse[:2]).all()


@pytest.mark.parametrize("rows", [16, 32, 128])
def test_windows_and_scales_at_the_ends_of_their_range(rows):
    lce.set_tuning(kv4_rows=rows)
    b = Batch(27, [90, 3], [5, 3], 2, 1, 64, "bf16")
    for causal in (True, False):
        for window in (2 ** 31 - 1, 2 ** 30, 91):
            attend(b, causal, window)
    b = Batch(27, [2, 90], [9, 3], 2, 1, 64, "bf16")     # positions below 0
    attend(b, False, 2 ** 31 - 1)
    # scores of about 10^34: each row is the token with the largest one
    args = b.device(lce)
    args[1].mul_(2.0 ** 100)
    out, lse = lce.kv4_attention(*args, scale=1e3, return_lse=True)
    q = args[1].cpu().double().numpy()
    for t in range(9, 12):
        for h in range(2):
            best = np.argmax((b.k[1][:, 0] @ q[t, h])[:88 + t - 9])
            assert np.array_equal(out[t, h].cpu().double().numpy(), b.v[1][best, 0])
    assert lse[9:].isfinite().all()


def test_same_bits_every_time_and_workspace_left_ready():
    b = Batch(18, [900, 40], [1, 1], 16, 2, 128, "bf16")
    args = b.device(lce)
    ws = lce.kv4_workspace(args[0], args[1], args[2])
    with lce.tuning(kv4_chunk=1):
        first = lce.kv4_attention(*args, return_lse=True, workspace=ws)
        pages = lce.kv4_select(*args, 3, workspace=ws)
        for _ in range(5):
            again = lce.kv4_attention(*args, return_lse=True, workspace=ws)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
            assert torch.equal(lce.kv4_select(*args, 3, workspace=ws), pages)
            assert not ws[:lce.KV4_WORKSPACE_ZERO].any()


def test_streams_and_graphs():
    """On a stream of its own, and captured: every replay is checked, with eager work between."""
    b = Batch(19, [700, 130], [1, 1], 8, 2, 128, "f16")
    cache, q, table, start, lengths = b.device(lce)
    with lce.tuning(kv4_chunk=2):
        want = lce.kv4_attention(cache, q, table, start, lengths)
        ws = lce.kv4_workspace(cache, q, table)
        out, pages = torch.empty_like(q), torch.empty(2, 2, 4, dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            lce.kv4_attention(cache, q, table, start, lengths, out=out, workspace=ws)
        side.synchronize()
        assert torch.equal(out, want)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lce.kv4_select(cache, q, table, start, lengths, 4, out=pages, workspace=ws)
            lce.kv4_attention(cache, q, table, start, lengths, pages=pages, out=out, workspace=ws)
        for i in range(4):
            q.copy_(torch.randn_like(q))
            ws2 = lce.kv4_workspace(cache, q, table)
            chosen = lce.kv4_select(cache, q, table, start, lengths, 4, workspace=ws2)
            want = lce.kv4_attention(cache, q, table, start, lengths, pages=chosen, workspace=ws2)
            out.fill_(0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(pages, chosen) and torch.equal(out, want), i


def test_the_binding_says_what_is_wrong():
    b = Batch(26, [70, 3], [2, 1], 4, 2, 64, "bf16")
    cache, q, table, start, lengths = b.device(lce)
    k = torch.zeros(3, 2, 64, device="cuda")
    slots = torch.arange(3, device="cuda")
    lce.kv4_append(cache, k[:0], k[:0], slots[:0])
    for bad, error in (((k.double(), k.double(), slots), TypeError), ((k, k.half(), slots), TypeError),
                       ((k, k[:2], slots), ValueError), ((k[:, :1], k[:, :1], slots), ValueError),
                       ((k, k, slots.int()), TypeError), ((k, k, slots[:2]), ValueError),
                       ((k, k, slots.cpu()), ValueError), ((k.cpu(), k, slots), ValueError),
                       ((k, k, [0, 1, 2]), TypeError), ((None, k, slots), TypeError),
                       ((k[0], k[0], slots), ValueError),
                       ((k.transpose(1, 2).contiguous().transpose(1, 2), k, slots), ValueError)):
        with pytest.raises(error):
            lce.kv4_append(cache, *bad)
    odd = torch.zeros(3, 2, 65, device="cuda")[:, :, :64]
    with pytest.raises(lce.LceError):
        lce.kv4_append(cache, odd, odd, slots)
    good = dict(q=q, table=table, q_start=start, lengths=lengths)
    for name, value, error in (("q", q.float(), TypeError), ("q", q.cpu(), ValueError),
                               ("q", q[:, :, :32], ValueError), ("q", q[0], ValueError),
                               ("q", None, TypeError), ("table", table.long(), TypeError),
                               ("table", table[0], ValueError), ("table", table[:, :1], ValueError),
                               ("q_start", start[:2], ValueError), ("q_start", start.cpu(), ValueError),
                               ("lengths", lengths[:1], ValueError), ("lengths", [70, 3], TypeError)):
        with pytest.raises(error):
            lce.kv4_attention(cache, **{**good, name: value})
        with pytest.raises(error):
            lce.kv4_select(cache, **{**good, name: value}, count=2)
    with pytest.raises(lce.LceError):
        lce.kv4_attention(cache, q[:, :3].contiguous(), table, start, lengths)
    with pytest.raises(lce.LceError):
        lce.kv4_select(cache, *good.values(), 0)
    for kw in (dict(out=q.float()), dict(out=q[:2]), dict(pages=table[:, None]),
               dict(workspace=torch.zeros(10, device="cuda")), dict(pages=torch.zeros(3, 2, 0).int().cuda())):
        with pytest.raises((TypeError, ValueError)):
            lce.kv4_attention(cache, **good, **kw)
    with pytest.raises(lce.LceError):
        lce.kv4_attention(cache, **good, workspace=torch.zeros(10, dtype=torch.uint8, device="cuda"))
    for kw in (dict(dtype=torch.int32), dict(out=(k, k[:2])), dict(out=(k.cpu(), k))):
        with pytest.raises((TypeError, ValueError)):
            lce.kv4_read(cache, slots, **kw)
    with pytest.raises(TypeError):
        lce.kv4_read(cache, slots.int())
    with pytest.raises(ValueError):
        lce.kv4_read(cache, slots[None])
    with pytest.raises(ValueError):
        lce.KV4Cache(2, 64, data=torch.zeros(3, 2, 64, dtype=torch.uint8, device="cuda"))
    out = torch.empty(3, 2, 64, device="cuda"), torch.empty(3, 2, 64, device="cuda")
    assert lce.kv4_read(cache, slots, out=out)[0] is out[0]
    assert torch.equal(out[0], lce.kv4_read(cache, slots, dtype=torch.float32)[0])


# ---- lists of pages, and choosing them

@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads", [(2, 2), (8, 2), (20, 1)])
@pytest.mark.parametrize("chunk", [0, 1])
def test_lists(dim, dtype, q_heads, kv_heads, chunk):
    lengths, queries = [400, 65, 1, 0, 130], [2, 1, 1, 0, 5]
    b = Batch(20, lengths, queries, q_heads, kv_heads, dim, dtype)
    pages = np.full((b.tokens, kv_heads, 5), -1, np.int32)
    for t in range(b.tokens):
        for h in range(kv_heads):
            n = b.rng.integers(0, 6)
            pages[t, h, :n] = b.rng.permutation(9)[:n]     # past some lengths, in any order
    pages[0, 0, 4] = 2 ** 31 - 1
    with lce.tuning(kv4_chunk=chunk):
        attend(b, pages=pages)
        attend(b, causal=False, window=90, pages=pages)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tables_and_lists_so_wide_that_loads_pass_the_caches(dtype):
    """What the call says of its size decides; the tokens are few all the same."""
    b = Batch(28, [300, 70, 1], [1, 1, 1], 8, 2, 128, dtype, width=20000)
    attend(b)
    pages = np.full((b.tokens, 2, 9000), -1, np.int32)
    for t in range(3):
        for h in range(2):
            pages[t, h, b.rng.permutation(9000)[:5]] = b.rng.permutation(5)
    attend(b, pages=pages)


def test_a_list_of_all_pages_is_no_list():
    b = Batch(21, [500, 64], [3, 1], 8, 2, 128, "bf16")
    every = np.broadcast_to(np.arange(8, dtype=np.int32), (4, 2, 8)).copy()
    attend(b, pages=every)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 2), (20, 1)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 150)])
@pytest.mark.parametrize("chunk", [0, 1, 3])
def test_select(dim, q_heads, kv_heads, causal, window, chunk):
    lengths, queries = [900, 65, 1, 0, 330, 64], [2, 1, 1, 0, 5, 2]
    b = Batch(22, lengths, queries, q_heads, kv_heads, dim, "bf16")
    args = b.device(lce)
    with lce.tuning(kv4_chunk=chunk):
        for count, first, last in ((4, 1, 1), (1, 0, 0), (6, 0, 2), (3, 5, 5), (40, 1, 1)):
            got = lce.kv4_select(*args, count, keep_first=first, keep_last=last, causal=causal,
                                 window=window)
            assert np.array_equal(got.cpu().numpy(), b.select(count, first, last, causal, window))


@pytest.mark.parametrize("chunk", [0, 7])
def test_select_of_many_pages_with_many_ties(chunk):
    """More pages than threads, and keys of few kinds, so that most scores are tied."""
    b = Batch(23, [64], [1], 2, 1, 64, "f16")
    pages, width = 40, 700
    rng = np.random.default_rng(1)
    data = rng.integers(0, 256, (pages, 1, 76 * 64)).astype(np.uint8)
    table = rng.integers(0, pages, (1, width)).astype(np.int32)
    n = width * PAGE - 13
    qs = np.where(b.q[0].numpy() < 0, -1, 1).astype(np.int64)
    bits = np.unpackbits(data[:, 0, 68 * 64:].reshape(pages, PAGE, 8), axis=-1, bitorder="little")
    score = ((1 - 2 * bits.astype(np.int64)) @ qs.T).sum(-1)
    best = score[table[0]]
    best[-1, PAGE - 13:] = -10 ** 6
    best = best.max(-1)
    cache = lce.KV4Cache(1, 64, data=torch.from_numpy(data).cuda())
    args = (b.q.cuda(), torch.from_numpy(table).cuda(),
            torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda())
    with lce.tuning(kv4_chunk=chunk):
        for count in (1, 5, 100, 699, 700, 800):
            got = lce.kv4_select(cache, *args, count, keep_first=0, keep_last=0).cpu().numpy()[0, 0]
            order = np.lexsort((np.arange(width), -best))[:count]
            want = np.full(count, -1)
            want[:len(order)] = np.sort(order)
            assert np.array_equal(got, want), count


def test_select_of_sign_zero_and_nan_queries():
    """-0 and NaN count as +1, as bitpack has them."""
    b = Batch(24, [200], [1], 2, 1, 64, "bf16")
    b.q[0, 0, :20] = -0.0
    got = lce.kv4_select(*b.device(lce), 2, keep_first=0, keep_last=0)
    b.q[0, 0, :20] = 0.0
    assert np.array_equal(got.cpu().numpy(), b.select(2, 0, 0))
    b.q[0, 0, :20] = NAN
    again = lce.kv4_select(*b.device(lce), 2, keep_first=0, keep_last=0)
    assert torch.equal(got, again)


# ---- all of it together

def test_the_decoding_example():
    """Prompts and steps as a serving loop runs them.  With all pages kept, sparse steps are
    dense ones; the 4-bit format's error of each key and value, about 0.11 of its size
    (a step of at most a quarter of a value between 1 and 2 of its binade, half of that at
    most, and a shared scale), is averaged by the sums and stays below 0.25."""
    import importlib.util
    import os
    from tests.conftest import ROOT
    spec = importlib.util.spec_from_file_location("kv4_decoding",
                                                  os.path.join(ROOT, "examples", "kv4_decoding.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run(seqs=3, prompt=300, steps=10, keep=6, q_heads=8, kv_heads=2, dim=64)
    assert r["prompt"] < 0.25 and r["dense"] < 0.25
    assert abs(r["sparse"] - r["dense"]) < 0.02        # 6 pages hold 310 tokens
    assert abs(r["size"] - 76 / 256) < 1e-6
