"""Attention over the 4-bit cache at the ends of its types' ranges, against the definition in
64 bits (kv4_util)."""
import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests.kv4_util import PAGE, Batch

pytestmark = pytest.mark.gpu

MOST = 65504.0        # the largest float16


def check(b, out, lse, scale, causal=True, window=0, pages=None):
    want, want_lse, bound, lse_bound = b.attention(scale, causal, window, pages)
    off = np.abs(out.cpu().double().numpy() - want)
    assert (off <= bound).all(), (np.argwhere(~(off <= bound))[:5], np.nanmax(off / bound))
    got = lse.cpu().double().numpy()
    empty = np.isinf(want_lse)
    assert np.array_equal(np.isneginf(got), empty)
    assert (np.abs(got[~empty] - want_lse[~empty]) <= lse_bound[~empty]).all()


def attend(b, causal=True, window=0, pages=None, scale=None):
    scale = b.dim ** -0.5 if scale is None else scale
    dev = None if pages is None else torch.from_numpy(pages).cuda()
    return lce.kv4_attention(*b.device(lce), scale=scale, causal=causal, window=window, pages=dev,
                             return_lse=True)


# ---- float16 queries over values that float16 does not hold: they count as +-65504, on
# ---- whole pages and on others, and what shares their scales keeps its own values

def large_values(seed, lengths, dim, heads):
    """Every ninth token of a head has a group of values around 2^14 to 2^18, with small ones
    among them (code 1 of a scale of 2^14 to 2^17), a few tokens around 2^60."""
    rng = np.random.default_rng(seed)
    odd = []
    for b, n in enumerate(lengths):
        for h in range(heads):
            for j in range(h, n, 9):
                g = int(rng.integers(0, dim // 32))
                up = 2.0 ** (60 if j % 5 == 0 else int(rng.integers(13, 17)))
                x = rng.uniform(-4, 4, 32) * np.where(rng.random(32) < 0.5, 0.2, 1.0)
                odd += [(b, j, h, 32 * g + c, "v", x[c] * up) for c in range(32)]
    return odd


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 70)])
def test_values_past_float16(dim, rows, causal, window):
    lengths, queries = [200, 128, 77, 130], [1, 90, 5, 130]
    b = Batch(31, lengths, queries, 4, 2, dim, "f16", odd=large_values(dim, lengths, dim, 2))
    assert max(np.abs(v).max() for v in b.v) > MOST
    b.v = [np.clip(v, -MOST, MOST) for v in b.v]
    for chunk in (0, 1):
        with lce.tuning(kv4_rows=rows, kv4_chunk=chunk):
            out, lse = attend(b, causal, window)
        check(b, out, lse, dim ** -0.5, causal, window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_values_past_float16_in_lists(dim):
    lengths, queries = [300, 70], [2, 1]
    b = Batch(32, lengths, queries, 8, 2, dim, "f16", odd=large_values(7, lengths, dim, 2))
    b.v = [np.clip(v, -MOST, MOST) for v in b.v]
    pages = np.full((3, 2, 4), -1, np.int32)
    pages[:2, 0, :3], pages[:2, 1, :4], pages[2, :, :2] = [0, 2, 4], [4, 1, 3, 0], [0, 1]
    out, lse = attend(b, pages=pages)
    check(b, out, lse, dim ** -0.5, pages=pages)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_float16_results_do_not_depend_on_the_page_being_whole(dim, rows):
    """One token of 65536 beside 16384 in one group: alone on its page, and with 64 tokens."""
    odd = [(0, 0, 0, 0, "v", 65536.0), (0, 0, 0, 1, "v", 16384.0), (0, 0, 0, 2, "v", -2.0 ** 17)]
    with lce.tuning(kv4_rows=rows):
        for n in (1, PAGE):
            b = Batch(33, [n], [1], 1, 1, dim, "f16", odd=odd)
            b.k[0][:] = 0                              # equal scores: the mean of the values
            b.q[:] = 0
            b.v = [np.clip(v, -MOST, MOST) for v in b.v]
            out, lse = attend(b)
            check(b, out, lse, dim ** -0.5)
            if n == 1:
                assert out[0, 0, :3].tolist() == [MOST, 16384.0, -MOST]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("byte", [141, 252, 254])
def test_bytes_of_slots_never_written_do_not_count(dtype, dim, rows, byte):
    """Codes 6 and scales of any size past the sequences' ends leave no trace."""
    b = Batch(34, [100, 70, 3], [40, 2, 1], 4, 2, dim, dtype)
    with lce.tuning(kv4_rows=rows):
        clean = attend(b)
        for s, n in enumerate(b.lengths):
            for t in range(n % PAGE, PAGE):
                rec = b.cache.data[b.table[s, n // PAGE]]
                for part, fill in zip(b.cache.places(t), (0x77, 0x77, byte, byte, 0x55)):
                    rec[:, part] = fill
        junk = attend(b)
    assert torch.equal(clean[0], junk[0]) and torch.equal(clean[1], junk[1])


# ---- weights and scores at the ends of their ranges

def fill(cache, keys, values):
    """keys, values [tokens, dim] of the cache's only head, in pages in order; the call's
    table, q_start and lengths for one sequence with one new token."""
    n = keys.shape[0]
    lce.kv4_append(cache, keys.cuda().bfloat16()[:, None].contiguous(),
                   values.cuda().bfloat16()[:, None].contiguous(), torch.arange(n).cuda())
    return (torch.arange(cache.pages, dtype=torch.int32).cuda()[None].contiguous(),
            torch.tensor([0, 1], dtype=torch.int32).cuda(),
            torch.tensor([n], dtype=torch.int32).cuda())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_scores_whose_last_place_is_sixteen(dtype, rows):
    """Scores of 2^27 + 16, then of 2^27 + 32 (log2): adjacent float32, 16 apart.  Weights
    of 2^16 would be past float16."""
    scale = np.float32(1 / np.log2(np.e))
    while scale * np.float32(np.log2(np.e)) != 1:
        scale = np.nextafter(scale, np.float32(0))
    keys, values = torch.zeros(300, 64), torch.ones(300, 64)
    keys[:, 0], keys[:, 32], keys[256:, 32], values[256:] = 2.0 ** 27, 16, 32, 2
    q = torch.zeros(1, 1, 64, dtype=dtype)
    q[..., 0] = q[..., 32] = 1
    cache = lce.KV4Cache(1, 64, pages=5)
    with lce.tuning(kv4_rows=rows, kv4_chunk=5):
        out, lse = lce.kv4_attention(cache, q.cuda(), *fill(cache, keys, values),
                                     scale=float(scale), return_lse=True)
    # 44 tokens of 2, and 256 of 1 that weigh 2^-16 each: within 4e-5 of 2
    assert (out == 2).all()
    # the maximum and the sum's logarithm (6), in a last place of 16; then of 8
    assert abs(lse.item() - (2.0 ** 27 + 32 + np.log2(44)) * np.log(2)) <= 8 + 4 + 8


def one_large(gap, dtype, rows, n=65536):
    """Attention over one token in each of the first four pages that weighs e^gap times as
    much as each of n - 4 others, whose values are 1; what the others weigh together."""
    keys, values = torch.zeros(n, 64), torch.ones(n, 64)
    keys[0:256:64, 0], values[0:256:64] = 1, 0
    q = torch.zeros(1, 1, 64, dtype=dtype)
    q[..., 0] = 1
    cache = lce.KV4Cache(1, 64, pages=n // PAGE)
    with lce.tuning(kv4_rows=rows, kv4_chunk=n // PAGE):
        out, lse = lce.kv4_attention(cache, q.cuda(), *fill(cache, keys, values), scale=gap,
                                     return_lse=True)
    return out.cpu().double().numpy(), lse.item(), (n - 4) * np.exp(-gap)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("gap", [5.0, 16.0, 17.0, 17.4])
def test_sums_of_many_small_weights_beside_a_large_one(dtype, rows, gap):
    """Sums of weights lose 2^-24 of the largest term at each of at most 4096 additions (16
    of a page, 1024 pages)."""
    _, lse, small = one_large(gap, dtype, rows)
    assert abs(lse - (gap + np.log(4 + small))) <= 4096 * 2.0 ** -24 + 2.0 ** -18


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("gap", [5.0, 16.0, 17.0, 17.4])
def test_many_small_weights_beside_a_large_one(dtype, rows, gap):
    """A weight is rounded to half a last place of its type, in float16 to half of 2^-24 at
    least, of which the largest is 2^7 times 2^24; so is the result; and sums lose 2^-24 of
    the largest term at each of 4096 additions."""
    out, _, small = one_large(gap, dtype, rows)
    want = small / (4 + small)
    ulp = 2.0 ** (-11 if dtype == torch.float16 else -8)
    bound = want * (2 * ulp + 4096 * 2.0 ** -24)
    if dtype == torch.float16:
        bound += 65532 * 2.0 ** -32 / (4 + small) + 2.0 ** -25
    assert np.abs(out - want).max() <= bound


# ---- rows that have nothing to do with each other

@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_a_channel_without_a_number_takes_its_row_alone(value, dtype, dim, rows):
    b = Batch(44, [70], [2], 4, 2, dim, dtype)
    with lce.tuning(kv4_rows=rows):
        clean = attend(b)
        for c in range(5, dim, 32):
            q = b.q.clone()
            b.q[1, 2, c] = value
            out, lse = attend(b)
            b.q = q
            assert out[1, 2].isnan().all() and lse[1, 2].isnan()
            out[1, 2], lse[1, 2] = clean[0][1, 2], clean[1][1, 2]
            assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
def test_no_bit_of_a_row_depends_on_the_rows_beside_it(dtype, dim, rows):
    """A row whose scores grow from page to page, or are past 2^23, among ordinary ones."""
    b = Batch(45, [400], [2], 4, 1, dim, dtype)
    with lce.tuning(kv4_rows=rows, kv4_chunk=7):
        clean = attend(b)
        for up in (2.0 ** 6, 2.0 ** 15):
            b.q[1, 2] = (b.q[1, 2].double() / b.q[1, 2].abs().max().double() * up).to(b.q.dtype)
            out, lse = attend(b)
            out[1, 2], lse[1, 2] = clean[0][1, 2], clean[1][1, 2]
            assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


# ---- queries whose channels are of very different sizes

def spread_keys(seed, n, dim, up):
    """Keys whose groups of 32 channels have scales 2^up[g], as Batch takes them."""
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((n, dim)) * np.exp2(np.repeat(up, 32))
    return [(0, j, 0, c, "k", k[j, c]) for j in range(n) for c in range(dim)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("step", [16, 20, 24])
def test_groups_of_channels_far_apart(dtype, dim, rows, step):
    """Groups of a query 2^-step of each other's size, against keys that are as much
    larger there: each counts as much as the others."""
    if dtype == "f16":
        step -= 6                                      # to the ends of its normal numbers
    down = -step * (np.arange(dim // 32) % 2)
    b = Batch(41, [90], [3], 2, 1, dim, dtype, odd=spread_keys(41, 90, dim, -down))
    q = b.q.double() * torch.from_numpy(np.exp2(np.repeat(down, 32)))
    b.q = q.to(b.q.dtype)
    with lce.tuning(kv4_rows=rows):
        out, lse = attend(b)
    check(b, out, lse, dim ** -0.5)


@pytest.mark.parametrize("dtype,left", [("bf16", 2.0 ** -21), ("f16", 2.0 ** -25)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("down", [12, 16, 20])
def test_channels_of_one_group_far_apart(dtype, left, dim, rows, down):
    """One loud channel of each group of a query, of which the keys have nothing: the others
    are off by at most `left` of it."""
    quiet = np.arange(dim) % 32 != 7
    odd = [(0, j, 0, c, "k", 0.0) for j in range(90) for c in range(7, dim, 32)]
    b = Batch(42, [90], [3], 2, 1, dim, dtype, odd=odd)
    q = b.q.double().numpy()
    q[..., quiet] *= 2.0 ** -down
    q[..., ~quiet] = 1.5
    b.q = torch.from_numpy(q).to(b.q.dtype)
    scale = 2.0 ** down * dim ** -0.5
    with lce.tuning(kv4_rows=rows):
        out, lse = attend(b, scale=scale)
    want, want_lse, bound, lse_bound = b.attention(scale)
    score = scale * 1.5 * left * np.abs(b.k[0][:, 0]).sum(-1).max()
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    bound += np.expm1(2 * score) * np.abs(b.v[0][:, 0]).max()
    assert (np.abs(out - want) <= bound).all() and (np.abs(lse - want_lse) <= lse_bound + score).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("down", [100, 114, 118, 126, 131])
def test_bfloat16_queries_down_to_the_smallest(dim, rows, down):
    b = Batch(43, [90], [3], 2, 1, dim, "bf16", odd=spread_keys(43, 90, dim, np.full(dim // 32, 100)))
    b.q = (b.q.double() * 2.0 ** -down).to(b.q.dtype)
    assert b.q.any()
    scale = 2.0 ** (down - 100) * dim ** -0.5
    with lce.tuning(kv4_rows=rows):
        out, lse = attend(b, scale=scale)
    check(b, out, lse, scale)


# ---- arguments past 32 bits

def test_sizes_that_an_int32_would_hold_as_others():
    """A window of 2^32 + 5 was one of 5."""
    b = Batch(46, [200], [2], 4, 2, 64, "bf16")
    args = b.device(lce)
    for call, kw in ((lce.kv4_attention, dict(window=2 ** 32 + 5)),
                     (lce.kv4_attention, dict(window=-2 ** 32)),
                     (lce.kv4_attention, dict(max_q=2 ** 32 + 1)),
                     (lce.kv4_attention, dict(max_len=2 ** 31)),
                     (lce.kv4_select, dict(count=2, keep_first=2 ** 32)),
                     (lce.kv4_select, dict(count=2, keep_last=2 ** 32 + 1)),
                     (lce.kv4_select, dict(count=2, window=2 ** 32 + 70)),
                     (lce.kv4_select, dict(count=2 ** 32 + 2))):
        with pytest.raises(ValueError, match="int32"):
            call(*args, **kw)
    for kw in (dict(window=-1), dict(max_q=-1)):
        with pytest.raises(lce.LceError):
            lce.kv4_attention(*args, **kw)


# ---- workspaces of the size that a call asks for

@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [0, 16, 32, 128])
@pytest.mark.parametrize("lengths,queries,width", [
    ([1], [1], None), ([700], [1], None), ([700, 64, 1], [300, 5, 1], None),
    ([200] * 20, [3] * 20, 9), ([100, 30], [2, 1], 3000)])
def test_calls_stay_inside_the_workspace_they_ask_for(dim, rows, lengths, queries, width):
    b = Batch(47, lengths, queries, 4, 2, dim, "bf16", width=width)
    args = b.device(lce)
    pages = np.full((b.tokens, 2, 3), -1, np.int32)
    pages[:, :, 0] = 0
    guard = 1 << 16
    with lce.tuning(kv4_rows=rows, kv4_chunk=1):
        for only in ("attention", "select"):
            n = lce.kv4_workspace(*args[:3], only=only).numel()
            ws = torch.full((n + guard,), 0xA5, dtype=torch.uint8, device="cuda")
            ws[:lce.KV4_WORKSPACE_ZERO] = 0
            if only == "select":
                got = lce.kv4_select(*args, 2, workspace=ws[:n])
                assert np.array_equal(got.cpu().numpy(), b.select(2))
            else:
                out, lse = lce.kv4_attention(*args, workspace=ws[:n], return_lse=True)
                check(b, out, lse, dim ** -0.5)
                out, lse = lce.kv4_attention(*args, workspace=ws[:n], return_lse=True,
                                             pages=torch.from_numpy(pages).cuda())
                check(b, out, lse, dim ** -0.5, pages=pages)
            assert (ws[n:] == 0xA5).all() and not ws[:lce.KV4_WORKSPACE_ZERO].any()
            with pytest.raises(lce.LceError):
                (lce.kv4_select(*args, 2, workspace=ws[:n - 1]) if only == "select"
                 else lce.kv4_attention(*args, workspace=ws[:n - 1]))


def test_a_list_does_not_hide_what_is_wrong_with_q():
    b = Batch(48, [70], [1], 4, 2, 64, "bf16")
    cache, q, *rest = b.device(lce)
    pages = torch.zeros(1, 2, 1, dtype=torch.int32, device="cuda")
    for bad, error in ((None, TypeError), ([0], TypeError), (q.cpu(), ValueError), (q[0], ValueError)):
        with pytest.raises(error, match="q must"):
            lce.kv4_attention(cache, bad, *rest, pages=pages)
    for table, error in ((None, TypeError), (rest[0].long(), TypeError), (rest[0][0], ValueError)):
        with pytest.raises(error, match="table must"):
            lce.kv4_workspace(cache, q, table)
    with pytest.raises(ValueError, match="only must"):
        lce.kv4_workspace(cache, q, rest[0], only="read")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("chunk", [1, 9])
def test_a_mean_of_the_largest_values_is_finite(dim, rows, chunk):
    """All values count as 65504 in float16, and so does every mean of them: half a last
    place more, as weights are rounded, would be an infinity."""
    n = 300
    keys, values = torch.zeros(n, dim), torch.full((n, dim), 2.0 ** 17)
    values[:, 1::2] *= -1
    keys[256:, 0], keys[1:256, 1] = 1, 1               # page 4, in the wave of page 0
    q = torch.zeros(1, 24, dim, dtype=torch.float16)
    q[0, :, 0], q[0, :, 1] = torch.linspace(0.03, 8, 24), -60
    cache = lce.KV4Cache(1, dim, pages=5)
    with lce.tuning(kv4_rows=rows, kv4_chunk=chunk):
        out = lce.kv4_attention(cache, q.cuda(), *fill(cache, keys, values), scale=float(np.log(2)))
    want = torch.full((dim,), MOST, dtype=torch.float64)
    want[1::2] *= -1
    # weights rounded by half a last place, 2^-11, and the result by as much
    assert ((out[0].cpu().double() - want).abs() <= 2 * 2.0 ** -11 * MOST).all()
