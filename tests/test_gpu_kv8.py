"""The 8-bit cache's operators on the GPU against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2011_09398_amd as lce
from tests import kv8_util as ref

pytestmark = pytest.mark.gpu
PAGE = ref.PAGE


def values(rng, n, heads, dim, dtype, size=1.0):
    x = rng.standard_normal((n, heads, dim)) * np.exp(rng.standard_normal((n, 1, 1))) * size
    return torch.from_numpy(x).to(ref.DTYPES[dtype])


class Sequences:
    """A cache on the GPU and its oracle, appended to side by side."""

    def __init__(self, seed, seqs, width, heads, dim, fill=0xA5):
        self.rng = np.random.default_rng(seed)
        self.cache = ref.Cache(seqs * width + 2, heads, dim, fill)
        self.handle = lce.KV8Cache(heads, dim, data=torch.from_numpy(self.cache.data.copy()).cuda())
        order = self.rng.permutation(self.cache.pages)[:seqs * width]
        self.table = order.reshape(seqs, width).astype(np.int32)
        self.lengths = [0] * seqs
        self.heads, self.dim = heads, dim

    def append(self, counts, dtype, size=1.0, k=None, v=None):
        total = sum(counts)
        k = values(self.rng, total, self.heads, self.dim, dtype, size) if k is None else k
        v = values(self.rng, total, self.heads, self.dim, dtype, size) if v is None else v
        at = 0
        for b, n in enumerate(counts):
            self.lengths[b] += n
            if n:
                self.cache.append(self.table[b], self.lengths[b], k[at:at + n].double().numpy(),
                                  v[at:at + n].double().numpy())
            at += n
        start = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
        args = (self.handle, k.cuda(), v.cuda(), torch.from_numpy(self.table).cuda(), start,
                torch.tensor(self.lengths, dtype=torch.int32).cuda())
        lce.kv8_append(*args)
        return args

    def check(self):
        got = self.handle.data.cpu().numpy()
        bad = np.argwhere(got != self.cache.data)
        assert not len(bad), (len(bad), bad[:5].tolist(), [int(got[tuple(x)]) for x in bad[:5]],
                              [int(self.cache.data[tuple(x)]) for x in bad[:5]])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,dim", [(1, 64), (3, 128), (2, 256)])
def test_append_writes_the_defined_bytes(heads, dim, dtype):
    s = Sequences(dim + heads, 5, 4, heads, dim)
    for counts, size in (([0, 1, 17, 64, 100], 1.0), ([3, 1, 1, 0, 5], 0.01), ([1, 1, 1, 1, 1], 30.0),
                         ([70, 15, 16, 13, 66], 2.0), ([1, 0, 0, 2, 1], 1e-4 if dtype == "f16" else 1e-30)):
        s.append(counts, dtype, size)
        s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_append_token_by_token(dtype):
    s = Sequences(7, 2, 1, 2, 64)
    for i in range(40):
        s.append([1, 1], dtype, 2.0 ** (i % 13 - 6))
    s.check()


def test_append_twice_changes_nothing_more():
    s = Sequences(8, 3, 2, 2, 128)
    s.append([20, 7, 64], "bf16")
    args = s.append([9, 30, 2], "bf16", 5.0)
    for _ in range(2):
        lce.kv8_append(*args)
    s.check()


def test_append_ends_of_the_types_range():
    s = Sequences(9, 1, 2, 2, 64)
    x = torch.zeros(64, 2, 64, dtype=torch.float32)
    x[:16] = torch.tensor([3.4028234e38, -3.4028234e38] * 32)
    x[16:32] = 2.0 ** -149                         # below every scale
    x[32:48, :, 0] = 448.0                         # exactly the largest code
    x[32:48, :, 1] = 448.0 * 2.0 ** -15            # subnormal codes
    x[32:48, :, 2] = -(2.0 ** -10)                 # half the smallest: to even
    x[32:48, :, 3] = 2.0 ** -10 * 1.0001
    x[48:64] = 448.0000305                         # one bit past it
    s.append([64], "f32", k=x, v=x.flip(2).contiguous())
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_append_infinities_and_nans(dtype):
    s = Sequences(10, 2, 2, 2, 128)
    k, v = (values(s.rng, 60, 2, 128, dtype) for _ in range(2))
    k[3, 0, 7], k[20, 1, 127], v[21, 1, 5], v[50, 0, 0] = (float("inf"), float("nan"), float("-inf"),
                                                          float("nan"))
    s.append([33, 27], dtype, k=k, v=v)
    s.append([5, 5], dtype, 100.0)                 # a NaN key stays one when its block's scale grows
    s.check()
    got, _ = lce.kv8_read(s.handle, torch.tensor([int(s.table[0, 0]) * PAGE + 3]).cuda())
    assert torch.isnan(got[0, 0]).all() and torch.isfinite(got[0, 1]).all()


def test_append_drops_what_has_no_place():
    """Pages outside the cache, tokens before a sequence's beginning, empty calls."""
    s = Sequences(11, 3, 2, 2, 64)
    s.append([10, 10, 10], "bf16")
    s.table[1, 0], s.table[2, 0] = -1, s.cache.pages
    s.append([30, 30, 30], "bf16")
    s.check()
    before = s.handle.data.clone()
    k = values(s.rng, 50, 2, 64, "bf16")
    start = torch.tensor([0, 50, 50, 50], dtype=torch.int32).cuda()
    table = torch.from_numpy(s.table).cuda()
    lengths = torch.tensor([20, 0, 0], dtype=torch.int32).cuda()
    lce.kv8_append(s.handle, k.cuda(), k.cuda(), table, start, lengths)
    s.cache.append(s.table[0], 20, k.double().numpy(), k.double().numpy())
    s.check()
    assert not torch.equal(before, s.handle.data)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16).cuda()
    lce.kv8_append(s.handle, none, none, table, torch.zeros(4, dtype=torch.int32).cuda(), lengths)
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_takes_views(dtype):
    """Keys and values inside one projection's rows, and heads first."""
    s = Sequences(12, 2, 2, 2, 64)
    rows = values(s.rng, 37, 7, 64, dtype).cuda()
    heads_first = values(s.rng, 2, 37, 64, dtype).cuda()
    k, v = rows[:, 3:5], heads_first.transpose(0, 1)
    s.lengths = [20, 17]
    s.cache.append(s.table[0], 20, k[:20].cpu().double().numpy(), v[:20].cpu().double().numpy())
    s.cache.append(s.table[1], 17, k[20:].cpu().double().numpy(), v[20:].cpu().double().numpy())
    lce.kv8_append(s.handle, k, v, torch.from_numpy(s.table).cuda(),
                   torch.tensor([0, 20, 37], dtype=torch.int32).cuda(),
                   torch.tensor(s.lengths, dtype=torch.int32).cuda())
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_read_every_code(dim, dtype):
    rng = np.random.default_rng(dim)
    cache = ref.Cache(3, 2, dim, 0)
    cache.data[..., :128 * dim] = rng.integers(0, 256, (3, 2, 128 * dim))
    cache.data[..., 128 * dim:] = rng.integers(100, 150, (3, 2, 128))
    cache.data[2, :, 128 * dim:128 * dim + 8] = [1, 247, 127, 2, 247, 1, 3, 127]
    slots = np.concatenate((rng.permutation(192), [-1, 192, 2 ** 62, -2 ** 63, 5, 5]))
    handle = lce.KV8Cache(2, dim, data=torch.from_numpy(cache.data).cuda())
    k, v = lce.kv8_read(handle, torch.from_numpy(slots).cuda(), dtype=ref.DTYPES[dtype])
    for i, slot in enumerate(slots.tolist()):
        for got, want in zip((k, v), cache.read(slot) if 0 <= slot < 192 else [np.zeros((2, dim))] * 2):
            want = torch.from_numpy(want).float().to(ref.DTYPES[dtype])
            assert torch.equal(got[i].cpu().nan_to_num(7, 8, 9), want.nan_to_num(7, 8, 9)), (i, slot)
    out = (torch.empty_like(k), torch.empty_like(v))
    lce.kv8_read(handle, torch.from_numpy(slots).cuda(), out=out)
    assert torch.equal(out[0].nan_to_num(7), k.nan_to_num(7))


def test_read_long_goes_past_the_caches():
    rng = np.random.default_rng(1)
    data = torch.from_numpy(rng.integers(0, 127, (1100, 4, 128 * 64 + 128)).astype(np.uint8)).cuda()
    handle = lce.KV8Cache(4, 64, data=data)
    slots = torch.randperm(1100 * 64, generator=torch.Generator().manual_seed(0)).cuda()
    for dtype in (torch.float32, torch.bfloat16):
        k, v = lce.kv8_read(handle, slots, dtype=dtype)
        for i in (0, 1, 4097, 70399):
            a, b = lce.kv8_read(handle, slots[i:i + 1], dtype=dtype)
            assert torch.equal(k[i], a[0]) and torch.equal(v[i], b[0])


# ---- attention

def check(batch, lce_args=None, **kw):
    """The call against the oracle, within the bounds that the oracle derives."""
    opts = {k: v for k, v in kw.items() if k in ("causal", "window", "cap", "slopes", "prefix")}
    scale = batch.dim ** -0.5
    want, want_lse, bound, lse_bound = batch.attention(scale, weights=kw.get("weights"), **opts)
    cache, q, table, start, lengths = batch.device(lce)
    opts["softcap"] = opts.pop("cap", 0.0)
    for name, dtype in (("slopes", torch.float32), ("prefix", torch.int32)):
        if opts.get(name) is not None:
            opts[name] = torch.as_tensor(opts[name], dtype=dtype).cuda()
    out, lse = lce.kv8_attention(cache, q, table, start, lengths, return_lse=True, **opts,
                                 **(lce_args or {}))
    got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(got))
    with np.errstate(invalid="ignore"):
        off = np.where(nan, 0, np.abs(got - want) - bound)
        assert off.max() <= 0, (off.max(), np.argwhere(off > 0)[:5].tolist())
        seen = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse))
        assert (np.abs(got_lse - want_lse)[seen] <= lse_bound[seen]).all()
    return out, lse


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 130, 300]
ONE = [0, 1, 1, 1, 1, 1, 1, 1, 1, 1]
SOME = [0, 1, 5, 0, 17, 2, 64, 3, 7, 20]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(1, 1, 64), (8, 2, 64), (4, 4, 128), (10, 2, 128),
                                                  (16, 1, 128), (20, 1, 256), (3, 3, 256)])
@pytest.mark.parametrize("queries", [ONE, SOME])
def test_attention(q_heads, kv_heads, dim, dtype, queries):
    check(ref.Batch(dim + q_heads, LENGTHS, queries, q_heads, kv_heads, dim, dtype))


@pytest.mark.parametrize("dtype,weights", [("bf16", 2.0 ** -14), ("f16", 2.0 ** -20)])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 2, 64), (7, 1, 128), (16, 2, 256)])
@pytest.mark.parametrize("chunk", [0, 1])
def test_few_rows_have_weights_of_two_parts(q_heads, kv_heads, dim, dtype, weights, chunk):
    """Up to eight rows of a head: a weight's leading bits (bfloat16: cut off below 2^-7 of it,
    float16: 2^-10) and as many of what is left."""
    queries = [1 if n else 0 for n in LENGTHS]
    if q_heads // kv_heads <= 4:
        queries[5] = queries[-1] = 2
    batch = ref.Batch(dim + q_heads, LENGTHS, queries, q_heads, kv_heads, dim, dtype, loud=3.0)
    with lce.tuning(kv8_chunk=chunk):
        check(batch, weights=weights)
        check(batch, weights=weights, cap=20.0, window=100)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("opts", [
    dict(causal=False), dict(window=1), dict(window=40), dict(window=100, causal=False),
    dict(prefix=[0, 1, 3, 16, 2 ** 31 - 1, 30, -5, 64, 129, 290]),
    dict(prefix=[9] * 10, window=20)], ids=str)
def test_masks(dim, dtype, opts):
    check(ref.Batch(dim, LENGTHS, SOME, 4, 2, dim, dtype), **opts)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("opts", [
    dict(cap=1.0), dict(cap=30.0), dict(cap=1e6), dict(slopes=[0.5, 0.0, -0.01, 2.0]),
    dict(cap=5.0, slopes=[0.1, 1.0, 0.01, 0.3], window=70),
    dict(slopes=[0.1, 1.0, 0.01, 0.3], causal=False),
    dict(cap=5.0, slopes=[0.1, 1.0, 0.01, 0.3], prefix=[40] * 10)], ids=str)
def test_changed_scores(dim, dtype, opts):
    check(ref.Batch(dim, LENGTHS, SOME, 4, 2, dim, dtype, loud=4.0), **opts)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("chunk", [0, 1, 3])
def test_every_schedule(dim, dtype, rows, chunk):
    """Tiles of each height, whole and split, with masks that move through them."""
    batch = ref.Batch(dim + rows, [700, 130, 1, 64, 333], [40, 9, 1, 2, 33], 8, 2, dim, dtype)
    for opts in (dict(), dict(window=100), dict(cap=10.0, prefix=[600, 2, 0, 70, 310])):
        with lce.tuning(kv8_rows=rows, kv8_chunk=chunk):
            check(batch, **opts)
            name = lce.last_schedule()
        # (a window of 100 spans three pages, which one workgroup takes)
        split = chunk == 1 or chunk == 3 and "window" not in opts
        assert name.startswith("kv8-") and name.endswith("-split") == split


def launched(length, queries, heads, kv_heads, dim, rows=0, seqs=1, **kw):
    """The schedule of a call over an empty table (every page is outside the cache), and that
    its rows see nothing."""
    cache = lce.KV8Cache(kv_heads, dim, pages=1)
    table = torch.full((seqs, -(-length // 64)), -1, dtype=torch.int32, device="cuda")
    start = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * queries
    q = torch.randn(seqs * queries, heads, dim, device="cuda").bfloat16()
    with lce.tuning(kv8_rows=rows):
        out, lse = lce.kv8_attention(cache, q, table, start, torch.full_like(start[1:], length),
                                     return_lse=True, **kw)
    assert not out.any() and torch.isneginf(lse).all()
    return lce.last_schedule()


def test_the_rule_for_heights():
    for rows in (16, 32, 128):
        assert launched(70, 3, 4, 2, 64, rows=rows) == f"kv8-{rows}"
        assert launched(70, 3, 4, 2, 256, rows=rows) == "kv8-16"      # no other has a kernel
    # one token each, a few tokens, long sequences
    assert launched(100, 1, 8, 2, 128, seqs=3) == "kv8-16"
    assert launched(20000, 1, 8, 2, 128) == "kv8-16-split"
    assert launched(300, 5, 24, 4, 64, seqs=4).startswith("kv8-16")
    # 512 tiles of 128 rows, of 64 channels 2048
    assert launched(2048, 2048, 32, 8, 128) == "kv8-128"
    assert launched(2047, 2047, 32, 8, 128) == "kv8-32"
    assert launched(8192, 8192, 32, 8, 64) == "kv8-128"
    assert launched(2048, 2048, 32, 8, 64) == "kv8-32"
    # 1024 tiles of 32
    assert launched(1024, 1024, 32, 8, 128).startswith("kv8-32")
    assert launched(1023, 1023, 32, 8, 128).startswith("kv8-16")
    # rows that share pages: 128 of them, 256
    assert launched(1000, 32, 32, 8, 128, seqs=80).startswith("kv8-128")
    assert launched(1000, 31, 32, 8, 128, seqs=80).startswith("kv8-16")
    assert launched(1000, 64, 32, 8, 128, seqs=16).startswith("kv8-32")
    assert launched(1000, 63, 32, 8, 128, seqs=17).startswith("kv8-16")


def test_longest_hints_and_workspaces():
    batch = ref.Batch(3, [2000, 77, 640], [1, 1, 3], 8, 2, 128, "bf16")
    cache, q, table, start, lengths = batch.device(lce)
    ws = lce.kv8_workspace(cache, q, table)
    for hints in (dict(), dict(max_q=3, max_len=2000), dict(max_q=1, max_len=1),
                  dict(max_q=2 ** 31 - 1, max_len=2 ** 31 - 1)):
        for w in (None, ws):
            check(batch, dict(workspace=w, **hints))
    assert not ws[:lce.KV8_WORKSPACE_ZERO].any()


@pytest.mark.parametrize("rows,counts,window", [(0, [256, 256], 4600), (16, [300, 212], 4600),
                                                (32, [512, 512], 4550), (128, [2048, 2048], 4600)])
def test_states_stay_in_the_workspace(rows, counts, window):
    """A hint of one new token where there are many, and windows that end inside pages: there
    is room for as many splits of a tile as pages that windows usually span would make, and
    not for another."""
    gen = torch.Generator("cuda").manual_seed(5)
    cache = lce.KV8Cache(8, 64, pages=160)
    table = torch.arange(160, dtype=torch.int32, device="cuda").reshape(2, 80)
    lengths = torch.tensor([5000, 5100], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(10100, 8, 64, generator=gen, device="cuda", dtype=torch.bfloat16)
            for _ in range(2))
    begin = torch.tensor([0, 5000, 10100], dtype=torch.int32, device="cuda")
    lce.kv8_append(cache, k, v, table, begin, lengths)
    start = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device="cuda")
    q = torch.randn(sum(counts), 32, 64, generator=gen, device="cuda", dtype=torch.bfloat16)
    need = lce.kv8_workspace(cache, q, table).numel()
    behind = 4 << 20
    space = torch.full((need + behind,), 0x5A, dtype=torch.uint8, device="cuda")
    space[:lce.KV8_WORKSPACE_ZERO] = 0
    with lce.tuning(kv8_rows=rows):
        out = lce.kv8_attention(cache, q, table, start, lengths, window=window, max_q=1,
                                workspace=space[:need])
        with lce.tuning(kv8_chunk=80):
            whole = lce.kv8_attention(cache, q, table, start, lengths, window=window, max_q=1,
                                      workspace=space[:need])
    assert (space[need:] == 0x5A).all() and not space[:lce.KV8_WORKSPACE_ZERO].any()
    # each rounds the result and weights of values of at most `most` by half a step of bfloat16
    most = v.float().abs().max().item() * (1 + 2.0 ** -4)
    assert (out.float() - whole.float()).abs().max().item() <= 4 * 2.0 ** -8 * most


def test_rows_of_no_sequence_stay():
    batch = ref.Batch(4, [70, 20], [3, 2], 4, 2, 64, "bf16")
    cache, q, table, start, lengths = batch.device(lce)
    q = torch.cat((q, q, q))
    out = torch.full_like(q, 7.0)
    start = torch.tensor([2, 5, 7], dtype=torch.int32).cuda()
    _, lse = lce.kv8_attention(cache, q, table, start, lengths, out=out, return_lse=True)
    assert (out[:2] == 7).all() and (out[7:] == 7).all() and not (out[2:7] == 7).any()


def test_what_is_not_finite_stays_with_the_rows_that_see_it():
    odd = [(0, 50, 0, 3, "k", np.nan), (1, 5, 1, 0, "v", np.inf), (2, 129, 0, 9, "k", -np.inf)]
    for dim in (64, 128, 256):
        for dtype in ("bf16", "f16"):
            batch = ref.Batch(5, [70, 40, 130], [40, 40, 3], 4, 2, dim, dtype, odd=odd)
            for rows in (16, 32, 128):
                with lce.tuning(kv8_rows=rows):
                    out, _ = check(batch)
                    assert torch.isnan(out).any() and torch.isfinite(out).any()
                    check(batch, window=10)


def test_queries_that_are_not_finite():
    batch = ref.Batch(6, [70, 40], [3, 40], 4, 2, 128, "bf16")
    batch.q[1, 2, 5], batch.q[20, 0, 0] = float("nan"), float("inf")
    cache, q, table, start, lengths = batch.device(lce)
    for rows in (16, 32, 128):
        with lce.tuning(kv8_rows=rows):
            out = lce.kv8_attention(cache, q, table, start, lengths)
        bad = torch.isnan(out).any(-1)
        assert bad[1, 2] and bad[20, 0] and bad.sum() == 2


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,spread", [("bf16", 60.0), ("bf16", 12.0), ("f16", 12.0)])
def test_blocks_of_very_different_sizes(dim, dtype, spread):
    """Values from 2^-spread to 2^spread, keys over a fraction of that (float16: results
    that fit it)."""
    batch = ref.Batch(7, [500, 90], [20, 1], 4, 2, dim, dtype, spread=spread)
    for rows in (16, 32, 128):
        with lce.tuning(kv8_rows=rows):
            check(batch)
            check(batch, cap=20.0)
    with lce.tuning(kv8_chunk=1):
        check(batch)


def test_largest_values_stay_finite():
    """Means of values near the ends of float32's and bfloat16's range."""
    for dtype, top in (("bf16", 3.0e38), ("f16", 6.0e4)):
        s = Sequences(13, 1, 4, 1, 64)
        k = values(s.rng, 200, 1, 64, "f32", 0.1)
        v = torch.full((200, 1, 64), top)
        s.append([200], "f32", k=k, v=v)
        s.check()
        q = values(s.rng, 1, 2, 64, dtype).cuda()
        args = (torch.from_numpy(s.table).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda(),
                torch.tensor([200], dtype=torch.int32).cuda())
        held = float(ref.E4M3[s.cache.data[s.table[0, 0], 0, 64 * 64]]
                     * 2.0 ** (int(s.cache.data[s.table[0, 0], 0, 128 * 64 + 4]) - 127))
        for chunk in (0, 1):
            with lce.tuning(kv8_chunk=chunk):
                out = lce.kv8_attention(s.handle, q, *args).double()
            assert torch.isfinite(out).all()
            assert ((out / held - 1).abs() <= 4 * ref.HALF_ULP[dtype]).all()


@pytest.mark.parametrize("queries", [1, 9, 80])
@pytest.mark.parametrize("under", [30.1, 31.6, 27.3])
def test_float16_weights_far_under_the_largest(queries, under):
    """A token of weight 1 and value 0, and many of weight 2^-under and value 1: weights have a
    last place of 2^-31 of the largest, of which half is lost."""
    n, dim = 20000, 64
    cache = lce.KV8Cache(1, dim, pages=-(-n // 64))
    table = torch.arange(cache.pages, dtype=torch.int32, device="cuda")[None]
    k, v = torch.zeros(n, 1, dim).half(), torch.ones(n, 1, dim).half()
    k[0, 0, 0], v[0] = 16, 0
    length = torch.tensor([n], dtype=torch.int32).cuda()
    lce.kv8_append(cache, k.cuda(), v.cuda(), table, torch.tensor([0, n]).int().cuda(), length)
    q = torch.zeros(queries, 1, dim).half()
    q[:, 0, 0] = 16
    out = lce.kv8_attention(cache, q.cuda(), table, torch.tensor([0, queries]).int().cuda(), length,
                            scale=under * math.log(2) / 256, causal=False)
    want = (n - 1) * 2.0 ** -under / (1 + (n - 1) * 2.0 ** -under)
    # scores of 22 in float32 are off by 2^-20 or less, the result by half a step of 2^-24
    bound = n * 2.0 ** -32 + want * 2.0 ** -11 + 2.0 ** -25
    assert (out.double().cpu() - want).abs().max().item() <= bound


@pytest.mark.parametrize("rows", [16, 32, 128])
@pytest.mark.parametrize("opts", [dict(softcap=1e-6), dict(softcap=1e-6, slopes=True),
                                  dict(scale=1e30)], ids=str)
def test_scores_of_zero_beside_the_largest_keys(rows, opts):
    """A block whose scale times the call's, or over its cap, is past float32's range: its
    zero keys score 0."""
    n, dim = 40, 64
    v = torch.randn(n, 1, dim, generator=torch.Generator().manual_seed(1)).bfloat16()
    k = torch.zeros(n, 1, dim).bfloat16()
    k[3, 0, 5] = -1e36
    cache = lce.KV8Cache(1, dim, pages=1)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    start, length = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([0, n], [n]))
    lce.kv8_append(cache, k.cuda(), v.cuda(), table, start, length)
    seen = lce.kv8_read(cache, torch.arange(n).cuda(), dtype=torch.float32)[1][:, 0].double().cpu()
    q = torch.ones(n, 1, dim).bfloat16().cuda()
    if opts.get("slopes"):
        opts = dict(opts, slopes=torch.zeros(1, device="cuda"))
    with lce.tuning(kv8_rows=rows):
        out = lce.kv8_attention(cache, q, table, start, length, causal=False, **opts)[:, 0].cpu()
    # capped, all weights are alike to 2e-6; else the token of the score below all has none
    some = seen if "softcap" in opts else torch.cat((seen[:3], seen[4:]))
    mean, size = some.mean(0), some.abs().mean(0)
    # weights' and the result's rounding, each half a step of bfloat16, and float32 sums
    bound = 2.0 ** -8 * 1.01 * (size + mean.abs()) + 1e-5 * size
    assert ((out.double() - mean).abs() <= bound).all()


def test_pages_outside_the_cache_are_hidden():
    batch = ref.Batch(8, [300, 100], [2, 1], 4, 2, 64, "bf16")
    whole = batch.attention(64 ** -0.5)[0]
    cache, q, table, start, lengths = batch.device(lce)
    table[0, 1], table[1, 0] = -1, cache.pages
    out = lce.kv8_attention(cache, q, table, start, lengths).cpu().double().numpy()
    keep = np.arange(300) // PAGE != 1
    batch.k[0], batch.v[0] = batch.k[0][keep], batch.v[0][keep]
    batch.k[1], batch.v[1] = batch.k[1][64:], batch.v[1][64:]
    batch.lengths = [236, 36]
    want, _, bound, _ = batch.attention(64 ** -0.5)
    assert (np.abs(out - want) <= bound).all() and not np.allclose(whole, want, atol=1e-2)


def test_lengths_and_starts_out_of_range():
    """Taken as the nearest bound: nothing outside a buffer is touched."""
    batch = ref.Batch(9, [128, 60], [2, 1], 4, 2, 64, "bf16", width=2)
    cache, q, table, start, lengths = batch.device(lce)
    table[1, 1] = 0
    lengths[0], lengths[1] = 2 ** 31 - 1, -5
    start[0], start[2] = -7, 2 ** 31 - 1
    out, lse = lce.kv8_attention(cache, q, table, start, lengths, return_lse=True)
    want = batch.attention(64 ** -0.5)[0]
    assert np.abs(out[:2].cpu().double().numpy() - want[:2]).max() < 0.05
    assert not out[2].any() and torch.isneginf(lse[2]).all()


def test_same_bits_each_time_and_beside_other_rows():
    batch = ref.Batch(10, [900, 70, 300], [4, 1, 2], 8, 2, 128, "bf16")
    cache, q, table, start, lengths = batch.device(lce)
    with lce.tuning(kv8_chunk=2):
        out = lce.kv8_attention(cache, q, table, start, lengths)
        for _ in range(3):
            assert torch.equal(out, lce.kv8_attention(cache, q, table, start, lengths))


def test_strided_queries():
    batch = ref.Batch(11, [90, 33], [5, 1], 4, 2, 128, "f16")
    cache, q, table, start, lengths = batch.device(lce)
    want = lce.kv8_attention(cache, q, table, start, lengths)
    rows = torch.zeros(6, 9, 128, dtype=q.dtype, device="cuda")
    rows[:, 2:6] = q
    assert torch.equal(want, lce.kv8_attention(cache, rows[:, 2:6], table, start, lengths))
    first = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(want, lce.kv8_attention(cache, first, table, start, lengths))


def test_refusals_of_what_is_no_number_and_of_one_output_twice():
    batch = ref.Batch(3, [5], [1], 4, 2, 64, "bf16")
    args = batch.device(lce)
    for kw in (dict(softcap=None), dict(softcap="2"), dict(scale="1"), dict(window=None),
               dict(window=1.5), dict(max_q=1.5)):
        with pytest.raises(TypeError):
            lce.kv8_attention(*args, **kw)
    for kw in (dict(scale=1e300), dict(softcap=1e300), dict(window=-1), dict(max_len=2 ** 31)):
        with pytest.raises((ValueError, lce.LceError)):
            lce.kv8_attention(*args, **kw)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    one = torch.empty(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        lce.kv8_read(args[0], slots, out=(one, one))
    with pytest.raises(TypeError):
        lce.kv8_read(args[0], slots, out=(None, one))
    plan, positions = lce.Rotary(64), torch.zeros(3, dtype=torch.int64, device="cuda")
    for out in (one[:1].expand(3, 2, 64), one[:, :1].expand(3, 2, 64)):
        with pytest.raises(lce.LceError):
            lce.rotary(plan, positions, one, out=out)


def test_far_into_a_large_buffer():
    """A cache of more than 4 GiB: pages whose offsets pass 32 bits."""
    heads, dim = 8, 256
    pages = (5 << 30) // (heads * (128 * dim + 128))
    data = torch.zeros(pages, heads, 128 * dim + 128, dtype=torch.uint8, device="cuda")
    handle = lce.KV8Cache(heads, dim, data=data)
    small = lce.KV8Cache(heads, dim, pages=3)
    rng = np.random.default_rng(2)
    k, v = (values(rng, 130, heads, dim, "bf16").cuda() for _ in range(2))
    q = values(rng, 1, heads, dim, "bf16").cuda()
    start = torch.tensor([0, 130], dtype=torch.int32).cuda()
    one = torch.tensor([0, 1], dtype=torch.int32).cuda()
    lengths = torch.tensor([130], dtype=torch.int32).cuda()
    outs = []
    for cache, table in ((handle, [pages - 1, 0, pages // 2 + 1]), (small, [0, 1, 2])):
        table = torch.tensor([table], dtype=torch.int32).cuda()
        lce.kv8_append(cache, k, v, table, start, lengths)
        place = torch.arange(130).cuda()
        outs.append((lce.kv8_attention(cache, q, table, one, lengths),)
                    + lce.kv8_read(cache, table[0].long()[place // 64] * 64 + place % 64))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# ---- together

def test_a_decoding_step_in_a_graph():
    """Rotary positions, append and attention of one token a sequence, captured once and
    replayed as sequences grow; each replay against the same calls made eagerly."""
    rng = np.random.default_rng(12)
    seqs, q_heads, kv_heads, dim, steps = 3, 8, 2, 128, 20
    caches = [lce.KV8Cache(kv_heads, dim, pages=seqs * 2) for _ in range(2)]
    for c in caches:
        c.data.zero_()
    plan = lce.Rotary(dim)
    table = torch.randperm(seqs * 2, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    table = table.view(seqs, 2).cuda()
    lengths = torch.tensor([0, 50, 60], dtype=torch.int32).cuda()
    start = torch.arange(seqs + 1, dtype=torch.int32).cuda()
    past = values(rng, 110, kv_heads, dim, "bf16").cuda()
    for c in caches:
        lce.kv8_append(c, past, past, table, torch.tensor([0, 0, 50, 110], dtype=torch.int32).cuda(),
                       lengths)
    q, k, v = (values(rng, seqs, h, dim, "bf16").cuda() for h in (q_heads, kv_heads, kv_heads))
    at = torch.zeros(seqs, dtype=torch.int64).cuda()
    out = torch.empty_like(q)
    spaces = [lce.kv8_workspace(c, q, table) for c in caches]

    def step(cache, into, space):
        a, b = lce.rotary(plan, at, q, k)
        lce.kv8_append(cache, b, v, table, start, lengths)
        lce.kv8_attention(cache, a, table, start, lengths, out=into, workspace=space, max_q=1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lengths += 1
    with torch.cuda.stream(side):
        step(caches[0], out, spaces[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out, spaces[0])
    lengths -= 1
    other = torch.empty_like(out)
    for _ in range(steps):
        q.copy_(values(rng, seqs, q_heads, dim, "bf16"))
        k.copy_(values(rng, seqs, kv_heads, dim, "bf16", 3.0))
        v.copy_(values(rng, seqs, kv_heads, dim, "bf16"))
        at.copy_(lengths)
        lengths += 1
        graph.replay()
        step(caches[1], other, spaces[1])
        torch.cuda.synchronize()
        assert torch.equal(out, other)
        assert torch.isfinite(out).all()


def test_other_streams():
    batch = ref.Batch(14, [900, 70], [2, 1], 8, 2, 128, "bf16")
    cache, q, table, start, lengths = batch.device(lce)
    want = lce.kv8_attention(cache, q, table, start, lengths)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(lce.kv8_attention(cache, q, table, start, lengths))
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for o in outs)


def test_prompts_and_steps_against_float64():
    """Prompts and then single tokens, through rotary positions, the cache and attention:
    as far from attention over unquantized keys and values as 8 bits make it."""
    rng = np.random.default_rng(15)
    q_heads, kv_heads, dim, prompt, steps = 4, 2, 64, 90, 5
    plan = lce.Rotary(dim, scaling="linear", factor=2.0)
    cache = lce.KV8Cache(kv_heads, dim, pages=2)
    table = torch.tensor([[1, 0]], dtype=torch.int32).cuda()
    q, k, v = (rng.standard_normal((prompt + steps, h, dim)) for h in (q_heads, kv_heads, kv_heads))
    got = []
    for lo, hi in [(0, prompt)] + [(prompt + i, prompt + i + 1) for i in range(steps)]:
        at = torch.arange(lo, hi).cuda()
        a, b, c = (torch.from_numpy(x[lo:hi]).bfloat16().cuda() for x in (q, k, v))
        a, b = lce.rotary(plan, at, a, b)
        start = torch.tensor([0, hi - lo], dtype=torch.int32).cuda()
        length = torch.tensor([hi], dtype=torch.int32).cuda()
        lce.kv8_append(cache, b, c, table, start, length)
        got.append(lce.kv8_attention(cache, a, table, start, length))
    got = torch.cat(got).cpu().double().numpy()
    f = plan.freqs.numpy()
    at = np.arange(prompt + steps)
    q, k = ref.rotary(q, at, f, 1.0, False), ref.rotary(k, at, f, 1.0, False)
    for h in range(q_heads):
        s = q[:, h] @ k[:, h // 2].T * dim ** -0.5
        s = np.where(np.tri(len(s), dtype=bool), s, -np.inf)
        w = np.exp(s - s.max(-1, keepdims=True))
        want = w / w.sum(-1, keepdims=True) @ v[:, h // 2]
        # codes are within 2^-4 of a value: keys move a score by some 2^-4 / sqrt(3), values
        # by as much of themselves
        assert np.linalg.norm(got[:, h] - want) <= 0.1 * np.linalg.norm(want)


def test_calls_beside_another_current_device(monkeypatch):
    """Where another device is current, calls make theirs current and put it back."""
    batch = ref.Batch(16, [90], [2], 4, 2, 64, "bf16")
    cache, q, table, start, lengths = batch.device(lce)
    want = lce.kv8_attention(cache, q, table, start, lengths)
    entered = []
    real = torch.cuda.device

    class Device(real):
        def __enter__(self):
            entered.append(self.idx)
            return super().__enter__()

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", Device)
    got = lce.kv8_attention(cache, q, table, start, lengths)
    assert entered and set(entered) == {0} and torch.equal(got, want)
