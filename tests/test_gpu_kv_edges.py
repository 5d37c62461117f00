"""The 4-bit cache where bounds are passed, rows fall short of what the host was told, softmaxes are steep and numbers extreme: against the 64-bit reference."""
import math

import pytest
import torch

import paper_2407_11062_amd as eq
import kv_reference as ref
from test_gpu_kv_cache import DTYPES, Setup, as_type, check, rows, same

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def batch(s, counts, lens=None, max_len=None, max_new=None, table=None):
    starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
    lens = s.lens if lens is None else lens
    return eq.KvBatch((s.table if table is None else table).contiguous().cuda(), i32(lens), i32(starts), tokens=starts[-1],
                      max_new=max(counts) if max_new is None else max_new, max_len=max(lens) if max_len is None else max_len)


def held_to(got, lse, want, dtype, what, rows_of=slice(None)):
    """results of one sequence's rows against (out, lse, bounds) of the reference"""
    o, l, to, tl = (x[rows_of] for x in want)
    got, lse = got.cpu(), lse.cpu().double()
    assert torch.equal(got.isnan(), o.isnan()) and torch.equal(lse == -math.inf, l == -math.inf), what
    over = (got.double() - o).abs() - to - (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * o.abs()
    assert over.nan_to_num().max() <= 0, f"{what}: {over.nan_to_num().max()} beyond the bound"
    fine = l.isfinite()
    over = ((lse - l).abs() - tl)[fine]
    assert over.numel() == 0 or over.nan_to_num().max() <= 0, f"{what}: lse {over.max()} beyond the bound"


# ---- bounds that are passed --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("by_table", [False, True])
@pytest.mark.parametrize("reach", [64, 96])
def test_tokens_beyond_a_bound_are_not_written_and_read_as_zeros(reach, by_table, dtype):
    """ten tokens at 90 .. 99 where the call was told of `reach` positions, by the host's number or by the table's width; a whole sequence beside it"""
    s = Setup([(10, 100), (4, 50)], 2, 128, 64, dtype, page=32).fill()
    everything = s.batch(s.lens)
    k0, v0 = eq.eqat_kv_read(s.cache, everything)
    b = batch(s, [10, 4], max_len=100 if by_table else reach, table=s.table[:, :reach // 32] if by_table else None)
    k, v = (rows(s.gen, 14, 2, 128, dtype) for _ in "kv")
    eq.eqat_kv_write(s.cache, b, k.cuda(), v.cuda())
    k1, v1 = eq.eqat_kv_read(s.cache, everything)
    inside = max(0, reach - 90)
    for before, now, new in ((k0, k1, k), (v0, v1, v)):
        want = before.clone().cpu()
        want[90:90 + inside] = as_type(ref.held(new[:inside], 64), dtype)
        want[146:] = as_type(ref.held(new[10:], 64), dtype)
        assert same(now.cpu(), want)
    for got, new in zip(eq.eqat_kv_read(s.cache, b, k=torch.full_like(k, 7.0).cuda(), v=torch.full_like(v, 7.0).cuda()), (k, v)):
        want = as_type(ref.held(new, 64), dtype)
        want[inside:10] = 0
        assert same(got.cpu(), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,ratio", [(3, 2), (90, 2), (300, 8)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 40), (False, 25)])
def test_queries_beyond_a_bound_stand_where_they_stand(n, ratio, causal, window, dtype):
    """attention of the newest tokens of 400 where the call was told of 350 positions: those from 350 on are not there, the queries at their own positions"""
    s = Setup([(n, 400), (2, 30)], 2, 128, 64, dtype, page=32, seed=n + window).fill()
    b = batch(s, [n, 2], max_len=350)
    q = rows(s.gen, n + 2, 2 * ratio, 128, dtype)
    lse = torch.empty((n + 2, 2 * ratio), dtype=torch.float32, device="cuda")
    out = eq.eqat_kv_attention(s.cache, b, q.cuda(), causal=causal, window=window, lse=lse)
    some = slice(0, n, max(1, n // 40))
    want = ref.attention(q[:n], s.k[0], s.v[0], 64, causal=causal, window=window, gone=torch.arange(400) >= 350)
    held_to(out[:n][some], lse[:n][some], want, dtype, "beyond", some)
    held_to(out[n:], lse[n:], ref.attention(q[n:], s.k[1], s.v[1], 64, causal=causal, window=window), dtype, "beside")
    if window == 25 and not causal:
        assert bool((out[n - 1] == 0).all())                       # the last query sees from 375 on: nothing that is there


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,most,ratio", [(9, 5, 2), (150, 100, 2)])
def test_more_new_tokens_than_the_bound(n, most, ratio, dtype):
    """the first `most` of a sequence's new tokens, at their own positions; the rows of the others stay as they are"""
    s = Setup([(n, 200), (2, 30)], 2, 128, 64, dtype, page=32).fill()
    everything = s.batch(s.lens)
    before = eq.eqat_kv_read(s.cache, everything)
    b = batch(s, [n, 2], max_new=most)
    new = [rows(s.gen, n + 2, 2, 128, dtype) for _ in "kv"]
    eq.eqat_kv_write(s.cache, b, *(x.cuda() for x in new))
    first = 200 - n
    for was, now, x, xs in zip(before, eq.eqat_kv_read(s.cache, everything), new, (s.k, s.v)):
        want = was.clone().cpu()
        want[first:first + most] = as_type(ref.held(x[:most], 64), dtype)
        want[228:] = as_type(ref.held(x[n:], 64), dtype)
        assert same(now.cpu(), want)
        xs[0][first:first + most], xs[1][28:] = x[:most], x[n:]
    for got, x in zip(eq.eqat_kv_read(s.cache, b, *(torch.full((n + 2, 2, 128), 7.0, dtype=dtype, device="cuda") for _ in "kv")), new):
        want = as_type(ref.held(x, 64), dtype)
        want[most:n] = 7.0
        assert same(got.cpu(), want)
    q = rows(s.gen, n + 2, 2 * ratio, 128, dtype)
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    eq.eqat_kv_attention(s.cache, b, q.cuda(), out=out, lse=lse)
    held_to(out[:most], lse[:most], ref.attention(q[:n], s.k[0], s.v[0], 64), dtype, "first", slice(0, most))
    held_to(out[n:], lse[n:], ref.attention(q[n:], s.k[1], s.v[1], 64), dtype, "beside")
    assert bool((out[most:n] == 7).all()) and bool((lse[most:n] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,window", [(7, 0), (7, 2), (7, 2 ** 31 - 1), (90, 0), (90, 2 ** 31 - 1)])
def test_more_new_tokens_than_are_held(n, window, dtype):
    """five tokens held, `n` of them new: the first rows stand before the beginning, are not written, read as zeros, see nothing"""
    s = Setup([(5, 5), (0, 0), (2, 40)], 2, 128, 64, dtype, page=32).fill()
    before = s.cache.pool.clone()
    b = batch(s, [n, 3, 2])
    new = [torch.cat([rows(s.gen, n - 5, 2, 128, dtype), x[0], rows(s.gen, 3, 2, 128, dtype), x[2][38:]]) for x in (s.k, s.v)]
    eq.eqat_kv_write(s.cache, b, *(x.cuda() for x in new))
    assert torch.equal(before, s.cache.pool)
    for got, x in zip(eq.eqat_kv_read(s.cache, b, *(torch.full((n + 5, 2, 128), 7.0, dtype=dtype, device="cuda") for _ in "kv")), new):
        want = as_type(ref.held(x, 64), dtype)
        want[:n - 5], want[n:n + 3] = 0, 0
        assert same(got.cpu(), want)
    q = rows(s.gen, n + 5, 4, 128, dtype)
    lse = torch.empty((n + 5, 4), dtype=torch.float32, device="cuda")
    out = eq.eqat_kv_attention(s.cache, b, q.cuda(), window=window, lse=lse)
    assert bool((out[:n - 5] == 0).all()) and bool((out[n:n + 3] == 0).all()) and bool((lse[:n - 5] == -math.inf).all()) and bool((lse[n:n + 3] == -math.inf).all())
    many = 2 * n > 64                                             # (the reference's bounds of a sequence of many rows)
    padded = torch.cat([rows(s.gen, 40, 4, 128, dtype), q[n - 5:n]]) if many else q[n - 5:n]
    held_to(out[n - 5:n], lse[n - 5:n], ref.attention(padded, s.k[0], s.v[0], 64, window=window), dtype, "held", slice(-5, None))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [2, 80])
def test_lengths_of_any_size(n, dtype):
    """a length at the end of 32 bits, one that is negative: nothing is written or read beyond the table, queries see what a window leaves of what is there"""
    s = Setup([(0, 96), (0, 64), (1, 33)], 2, 128, 64, dtype, page=32).fill()
    before = s.cache.pool.clone()
    b = batch(s, [n, n, 1], lens=[2 ** 31 - 1, -7, 33], max_len=96, table=s.table[:, :3])
    k, v = (torch.cat([rows(s.gen, 2 * n, 2, 128, dtype), x[2][32:]]).cuda() for x in (s.k, s.v))
    eq.eqat_kv_write(s.cache, b, k, v)
    assert torch.equal(before, s.cache.pool)
    kr, _ = eq.eqat_kv_read(s.cache, b)
    assert bool((kr[:2 * n] == 0).all()) and same(kr[2 * n:].cpu(), as_type(ref.held(s.k[2][32:], 64), dtype))
    q = rows(s.gen, 2 * n + 1, 2, 128, dtype)
    for causal, window in ((True, 0), (True, 500), (False, 500), (True, 2 ** 31 - 1)):
        lse = torch.empty((2 * n + 1, 2), dtype=torch.float32, device="cuda")
        out = eq.eqat_kv_attention(s.cache, b, q.cuda(), causal=causal, window=window, lse=lse)
        assert bool((out[n:2 * n] == 0).all())
        if window == 500:
            assert bool((out[:n] == 0).all())
        elif window == 0:
            held_to(out[:n], lse[:n], ref.attention(q[:n], s.k[0], s.v[0], 64, causal=False), dtype, "all")


def test_a_captured_step_replayed_past_the_end():
    """the replays whose token no longer fits leave the cache as it is"""
    s = Setup([(0, 62), (0, 20)], 2, 128, 64, torch.bfloat16, page=32).fill()
    table, lens = s.table[:, :2].contiguous().cuda(), i32([62, 20])
    b = eq.KvBatch(table, lens, i32([0, 1, 2]), tokens=2, max_new=1, max_len=64)
    k, v = (torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    def step():
        lens.add_(1)
        eq.eqat_kv_write(s.cache, b, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    lens.copy_(i32([62, 20]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    tokens = [[], []]
    for t in range(5):
        new = [rows(s.gen, 2, 2, 128, torch.bfloat16) for _ in "kv"]
        k.copy_(new[0]); v.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        tokens[0].append(new[0]); tokens[1].append(new[1])
    assert lens.tolist() == [67, 25]
    now = eq.eqat_kv_read(s.cache, eq.KvBatch(table, i32([64, 25]), i32([0, 64, 89]), tokens=89, max_new=64, max_len=64))
    for got, xs, new in zip(now, (s.k, s.v), tokens):
        want = torch.cat([xs[0]] + [x[:1] for x in new[:2]] + [xs[1]] + [x[1:] for x in new])
        assert same(got.cpu(), as_type(ref.held(want, 64), torch.bfloat16))


# ---- rows that change between replays ----------------------------------------------------------------------------------------
def test_replays_in_which_a_sequence_falls_short():
    """captured with four sequences of 128 new tokens; replayed with starts that leave one of them a single token, or none"""
    H, R, D, g = 2, 2, 128, 64
    s = Setup([(128, 300)] * 4, H, D, g, torch.bfloat16, page=32).fill()
    lens, starts = i32([300] * 4), i32([0, 128, 256, 384, 512])
    b = eq.KvBatch(s.table.cuda(), lens, starts, tokens=512, max_new=128, max_len=300)
    q, out = torch.zeros(512, H * R, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(512, H * R, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(512, H * R, device="cuda")
    ws = eq.kv_workspace(s.cache, b, H * R)
    def step():
        eq.eqat_kv_attention(s.cache, b, q, out=out, lse=lse, ws=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for counts in ([128, 128, 128, 1], [128, 20, 0, 128], [1, 1, 1, 1], [128, 128, 128, 128]):
        starts.copy_(i32([sum(counts[:i]) for i in range(5)]))
        qh = rows(s.gen, 512, H * R, D, torch.bfloat16)
        q.copy_(qh)
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        at = 0
        for i, n in enumerate(counts):
            if n:
                some = slice(at, at + n, max(1, n // 10))
                padded = torch.cat([rows(s.gen, 40, H * R, D, torch.bfloat16), qh[at:at + n]])                # (the bounds of a sequence of many rows: one kernel takes all of this call)
                held_to(out[some], lse[some], ref.attention(padded, s.k[i], s.v[i], g), torch.bfloat16, f"{counts} {i}", slice(40, 40 + n, max(1, n // 10)))
            at += n
        assert bool((out[at:] == 7).all()) and bool((lse[at:] == 7).all())


# ---- steep softmaxes, small values, extreme queries and scales ---------------------------------------------------------------
def steep(seqs, gap, dtype, H=2, D=128, g=64, every=32):
    """Every `every` positions a key that stands 2^gap above the others, its value zero: results are made of small probabilities alone."""
    direction = torch.randn(D, generator=torch.Generator().manual_seed(int(gap)))
    up = gap * math.log(2.0) * math.sqrt(D) / direction.square().sum() * direction
    def keys(xs):
        for x in xs:
            x.mul_(0.05)
            x[::every] = up.to(dtype)
    def values(xs):
        for x in xs:
            x[::every] = 0
    def queries(q):
        q[:] = direction.to(dtype)
    return Setup(seqs, H, D, g, dtype, key_edit=keys, value_edit=values).fill(), queries


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gap", [12, 20, 26])
@pytest.mark.parametrize("D,g", [(64, 32), (128, 64), (256, 256)])
def test_steep_softmaxes_of_few_rows(D, g, gap, dtype):
    """(in fp32 too: what lies 2^26 below the greatest is held to the same share of itself)"""
    s, queries = steep([(1, 33), (3, 300), (1, 1700)], gap, dtype, D=D, g=g)
    check(s, 4, q_edit=queries)


@pytest.mark.parametrize("gap", [12, 20, 26])
@pytest.mark.parametrize("D,g,H,n,past,ratio", [(64, 32, 2, 150, 0, 2), (128, 64, 2, 150, 0, 2), (256, 128, 2, 150, 0, 2), (128, 128, 8, 1100, 0, 8), (128, 64, 1, 80, 1420, 2)])
def test_steep_softmaxes_of_prompts(D, g, H, n, past, ratio, gap):
    """workgroups of few and of many rows, teams, units that are cut"""
    s, queries = steep([(n, past + n)], gap, torch.bfloat16, H=H, D=D, g=g, every=64)
    q = torch.empty(n, H * ratio, D, dtype=torch.bfloat16)
    queries(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    out = eq.eqat_kv_attention(s.cache, s.batch([n]), q.cuda(), lse=lse)
    some = slice(1, n, n // 12)
    for head in (0, H * ratio - 1):
        one = slice(head // ratio, head // ratio + 1)
        want = ref.attention(q[:, head:head + 1], s.k[0][:, one], s.v[0][:, one], g)
        held_to(out[some, head:head + 1], lse[some, head:head + 1], want, torch.bfloat16, "steep", some)


@pytest.mark.parametrize("size", [1e-6, 1e-5, 1e-4])
def test_small_values(size):
    """a few steps of the cache's smallest: what they stand for is summed as well as larger values are"""
    def small(xs):
        for x in xs:
            x.mul_(size)
    check(Setup([(1, 33), (3, 300), (1, 1700)], 2, 128, 64, torch.bfloat16, value_edit=small).fill(), 4)
    def mixed(xs):
        for x in xs:
            x[:len(x) // 2].mul_(size)
            x[len(x) // 2:].mul_(3e3)
    check(Setup([(1, 33), (3, 300), (1, 1700)], 2, 128, 64, torch.bfloat16, value_edit=mixed).fill(), 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [4, 90])
@pytest.mark.parametrize("scale", [1e8, 1e10, 2.0 ** 100])
def test_large_scales(scale, n, dtype):
    """scores that are far apart: one key a row, whatever the roundings"""
    s = Setup([(n, 300)], 2, 128, 64, dtype).fill()
    def sizes(q):
        q[1::2] *= 1e-3
        q[0] *= 2.0 ** -100
        q[2] = 0
    check(s, 2, scale=scale, q_edit=sizes)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [4, 90])
@pytest.mark.parametrize("size", [2.0 ** 112, 2.0 ** 117, 2.0 ** 121, 2.0 ** -110, 2.0 ** -124])
def test_queries_of_extreme_sizes(size, n, dtype):
    s = Setup([(n, 300)], 2, 128, 64, dtype).fill()
    def sizes(q):
        q[1::2] *= size
        q[2] = 0
    check(s, 2, q_edit=sizes)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [4, 90])
@pytest.mark.parametrize("scale", [1e-12, 1e-24, 1e-38])
def test_small_scales(scale, n, dtype):
    """all that a row sees counts alike, what it does not see stays hidden"""
    s = Setup([(n, 300)], 2, 128, 64, dtype).fill()
    def sizes(q):
        q[1::2] *= 1e-3
        q[0] *= 2.0 ** -100
        q[2] = 0
    check(s, 2, scale=scale, q_edit=sizes)


# ---- one workspace for several caches ----------------------------------------------------------------------------------------
def test_a_workspace_serves_caches_of_other_shapes():
    """layers whose heads differ in size and number share a workspace, zeroed once, large enough for each of them"""
    def setup(seqs, H, D, g, ratio, dtype=torch.bfloat16):
        s = Setup(seqs, H, D, g, dtype).fill()
        b = s.batch([n for n, _ in s.seqs])
        q = rows(s.gen, b.tokens, H * ratio, D, dtype).cuda()
        return s, b, q, H * ratio
    shapes = [setup([(1, 3000 + i) for i in range(5)], 8, 128, 128, 4), setup([(1, 4300 - 70 * i) for i in range(32)], 8, 64, 64, 1), setup([(1, 5000), (100, 700)], 300, 64, 64, 1),
              setup([(90, 900), (2, 40)], 2, 128, 32, 2), setup([(2, 3000)], 3, 256, 64, 4, torch.float32)]
    alone = [eq.eqat_kv_attention(s.cache, b, q) for s, b, q, _ in shapes]
    ws = torch.zeros(max(len(eq.kv_workspace(s.cache, b, heads)) for s, b, _, heads in shapes), dtype=torch.uint8, device="cuda")
    for turn in range(2):
        for (s, b, q, _), want in zip(shapes, alone):
            out = torch.full_like(q, 7.0)
            eq.eqat_kv_attention(s.cache, b, q, out=out, ws=ws)
            assert torch.equal(out, want), (turn, s.H, s.D)


@pytest.mark.parametrize("n,L,B", [(70, 100, 80), (33, 700, 130), (200, 200, 66)])
def test_prompts_of_more_sequences_than_lanes(n, L, B):
    """some of them without new tokens, some with few"""
    seqs = [((n, 2, 0)[i % 3], max(n, L - 3 * i)) for i in range(B)]
    check(Setup(seqs, 2, 128, 64, torch.bfloat16, page=32).fill(), 2)
