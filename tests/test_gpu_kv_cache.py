"""The 4-bit key-value cache on the GPU: what is written and read back is the definition's, bit for bit, and attention over it is the 64-bit attention over the
values it stands for, at the sizes, masks and layouts where it can go wrong."""
import math

import pytest
import torch

import paper_2407_11062_amd as eq
import kv_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
GRID = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128), (256, 256)]


def rows(gen, T, H, D, dtype, key=False):
    x = torch.randn(T, H, D, generator=gen)
    if key:
        x = x * torch.randn(H, D, generator=gen).mul(0.5).exp() + torch.randn(H, D, generator=gen)
    return x.to(dtype)


class Setup:
    """A cache whose memory was full of NaN steps, and sequences on pages in no order: seqs = [(new, length)]."""

    def __init__(self, seqs, H, D, g, dtype, page=64, seed=1, key_edit=None, value_edit=None, slack=3):
        gen = torch.Generator().manual_seed(seed)
        self.seqs, self.H, self.D, self.g, self.dtype, self.page, self.gen = seqs, H, D, g, dtype, page, gen
        n_pages = [-(-L // page) for _, L in seqs]
        pool = sum(n_pages) + slack
        order = torch.randperm(pool, generator=gen)[:sum(n_pages)].tolist()
        width = max(n_pages + [1]) + 1
        self.table = torch.full((len(seqs), width), pool + 7, dtype=torch.int32)            # unused entries name no page
        for b, n in enumerate(n_pages):
            self.table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        self.cache = eq.KvCache(H, D, g, page, pool, dtype=dtype)
        self.cache.pool.fill_(0xFF)
        self.k = [rows(gen, L, H, D, dtype, key=True) for _, L in seqs]
        self.v = [rows(gen, L, H, D, dtype) for _, L in seqs]
        if key_edit:
            key_edit(self.k)
        if value_edit:
            value_edit(self.v)
        self.lens = [L for _, L in seqs]

    def batch(self, counts, lens=None, table=None, slack=0):
        starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
        lens = self.lens if lens is None else lens
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        return eq.KvBatch((self.table if table is None else table).cuda(), i32(lens), i32(starts), tokens=starts[-1], max_new=max(counts) + slack,
                          max_len=max(lens) + slack)

    def fill(self):
        k, v = torch.cat(self.k).cuda(), torch.cat(self.v).cuda()
        eq.eqat_kv_write(self.cache, self.batch(self.lens), k, v)
        return self

    def new(self, x):
        return torch.cat([t[len(t) - n:] for t, (n, _) in zip(x, self.seqs)])


def as_type(x64, dtype):
    """exact value -> binary32 (the kernel's one rounding: s c is exact there) -> the tensor's type"""
    return x64.float().to(dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=1e30), torch.nan_to_num(b.float(), nan=1e30)) and torch.equal(a.isnan(), b.isnan())


# ---- writing and reading back ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,g", GRID)
def test_what_was_written_is_read_back_as_the_definition_says(D, g, dtype):
    s = Setup([(5, 70), (0, 0), (33, 33), (1, 1), (0, 40), (64, 129)], 3, D, g, dtype, page=96, seed=D + g).fill()
    k, v = eq.eqat_kv_read(s.cache, s.batch(s.lens))
    assert same(k.cpu(), as_type(ref.held(torch.cat(s.k), g), dtype))
    assert same(v.cpu(), as_type(ref.held(torch.cat(s.v), g), dtype))
    # the newest tokens alone, one of the two
    only_v = eq.eqat_kv_read(s.cache, s.batch([n for n, _ in s.seqs]), want=("v",))
    assert only_v[0] is None and same(only_v[1].cpu(), as_type(ref.held(s.new(s.v), g), dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,g,H", [(128, 128, 8), (128, 32, 1), (64, 32, 5), (256, 256, 2)])
def test_tokens_written_one_by_one_are_those_written_at_once(D, g, H, dtype):
    s = Setup([(0, 37), (0, 64), (0, 5)], H, D, g, dtype, page=32, seed=7)
    at_once = s.batch(s.lens)
    eq.eqat_kv_write(s.cache, at_once, torch.cat(s.k).cuda(), torch.cat(s.v).cuda())
    k, v = eq.eqat_kv_read(s.cache, at_once)
    s.cache.pool.fill_(0xFF)
    for t in range(64):                                    # one token of every sequence that is this long, as decoding goes
        counts = [1 if t < L else 0 for L in s.lens]
        b = s.batch(counts, lens=[min(t + 1, L) for L in s.lens])
        eq.eqat_kv_write(s.cache, b, *(torch.cat([x[t:t + 1] if t < len(x) else x[:0] for x in xs]).cuda() for xs in (s.k, s.v)))
    k1, v1 = eq.eqat_kv_read(s.cache, at_once)
    assert same(k, k1) and same(v, v1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_codes_at_and_beside_ties(dtype):
    """groups whose steps are powers of two, elements on every tie between two codes and a few units in the last place beside it"""
    D = g = 128
    T = 64
    x = torch.empty(T, 1, D)
    for t in range(T):
        s, m = 2.0 ** ((t % 16) - 8), float(t - 32) * 2.0 ** ((t % 16) - 9)
        ties = torch.arange(15) + 0.5
        e = torch.cat([torch.tensor([0.0, 15.0]), ties, ties, ties, torch.arange(D - 47) % 16.0])
        x[t, 0] = m + s * e
        if dtype == torch.float32:
            near = x[t, 0].clone()
            near[17:32], near[32:47] = torch.nextafter(near[17:32], torch.tensor(math.inf)), torch.nextafter(near[32:47], torch.tensor(-math.inf))
            x[t, 0] = near
    def put(xs):
        xs[0].copy_(x.to(dtype))
    s = Setup([(T, T)], 1, D, g, dtype, key_edit=put, value_edit=put).fill()
    k, v = eq.eqat_kv_read(s.cache, s.batch(s.lens))
    want = as_type(ref.held(x.to(dtype), g), dtype)
    assert same(k.cpu(), want) and same(v.cpu(), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_groups_that_are_constant_tiny_huge_or_not_finite(dtype):
    D, g = 128, 32
    def edit(xs):
        x = xs[0]
        x[0] = 0.0
        x[1] = 3.25
        x[2] *= 1e-6
        x[3] *= 1e4
        x[4, 0, 5] = math.nan
        x[5, 1, 40] = math.inf
        x[6, 0, 70] = -math.inf
        x[7, 0, 100] = 1e6               # beyond binary16: the step is not finite
        x[8, 1, 3] = -7e4                # the least element is not
        x[9, 0, 3] = 7e4                 # the greatest is, though step and least element are binary16 numbers
        x[9, 1, 3], x[9, 1, 4] = 65280.0, -65280.0          # the largest of both types
        x[10, 0, 64:96] = -65504.0
    s = Setup([(11, 11)], 2, D, g, dtype, key_edit=edit, value_edit=edit).fill()
    k, v = eq.eqat_kv_read(s.cache, s.batch(s.lens))
    for got, xs in ((k, s.k), (v, s.v)):
        want = as_type(ref.held(xs[0], g), dtype)
        assert same(got.cpu(), want)
        assert want[4, 0, :32].isnan().all() and not want[4, 0, 32:].isnan().any() and want[8, 1, :32].isnan().all() and want[9, 0, :32].isnan().all() and want[9, 1].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_are_slices_and_outputs_with_strides(dtype):
    """keys and values as slices of the rows of a stacked projection; results into slices; heads in another order (a negative head stride is none torch makes)"""
    H, R, D, g, T = 4, 3, 128, 64, 77
    s = Setup([(T, T)], H, D, g, dtype)
    qkv = torch.randn(T, (R + 2) * H * D).to(dtype).cuda()
    k, v = (qkv[:, (R + i) * H * D:(R + 1 + i) * H * D].view(T, H, D) for i in range(2))
    b = s.batch([T])
    eq.eqat_kv_write(s.cache, b, k, v)
    wide = torch.full((T, 3, H, D), 7.0, dtype=dtype, device="cuda")
    by_head = torch.full((H, T, D), 7.0, dtype=dtype, device="cuda")
    eq.eqat_kv_read(s.cache, b, k=wide[:, 1], v=by_head.transpose(0, 1))
    assert same(wide[:, 1].cpu(), as_type(ref.held(k.cpu(), g), dtype)) and same(by_head.transpose(0, 1).cpu(), as_type(ref.held(v.cpu(), g), dtype))
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 2] == 7).all())
    by_head_k = k.transpose(0, 1).contiguous().transpose(0, 1)
    s.cache.pool.fill_(0xFF)
    eq.eqat_kv_write(s.cache, b, by_head_k, v)
    assert same(eq.eqat_kv_read(s.cache, b)[0].cpu(), as_type(ref.held(k.cpu(), g), dtype))
    # attention: queries as the slice of the same rows, results by head
    q = qkv[:, :R * H * D].view(T, R * H, D)
    plain = eq.eqat_kv_attention(s.cache, b, q.contiguous())
    out = torch.empty((R * H, T, D), dtype=dtype, device="cuda").transpose(0, 1)
    eq.eqat_kv_attention(s.cache, b, q, out=out)
    assert torch.equal(plain, out)


def test_a_write_touches_its_own_tokens_only():
    """every byte of the pool that does not hold a written token stays"""
    H, D, g, dtype = 2, 128, 64, torch.bfloat16
    s = Setup([(0, 90), (0, 64)], H, D, g, dtype, page=32).fill()
    all_of = s.batch(s.lens)
    k0, v0 = eq.eqat_kv_read(s.cache, all_of)
    before = s.cache.pool.clone()
    b = s.batch([3, 0])                                     # tokens 87 .. 89 of the first sequence again, as they were
    eq.eqat_kv_write(s.cache, b, s.k[0][87:].cuda(), s.v[0][87:].cuda())
    assert torch.equal(before, s.cache.pool)
    eq.eqat_kv_write(s.cache, b, s.k[0][:3].cuda(), s.v[0][:3].cuda())
    k1, v1 = eq.eqat_kv_read(s.cache, all_of)
    changed = torch.zeros(len(k0), dtype=torch.bool)
    changed[87:90] = True
    for x0, x1 in ((k0, k1), (v0, v1)):
        assert torch.equal(x0[~changed], x1[~changed]) and not torch.equal(x0[changed], x1[changed])
    page = int(s.table[0, 87 // 32])
    rest = torch.ones(len(before), dtype=torch.bool)
    size = len(before) // s.cache.desc.pages
    rest[page * size:(page + 1) * size] = False
    assert torch.equal(before.cpu()[rest], s.cache.pool.cpu()[rest])


# ---- attention -----------------------------------------------------------------------------------------------------------------
def check(s, ratio, causal=True, window=0, scale=None, gone=None, table=None, lens=None, q_edit=None, slack=0, want_lse=True):
    counts = [n for n, _ in s.seqs]
    q = rows(s.gen, sum(counts), s.H * ratio, s.D, s.dtype)
    if q_edit:
        q_edit(q)
    b = s.batch(counts, table=table, lens=lens, slack=slack)
    lse = torch.empty((sum(counts), s.H * ratio), dtype=torch.float32, device="cuda") if want_lse else None
    ws = eq.kv_workspace(s.cache, b, s.H * ratio)
    qd = q.cuda()
    out = eq.eqat_kv_attention(s.cache, b, qd, scale=scale or 0.0, causal=causal, window=window, lse=lse, ws=ws)
    again = eq.eqat_kv_attention(s.cache, b, qd, scale=scale or 0.0, causal=causal, window=window, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(out, nan=1e30), torch.nan_to_num(again, nan=1e30))
    at = 0
    for i, (n, L) in enumerate(s.seqs):
        if n:
            o, l, to, tl = ref.attention(q[at:at + n], s.k[i], s.v[i], s.g, scale, causal, window, gone[i] if gone else None)
            got = out[at:at + n].cpu()
            assert torch.equal(got.isnan(), o.isnan()), f"sequence {i}: NaN in other places"
            fine = ~o.isnan()
            rounding = (2.0 ** -8 if s.dtype == torch.bfloat16 else 2.0 ** -23) * o.abs()
            over = ((got.double() - o).abs() - to - rounding)[fine]
            assert over.numel() == 0 or over.max() <= 0, f"sequence {i}: {over.max()} beyond the bound"
            if want_lse:
                gl = lse[at:at + n].cpu().double()
                assert torch.equal(gl.isnan(), l.isnan()) and torch.equal(gl == -math.inf, l == -math.inf)
                fine = l.isfinite()
                over = ((gl - l).abs() - tl)[fine]
                assert over.numel() == 0 or over.max() <= 0, f"sequence {i}: lse {over.max()} beyond the bound"
        at += n
    return q, out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,g", GRID)
def test_attention_of_a_token_each(D, g, dtype):
    check(Setup([(1, 1), (1, 31), (1, 32), (1, 33), (0, 50), (1, 300), (0, 0), (1, 257)], 2, D, g, dtype, page=32, seed=D * g).fill(), 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,ratio", [(1, 1), (8, 1), (1, 7), (3, 5), (2, 16), (1, 17), (1, 71), (40, 1)])
def test_head_layouts(H, ratio, dtype):
    check(Setup([(1, 77), (3, 140), (2, 2)], H, 128, 64, dtype, seed=H * ratio).fill(), ratio)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,g", [(64, 64), (128, 32), (128, 128), (256, 128)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 33), (False, 40), (True, 500)])
def test_masks_over_several_tokens(D, g, causal, window, dtype):
    check(Setup([(5, 100), (64, 64), (17, 201), (1, 96), (40, 41)], 2, D, g, dtype, page=96, seed=window + D).fill(), 2, causal=causal, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H,L", [(1, 1, 5000), (1, 8, 2777), (3, 2, 4097), (70, 1, 200), (200, 1, 40)])
def test_long_sequences_are_cut_and_joined(B, H, L, dtype):
    """one long sequence over many workgroups; more sequences than lanes; lengths that differ much"""
    seqs = [(1, max(1, L - 13 * i)) for i in range(B)]
    check(Setup(seqs, H, 128, 128, dtype, page=64, seed=L).fill(), 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("D,g,H", [(128, 64, 8), (256, 128, 24), (64, 32, 1)])
def test_more_short_units_than_workgroups(D, g, H, window, dtype):
    """several units of a workgroup one after the other, some of them cut, beside sequences that are long or have no new token"""
    lens = [3, 31, 32, 33, 90, 64, 5, 200, 3, 40] * (3 if H > 1 else 30) + [1500, 700]
    s = Setup([((3, 2, 0)[i % 3], L) for i, L in enumerate(lens)], H, D, g, dtype, page=32).fill()
    check(s, 16, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,D,g", [(8, 64, 32), (40, 64, 64), (24, 128, 128), (300, 64, 64)])
def test_shares_of_many_records(H, D, g, dtype):
    """workgroups of two a compute unit, and of heads that do not divide them"""
    s = Setup([(1, L) for L in [2000 if H < 100 else 300] * 2 + [3 + 7 * i % 50 for i in range(90 if H < 40 else 20)]], H, D, g, dtype, page=32).fill()
    check(s, 1)
    assert D != 64 or len(s.seqs) * H * (max(s.lens) // 32) >= 64 * 512


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,g,T,ratio", [(128, 128, 333, 1), (128, 32, 130, 4), (64, 64, 257, 2), (256, 64, 96, 2), (128, 64, 700, 1)])
def test_prompts(D, g, T, ratio, dtype):
    check(Setup([(T, T), (T // 2, T // 2 + 45), (1, 80), (0, 20)], 2, D, g, dtype, seed=T).fill(), ratio)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("seqs,H,ratio", [([(70, 2600)], 2, 4), ([(33, 2100), (3, 2500), (0, 9)], 1, 8), ([(100, 900), (90, 700)], 1, 3)])
def test_prompts_behind_long_pasts(seqs, H, ratio, dtype):
    """units cut over workgroups and joined, by the kernel that streams (from 2048 positions on) and by the one that rebuilds"""
    check(Setup(seqs, H, 128, 64, dtype, page=64, seed=sum(map(sum, seqs))).fill(), ratio)


def close_to_fp32(s, q, b, window, nan=False):
    """A prompt in bf16 against the same values in fp32, whose kernel rebuilds nothing and is held to 64 bits above: the bounds of the rounding to binary16 and bf16."""
    out = eq.eqat_kv_attention(s.cache, b, q, window=window)
    twin = eq.KvCache(s.H, s.D, s.g, s.page, s.cache.desc.pages, dtype=torch.float32)
    eq.eqat_kv_write(twin, s.batch(s.lens), torch.cat(s.k).float().cuda(), torch.cat(s.v).float().cuda())
    exact = eq.eqat_kv_attention(twin, b, q.float(), window=window)
    assert torch.equal(out.isnan(), exact.isnan())
    held = ref.held(torch.cat(s.k), s.g).cuda().float().nan_to_num().abs().transpose(0, 1)                    # [H, L, D]
    R = q.shape[1] // s.H
    most = torch.stack([(q[:, h].float().abs() @ held[h // R].T.contiguous()).amax(-1) for h in range(q.shape[1])], 1) / math.sqrt(s.D)
    vs, vm, vc = ref.steps(torch.cat(s.v), s.g)
    span = (vm.abs().unsqueeze(-1) + vs.unsqueeze(-1) * vc).nan_to_num().max().item()
    bound = span * (2.0 ** -11 + 2 * (2.0 ** -11 * most[..., None] + 2.0 ** -18)) + 2.0 ** -8 * exact.abs()       # a key and a query: 2^-12 each
    assert ((out.float() - exact).abs().nan_to_num() <= bound.nan_to_num(nan=1.0)).all()
    return out


@pytest.mark.parametrize("D,g", GRID)
@pytest.mark.parametrize("window", [0, 200])
def test_large_prompts(D, g, window):
    """workgroups of 256 rows (heads of 256: 128): a sequence whose last rows leave most of one empty, one shorter than a tile, one behind a past"""
    seqs = [(1061, 1061), (40, 40), (300, 777)]
    s = Setup(seqs, 8, D, g, torch.bfloat16, page=96, seed=D + g).fill()
    q = rows(s.gen, sum(n for n, _ in seqs), 64, D, torch.bfloat16).cuda()
    close_to_fp32(s, q, s.batch([n for n, _ in seqs]), window)


def test_large_prompts_with_values_and_keys_that_are_not_finite():
    def bad(xs):
        xs[0][1030:, :, 3] = math.nan
        xs[0][500, 2] = math.inf
        xs[1][39, 0, 100] = math.nan
    seqs = [(1061, 1061), (40, 40)]
    for kw in (dict(value_edit=bad), dict(key_edit=bad)):
        s = Setup(seqs, 8, 128, 64, torch.bfloat16, seed=3, **kw).fill()
        q = rows(s.gen, 1101, 64, 128, torch.bfloat16).cuda()
        for window in (0, 300):
            out = close_to_fp32(s, q, s.batch([1061, 40]), window)
            assert not out[:500].isnan().any() and out.isnan().any()


def test_large_and_small_queries_in_prompts():
    """rows whose scores would leave binary16, or lie below it, with the scale in them"""
    s = Setup([(200, 200)], 2, 128, 64, torch.bfloat16).fill()
    def sizes(q):
        q[::3] *= 1e-5
        q[1::7] *= 1e6
        q[5] = 0
    check(s, 2, q_edit=sizes)


def test_a_workspace_serves_smaller_batches():
    s = Setup([(3000, 3000), (200, 2100)], 2, 128, 64, torch.bfloat16).fill()
    heads = 8
    ws = eq.kv_workspace(s.cache, s.batch([3000, 200]), heads)
    for counts, lens in (([3000, 200], [3000, 2100]), ([100, 30], [600, 2100]), ([1, 1], [3000, 2100]), ([17, 0], [40, 0]), ([300, 0], [700, 0])):
        b = s.batch(counts, lens=lens)
        q = rows(s.gen, sum(counts), heads, 128, torch.bfloat16).cuda()
        assert len(eq.kv_workspace(s.cache, b, heads)) <= len(ws)
        assert torch.equal(eq.eqat_kv_attention(s.cache, b, q, ws=ws), eq.eqat_kv_attention(s.cache, b, q))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 6, 150])
def test_what_a_query_does_not_see_does_not_reach_it(n, dtype):
    """NaN and infinities in later keys and values, and in those that a window leaves out"""
    def bad(xs):
        x = xs[0]
        x[3, 0, 5] = math.nan
        x[len(x) - n // 2 - 1:, :, 77] = math.inf
        x[len(x) - 1:, 0] = -math.inf
    s = Setup([(n, 220)], 2, 128, 32, dtype, key_edit=bad, value_edit=bad).fill()
    check(s, 4, window=100)
    check(s, 4)
    s = Setup([(n, 220)], 2, 128, 32, dtype, value_edit=bad).fill()
    check(s, 2, window=100)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_see_nothing_are_zeros(dtype):
    """all pages of a sequence outside the pool; some of them; none of the pages of the other sequences is touched by it"""
    s = Setup([(2, 130), (3, 200), (70, 100)], 2, 128, 64, dtype, page=32).fill()
    table = s.table.clone()
    table[0, :] = -1
    table[1, 2] = 1 << 30
    table[2, :] = 2 ** 31 - 1
    gone = [torch.ones(130, dtype=torch.bool), (torch.arange(200) // 32) == 2, torch.ones(100, dtype=torch.bool)]
    q, out = check(s, 2, table=table, gone=gone)
    assert bool((out[:2] == 0).all()) and bool((out[5:] == 0).all())
    # reading: zeros; writing: nothing
    k, v = eq.eqat_kv_read(s.cache, s.batch(s.lens, table=table))
    assert bool((k[:130] == 0).all()) and bool((v[130 + 64:130 + 96] == 0).all()) and not bool((v[130:194] == 0).all())
    before = s.cache.pool.clone()
    eq.eqat_kv_write(s.cache, s.batch([2, 0, 70], table=table), torch.zeros(72, 2, 128, dtype=dtype, device="cuda"), torch.zeros(72, 2, 128, dtype=dtype, device="cuda"))
    assert torch.equal(before, s.cache.pool)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scales_and_queries_of_all_sizes(dtype):
    s = Setup([(4, 300)], 2, 128, 64, dtype).fill()
    check(s, 2, scale=0.001)
    check(s, 2, scale=2.5)
    def sizes(q):
        q[0] *= 1e-20
        q[1] *= 30
        q[2] = 0
        q[3, 1] = math.nan
    check(s, 2, q_edit=sizes)
    def wide(vs):
        vs[0][:200] *= 1e-3
        vs[0][200:] *= 3e3
    check(Setup([(4, 300)], 2, 128, 64, dtype, value_edit=wide).fill(), 2)
    def narrow(vs):
        vs[0][:] *= 1e-3
    check(Setup([(4, 300), (200, 200)], 2, 128, 128, dtype, value_edit=lambda vs: [v.mul_(1e-3) for v in vs]).fill(), 2)


@pytest.mark.parametrize("D,g", GRID)
@pytest.mark.parametrize("window", [1, 8, 100, 0])
def test_fp32_results_are_as_near_as_binary32_arithmetic(D, g, window):
    """In the 2-norm of a row: a probability is off by 2^-24 of its exponent (below 2^5 here) and a few roundings, a product by 2^-24, and a sum of up to 400 adds
    to that the square root of their number at the most: 2^-19 holds for every row, where one low part that is missing or belongs to another high part shows as 2^-13."""
    s = Setup([(40, 400)], 2, D, g, torch.float32, seed=3).fill()
    q = rows(s.gen, 40, 4, D, torch.float32)
    out = eq.eqat_kv_attention(s.cache, s.batch([40]), q.cuda(), window=window).cpu().double()
    o = ref.attention(q, s.k[0], s.v[0], g, window=window)[0]
    assert ((out - o).norm(dim=-1) <= 2.0 ** -19 * o.norm(dim=-1)).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_bounds_larger_than_the_batch(dtype):
    """a captured graph's bounds: more new tokens and longer sequences than there are"""
    check(Setup([(1, 100), (2, 300)], 2, 128, 128, dtype).fill(), 2, slack=57)


def test_a_pool_beyond_32_bits():
    """pages whose offsets pass 2^32 bytes"""
    H, D, g, page = 8, 128, 128, 256
    per_page = eq.KvCache(H, D, g, page, 1).pool.numel()
    pages = (5 << 30) // per_page
    cache = eq.KvCache(H, D, g, page, pages)
    table = torch.tensor([[pages - 1, 3, (1 << 32) // per_page + 1]], dtype=torch.int32, device="cuda")
    L = 3 * page - 5
    b = eq.KvBatch(table, torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, L], dtype=torch.int32, device="cuda"), tokens=L, max_new=L, max_len=L)
    gen = torch.Generator().manual_seed(5)
    k, v = rows(gen, L, H, D, torch.bfloat16, key=True), rows(gen, L, H, D, torch.bfloat16)
    eq.eqat_kv_write(cache, b, k.cuda(), v.cuda())
    kr, vr = eq.eqat_kv_read(cache, b)
    assert same(kr.cpu(), as_type(ref.held(k, g), torch.bfloat16)) and same(vr.cpu(), as_type(ref.held(v, g), torch.bfloat16))
    b1 = eq.KvBatch(table, b.keep[1], torch.tensor([0, 1], dtype=torch.int32, device="cuda"), tokens=1, max_new=1, max_len=L)
    q = rows(gen, 1, H, D, torch.bfloat16)
    out = eq.eqat_kv_attention(cache, b1, q.cuda())
    o, _, to, _ = ref.attention(q, k, v, g)
    assert bool(((out.cpu().double() - o).abs() <= to + 2.0 ** -8 * o.abs()).all())


def test_graph_replays_with_other_lengths_and_pages():
    """write and attend captured once; lengths, pages and tensors change between the replays, with eager work in between"""
    H, R, D, g, page, B = 2, 4, 128, 64, 32, 3
    s = Setup([(0, 150), (0, 150), (0, 150)], H, D, g, torch.bfloat16, page=page)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, lens, starts = s.table.cuda(), i32([1, 1, 1]), i32([0, 1, 2, 3])
    b = eq.KvBatch(table, lens, starts, tokens=B, max_new=1, max_len=160)
    k, v = (torch.zeros(B, H, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    q, out = torch.zeros(B, H * R, D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H * R, D, dtype=torch.bfloat16, device="cuda")
    ws = eq.kv_workspace(s.cache, b, H * R)
    def step():
        eq.eqat_kv_write(s.cache, b, k, v)
        eq.eqat_kv_attention(s.cache, b, q, out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for it, L in enumerate([37, 150, 1, 97]):
        now = [L, max(1, L // 2), max(1, L - 1)]
        filled = s.batch(now, lens=now)
        eq.eqat_kv_write(s.cache, filled, *(torch.cat([x[:n] for x, n in zip(xs, now)]).cuda() for xs in (s.k, s.v)))
        lens.copy_(i32(now))
        k.copy_(torch.stack([x[n - 1] for x, n in zip(s.k, now)]))
        v.copy_(torch.stack([x[n - 1] for x, n in zip(s.v, now)]))
        q.copy_(rows(s.gen, B, H * R, D, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager = eq.eqat_kv_attention(s.cache, b, q)
        assert torch.equal(got, eager), it
        for i, n in enumerate(now):
            o, _, to, _ = ref.attention(q[i:i + 1].cpu(), s.k[i][:n], s.v[i][:n], g)
            assert bool(((got[i:i + 1].cpu().double() - o).abs() <= to + 2.0 ** -8 * o.abs()).all())


def test_calls_on_another_stream():
    s = Setup([(1, 500)], 2, 128, 64, torch.bfloat16).fill()
    q = rows(s.gen, 1, 8, 128, torch.bfloat16).cuda()
    b = s.batch([1])
    here = eq.eqat_kv_attention(s.cache, b, q)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        there = eq.eqat_kv_attention(s.cache, b, q)
    other.synchronize()
    assert torch.equal(here, there)


@pytest.mark.parametrize("dtype", DTYPES)
def test_nothing_outside_the_tensors_is_written(dtype):
    """pool, results and workspace between bands of a pattern"""
    GUARD = 4096
    def banded(n):
        raw = torch.full((2 * GUARD + (n + 255) // 256 * 256,), 0xC3, dtype=torch.uint8, device="cuda")
        return raw, raw[GUARD:GUARD + n]
    H, R, D, g = 2, 3, 128, 32
    s = Setup([(1, 700), (3, 77), (150, 150)], H, D, g, dtype, page=32)
    raws = []
    raw, pool = banded(s.cache.pool.numel())
    raws.append((raw, len(pool)))
    s.cache = eq.KvCache(H, D, g, 32, s.cache.desc.pages, dtype=dtype, pool=pool)
    s.fill()
    counts = [n for n, _ in s.seqs]
    b = s.batch(counts)
    need = len(eq.kv_workspace(s.cache, b, H * R))
    raw, ws = banded(need)
    ws.zero_()
    raws.append((raw, need))
    es = torch.empty(0, dtype=dtype).element_size()
    T = sum(counts)
    outs = []
    for heads, es_ in ((H * R, es), (H, es), (H, es)):
        raw, o = banded(T * heads * D * es_)
        raws.append((raw, len(o)))
        outs.append(o.view(dtype).view(T, heads, D))
    raw, l = banded(T * H * R * 4)
    raws.append((raw, len(l)))
    eq.eqat_kv_attention(s.cache, b, rows(s.gen, T, H * R, D, dtype).cuda(), out=outs[0], lse=l.view(torch.float32).view(T, H * R), ws=ws)
    eq.eqat_kv_read(s.cache, b, k=outs[1], v=outs[2])
    torch.cuda.synchronize()
    for raw, n in raws:
        assert bool((raw[:GUARD] == 0xC3).all()) and bool((raw[GUARD + n:] == 0xC3).all())
