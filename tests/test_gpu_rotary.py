"""Rotary positions against complex turns in 64 bits, and the turned write into the 4-bit cache against its two halves."""
import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref

pytestmark = pytest.mark.gpu


def heads(seed, T, H, D, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty((T, H, D), device="cuda").normal_(generator=gen).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def freq(part, stretch=1.0):
    return eq.rotary_frequencies(part, stretch=stretch).cuda()


# head size, elements turned: whole heads, half, a quarter; halves that 8, 4, 2 and no more divide
SIZES = [(128, 128), (64, 64), (256, 256), (80, 80), (80, 20), (96, 24), (128, 6), (8, 8), (8, 2), (72, 72), (1024, 1024), (512, 128)]


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("D, part", SIZES)
def test_turns(D, part, interleaved, dtype):
    for T, H, Hk in ((1, 1, 1), (5, 7, 1), (33, 4, 2)):
        q, k, f = heads(1, T, H, D, dtype), heads(2, T, Hk, D, dtype), freq(part, 8.0)
        pos = i32([(37 * t * t) % 5000 for t in range(T)])
        rot = eq.Rotary(f, D, interleaved, amplitude=1.25)
        for inverse in (False, True):
            qo, ko = eq.eqat_rotary(rot, pos, q, k, inverse=inverse)
            for got, x in ((qo, q), (ko, k)):
                ref.within(got, *ref.turned(x, pos, f, interleaved, 1.25, inverse))
        only, none = eq.eqat_rotary(rot, pos, q)
        assert none is None and torch.equal(only, eq.eqat_rotary(rot, pos, q, k)[0])


def test_far_positions():
    pos = i32([0, 1, 4095, 100003, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -1, -(1 << 31)])
    f = freq(128)
    q = heads(1, len(pos), 2, 128, torch.float32)
    got, _ = eq.eqat_rotary(eq.Rotary(f, 128), pos, q)
    # beyond 2^24 the angle itself, 2^-53 of up to 2^31 turned by 1 each, is good to 2^-22: within the bound's 8 roundings of 2^-24 with 2^-22 more
    y, bound = ref.turned(q, pos, f)
    ref.within(got, y, bound + 4 * ref.F32 * 2.0 * q.double().abs().amax())


@pytest.mark.parametrize("T", (1, 3, 1000, 2111))
def test_many_heads_and_tokens(T):
    q, k, f = heads(1, T, 72, 128, torch.bfloat16), heads(2, T, 9, 128, torch.bfloat16), freq(128)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 70000
    qo, ko = eq.eqat_rotary(eq.Rotary(f, 128), pos, q, k)
    ref.within(qo, *ref.turned(q, pos, f))
    ref.within(ko, *ref.turned(k, pos, f))


@pytest.mark.parametrize("interleaved, part", [(False, 128), (True, 128), (False, 20), (True, 20)])
def test_slices_in_place_and_what_lies_between(interleaved, part):
    T, H, Hk, D = 19, 6, 2, 128
    f, pos = freq(part), i32(list(range(3, 22)))
    qkv = heads(1, T, H + 2 * Hk, D, torch.bfloat16)
    kept = qkv.clone()
    rot = eq.Rotary(f, D, interleaved)
    q, k = qkv[:, :H], qkv[:, H:H + Hk]
    eq.eqat_rotary(rot, pos, q, k, q_out=q, k_out=k)
    ref.within(q, *ref.turned(kept[:, :H], pos, f, interleaved))
    ref.within(k, *ref.turned(kept[:, H:H + Hk], pos, f, interleaved))
    assert torch.equal(qkv[:, H + Hk:], kept[:, H + Hk:])
    # heads outermost, and into a wider buffer
    t = heads(2, H, T, D, torch.bfloat16).transpose(0, 1)
    wide = torch.full((T, H, D + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eqat_rotary(rot, pos, t, q_out=wide[..., :D])
    ref.within(wide[..., :D], *ref.turned(t, pos, f, interleaved))
    assert (wide[..., D:] == 7).all()


def test_the_inverse_is_the_gradient():
    """<turned(x), g> = <x, inverse(g)> up to the roundings of both, and the inverse undoes a turn of amplitude 1"""
    T, H, D = 11, 3, 64
    f, pos = freq(48), i32(list(range(T)))
    rot = eq.Rotary(f, D, amplitude=1.5)
    x, g = heads(1, T, H, D, torch.float32), heads(2, T, H, D, torch.float32)
    y, _ = eq.eqat_rotary(rot, pos, x)
    b, _ = eq.eqat_rotary(rot, pos, g, inverse=True)
    terms = 1.5 * (x.double().abs() * g.double().abs()).sum() * 2
    assert abs(float((y.double() * g.double()).sum() - (x.double() * b.double()).sum())) <= float(terms) * 20 * ref.F32
    rot = eq.Rotary(f, D)
    back, _ = eq.eqat_rotary(rot, pos, eq.eqat_rotary(rot, pos, x)[0], inverse=True)
    assert float((back - x).abs().max()) <= 40 * ref.F32 * float(x.abs().max())


def test_no_tokens():
    q = heads(1, 0, 4, 64, torch.bfloat16)
    assert eq.eqat_rotary(eq.Rotary(freq(64), 64), i32([]), q)[0].shape == (0, 4, 64)


def pages(lens, page, extra=1):
    n = [-(-x // page) for x in lens]
    order = torch.randperm(sum(n) + extra, generator=torch.Generator().manual_seed(3))
    table, at = torch.zeros((len(lens), max(n)), dtype=torch.int32), 0
    for b, m in enumerate(n):
        table[b, :m] = order[at:at + m]
        at += m
    return table.cuda(), sum(n) + extra


def two_calls(cache, batch, rot, pos, q, k, v):
    qo, ko = eq.eqat_rotary(rot, pos, q, k)
    eq.eqat_kv_write(cache, batch, ko, v)
    return qo


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("D, group, part, interleaved", [
    (128, 128, 128, False), (128, 64, 128, True), (128, 32, 64, False), (128, 128, 32, False), (128, 64, 20, False), (128, 64, 20, True), (64, 64, 64, False), (64, 32, 10, False), (64, 32, 64, True),
    (256, 256, 256, False), (256, 64, 192, False), (256, 32, 128, False), (256, 128, 64, False), (256, 128, 250, True)])
def test_turned_write_is_the_two_calls(D, group, part, interleaved, dtype):
    H, R = 3, 5
    new, lens = [1, 40, 0, 33, 5], [1, 100, 77, 33, 69]
    T, starts = sum(new), [sum(new[:i]) for i in range(len(new) + 1)]
    table, n = pages(lens, 32)
    batch = eq.KvBatch(table, i32(lens), i32(starts), tokens=T, max_new=max(new), max_len=max(lens))
    qkv = heads(1, T, H * R + 2 * H, D, dtype)
    q, k, v = qkv[:, :H * R], qkv[:, H * R:H * R + H], qkv[:, H * R + H:]
    rot = eq.Rotary(freq(part), D, interleaved, amplitude=1.125)
    caches = [eq.KvCache(H, D, group, 32, n, dtype=dtype) for _ in range(2)]
    for c in caches:
        c.pool.fill_(85)
    pos = torch.cat([torch.arange(l - m, l) for m, l in zip(new, lens)]).int().cuda()
    want = two_calls(caches[0], batch, rot, pos, q, k, v)
    kept = qkv.clone()
    got = eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v)
    assert torch.equal(got, want) and torch.equal(caches[0].pool, caches[1].pool) and torch.equal(qkv, kept)
    eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v, q_out=q)          # in place
    assert torch.equal(q, want) and torch.equal(caches[0].pool, caches[1].pool) and torch.equal(qkv[:, H * R:], kept[:, H * R:])


def test_turned_write_beyond_the_bounds():
    """rows behind the last sequence and beyond max_new stay; tokens past max_len and on missing pages are turned, and not written"""
    H, D, page = 2, 64, 32
    lens, starts = [70, 40, 10], [0, 6, 8, 11]
    table, n = pages(lens, page)
    table[1, 1] = -1                      # positions 32 .. of the second sequence are on no page
    batch = eq.KvBatch(table, i32(lens), i32(starts), tokens=14, max_new=4, max_len=67)
    q, k, v = (heads(i, 14, H, D, torch.bfloat16) for i in range(3))
    rot = eq.Rotary(freq(D), D)
    caches = [eq.KvCache(H, D, 64, page, n) for _ in range(2)]
    for c in caches:
        c.pool.fill_(85)
    pos = i32([64, 65, 66, 67, 68, 69, 38, 39, 7, 8, 9, 0, 0, 0])
    full = two_calls(caches[0], batch, rot, pos, q, k, v)
    out = torch.full_like(q, 7.0)
    eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v, q_out=out)
    taken = [0, 1, 2, 3, 6, 7, 8, 9, 10]
    left = [i for i in range(14) if i not in taken]
    assert torch.equal(out[taken], full[taken]) and (out[left] == 7).all() and torch.equal(caches[0].pool, caches[1].pool)
    # nothing new at all
    none = eq.KvBatch(table, i32(lens), i32([0, 0, 0, 0]), tokens=14, max_new=0, max_len=67)
    out.fill_(7.0)
    eq.eqat_kv_rotary_write(caches[1], none, rot, q, k, v, q_out=out)
    assert (out == 7).all() and torch.equal(caches[0].pool, caches[1].pool)


def test_more_new_tokens_than_held():
    H, D = 2, 64
    table, n = pages([8], 32)
    batch = eq.KvBatch(table, i32([3]), i32([0, 8]), tokens=8, max_new=8, max_len=32)
    q, k, v = (heads(i, 8, H, D, torch.bfloat16) for i in range(3))
    rot = eq.Rotary(freq(D), D)
    caches = [eq.KvCache(H, D, 32, 32, n) for _ in range(2)]
    for c in caches:
        c.pool.fill_(85)
    want = two_calls(caches[0], batch, rot, i32(list(range(-5, 3))), q, k, v)
    got = eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v)
    assert torch.equal(got, want) and torch.equal(caches[0].pool, caches[1].pool)


def test_more_sequences_than_lanes_and_heads_than_a_workgroup_takes():
    B, H, R, D = 150, 5, 13, 128
    lens = [1 + (7 * b) % 90 for b in range(B)]
    table, n = pages(lens, 32)
    batch = eq.KvBatch(table, i32(lens), i32(list(range(B + 1))), tokens=B, max_new=1, max_len=96)
    q, k, v = heads(1, B, H * R, D, torch.bfloat16), heads(2, B, H, D, torch.bfloat16), heads(3, B, H, D, torch.bfloat16)
    rot = eq.Rotary(freq(D, 4.0), D)
    caches = [eq.KvCache(H, D, 64, 32, n) for _ in range(2)]
    for c in caches:
        c.pool.fill_(85)
    want = two_calls(caches[0], batch, rot, i32([x - 1 for x in lens]), q, k, v)
    assert torch.equal(eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v), want) and torch.equal(caches[0].pool, caches[1].pool)


def test_replayed_with_other_lengths():
    H, R, D, B = 2, 4, 128, 3
    table, n = pages([96] * B, 32)
    lens = i32([5, 31, 64])
    batch = eq.KvBatch(table, lens, i32(list(range(B + 1))), tokens=B, max_new=1, max_len=96)
    q, k, v = heads(1, B, H * R, D, torch.bfloat16), heads(2, B, H, D, torch.bfloat16), heads(3, B, H, D, torch.bfloat16)
    rot, out = eq.Rotary(freq(D), D), torch.empty_like(q)
    caches = [eq.KvCache(H, D, 64, 32, n) for _ in range(2)]
    for c in caches:
        c.pool.fill_(85)
    eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v, q_out=out)
    two_calls(caches[0], batch, rot, lens - 1, q, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(1)
        eq.eqat_kv_rotary_write(caches[1], batch, rot, q, k, v, q_out=out)
    for i in range(4):
        q.copy_(heads(10 + i, B, H * R, D, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = two_calls(caches[0], batch, rot, lens - 1, q, k, v)
        assert torch.equal(out, want) and torch.equal(caches[0].pool, caches[1].pool)


def test_offsets_beyond_32_bits():
    T, H, D = 270_000, 64, 128                       # 4.4 GB, in place
    q = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")
    tail = heads(1, 2, H, D, torch.bfloat16)
    q[-2:] = tail
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rot = eq.Rotary(freq(D), D)
    eq.eqat_rotary(rot, pos, q, q_out=q)
    assert torch.equal(q[-2:], eq.eqat_rotary(rot, pos[-2:].clone(), tail)[0]) and not q[:-2].any()


def test_more_workgroups_than_a_launch_holds():
    """68 tokens to a workgroup, and 2^24 workgroups of 256 threads are 2^32 threads: 37 GB, in place"""
    T, D, part = 1_150_000_000, 16, 2
    q = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 1, 570_425_343, 570_425_344, 1_140_850_687, 1_140_850_688, T - 1], device="cuda")
    rows = heads(3, some.numel(), 1, D, torch.bfloat16)
    q[some], pos[some] = rows, torch.arange(1, 8, dtype=torch.int32, device="cuda")
    rot = eq.Rotary(freq(part), D)
    want = eq.eqat_rotary(rot, pos[some], rows)[0]
    eq.eqat_rotary(rot, pos, q, q_out=q)
    assert torch.equal(q[some], want)
    assert int(torch.stack([c.ne(0).sum() for c in q.view(torch.int16).view(-1).chunk(16)]).sum()) == int(want.ne(0).sum())
