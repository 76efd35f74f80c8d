"""New rows into caches, slots back out of them and compaction of e4m3 caches, against the definitions in 64 bits."""
import math

import pytest
import torch

from chunk_util import PAGE, Cache, as_bytes, gen, i32, quantise64, two_to

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def sv():
    import paper_2509_11815_amd as sv
    sv.load_library()
    return sv


def rows(g, B, N, heads, D, dtype, fused):
    """New K and V rows, on their own or as parts of a fused projection's output."""
    if not fused:
        return [torch.empty((B, N, heads, D), dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2)]
    x = torch.empty((B, N, 3 + 2 * heads, D), dtype=dtype, device="cuda").normal_(generator=g)
    return [x[:, :, 3:3 + heads], x[:, :, 3 + heads:]]


def held(cache):
    return [as_bytes(t).clone() for t in (cache.k, cache.v, *(cache.scales or ()))]


def expect_append(cache, prefix, new, k_new, v_new):
    """The caches' memory as it has to be afterwards."""
    want = held(cache)
    for b, (P, n) in enumerate(zip(prefix, new)):
        for i, (r, t) in enumerate(cache.places(b, range(P, P + n))):
            for which, x in enumerate((k_new, v_new)):
                if cache.ks is None:
                    want[which][r, :, t] = x[b, i].to(want[which].dtype)
                else:
                    code, e = quantise64(x[b, i])
                    want[which][r, :, t] = code.float().to(E4M3).view(torch.uint8)
                    want[2 + which][r, :, t] = (e + 127).to(torch.uint8)
    return want


def same(got, want, nan_codes=False):
    for g, w in zip(got, want):
        if g.dtype.is_floating_point:
            g, w = (t.view({2: torch.int16, 4: torch.int32}[t.element_size()]) for t in (g, w))
        elif nan_codes:
            g, w = (torch.where(t & 0x7F == 0x7F, torch.full_like(t, 0x7F), t) for t in (g, w))
        assert torch.equal(g, w)


CASES = [([0], [1]), ([5, 40, 0, 31], [1, 1, 1, 1]), ([0], [100]), ([3, 0, 77, 16], [33, 0, 16, 50]), ([15, 1], [2, 64])]


@pytest.mark.parametrize("prefix,new", CASES)
@pytest.mark.parametrize("heads,D", [(1, 64), (3, 128), (5, 64), (8, 128)])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("dtype,kind", [(BF16, E4M3), (F32, E4M3), (BF16, BF16), (F32, F32)])
def test_append(sv, prefix, new, heads, D, paged, dtype, kind):
    g = gen(len(prefix) + heads)
    cache = Cache(g, [p + n for p, n in zip(prefix, new)], heads, D, kind, paged)
    k, v = rows(g, len(prefix), max(new) + 2, heads, D, dtype, fused=heads != 3)
    for b, n in enumerate(new):
        k[b, n:] = math.nan                      # rows past the count are never to matter
        v[b, n:] = math.nan
    want = expect_append(cache, prefix, new, k, v)
    err = i32([0])
    sv.specvlm_kv_append(k, v, cache.k, cache.v, i32(prefix), num_new=i32(new), block_table=cache.table, scales=cache.scales, err_flag=err)
    assert int(err) == 0
    same(held(cache), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_quantisation_edges(sv, dtype, D):
    """Zeros, the greatest and least numbers, exact borders of the exponent rule, ties of the rounding, infinities and NaN."""
    g = gen(2)
    x = torch.empty((1, 64, 1, D), dtype=F32, device="cuda").normal_(generator=g)
    x[0, 0] = 0.0
    x[0, 1] *= 2.0 ** -130
    x[0, 2] *= 2.0 ** 120
    x[0, 3] = 3.3895e38
    x[0, 4, 0, ::2] = -3.0e38
    for i, top in enumerate((448.0, 449.0, 447.0, 448.0 * 2 ** -9, 464.0, 512.0, 224.0)):
        x[0, 5 + i].clamp_(-1, 1)
        x[0, 5 + i, 0, 7] = top
    x[0, 12] = torch.arange(D, device="cuda") * 0.25 + 16.0 + 1.0          # halves of a step of codes 16 .. 32
    x[0, 12, 0, 0] = 448.0
    x[0, 13, 0, 3] = math.inf
    x[0, 14, 0, 5] = -math.inf
    x[0, 15, 0, 9] = math.nan
    x[0, 16] = math.nan
    x[0, 17] = math.inf
    x[0, 18] = 2.0 ** -149
    x[0, 19] = torch.where(torch.arange(D, device="cuda") == 1, 1.0, 2.0 ** -20)       # below half of the least code: zeros
    x[0, 20] = -0.0
    x = x.to(dtype)
    cache = Cache(g, [64], 1, D, E4M3, False)
    sv.specvlm_kv_append(x, x, cache.k, cache.v, i32([0]), scales=cache.scales)
    code, e = quantise64(x[0, :, 0])
    got, exponent = cache.k[0, 0, :64], cache.ks[0, 0, :64].long() - 127
    assert torch.equal(exponent, e)
    assert torch.equal(torch.isnan(got.float()), torch.isnan(code))
    assert torch.equal(torch.nan_to_num(got.double(), nan=0.0), torch.nan_to_num(code, nan=0.0))
    k, v = sv.specvlm_kv_read(cache.k, cache.v, i32([64]), 64, scales=cache.scales, dtype=dtype)
    value = (code * two_to(e)[:, None]).to(dtype)
    assert torch.equal(torch.nan_to_num(k[0, :, 0], nan=5.0), torch.nan_to_num(value, nan=5.0)) and bool(torch.isfinite(k[0, :13]).all())
    assert torch.equal(as_bytes(cache.k)[0, :, :64], as_bytes(cache.v)[0, :, :64])


@pytest.mark.parametrize("start,count", [([0], [1]), ([0, 7, 100], [40, 0, 33]), ([31, 2], [16, 100]), ([0] * 5, [64, 1, 2, 3, 0])])
@pytest.mark.parametrize("heads,D", [(1, 128), (5, 64), (8, 128)])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (E4M3, F32), (BF16, BF16), (F32, F32)])
def test_read(sv, start, count, heads, D, paged, kind, dtype):
    g = gen(heads + len(count))
    cache = Cache(g, [a + n for a, n in zip(start, count)], heads, D, kind, paged)
    N = max(count) + 3
    out = rows(g, len(start), N, heads, D, dtype, fused=heads == 5)
    before = [t.clone() for t in out]
    err = i32([0])
    got = sv.specvlm_kv_read(cache.k, cache.v, i32(count), start=i32(start), block_table=cache.table, scales=cache.scales, out=out,
                             err_flag=err)
    assert int(err) == 0 and got[0] is out[0] and got[1] is out[1]
    fresh = sv.specvlm_kv_read(cache.k, cache.v, i32(count), N, start=i32(start), block_table=cache.table, scales=cache.scales,
                               dtype=dtype)
    for b, (a, n) in enumerate(zip(start, count)):
        for which in range(2):
            if n:
                want = cache.rows64(b, range(a, a + n), which)
                assert torch.equal(out[which][b, :n].double(), want) and torch.equal(fresh[which][b, :n].double(), want)
            assert torch.equal(out[which][b, n:], before[which][b, n:]) and not fresh[which][b, n:].any()


@pytest.mark.parametrize("kind", [E4M3, BF16])
@pytest.mark.parametrize("paged", [False, True])
def test_bad_requests_are_reported_and_left(sv, kind, paged):
    g = gen(3)
    cache = Cache(g, [64, 64], 2, 64, kind, paged)
    k, v = rows(g, 2, 8, 2, 64, BF16, fused=False)
    for new, prefix, bit in (([9, 8], [0, 0], 2), ([-1, 8], [0, 0], 2), ([8, 8], [-1, 0], 4), ([8, 8], [cache.capacity - 7, 0], 4),
                             ([8, 8], [2 ** 31 - 1, 0], 4), ([8, 8], [-2 ** 31, 0], 4), ([8, 0], [cache.capacity + 1, 0], 4)):
        want = expect_append(cache, prefix, [0, new[1]], k, v)
        err = i32([0])
        sv.specvlm_kv_append(k, v, cache.k, cache.v, i32(prefix), num_new=i32(new), block_table=cache.table, scales=cache.scales, err_flag=err)
        assert int(err) == bit
        same(held(cache), want)
        out = [torch.full_like(t, 7.0) for t in (k, v)]
        err = i32([0])
        sv.specvlm_kv_read(cache.k, cache.v, i32(new), start=i32(prefix), block_table=cache.table, scales=cache.scales, out=out, err_flag=err)
        assert int(err) == bit and bool((out[0][0] == 7.0).all()) and bool((out[1][0] == 7.0).all())


@pytest.mark.parametrize("kind", [E4M3, BF16])
def test_block_ids_outside_the_pool(sv, kind):
    g = gen(4)
    cache = Cache(g, [64], 2, 128, kind, True)
    k, v = rows(g, 1, 40, 2, 128, BF16, fused=False)
    good = cache.table
    for bad in (-1, cache.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        want = expect_append(cache, [10], [40], k, v)
        for w, h in zip(want, held(cache)):                # (block 1 of the request keeps what it holds)
            w[int(good[0, 1])] = h[int(good[0, 1])]
        table = good.clone()
        table[0, 1] = bad
        err = i32([0])
        sv.specvlm_kv_append(k, v, cache.k, cache.v, i32([10]), block_table=table, scales=cache.scales, err_flag=err)
        assert int(err) == 16
        same(held(cache), want)
        out = [torch.full_like(t, 7.0) for t in (k, v)]
        err = i32([0])
        sv.specvlm_kv_read(cache.k, cache.v, i32([40]), start=i32([10]), block_table=table, scales=cache.scales, out=out, err_flag=err)
        assert int(err) == 16
        for which in range(2):
            assert bool((out[which][0, 6:22] == 7.0).all())
            for lo, hi in ((0, 6), (22, 40)):
                assert torch.equal(out[which][0, lo:hi].double(), cache.rows64(0, range(10 + lo, 10 + hi), which))


def compacted(cache, prefix, path, length):
    want = held(cache)
    old = held(cache)
    for b, P in enumerate(prefix):
        m = int(length[b])
        source = cache.places(b, [P + int(path[b][j]) for j in range(m + 1)])
        for (r0, t0), (r1, t1) in zip(source, cache.places(b, range(P, P + m + 1))):
            for w, o in zip(want, old):
                w[:, r1, :, t1] = o[:, r0, :, t0]
    return want


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,D,layers", [(1, 64, 1), (3, 128, 2), (32, 128, 3), (5, 64, 4)])
@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("by_ptr", [False, True])
def test_compaction(sv, paged, heads, D, layers, alias, by_ptr):
    g = gen(heads + layers)
    prefix, nodes = [30, 0, 65], 64
    paths = [[0, 2, 3, 17, 40, -1, -1, -1], [0, -1, -1, -1, -1, -1, -1, -1], [0, 1, 9, 10, 11, 30, 62, 63]]
    length = [4, 0, 7]
    cache = Cache(g, [p + nodes for p in prefix], heads, D, E4M3, paged, layers=layers)
    want = compacted(cache, prefix, paths, length)
    P, path, m = i32(prefix), i32(paths), i32(length)
    moved = torch.zeros((3, 8, 2), dtype=torch.int32, device="cuda")
    err = i32([0])
    kw = dict(block_table=cache.table, moved_idx=moved, err_flag=err, new_prefix_len=P if alias else None)
    if by_ptr:
        ptrs = tuple(torch.tensor([t[l].data_ptr() for l in range(layers)], dtype=torch.int64, device="cuda") for t in (cache.k, cache.v, cache.ks, cache.vs))
        new, _ = sv.specvlm_kv_compact_quantized(cache.k[0], cache.v[0], (cache.ks[0], cache.vs[0]), P, path, m, layer_ptrs=ptrs, **kw)
    else:
        new, _ = sv.specvlm_kv_compact_quantized(cache.k, cache.v, cache.scales, P, path, m, **kw)
    same(held(cache), want)
    assert int(err) == 0 and new.tolist() == [p + n + 1 for p, n in zip(prefix, length)]
    for b in range(3):
        for j in range(8):
            assert moved[b, j].tolist() == ([prefix[b] + paths[b][j], prefix[b] + j] if j <= length[b] else [-1, -1])


def test_compaction_longest_path(sv):
    """A path of 64 nodes out of 64 moves nothing; one of every second slot moves them all."""
    g = gen(1)
    cache = Cache(g, [64 + 40], 4, 128, E4M3, True, layers=2)
    path = [list(range(0, 64, 2)) + [-1] * 32]
    want = compacted(cache, [40], path, [31])
    sv.specvlm_kv_compact_quantized(cache.k, cache.v, cache.scales, i32([40]), i32(path), i32([31]), block_table=cache.table)
    same(held(cache), want)
    before = held(cache)
    sv.specvlm_kv_compact_quantized(cache.k, cache.v, cache.scales, i32([40]), i32([list(range(64))]), i32([63]), block_table=cache.table)
    same(held(cache), before)


def test_compaction_bad_blocks_stay(sv):
    g = gen(1)
    cache = Cache(g, [80], 2, 64, E4M3, True, layers=2)
    before = held(cache)
    table = cache.table.clone()
    table[0, 3] = -3
    err = i32([0])
    sv.specvlm_kv_compact_quantized(cache.k, cache.v, cache.scales, i32([16]), i32([[0, 40]]), i32([1]), block_table=table, err_flag=err)
    assert int(err) == 16
    same(held(cache), before)
