"""Attention of token chunks over bf16 and e4m3 caches, against the definition in 64 bits."""
import pytest
import torch

from chunk_util import Cache, attention64, check_attention, gen, i32, random_tree

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def sv():
    import paper_2509_11815_amd as sv
    sv.load_library()
    return sv


def queries(g, B, N, H, D, fused=False):
    """[B, N, H, D], on its own or as a part of a wider projection's output."""
    if not fused:
        return torch.empty((B, N, H, D), dtype=BF16, device="cuda").normal_(generator=g)
    return torch.empty((B, N, H + 4, D), dtype=BF16, device="cuda").normal_(generator=g)[:, :, 2:-2]


def run(sv, seed, H, G, D, N, prefix, new, dtype, paged, tree=False, fused=False, **kw):
    g = gen(seed)
    cache = Cache(g, [p + n for p, n in zip(prefix, new)], G, D, dtype, paged)
    parent = torch.stack([random_tree(g, N) for _ in prefix]) if tree else None
    return check_attention(sv, queries(g, len(prefix), N, H, D, fused), cache, prefix, new, parent=parent, **kw)


KINDS = [(BF16, False), (BF16, True), (E4M3, False), (E4M3, True)]
kinds = pytest.mark.parametrize("dtype,paged", KINDS, ids=["bf16", "bf16-paged", "e4m3", "e4m3-paged"])


@kinds
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [0, 1, 15, 31, 32, 100, 127, 128, 129, 1000, 4500])
def test_one_token(sv, dtype, paged, D, P):
    run(sv, P + D, 8, 2, D, 1, [P], [1], dtype, paged)


@kinds
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,P", [(2, 0), (7, 3), (33, 40), (64, 0), (65, 17), (130, 500), (257, 0), (300, 77), (513, 1290)])
def test_one_chunk(sv, dtype, paged, D, N, P):
    run(sv, N + P, 4, 2, D, N, [P], [N], dtype, paged, fused=True)


@kinds
@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (7, 7), (8, 1), (12, 4), (40, 8), (64, 2), (33, 1)])
def test_heads(sv, dtype, paged, H, G):
    run(sv, H, H, G, 128, 9, [200, 3], [9, 5], dtype, paged)


@kinds
@pytest.mark.parametrize("D", [64, 128])
def test_ragged_batch_with_idle_requests(sv, dtype, paged, D):
    run(sv, 5, 8, 2, D, 70, [0, 900, 33, 5000, 0, 17, 250], [70, 0, 1, 64, 0, 69, 16], dtype, paged)


@kinds
@pytest.mark.parametrize("N,prefix", [(1, [0]), (2, [31, 0]), (60, [768, 33, 0]), (64, [3264]), (64, [16, 15, 100]), (33, [4864, 4000])])
@pytest.mark.parametrize("D", [64, 128])
def test_trees(sv, dtype, paged, D, N, prefix):
    new = [max(1, N - 7 * b) for b in range(len(prefix))]
    run(sv, N, 8, 4, D, N, prefix, new, dtype, paged, tree=True)


@kinds
def test_softmax_scale(sv, dtype, paged):
    run(sv, 3, 8, 2, 128, 20, [300], [20], dtype, paged, softmax_scale=0.31)


@kinds
def test_large_scores_and_far_maxima(sv, dtype, paged):
    """Scores far apart, the greatest one late: the reference maximum has to move."""
    g = gen(11)
    cache = Cache(g, [700], 2, 128, dtype, paged)
    q = queries(g, 1, 40, 8, 128) * 12
    check_attention(sv, q, cache, [660], [40])


def test_a_chunk_is_its_tokens_one_at_a_time(sv):
    g = gen(4)
    N, P = 37, 211
    cache = Cache(g, [P + N], 2, 128, E4M3, True)
    q = queries(g, 1, N, 8, 128)
    whole = sv.specvlm_chunk_attn(q, cache.k, cache.v, i32([P]), block_table=cache.table, scales=cache.scales)
    bound = attention64(q, cache, 0, P, N)[2]
    for i in range(N):
        one = sv.specvlm_chunk_attn(q[:, i:i + 1].contiguous(), cache.k, cache.v, i32([P + i]), block_table=cache.table, scales=cache.scales)
        # each of the two is off by no more than its bound from the exact result, which is the same; results are not bounded by 1 (e4m3 rows here
        # have scales up to e^2 or so), and half a bf16 step of 4 .. 8 alone is 2^-6
        assert bool(((whole[0, i].double() - one[0, 0].double()).abs() <= 2 * bound[i]).all())


def test_chain_tree_is_causal(sv):
    g = gen(6)
    N = 50
    cache = Cache(g, [400 + N], 4, 64, BF16, False)
    q = queries(g, 1, N, 8, 64)
    chain = torch.arange(-1, N - 1, dtype=torch.int32, device="cuda")[None]
    a, la = check_attention(sv, q, cache, [400], [N])
    b, lb = check_attention(sv, q, cache, [400], [N], parent=chain)
    assert torch.equal(a, b) and torch.equal(la, lb)


@kinds
def test_bad_requests_are_reported_and_left(sv, dtype, paged):
    """num_new, lengths and trees that do not hold: the request's rows stay, the others are served."""
    g = gen(8)
    cache = Cache(g, [64, 64, 64, 64], 2, 64, dtype, paged)
    q = queries(g, 4, 10, 4, 64)
    chain = torch.arange(-1, 9, dtype=torch.int32, device="cuda").repeat(4, 1)
    good, _ = check_attention(sv, q, cache, [54] * 4, [10] * 4, parent=chain)
    for new, prefix, bad_parent, bit in (([11, 10, 10, 10], [54] * 4, None, 2), ([-1, 10, 10, 10], [54] * 4, None, 2),
                                         ([10] * 4, [cache.capacity - 9, 54, 54, 54], None, 4), ([10] * 4, [-1, 54, 54, 54], None, 4),
                                         ([10] * 4, [2 ** 31 - 1, 54, 54, 54], None, 4), ([10] * 4, [-2 ** 31, 54, 54, 54], None, 4),
                                         ([10] * 4, [54] * 4, 3, 1), ([10] * 4, [54] * 4, 5, 1)):
        parent = chain.clone()
        if bad_parent is not None:
            parent[0, 3] = bad_parent
        out = torch.full_like(q, 7.0)
        err = i32([0])
        sv.specvlm_chunk_attn(q, cache.k, cache.v, i32(prefix), num_new=i32(new), parent=parent, block_table=cache.table,
                              scales=cache.scales, out=out, err_flag=err)
        assert int(err) == bit, (new, prefix, bad_parent)
        assert bool((out[0] == 7.0).all()) and torch.equal(out[1:], good[1:])


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_block_ids_outside_the_pool(sv, dtype):
    g = gen(9)
    cache = Cache(g, [100, 100], 2, 128, dtype, True)
    q = queries(g, 2, 3, 4, 128)
    good, _ = check_attention(sv, q, cache, [97, 97], [3, 3])
    for bad in (-1, cache.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        table = cache.table.clone()
        table[0, 2] = bad
        err = i32([0])
        out = sv.specvlm_chunk_attn(q, cache.k, cache.v, i32([97, 97]), block_table=table, scales=cache.scales, err_flag=err)
        assert int(err) == 16 and torch.equal(out[1], good[1])


@kinds
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G,N,prefix,new", [(4, 4, 300, [0], [300]), (8, 2, 129, [63, 0, 1000], [129, 128, 1]), (3, 1, 1000, [0, 500], [1000, 333]),
                                              (2, 2, 2050, [31], [2050]), (5, 1, 200, [2111, 0], [200, 52]), (8, 1, 33, [1, 2, 3], [33, 32, 0]),
                                              (1, 1, 512, [2000], [256]), (7, 1, 1100, [40], [1100])])
def test_long_chunks(sv, dtype, paged, D, H, G, N, prefix, new):
    run(sv, N + H, H, G, D, N, prefix, new, dtype, paged, fused=True)
