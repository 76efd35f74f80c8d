"""What the cache calls and the attention of token chunks refuse, before any HIP call (no GPU needed)."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED = 0, 1, 2
NULL, FAKE, ODD = ctypes.c_void_p(None), ctypes.c_void_p(4096), ctypes.c_void_p(4104)


@pytest.fixture(scope="module")
def lib():
    import paper_2509_11815_amd as sv
    return sv.load_library()


def desc(e4m3=False, paged=False, **changes):
    from paper_2509_11815_amd.binding import AttnDesc
    d = AttnDesc()
    d.dtype, d.B, d.H_q, d.H_kv, d.D, d.N_max = 0, 2, 8, 2, 128, 40
    d.q_stride_b, d.q_stride_n, d.q_stride_h = 40 * 8 * 128, 8 * 128, 128
    d.o_stride_b, d.o_stride_n, d.o_stride_h = 40 * 8 * 128, 8 * 128, 128
    if paged:
        d.paged, d.block_size, d.max_blocks_per_req, d.num_blocks = 1, 16, 32, 70
        d.kv_stride_b, d.kv_stride_h, d.kv_stride_t = 2 * 16 * 128, 16 * 128, 128
    else:
        d.kv_capacity = 500
        d.kv_stride_b, d.kv_stride_h, d.kv_stride_t = 2 * 500 * 128, 500 * 128, 128
    for name, value in changes.items():
        setattr(d, name, value)
    return d


def scales(k=4096, v=4096, stride_b=1000, stride_h=500):
    from paper_2509_11815_amd.binding import KvScales
    return KvScales(k, v, stride_b, stride_h)


def rows(lib, d, s=None, *, append=True, rows=FAKE, cache=FAKE, strides=(40 * 2 * 128, 2 * 128, 128), table=NULL, prefix=FAKE):
    s = ctypes.byref(s) if s is not None else None
    if append:
        return lib.specvlm_kv_append(ctypes.byref(d), rows, rows, *strides, NULL, prefix, table, cache, cache, s, NULL, NULL)
    return lib.specvlm_kv_read(ctypes.byref(d), cache, cache, s, prefix, NULL, table, rows, rows, *strides, NULL, NULL)


@pytest.mark.parametrize("append", [True, False])
def test_rows(lib, append):
    call = lambda *a, **kw: rows(lib, *a, append=append, **kw)
    assert call(desc(dtype=2)) == INVALID
    assert call(desc(B=0)) == INVALID and call(desc(B=65536)) == INVALID and call(desc(H_kv=0)) == INVALID and call(desc(D=96)) == INVALID
    assert call(desc(N_max=0)) == INVALID and call(desc(N_max=65537)) == INVALID
    assert call(desc(kv_capacity=0)) == INVALID and call(desc(kv_stride_t=120)) == INVALID and call(desc(kv_stride_h=500 * 128 + 4)) == INVALID
    assert call(desc(kv_stride_b=-8)) == INVALID and call(desc(kv_stride_t=(1 << 24) + 8)) == INVALID
    assert call(desc(kv_capacity=(1 << 30) + 1)) == INVALID                        # slot numbers and a tile behind them: below 2^31
    assert call(desc(paged=True, max_blocks_per_req=(1 << 26) + 1), table=FAKE) == INVALID
    assert call(desc(), rows=ODD) == INVALID and call(desc(), cache=ODD) == INVALID
    assert call(desc(), rows=NULL) == INVALID and call(desc(), cache=NULL) == INVALID
    assert call(desc(), strides=(1, 256, 128)) == INVALID and call(desc(), strides=(8, 256, 120)) == INVALID
    assert call(desc(), strides=(-8, 256, 128)) == INVALID and call(desc(), strides=(8, 4, 128)) == INVALID
    assert call(desc(paged=True)) == INVALID                        # no block table
    assert call(desc(), table=FAKE) == INVALID                      # ... and one too many
    assert call(desc(paged=True, block_size=32), table=FAKE) == INVALID
    assert call(desc(paged=True, num_blocks=0), table=FAKE) == INVALID
    assert call(desc(kv_stride_t=136), scales()) == INVALID         # e4m3 rows: 16-byte vectors
    assert call(desc(), scales(k=None)) == INVALID and call(desc(), scales(v=None)) == INVALID
    assert call(desc(), scales(stride_b=-1)) == INVALID and call(desc(), scales(stride_h=-1)) == INVALID
    if append:
        assert call(desc(), prefix=NULL) == INVALID


def test_compaction(lib):
    def call(d, s, L=2, base=FAKE, layer=1 << 20, ptrs=(NULL,) * 4, scale_layer=1 << 13, cap=8, table=NULL, new=FAKE):
        s = ctypes.byref(s) if s is not None else None
        return lib.specvlm_kv_compact_quantized(ctypes.byref(d), L, base, base, layer, ptrs[0], ptrs[1], s, scale_layer, ptrs[2], ptrs[3],
                                                table, FAKE, FAKE, cap, FAKE, new, NULL, NULL, NULL)
    assert call(desc(), None) == INVALID
    assert call(desc(kv_stride_t=136), scales()) == INVALID
    assert call(desc(), scales(), L=0) == INVALID and call(desc(), scales(), L=32768) == INVALID
    assert call(desc(), scales(), cap=0) == INVALID and call(desc(), scales(), cap=65) == INVALID
    assert call(desc(), scales(), base=ODD) == INVALID and call(desc(), scales(), base=NULL) == INVALID
    assert call(desc(), scales(), layer=8) == INVALID and call(desc(), scales(), layer=-16) == INVALID
    assert call(desc(), scales(), scale_layer=-1) == INVALID and call(desc(), scales(), new=NULL) == INVALID
    assert call(desc(), scales(k=None)) == INVALID
    assert call(desc(), scales(), ptrs=(FAKE, FAKE, NULL, NULL)) == INVALID        # all four or none
    assert call(desc(paged=True), scales()) == INVALID and call(desc(), scales(), table=FAKE) == INVALID


def attention(lib, d, s=None, *, q=FAKE, o=FAKE, cache=FAKE, table=NULL, prefix=FAKE, parent=NULL, ws=NULL, bytes=0):
    s = ctypes.byref(s) if s is not None else None
    return lib.specvlm_chunk_attn(ctypes.byref(d), q, cache, cache, s, table, prefix, NULL, parent, o, NULL, ws, bytes, NULL, NULL)


def test_attention(lib):
    call = lambda *a, **kw: attention(lib, *a, **kw)
    assert call(desc(dtype=1)) == UNSUPPORTED and call(desc(dtype=3)) == INVALID
    assert call(desc(H_q=7)) == INVALID and call(desc(H_q=0)) == INVALID and call(desc(D=32)) == INVALID
    assert call(desc(N_max=0)) == INVALID and call(desc(N_max=65537)) == INVALID and call(desc(N_max=65), parent=FAKE) == INVALID
    assert call(desc(H_q=512, N_max=65536)) == INVALID
    assert call(desc(kv_capacity=(1 << 30) + 1)) == INVALID
    assert call(desc(paged=True, max_blocks_per_req=(1 << 26) + 1), table=FAKE) == INVALID
    assert call(desc(softmax_scale=-1.0)) == INVALID and call(desc(softmax_scale=float("inf"))) == INVALID
    assert call(desc(softmax_scale=float("nan"))) == INVALID
    assert call(desc(num_splits=2)) == INVALID and call(desc(num_splits=-1)) == INVALID
    for name in ("q_stride_b", "q_stride_n", "q_stride_h", "o_stride_b", "o_stride_n", "o_stride_h"):
        assert call(desc(**{name: -8})) == INVALID and call(desc(**{name: 1028})) == INVALID
    assert call(desc(q_stride_h=64)) == INVALID and call(desc(o_stride_h=64)) == INVALID
    for name in ("q", "o", "cache"):
        assert call(desc(), **{name: ODD}) == INVALID and call(desc(), **{name: NULL}) == INVALID
    assert call(desc(), prefix=NULL) == INVALID
    assert call(desc(), table=FAKE) == INVALID and call(desc(paged=True)) == INVALID
    assert call(desc(kv_stride_t=136), scales()) == INVALID and call(desc(), scales(v=None)) == INVALID
    assert call(desc(), ws=ctypes.c_void_p(4096 + 128), bytes=1 << 20) == INVALID
    assert lib.specvlm_chunk_attn(None, FAKE, FAKE, FAKE, None, NULL, FAKE, NULL, NULL, FAKE, NULL, NULL, 0, NULL, NULL) == INVALID


def test_workspace_bytes(lib):
    from paper_2509_11815_amd.binding import CHUNK_WORKSPACE_BYTES
    most = 0
    for B in (1, 2, 16, 300, 65535):
        for H, G in ((1, 1), (8, 2), (40, 40), (64, 8)):
            for N in (1, 7, 64, 300, 65536):
                for capacity in (1, 100, 5000, 1 << 20, 2 ** 31 - 1):
                    for D in (64, 128):
                        d = desc(B=B, H_q=H, H_kv=G, N_max=N, kv_capacity=capacity, D=D)
                        most = max(most, lib.specvlm_chunk_attn_workspace_bytes(ctypes.byref(d)))
    assert most <= CHUNK_WORKSPACE_BYTES
    assert lib.specvlm_chunk_attn_workspace_bytes(ctypes.byref(desc(D=96))) == 0
    assert lib.specvlm_chunk_attn_workspace_bytes(ctypes.byref(desc(num_splits=1))) == 0
    assert lib.specvlm_chunk_attn_workspace_bytes(None) == 0


def test_binding_refuses_host_tensors():
    import torch

    import paper_2509_11815_amd as sv
    k = torch.zeros((1, 2, 32, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, 3, 4, 64), dtype=torch.bfloat16)
    P = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        sv.specvlm_chunk_attn(q, k, k, P)
    with pytest.raises(TypeError):
        sv.specvlm_kv_append(q[:, :, :2], q[:, :, :2], k, k, P)
    with pytest.raises(TypeError):
        sv.specvlm_kv_read(k, k, P, 4)
    with pytest.raises(TypeError):
        sv.specvlm_kv_compact_quantized(k[None], k[None], (k, k), P, P[None], P)
