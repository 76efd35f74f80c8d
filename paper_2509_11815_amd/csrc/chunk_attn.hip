// Attention of a chunk of new tokens over a bf16 or e4m3 cache that holds them: causal, or a draft tree of up to 64 nodes.
//
//   rows      the (token, query head) pairs of a KV head's group, token by token, so that a block of rows has few tokens and a tight causal
//             edge.  Here: at most 32 of them, decoding and short chunks; more are chunk_rows.hip's
//   product   v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T += V^T P^T: exp2(S^T) packed to bf16 is the second product's operand as it is
//   fetch     16 bytes a lane through registers, a tile ahead of its use; e4m3 codes become bf16 on the way to LDS (exact, the row's scale goes
//             into the conversion), so both kinds of cache share everything behind it.  No slot at or past the request's length is read
//   softmax   one pass, the reference maximum moves only where a score lies 2^8 above it; maximum, sum and accumulators in fp32
//   merge     four wavefronts with a key stream each (tiles of 32 keys, every fourth) meet in LDS, ranges of keys through the workspace
//
// Bound by the stream of K and V (one token over 131 000 slots of 8 heads 91 us, 5.9 TB/s; sixteen over 64 - 16 383 in e4m3 34 us) and, where that
// is short, by its chain of latencies (one over 768 slots of 32 heads 10.8 us).  Two workgroups a compute unit: nothing of the next tile is in registers but what has been loaded of it.
#include "chunk_common.hpp"

namespace specvlm {

namespace {

template <int D, bool E4M3, bool PAGED>
__device__ __forceinline__ void attend32(const ChunkParams& p) {
    constexpr int NC = D / 16;                 // contraction steps of K Q^T
    constexpr int NT = D / 32;                 // output blocks of 32 head dims
    constexpr int ROWG = D / 8;                // 16-byte granules of a bf16 row
    constexpr int ROWB = D * 2;                // bytes of a row in LDS
    constexpr int LPR = (E4M3 ? D : 2 * D) / 16;   // lanes per cached row
    constexpr int RPI = 64 / LPR;              // rows per load instruction
    constexpr int KI = kKeys / RPI;            // load instructions per tile
    constexpr int kTileBytes = kKeys * ROWB;
    constexpr int kMergeBytes = NT * 3 * 4096;
    constexpr int kLds = kMergeBytes > kWaveWgs * 2 * kTileBytes ? kMergeBytes : kWaveWgs * 2 * kTileBytes;

    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[kLds];
    __shared__ float s_m[kWaveWgs][32];
    __shared__ float s_l[kWaveWgs][32];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    Item it;
    if (!find_item<32, 2, 4>(p, lane, it)) return;
    it = uniform(it);
    const int b = it.b, hk = it.hk, n = it.n, P = it.P, S = P + n;
    const int row0 = it.rb * 32;
    const Rows<1> rows(p, hk, n, row0, l32);
    unsigned long long anc[1] = {};
    if (p.parent && !ancestors(p, it, lane, rows.token, anc)) return;
    const int first_token = divide(row0, p.magic_group);
    const int last_token = Work<ChunkParams, 32>::last_token(p, n, it.rb);
    const int all_see = p.parent ? P : P + first_token + 1;          // slots that every row of the block sees
    const int end = p.parent ? S : P + last_token + 1;               // slots that some row sees
    // Tiles of this segment, up to the block's end; this wavefront's stream has every fourth.
    const int ntile = min((end - 1) / kKeys + 1, it.to * kWaveWgs);
    const int tile0 = it.from * kWaveWgs + wave;
    const int my_tiles = tile0 < ntile ? (ntile - tile0 + kWaveWgs - 1) / kWaveWgs : 0;

    // ---- tile fetch -------------------------------------------------------------------------
    const int lrow = lane / LPR, lpos = lane % LPR;
    const int es = E4M3 ? 1 : 2;
    const uint32_t row_bytes = static_cast<uint32_t>(p.g.stride_t) * es;
    const int64_t head_off = (hk * p.g.stride_h + (PAGED ? 0 : b * p.g.stride_b)) * es;
    const int64_t s_off = hk * p.s_sh + (PAGED ? 0 : b * p.s_sb);
    const int last_blk = (S - 1) >> 4;
    bool bad_block = false;
    // Block ids: lane 2i + x holds that of half x of tile i (mod 32) of the stream, and the next 32 tiles' are on their way
    int ids = 0, ids_next = 0;
    auto request_ids = [&](int j) __attribute__((always_inline)) {
        const int blk = min((tile0 + (j + (lane >> 1)) * kWaveWgs) * 2 + (lane & 1), last_blk);
        return p.g.block_table[static_cast<int64_t>(b) * p.g.max_blocks + blk];
    };
    auto take_ids = [&](int raw) __attribute__((always_inline)) {
        bad_block = bad_block || static_cast<uint32_t>(raw) >= static_cast<uint32_t>(p.g.num_blocks);
        ids = min(max(raw, 0), p.g.num_blocks - 1);
    };
    struct Raw { u32x4 w[KI]; uint32_t e[E4M3 ? KI : 1]; };
    auto load = [&](Raw& raw, const unsigned char* cache, const unsigned char* scales, int j) __attribute__((always_inline)) {
        const int slot0 = (tile0 + j * kWaveWgs) * kKeys;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const unsigned char *base, *sbase = scales + s_off;
            uint32_t row;
            if constexpr (PAGED) {
                const int x = i * RPI / 16;
                const int blk = __builtin_amdgcn_readlane(ids, (2 * j + x) & 63);
                base = cache + head_off + blk * (p.g.stride_b * es);
                sbase += blk * p.s_sb;
                row = min(i * RPI % 16 + lrow, (slot0 >> 4) + x >= last_blk ? (S - 1) & 15 : 15);
            } else {
                base = cache + head_off + static_cast<int64_t>(slot0) * row_bytes;
                sbase += slot0;
                row = min(i * RPI + lrow, S - 1 - slot0);
            }
            raw.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + (row * row_bytes + lpos * 16)));
            if constexpr (E4M3) raw.e[i] = sbase[row];
        }
    };
    // Into LDS as bf16 rows: granule g of K row r at g ^ (r % ROWG), the 64-byte chunk c of V row r at c ^ vswz(r), so that the operand
    // reads below meet no bank twice.
    auto vswz = [](int r) { return D == 128 ? (r & 3) : ((r >> 1) & 1); };
    unsigned char* const kbuf = s_mem + wave * 2 * kTileBytes;
    unsigned char* const vbuf = kbuf + kTileBytes;
    auto store = [&](const Raw& raw, auto is_v) __attribute__((always_inline)) {
        constexpr bool V = decltype(is_v)::value;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int r = i * RPI + lrow;
            unsigned char* const to = (V ? vbuf : kbuf) + r * ROWB;
            const int swz = V ? vswz(r) << 2 : r & (ROWG - 1);
            if constexpr (E4M3) {
                const float scale = __uint_as_float(raw.e[i] << 23);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 w;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        w[2 * x] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw.w[i][2 * h + x], scale, false));
                        w[2 * x + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw.w[i][2 * h + x], scale, true));
                    }
                    *reinterpret_cast<u32x4*>(to + (((2 * lpos + h) ^ swz) << 4)) = w;
                }
            } else {
                *reinterpret_cast<u32x4*>(to + ((lpos ^ swz) << 4)) = raw.w[i];
            }
        }
    };

    // ---- operands ---------------------------------------------------------------------------
    uint32_t kaddr[NC];                        // lane (key l32, half hf): dims 16c + 8hf .. +7; the query rows likewise
#pragma unroll
    for (int c = 0; c < NC; ++c) kaddr[c] = l32 * ROWB + (((2 * c + hf) ^ (l32 & (ROWG - 1))) << 4);
    // va[x] element e is key 16x + 8 (e / 4) + 4 hf + e % 4, dim 32t + l32 of block t (attn_streams.hip has the same reads)
    const int k0 = 4 * hf + ((lane & 15) >> 2);
    const uint32_t vaddr = k0 * ROWB + ((lane >> 4) & 1) * 32 + (lane & 3) * 8 + (vswz(k0) << 6);
    bf16x8 ka[NC], va[2], qf[NC];
    auto read_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) ka[c] = *reinterpret_cast<const bf16x8*>(kbuf + kaddr[c]);
    };
    auto read_v = [&](int t) __attribute__((always_inline)) {
        const uint32_t a = vaddr ^ (t << 6);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const s16x4 lo = lds_read_tr16(vbuf + a + (16 * x) * ROWB);
            const s16x4 hi = lds_read_tr16(vbuf + a + (16 * x + 8) * ROWB);
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            va[x] = __builtin_bit_cast(bf16x8, both);
        }
    };
    // Softmax state of row l32 (both halves agree): reference maximum, the same times c2 (0 while no key was seen), the score that moves it, and
    // this lane's part of the sum of the row's weights.  acc[t][i]: O^T row 32t + 8 (i / 4) + 4 hf + i % 4.
    float m_run[1] = {-INFINITY}, mrc = 0.f, thr = -INFINITY, l_run[1] = {0.f};
    f32x16 acc[1][NT];
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[0][t] = zero;
    // Tiles on their way through registers: one, of e4m3 caches two (tile j in set j % 2)
    constexpr int SETS = E4M3 ? 2 : 1;
    Raw kraw[SETS], vraw[SETS];
    auto bring = [&](int set, int tile) __attribute__((always_inline)) {
        if (tile >= my_tiles) return;
        if (PAGED && tile && (tile & 31) == 0) {
            take_ids(ids_next);
            if (tile + 32 < my_tiles) ids_next = request_ids(tile + 32);
        }
        load(kraw[set], p.k, p.ks, tile);
        load(vraw[set], p.v, p.vs, tile);
    };
    if (my_tiles > 0) {
        if constexpr (PAGED) {
            take_ids(request_ids(0));
            if (my_tiles > 32) ids_next = request_ids(32);
        }
        bring(0, 0);
        if constexpr (SETS == 2) bring(1, 1);
        const uint16_t* row = p.q + b * p.q_sb + rows.token[0] * p.q_sn + rows.head[0] * p.q_sh + 8 * hf;
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(row + 16 * c);
        store(kraw[0], std::false_type{});
        store(vraw[0], std::true_type{});
        bring(0, SETS);
        wave_order();
    }
    auto step = [&](auto next_set, int j) __attribute__((always_inline)) {
        constexpr int NEXT_SET = decltype(next_set)::value;
        const int slot0 = (tile0 + j * kWaveWgs) * kKeys;
        read_k();
        f32x16 s;
#pragma unroll
        for (int c = 0; c < NC; ++c) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[c], qf[c], c ? s : zero, 0, 0, 0);
        if (slot0 + kKeys > all_see) hide(s, p.parent ? visible_tree(P, anc[0], slot0) : visible_causal(P, rows.token[0], slot0), hf);
        const float lmax = max16(s);
        if (__builtin_expect(__any(lmax > thr), 0)) {
            const float m_new = fmaxf(m_run[0], fmaxf(lmax, other_half(lmax)));
            const float m_safe = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m_run[0] == -INFINITY ? 1.f : fast_exp2((m_run[0] - m_safe) * p.c2);
            m_run[0] = m_new;
            thr = m_new + p.tau;
            mrc = m_safe * p.c2;
            l_run[0] *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[0][t] *= alpha;
        }
        float pr[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) pr[i] = fast_exp2(fmaf(s[i], p.c2, -mrc));
        float sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = (pr[4 * i] + pr[4 * i + 1]) + (pr[4 * i + 2] + pr[4 * i + 3]);
        l_run[0] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        bf16x8 pf[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(pr[8 * x + 2 * e], pr[8 * x + 2 * e + 1]);
            pf[x] = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            read_v(t);
#pragma unroll
            for (int x = 0; x < 2; ++x) acc[0][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[x], pf[x], acc[0][t], 0, 0, 0);
        }
        wave_order();
        if (j + 1 < my_tiles) {
            store(kraw[NEXT_SET], std::false_type{});
            store(vraw[NEXT_SET], std::true_type{});
            bring(NEXT_SET, j + 1 + SETS);
            wave_order();
        }
    };
    if constexpr (SETS == 2) {
        for (int j = 0; j < my_tiles; j += 2) {
            step(std::integral_constant<int, 1>{}, j);
            if (j + 1 < my_tiles) step(std::integral_constant<int, 0>{}, j + 1);
        }
    } else {
        for (int j = 0; j < my_tiles; ++j) step(std::integral_constant<int, 0>{}, j);
    }
    if (PAGED && __any(bad_block) && lane == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_BLOCK);
    finish<D, 1>(p, it, rows, acc, m_run, l_run, s_mem, s_m, s_l);
}

template <int D, bool E4M3, bool PAGED>
__global__ __launch_bounds__(kWaveWgs * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void chunk_few_kernel(ChunkParams p) {
    attend32<D, E4M3, PAGED>(p);
}

template <int D>
void launch_few(const ChunkParams& p, bool e4m3, dim3 grid, hipStream_t stream) {
    auto* const kernel = e4m3 ? (p.g.block_table ? chunk_few_kernel<D, true, true> : chunk_few_kernel<D, true, false>)
                              : (p.g.block_table ? chunk_few_kernel<D, false, true> : chunk_few_kernel<D, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kWaveWgs * 64), 0, stream, p);
}

struct ChunkPlan {
    int qb;                  // blocks of 32 rows per workgroup; 0: wavefronts with 64 rows each share the tiles
    int row_blocks, target, places;          // see ChunkParams
    int64_t workgroups;
    size_t bytes;            // workspace
};

// How a call is divided, with `bytes` of workspace.
ChunkPlan chunk_plan(const specvlm_attn_desc& d, bool tree, size_t bytes) {
    ChunkPlan plan;
    const int64_t rows = static_cast<int64_t>(d.H_q / d.H_kv) * d.N_max;
    // Key streams while every 64 rows have a compute unit, whatever the keys: 32 heads and 256 tokens over nothing 10.7 us, of a shared block's
    // 17.1; over 1000 slots 26 of 39; 512 tokens over 8000 in bf16 93 of 97, in e4m3 96 of 91.  With twice as many blocks shared tiles are ahead
    // (1024 tokens over 8000: 173 of 191; four chunks of 256 with eight KV heads 108 of 181).  Up to 128 rows a shared block would be half empty.
    plan.qb = rows <= 32 ? 1 : rows <= 128 || tree || d.B * static_cast<int64_t>(d.H_kv) * ((rows + 63) / 64) <= 256 ? 2 : 0;
    const int block = plan.qb ? 32 * plan.qb : kSharedRows;
    plan.row_blocks = static_cast<int>((rows + block - 1) / block);
    const int64_t pairs = static_cast<int64_t>(d.B) * d.H_kv * plan.row_blocks;
    plan.target = plan.places = 0;
    plan.workgroups = pairs;
    plan.bytes = 0;
    const int64_t slots = bytes < kChunkCounterBytes ? 0 : (bytes - kChunkCounterBytes) / (2 * part_bytes(block, d.D));
    if (d.num_splits == 1 || pairs > kMostPairs || slots < 8) return plan;
    // A place for a workgroup on every compute unit, for two of 32 rows.  Key streams: a part for every place, up to two or three times as many
    plan.places = plan.qb == 1 ? 512 : 256;
    const int64_t most = std::min<int64_t>(!plan.qb ? plan.places : std::max<int64_t>((plan.qb == 1 ? 2 : 3) * plan.places, pairs), slots);
    if (plan.qb && most < pairs) return plan;
    plan.target = static_cast<int>(most);
    // (shared: stretches, or an item each and one more for every half)
    plan.workgroups = (std::max<int64_t>(plan.target, plan.qb ? 0 : pairs + plan.target / 2) + 7) / 8 * 8;
    plan.bytes = kChunkCounterBytes + static_cast<size_t>(plan.target) * 2 * part_bytes(block, d.D);
    return plan;
}

}  // namespace

size_t chunk_workspace_bytes(const specvlm_attn_desc& d) { return std::max(chunk_plan(d, false, SPECVLM_CHUNK_WORKSPACE_BYTES).bytes,
                                                                              d.N_max > SPECVLM_MAX_NODES ? 0 : chunk_plan(d, true, SPECVLM_CHUNK_WORKSPACE_BYTES).bytes); }

int32_t launch_chunk_attn(const ChunkArgs& a) {
    const specvlm_attn_desc& d = a.d;
    const ChunkPlan plan = chunk_plan(d, a.parent != nullptr, a.workspace_bytes);
    if (plan.workgroups >= int64_t{1} << 31) return SPECVLM_INVALID_ARG;
    ChunkParams p;
    p.g = KvGeom{d.kv_stride_b, d.kv_stride_h, d.kv_stride_t, d.paged ? a.block_table : nullptr, d.max_blocks_per_req, d.num_blocks,
                 d.paged ? d.max_blocks_per_req * SPECVLM_PAGE_SIZE : d.kv_capacity};
    p.k = static_cast<const unsigned char*>(a.k); p.v = static_cast<const unsigned char*>(a.v);
    p.ks = a.scales ? a.scales->k_dev : nullptr; p.vs = a.scales ? a.scales->v_dev : nullptr;
    p.s_sb = a.scales ? a.scales->stride_b : 0; p.s_sh = a.scales ? a.scales->stride_h : 0;
    p.q = static_cast<const uint16_t*>(a.q); p.o = static_cast<uint16_t*>(a.o); p.lse = a.lse;
    p.q_sb = d.q_stride_b; p.q_sn = d.q_stride_n; p.q_sh = d.q_stride_h;
    p.o_sb = d.o_stride_b; p.o_sn = d.o_stride_n; p.o_sh = d.o_stride_h;
    p.prefix_len = a.prefix_len; p.num_new = a.num_new; p.parent = a.parent; p.err_flag = a.err_flag;
    p.B = d.B; p.N_max = d.N_max; p.H_q = d.H_q; p.H_kv = d.H_kv; p.group = d.H_q / d.H_kv;
    p.row_blocks = plan.row_blocks;
    p.magic_group = divisor(p.group);
    p.scale = a.scale;
    p.c2 = a.scale * kLog2e;
    p.tau = std::fmin(kTau / p.c2, 1e30f);
    p.target = plan.target;
    p.places = plan.places;
    p.ws_cnt = static_cast<int32_t*>(a.workspace);
    p.ws_part = static_cast<unsigned char*>(a.workspace) + kChunkCounterBytes;
    const unsigned workgroups = static_cast<unsigned>(plan.workgroups);
    if (plan.qb != 1) launch_chunk_rows(p, d.D, a.scales != nullptr, !plan.qb, workgroups, a.stream);
    else if (d.D == 128) launch_few<128>(p, a.scales != nullptr, dim3(workgroups), a.stream);
    else launch_few<64>(p, a.scales != nullptr, dim3(workgroups), a.stream);
    return check_launch();
}

}  // namespace specvlm
