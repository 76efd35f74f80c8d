// Attention of a chunk of new tokens over a bf16 or e4m3 cache that holds them: causal, or a draft tree of up to 64 nodes.
//
//   rows      the (token, query head) pairs of a KV head's group, token by token, so that a block of 64 rows has few tokens and a tight
//             causal edge; a workgroup has 64 rows, its four wavefronts a key stream each (tiles of 32 keys, every fourth)
//   product   v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T += V^T P^T: exp2(S^T) packed to bf16 is the second product's operand as it is
//   fetch     16 bytes a lane through registers, a tile ahead of its use; e4m3 codes become bf16 on the way to LDS (exact, the row's scale goes
//             into the conversion), so both kinds of cache share everything behind it.  No slot at or past the request's length is read
//   softmax   one pass, the reference maximum moves only where a score lies 2^8 above it; maximum, sum and accumulators in fp32
//   merge     the four streams meet in LDS
#include <type_traits>

#include "attn_common.hpp"
#include "attn_rows.hpp"

namespace specvlm {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct ChunkParams {
    KvGeom g;                                // strides in elements of the cache
    const unsigned char *k, *v, *ks, *vs;    // cache; scales (e4m3)
    int64_t s_sb, s_sh;
    const uint16_t* q;
    uint16_t* o;
    float* lse;
    int64_t q_sb, q_sn, q_sh, o_sb, o_sn, o_sh;
    const int32_t *prefix_len, *num_new, *parent;
    int32_t* err_flag;
    int B, N_max, H_q, H_kv, group, row_blocks;
    uint32_t magic_group;
    float scale, c2, tau;                    // softmax scale; times log2 e; how far a score may lie above the reference
};

__device__ __forceinline__ float max16(const f32x16& a) {
    auto max3 = [](float x, float y, float z) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z); };
    const float u = max3(a[0], a[1], a[2]), v = max3(a[3], a[4], a[5]), w = max3(a[6], a[7], a[8]), x = max3(a[9], a[10], a[11]);
    const float y = max3(a[12], a[13], a[14]);
    return max3(max3(u, v, w), max3(x, y, a[15]), a[15]);
}

// What the other half of the wavefront (lane ^ 32) holds.
__device__ __forceinline__ float other_half(float x) {
    const uint32_t a = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// LDS traffic between lanes of one wavefront needs no wait (it is in order) but must stay in order.
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }

template <int D, int QB, bool E4M3, bool PAGED>
__device__ __forceinline__ void attend(const ChunkParams& p) {
    constexpr int NC = D / 16;                 // contraction steps of K Q^T
    constexpr int NT = D / 32;                 // output blocks of 32 head dims
    constexpr int ROWG = D / 8;                // 16-byte granules of a bf16 row
    constexpr int ROWB = D * 2;                // bytes of a row in LDS
    constexpr int LPR = (E4M3 ? D : 2 * D) / 16;   // lanes per cached row
    constexpr int RPI = 64 / LPR;              // rows per load instruction
    constexpr int KI = kKeys / RPI;            // load instructions per tile
    constexpr int kTileBytes = kKeys * ROWB;
    constexpr int ROWS = QB * 32;
    constexpr int NB = QB * NT;                // (32 rows, 32 dims) blocks of the result
    constexpr int OWN = NB >= kWaveWgs ? NB / kWaveWgs : 1;
    constexpr int kMergeBytes = NB * 3 * 4096;
    constexpr int kLds = kMergeBytes > kWaveWgs * 2 * kTileBytes ? kMergeBytes : kWaveWgs * 2 * kTileBytes;

    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[kLds];
    __shared__ float s_m[kWaveWgs][ROWS];
    __shared__ float s_l[kWaveWgs][ROWS];

    const uint32_t pair = blockIdx.x / static_cast<uint32_t>(p.row_blocks);
    const int rb = blockIdx.x - pair * p.row_blocks;
    const int b = pair / static_cast<uint32_t>(p.H_kv);
    const int hk = pair - b * p.H_kv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;

    typedef const __attribute__((address_space(4))) int32_t* const_i32;
    const int n = p.num_new ? ((const_i32)p.num_new)[b] : p.N_max;
    const int P = ((const_i32)p.prefix_len)[b];
    int err = 0;
    if (n < 0 || n > p.N_max) err |= SPECVLM_ERR_BAD_NUM_NODES;
    else if (P < 0 || P > p.g.capacity - n) err |= SPECVLM_ERR_BAD_LENGTH;
    const bool reports = rb == 0 && hk == 0 && tid == 0 && p.err_flag;
    if (err) {
        if (reports) atomicOr(p.err_flag, err);
        return;
    }
    const int row0 = rb * ROWS;
    if (row0 >= p.group * n) return;
    const int S = P + n;

    // Rows of this lane: token and head of the group.
    int token[QB], head[QB];
    bool real[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int R = row0 + qb * 32 + l32;
        token[qb] = divide(R, p.magic_group);
        head[qb] = hk * p.group + R - token[qb] * p.group;
        real[qb] = token[qb] < n;
        if (!real[qb]) { token[qb] = n - 1; head[qb] = hk * p.group; }
    }
    const int first_token = divide(row0, p.magic_group);
    const int last_token = min(static_cast<int>(divide(row0 + ROWS - 1, p.magic_group)), n - 1);

    // Ancestor-or-self masks of a tree: pointer doubling over the lanes (lane i holds node i)
    uint32_t anc_lo[QB], anc_hi[QB];
    if (p.parent) {
        int par = lane < n ? p.parent[static_cast<int64_t>(b) * p.N_max + lane] : -1;
        const bool bad_par = lane < n && (lane == 0 ? par != -1 : (par < 0 || par >= lane));
        if (__any(bad_par)) {                              // the same in every workgroup of the request
            if (reports) atomicOr(p.err_flag, SPECVLM_ERR_BAD_PARENT);
            return;
        }
        uint32_t mlo = lane < 32 ? 1u << (lane & 31) : 0u, mhi = lane < 32 ? 0u : 1u << (lane & 31);
        int up = par;
#pragma unroll 1
        while (__any(up >= 0)) {
            const int src = max(up, 0) * 4;
            const uint32_t alo = __builtin_amdgcn_ds_bpermute(src, mlo), ahi = __builtin_amdgcn_ds_bpermute(src, mhi);
            const int up2 = __builtin_amdgcn_ds_bpermute(src, up);
            if (up >= 0) { mlo |= alo; mhi |= ahi; up = up2; }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            anc_lo[qb] = __builtin_amdgcn_ds_bpermute(token[qb] * 4, mlo);
            anc_hi[qb] = __builtin_amdgcn_ds_bpermute(token[qb] * 4, mhi);
        }
    }
    const int all_see = p.parent ? P : P + first_token + 1;          // slots that every row of the block sees
    const int end = p.parent ? S : P + last_token + 1;               // slots that some row sees
    const int ntile = (end + kKeys - 1) / kKeys;
    const int my_tiles = wave < ntile ? (ntile - wave + kWaveWgs - 1) / kWaveWgs : 0;

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
        const int blk = min((wave + (j + (lane >> 1)) * kWaveWgs) * 2 + (lane & 1), last_blk);
        return p.g.block_table[static_cast<int64_t>(b) * p.g.max_blocks + blk];
    };
    auto take_ids = [&](int raw) __attribute__((always_inline)) {
        bad_block = bad_block || static_cast<uint32_t>(raw) >= static_cast<uint32_t>(p.g.num_blocks);
        ids = min(max(raw, 0), p.g.num_blocks - 1);
    };
    struct Raw { u32x4 w[KI]; uint32_t e[E4M3 ? KI : 1]; };
    auto load = [&](Raw& raw, const unsigned char* cache, const unsigned char* scales, int j) __attribute__((always_inline)) {
        const int slot0 = (wave + j * kWaveWgs) * kKeys;
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
            raw.w[i] = *reinterpret_cast<const u32x4*>(base + (row * row_bytes + lpos * 16));
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
    // va[t][x] element e is key 16x + 8 (e / 4) + 4 hf + e % 4, dim 32t + l32 (attn_streams.hip has the same reads)
    const int k0 = 4 * hf + ((lane & 15) >> 2);
    const uint32_t vaddr = k0 * ROWB + ((lane >> 4) & 1) * 32 + (lane & 3) * 8 + (vswz(k0) << 6);
    bf16x8 ka[NC], va[NT][2], qf[QB][NC];
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
            va[t][x] = __builtin_bit_cast(bf16x8, both);
        }
    };
    // Softmax state of row 32 qb + l32 (both halves agree): reference maximum, the same times c2 (0 while no key was seen), the score that
    // moves it, and this lane's part of the sum of the row's weights.  acc[qb][t][i]: O^T row 32t + 8 (i / 4) + 4 hf + i % 4.
    float m_run[QB], mrc[QB], thr[QB], l_run[QB], lmax[QB];
    f32x16 acc[QB][NT], s[QB], s_next[QB];
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m_run[qb] = -INFINITY;
        thr[qb] = -INFINITY;
        mrc[qb] = 0.f;
        l_run[qb] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[qb][t] = zero;
    }
    auto scores = [&](f32x16& d, int qb) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[c], qf[qb][c], c ? d : zero, 0, 0, 0);
    };
    bf16x8 pf[QB][2];
    auto weights = [&](int qb) __attribute__((always_inline)) {
        float pr[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) pr[i] = fast_exp2(fmaf(s[qb][i], p.c2, -mrc[qb]));
        float sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = (pr[4 * i] + pr[4 * i + 1]) + (pr[4 * i + 2] + pr[4 * i + 3]);
        l_run[qb] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(pr[8 * x + 2 * e], pr[8 * x + 2 * e + 1]);
            pf[qb][x] = __builtin_bit_cast(bf16x8, w);
        }
    };
    Raw kraw, vraw;
    if (my_tiles > 0) {
        if constexpr (PAGED) {
            take_ids(request_ids(0));
            if (my_tiles > 32) ids_next = request_ids(32);
        }
        load(kraw, p.k, p.ks, 0);
        load(vraw, p.v, p.vs, 0);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const uint16_t* row = p.q + b * p.q_sb + token[qb] * p.q_sn + head[qb] * p.q_sh + 8 * hf;
#pragma unroll
            for (int c = 0; c < NC; ++c) qf[qb][c] = *reinterpret_cast<const bf16x8*>(row + 16 * c);
        }
        store(kraw, std::false_type{});
        store(vraw, std::true_type{});
        if (my_tiles > 1) {
            load(kraw, p.k, p.ks, 1);
            load(vraw, p.v, p.vs, 1);
        }
        wave_order();
        read_k();
#pragma unroll
        for (int t = 0; t < NT; ++t) read_v(t);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) scores(s[qb], qb);
        wave_order();
        if (my_tiles > 1) {
            store(kraw, std::false_type{});
            wave_order();
            read_k();
            if (my_tiles > 2) load(kraw, p.k, p.ks, 2);
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) lmax[qb] = max16(s[qb]);
    }
    // One tile.  At its start s holds its scores and lmax their maxima; va its V operands, ka the next tile's K operands; vraw and kraw V of the
    // next tile and K of the one after it.
    auto step = [&](auto next, int j) __attribute__((always_inline)) {
        constexpr bool NEXT = decltype(next)::value;
        const int slot0 = (wave + j * kWaveWgs) * kKeys;
        if (slot0 + kKeys > all_see) {
            // bit k of `visible`: key slot0 + k.  Its place among this lane's scores is a constant once the lane's half is shifted out
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                uint32_t visible;
                if (p.parent) {
                    const int before = P - slot0;          // keys of the tile in the prefix, < 32
                    const unsigned long long anc = (static_cast<unsigned long long>(anc_hi[qb]) << 32) | anc_lo[qb];
                    visible = before > 0 ? (anc_lo[qb] << before) | ((1u << before) - 1u) : static_cast<uint32_t>(anc >> -before);
                } else {
                    const int seen = P + token[qb] + 1 - slot0;
                    visible = seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u;
                }
                visible >>= 4 * hf;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t on = static_cast<uint32_t>(static_cast<int32_t>(visible << (31 - (8 * (i >> 2) + (i & 3)))) >> 31);
                    s[qb][i] = __uint_as_float((on & __float_as_uint(s[qb][i])) | (~on & 0xFF800000u));
                }
                lmax[qb] = max16(s[qb]);
            }
        }
        bool moves = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) moves = moves | (lmax[qb] > thr[qb]);
        if (__builtin_expect(__any(moves), 0)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const float m_new = fmaxf(m_run[qb], fmaxf(lmax[qb], other_half(lmax[qb])));
                const float m_safe = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = m_run[qb] == -INFINITY ? 1.f : fast_exp2((m_run[qb] - m_safe) * p.c2);
                m_run[qb] = m_new;
                thr[qb] = m_new + p.tau;
                mrc[qb] = m_safe * p.c2;
                l_run[qb] *= alpha;
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[qb][t] *= alpha;
            }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            if constexpr (NEXT) scores(s_next[qb], qb);
            weights(qb);
        }
        wave_order();
        if constexpr (NEXT) {
            store(vraw, std::true_type{});
            if (j + 2 < my_tiles) {
                store(kraw, std::false_type{});
                if (PAGED && ((j + 3) & 31) == 0) {
                    // (V of tile j + 2 still needs the ids of its own 32 tiles: before they change)
                    load(vraw, p.v, p.vs, j + 2);
                    take_ids(ids_next);
                    if (j + 3 + 32 < my_tiles) ids_next = request_ids(j + 3 + 32);
                } else {
                    load(vraw, p.v, p.vs, j + 2);
                }
                if (j + 3 < my_tiles) load(kraw, p.k, p.ks, j + 3);
                wave_order();
                read_k();
            }
            wave_order();
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) acc[qb][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t][x], pf[qb][x], acc[qb][t], 0, 0, 0);
            if constexpr (NEXT) read_v(t);
        }
        if constexpr (NEXT) {
            wave_order();
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) { s[qb] = s_next[qb]; lmax[qb] = max16(s[qb]); }
        }
    };
    {
        int j = 0;
        for (; j < my_tiles - 1; ++j) step(std::true_type{}, j);
        if (my_tiles > 0) step(std::false_type{}, j);
    }
    if (PAGED && __any(bad_block) && lane == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_BLOCK);

    // ---- merge of the four streams ------------------------------------------------------------
    // Block x: rows 32 (x / NT), dims 32 (x % NT); wavefront w owns blocks OWN w .. (head size 64 and 32 rows: the first two have one each).
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        l_run[qb] += other_half(l_run[qb]);
        if (hf == 0) {
            s_m[wave][qb * 32 + l32] = m_run[qb];
            s_l[wave][qb * 32 + l32] = l_run[qb];
        }
    }
    __syncthreads();                                       // every stream is done with its tiles
    f32x16 out[OWN];
#pragma unroll
    for (int o = 0; o < NB / OWN; ++o) {
        if (o == wave) {                                   // uniform
#pragma unroll
            for (int e = 0; e < OWN; ++e) out[e] = acc[(o * OWN + e) / NT][(o * OWN + e) % NT];
        } else {
            const int idx = wave < o ? wave : wave - 1;
#pragma unroll
            for (int e = 0; e < OWN; ++e) {
                f32x4* dst = reinterpret_cast<f32x4*>(s_mem) + ((o * OWN + e) * 3 + idx) * 4 * 64 + lane;
                const f32x16& a = acc[(o * OWN + e) / NT][(o * OWN + e) % NT];
#pragma unroll
                for (int u = 0; u < 4; ++u) dst[u * 64] = f32x4{a[4 * u], a[4 * u + 1], a[4 * u + 2], a[4 * u + 3]};
            }
        }
    }
    __syncthreads();
    if (wave >= NB / OWN) return;
#pragma unroll
    for (int e = 0; e < OWN; ++e) {
        const int block = wave * OWN + e;
        const int qb = block / NT, t = block % NT;
        float m[kWaveWgs], w[kWaveWgs];
#pragma unroll
        for (int x = 0; x < kWaveWgs; ++x) m[x] = s_m[x][qb * 32 + l32];
        const float M = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        const float m_safe = M == -INFINITY ? 0.f : M;
        float L = 0.f;
#pragma unroll
        for (int x = 0; x < kWaveWgs; ++x) {               // (in this order in every owner of the rows)
            w[x] = fast_exp2((m[x] - m_safe) * p.c2);
            L += s_l[x][qb * 32 + l32] * w[x];
        }
        out[e] *= wave == 0 ? w[0] : wave == 1 ? w[1] : wave == 2 ? w[2] : w[3];
        const f32x4* src = reinterpret_cast<const f32x4*>(s_mem) + block * 3 * 4 * 64 + lane;
#pragma unroll
        for (int idx = 0; idx < 3; ++idx) {
            const float wx = wave <= idx ? w[idx + 1] : w[idx];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x4 v = src[(idx * 4 + u) * 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) out[e][4 * u + i] += v[i] * wx;
            }
        }
        const bool live = QB == 1 ? real[0] : qb ? real[QB - 1] : real[0];
        const int tok = QB == 1 ? token[0] : qb ? token[QB - 1] : token[0], h = QB == 1 ? head[0] : qb ? head[QB - 1] : head[0];
        const float inv = 1.f / L;
        uint16_t* const row = p.o + b * p.o_sb + tok * p.o_sn + h * p.o_sh + 32 * t + 8 * hf;
#pragma unroll
        for (int u = 0; u < 2; ++u) {                      // 16 dims: registers 8u .. 8u + 7
            uint32_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = pack_bf16x2(out[e][8 * u + 2 * i] * inv, out[e][8 * u + 2 * i + 1] * inv);
            // the halves of the wavefront hold dims 0-3, 8-11 and 4-7, 12-15: the lower keeps 0-7, the upper 8-15
            const auto r0 = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
            const auto r1 = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
            if (live) *reinterpret_cast<u32x4*>(row + 16 * u) = u32x4{r0[0], r1[0], r0[1], r1[1]};
        }
        if (live && p.lse && hf == 0 && t == 0) p.lse[(static_cast<int64_t>(b) * p.H_q + h) * p.N_max + tok] = M * p.scale + __log2f(L) * kLn2;
    }
}

template <int D, int QB, bool E4M3, bool PAGED>
__global__ __launch_bounds__(kWaveWgs * 64) __attribute__((amdgpu_waves_per_eu(1, 1))) void chunk_attn_kernel(ChunkParams p) {
    attend<D, QB, E4M3, PAGED>(p);
}

template <int D, int QB>
void launch_as(const ChunkParams& p, bool e4m3, dim3 grid, hipStream_t stream) {
    auto* const kernel = e4m3 ? (p.g.block_table ? chunk_attn_kernel<D, QB, true, true> : chunk_attn_kernel<D, QB, true, false>)
                              : (p.g.block_table ? chunk_attn_kernel<D, QB, false, true> : chunk_attn_kernel<D, QB, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kWaveWgs * 64), 0, stream, p);
}

}  // namespace

size_t chunk_workspace_bytes(const specvlm_attn_desc&) { return 0; }

int32_t launch_chunk_attn(const ChunkArgs& a) {
    const specvlm_attn_desc& d = a.d;
    constexpr int kRows = 64;
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
    p.row_blocks = (p.group * d.N_max + kRows - 1) / kRows;
    p.magic_group = divisor(p.group);
    p.scale = a.scale;
    p.c2 = a.scale * kLog2e;
    p.tau = std::fmin(kTau / p.c2, 1e30f);
    const int64_t workgroups = static_cast<int64_t>(d.B) * d.H_kv * p.row_blocks;
    if (workgroups >= int64_t{1} << 31) return SPECVLM_INVALID_ARG;
    const dim3 grid(static_cast<unsigned>(workgroups));
    if (d.D == 128) launch_as<128, 2>(p, a.scales != nullptr, grid, a.stream);
    else launch_as<64, 2>(p, a.scales != nullptr, grid, a.stream);
    return check_launch();
}

}  // namespace specvlm
