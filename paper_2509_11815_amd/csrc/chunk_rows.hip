// Attention of token chunks, 64 query rows a wavefront: for chunks of the prompt and draft trees, where the matrix products count.
//
//   shared    four wavefronts share every tile of 32 keys, 256 rows a workgroup; one barrier a tile
//   streams   all four have the same 64 rows and a key stream each (every fourth tile), which meet in LDS; keys divided among workgroups
//
// Per tile and wavefront: 32 matrix instructions of 32 x 32 x 16, 32 exponentials a lane, 24 operand reads.  One wavefront a SIMD (it needs
// most of 512 registers), so that its own instructions have to fill the matrix instructions' shadow: the tile is done in two halves, each
// with the weights of one block of 32 rows beside the products of the other.  Chip-wide, matrix instructions on real operands are bound by power
// (a stream of them alone: 1.6 PFLOP/s, with four multiply-adds beside each 1.2), so every instruction left out counts.
// Measured: a first chunk of 3008 tokens of 32 heads 94 us (0.79 PFLOP/s), 1024, 1024 and 333 tokens over 4096, 7001 and 5120 e4m3 slots of 8 heads 250
// (0.92), four trees of 60 nodes over 4864 e4m3 slots of 40 heads 64 - 70 (3.0 - 3.2 TB/s).
#include "chunk_common.hpp"

namespace specvlm {

namespace {

// A shared block's part of a wavefront's 64 rows joins the other parts.  The last to come has the whole result afterwards, the same whoever that
// is (the parts are added in their order), and returns true; its own part does not go through memory.
// A part: [wavefront][2 NT blocks][4][64 lanes] vectors of four fp32, then (maximum, sum) pairs.
template <int NT>
__device__ __forceinline__ bool join(const ChunkParams& p, const Item& it, int wave, int lane, float (&M)[2], float (&L)[2], f32x16 (&acc)[2][NT]) {
    constexpr int kCoherent = 16;                          // device-coherent (sc1) loads, which the compiler counts
    constexpr int kPart = part_bytes(kSharedRows, 32 * NT), kWave = 2 * NT * 4096;
    const int l32 = lane & 31, hf = lane >> 5;
    int32_t* const cnt = p.ws_cnt + ((static_cast<int64_t>(it.b) * p.H_kv + it.hk) * p.row_blocks + it.rb) * kCounterStride + wave;
    int before = 0;
    if (lane == 0) before = __hip_atomic_load(cnt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (u(before) != it.parts - 1) {
        unsigned char* const mine = p.ws_part + part_at(it, it.part, kPart);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    u32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(acc[qb][t][4 * v + i]);
                    store16_coherent(mine + wave * kWave + (((qb * NT + t) * 4 + v) * 64 + lane) * 16, x);
                }
            if (hf == 0) store8_coherent(mine + 4 * kWave + (wave * 64 + qb * 32 + l32) * 8, u32x2{__float_as_uint(M[qb]), __float_as_uint(L[qb])});
        }
        wait_vmcnt<0>();
        if (lane == 0) before = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (u(before) != it.parts - 1) return false;
    }
    if (lane == 0) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ws_part, 0, 0x7FFFFFFF, 0x00027000);
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int ml_off = 4 * kWave + (wave * 64 + qb * 32 + l32) * 8;
        auto pair = [&](int i) __attribute__((always_inline)) {
            return __builtin_amdgcn_raw_buffer_load_b64(rsrc, ml_off, static_cast<int>(part_at(it, i, kPart)), kCoherent);
        };
        float most = M[qb];
        for (int i = 0; i < it.parts; ++i)
            if (i != it.part) most = fmaxf(most, __uint_as_float(pair(i)[0]));
        const float m_safe = most == -INFINITY ? 0.f : most;
        const float own = fast_exp2((M[qb] - m_safe) * p.c2);
        float sum = 0.f;
        f32x16 out[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) out[t][i] = 0.f;
        for (int i = 0; i < it.parts; ++i) {
            if (i == it.part) {
                sum += L[qb] * own;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) out[t][e] = fmaf(acc[qb][t][e], own, out[t][e]);
                continue;
            }
            const int at = static_cast<int>(part_at(it, i, kPart));
            const auto ml = pair(i);
            u32x4 x[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    x[t][v] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, wave * kWave + (((qb * NT + t) * 4 + v) * 64 + lane) * 16, at, kCoherent);
            const float w = fast_exp2((__uint_as_float(ml[0]) - m_safe) * p.c2);
            sum += __uint_as_float(ml[1]) * w;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[t][4 * v + e] = fmaf(__uint_as_float(x[t][v][e]), w, out[t][4 * v + e]);
        }
        M[qb] = most;
        L[qb] = sum;
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[qb][t] = out[t];
    }
    return true;
}

template <int D, bool E4M3, bool PAGED, bool SHARED>
__device__ __forceinline__ void attend64(const ChunkParams& p) {
    constexpr int QB = 2;
    constexpr int NC = D / 16, NT = D / 32, ROWG = D / 8, ROWB = D * 2;
    constexpr int LPR = (E4M3 ? D : 2 * D) / 16;   // lanes per cached row
    constexpr int RPI = 64 / LPR;              // rows per load instruction
    constexpr int KI = (SHARED ? 16 : 32) / RPI;   // load instructions of a wavefront per tensor and tile: half a tile of K or V, or whole ones of both
    constexpr int STEP = SHARED ? 1 : kWaveWgs;    // tiles from one of a stream to its next
    constexpr int kTileBytes = kKeys * ROWB;
    // Tiles of K, and of V, in LDS, and how many tiles before a tile's weights its K and V are asked for (e4m3: from memory into registers two
    // tiles before that).
    constexpr int SLOTS = SHARED ? (E4M3 ? 2 : 4) : (E4M3 ? 1 : 2);
    constexpr int K_LEAD = E4M3 ? 2 : SHARED ? 4 : 3, V_LEAD = K_LEAD - 1;
    constexpr int SETS = E4M3 ? 2 : 0;
    constexpr int kAreaBytes = 2 * SLOTS * kTileBytes;     // of a stream
    constexpr int kMergeBytes = SHARED ? 0 : QB * NT * 3 * 4096;
    constexpr int kTiles = (SHARED ? 1 : kWaveWgs) * kAreaBytes;

    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[kTiles > kMergeBytes ? kTiles : kMergeBytes];
    __shared__ float s_m[SHARED ? 1 : kWaveWgs][QB * 32];
    __shared__ float s_l[SHARED ? 1 : kWaveWgs][QB * 32];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    using W = Work<ChunkParams, SHARED ? kSharedRows : 64>;
    __shared__ std::conditional_t<SHARED, Segments, int> s_segments;
    Item it;
    for (int turn = 0; ; ++turn) {
    if constexpr (SHARED) {
        if (!next_segment<kSharedRows, !E4M3>(p, s_segments, turn, it)) return;
    } else {
        if (turn || !find_item<64, 3, 14>(p, threadIdx.x & 63, it)) return;
        it = uniform(it);
    }
    const int lane = this_thread() & 63, l32 = lane & 31, hf = lane >> 5;
    const int b = it.b, hk = it.hk, n = it.n, P = it.P, S = P + n;
    const int row0 = it.rb * (SHARED ? kSharedRows : 64) + (SHARED ? wave * 64 : 0);       // of the wavefront
    const Rows<QB> rows(p, hk, n, row0, l32);
    unsigned long long anc[QB] = {};
    if constexpr (!SHARED) {
        if (p.parent && !ancestors(p, it, lane, rows.token, anc)) continue;
    }
    const bool tree = !SHARED && p.parent;
    const int first_token = min(static_cast<int>(divide(row0, p.magic_group)), n - 1);
    const int last_token = W::last_token(p, n, it.rb);
    const int all_see = tree ? P : P + first_token + 1;    // slots that every row of the wavefront sees
    const int end = tree ? S : P + last_token + 1;         // slots that some row of the workgroup sees
    // Tiles of this segment: first; number.  Streams: up to the block's end, this wavefront's has every fourth.
    int tile0 = it.from, ntile = it.to - it.from;
    if constexpr (!SHARED) {
        tile0 = it.from * kWaveWgs + wave;
        const int past = min((end - 1) / kKeys + 1, it.to * kWaveWgs);
        ntile = tile0 < past ? (past - tile0 + kWaveWgs - 1) / kWaveWgs : 0;
    }

    // ---- tile fetch -------------------------------------------------------------------------
    const bool is_v = SHARED && wave >> 1;     // shared: wavefronts 0, 1 bring the halves of K tiles, 2, 3 those of V tiles
    const int half = SHARED ? wave & 1 : 0;
    const int lrow = lane / LPR, lpos = lane % LPR;
    constexpr int es = E4M3 ? 1 : 2;
    const uint32_t row_bytes = static_cast<uint32_t>(p.g.stride_t) * es;
    const int64_t head_off = (hk * p.g.stride_h + (PAGED ? 0 : b * p.g.stride_b)) * es;
    const int64_t scale_off = hk * p.s_sh + (PAGED ? 0 : b * p.s_sb);
    const int last_blk = (S - 1) >> 4;
    bool bad_block = false;
    // Block ids.  Shared: lane i has the block of this wavefront's half of tile i (mod 64); streams: lane 2i + x that of half x of tile i (mod 32).
    // The next 64 are on their way.
    constexpr int kIdTiles = SHARED ? 64 : 32;
    int ids = 0, ids_next = 0;
    auto request_ids = [&](int tile) __attribute__((always_inline)) {
        const int blk = SHARED ? (tile0 + tile + lane) * 2 + half : (tile0 + (tile + (lane >> 1)) * STEP) * 2 + (lane & 1);
        return p.g.block_table[static_cast<int64_t>(b) * p.g.max_blocks + min(blk, last_blk)];
    };
    auto take_ids = [&](int raw) __attribute__((always_inline)) {
        bad_block = bad_block || static_cast<uint32_t>(raw) >= static_cast<uint32_t>(p.g.num_blocks);
        ids = min(max(raw, 0), p.g.num_blocks - 1);
    };
    // Before the first request for a tile (K's, where a wavefront brings both): the ids of its 32 or 64 tiles.
    auto ids_for = [&](int tile) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            if (tile && (tile & (kIdTiles - 1)) == 0) {
                take_ids(ids_next);
                ids_next = request_ids(tile + kIdTiles);
            }
        }
    };
    // Where instruction i's rows of tile `tile` lie: element 0 of the 16-row half's first row, and the row of the half that is the last to exist
    // (rows behind it are replaced by that one: nothing past the request's slots is read).
    struct Half { const unsigned char *base, *sbase; int last; };
    auto half_of = [&](const unsigned char* cache, const unsigned char* scales, int tile, int x) __attribute__((always_inline)) {
        Half at;
        const int slot0 = (tile0 + tile * STEP) * kKeys + (SHARED ? half : x) * 16;
        if constexpr (PAGED) {
            const int blk = __builtin_amdgcn_readlane(ids, SHARED ? tile & 63 : (2 * tile + x) & 63);
            at.base = cache + head_off + blk * (p.g.stride_b * es);
            at.sbase = scales + scale_off + blk * p.s_sb;
            at.last = (slot0 >> 4) >= last_blk ? (S - 1) & 15 : 15;
        } else {
            const int from = min(slot0, (S - 1) & ~15);
            at.base = cache + head_off + static_cast<int64_t>(from) * row_bytes;
            at.sbase = scales + scale_off + from;
            at.last = S - 1 - from;
        }
        return at;
    };
    auto vswz = [](int r) { return D == 128 ? (r & 3) : ((r >> 1) & 1); };
    // (e4m3 streams: the rows of a store lie KI apart, so that their lowest bits go last)
    auto kswz = [](int r) { return E4M3 && !SHARED ? (r & (ROWG - 1)) / KI | (r & (KI - 1)) * (ROWG / KI) : r & (ROWG - 1); };
    // K row r in LDS: granule g at g ^ kswz(r); V row r: 64-byte chunk c at c ^ vswz(r), so that the operand reads meet no bank twice
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    unsigned char* const area = s_mem + (SHARED ? 0 : wave * kAreaBytes);
    constexpr int kVArea = SLOTS * kTileBytes;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)area + half * (kTileBytes / 2);
    // bf16: straight into LDS, 1 KB an instruction; a lane asks for the granule that belongs where it writes
    auto fetch = [&](bool v, int tile) __attribute__((always_inline)) {
        if (tile >= ntile) return;
        if (SHARED || !v) ids_for(tile);
        const uint32_t dst = lds0 + (v ? kVArea : 0) + (tile & (SLOTS - 1)) * kTileBytes;
#pragma unroll
        for (int x = 0; x < (SHARED ? 1 : 2); ++x) {
            const Half at = half_of(v ? p.v : p.k, nullptr, tile, x);
#pragma unroll
            for (int i = 0; i < KI / (SHARED ? 1 : 2); ++i) {
                const int r = i * RPI + lrow;
                const int swz = v ? vswz(r) << 2 : (x * 16 + half * 16 + r) & (ROWG - 1);
                dma16s(at.base, static_cast<uint32_t>(min(r, at.last)) * row_bytes + ((lpos ^ swz) << 4), dst + x * (kTileBytes / 2) + i * 1024);
            }
        }
    };
    // e4m3: through registers, where codes become bf16 (exact; the row's scale goes into the conversion).  Streams: a lane has KI rows beside one
    // another and their scales in one load, for a byte a lane takes the address unit as long as sixteen (four trees over 4864 slots 66.8 -> 64.3 us);
    // shared, where a wavefront brings a quarter as much, a row of every load instruction (1024, 1024 and 333 tokens 252 us, beside one another 276).
    constexpr bool BESIDE = !SHARED;
    struct Raw { u32x4 w[KI]; uint32_t e[BESIDE ? 1 : KI]; };
    const int my_row = BESIDE ? lrow * KI : lrow;
    const uint32_t my_off = (my_row & 15) * row_bytes + lpos * 16;
    auto load = [&](Raw& raw, bool v, int tile) __attribute__((always_inline)) {
        if (tile >= ntile) return;
        if (SHARED || !v) ids_for(tile);
        const unsigned char *const cache = v ? p.v : p.k, *const scales = v ? p.vs : p.ks;
        const Half low = half_of(cache, scales, tile, 0);
        if constexpr (!BESIDE) {
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                const uint32_t row = min(i * RPI + lrow, low.last);
                raw.w[i] = *reinterpret_cast<const u32x4*>(low.base + (row * row_bytes + lpos * 16));
                raw.e[i] = low.sbase[row];
            }
        } else {
            const Half high = half_of(cache, scales, tile, 1), at = hf ? high : low;
            if (__builtin_expect((tile0 + tile * STEP + 1) * kKeys <= S, 1)) {
#pragma unroll
                for (int i = 0; i < KI; ++i) raw.w[i] = *reinterpret_cast<const u32x4*>(at.base + static_cast<uint64_t>(i * row_bytes) + my_off);
                std::conditional_t<KI == 4, uint32_t, uint16_t> e;
                __builtin_memcpy(&e, at.sbase + (my_row & 15), sizeof e);
                raw.e[0] = e;
            } else {
                raw.e[0] = 0;
#pragma unroll
                for (int i = 0; i < KI; ++i) {
                    const uint32_t row = min((my_row & 15) + i, at.last);
                    raw.w[i] = *reinterpret_cast<const u32x4*>(at.base + (row * row_bytes + lpos * 16));
                    raw.e[0] |= static_cast<uint32_t>(at.sbase[row]) << (8 * i);
                }
            }
        }
    };
    auto store = [&](const Raw& raw, bool v, int tile) __attribute__((always_inline)) {
        unsigned char* const at = area + (v ? kVArea : 0) + (tile & (SLOTS - 1)) * kTileBytes;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int r = half * 16 + my_row + (BESIDE ? i : i * RPI);
            const int swz = v ? vswz(r) << 2 : kswz(r);
            const float scale = __uint_as_float(!BESIDE ? raw.e[i] << 23 : (i < 3 ? raw.e[0] << (23 - 8 * i) : raw.e[0] >> 1) & 0x7F800000u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 w;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    w[2 * x] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw.w[i][2 * h + x], scale, false));
                    w[2 * x + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw.w[i][2 * h + x], scale, true));
                }
                *reinterpret_cast<u32x4*>(at + r * ROWB + (((2 * lpos + h) ^ swz) << 4)) = w;
            }
        }
    };

    // ---- operands ---------------------------------------------------------------------------
    uint32_t kaddr[NC];                        // lane (key l32, half hf): dims 16c + 8hf .. +7; the query rows likewise
#pragma unroll
    for (int c = 0; c < NC; ++c) kaddr[c] = l32 * ROWB + (((2 * c + hf) ^ kswz(l32)) << 4);
    // va[t][x] element e is key 16x + 8 (e / 4) + 4 hf + e % 4, dim 32t + l32 (attn_streams.hip has the same reads)
    const int k0 = 4 * hf + ((lane & 15) >> 2);
    const uint32_t vaddr = k0 * ROWB + ((lane >> 4) & 1) * 32 + (lane & 3) * 8 + (vswz(k0) << 6);
    bf16x8 ka[NC], va[NT][2], qf[QB][NC];
    auto read_k = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) ka[c] = *reinterpret_cast<const bf16x8*>(area + (tile & (SLOTS - 1)) * kTileBytes + kaddr[c]);
    };
    auto read_v = [&](int t, int tile) __attribute__((always_inline)) {
        const uint32_t a = (vaddr ^ (t << 6)) + kVArea + (tile & (SLOTS - 1)) * kTileBytes;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const s16x4 lo = lds_read_tr16(area + a + (16 * x) * ROWB);
            const s16x4 hi = lds_read_tr16(area + a + (16 * x + 8) * ROWB);
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            va[t][x] = __builtin_bit_cast(bf16x8, both);
        }
    };
    // Softmax state of row 32 qb + l32 (both halves agree): reference maximum, the same times c2 (0 while no key was seen), the score that
    // moves it, and this lane's part of the sum of the row's weights.  acc[qb][t][i]: O^T row 32t + 8 (i / 4) + 4 hf + i % 4.
    float m_run[QB], mrc[QB], thr[QB], l_run[QB];
    f32x16 acc[QB][NT], s[QB];
    bf16x8 pf[QB][2];
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
    auto scores = [&](int qb, int c) __attribute__((always_inline)) {
        s[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[c], qf[qb][c], c ? s[qb] : zero, 0, 0, 0);
    };
    auto product = [&](int qb, int t) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x) acc[qb][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t][x], pf[qb][x], acc[qb][t], 0, 0, 0);
    };
    auto weights = [&](int qb) __attribute__((always_inline)) {    // exp2(S^T) rounded to bf16 is the other operand of the product with V
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
    // Masks and the reference maximum of one block of rows for tile j.  The reference only moves when some score lies 2^kTau above it (or on the
    // first visible key).
    auto settle = [&](int qb, int j) __attribute__((always_inline)) {
        const int slot0 = (tile0 + j * STEP) * kKeys;
        if (slot0 + kKeys > all_see) hide(s[qb], tree ? visible_tree(P, anc[qb], slot0) : visible_causal(P, rows.token[qb], slot0), hf);
        const float lmax = max16(s[qb]);
        if (__builtin_expect(__any(lmax > thr[qb]), 0)) {
            const float m_new = fmaxf(m_run[qb], fmaxf(lmax, other_half(lmax)));
            const float m_safe = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m_run[qb] == -INFINITY ? 1.f : fast_exp2((m_run[qb] - m_safe) * p.c2);
            m_run[qb] = m_new;
            thr[qb] = m_new + p.tau;
            mrc[qb] = m_safe * p.c2;
            l_run[qb] *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[qb][t] *= alpha;
        }
    };
    // What was written to LDS is there for all who read it: of a shared tile everybody (not __syncthreads(): it would wait for the loads that are
    // on their way), of a stream's own this wavefront, whose LDS operations are in order.
    auto meet = [&]() __attribute__((always_inline)) {
        if constexpr (SHARED) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("" ::: "memory");
    };
    // e4m3: set x of K holds tiles x (mod 2) and of V tiles x + 1 (mod 2); shared: what the wavefront brings, in raw_k
    Raw raw_k[SETS ? SETS : 1], raw_v[SETS && !SHARED ? SETS : 1];
    auto request_q = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const uint16_t* row = p.q + b * p.q_sb + rows.token[qb] * p.q_sn + rows.head[qb] * p.q_sh + 8 * hf;
#pragma unroll
            for (int c = 0; c < NC; ++c) qf[qb][c] = *reinterpret_cast<const bf16x8*>(row + 16 * c);
        }
    };
    auto mix = [&](auto products) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < decltype(products)::value; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // a matrix product
            __builtin_amdgcn_sched_group_barrier(0x402, 4, 0);      // and vector instructions in its shadow
        }
    };
    auto pin = [&](int qb) __attribute__((always_inline)) {          // (the weights are computed here, not behind a branch where they are used)
#pragma unroll
        for (int x = 0; x < 2; ++x) asm volatile("" : "+v"(pf[qb][x]));
    };
    // K of tile j + K_LEAD and V of tile j + V_LEAD on their way (e4m3: into LDS, and what follows from memory into the same registers)
    auto bring = [&](auto odd, int j) __attribute__((always_inline)) {
        constexpr int SET = SETS == 2 ? decltype(odd)::value : 0;
        if constexpr (!E4M3) {
            if constexpr (SHARED) {
                fetch(is_v, j + (is_v ? V_LEAD : K_LEAD));
            } else {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tiles that give way have been read
                fetch(true, j + V_LEAD);             // (before the ids change: V is a tile behind K)
                fetch(false, j + K_LEAD);
            }
        } else if constexpr (SHARED) {
            store(raw_k[SET], is_v, j + (is_v ? V_LEAD : K_LEAD));   // (past the last: what was there)
            load(raw_k[SET], is_v, j + (is_v ? V_LEAD : K_LEAD) + 2);
        } else {
            asm volatile("" ::: "memory");
            store(raw_v[SET], true, j + V_LEAD);
            load(raw_v[SET], true, j + V_LEAD + 2);        // (before the ids change)
            store(raw_k[SET], false, j + K_LEAD);
            load(raw_k[SET], false, j + K_LEAD + 2);
        }
    };
    auto land = [&](int j) __attribute__((always_inline)) {
        if constexpr (!E4M3) {
            // what the next tile needs has landed: all but what was asked for in the last two tiles (shared) or the last one
            if (j + K_LEAD < ntile) wait_vmcnt<2 * KI>();
            else wait_vmcnt<0>();
        }
        meet();
    };
    // One tile j in two halves, each with the weights of one block of rows beside the products of the other:
    //   weights of block 0 | block 1: V product of tile j - 1, scores of tile j      (behind their last use, V of j and K of j + 1 are read)
    //   weights of block 1 | block 0: V product of tile j, scores of tile j + 1
    // At its start s[0] holds block 0's scores of tile j, ka K of tile j, va V of tile j - 1.
    constexpr int FIRST = 1;                   // products that stand before a half's branches: the matrix pipe has them meanwhile
    auto step = [&](auto odd, auto next, int j) __attribute__((always_inline)) {
        constexpr bool NEXT = decltype(next)::value;
#pragma unroll
        for (int t = 0; t < FIRST; ++t) {
            product(1, t);
            read_v(t, j);
        }
        settle(0, j);
#pragma unroll
        for (int t = FIRST; t < NT; ++t) {
            product(1, t);
            read_v(t, j);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) scores(1, c);
        weights(0);
        if constexpr (NEXT) read_k(j + 1);
        mix(std::integral_constant<int, 2 * (NT - FIRST) + NC>{});
        pin(0);
        if constexpr (NEXT) bring(odd, j);
#pragma unroll
        for (int t = 0; t < FIRST; ++t) product(0, t);
        settle(1, j);
#pragma unroll
        for (int t = FIRST; t < NT; ++t) product(0, t);
        if constexpr (NEXT) {
#pragma unroll
            for (int c = 0; c < NC; ++c) scores(0, c);
        }
        weights(1);
        mix(std::integral_constant<int, 2 * (NT - FIRST) + (NEXT ? NC : 0)>{});
        pin(1);
        if constexpr (NEXT) land(j);
    };
    if (ntile > 0) {
        if constexpr (PAGED) {
            take_ids(request_ids(0));
            ids_next = request_ids(kIdTiles);
        }
        if constexpr (!E4M3 && SHARED) {
            fetch(is_v, 0);
            if (!is_v) fetch(false, 1);
            request_q();
            fetch(is_v, is_v ? 1 : 2);
            fetch(is_v, is_v ? 2 : 3);
            if (ntile > 3) wait_vmcnt<2 * KI>();
            else wait_vmcnt<0>();
        } else if constexpr (!E4M3) {
            fetch(false, 0);
            fetch(true, 0);
            fetch(false, 1);
            request_q();
            wait_vmcnt<0>();
        } else if constexpr (SHARED) {
            if (is_v) {
                load(raw_k[1], true, 0);
                load(raw_k[0], true, 1);
            } else {
                load(raw_k[0], false, 0);
                load(raw_k[1], false, 1);
            }
            request_q();
            if (is_v) {
                store(raw_k[1], true, 0);
                load(raw_k[1], true, 2);
            } else {
                store(raw_k[0], false, 0);
                store(raw_k[1], false, 1);
                load(raw_k[0], false, 2);
                load(raw_k[1], false, 3);
            }
        } else {
            load(raw_k[0], false, 0);
            load(raw_v[1], true, 0);
            load(raw_k[1], false, 1);
            load(raw_v[0], true, 1);
            request_q();
            store(raw_k[0], false, 0);
            load(raw_k[0], false, 2);
            store(raw_v[1], true, 0);
            load(raw_v[1], true, 2);
        }
        meet();
        read_k(0);
        // a later tile takes the place of K of the first
        if constexpr (SHARED) {
            meet();
        } else if constexpr (E4M3) {
            meet();
            store(raw_k[1], false, 1);
            load(raw_k[1], false, 3);
            meet();
        } else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(true, 1);
            fetch(false, 2);
        }
        // (the query rows stay in accumulation registers, which the products read as they are)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int c = 0; c < NC; ++c) asm volatile("" : "+a"(qf[qb][c]));
#pragma unroll
        for (int c = 0; c < NC; ++c) scores(0, c);
        // (there is no tile before the first: its product adds zeros)
#pragma unroll
        for (int x = 0; x < 2; ++x) pf[1][x] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) va[t][x] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, 1> odd;
        int j = 0;
        if constexpr (SETS == 2) {
            for (; j + 2 < ntile; j += 2) {
                step(even, std::true_type{}, j);
                step(odd, std::true_type{}, j + 1);
            }
            if (j + 1 < ntile) step(even, std::true_type{}, j++);
        } else {
            for (; j + 1 < ntile; ++j) step(even, std::true_type{}, j);
        }
        step(even, std::false_type{}, j);      // (the last tile brings nothing)
#pragma unroll
        for (int t = 0; t < NT; ++t) product(1, t);
    }
    if (PAGED && __any(bad_block) && lane == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_BLOCK);
    if constexpr (SHARED) {
        float M[QB], L[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            M[qb] = m_run[qb];
            L[qb] = l_run[qb] + other_half(l_run[qb]);
        }
        if (it.parts > 1 && !join(p, it, wave, lane, M, L, acc)) continue;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const float inv = 1.f / L[qb];
            uint16_t* const row = p.o + b * p.o_sb + rows.token[qb] * p.o_sn + rows.head[qb] * p.o_sh + 8 * hf;
#pragma unroll
            for (int t = 0; t < NT; ++t) store_block(acc[qb][t], inv, row + 32 * t, rows.real[qb]);
            if (rows.real[qb] && p.lse && hf == 0)
                p.lse[(static_cast<int64_t>(b) * p.H_q + rows.head[qb]) * p.N_max + rows.token[qb]] = M[qb] * p.scale + __log2f(L[qb]) * kLn2;
        }
    } else {
        finish<D, QB>(p, it, rows, acc, m_run, l_run, s_mem, s_m, s_l);
    }
    }
}

template <int D, bool E4M3, bool PAGED, bool SHARED>
__global__ __launch_bounds__(kWaveWgs * 64) __attribute__((amdgpu_waves_per_eu(1, D == 64 ? 2 : 1))) void chunk_rows_kernel(ChunkParams p) {
    attend64<D, E4M3, PAGED, SHARED>(p);
}

template <int D, bool SHARED>
void launch_as(const ChunkParams& p, bool e4m3, dim3 grid, hipStream_t stream) {
    auto* const kernel = e4m3 ? (p.g.block_table ? chunk_rows_kernel<D, true, true, SHARED> : chunk_rows_kernel<D, true, false, SHARED>)
                              : (p.g.block_table ? chunk_rows_kernel<D, false, true, SHARED> : chunk_rows_kernel<D, false, false, SHARED>);
    hipLaunchKernelGGL(kernel, grid, dim3(kWaveWgs * 64), 0, stream, p);
}

}  // namespace

void launch_chunk_rows(const ChunkParams& p, int D, bool e4m3, bool shared, unsigned workgroups, hipStream_t stream) {
    if (D == 128) shared ? launch_as<128, true>(p, e4m3, dim3(workgroups), stream) : launch_as<128, false>(p, e4m3, dim3(workgroups), stream);
    else shared ? launch_as<64, true>(p, e4m3, dim3(workgroups), stream) : launch_as<64, false>(p, e4m3, dim3(workgroups), stream);
}

}  // namespace specvlm
