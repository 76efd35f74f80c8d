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
#include "wave_ops.hpp"

namespace specvlm {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kSharedRows = 256;             // rows of a workgroup whose wavefronts share tiles
constexpr int kLeastRounds = 2;              // rounds a range of keys has at least: below that the meeting of the partial results costs more
constexpr int kMostColumns = 64;             // ranges of keys of one (request, KV head, row block)
constexpr int kMostPairs = 1024;             // (request, KV head, row block)s of a call whose keys are divided: more fill the chip by themselves
constexpr size_t kChunkCounterBytes = kMostPairs * kCounterStride * 4;     // tickets: a 128-byte line each

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
    int target;                              // workgroups to divide the keys among, 0: one range of keys for every (request, KV head, row block)
    int32_t* ws_cnt;                         // [pairs] arrival tickets, kCounterStride words apart, zero between calls
    unsigned char* ws_part;                  // [items] partial results, see merge_ranges()
};

// A workgroup's part of the call: column x of the c ranges of keys of (request, KV head, row block).
struct Item { int b, hk, rb, x, c, n, P, index; };

__device__ __forceinline__ int wave_sum_int(int x) {
    x = row_sum(x);
    return (__builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16)) + (__builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48));
}

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int x, int lane) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);           // row_shr:1, zero where there is none
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    const int a = __builtin_amdgcn_readlane(x, 15), b = a + __builtin_amdgcn_readlane(x, 31), c = b + __builtin_amdgcn_readlane(x, 47);
    return x + (lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? b : c);
}

__device__ __forceinline__ int length_error(const ChunkParams& p, int n, int P) {
    return n < 0 || n > p.N_max ? SPECVLM_ERR_BAD_NUM_NODES : P < 0 || P > p.g.capacity - n ? SPECVLM_ERR_BAD_LENGTH : 0;
}

// A 32 x 32 block of O^T (dims 8 (i / 4) + 4 (lane / 32) + i % 4 of the lane's row) times inv, as bf16; `to`: the row's dims 8 (lane / 32) ..
__device__ __forceinline__ void store_block(const f32x16& a, float inv, uint16_t* to, bool live) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {                          // 16 dims: registers 8u .. 8u + 7
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pack_bf16x2(a[8 * u + 2 * i] * inv, a[8 * u + 2 * i + 1] * inv);
        // the halves of the wavefront hold dims 0-3, 8-11 and 4-7, 12-15: the lower keeps 0-7, the upper 8-15
        const auto r0 = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
        const auto r1 = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
        if (live) *reinterpret_cast<u32x4*>(to + 16 * u) = u32x4{r0[0], r1[0], r0[1], r1[1]};
    }
}

// What a workgroup has to do, worked out by each from the lengths, which the host does not know.  Every range of keys of every (request, KV
// head, row block) gets about the same number of rounds (a round: a tile of every wavefront): the least `len` for which the ranges are no
// more than `target` workgroups (or one each).  Returns false where there is nothing to do.
template <int ROWS>
__device__ __forceinline__ bool find_item(const ChunkParams& p, int lane, Item& it) {
    typedef const __attribute__((address_space(4))) int32_t* const_i32;
    if (!p.target) {
        const uint32_t pair = blockIdx.x / static_cast<uint32_t>(p.row_blocks);
        it.rb = blockIdx.x - pair * p.row_blocks;
        it.b = pair / static_cast<uint32_t>(p.H_kv);
        it.hk = pair - it.b * p.H_kv;
        it.n = p.num_new ? ((const_i32)p.num_new)[it.b] : p.N_max;
        it.P = ((const_i32)p.prefix_len)[it.b];
        it.x = 0;
        it.c = 1;
        it.index = blockIdx.x;
        if (const int err = length_error(p, it.n, it.P)) {
            if (it.rb == 0 && it.hk == 0 && threadIdx.x == 0 && p.err_flag) atomicOr(p.err_flag, err);
            return false;
        }
        return it.rb * ROWS < p.group * it.n;
    }
    int n = 0, P = 0, rounds = 0, units = 0;               // of request b0 + lane
    auto look = [&](int b0, bool report) __attribute__((always_inline)) {
        const int b = b0 + lane;
        rounds = units = 0;
        if (b < p.B) {
            n = p.num_new ? p.num_new[b] : p.N_max;
            P = p.prefix_len[b];
            if (const int err = length_error(p, n, P)) {
                if (report && p.err_flag) atomicOr(p.err_flag, err);
            } else if (n) {
                rounds = static_cast<int>((static_cast<uint32_t>(P + n - 1) + kSharesRound) / kSharesRound);
                units = (p.group * n + ROWS - 1) / ROWS * p.H_kv;
            }
        }
    };
    // (more than 64 requests: looked at 64 at a time, again for every pass)
    const bool first = blockIdx.x == 0 && threadIdx.x < 64;
    float total = 0.f;
    int pairs = 0, longest = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        look(b0, first);
        total += wave_sum(static_cast<float>(rounds) * units);
        pairs += wave_sum_int(units);
        longest = max(longest, static_cast<int>(wave_max(static_cast<float>(rounds))));      // (up to 2^24: exact)
    }
    const int most = max(p.target, pairs);
    int len = max(static_cast<int>(ceilf(total / p.target)), max(kLeastRounds, (longest + kMostColumns - 1) / kMostColumns));
    int all;
    for (;; len += 1 + (len >> 4)) {
        all = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            if (p.B > 64) look(b0, false);
            all += wave_sum_int(units * ((rounds + len - 1) / len));
        }
        if (all <= most || len >= longest) break;
    }
    // every XCD has a contiguous range of the items, so that the row blocks of a head's keys share an L2
    const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3, share = all >> 3, more = all & 7;
    if (place >= share + (xcd < more)) return false;
    it.index = xcd * share + min(xcd, more) + place;
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64) look(b0, false);
        const int mine = units * ((rounds + len - 1) / len), upto = before + wave_scan(mine, lane);
        const unsigned long long here = __ballot(it.index < upto);
        if (here) {
            const int at = __builtin_ctzll(here);
            it.b = b0 + at;
            it.n = __builtin_amdgcn_readlane(n, at);
            it.P = __builtin_amdgcn_readlane(P, at);
            const uint32_t local = it.index - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
            const uint32_t units_of = __builtin_amdgcn_readlane(units, at), blocks = units_of / static_cast<uint32_t>(p.H_kv);
            it.c = (__builtin_amdgcn_readlane(rounds, at) + len - 1) / len;
            it.x = local / units_of;
            const uint32_t rest = local - it.x * units_of;
            it.hk = rest / blocks;
            it.rb = rest - it.hk * blocks;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

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

// Items between two ranges of keys of one (request, KV head, row block): find_item() puts the request's (head, block) pairs in between.
__device__ __forceinline__ int step_of(const ChunkParams& p, const Item& it, int rows) { return (p.group * it.n + rows - 1) / rows * p.H_kv; }

// The partial results of an item's ranges of keys, in their order, by the 256 threads of the workgroup that came last.  A unit is four head
// dims of a row; where the block has few rows, threads share a unit's ranges and meet in LDS.
template <int D, int ROWS>
__device__ __forceinline__ void merge_ranges(const ChunkParams& p, const Item& it, const unsigned char* parts, int64_t part_step, unsigned char* lds) {
    constexpr int kCoherent = 16;                          // device-coherent (sc1) loads, which the compiler counts
    constexpr int NT = D / 32;
    const int tid = threadIdx.x, row0 = it.rb * ROWS;
    const int rows = min(ROWS, p.group * it.n - row0);
    float* const s_w = reinterpret_cast<float*>(lds);      // [rows][c] maxima, then weights
    float* const s_inv = s_w + ROWS * kMostColumns;        // [rows]
    float* const s_sum = s_inv + ROWS;                     // [256][4]
    auto load = [&](int64_t off, auto wide) __attribute__((always_inline)) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(parts), 0, 0x7FFFFFFF, 0x00027000);
        if constexpr (decltype(wide)::value) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, static_cast<int>(off), 0, kCoherent);
        else return __builtin_amdgcn_raw_buffer_load_b64(rsrc, static_cast<int>(off), 0, kCoherent);
    };
    // eight threads a row: its maximum over the ranges, their weights, the sum
    for (int r = tid >> 3; r < rows; r += 32) {
        const int i0 = tid & 7;
        float m[kMostColumns / 8], l[kMostColumns / 8], M = -INFINITY, L = 0.f;
#pragma unroll
        for (int k = 0; k < kMostColumns / 8; ++k) {
            m[k] = -INFINITY;
            l[k] = 0.f;
            if (i0 + 8 * k < it.c) {
                const u32x2 ml = load((i0 + 8 * k) * part_step + ROWS * D * 4 + r * 8, std::false_type{});
                m[k] = __uint_as_float(ml[0]);
                l[k] = __uint_as_float(ml[1]);
            }
        }
#pragma unroll
        for (int k = 0; k < kMostColumns / 8; ++k) M = __builtin_elementwise_maximum(M, m[k]);
        M = __builtin_elementwise_maximum(M, dpp<0x141>(M));
        M = __builtin_elementwise_maximum(M, dpp<0x4E>(M));
        M = __builtin_elementwise_maximum(M, dpp<0xB1>(M));
        const float m_safe = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < kMostColumns / 8; ++k) {
            const float w = fast_exp2((m[k] - m_safe) * p.c2);
            L += l[k] * w;
            if (i0 + 8 * k < it.c) s_w[r * kMostColumns + i0 + 8 * k] = w;
        }
        L += dpp<0x141>(L);
        L += dpp<0x4E>(L);
        L += dpp<0xB1>(L);
        if (i0 == 0) {
            s_inv[r] = 1.f / L;
            if (p.lse) {
                const int token = divide(row0 + r, p.magic_group);
                const int h = it.hk * p.group + row0 + r - token * p.group;
                p.lse[(static_cast<int64_t>(it.b) * p.H_q + h) * p.N_max + token] = M * p.scale + __log2f(L) * kLn2;
            }
        }
    }
    __syncthreads();
    // Units of 32 rows at a time: (dims 32t + 8u + 4hf .., row), rows innermost, so that threads beside one another read beside one another.
    for (int q = 0; q < ROWS; q += 32) {
        const int here = min(32, rows - q);
        if (here <= 0) break;
        const int units = here * (D / 4);
        int share = 1;                                     // threads of a unit
        while (units * share * 2 <= 256) share *= 2;
        for (int first = 0; first < units; first += 256 / share) {
            const int part = tid * share / 256;            // (share is a power of two)
            const int unit = first + tid - part * (256 / share);
            const bool mine = unit < units;
            const int dims = mine ? unit / here : 0, r = mine ? unit - dims * here : 0;
            const int hf = dims & 1, block = q / 32 * NT + (dims >> 3), u = (dims >> 1) & 3;
            const int off = ((block * 4 + u) * 64 + hf * 32 + r) * 16;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            constexpr int BATCH = 8;
            for (int i = part; i < it.c; i += share * BATCH) {
                u32x4 x[BATCH];
#pragma unroll
                for (int k = 0; k < BATCH; ++k) x[k] = load(min(i + k * share, it.c - 1) * part_step + off, std::true_type{});
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const float w = i + k * share < it.c ? s_w[(q + r) * kMostColumns + i + k * share] : 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = fmaf(__uint_as_float(x[k][e]), w, sum[e]);
                }
            }
            if (share > 1) {
                __syncthreads();
                reinterpret_cast<f32x4*>(s_sum)[tid] = sum;
                __syncthreads();
                if (part == 0)
                    for (int k = 1; k < share; ++k) {
                        const f32x4 other = reinterpret_cast<const f32x4*>(s_sum)[tid + k * (256 / share)];
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[e] += other[e];
                    }
            }
            if (mine && part == 0) {
                const float inv = s_inv[q + r];
                const int token = divide(row0 + q + r, p.magic_group);
                const int h = it.hk * p.group + row0 + q + r - token * p.group;
                uint16_t* const to = p.o + it.b * p.o_sb + token * p.o_sn + h * p.o_sh + dims * 4;
                *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
            }
        }
    }
}

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
    constexpr bool LEAN = QB == 1;             // little in registers, so that two workgroups fit a compute unit
    constexpr int NB = QB * NT;                // (32 rows, 32 dims) blocks of the result
    constexpr int OWN = NB >= kWaveWgs ? NB / kWaveWgs : 1;
    constexpr int kMergeBytes = NB * 3 * 4096;
    constexpr int kLds = kMergeBytes > kWaveWgs * 2 * kTileBytes ? kMergeBytes : kWaveWgs * 2 * kTileBytes;

    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[kLds];
    __shared__ float s_m[kWaveWgs][ROWS];
    __shared__ float s_l[kWaveWgs][ROWS];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;
    Item it;
    if (!find_item<ROWS>(p, lane, it)) return;
    const int b = it.b, hk = it.hk, n = it.n, P = it.P, S = P + n;
    const int row0 = it.rb * ROWS;

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
            if (it.rb == 0 && it.hk == 0 && it.x == 0 && tid == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_PARENT);
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
    // Tiles of this range of keys: whole rounds of the request, up to the block's end; this wavefront's stream has every fourth.
    const int rounds = static_cast<int>((static_cast<uint32_t>(S - 1) + kSharesRound) / kSharesRound);
    const int first_round = it.x * rounds / it.c, next_round = (it.x + 1) * rounds / it.c;
    const int ntile = min((end - 1) / kKeys + 1, next_round * kWaveWgs);
    const int tile0 = first_round * kWaveWgs + wave;
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
        if constexpr (!LEAN) {
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
    }
    // Masks and reference maxima of the tile of slot0, whose scores s and their maxima lmax are.
    auto settle = [&](int slot0) __attribute__((always_inline)) {
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
    };
    // One tile.  At its start s holds its scores and lmax their maxima; va its V operands, ka the next tile's K operands; vraw and kraw V of the
    // next tile and K of the one after it.
    auto step = [&](auto next, int j) __attribute__((always_inline)) {
        constexpr bool NEXT = decltype(next)::value;
        settle((tile0 + j * kWaveWgs) * kKeys);
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
    // The same without anything of the next tile in registers but what has been loaded of it: two workgroups fit a compute unit.
    auto lean_step = [&](int j) __attribute__((always_inline)) {
        read_k();
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) { scores(s[qb], qb); lmax[qb] = max16(s[qb]); }
        settle((tile0 + j * kWaveWgs) * kKeys);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) weights(qb);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            read_v(t);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) acc[qb][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t][x], pf[qb][x], acc[qb][t], 0, 0, 0);
        }
        wave_order();
        if (j + 1 < my_tiles) {
            store(kraw, std::false_type{});
            store(vraw, std::true_type{});
            if (j + 2 < my_tiles) {
                if (PAGED && ((j + 2) & 31) == 0) {
                    take_ids(ids_next);
                    if (j + 2 + 32 < my_tiles) ids_next = request_ids(j + 2 + 32);
                }
                load(kraw, p.k, p.ks, j + 2);
                load(vraw, p.v, p.vs, j + 2);
            }
            wave_order();
        }
    };
    if constexpr (LEAN) {
        for (int j = 0; j < my_tiles; ++j) lean_step(j);
    } else {
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
    float M[OWN], L[OWN];
    if (wave < NB / OWN) {
#pragma unroll
        for (int e = 0; e < OWN; ++e) {
            const int block = wave * OWN + e;
            const int qb = block / NT;
            float m[kWaveWgs], w[kWaveWgs];
#pragma unroll
            for (int x = 0; x < kWaveWgs; ++x) m[x] = s_m[x][qb * 32 + l32];
            M[e] = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
            const float m_safe = M[e] == -INFINITY ? 0.f : M[e];
            L[e] = 0.f;
#pragma unroll
            for (int x = 0; x < kWaveWgs; ++x) {           // (in this order in every owner of the rows)
                w[x] = fast_exp2((m[x] - m_safe) * p.c2);
                L[e] += s_l[x][qb * 32 + l32] * w[x];
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
        }
    }
    if (it.c == 1) {
        if (wave < NB / OWN) {
#pragma unroll
            for (int e = 0; e < OWN; ++e) {
                const int block = wave * OWN + e, qb = block / NT, t = block % NT;
                const bool live = qb ? real[QB - 1] : real[0];
                const int tok = qb ? token[QB - 1] : token[0], h = qb ? head[QB - 1] : head[0];
                const float inv = 1.f / L[e];
                store_block(out[e], inv, p.o + b * p.o_sb + tok * p.o_sn + h * p.o_sh + 32 * t + 8 * hf, live);
                if (live && p.lse && hf == 0 && t == 0) p.lse[(static_cast<int64_t>(b) * p.H_q + h) * p.N_max + tok] = M[e] * p.scale + __log2f(L[e]) * kLn2;
            }
        }
        return;
    }
    // ---- partial result of this range of keys, and the merge by the last of them -----------------
    // A partial: [block][4][64 lanes] vectors of four fp32 (the accumulators as they are, rows of the group that exist only), then a (maximum,
    // sum) pair per row.
    constexpr int kPartBytes = ROWS * (D + 2) * 4;
    unsigned char* const parts = p.ws_part + static_cast<int64_t>(it.index - it.x * step_of(p, it, ROWS)) * kPartBytes;
    const int64_t part_step = static_cast<int64_t>(step_of(p, it, ROWS)) * kPartBytes;
    if (wave < NB / OWN) {
        unsigned char* const mine = parts + it.x * part_step;
#pragma unroll
        for (int e = 0; e < OWN; ++e) {
            const int block = wave * OWN + e, qb = block / NT;
            if (!(qb ? real[QB - 1] : real[0])) continue;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(out[e][4 * u + i]);
                store16_coherent(mine + ((block * 4 + u) * 64 + lane) * 16, x);
            }
            if (block % NT == 0 && hf == 0)
                store8_coherent(mine + ROWS * D * 4 + (qb * 32 + l32) * 8, u32x2{__float_as_uint(M[e]), __float_as_uint(L[e])});
        }
    }
    wait_vmcnt<0>();
    __syncthreads();                                       // (LDS is free as well)
    int* const s_last = reinterpret_cast<int*>(s_m);
    if (tid == 0) {
        int32_t* const cnt = p.ws_cnt + ((static_cast<int64_t>(b) * p.H_kv + hk) * p.row_blocks + it.rb) * kCounterStride;
        const int ticket = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = ticket == it.c - 1;
        if (last) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = last;
    }
    __syncthreads();
    if (!*s_last) return;
    asm volatile("" ::: "memory");
    merge_ranges<D, ROWS>(p, it, parts, part_step, s_mem);
}

// 256 rows a workgroup: every wavefront has 64 rows of its own, and all four share each tile of 32 keys.
template <int D, bool E4M3, bool PAGED>
__device__ __forceinline__ void attend_rows(const ChunkParams& p) {
    constexpr int QB = 2;
    constexpr int NC = D / 16, NT = D / 32, ROWG = D / 8, ROWB = D * 2;
    constexpr int LPR = (E4M3 ? D : 2 * D) / 16;   // lanes per cached row
    constexpr int RPI = 64 / LPR;              // rows per load instruction
    constexpr int KI = 16 / RPI;               // load instructions of a wavefront per tile: 16 rows of K or of V
    constexpr int kTileBytes = kKeys * ROWB;

    __shared__ __attribute__((aligned(1024))) unsigned char s_mem[4 * kTileBytes];      // two K tiles, two V tiles

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;
    // the blocks with the most keys first; the blocks of a head's keys on one XCD where the number of heads allows it
    const uint32_t pairs = static_cast<uint32_t>(p.B) * p.H_kv;
    const uint32_t level = blockIdx.x / pairs, pair = blockIdx.x - level * pairs;
    const int rb = p.row_blocks - 1 - level;
    const int b = pair / static_cast<uint32_t>(p.H_kv), hk = pair - b * p.H_kv;
    typedef const __attribute__((address_space(4))) int32_t* const_i32;
    const int n = p.num_new ? ((const_i32)p.num_new)[b] : p.N_max;
    const int P = ((const_i32)p.prefix_len)[b];
    if (const int err = length_error(p, n, P)) {
        if (rb == 0 && hk == 0 && tid == 0 && p.err_flag) atomicOr(p.err_flag, err);
        return;
    }
    const int row0 = rb * kSharedRows;
    if (row0 >= p.group * n) return;
    const int S = P + n;

    int token[QB], head[QB];
    bool real[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int R = row0 + wave * 64 + qb * 32 + l32;
        token[qb] = divide(R, p.magic_group);
        head[qb] = hk * p.group + R - token[qb] * p.group;
        real[qb] = token[qb] < n;
        if (!real[qb]) { token[qb] = n - 1; head[qb] = hk * p.group; }
    }
    const int first_token = min(static_cast<int>(divide(row0 + wave * 64, p.magic_group)), n - 1);
    const int last_token = min(static_cast<int>(divide(row0 + kSharedRows - 1, p.magic_group)), n - 1);
    const int all_see = P + first_token + 1;   // slots that every row of the wavefront sees
    const int ntile = (P + last_token) / kKeys + 1;

    // ---- tile fetch: wavefronts 0, 1 bring the halves of K tiles, 2, 3 those of V tiles ---------
    const bool is_v = wave >> 1;
    const int half = wave & 1;
    const int lrow = lane / LPR, lpos = lane % LPR;
    const int es = E4M3 ? 1 : 2;
    const uint32_t row_bytes = static_cast<uint32_t>(p.g.stride_t) * es;
    const unsigned char* const cache = (is_v ? p.v : p.k) + (hk * p.g.stride_h + (PAGED ? 0 : b * p.g.stride_b)) * es;
    const unsigned char* const scales = (is_v ? p.vs : p.ks) + (hk * p.s_sh + (PAGED ? 0 : b * p.s_sb));
    const int last_blk = (S - 1) >> 4;
    bool bad_block = false;
    int ids = 0, ids_next = 0;                 // lane i: the block of this half of tile i (mod 64), and of the next 64 tiles
    auto request_ids = [&](int tile) __attribute__((always_inline)) {
        return p.g.block_table[static_cast<int64_t>(b) * p.g.max_blocks + min((tile + lane) * 2 + half, last_blk)];
    };
    auto take_ids = [&](int raw) __attribute__((always_inline)) {
        bad_block = bad_block || static_cast<uint32_t>(raw) >= static_cast<uint32_t>(p.g.num_blocks);
        ids = min(max(raw, 0), p.g.num_blocks - 1);
    };
    struct Raw { u32x4 w[KI]; uint32_t e[E4M3 ? KI : 1]; };
    // Tiles are asked for in order, 0, 1, 2 ..; one past the last is not.
    auto load = [&](Raw& raw, int tile) __attribute__((always_inline)) {
        if (tile >= ntile) return;
        const int slot0 = tile * kKeys + half * 16;
        const unsigned char *base, *sbase;
        int last;                              // row of the half that is the last to exist (or before it, then some row of the tile again)
        if constexpr (PAGED) {
            if (tile && (tile & 63) == 0) {
                take_ids(ids_next);
                ids_next = request_ids(tile + 64);
            }
            const int blk = __builtin_amdgcn_readlane(ids, tile & 63);
            base = cache + blk * (p.g.stride_b * es);
            sbase = scales + blk * p.s_sb;
            last = (slot0 >> 4) >= last_blk ? (S - 1) & 15 : 15;
        } else {
            const int from = min(slot0, (S - 1) & ~15);
            base = cache + static_cast<int64_t>(from) * row_bytes;
            sbase = scales + from;
            last = S - 1 - from;
        }
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const uint32_t row = min(i * RPI + lrow, last);
            raw.w[i] = *reinterpret_cast<const u32x4*>(base + (row * row_bytes + lpos * 16));
            if constexpr (E4M3) raw.e[i] = sbase[row];
        }
    };
    auto vswz = [](int r) { return D == 128 ? (r & 3) : ((r >> 1) & 1); };
    uint32_t to[KI][E4M3 ? 2 : 1];             // where this lane's granules go in a tile
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        const int r = half * 16 + i * RPI + lrow;
        const int swz = is_v ? vswz(r) << 2 : r & (ROWG - 1);
#pragma unroll
        for (int h = 0; h < (E4M3 ? 2 : 1); ++h) to[i][h] = (is_v ? 2 * kTileBytes : 0) + r * ROWB + (((E4M3 ? 2 * lpos + h : lpos) ^ swz) << 4);
    }
    auto store = [&](const Raw& raw, int slot) __attribute__((always_inline)) {
        unsigned char* const tile = s_mem + slot * kTileBytes;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
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
                    *reinterpret_cast<u32x4*>(tile + to[i][h]) = w;
                }
            } else {
                *reinterpret_cast<u32x4*>(tile + to[i][0]) = raw.w[i];
            }
        }
    };

    // ---- operands, as in attend() -----------------------------------------------------------
    uint32_t kaddr[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) kaddr[c] = l32 * ROWB + (((2 * c + hf) ^ (l32 & (ROWG - 1))) << 4);
    const int k0 = 4 * hf + ((lane & 15) >> 2);
    const uint32_t vaddr = 2 * kTileBytes + k0 * ROWB + ((lane >> 4) & 1) * 32 + (lane & 3) * 8 + (vswz(k0) << 6);
    bf16x8 ka[NC], va[NT][2], qf[QB][NC];
    auto read_k = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) ka[c] = *reinterpret_cast<const bf16x8*>(s_mem + slot * kTileBytes + kaddr[c]);
    };
    auto read_v = [&](int t, int slot) __attribute__((always_inline)) {
        const uint32_t a = (vaddr ^ (t << 6)) + slot * kTileBytes;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const s16x4 lo = lds_read_tr16(s_mem + a + (16 * x) * ROWB);
            const s16x4 hi = lds_read_tr16(s_mem + a + (16 * x + 8) * ROWB);
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            va[t][x] = __builtin_bit_cast(bf16x8, both);
        }
    };
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
    auto settle = [&](int slot0) __attribute__((always_inline)) {
        if (slot0 + kKeys > all_see) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const int seen = P + token[qb] + 1 - slot0;
                const uint32_t visible = (seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u) >> (4 * hf);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t on = static_cast<uint32_t>(static_cast<int32_t>(visible << (31 - (8 * (i >> 2) + (i & 3)))) >> 31);
                    s[qb][i] = __uint_as_float((on & __float_as_uint(s[qb][i])) | (~on & 0xFF800000u));
                }
                lmax[qb] = max16(s[qb]);
            }
        }
        if (__builtin_expect(__any((lmax[0] > thr[0]) | (lmax[1] > thr[1])), 0)) {
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
    };
    auto meet = [&]() __attribute__((always_inline)) {     // (not __syncthreads(): it would wait for the loads that are on their way)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // K tiles are two ahead of the one whose weights are computed, V tiles one.  raw[x] of a wavefront that brings K holds tiles x (mod 2), of one
    // that brings V tiles x + 1 (mod 2).
    Raw raw[2];
    if constexpr (PAGED) {
        take_ids(request_ids(0));
        ids_next = request_ids(64);
    }
    if (is_v) {
        load(raw[1], 0);
        load(raw[0], 1);
    } else {
        load(raw[0], 0);
        load(raw[1], 1);
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const uint16_t* row = p.q + b * p.q_sb + token[qb] * p.q_sn + head[qb] * p.q_sh + 8 * hf;
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[qb][c] = *reinterpret_cast<const bf16x8*>(row + 16 * c);
    }
    if (is_v) {
        store(raw[1], 0);
        load(raw[1], 2);
    } else {
        store(raw[0], 0);
        store(raw[1], 1);
        load(raw[0], 2);
        load(raw[1], 3);
    }
    meet();
    read_k(0);
#pragma unroll
    for (int t = 0; t < NT; ++t) read_v(t, 0);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) scores(s[qb], qb);
    read_k(1);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) lmax[qb] = max16(s[qb]);
    // One tile: s holds its scores, lmax their maxima, va its V operands, ka the next tile's K operands.
    auto step = [&](auto odd, auto next, int j) __attribute__((always_inline)) {
        constexpr int ODD = decltype(odd)::value;
        constexpr bool NEXT = decltype(next)::value;
        settle(j * kKeys);
        if constexpr (NEXT) {
            store(raw[ODD], is_v ? ODD ^ 1 : ODD);         // K of tile j + 2 (none: what was there), V of tile j + 1
            load(raw[ODD], j + (is_v ? 3 : 4));
            scores(s_next[0], 0);
        }
        weights(0);
        if constexpr (NEXT) scores(s_next[1], 1);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) acc[0][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t][x], pf[0][x], acc[0][t], 0, 0, 0);
        weights(1);
        if constexpr (NEXT) {
            meet();
            read_k(ODD);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int x = 0; x < 2; ++x) acc[1][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t][x], pf[1][x], acc[1][t], 0, 0, 0);
            if constexpr (NEXT) read_v(t, ODD ^ 1);
        }
        if constexpr (NEXT) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) { s[qb] = s_next[qb]; lmax[qb] = max16(s[qb]); }
        }
    };
    {
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, 1> odd;
        int j = 0;
        for (; j + 2 < ntile; j += 2) {
            step(even, std::true_type{}, j);
            step(odd, std::true_type{}, j + 1);
        }
        if (j + 1 < ntile) step(even, std::true_type{}, j++);
        step(even, std::false_type{}, j);                  // (nothing of it depends on the tile's parity)
    }
    if (PAGED && __any(bad_block) && lane == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_BLOCK);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float L = l_run[qb] + other_half(l_run[qb]);
        const float inv = 1.f / L;
        uint16_t* const row = p.o + b * p.o_sb + token[qb] * p.o_sn + head[qb] * p.o_sh + 8 * hf;
#pragma unroll
        for (int t = 0; t < NT; ++t) store_block(acc[qb][t], inv, row + 32 * t, real[qb]);
        if (real[qb] && p.lse && hf == 0) p.lse[(static_cast<int64_t>(b) * p.H_q + head[qb]) * p.N_max + token[qb]] = m_run[qb] * p.scale + __log2f(L) * kLn2;
    }
}

template <int D, bool E4M3, bool PAGED>
__global__ __launch_bounds__(kWaveWgs * 64) __attribute__((amdgpu_waves_per_eu(1, 1))) void chunk_attn_rows_kernel(ChunkParams p) {
    attend_rows<D, E4M3, PAGED>(p);
}

template <int D, int QB, bool E4M3, bool PAGED>
__global__ __launch_bounds__(kWaveWgs * 64) __attribute__((amdgpu_waves_per_eu(QB == 1 ? 2 : 1, QB == 1 ? 2 : 1))) void chunk_attn_kernel(ChunkParams p) {
    attend<D, QB, E4M3, PAGED>(p);
}

template <int D, int QB>
void launch_as(const ChunkParams& p, bool e4m3, dim3 grid, hipStream_t stream) {
    auto* const kernel = e4m3 ? (p.g.block_table ? chunk_attn_kernel<D, QB, true, true> : chunk_attn_kernel<D, QB, true, false>)
                              : (p.g.block_table ? chunk_attn_kernel<D, QB, false, true> : chunk_attn_kernel<D, QB, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kWaveWgs * 64), 0, stream, p);
}


template <int D>
void launch_rows(const ChunkParams& p, bool e4m3, dim3 grid, hipStream_t stream) {
    auto* const kernel = e4m3 ? (p.g.block_table ? chunk_attn_rows_kernel<D, true, true> : chunk_attn_rows_kernel<D, true, false>)
                              : (p.g.block_table ? chunk_attn_rows_kernel<D, false, true> : chunk_attn_rows_kernel<D, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kWaveWgs * 64), 0, stream, p);
}

struct ChunkPlan {
    int qb;                  // blocks of 32 rows per workgroup; 0: wavefronts with 64 rows each share the tiles
    int row_blocks, target;  // see ChunkParams
    int64_t workgroups;
    size_t bytes;            // workspace
};

// How a call is divided, with `bytes` of workspace.
ChunkPlan chunk_plan(const specvlm_attn_desc& d, bool tree, size_t bytes) {
    ChunkPlan plan;
    const int64_t rows = static_cast<int64_t>(d.H_q / d.H_kv) * d.N_max;
    plan.qb = rows <= 32 ? 1 : rows <= 128 || tree ? 2 : 0;
    const int block = plan.qb ? 32 * plan.qb : kSharedRows;
    plan.row_blocks = static_cast<int>((rows + block - 1) / block);
    const int64_t pairs = static_cast<int64_t>(d.B) * d.H_kv * plan.row_blocks;
    plan.target = 0;
    plan.workgroups = pairs;
    plan.bytes = 0;
    const int64_t capacity = d.paged ? static_cast<int64_t>(d.max_blocks_per_req) * SPECVLM_PAGE_SIZE : d.kv_capacity;
    const int64_t rounds = (capacity + kSharesRound - 1) / kSharesRound;
    if (!plan.qb || d.num_splits == 1 || pairs > kMostPairs || rounds <= kLeastRounds || bytes < kChunkCounterBytes) return plan;
    const int64_t part = static_cast<int64_t>(32) * plan.qb * (d.D + 2) * 4;
    const int64_t slots = (bytes - kChunkCounterBytes) / part;
    const int64_t want = std::max<int64_t>(plan.qb == 1 ? 512 : 256, pairs);
    const int64_t most = std::min(want, pairs * std::min<int64_t>(kMostColumns, (rounds + kLeastRounds - 1) / kLeastRounds));
    if (slots < pairs) return plan;
    plan.target = static_cast<int>(std::min(most, slots));
    plan.workgroups = (plan.target + 7) / 8 * 8;
    plan.bytes = kChunkCounterBytes + plan.target * part;
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
    p.ws_cnt = static_cast<int32_t*>(a.workspace);
    p.ws_part = static_cast<unsigned char*>(a.workspace) + kChunkCounterBytes;
    const dim3 grid(static_cast<unsigned>(plan.workgroups));
    if (!plan.qb) d.D == 128 ? launch_rows<128>(p, a.scales != nullptr, grid, a.stream) : launch_rows<64>(p, a.scales != nullptr, grid, a.stream);
    else if (d.D == 128) plan.qb == 1 ? launch_as<128, 1>(p, a.scales != nullptr, grid, a.stream) : launch_as<128, 2>(p, a.scales != nullptr, grid, a.stream);
    else plan.qb == 1 ? launch_as<64, 1>(p, a.scales != nullptr, grid, a.stream) : launch_as<64, 2>(p, a.scales != nullptr, grid, a.stream);
    return check_launch();
}

}  // namespace specvlm
