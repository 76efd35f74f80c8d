// Shared by the kernels of the attention of token chunks: parameters, the division of a call among workgroups, the merge of ranges of keys.
#pragma once
#include <type_traits>

#include "attn_common.hpp"
#include "attn_rows.hpp"
#include "chunk_share.hpp"
#include "wave_ops.hpp"

namespace specvlm {

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
    int target, places;                      // workgroups to divide the call among at most (0: one for every (request, KV head, row block)), and at once
    int32_t* ws_cnt;                         // [items] arrival tickets, kCounterStride words apart, zero between calls
    unsigned char* ws_part;                  // two partial results a workgroup
};

// The kernels with 64 rows a wavefront (chunk_rows.hip); `shared`: 256 rows a workgroup.
void launch_chunk_rows(const ChunkParams& p, int D, bool e4m3, bool shared, unsigned workgroups, hipStream_t stream);

constexpr int kSharedRows = 256;             // rows of a workgroup whose wavefronts share tiles
static_assert(kChunkKeys == kKeys, "keys per tile");
constexpr int kLeastRounds = 2;              // rounds a part has at least where the keys of an item are divided
constexpr int kMostPairs = 4096;             // (request, KV head, row block)s of a call that is divided: more even out by themselves
constexpr size_t kChunkCounterBytes = kMostPairs * kCounterStride * 4;     // tickets: a 128-byte line each
constexpr int part_bytes(int rows, int D) { return rows * (D + 2) * 4; }   // accumulators, then a (maximum, sum) pair a row, in fp32

namespace {        // (device functions of each file's kernels)

typedef float f32x16 __attribute__((ext_vector_type(16)));


__device__ __forceinline__ int wave_sum_int(int x) {
    x = row_sum(x);
    return (__builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16)) + (__builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48));
}

static_assert(SPECVLM_ERR_BAD_NUM_NODES == 2 && SPECVLM_ERR_BAD_LENGTH == 4, "chunk_length_error()");
__device__ __forceinline__ int length_error(const ChunkParams& p, int n, int P) { return chunk_length_error(n, P, p.N_max, p.g.capacity); }

// The greatest of sixteen scores, NaN where one is.
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

// The same item in scalar registers.
__device__ __forceinline__ Item uniform(const Item& x) {
    return Item{u(x.b), u(x.hk), u(x.rb), u(x.n), u(x.P), u(x.from), u(x.to), u(x.steps), u(x.part), u(x.parts), u(x.first)};
}

// The thread's number, anew: what a segment's code derives from it is worked out there and not kept in registers from one segment to the next.
__device__ __forceinline__ int this_thread() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
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

// Calls whose workgroups have key streams: one segment each, worked out by every workgroup from the lengths.  All parts of all items get about
// the same number of rounds (a round: a tile of every stream, 128 keys).  Returns false where there is nothing to do.
// (Equal stretches as in Share leave no workgroup with more than the mean, but most with the end of one item and the beginning of the next, and
// each segment is a chain of latencies: one token over 768 keys of 32 heads 10.9 -> 19.5 us, sixteen over 64 - 16383 36.7 -> 42.4.)
template <int ROWS, int kTurns, int kFixed>
__device__ __forceinline__ bool find_item(const ChunkParams& p, int lane, Item& it) {
    typedef const __attribute__((address_space(4))) int32_t* const_i32;
    if (!p.target) {
        const uint32_t pair = blockIdx.x / static_cast<uint32_t>(p.row_blocks);
        it.rb = blockIdx.x - pair * p.row_blocks;
        it.b = pair / static_cast<uint32_t>(p.H_kv);
        it.hk = pair - it.b * p.H_kv;
        it.n = p.num_new ? ((const_i32)p.num_new)[it.b] : p.N_max;
        it.P = ((const_i32)p.prefix_len)[it.b];
        it.part = it.first = 0;
        it.parts = 1;
        if (const int err = length_error(p, it.n, it.P)) {
            if (it.rb == 0 && it.hk == 0 && threadIdx.x == 0 && p.err_flag) atomicOr(p.err_flag, err);
            return false;
        }
        if (it.rb * ROWS >= p.group * it.n) return false;
        it.from = 0;
        it.to = it.steps = Work<ChunkParams, ROWS>::rounds(it.P, it.n);
        return true;
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
                rounds = Work<ChunkParams, ROWS>::rounds(P, n);
                units = Work<ChunkParams, ROWS>::blocks(p, n) * p.H_kv;
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
    // The least number of rounds a part for which the parts are no more than one workgroup for every place on the chip (or one part an item).
    // Where that leaves places empty because items have few rounds, twice or three times as many shorter parts: kFixed rounds are what a part costs
    // beside its own (64 rows: 14, four trees over 4864 slots of 40 heads 67 us, with 4 or 8 80 - 86).
    auto parts_of = [&](int len) __attribute__((always_inline)) {
        int sum = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            if (p.B > 64) look(b0, false);
            sum += wave_sum_int(units * ((rounds + len - 1) / len));
        }
        return sum;
    };
    const int shortest = max(kLeastRounds, (longest + kMostParts - 1) / kMostParts);
    int len = longest, all = pairs, best = 1 << 30;
    for (int turns = 1; turns <= kTurns; ++turns) {
        const int most = min(turns * p.places, p.target);
        int l = max(static_cast<int>(ceilf(total / most)), shortest), sum;
        for (; (sum = parts_of(l)) > most && l < longest; l += 1 + (l >> 4)) {}
        l = min(l, longest);
        const int cost = (sum + p.places - 1) / p.places * (l + kFixed);
        if (cost < best) { best = cost; len = l; all = sum; }
        if (l <= shortest) break;
    }
    // every XCD has a contiguous range of the items, so that the row blocks of a head's keys share an L2
    const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3, share = all >> 3, more = all & 7;
    if (place >= share + (xcd < more)) return false;
    const int index = xcd * share + min(xcd, more) + place;
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64) look(b0, false);
        const int mine = units * ((rounds + len - 1) / len), upto = before + wave_scan(mine, lane);
        const unsigned long long here = __ballot(index < upto);
        if (here) {
            const int at = __builtin_ctzll(here);
            it.b = b0 + at;
            it.n = __builtin_amdgcn_readlane(n, at);
            it.P = __builtin_amdgcn_readlane(P, at);
            const uint32_t local = index - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
            const uint32_t blocks = static_cast<uint32_t>(__builtin_amdgcn_readlane(units, at)) / static_cast<uint32_t>(p.H_kv);
            it.steps = __builtin_amdgcn_readlane(rounds, at);
            it.parts = (it.steps + len - 1) / len;
            const uint32_t item = local / static_cast<uint32_t>(it.parts);
            it.part = local - item * it.parts;
            it.first = index - it.part;
            it.hk = item / blocks;
            it.rb = item - it.hk * blocks;
            it.from = static_cast<int>(static_cast<uint32_t>(it.part) * it.steps / it.parts);
            it.to = static_cast<int>((static_cast<uint32_t>(it.part) + 1) * it.steps / it.parts);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Where a workgroup's share begins.  False: nothing to do.
template <int ROWS, bool HALVES>
__device__ __forceinline__ bool begin_share(Share<ChunkParams, ROWS, HALVES>& s, int lane) {
    using W = Work<ChunkParams, ROWS>;
    const ChunkParams& p = s.p;
    s.done = false;
    s.skip = 0;
    // An item a workgroup, the blocks with the most keys first
    auto undivided = [&](bool report) __attribute__((always_inline)) {
        s.whole = true;
        const uint32_t pairs = static_cast<uint32_t>(p.B) * p.H_kv;
        const uint32_t level = blockIdx.x / pairs, pair = blockIdx.x - level * pairs;
        s.rb = p.row_blocks - 1 - level;
        if (s.rb < 0) return false;
        s.b = pair / static_cast<uint32_t>(p.H_kv);
        s.hk = pair - s.b * p.H_kv;
        const int n = p.num_new ? p.num_new[s.b] : p.N_max, P = p.prefix_len[s.b];
        if (const int err = length_error(p, n, P)) {
            if (report && s.rb == 0 && s.hk == 0 && threadIdx.x == 0 && p.err_flag) atomicOr(p.err_flag, err);
            return false;
        }
        return s.request(s.b, u(n), u(P)) && s.rb < s.blocks;
    };
    if (!p.target) return undivided(true);
    s.whole = false;
    const bool report = blockIdx.x == 0 && threadIdx.x < 64 && p.err_flag;
    // lane i: request b0 + i; more than 64 requests are looked at 64 at a time, and once more for the place
    double weight = 0.0, sum = 0.0;
    int items = 0, n = 0, P = 0;
    float heaviest = 0.f, lightest = INFINITY;             // last blocks of the requests
    auto look = [&](int b0, bool first) __attribute__((always_inline)) {
        const int at = b0 + lane;
        int here = 0;
        double most = 0.0;
        weight = 0.0;
        if (at < p.B) {
            n = p.num_new ? p.num_new[at] : p.N_max;
            P = p.prefix_len[at];
            if (const int err = length_error(p, n, P)) {
                if (first && report) atomicOr(p.err_flag, err);
            } else if (n) {
                const int blocks = W::blocks(p, n);
                here = blocks * p.H_kv;
                weight = W::before(p, n, P, blocks) * p.H_kv;
                if (first) most = W::weight(p, n, P, blocks - 1);
            }
        }
        if (first) {
            items += wave_sum_int(here);
            heaviest = fmaxf(heaviest, wave_max(here ? static_cast<float>(most) : 0.f));
            lightest = fminf(lightest, -wave_max(here ? -static_cast<float>(most) : -INFINITY));
        }
    };
    // Sum over the lanes up to this one (exact: whole numbers)
    auto scan = [&](double x) __attribute__((always_inline)) {
        for (int d = 1; d < min(64, p.B); d *= 2) {
            const double other = __shfl_up(x, d);
            if (lane >= d) x += other;
        }
        return x;
    };
    double upto = 0.0;
    const int last_lane = min(64, p.B) - 1;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        look(b0, true);
        upto = scan(weight);
        sum += __shfl(upto, last_lane);
    }
    if (!items) return false;
    s.divide_line(sum, items, heaviest);
    if constexpr (HALVES) {
        const int halved = s.choose(sum, items, heaviest, lightest == heaviest);
        if (halved >= 0) return s.whole_item(blockIdx.x, halved);
    } else {
        if (s.undivided_is_faster(sum, items, heaviest, lightest == heaviest)) return undivided(false);
    }
    s.mine = s.stretch_of(blockIdx.x);
    if (s.mine < 0) return false;
    const double at = s.cut(s.mine);
    double past = 0.0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64) {
            look(b0, false);
            upto = scan(weight);
        }
        const unsigned long long here = __ballot(lane <= last_lane && past + upto > at);
        if (here || b0 + 64 >= p.B) {
            const int to = here ? __builtin_ctzll(here) : last_lane;
            if (!s.request(u(b0 + to), __builtin_amdgcn_readlane(n, to), __builtin_amdgcn_readlane(P, to))) return false;  // (cannot be: the line ends with an item)
            s.find_block(past + __shfl(upto - weight, to));
            return !s.done;
        }
        past += __shfl(upto, last_lane);
    }
    return false;
}

// The parts of an item, in their order, by the 256 threads of the workgroup that came last.  A unit is four head dims of a row; where the
// block has few rows, threads share a unit's parts and meet in LDS. 
template <int D, int ROWS>
__device__ __forceinline__ void merge_parts(const ChunkParams& p, const Item& it, unsigned char* lds) {
    constexpr int kCoherent = 16;                          // device-coherent (sc1) loads, which the compiler counts
    constexpr int NT = D / 32, kPart = part_bytes(ROWS, D);
    const int tid = this_thread(), row0 = it.rb * ROWS;
    const int rows = min(ROWS, p.group * it.n - row0);
    float* const s_w = reinterpret_cast<float*>(lds);      // [rows][kMostParts] weights
    float* const s_inv = s_w + ROWS * kMostParts;        // [rows]
    float* const s_sum = s_inv + ROWS;                     // [256][4]
    auto load = [&](int64_t off, auto wide) __attribute__((always_inline)) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ws_part, 0, 0x7FFFFFFF, 0x00027000);
        if constexpr (decltype(wide)::value) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, static_cast<int>(off), 0, kCoherent);
        else return __builtin_amdgcn_raw_buffer_load_b64(rsrc, static_cast<int>(off), 0, kCoherent);
    };
    // eight threads a row: its maximum over the parts, their weights, the sum
    for (int r = tid >> 3; r < rows; r += 32) {
        const int i0 = tid & 7;
        float m[kMostParts / 8], l[kMostParts / 8], M = -INFINITY, L = 0.f;
#pragma unroll
        for (int k = 0; k < kMostParts / 8; ++k) {
            m[k] = -INFINITY;
            l[k] = 0.f;
            if (i0 + 8 * k < it.parts) {
                const u32x2 ml = load(part_at(it, i0 + 8 * k, kPart) + ROWS * D * 4 + r * 8, std::false_type{});
                m[k] = __uint_as_float(ml[0]);
                l[k] = __uint_as_float(ml[1]);
            }
        }
#pragma unroll
        for (int k = 0; k < kMostParts / 8; ++k) M = __builtin_elementwise_maximum(M, m[k]);
        M = __builtin_elementwise_maximum(M, dpp<0x141>(M));
        M = __builtin_elementwise_maximum(M, dpp<0x4E>(M));
        M = __builtin_elementwise_maximum(M, dpp<0xB1>(M));
        const float m_safe = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < kMostParts / 8; ++k) {
            const float w = fast_exp2((m[k] - m_safe) * p.c2);
            L += l[k] * w;
            if (i0 + 8 * k < it.parts) s_w[r * kMostParts + i0 + 8 * k] = w;
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
            for (int i = part; i < it.parts; i += share * BATCH) {
                u32x4 x[BATCH];
#pragma unroll
                for (int k = 0; k < BATCH; ++k) x[k] = load(part_at(it, min(i + k * share, it.parts - 1), kPart) + off, std::true_type{});
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const float w = i + k * share < it.parts ? s_w[(q + r) * kMostParts + i + k * share] : 0.f;
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

// The workgroup's next segment; false: there is none.  One barrier, behind which LDS is free for it.
struct Segments {
    ShareState state;
    Item item[2];
    int some[2];
};
template <int ROWS, bool HALVES>
__device__ __forceinline__ bool next_segment(const ChunkParams& p, Segments& lds, int turn, Item& it) {
    const int lane = this_thread() & 63, at = turn & 1;    // (two places: a slow wavefront may still read the last one)
    if (threadIdx.x < 64) {
        Share<ChunkParams, ROWS, HALVES> share(p);
        Item found;
        bool some;
        if (turn) {
            share.take(lds.state);
            some = share.next(found);
        } else {
            some = begin_share(share, lane) && share.next(found);
        }
        if (lane == 0) {
            if (some) {
                lds.item[at] = found;
                share.keep(lds.state);
            }
            lds.some[at] = some;
        }
    }
    __syncthreads();
    if (!u(lds.some[at])) return false;
    it = uniform(lds.item[at]);
    return true;
}

// Rows of a lane's blocks of 32: token and head; rows that do not exist count as the last token's.
template <int QB>
struct Rows {
    int token[QB], head[QB];
    bool real[QB];
    __device__ __forceinline__ Rows(const ChunkParams& p, int hk, int n, int row0, int l32) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int R = row0 + qb * 32 + l32;
            token[qb] = divide(R, p.magic_group);
            head[qb] = hk * p.group + R - token[qb] * p.group;
            real[qb] = token[qb] < n;
            if (!real[qb]) { token[qb] = n - 1; head[qb] = hk * p.group; }
        }
    }
};

// Ancestor-or-self masks of the nodes that a lane's rows are: pointer doubling over the lanes (lane i holds node i).  False: not a tree.
template <int QB>
__device__ __forceinline__ bool ancestors(const ChunkParams& p, const Item& it, int lane, const int (&token)[QB], unsigned long long (&anc)[QB]) {
    const int par = lane < it.n ? p.parent[static_cast<int64_t>(it.b) * p.N_max + lane] : -1;
    const bool bad_par = lane < it.n && (lane == 0 ? par != -1 : (par < 0 || par >= lane));
    if (__any(bad_par)) {                                  // the same in every workgroup of the request
        if (it.rb == 0 && it.hk == 0 && it.part == 0 && threadIdx.x == 0 && p.err_flag) atomicOr(p.err_flag, SPECVLM_ERR_BAD_PARENT);
        return false;
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
        const uint32_t lo = __builtin_amdgcn_ds_bpermute(token[qb] * 4, mlo), hi = __builtin_amdgcn_ds_bpermute(token[qb] * 4, mhi);
        anc[qb] = (static_cast<unsigned long long>(hi) << 32) | lo;
    }
    return true;
}

// Bit k: whether a row sees slot slot0 + k, for a tile that reaches past what all rows see.
__device__ __forceinline__ uint32_t visible_causal(int P, int token, int slot0) {
    const int seen = P + token + 1 - slot0;
    return seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u;
}
__device__ __forceinline__ uint32_t visible_tree(int P, unsigned long long anc, int slot0) {
    const int before = P - slot0;                          // keys of the tile in the prefix, < 32
    return before > 0 ? (static_cast<uint32_t>(anc) << before) | ((1u << before) - 1u) : static_cast<uint32_t>(anc >> -before);
}

// Scores of keys that the lane's row does not see become -inf.  A key's place among the lane's scores is a constant once the lane's half is
// shifted out, so a score takes two instructions.
__device__ __forceinline__ void hide(f32x16& s, uint32_t visible, int hf) {
    asm volatile("" : "+v"(visible));          // (stays behind its branch: few tiles need it, and the compiler would do it for all)
    visible >>= 4 * hf;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t on = static_cast<uint32_t>(static_cast<int32_t>(visible << (31 - (8 * (i >> 2) + (i & 3)))) >> 31);
        s[i] = __uint_as_float((on & __float_as_uint(s[i])) | (~on & 0xFF800000u));
    }
}

// The four key streams of a workgroup meet in LDS, and the result is stored, or joins the item's other parts.
template <int D, int QB>
__device__ __forceinline__ void finish(const ChunkParams& p, const Item& it, const Rows<QB>& rows, const f32x16 (&acc)[QB][D / 32], const float (&m_run)[QB],
                                       const float (&l_run)[QB], unsigned char* s_mem, float (*s_m)[QB * 32], float (*s_l)[QB * 32]) {
    constexpr int NT = D / 32, ROWS = QB * 32;
    constexpr int NB = QB * NT;                            // (32 rows, 32 dims) blocks of the result
    constexpr int OWN = NB >= kWaveWgs ? NB / kWaveWgs : 1;
    const int tid = this_thread(), lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = it.b, hk = it.hk;
    // Block x: rows 32 (x / NT), dims 32 (x % NT); wavefront w owns blocks OWN w .. (head size 64 and 32 rows: the first two have one each).
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float l = l_run[qb] + other_half(l_run[qb]);
        if (hf == 0) {
            s_m[wave][qb * 32 + l32] = m_run[qb];
            s_l[wave][qb * 32 + l32] = l;
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
    if (it.parts == 1) {
        if (wave < NB / OWN) {
#pragma unroll
            for (int e = 0; e < OWN; ++e) {
                const int block = wave * OWN + e, qb = block / NT, t = block % NT;
                const bool live = qb ? rows.real[QB - 1] : rows.real[0];
                const int tok = qb ? rows.token[QB - 1] : rows.token[0], h = qb ? rows.head[QB - 1] : rows.head[0];
                const float inv = 1.f / L[e];
                store_block(out[e], inv, p.o + b * p.o_sb + tok * p.o_sn + h * p.o_sh + 32 * t + 8 * hf, live);
                if (live && p.lse && hf == 0 && t == 0) p.lse[(static_cast<int64_t>(b) * p.H_q + h) * p.N_max + tok] = M[e] * p.scale + __log2f(L[e]) * kLn2;
            }
        }
        return;
    }
    // ---- this part of the result, and the merge by the workgroup that comes last -----------------
    // A part: [block][4][64 lanes] vectors of four fp32 (the accumulators as they are, rows that exist only), then a (maximum, sum) pair per row.
    if (wave < NB / OWN) {
        unsigned char* const mine = p.ws_part + part_at(it, it.part, part_bytes(ROWS, D));
#pragma unroll
        for (int e = 0; e < OWN; ++e) {
            const int block = wave * OWN + e, qb = block / NT;
            if (!(qb ? rows.real[QB - 1] : rows.real[0])) continue;
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
        const bool last = ticket == it.parts - 1;
        if (last) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = last;
    }
    __syncthreads();
    if (!*s_last) return;
    asm volatile("" ::: "memory");
    merge_parts<D, ROWS>(p, it, s_mem);
}

}  // namespace

}  // namespace specvlm
