// New K/V rows into a cache and cached slots back into dense rows, as they are or as e4m3 codes with one power-of-two scale per row.
//
// Both are one pass over memory.  A workgroup has the 16 slots that share a page (of a contiguous cache: 16 aligned slots) and four KV
// heads: one block-table entry, and a head's codes (16 rows, 2 KB at head size 128) and scales (16 bytes) in one piece.  A lane holds 8
// elements of a row, 16 or 8 lanes a row; every load of a workgroup is on its way before the first is used.  Stores are non-temporal: what a call
// writes is more than the L2s hold or is next used by another launch (read 27 649 rows of 40 heads 171 -> 154 us, append 8447 of 32 heads in bf16
// 48 -> 41; non-temporal loads lose: of a fused buffer's lines a workgroup takes a part).
//
//   quantise  e = smallest whole number with max |x| <= 448 * 2^e, from the bits of the greatest magnitude (lanes of a row meet by DPP).
//             x * 2^-e is exact, so the only rounding is that to e4m3.  One scale a row and not one per 32 elements: a code has an
//             exponent of its own, and a row's small entries keep their 4 significant bits down to 2^-14 of its greatest.
#include "wave_ops.hpp"

namespace specvlm {

namespace {

constexpr int kCacheThreads = 256;
constexpr int kHeadsPerWg = 4;
constexpr int kLeastExponent = -100;         // value = code * 2^e stays a normal bf16 number: the least code is 2^-9
constexpr int kMostExponent = 120;           // of fp32's greatest numbers; codes above 240 would be infinities there

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct CacheParams {
    KvGeom g;                                // strides in elements of the cache
    unsigned char *k, *v;                    // cache
    unsigned char *ks, *vs;                  // scales (quantised)
    int64_t s_sb, s_sh;
    unsigned char *k_rows, *v_rows;          // dense rows outside
    int64_t r_sb, r_sn, r_sh;                // elements
    const int32_t *first, *count;            // first slot (nullptr: 0), rows (nullptr: N_max)
    int32_t* err_flag;
    int N_max, H_kv;
};

// Eight elements of a dense row as fp32.
template <typename T>
struct Eight {
    u32x4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const unsigned char* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
    }
    __device__ __forceinline__ void store(unsigned char* p) const {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<u32x4*>(p) + i);
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e >> 2][e & 3]);
        else return __uint_as_float((e & 1) ? w[0][e >> 1] & 0xFFFF0000u : w[0][e >> 1] << 16);
    }
};

// Greatest over the LANES (8 or 16) lanes of a row.
template <int LANES>
__device__ __forceinline__ uint32_t row_lanes_max(uint32_t x) {
    auto meet = [&](uint32_t y) { x = x > y ? x : y; };
    if constexpr (LANES == 16) meet(dpp<kRor8>(static_cast<int>(x)));
    meet(dpp<0x141>(static_cast<int>(x)));        // row_half_mirror: lane 7 - i of the eight
    meet(dpp<0x4E>(static_cast<int>(x)));         // quad_perm 2, 3, 0, 1
    meet(dpp<0xB1>(static_cast<int>(x)));         // quad_perm 1, 0, 3, 2
    return x;
}

// The workgroup's place: (16-slot tile of a request's rows, group of heads, request), and what part of the tile the call has.
// Returns false where it has none.
struct Place {
    int b, hk0, slot0, first, n;             // first slot of the tile; of the call's rows; their number
    int64_t base, s_base;                    // element offset of the tile's first slot at head 0, in the cache and in the scales
};
__device__ __forceinline__ bool place_of(const CacheParams& p, Place& at) {
    at.b = blockIdx.z;
    at.hk0 = blockIdx.y * kHeadsPerWg;
    at.first = p.first ? p.first[at.b] : 0;
    at.n = p.count ? p.count[at.b] : p.N_max;
    int err = 0;
    if (at.n < 0 || at.n > p.N_max) err |= SPECVLM_ERR_BAD_NUM_NODES;
    else if (at.first < 0 || at.first > p.g.capacity - at.n) err |= SPECVLM_ERR_BAD_LENGTH;
    if (err) {
        if (p.err_flag && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.err_flag, err);
        return false;
    }
    if (!at.n) return false;
    const int64_t tile = (at.first >> 4) + static_cast<int64_t>(blockIdx.x);
    if (tile * 16 >= static_cast<int64_t>(at.first) + at.n) return false;
    at.slot0 = static_cast<int>(tile) * 16;
    if (p.g.block_table) {
        const int blk = p.g.block_table[static_cast<int64_t>(at.b) * p.g.max_blocks + tile];
        if (blk < 0 || blk >= p.g.num_blocks) {
            if (p.err_flag && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.err_flag, SPECVLM_ERR_BAD_BLOCK);
            return false;
        }
        at.base = blk * p.g.stride_b;
        at.s_base = blk * p.s_sb;
    } else {
        at.base = at.b * p.g.stride_b + at.slot0 * p.g.stride_t;
        at.s_base = at.b * p.s_sb + at.slot0;
    }
    return true;
}

// Row x of a thread: (tensor, head, slot of the tile); a pass of the workgroup has 256 / LANES rows of one tensor.
template <int LANES>
struct RowOf {
    static constexpr int kHeadsAPass = kCacheThreads / LANES / 16;            // 1 or 2
    static constexpr int kPasses = kHeadsPerWg / kHeadsAPass;                 // per tensor
    static __device__ __forceinline__ int slot(int tid) { return tid / LANES & 15; }
    static __device__ __forceinline__ int head(int tid, int pass) { return pass * kHeadsAPass + tid / (LANES * 16); }
};

__device__ __forceinline__ float two_to(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }

template <typename T, int D, bool QUANTISE>
__global__ __launch_bounds__(kCacheThreads) void kv_append_kernel(CacheParams p) {
    constexpr int LANES = D / 8;
    using Rows = RowOf<LANES>;
    Place at;
    if (!place_of(p, at)) return;
    const int tid = threadIdx.x, slot = Rows::slot(tid), d = (tid & (LANES - 1)) * 8;
    const int i = at.slot0 + slot - at.first;
    const bool live = i >= 0 && i < at.n;
    Eight<T> x[2][Rows::kPasses];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int pass = 0; pass < Rows::kPasses; ++pass) {
            const int hk = at.hk0 + Rows::head(tid, pass);
            if (live && hk < p.H_kv)
                x[which][pass].load((which ? p.v_rows : p.k_rows) + (at.b * p.r_sb + i * p.r_sn + hk * p.r_sh + d) * static_cast<int>(sizeof(T)));
            else
                x[which][pass] = {};
        }
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int pass = 0; pass < Rows::kPasses; ++pass) {
            const int hk = at.hk0 + Rows::head(tid, pass);
            const bool mine = live && hk < p.H_kv;
            const int64_t to = at.base + hk * p.g.stride_h + slot * p.g.stride_t + d;
            const Eight<T>& v = x[which][pass];
            unsigned char* cache = which ? p.v : p.k;
            if constexpr (!QUANTISE) {
                if (mine) v.store(cache + to * static_cast<int>(sizeof(T)));
            } else {
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t a = __float_as_uint(v.get(e)) & 0x7FFFFFFFu;
                    most = a < 0x7F800000u && a > most ? a : most;
                }
                most = row_lanes_max<LANES>(most);
                // most = m 2^k, 1 <= m < 2, and 448 = 1.75 * 2^8
                const int e = max(static_cast<int>(most >> 23) - 127 - 8 + ((most & 0x7FFFFFu) > 0x600000u), kLeastExponent);
                const float scale = two_to(-e);
                float y[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    y[c] = v.get(c) * scale;
                    if (e == kMostExponent && fabsf(y[c]) > 240.f) y[c] = copysignf(240.f, y[c]);
                    if ((__float_as_uint(v.get(c)) & 0x7F800000u) == 0x7F800000u) y[c] = __uint_as_float(0x7FC00000u);
                }
                u32x2 codes;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    int pair = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
                    codes[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], pair, true);
                }
                if (mine) {
                    __builtin_nontemporal_store(codes, reinterpret_cast<u32x2*>(cache + to));
                    if (d == 0) (which ? p.vs : p.ks)[at.s_base + hk * p.s_sh + slot] = static_cast<unsigned char>(e + 127);
                }
            }
        }
}

template <typename T, int D, bool QUANTISED>
__global__ __launch_bounds__(kCacheThreads) void kv_read_kernel(CacheParams p) {
    constexpr int LANES = D / 8;
    using Rows = RowOf<LANES>;
    Place at;
    if (!place_of(p, at)) return;
    const int tid = threadIdx.x, slot = Rows::slot(tid), d = (tid & (LANES - 1)) * 8;
    const int i = at.slot0 + slot - at.first;
    if (i < 0 || i >= at.n) return;
    Eight<T> x[2][Rows::kPasses];
    u32x2 codes[2][Rows::kPasses];
    uint32_t exponent[2][Rows::kPasses];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int pass = 0; pass < Rows::kPasses; ++pass) {
            const int hk = at.hk0 + Rows::head(tid, pass);
            if (hk >= p.H_kv) continue;
            const int64_t from = at.base + hk * p.g.stride_h + slot * p.g.stride_t + d;
            const unsigned char* cache = which ? p.v : p.k;
            if constexpr (QUANTISED) {
                codes[which][pass] = *reinterpret_cast<const u32x2*>(cache + from);
                exponent[which][pass] = (which ? p.vs : p.ks)[at.s_base + hk * p.s_sh + slot];
            } else {
                x[which][pass].load(cache + from * static_cast<int>(sizeof(T)));
            }
        }
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int pass = 0; pass < Rows::kPasses; ++pass) {
            const int hk = at.hk0 + Rows::head(tid, pass);
            if (hk >= p.H_kv) continue;
            if constexpr (QUANTISED) {
                const float scale = __uint_as_float(exponent[which][pass] << 23);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const u32x2& c = codes[which][pass];
                    if constexpr (sizeof(T) == 2) {
                        x[which][pass].w[0][2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, false));
                        x[which][pass].w[0][2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, true));
                    } else {
                        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], scale, false);
                        const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], scale, true);
                        x[which][pass].w[w] = u32x4{__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1])};
                    }
                }
            }
            x[which][pass].store((which ? p.v_rows : p.k_rows) + (at.b * p.r_sb + i * p.r_sn + hk * p.r_sh + d) * static_cast<int>(sizeof(T)));
        }
}

template <typename T, int D>
void launch_as(const CacheParams& p, bool append, bool quantised, dim3 grid, hipStream_t stream) {
    auto* const kernel = append ? (quantised ? kv_append_kernel<T, D, true> : kv_append_kernel<T, D, false>)
                                : (quantised ? kv_read_kernel<T, D, true> : kv_read_kernel<T, D, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kCacheThreads), 0, stream, p);
}

}  // namespace

int32_t launch_kv_rows(const specvlm_attn_desc& d, bool append, void* k_cache, void* v_cache, const specvlm_kv_scales* scales,
                       void* k_rows, void* v_rows, int64_t stride_b, int64_t stride_n, int64_t stride_h, const int32_t* first,
                       const int32_t* count, const int32_t* block_table, int32_t* err_flag, hipStream_t stream) {
    CacheParams p;
    p.g = KvGeom{d.kv_stride_b, d.kv_stride_h, d.kv_stride_t, d.paged ? block_table : nullptr, d.max_blocks_per_req, d.num_blocks,
                 d.paged ? d.max_blocks_per_req * SPECVLM_PAGE_SIZE : d.kv_capacity};
    p.k = static_cast<unsigned char*>(k_cache); p.v = static_cast<unsigned char*>(v_cache);
    p.ks = scales ? scales->k_dev : nullptr; p.vs = scales ? scales->v_dev : nullptr;
    p.s_sb = scales ? scales->stride_b : 0; p.s_sh = scales ? scales->stride_h : 0;
    p.k_rows = static_cast<unsigned char*>(k_rows); p.v_rows = static_cast<unsigned char*>(v_rows);
    p.r_sb = stride_b; p.r_sn = stride_n; p.r_sh = stride_h;
    p.first = first; p.count = count; p.err_flag = err_flag;
    p.N_max = d.N_max; p.H_kv = d.H_kv;
    // rows that begin anywhere in a tile touch one tile more than their number needs
    const dim3 grid((d.N_max + 15 + 15) / 16, (d.H_kv + kHeadsPerWg - 1) / kHeadsPerWg, d.B);
    if (d.dtype == SPECVLM_BF16) {
        if (d.D == 128) launch_as<uint16_t, 128>(p, append, scales != nullptr, grid, stream);
        else launch_as<uint16_t, 64>(p, append, scales != nullptr, grid, stream);
    } else {
        if (d.D == 128) launch_as<float, 128>(p, append, scales != nullptr, grid, stream);
        else launch_as<float, 64>(p, append, scales != nullptr, grid, stream);
    }
    return check_launch();
}

}  // namespace specvlm
