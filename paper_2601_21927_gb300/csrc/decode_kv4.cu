// GQA decode over a four-bit cache (sonic_attn_decode_kv4).
//
//   O = softmax(scale q K^T) V,  K = c_K s_K,  V = c_V s_V  (kv4_dev.cuh)
//
// One key of one KV head is D / 2 + D / 16 bytes of K and as many of V (144 together at D = 128)
// against 4 D G flops: 25 per byte at G = 7, so HBM bounds it, and next to that the instructions
// that turn codes into operands: 64 values a lane for 16 keys.  Hence
//   - keys in the M dimension of 16 x 8 x 16 products (S^T = K q^T, O^T += V^T P^T), so up to 8
//     query heads cost no more than one, and every code is converted once;
//   - each warp copies its tiles into a ring of its own (cp.async, two tiles ahead), so no warp
//     waits for another and bytes in flight cost no registers;
//   - with the reduction's dimensions taken in the order in which a lane holds them (q is staged to
//     match), each lane's 16 bytes of a K row are eight operand registers' worth.  V needs pairs of
//     keys in one register: a shift and a mask interleave the nibbles of two rows, then the same
//     conversion;
//   - one cvt and one f16x2 multiply per pair of values; the products are exact in fp16;
//   - scores are compared with a running reference, which is only raised (a shuffle reduction and
//     a rescale) when one exceeds it by 2^8;  P is 2^7 at the reference and at most 2^15, and so keeps
//     fp16's full width down to 2^-21 of the reference's weight, and below that is off by 2^-32 of it.
// tcgen05 is no help here: its operands come from shared memory, so the converted values would
// have to be written there and fenced first (its own 4-bit types take no bf16 q and no per-row
// scales of V).
//
// A unit is a (layer, sequence, KV head).  Many short units get a warp each, with no barrier and
// nothing to merge; few units a cluster of 1 to 8 blocks each, whose warps take 16 keys in turn and
// merge through each other's shared memory: one launch.  In other calls (mode_of) persistent blocks
// take equal shares of the keys of one KV head (line.cuh).  The 8 warps of a
// block walk one piece (the share's part of one sequence) together, 16 keys each in turn, each
// with its own softmax state, merged in shared memory at the piece's end; in long shares, pieces
// of at most kSoloKeys keys go to one warp each instead, without a barrier.  Sequences cut
// between blocks leave (max, sum, accumulator) in the workspace for decode_kv4_merge.
// Equal shares for each warp instead of each block were slower on long sequences (eight times the
// parts to merge: 150 us for 138 on 56 up to 16,384 in 4 layers, 246 us on 4 of 60,000).
#include <algorithm>
#include <type_traits>

#include "kv4_dev.cuh"
#include "line.cuh"
#include "sonic_host.h"

namespace sonic {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMinShare = 16 * kWarps;  // keys: one step of a block
constexpr int kSoloKeys = 128;
constexpr int kSoloShare = 1024;  // shares from which short pieces go to single warps
constexpr int kClusterMost = 8;   // blocks of a cluster
constexpr int kSeqCache = 1024;   // sequences whose rows are kept in shared memory
constexpr float kRaise = 8.0f;    // scores above the reference by more raise it
constexpr float kShift = 7.0f;    // P = 2^(s - ref + kShift) <= 2^15

struct Params {
    const uint16_t *q;
    const uint8_t *kc, *ks, *vc, *vs;
    uint16_t *O;
    const int32_t *lens, *kv_start;
    float *lse;
    float *part_acc;   // [slots][D]
    float2 *part_ml;   // [slots]
    int32_t *status;
    int32_t B, Hq, Hkv, G, n_layers, rows, max_len, groups;
    int64_t q_ls, o_ls, codes_ls, scales_ls;
    float scale_log2;
};

__device__ __forceinline__ int seq_len(const Params &p, int b, bool tell = false) {
    const int raw = p.lens[b], start = p.kv_start[b];
    const int len = min(max(raw, 0), p.max_len);
    const bool out = start < 0 || (int64_t)start + len > p.rows;
    if (tell && (out || raw > p.max_len || raw < 0)) set_status(p.status, SONIC_ERR_INVALID_ARGUMENT);
    return out ? 0 : len;
}

__device__ __forceinline__ long long share_of(long long n, int groups) {
    const long long per = ((n + groups - 1) / groups + 15) & ~15LL;
    return per < kMinShare ? kMinShare : per;
}

// A warp's ring of tiles of 16 keys in shared memory, filled with cp.async ahead of their use.
// Lane (g, c) = (lane / 4, lane % 4) reads the c-th quarter of K rows g and g + 8 of a tile and
// the g-th eighth of four V rows.  Row k of the products is key pi(k) = k ^ (k / 2 % 2) of the tile,
// and V's 16-byte chunks are placed so that none of these reads meets a bank conflict:
//   D = 128 (64-byte rows): chunk j of key r at r * 64 + (j ^ 2 (r / 4 % 2)) * 16; reduction rows
//           2c of the four c are keys 0, 3, 4, 7: two in each half of the banks, and of these
//           two the chunks 0, 1 in different quarters;
//   D = 64  (32-byte rows): the key of row 2c + i at place c + 4i.
template <int D>
struct Ring {
    static constexpr int kStages = 3;
    static constexpr int kCodes = 16 * (D / 2), kScales = 16 * (D / 16);
    static constexpr int kV = kCodes, kKs = 2 * kCodes, kVs = kKs + kScales;
    static constexpr int kTile = kVs + kScales;  // 2304, 1152 bytes
    static constexpr int kBytes = kStages * kTile;
};

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void *p) {
    asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

// A lane's places in the ring.
template <int D>
struct Lane {
    uint32_t k, v, s;            // its copies' places in a tile
    uint32_t rk, rs, rv[2], rt[2];  // its reads: K codes and scales, V codes and scales
};

template <int D>
__device__ __forceinline__ Lane<D> lane_places(uint32_t ring) {
    using R = Ring<D>;
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int key = g ^ (g >> 1 & 1), row = lane / (D / 32);
    Lane<D> p;
    p.k = ring + lane * 16;
    p.v = ring + R::kV;
    if constexpr (D == 128)
        p.v += row * 64 + ((lane & 3) ^ (row >> 2 << 1)) * 16;
    else
        p.v += ((row & 8) + (row >> 1 & 3) + 4 * ((row & 1) ^ (row >> 1 & 1))) * 32 + (lane & 1) * 16;
    p.s = ring + R::kKs + lane * (D / 16);
    p.rk = ring + key * (D / 2) + c * (D / 8);
    p.rs = ring + R::kKs + key * (D / 16) + (D == 128 ? 2 * c : c);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 2 * c + (i ^ (c & 1));
        p.rv[i] = ring + R::kV + (D == 128 ? r * 64 + ((g >> 1) ^ (c & 2)) * 16 + (g & 1) * 8
                                           : (c + 4 * i) * 32 + g * 4);
        p.rt[i] = ring + R::kVs + r * (D / 16) + (D == 128 ? g : g >> 1);
    }
    return p;
}

// A tile of 16 keys, from this lane's addresses in it; `n` are the piece's, the others repeat the last
// (their P is zero).
template <int D>
__device__ __forceinline__ void fetch_tile(const Lane<D> &p, uint32_t slot, const uint8_t *k,
                                           const uint8_t *v, const uint8_t *s, int n) {
    int64_t at = 0, at8 = 8 * (D / 2), ats = 0;
    if (n < 16) {
        const int lane = threadIdx.x & 31, row = lane / (D / 32);
        at = min(0, n - 1 - row) * (D / 2);
        at8 = (min(8 + row, n - 1) - row) * (D / 2);
        ats = min(0, n - 1 - (lane & 15)) * (D / 16);
    }
    copy_async<16>(p.k + slot, k + at);
    copy_async<16>(p.v + slot, v + at);
    if constexpr (D == 128) {
        copy_async<16>(p.k + slot + 512, k + at8);
        copy_async<16>(p.v + slot + 512, v + at8);
    }
    copy_async<D / 16>(p.s + slot, s + ats);
}

template <typename T>
__device__ __forceinline__ T lds(uint32_t addr) {
    T v;
    if constexpr (sizeof(T) == 16)
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    else if constexpr (sizeof(T) == 8)
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}

// State of one warp: NT groups of 8 query heads; this lane's columns are heads 2c and 2c + 1 of each.
template <int D, int NT>
struct State {
    float acc[NT][D / 16][4];  // O^T: dims 16 j' ..; see write_result
    float m[NT][2], l[NT][2];  // reference and sum (this lane's keys)
};

template <int D, int NT>
__device__ __forceinline__ void clear_state(State<D, NT> &s) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s.acc[nt][j][e] = 0.f;
        s.m[nt][0] = s.m[nt][1] = -INFINITY;
        s.l[nt][0] = s.l[nt][1] = 0.f;
    }
}

// q of one (layer, sequence, KV head) as operands, scaled per head by a power of two so that its
// largest element lies in [2^13, 2^14): fp16 then holds bf16's 8 bits of every element down to
// 2^-27 of that one (and 2^-38 in part).  f: the factor from products to base-2 scores, for
// this lane's two columns.
template <int D, int NT>
__device__ __forceinline__ void load_q(const Params &p, int layer, int b, int kvh,
                                       uint32_t (&qf)[NT][D / 16][2], float (&f)[NT][2]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int h = nt * 8 + g;
        uint32_t w[D / 8];
        if (h < p.G) {
            const uint4 *src = reinterpret_cast<const uint4 *>(
                p.q + layer * p.q_ls + ((int64_t)b * p.Hq + kvh * p.G + h) * D + c * (D / 4));
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const uint4 x = src[i];
                w[4 * i] = x.x;
                w[4 * i + 1] = x.y;
                w[4 * i + 2] = x.z;
                w[4 * i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) w[i] = 0;
        }
        uint32_t top = 0;  // largest magnitude, as bf16 bits
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
            top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^(13 - e), e the exponent of the largest element, within what a float can hold
        const int up = min(max(13 - ((int)(top >> 7) - 127), -126), 126);
        const float k = __int_as_float((127 + up) << 23);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            qf[nt][s][0] = pack_f16x2(bf16lo(w[2 * s]) * k, bf16hi(w[2 * s]) * k);
            qf[nt][s][1] = pack_f16x2(bf16lo(w[2 * s + 1]) * k, bf16hi(w[2 * s + 1]) * k);
        }
        const float back = p.scale_log2 * __int_as_float((127 - up) << 23);
        f[nt][0] = __shfl_sync(0xffffffffu, back, 8 * c);
        f[nt][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4);
    }
}

// The sixteen keys of the tile at `slot`; those from `n` on are hidden.
template <int D, int NT>
__device__ __forceinline__ void step(const Lane<D> &pl, uint32_t slot, int n, const uint32_t (&qf)[NT][D / 16][2],
                                     const float (&f)[NT][2], State<D, NT> &st) {
    using R = Ring<D>;
    using KVec = typename std::conditional<D == 128, uint4, uint2>::type;
    using VVec = typename std::conditional<D == 128, uint2, uint32_t>::type;
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
    {
        const KVec x0 = lds<KVec>(pl.rk + slot), x1 = lds<KVec>(pl.rk + slot + 8 * (D / 2));
        const uint32_t at = pl.rs + slot;
        const uint32_t sk0 = D == 128 ? lds_u16(at) : lds_u8(at);
        const uint32_t sk1 = D == 128 ? lds_u16(at + 64) : lds_u8(at + 32);
        const uint32_t *k0 = reinterpret_cast<const uint32_t *>(&x0);
        const uint32_t *k1 = reinterpret_cast<const uint32_t *>(&x1);
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            uint32_t a[4], b[4];
            kv4_decode4(k0[w], a);
            kv4_decode4(k1[w], b);
            // (D = 128: words 0, 1 are the quarter's first block)
            const uint32_t sa = kv4_scale_f16x2(D == 128 && w >= 2 ? sk0 >> 8 : sk0 & 0xFFu);
            const uint32_t sb = kv4_scale_f16x2(D == 128 && w >= 2 ? sk1 >> 8 : sk1 & 0xFFu);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = mul_f16x2(a[i], sa);
                b[i] = mul_f16x2(b[i], sb);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    mma_f16(s[nt], a[2 * h], b[2 * h], a[2 * h + 1], b[2 * h + 1], qf[nt][2 * w + h][0],
                            qf[nt][2 * w + h][1]);
        }
    }
    if (n < 16) {
        const int g = (threadIdx.x & 31) >> 2, key = g ^ (g >> 1 & 1);  // of product row g
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (key >= n) s[nt][0] = s[nt][1] = -INFINITY;
            if (key + 8 >= n) s[nt][2] = s[nt][3] = -INFINITY;
        }
    }
    uint32_t pb[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float (&x)[4] = s[nt];
        const float t0 = fmaxf(x[0], x[2]) * f[nt][0], t1 = fmaxf(x[1], x[3]) * f[nt][1];
        const bool raise = t0 > st.m[nt][0] + kRaise || t1 > st.m[nt][1] + kRaise;
        if (__any_sync(0xffffffffu, raise)) {
            float n0 = t0, n1 = t1;
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, o));
                n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
            }
            n0 = fmaxf(n0, st.m[nt][0]);
            n1 = fmaxf(n1, st.m[nt][1]);
            const float a0 = ex2(st.m[nt][0] - n0), a1 = ex2(st.m[nt][1] - n1);
            st.m[nt][0] = n0;
            st.m[nt][1] = n1;
            st.l[nt][0] *= a0;
            st.l[nt][1] *= a1;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                st.acc[nt][j][0] *= a0;
                st.acc[nt][j][1] *= a1;
                st.acc[nt][j][2] *= a0;
                st.acc[nt][j][3] *= a1;
            }
        }
        const float o0 = kShift - st.m[nt][0], o1 = kShift - st.m[nt][1];
        const float p0 = ex2(fmaf(x[0], f[nt][0], o0)), p1 = ex2(fmaf(x[1], f[nt][1], o1));
        const float p2 = ex2(fmaf(x[2], f[nt][0], o0)), p3 = ex2(fmaf(x[3], f[nt][1], o1));
        st.l[nt][0] += p0 + p2;
        st.l[nt][1] += p1 + p3;
        pb[nt][0] = transpose8x8(pack_f16x2(p0, p1));
        pb[nt][1] = transpose8x8(pack_f16x2(p2, p3));
    }
    // O^T += V^T P^T: the two dims of a byte go to rows g and g + 8 of one product
    VVec x[4];
    uint32_t sv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // reduction rows 2c, 2c + 1, 2c + 8, 2c + 9
        x[i] = lds<VVec>(pl.rv[i & 1] + slot + (i >> 1) * 8 * (D / 2));
        sv[i] = lds_u8(pl.rt[i & 1] + slot + (i >> 1) * 8 * (D / 16));
    }
    const uint32_t s01 = (sv[0] | sv[1] << 16) << 7, s23 = (sv[2] | sv[3] << 16) << 7;
    const uint32_t *v0 = reinterpret_cast<const uint32_t *>(&x[0]);
    const uint32_t *v1 = reinterpret_cast<const uint32_t *>(&x[1]);
    const uint32_t *v2 = reinterpret_cast<const uint32_t *>(&x[2]);
    const uint32_t *v3 = reinterpret_cast<const uint32_t *>(&x[3]);
    constexpr uint32_t kLo = 0x0F0F0F0Fu, kHi = 0xF0F0F0F0u;
#pragma unroll
    for (int w = 0; w < D / 64; ++w) {
        uint32_t e01[4], o01[4], e23[4], o23[4];
        kv4_decode4((v0[w] & kLo) | ((v1[w] << 4) & kHi), e01);
        kv4_decode4(((v0[w] >> 4) & kLo) | (v1[w] & kHi), o01);
        kv4_decode4((v2[w] & kLo) | ((v3[w] << 4) & kHi), e23);
        kv4_decode4(((v2[w] >> 4) & kLo) | (v3[w] & kHi), o23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = mul_f16x2(e01[i], s01), a1 = mul_f16x2(o01[i], s01);
            const uint32_t a2 = mul_f16x2(e23[i], s23), a3 = mul_f16x2(o23[i], s23);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                mma_f16(st.acc[nt][4 * w + i], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
        }
    }
}

// Where an accumulator's element goes in a shared-memory row of one query head: lane g's
// D / 8 dims two words apart from the next lane's, and rows kLd words apart (2 kLd = 8 mod 32),
// so that a half-warp's 8-byte stores fall on different banks.
template <int D>
struct Smem {
    static constexpr int kDims = D / 8;                // dims of a lane
    static constexpr int kLd = 8 * (kDims + 2) + 4;    // 148, 84
};

template <int D, int NT>
__host__ __device__ constexpr size_t smem_bytes() {
    constexpr size_t state = (size_t)kWarps * NT * 8 * (Smem<D>::kLd + 2) * sizeof(float);
    constexpr size_t ring = (size_t)kWarps * Ring<D>::kBytes;
    return ring + state;
}

// A warp's stream of tiles: copies ahead of the products.
template <int D>
struct Feed {
    using R = Ring<D>;
    Lane<D> pl;
    const uint8_t *k, *v, *s;
    int ahead, stride;  // keys from the next tile to fetch on; from one tile to the next

    __device__ __forceinline__ void fetch(uint32_t slot) {
        if (ahead > 0) {
            fetch_tile<D>(pl, slot, k, v, s, ahead);
            k += stride * (D / 2);
            v += stride * (D / 2);
            s += stride * (D / 16);
            ahead -= stride;
        }
        copy_commit();
    }
    // The first tiles of `keys` keys from `row` on, `step` from one to the next, and q to L2.
    __device__ __forceinline__ void begin(const Params &p, int layer, int b, int kvh, int64_t row, int keys,
                                          int step) {
        const int lane = threadIdx.x & 31;
        const int64_t at = (int64_t)kvh * p.rows + row;
        ahead = keys;
        stride = step;
        k = p.kc + layer * p.codes_ls + at * (D / 2) + lane * 16;
        v = p.vc + layer * p.codes_ls + at * (D / 2) + lane * 16;
        // lanes 0-15 copy the scales of K, the others of V: one row each
        s = (lane < 16 ? p.ks : p.vs) + layer * p.scales_ls + (at + (lane & 15)) * (D / 16);
#pragma unroll
        for (int i = 0; i < R::kStages - 1; ++i) fetch(i * R::kTile);
        if (lane < p.G * D / 64)
            prefetch_l2(p.q + layer * p.q_ls + ((int64_t)b * p.Hq + kvh * p.G) * D + lane * 64);
    }
    // All of them, into the state (l: summed over the warp's lanes of a column).
    template <int NT>
    __device__ __forceinline__ void attend(int n, const uint32_t (&qf)[NT][D / 16][2], const float (&f)[NT][2],
                                           State<D, NT> &st) {
        while (n > 0) {
#pragma unroll
            for (int i = 0; i < R::kStages; ++i) {
                if (n <= 0) break;
                copy_wait<R::kStages - 2>();
                __syncwarp();  // every lane's copies have landed, and all have read the tile before
                fetch((i + R::kStages - 1) % R::kStages * R::kTile);
                step<D, NT>(pl, i * R::kTile, n, qf, f, st);
                n -= stride;
            }
        }
        __syncwarp();  // (the last tile is read; no copy is left)
    }
};

template <int D, int NT>
__device__ __forceinline__ void sum_lanes(State<D, NT> &st) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1)
                st.l[nt][e] += __shfl_xor_sync(0xffffffffu, st.l[nt][e], o);
}

// Blocks that an SM holds, by registers.  (Three at head_dim 64 with one group of heads, 74 registers,
// were slower than two: 169 us for 162 on 56 long sequences; with two groups two blocks took 65, one 73.)
template <int D, int NT>
constexpr int kResident = D == 128 && NT == 2 ? 1 : 2;

// The states of a block's warps in shared memory, behind the rings.
template <int D, int NT>
struct Shared {
    float *acc, *m, *l;  // [warps][NT * 8][kLd], [warps][NT * 8], [warps][NT * 8]

    __device__ __forceinline__ explicit Shared(float *smem) {
        acc = smem + kWarps * Ring<D>::kBytes / 4;
        m = acc + kWarps * NT * 8 * Smem<D>::kLd;
        l = m + kWarps * NT * 8;
    }
    __device__ __forceinline__ void put(int warp, const State<D, NT> &st) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int h = nt * 8 + 2 * c + e;
                float *a = acc + (warp * NT * 8 + h) * Smem<D>::kLd + g * (Smem<D>::kDims + 2);
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    *reinterpret_cast<float2 *>(a + 2 * j) =
                        make_float2(st.acc[nt][j][e], st.acc[nt][j][2 + e]);
                if (g == 0) {
                    m[warp * NT * 8 + h] = st.m[nt][e];
                    l[warp * NT * 8 + h] = st.l[nt][e];
                }
            }
    }
    // Maximum, sum and accumulators of dims d, d + 1 of head h over the warps.
    __device__ __forceinline__ float4 merge(int h, int d) const {
        float M = -INFINITY;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) M = fmaxf(M, m[k * NT * 8 + h]);
        if (M == -INFINITY) return make_float4(-INFINITY, 0.f, 0.f, 0.f);  // (no warp had keys)
        float L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
            const float e = ex2(m[k * NT * 8 + h] - M);
            const float2 a = *reinterpret_cast<const float2 *>(
                acc + (k * NT * 8 + h) * Smem<D>::kLd + d / Smem<D>::kDims * (Smem<D>::kDims + 2) +
                d % Smem<D>::kDims);
            L += e * l[k * NT * 8 + h];
            x += e * a.x;
            y += e * a.y;
        }
        return make_float4(M - kShift, L, x, y);
    }
};

// A warp's own result: heads 2c, 2c + 1 of each group of 8, dims g D / 8 .. of lane (g, c).
template <int D, int NT>
__device__ __forceinline__ void write_result(const Params &p, const State<D, NT> &st, uint16_t *out, int64_t unit) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int h = nt * 8 + 2 * c + e;
            if (h >= p.G) continue;
            const float l = st.l[nt][e], inv = 1.0f / l;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
                *reinterpret_cast<uint32_t *>(out + h * D + g * (D / 8) + 2 * j) =
                    pack_bf16x2(st.acc[nt][j][e] * inv, st.acc[nt][j][2 + e] * inv);
            if (g == 0 && p.lse != nullptr) p.lse[unit + h] = (st.m[nt][e] - kShift + __log2f(l)) * kLn2;
        }
}

template <int D, int NT>
__device__ __forceinline__ void write_part(const Params &p, const State<D, NT> &st, int64_t part) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int h = nt * 8 + 2 * c + e;
            if (h >= p.G) continue;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
                *reinterpret_cast<float2 *>(p.part_acc + (part + h) * D + g * (D / 8) + 2 * j) =
                    make_float2(st.acc[nt][j][e], st.acc[nt][j][2 + e]);
            if (g == 0) p.part_ml[part + h] = make_float2(st.m[nt][e] - kShift, st.l[nt][e]);
        }
}

// One (layer, sequence, KV head) per warp, for many short sequences: no barrier, no merge.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads, kResident<D, NT>) decode_kv4_warp_kernel(const Params p) {
    extern __shared__ __align__(16) float smem[];
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const int64_t u = (int64_t)blockIdx.x * kWarps + warp;
    if (u >= (int64_t)p.n_layers * p.B * p.Hkv) return;
    const int kvh = (int)(u % p.Hkv), seq = (int)(u / p.Hkv % p.B), layer = (int)(u / p.Hkv / p.B);
    const int len = seq_len(p, seq, lane == 0 && kvh == 0 && layer == 0);
    uint16_t *out = p.O + layer * p.o_ls + ((int64_t)seq * p.Hq + kvh * p.G) * D;
    const int64_t unit = ((int64_t)layer * p.B + seq) * p.Hq + kvh * p.G;
    if (len == 0) {
        for (int i = lane; i < p.G * (D / 2); i += 32) reinterpret_cast<uint32_t *>(out)[i] = 0u;
        if (p.lse != nullptr && lane < p.G) p.lse[unit + lane] = -INFINITY;
        return;
    }
    Feed<D> feed;
    feed.pl = lane_places<D>(smem_u32(smem) + warp * Ring<D>::kBytes);
    State<D, NT> st;
    uint32_t qf[NT][D / 16][2];
    float f[NT][2];
    feed.begin(p, layer, seq, kvh, p.kv_start[seq], len, 16);
    clear_state(st);
    load_q<D, NT>(p, layer, seq, kvh, qf, f);
    feed.attend(len, qf, f, st);
    sum_lanes(st);
    write_result(p, st, out, unit);
}

// One (layer, sequence, KV head) per cluster of blocks, which share its keys and merge through
// shared memory: no second launch.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads, kResident<D, NT>) decode_kv4_cluster_kernel(const Params p, int blocks) {
    extern __shared__ __align__(16) float smem[];
    __shared__ float4 s_part[NT * 8 * D / 2];  // the block's (max, sum, two dims) by (head, dims)
    const int tid = threadIdx.x;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (known to be the warp's)
    const int rank = blocks > 1 ? (int)cluster_rank() : 0;
    const int64_t u = blockIdx.x / blocks;
    const int kvh = (int)(u % p.Hkv), seq = (int)(u / p.Hkv % p.B), layer = (int)(u / p.Hkv / p.B);
    pdl_wait();
    pdl_trigger();
    const int len = seq_len(p, seq, rank == 0 && kvh == 0 && layer == 0);
    const int per = ((len + blocks - 1) / blocks + 15) & ~15, from = min(len, rank * per);
    const int n = min(len - from, per) - 16 * warp;  // keys from this warp's first on
    State<D, NT> st;
    clear_state(st);
    if (n > 0) {
        Feed<D> feed;
        feed.pl = lane_places<D>(smem_u32(smem) + warp * Ring<D>::kBytes);
        uint32_t qf[NT][D / 16][2];
        float f[NT][2];
        feed.begin(p, layer, seq, kvh, (int64_t)p.kv_start[seq] + from + 16 * warp, n, 16 * kWarps);
        load_q<D, NT>(p, layer, seq, kvh, qf, f);
        feed.attend(n, qf, f, st);
        sum_lanes(st);
    }
    Shared<D, NT> sh(smem);
    sh.put(warp, st);
    __syncthreads();
    const int items = p.G * (D / 2);
    for (int i = tid; i < items; i += kThreads) s_part[i] = sh.merge(i / (D / 2), i % (D / 2) * 2);
    if (blocks > 1)
        cluster_sync_all();
    else
        __syncthreads();
    uint16_t *out = p.O + layer * p.o_ls + ((int64_t)seq * p.Hq + kvh * p.G) * D;
    for (int i = rank * kThreads + tid; i < items; i += blocks * kThreads) {
        float4 part[kClusterMost];
        float M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int k = 0; k < kClusterMost; ++k)
            if (k < blocks) {
                part[k] = blocks > 1 ? ld_cluster_f4(smem_in_rank(&s_part[i], k)) : s_part[i];
                M = fmaxf(M, part[k].x);
            }
#pragma unroll
        for (int k = 0; k < kClusterMost; ++k)
            if (k < blocks && part[k].x > -INFINITY) {
                const float e = ex2(part[k].x - M);
                L += e * part[k].y;
                x += e * part[k].z;
                y += e * part[k].w;
            }
        const int h = i / (D / 2), d = i % (D / 2) * 2;
        *reinterpret_cast<uint32_t *>(out + h * D + d) = len > 0 ? pack_bf16x2(x / L, y / L) : 0u;
        if (d == 0 && p.lse != nullptr)
            p.lse[((int64_t)layer * p.B + seq) * p.Hq + kvh * p.G + h] =
                len > 0 ? (M + __log2f(L)) * kLn2 : -INFINITY;
    }
    if (blocks > 1) cluster_sync_all();  // no block leaves while another reads its part
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, kResident<D, NT>) decode_kv4_kernel(const Params p) {
    extern __shared__ __align__(16) float smem[];
    __shared__ LineShared line;
    __shared__ int s_len[kSeqCache], s_start[kSeqCache];
    Shared<D, NT> sh(smem);
    const int tid = threadIdx.x;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (known to be the warp's)
    pdl_wait();
    pdl_trigger();
    const bool cached = p.B <= kSeqCache;
    if (cached) {
        for (int b = tid; b < p.B; b += kThreads) {
            s_len[b] = seq_len(p, b, blockIdx.x == 0);
            s_start[b] = p.kv_start[b];
        }
        __syncthreads();
    } else if (blockIdx.x == 0) {
        for (int b = tid; b < p.B; b += kThreads) seq_len(p, b, true);
    }
    auto len_of = [&](int b) { return cached ? s_len[b] : seq_len(p, b); };
    auto start_of = [&](int b) { return cached ? s_start[b] : p.kv_start[b]; };
    const int kvh = (int)blockIdx.x % p.Hkv, grp = (int)blockIdx.x / p.Hkv;
    long long per = 0, x0 = 0;
    int layer = 0;
    line_find<kThreads>(p.B, len_of, [&](long long sum) {
        per = share_of(sum * p.n_layers, p.groups);
        x0 = grp * per;
        if (x0 >= sum * p.n_layers) return -1LL;
        layer = (int)(x0 / sum);
        return x0 - layer * sum;
    }, line);
    const long long n = line.sum * p.n_layers;
    if (x0 >= n) return;
    // This warp's walk along the share, piece by piece: the 8 warps take 16 keys each in turn of
    // most pieces; in long shares, one takes all of a short piece.
    const bool solo_ok = per >= kSoloShare;
    struct Walk {
        long long left;
        int layer, b, off, solo;
    };
    struct Piece {
        int layer, b, off, keys;
        bool alone;
    };
    auto next_piece = [&](Walk &k, Piece &w) -> bool {
        while (k.left > 0) {
            const int len = len_of(k.b);
            w.layer = k.layer;
            w.b = k.b;
            w.off = k.off;
            w.keys = (int)min((long long)(len - k.off), k.left);
            k.left -= w.keys;
            k.off = 0;
            if (++k.b == p.B) {
                k.b = 0;
                ++k.layer;
            }
            if (w.keys == 0) continue;
            w.alone = solo_ok && w.keys <= kSoloKeys;
            if (!w.alone || k.solo++ % kWarps == warp) return true;
        }
        return false;
    };
    Walk walk{min(per, n - x0), layer, line.seq, line.off, 0};

    Feed<D> feed;
    feed.pl = lane_places<D>(smem_u32(smem) + warp * Ring<D>::kBytes);
    // A piece's first tiles are on their way while the one before it is merged.
    auto begin = [&](const Piece &w) {
        const int first = w.alone ? 0 : 16 * warp;
        feed.begin(p, w.layer, w.b, kvh, (int64_t)start_of(w.b) + w.off + first, w.keys - first,
                   w.alone ? 16 : 16 * kWarps);
    };

    State<D, NT> st;
    uint32_t qf[NT][D / 16][2];
    float f[NT][2];
    Piece piece;
    bool more = next_piece(walk, piece);
    if (more) begin(piece);
    while (more) {
        const bool alone = piece.alone;
        const int take = piece.keys, seq = piece.b, lay = piece.layer, from = piece.off;
        clear_state(st);
        const int n = alone ? take : take - 16 * warp;  // keys from this warp's first on
        if (n > 0) load_q<D, NT>(p, lay, seq, kvh, qf, f);
        feed.attend(n, qf, f, st);
        more = next_piece(walk, piece);
        if (more) begin(piece);
        sum_lanes(st);
        // a share cuts at most two sequences: its first (from the middle on) has slot 0, its
        // last (from its start) slot 1
        const bool whole = take == len_of(seq);
        const int64_t part = ((int64_t)blockIdx.x * 2 + (from > 0 ? 0 : 1)) * p.G;
        const int64_t unit = ((int64_t)lay * p.B + seq) * p.Hq + kvh * p.G;
        uint16_t *out = p.O + lay * p.o_ls + ((int64_t)seq * p.Hq + kvh * p.G) * D;
        if (alone) {
            if (whole)
                write_result(p, st, out, unit);
            else
                write_part(p, st, part);
            continue;
        }
        __syncthreads();  // the states of the piece before are read
        sh.put(warp, st);
        __syncthreads();
        for (int i = tid; i < p.G * (D / 2); i += kThreads) {
            const int h = i / (D / 2), d = i % (D / 2) * 2;
            const float4 r = sh.merge(h, d);
            if (whole) {
                *reinterpret_cast<uint32_t *>(out + h * D + d) = pack_bf16x2(r.z / r.y, r.w / r.y);
                if (d == 0 && p.lse != nullptr) p.lse[unit + h] = (r.x + __log2f(r.y)) * kLn2;
            } else {
                *reinterpret_cast<float2 *>(p.part_acc + (part + h) * D + d) = make_float2(r.z, r.w);
                if (d == 0) p.part_ml[part + h] = make_float2(r.x, r.y);
            }
        }
    }
}

// The log-sum-exp merge of the sequences that were cut, zeros for the empty ones: a warp per
// (layer, sequence, query head); a block takes one (layer, sequence) and `heads` of its heads.
constexpr int kMergeThreads = 128;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) decode_kv4_merge_kernel(const Params p, int heads) {
    // The main kernel lets this one start once all work ahead of the call is complete, so the
    // lengths are read and the pieces found while it still runs.
    const int per_row = (p.Hq + heads - 1) / heads;
    const int64_t lb = blockIdx.x / per_row;
    const int b = (int)(lb % p.B), layer = (int)(lb / p.B);
    const int h0 = (int)(blockIdx.x % per_row) * heads, h1 = min(p.Hq, h0 + heads);
    const int len = seq_len(p, b);
    int n = 0;
    long long ga = 0;
    if (len > 0) {
        // the keys before this sequence and in all: two sums by the block
        long long before = 0, sum = 0;
        for (int i = threadIdx.x; i < p.B; i += kMergeThreads) {
            const int v = seq_len(p, i);
            sum += v;
            before += i < b ? v : 0;
        }
        __shared__ long long part[2][kMergeThreads / 32];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            before += __shfl_xor_sync(0xffffffffu, before, o);
        }
        if ((threadIdx.x & 31) == 0) {
            part[0][threadIdx.x >> 5] = sum;
            part[1][threadIdx.x >> 5] = before;
        }
        __syncthreads();
        sum = before = 0;
        for (int w = 0; w < kMergeThreads / 32; ++w) {
            sum += part[0][w];
            before += part[1][w];
        }
        const long long per = share_of(sum * p.n_layers, p.groups), s0 = layer * sum + before;
        ga = s0 / per;
        n = (int)((s0 + len - 1) / per - ga) + 1;
    }
    // (no block ends before the main kernel: the next call reuses its workspace)
    pdl_wait();
    pdl_trigger();
    if (n == 1) return;  // written by the main kernel
    const int lane = threadIdx.x & 31;
    constexpr int kDpl = D / 32;
    for (int h = h0 + (threadIdx.x >> 5); h < h1; h += kMergeThreads / 32) {
        const int kvh = h / p.G, hl = h % p.G;
        auto slot = [&](int i) {
            return (((ga + i) * p.Hkv + kvh) * 2 + (i == 0 ? 1 : 0)) * (int64_t)p.G + hl;
        };
        float M = -INFINITY;
        for (int i = lane; i < n; i += 32) M = fmaxf(M, p.part_ml[slot(i)].x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        float L = 0.f, a[kDpl] = {};
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const int64_t s = slot(i);
            const float2 ml = p.part_ml[s];
            const float e = ex2(ml.x - M);
            L += e * ml.y;
#pragma unroll
            for (int k = 0; k < kDpl / 2; ++k) {
                const float2 v =
                    *reinterpret_cast<const float2 *>(p.part_acc + s * D + lane * kDpl + 2 * k);
                a[2 * k] += e * v.x;
                a[2 * k + 1] += e * v.y;
            }
        }
        uint16_t *out = p.O + layer * p.o_ls + ((int64_t)b * p.Hq + h) * D + lane * kDpl;
#pragma unroll
        for (int k = 0; k < kDpl / 2; ++k)
            *reinterpret_cast<uint32_t *>(out + 2 * k) =
                n > 0 ? pack_bf16x2(a[2 * k] / L, a[2 * k + 1] / L) : 0u;
        if (lane == 0 && p.lse != nullptr)
            p.lse[((int64_t)layer * p.B + b) * p.Hq + h] = n > 0 ? (M + __log2f(L)) * kLn2 : -INFINITY;
    }
}

constexpr size_t kWsAlign = 16;

int64_t resident_blocks(const sonic_decode_kv4_args *a) {
    const bool wide = a->n_heads_q / a->n_heads_kv > 8;
    const int each = a->head_dim == 64 ? (wide ? kResident<64, 2> : kResident<64, 1>)
                                       : (wide ? kResident<128, 2> : kResident<128, 1>);
    return (int64_t)device_sm_count() * each;
}

// Blocks per KV head: those that fit the GPU at once, no more than there are shares' keys.
int groups_of(const sonic_decode_kv4_args *a) {
    const int64_t keys = (int64_t)a->n_layers * a->batch * std::max(a->max_len, 1);
    const int64_t most = (keys + kMinShare - 1) / kMinShare;
    return (int)std::max<int64_t>(1, std::min(most, resident_blocks(a) / a->n_heads_kv));
}

size_t acc_bytes(const sonic_decode_kv4_args *a, int groups) {
    return (size_t)groups * 2 * a->n_heads_q * a->head_dim * sizeof(float);
}

// How a call's units (layer, sequence, KV head) are worked on: a warp each, a cluster of 1, 2, 4 or
// 8 blocks each, or equal shares of the line of keys (kByLine).
//
// Reckoned in steps of a warp (16 keys; 0.47 us while HBM does not bound it): a wave of resident
// blocks costs 8 steps (launch, lengths, q, the merge of the warps; 6 where each warp is alone) and
// its longest unit's, the exchange within a cluster 3.  The cheapest is taken up to 85 steps.  Above
// that equal shares win, whatever the lengths (their time is that of the sum of the lengths, the
// others' that of the longest; they add a launch and a merge through HBM), but for units that fill
// the GPU's warps and are short enough to even out: up to kWarpKeys these keep a warp each.
// GPU time in us, D = 128.  Clusters (their size) / line, 32/8 heads: one sequence of 1,045 rows
// 6.2 (8) / 9.6, of 16,000 13.1 (8) / 21.4; 16 of 1,045 8.7 (1) / 16.4; 64 ragged ones up to 1,000
// 15.0 (1) / 22.7, up to 4,000 35.3 (1) / 37.0; 16 up to 16,000 33.4 (4) / 32.9; 64 up to 8,000
// 55.6 (2) / 53.7; 56 up to 16,000 in 4 layers of 28/4 heads 154 (2) / 138.  Warps / clusters of 1 /
// line: 64 up to 100 in 8 layers 13.7 / 48 / 57; 1,500 up to 40, 4/1 heads, 8.9 / 33 / 52; 64 up to
// 1,000 in 8 layers 61 / 81 / 92, in 32 layers 163 / 303 / 309; 500 up to 2,000 in 8 layers of 8/2
// heads 210 / 213 / 235, but 56 up to 4,000 in 4 layers of 28/4 heads 107 by warps, 63 by the line.
constexpr int kByWarp = -1, kByLine = 0;
constexpr int kWarpKeys = 2048;
int mode_of(const sonic_decode_kv4_args *a) {
    const int64_t units = (int64_t)a->n_layers * a->batch * a->n_heads_kv, resident = resident_blocks(a);
    int64_t best = 85;
    int mode = units >= resident * kWarps && a->max_len <= kWarpKeys ? kByWarp : kByLine;
    auto offer = [&](int m, int64_t blocks, int64_t fixed, int keys, int64_t extra) {
        const int64_t waves = (blocks + resident - 1) / resident;
        const int64_t cost = waves * (fixed + ((int64_t)a->max_len + keys - 1) / keys) + extra;
        if (cost <= best) {
            best = cost;
            mode = m;
        }
    };
    offer(kByWarp, (units + kWarps - 1) / kWarps, 6, 16, 0);
    for (int c = 1; c <= kClusterMost; c *= 2) offer(c, units * c, 8, c * 16 * kWarps, c > 1 ? 3 : 0);
    return mode;
}

template <int D, int NT>
cudaError_t launch(const Params &p, int mode, cudaStream_t stream) {
    const int64_t units = (int64_t)p.n_layers * p.B * p.Hkv;
    if (mode == kByWarp) {
        auto kern = decode_kv4_warp_kernel<D, NT>;
        constexpr size_t smem = (size_t)kWarps * Ring<D>::kBytes;
        const cudaError_t e =
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        return launch_pdl(kern, dim3((unsigned)((units + kWarps - 1) / kWarps)), kThreads, smem, stream, 1, p);
    }
    if (mode > 0) {
        auto kern = decode_kv4_cluster_kernel<D, NT>;
        constexpr size_t smem = smem_bytes<D, NT>();
        const cudaError_t e =
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        return launch_pdl(kern, dim3((unsigned)(units * mode)), kThreads, smem, stream, mode, p, mode);
    }
    auto kern = decode_kv4_kernel<D, NT>;
    constexpr size_t smem = smem_bytes<D, NT>();
    cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kern, dim3((unsigned)(p.groups * p.Hkv)), kThreads, smem, stream, 1, p);
    if (e != cudaSuccess) return e;
    // a block per four heads, or per sequence where there are so many that each block's sum of
    // the lengths would weigh
    const int heads = p.B <= 256 ? std::min(4, p.Hq) : p.Hq;
    const int64_t merges = (int64_t)p.n_layers * p.B * ((p.Hq + heads - 1) / heads);
    return launch_pdl(decode_kv4_merge_kernel<D>, dim3((unsigned)merges), kMergeThreads, 0, stream, 1,
                      p, heads);
}

}  // namespace
}  // namespace sonic

using namespace sonic;

extern "C" size_t sonic_decode_kv4_workspace_size(const sonic_decode_kv4_args *a) {
    if (a == nullptr || a->batch <= 0 || a->n_layers < 1 || a->n_heads_q < 1 || a->n_heads_kv < 1 ||
        a->head_dim < 1)
        return 0;
    const int groups = groups_of(a);
    return acc_bytes(a, groups) + (size_t)groups * 2 * a->n_heads_q * sizeof(float2) + kWsAlign;
}

extern "C" sonic_status_t sonic_attn_decode_kv4(const uint16_t *q, const sonic_kv4_cache *cache,
                                                const int32_t *lens, uint16_t *O,
                                                const sonic_decode_kv4_args *a,
                                                sonic_stream_t stream_) {
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (a == nullptr || a->batch < 0 || a->n_layers < 1 || a->n_heads_kv < 1 || a->n_heads_q < 1 ||
        a->n_heads_q % a->n_heads_kv != 0 || a->max_len < 0)
        return SONIC_ERR_INVALID_ARGUMENT;
    const int D = a->head_dim, G = a->n_heads_q / a->n_heads_kv;
    if (D != 64 && D != 128) return SONIC_ERR_UNSUPPORTED;
    if (G > 16) return SONIC_ERR_UNSUPPORTED;
    if (a->batch == 0) return SONIC_OK;
    if (q == nullptr || lens == nullptr || O == nullptr || a->kv_start == nullptr)
        return SONIC_ERR_INVALID_ARGUMENT;
    const sonic_status_t st = check_kv4(cache, a->n_layers, D, true);
    if (st != SONIC_OK) return st;
    if (!aligned16(q) || (reinterpret_cast<uintptr_t>(O) & 3) != 0) return SONIC_ERR_INVALID_ARGUMENT;
    if (a->n_layers > 1 && (a->q_layer_stride % 8 != 0 || a->o_layer_stride % 2 != 0))
        return SONIC_ERR_INVALID_ARGUMENT;
    if ((int64_t)a->n_layers * a->batch * a->n_heads_q > 0x7fffffffLL) return SONIC_ERR_UNSUPPORTED;
    const size_t need = sonic_decode_kv4_workspace_size(a);
    if (a->workspace == nullptr || a->workspace_bytes < need) return SONIC_ERR_WORKSPACE;

    Params p{};
    p.q = q;
    p.kc = cache->k_codes;
    p.ks = cache->k_scales;
    p.vc = cache->v_codes;
    p.vs = cache->v_scales;
    p.O = O;
    p.lens = lens;
    p.kv_start = a->kv_start;
    p.lse = a->lse;
    p.groups = groups_of(a);
    char *ws = reinterpret_cast<char *>(
        (reinterpret_cast<uintptr_t>(a->workspace) + kWsAlign - 1) & ~(uintptr_t)(kWsAlign - 1));
    p.part_acc = reinterpret_cast<float *>(ws);
    p.part_ml = reinterpret_cast<float2 *>(ws + acc_bytes(a, p.groups));
    p.status = a->status;
    p.B = a->batch;
    p.Hq = a->n_heads_q;
    p.Hkv = a->n_heads_kv;
    p.G = G;
    p.n_layers = a->n_layers;
    p.rows = cache->rows;
    p.max_len = a->max_len;
    p.q_ls = a->q_layer_stride;
    p.o_ls = a->o_layer_stride;
    p.codes_ls = cache->codes_layer_bytes;
    p.scales_ls = cache->scales_layer_bytes;
    const float scale = a->softmax_scale > 0.f ? a->softmax_scale : 1.0f / sqrtf((float)D);
    p.scale_log2 = scale * kLog2e;
    const int c = mode_of(a);
    const cudaError_t e = D == 128 ? (G <= 8 ? launch<128, 1>(p, c, stream) : launch<128, 2>(p, c, stream))
                                   : (G <= 8 ? launch<64, 1>(p, c, stream) : launch<64, 2>(p, c, stream));
    return e == cudaSuccess ? SONIC_OK : SONIC_ERR_CUDA;
}
