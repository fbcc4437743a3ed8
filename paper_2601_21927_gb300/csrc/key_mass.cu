// The attention weight that each cached row received (sonic_key_mass):
//   mass[t] = keep prev[t] + sum over queries i and heads h of exp(scale <q_ih, K_t> - lse_ih).
//
// The softmax is done: lse is known, so every key stands alone and K is read once, and a block
// that owns some keys adds up what concerns them, with no atomics and in a fixed order.  A block
// takes a run of keys of one sequence (of one layer and KV head; where the caller wants the sum over
// these, it works through them for its keys); runs are short enough for two waves of resident
// blocks, and at most kRunMost keys, and blocks past a sequence's end leave at once.
//
// Few query rows (a generation step; at most kStepRows of queries x heads): bound by HBM (256 bytes
// of bf16 or 72 of four-bit key at D = 128 against 2 D G flops).  Tiles of 16 keys are the M
// dimension of warp-wide 16 x 8 x 16 products; operands of q stay in registers, the next tile is in
// flight while one is worked on, warps share nothing; a key's sum is a lane's own sum over its
// columns and two shuffles.
// Windows of queries: 2 D flops and one exponential per key and row (57 kflop for 72 to 256 bytes with
// 32 rows of 7 heads), so bound by the exponentials (measured per clock and SM: 31 alone, 19 with the packed
// arithmetic around them: 7 clocks of an SM for the 128 keys of a tile and one row, where the products take 4).  S^T = K q^T on tcgen05, 128 keys
// by up to 256 rows, two accumulators in tensor memory; a thread's TMEM lane is a key, so the sum over
// rows stays in one register.  Four warps bring the next K tiles (four-bit rows are converted on
// the way) and sixteen take the exponentials: with eight, two to a scheduler, the chain from tensor
// memory to the sum was waited for (85 us for eight windows of 32 rows x 7 heads over 64k keys).
//
// Scores: the products of bf16 are exact, and those of fp16 (four-bit values, and q scaled by a power of two
// that its larger elements hold all their bits) but for q's rounding; fp32 sums.  scale s - lse is formed before the factor log2 e, so its rounding is relative to the
// small difference.
#include <algorithm>

#include "kv4_dev.cuh"
#include "sonic_host.h"

namespace sonic {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;
constexpr int kStepRows = 16;     // query rows (queries x heads of a group) kept in registers
constexpr int kWindowRows = 256;  // query rows of one product
constexpr int kRunMost = 2048;    // keys of a block
constexpr int kTile = 128;        // keys of a step of a block: 8 warps' 16, or one product's
// (a tile's rows are counted in 32 bits, up to a tile past a sequence's last)
constexpr int kMostRows = 0x7fffffff - 2 * kTile;
constexpr uint32_t kInf16 = 0x7F80;  // bits of bf16's infinity

struct Params {
    const uint16_t *q, *K;
    const uint8_t *kc, *ks;
    const float *lse, *prev;
    float *mass;
    const int32_t *lens, *kv_start, *q_start, *q_len;
    int32_t *status;
    int32_t B, Hq, Hkv, G, rows, q_rows, max_len, max_q_len;
    int32_t run, runs;                // keys of a block; blocks per (layer, sequence, KV head)
    int32_t unit_layers, sum_layers;  // layers with a block each; layers added up (one of them is 1)
    int32_t unit_heads, sum_heads;    // the same of KV heads
    int64_t kv_ls, q_ls, codes_ls, scales_ls;
    float scale, keep;
};

struct Seq {
    int len, start, nq, q0;
};

// Sequence b; len 0 where it is refused.
__device__ __forceinline__ Seq seq_of(const Params &p, int b, bool tell = false) {
    Seq s;
    s.len = p.lens[b];
    s.start = p.kv_start[b];
    s.nq = p.q_len != nullptr ? p.q_len[b] : 1;
    s.q0 = p.q_start != nullptr ? p.q_start[b] : b;
    const bool empty = s.len == 0 && p.q_len == nullptr;
    const bool bad = s.len < 0 || s.len > p.max_len || s.start < 0 ||
                     (int64_t)s.start + s.len > p.rows || s.nq < 0 || s.nq > p.max_q_len ||
                     (s.nq > s.len && !empty) || s.q0 < 0 || (int64_t)s.q0 + s.nq > p.q_rows;
    if (bad) {
        if (tell) set_status(p.status, SONIC_ERR_INVALID_ARGUMENT);
        s.len = 0;
    }
    return s;
}

// What a block works on.
struct Unit {
    int layer, b, kvh, from, take;  // its first key and its keys
    Seq s;
};
__device__ __forceinline__ Unit unit_of(const Params &p) {
    Unit u;
    const int run = (int)(blockIdx.x % p.runs);
    int64_t y = blockIdx.x / p.runs;
    u.kvh = (int)(y % p.unit_heads);
    y /= p.unit_heads;
    u.b = (int)(y % p.B);
    u.layer = (int)(y / p.B);
    u.s = seq_of(p, u.b, threadIdx.x == 0 && run == 0 && u.kvh == 0 && u.layer == 0);
    u.from = run * p.run;
    u.take = min(u.s.len - u.from, p.run);
    return u;
}

// 16 keys as loaded: lane (g, c) has its parts of rows g and g + 8.  bf16: bytes 64 i + 16 c of
// each 64-byte stretch i; four bits: the c-th quarter.  Either way word pair h of part i is
// the operand of reduction step 2 i + h, for the dims dim_of(i, c) + 4 h .. + 3.
template <int D, bool k4>
struct Keys {
    uint4 k[2][D / 32];
};
template <int D>
struct Keys<D, true> {
    uint32_t k[2][D / 32];
    uint32_t s[2];
};

template <int D, bool k4>
__device__ __forceinline__ int dim_of(int i, int c) {
    return k4 ? c * (D / 4) + 8 * i : 32 * i + 8 * c;
}

// This lane's address in the keys (or, four bits, the scales) of the tile from `row` on.
template <int D, bool k4>
__device__ __forceinline__ const uint8_t *key_base(const Params &p, int layer, int kvh, int64_t row, bool scales) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    if constexpr (k4) {
        const int64_t at = (int64_t)kvh * p.rows + row + g;
        return scales ? p.ks + layer * p.scales_ls + at * (D / 16) + c * (D / 64)
                      : p.kc + layer * p.codes_ls + at * (D / 2) + c * (D / 8);
    } else {
        return reinterpret_cast<const uint8_t *>(p.K + layer * p.kv_ls + ((row + g) * p.Hkv + kvh) * D + 8 * c);
    }
}

// The tile there, of which `n` keys are the unit's: the others repeat the last.
template <int D, bool k4>
__device__ __forceinline__ void load_keys(Keys<D, k4> &t, const uint8_t *src, const uint8_t *src_s, int64_t row_bytes,
                                          int n) {
    const int g = (threadIdx.x & 31) >> 2;
    int back = 0, step = 8;  // rows from the first to its place, and to the second
    if (n < 16) {
        back = min(0, n - 1 - g);
        step = min(8, n - 1 - g);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int by = i == 0 ? back : step;
        const uint8_t *k = src + by * row_bytes;
        if constexpr (k4) {
            const uint8_t *ks = src_s + by * (D / 16);
            if constexpr (D == 128) {
                const uint4 v = ld_once16(k);
                t.k[i][0] = v.x;
                t.k[i][1] = v.y;
                t.k[i][2] = v.z;
                t.k[i][3] = v.w;
                t.s[i] = *reinterpret_cast<const uint16_t *>(ks);
            } else {
                const uint2 v = ld_once8(k);
                t.k[i][0] = v.x;
                t.k[i][1] = v.y;
                t.s[i] = *ks;
            }
        } else {
#pragma unroll
            for (int j = 0; j < D / 32; ++j) t.k[i][j] = ld_once16(k + 64 * j);
        }
    }
}

template <int D>
struct Operand {
    uint32_t a[D / 16][4];
};

template <int D, bool k4>
__device__ __forceinline__ void make_operand(const Keys<D, k4> &t, Operand<D> &o) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            uint32_t w[4];
            if constexpr (k4) {
                kv4_decode4(t.k[r][i], w);
                const uint32_t s = kv4_scale_f16x2(D == 128 && i >= 2 ? t.s[r] >> 8 : t.s[r] & 0xFFu);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = mul_f16x2(w[e], s);
            } else {
                w[0] = t.k[r][i].x;
                w[1] = t.k[r][i].y;
                w[2] = t.k[r][i].z;
                w[3] = t.k[r][i].w;
            }
            o.a[2 * i][r] = w[0];
            o.a[2 * i][2 + r] = w[1];
            o.a[2 * i + 1][r] = w[2];
            o.a[2 * i + 1][2 + r] = w[3];
        }
    }
}

template <bool k4>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (k4) {
        mma_f16(c, a[0], a[1], a[2], a[3], b0, b1);
    } else {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
            "{%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
}

// Scores of 16 keys and 8 query rows.
template <int D, bool k4>
__device__ __forceinline__ void scores(float (&s)[4], const Operand<D> &o, const uint32_t (&qf)[D / 16][2]) {
    float h[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
        mma<k4>(s, o.a[k], qf[k][0], qf[k][1]);
        mma<k4>(h, o.a[D / 32 + k], qf[D / 32 + k][0], qf[D / 32 + k][1]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += h[e];
}

// Query row `row` of a (layer, sequence, KV head): query row / G, head row % G of the group.
__device__ __forceinline__ int64_t q_index(const Params &p, const Seq &s, int kvh, int row) {
    return (int64_t)(s.q0 + row / p.G) * p.Hq + kvh * p.G + row % p.G;
}

// A quarter of a query row (dims dim_of(0..D/32 - 1, c) + 0..7) as operand words; k4: fp16,
// scaled by 2^up so that the row's largest element lies in [2^13, 2^14).  Returns the factor
// from products to scores.  The four lanes of a row call it together.
template <int D, bool k4>
__device__ __forceinline__ float q_words(const Params &p, const uint16_t *row, bool none, int c, uint32_t (&w)[D / 8]) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row != nullptr) x = *reinterpret_cast<const uint4 *>(row + dim_of<D, k4>(i, c));
        w[4 * i] = x.x;
        w[4 * i + 1] = x.y;
        w[4 * i + 2] = x.z;
        w[4 * i + 3] = x.w;
    }
    if (none)  // (after the loads, so that these need not wait for its lse)
#pragma unroll
        for (int i = 0; i < D / 8; ++i) w[i] = 0;
    if constexpr (!k4) return p.scale;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int up = min(max(13 - ((int)(top >> 7) - 127), -126), 126);
    const float k = __int_as_float((127 + up) << 23);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) w[i] = pack_f16x2(bf16lo(w[i]) * k, bf16hi(w[i]) * k);
    return p.scale * __int_as_float((127 - up) << 23);
}

// -lse; -inf for a row that saw nothing (lse = -inf): like a row that is none, it has zeros for q, sees no
// key where keys are told apart, and adds nothing.
__device__ __forceinline__ float neg_lse(float lse) { return lse == -INFINITY ? -INFINITY : -lse; }

__device__ __forceinline__ float weight(float s, float f, float nl) {
    return ex2(fmaf(s, f, nl) * kLog2e);
}

// Rows of queries in registers (NT * 8 of them at most); a warp per tile of 16 keys, every kTile keys.
// kSum: the weights of several layers or heads are added up.
// (Four-bit keys: a third block on the SM, 85 registers, 57 us for 64 sequences up to 16,384 rows x 2 layers
// where two took 73 and a fourth 62; bf16 tiles fill the registers of two.)
template <int D, bool k4, int NT, bool kSum>
__global__ void __launch_bounds__(kThreads, k4 && NT == 1 && !kSum ? 3 : 2) mass_step_kernel(const Params p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    pdl_wait();
    pdl_trigger();
    const Unit u = unit_of(p);
    const Seq &s = u.s;
    if (u.take <= 16 * warp) return;
    const int rows = s.nq * p.G, row0 = s.start + u.from + 16 * warp, mine = u.take - 16 * warp;
    // (tile, layer, head), the heads fastest; the next one's keys are in flight
    const int sums = kSum ? p.sum_layers * p.sum_heads : 1;
    const int total = (mine + kTile - 1) / kTile * sums;
    const uint8_t *src = key_base<D, k4>(p, u.layer, u.kvh, row0, false);
    const uint8_t *src_s = k4 ? key_base<D, k4>(p, u.layer, u.kvh, row0, true) : nullptr;
    const int64_t row_bytes = k4 ? D / 2 : (int64_t)p.Hkv * D * 2;
    int ahead = mine, a_layer = u.layer, a_kvh = u.kvh;  // keys from the next tile to load on
    auto load = [&](Keys<D, k4> &t) {
        if (kSum) {
            const int r = row0 + mine - ahead;
            src = key_base<D, k4>(p, a_layer, a_kvh, r, false);
            if (k4) src_s = key_base<D, k4>(p, a_layer, a_kvh, r, true);
            bool end = true;
            if (p.sum_heads > 1) {
                end = ++a_kvh == p.sum_heads;
                if (end) a_kvh = 0;
            }
            if (end && p.sum_layers > 1) {
                end = ++a_layer == p.sum_layers;
                if (end) a_layer = 0;
            }
            load_keys<D, k4>(t, src, src_s, row_bytes, ahead);
            if (end) ahead -= kTile;
        } else {
            load_keys<D, k4>(t, src, src_s, row_bytes, ahead);
            ahead -= kTile;
            src += kTile * row_bytes;
            if (k4) src_s += kTile * (D / 16);
        }
    };
    Keys<D, k4> cur, nxt;
    load(cur);
    uint32_t qf[NT][D / 16][2];
    float f[NT][2], nl[NT][2];
    int limit[NT][2];  // the last key that the lane's query rows see
    bool blind = false;  // some row saw nothing, or there is no row: the keys may hold anything for it
    auto load_q = [&](int layer, int kvh) {
        bool sees_none = rows == 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = nt * 8 + g;
            const int64_t at = row < rows ? q_index(p, s, kvh, row) : 0;
            const float neg = row < rows ? neg_lse(p.lse[(int64_t)layer * p.q_rows * p.Hq + at]) : -INFINITY;
            const bool none = neg == -INFINITY;  // (a row that saw nothing may hold anything)
            uint32_t x[D / 8];
            const float back = q_words<D, k4>(p, row < rows ? p.q + layer * p.q_ls + at * D : nullptr, none, c, x);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                qf[nt][i][0] = x[2 * i];
                qf[nt][i][1] = x[2 * i + 1];
            }
            const int sees = none ? -1 : s.len - s.nq + row / p.G;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f[nt][e] = __shfl_sync(0xffffffffu, back, 8 * c + 4 * e);
                nl[nt][e] = __shfl_sync(0xffffffffu, neg, 8 * c + 4 * e);
                limit[nt][e] = __shfl_sync(0xffffffffu, sees, 8 * c + 4 * e);
                sees_none |= limit[nt][e] < 0 && nt * 8 + 2 * c + e < rows;
            }
        }
        blind = __any_sync(0xffffffffu, sees_none);
    };
    if (!kSum) load_q(u.layer, u.kvh);
    // lanes 4 g and 4 g + 1 write rows g and g + 8
    const bool reads = p.prev != nullptr && p.keep != 0.f;
    const int row = c == 0 ? g : g + 8;
    const int64_t out = ((int64_t)u.layer * p.unit_heads + u.kvh) * p.rows + row0 + row;
    float *mass = p.mass + out;
    const float *prev = reads ? p.prev + out : nullptr;
    float lo = 0.f, hi = 0.f;
    int left = mine, done = 0;  // keys from this tile on; (layer, head) pairs of it added
    for (int it = 0; it < total; ++it) {
        const bool writes = c < 2 && row < left;
        float before = 0.f;
        if (reads && writes) before = *prev;
        if (it + 1 < total) load(nxt);
        if (kSum) load_q(p.sum_layers > 1 ? done / p.sum_heads : u.layer, p.sum_heads > 1 ? done % p.sum_heads : u.kvh);
        Operand<D> o;
        make_operand<D, k4>(cur, o);
        const int pos = s.len - left - (s.len - u.from - u.take);  // the tile's first key in the sequence
        const bool cut = blind || pos + 16 > s.len - s.nq + 1;  // some query does not see some key
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float x[4];
            scores<D, k4>(x, o, qf[nt]);
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = weight(x[e], f[nt][e & 1], nl[nt][e & 1]);
            if (cut)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pos + g + 8 * (e >> 1) <= limit[nt][e & 1] ? w[e] : 0.f;
            lo += w[0] + w[1];
            hi += w[2] + w[3];
        }
        cur = nxt;
        if (kSum && ++done < sums) continue;
        lo += __shfl_xor_sync(0xffffffffu, lo, 1);
        hi += __shfl_xor_sync(0xffffffffu, hi, 1);
        lo += __shfl_xor_sync(0xffffffffu, lo, 2);
        hi += __shfl_xor_sync(0xffffffffu, hi, 2);
        if (writes) *mass = fmaf(p.keep, before, c == 0 ? lo : hi);
        lo = hi = 0.f;
        done = 0;
        left -= kTile;
        mass += kTile;
        if (reads) prev += kTile;
    }
}

// ---- windows of queries on tcgen05

constexpr int kEpilogue = 512;   // threads: four groups of 128, a TMEM lane (a key) each
constexpr int kProducer = 128;
constexpr int kWinThreads = kEpilogue + kProducer + 32;

template <int D, bool k4>
struct Win {
    // K tiles in shared memory: converted ones come from registers, bf16 ones by cp.async, which needs
    // a third to have two on their way
    static constexpr int kKStages = k4 ? 2 : 3;
    static constexpr int kKBytes = kTile * D * 2;  // an operand tile: [D / 64][128 keys][128 bytes], swizzled
    static constexpr int kOffQ = kKStages * kKBytes;  // q: [D / 64][N rows][128 bytes], swizzled
};

// Shared memory of a window kernel of N rows: operands, sums by (quarter of the rows, key), -lse, the
// last visible key and the factor to scores by row, barriers.
struct WinLayout {
    int acc, nl, last, f, bars, total;
};
template <int D, bool k4>
__host__ __device__ constexpr WinLayout win_layout(int N) {
    WinLayout w{};
    w.acc = Win<D, k4>::kOffQ + N * D * 2;
    w.nl = w.acc + 4 * kRunMost * 4;
    w.last = w.nl + kWindowRows * 4;
    w.f = w.last + kWindowRows * 4;
    w.bars = w.f + kWindowRows * 4;
    w.total = w.bars + 16 * 8;
    return w;
}

constexpr uint32_t idesc_f16_f32(uint32_t M, uint32_t N) {  // kind::f16 with fp16 operands, K-major
    return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

// Chunk j (16 bytes, 8 dims) of row r of an operand with `rows` rows.
__device__ __forceinline__ uint32_t swizzled(int rows, int r, int j) {
    return (uint32_t)((j >> 3) * rows * 128 + r * 128 + (((j & 7) ^ (r & 7)) << 4));
}

__device__ __forceinline__ void sts16(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

// Row t of a four-bit K tile as loaded, and as an operand.
template <int D>
struct Raw {
    uint4 k[D / 32];
    uint2 s;
};

template <int D>
__device__ __forceinline__ void load_raw(Raw<D> &x, const Params &p, int layer, int kvh, int64_t row) {
    const int64_t at = (int64_t)kvh * p.rows + row;
    const uint4 *kc = reinterpret_cast<const uint4 *>(p.kc + layer * p.codes_ls + at * (D / 2));
    const uint8_t *ks = p.ks + layer * p.scales_ls + at * (D / 16);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) x.k[i] = kc[i];
    x.s.x = ld_once4(ks);
    x.s.y = D == 128 ? ld_once4(ks + (D == 128 ? 4 : 0)) : 0;
}

template <int D>
__device__ __forceinline__ void store_raw(const Raw<D> &x, uint32_t base, int t) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const uint32_t w[4] = {x.k[i].x, x.k[i].y, x.k[i].z, x.k[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // eight codes: one chunk; two chunks to a scale
            const int blk = 2 * i + (j >> 1);
            const uint32_t sc = kv4_scale_f16x2(((blk < 4 ? x.s.x : x.s.y) >> (blk % 4 * 8)) & 0xFFu);
            uint32_t r[4];
            kv4_decode4(w[j], r);
            sts16(base + swizzled(kTile, t, 4 * i + j),
                  make_uint4(mul_f16x2(r[0], sc), mul_f16x2(r[1], sc), mul_f16x2(r[2], sc), mul_f16x2(r[3], sc)));
        }
    }
}

// A bf16 K tile by cp.async: 16-byte chunk t % (D / 8) of every (1024 / D)-th row.
template <int D>
__device__ __forceinline__ void copy_tile(const Params &p, int layer, int kvh, int row0, int last, uint32_t base,
                                          int t) {
    constexpr int kChunks = D / 8, kStep = kProducer / kChunks;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int r = t / kChunks + i * kStep;
        const uint16_t *src = p.K + layer * p.kv_ls + ((int64_t)min(row0 + r, last) * p.Hkv + kvh) * D + t % kChunks * 8;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + swizzled(kTile, r, t % kChunks)), "l"(src)
                     : "memory");
    }
}

// Sum of the weights of one key (a TMEM lane) over the 32 query rows from c0 on, and every 128th 32 after
// them, f the factor from products to scores; kCut: rows that do not see the key add nothing; kOwn:
// each row has a factor of its own.  Per two rows: three packed instructions, two exponentials and half a
// 16-byte read of -lse.  (With kOwn for all tiles the reads, 512 bytes to a warp each, were the bound: 9
// clocks of a scheduler per row and warp.)
template <bool kCut, bool kOwn>
__device__ __forceinline__ float sum_rows(uint32_t scores, int c0, int N, float f, const float *s_nl, const int *s_last,
                                          const float *s_f, int pos) {
    const uint64_t ff = (uint64_t)__float_as_uint(f) << 32 | __float_as_uint(f);
    constexpr uint64_t kLog2e2 = 0x3FB8AA3B3FB8AA3Bull;  // log2 e twice
    uint64_t sum[2] = {0, 0};
#pragma unroll 1
    for (; c0 < N; c0 += kEpilogue / 4) {
        uint32_t x[32];
        tmem_ld32(scores + c0, x);
        tmem_ld_wait();
        reg_fence32(x);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const ulonglong2 nl = *reinterpret_cast<const ulonglong2 *>(s_nl + c0 + i);
            ulonglong2 fs = make_ulonglong2(ff, ff);
            if (kOwn) fs = *reinterpret_cast<const ulonglong2 *>(s_f + c0 + i);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint64_t w;
                asm("{\n\t.reg .b64 x, y;\n\t"
                    "mov.b64 x, {%1, %2};\n\t"
                    "fma.rn.f32x2 y, x, %3, %4;\n\t"
                    "mul.rn.f32x2 %0, y, %5;\n\t}"
                    : "=l"(w)
                    : "r"(x[i + 2 * h]), "r"(x[i + 2 * h + 1]), "l"((uint64_t)(h == 0 ? fs.x : fs.y)),
                      "l"((uint64_t)(h == 0 ? nl.x : nl.y)), "l"(kLog2e2));
                float a = ex2(__uint_as_float((uint32_t)w)), b = ex2(__uint_as_float((uint32_t)(w >> 32)));
                if (kCut) {
                    const int2 lim = *reinterpret_cast<const int2 *>(s_last + c0 + i + 2 * h);
                    a = pos <= lim.x ? a : 0.f;
                    b = pos <= lim.y ? b : 0.f;
                }
                asm("{\n\t.reg .b64 x;\n\t"
                    "mov.b64 x, {%1, %2};\n\t"
                    "add.rn.f32x2 %0, %0, x;\n\t}"
                    : "+l"(sum[h])
                    : "f"(a), "f"(b));
            }
        }
    }
    auto both = [](uint64_t v) { return __uint_as_float((uint32_t)v) + __uint_as_float((uint32_t)(v >> 32)); };
    return both(sum[0]) + both(sum[1]);
}

template <int D, bool k4>
__global__ void __launch_bounds__(kWinThreads, 1) mass_window_kernel(const Params p, int N, int tmem_cols) {
    using W = Win<D, k4>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const WinLayout lay = win_layout<D, k4>(N);
    float *acc = reinterpret_cast<float *>(smem + lay.acc);  // [4][kRunMost]
    float *s_nl = reinterpret_cast<float *>(smem + lay.nl);
    int *s_last = reinterpret_cast<int *>(smem + lay.last);
    float *s_f = reinterpret_cast<float *>(smem + lay.f);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + lay.bars);
    uint64_t *k_full = bars, *k_empty = bars + W::kKStages;  // a K tile is in place / its product is done
    uint64_t *s_full = bars + 2 * W::kKStages;               // [2] a tile's scores are in their accumulator
    uint64_t *s_empty = s_full + 2;                          // [2] read out
    uint64_t *q_full = s_empty + 2, *idle = q_full + 1;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_dead;
    __shared__ uint32_t s_top[2];
    __shared__ int s_apart[2];  // some row of a stage saw nothing, or has a factor of its own
    volatile int *abort_flag = &s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    const Unit u = unit_of(p);
    if (u.take <= 0) return;
    const Seq &s = u.s;
    const int rows = s.nq * p.G;
    if (tid == 0) {
        for (int i = 0; i < W::kKStages; ++i) {
            mbar_init(&k_full[i], kProducer);
            mbar_init(&k_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], kEpilogue);
        }
        mbar_init(q_full, kEpilogue);
        mbar_init(idle, 1);
        s_abort = 0;
        s_top[0] = s_top[1] = 0;
        s_apart[0] = s_apart[1] = rows == 0;
        s_dead = timed_out(p.status);
        fence_mbar_init();
    }
    if (warp == kWinThreads / 32 - 1) {
        tmem_alloc(&s_tmem, (uint32_t)tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // only now: a kernel behind this one may hold tensor memory while it waits for this one's end, and
    // a block here that then asked for its own would wait for that
    pdl_trigger();
    const uint32_t tmem = s_tmem;
    const int row0 = s.start + u.from, last = row0 + u.take - 1;
    const int tiles = (u.take + kTile - 1) / kTile;
    const int chunks = max(1, (rows + N - 1) / N);
    // stage k: the query rows of one chunk of one (layer, head), against every tile
    const int stages = s_dead ? 0 : p.sum_layers * p.sum_heads * chunks;
    auto layer_of = [&](int st) { return p.sum_layers > 1 ? st / chunks / p.sum_heads : u.layer; };
    auto head_of = [&](int st) { return p.sum_heads > 1 ? st / chunks % p.sum_heads : u.kvh; };
    const uint32_t k_base = smem_u32(smem), q_base = k_base + W::kOffQ;
    if (warp < kEpilogue / 32) {
        // ------------------------------------------------------------ exponentials
        // All sixteen warps take a tile together: warps w, w + 4, .. have the same keys and every fourth
        // 32 of the rows each.  (In two groups with a tile each, both waited for products at once.)
        const int part = warp >> 2, key = (warp & 3) * 32 + lane;
        float *mine = acc + part * kRunMost;
        int T = 0;
        bool ok = true;
        for (int st = 0; st < stages; ++st) {
            // q, four threads to a row, a quarter of its chunks each: the products of the stage before
            // are done and its -lse read once all threads are here
            if (st > 0) named_barrier(1, kEpilogue);
            const int layer = layer_of(st), kvh = head_of(st), r0 = st % chunks * N, n = min(N, rows - r0);
            constexpr int kItems = kWindowRows * 4 / kEpilogue;
            uint32_t x[kItems][D / 8];
#pragma unroll
            for (int v = 0; v < kItems; ++v) {
                const int i = tid + v * kEpilogue, j = i >> 2, quarter = i & 3;
                const int64_t at = j < n ? q_index(p, s, kvh, r0 + j) : 0;
                const float neg = j < n ? neg_lse(p.lse[(int64_t)layer * p.q_rows * p.Hq + at]) : -INFINITY;
                const bool none = neg == -INFINITY;  // (a row that saw nothing may hold anything)
                if (none && j < n) s_apart[st & 1] = 1;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (j < n) w = *reinterpret_cast<const uint4 *>(p.q + layer * p.q_ls + at * D + 32 * k + 8 * quarter);
                    x[v][4 * k] = w.x;
                    x[v][4 * k + 1] = w.y;
                    x[v][4 * k + 2] = w.z;
                    x[v][4 * k + 3] = w.w;
                }
                if (none)
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) x[v][k] = 0;
                if (quarter == 0 && j < N) {
                    s_nl[j] = neg;
                    s_last[j] = none ? -1 : s.len - s.nq + (r0 + j) / p.G;
                }
            }
            float f = p.scale;
            if constexpr (k4) {
                // fp16, scaled by 2^up so that the largest element lies in [2^13, 2^14): one factor for all rows (see
                // sum_rows), but one of its own for a row whose largest lies more than 12 powers of two below.  So a
                // row's largest lies at 2 or above and its elements, off by at most 2^-25, by 2^-26 of it;
                // a score by 2^-26 max |q_d| sum |k_d| scale.
                uint32_t most[kItems], top = 0;  // largest finite magnitudes, as bf16 bits: of this quarter, of all rows
#pragma unroll
                for (int v = 0; v < kItems; ++v) {
                    uint32_t m = 0;
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) m = max(m, max(x[v][k] & 0x7FFFu, (x[v][k] >> 16) & 0x7FFFu));
                    if (m >= kInf16) {
                        // NaN or infinities stay in their row: all are scaled as if they were not there
                        m = 0;
#pragma unroll
                        for (int k = 0; k < D / 8; ++k) {
                            const uint32_t lo = x[v][k] & 0x7FFFu, hi = (x[v][k] >> 16) & 0x7FFFu;
                            m = max(m, max(lo < kInf16 ? lo : 0, hi < kInf16 ? hi : 0));
                        }
                    }
                    most[v] = m;
                    top = max(top, m);
                }
                top = __reduce_max_sync(0xffffffffu, top);
                if (lane == 0) atomicMax(&s_top[st & 1], top);
                named_barrier(1, kEpilogue);
                top = s_top[st & 1];
                if (tid == 0) s_top[st + 1 & 1] = 0;  // (read by all before this barrier)
#pragma unroll
                for (int v = 0; v < kItems; ++v) {
                    const int i = tid + v * kEpilogue;
                    uint32_t e = top >> 7;
                    if (__any_sync(0xffffffffu, (most[v] >> 7) + 12 < e)) {
                        uint32_t own = max(most[v], __shfl_xor_sync(0xffffffffu, most[v], 1));
                        own = max(own, __shfl_xor_sync(0xffffffffu, own, 2));
                        if (own > 0 && (own >> 7) + 12 < e) {
                            e = own >> 7;
                            s_apart[st & 1] = 1;
                        }
                    }
                    const int up = min(max(13 - ((int)e - 127), -126), 126);
                    const float scale = __int_as_float((127 + up) << 23);
                    f = p.scale * __int_as_float((127 - up) << 23);
                    if ((i & 3) == 0 && i < N * 4) s_f[i >> 2] = f;
#pragma unroll
                    for (int k = 0; k < D / 8; ++k)
                        x[v][k] = pack_f16x2(bf16lo(x[v][k]) * scale, bf16hi(x[v][k]) * scale);
                }
                const int up = min(max(13 - ((int)(top >> 7) - 127), -126), 126);
                f = p.scale * __int_as_float((127 - up) << 23);
            }
#pragma unroll
            for (int v = 0; v < kItems; ++v) {
                const int i = tid + v * kEpilogue;
                if (i < N * 4)
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)
                        sts16(q_base + swizzled(N, i >> 2, 4 * k + (i & 3)),
                              make_uint4(x[v][4 * k], x[v][4 * k + 1], x[v][4 * k + 2], x[v][4 * k + 3]));
            }
            if (tid == 0) s_apart[st + 1 & 1] = rows == 0;  // (its readers are past the barrier above)
            fence_proxy_async_smem();
            mbar_arrive(q_full);
            // (a warp goes on, or gives up, as one: tensor memory is read by whole warps)
            ok = ok && __all_sync(0xffffffffu, mbar_wait(q_full, st & 1, p.status, abort_flag));
            const bool apart = s_apart[st & 1];
            for (int t = 0; ok && t < tiles; ++t, ++T) {
                const int at = t * kTile + key, pos = u.from + at;  // the key's row in the sequence
                ok = __all_sync(0xffffffffu, mbar_wait(&s_full[T & 1], (T >> 1) & 1, p.status, abort_flag));
                if (!ok) break;
                tc_fence_after();
                // (whether some query does not see some key of the tile: a loop of its own, so that the
                // common one has no branch between its columns)
                const uint32_t tS = tmem + (T & 1) * (tmem_cols / 2) + ((uint32_t)(warp & 3) << 21);
                const bool cut = apart || u.from + t * kTile + kTile > s.len - s.nq + 1;
                const float sum = cut ? sum_rows<true, k4>(tS, 32 * part, N, f, s_nl, s_last, s_f, pos)
                                      : sum_rows<false, false>(tS, 32 * part, N, f, s_nl, s_last, s_f, pos);
                tc_fence_before();
                mbar_arrive(&s_empty[T & 1]);
                mine[at] = st > 0 ? mine[at] + sum : sum;
            }
        }
        // a warp that gave up leaves its part of every sum out: then the block writes none of its entries
        const bool none = named_barrier_or(1, kEpilogue, !ok);
        if (!none && stages > 0) {
            const int64_t out = ((int64_t)u.layer * p.unit_heads + u.kvh) * p.rows + row0;
            const bool reads = p.prev != nullptr && p.keep != 0.f;
            for (int at = tid; at < u.take; at += kEpilogue) {
                const float before = reads ? p.prev[out + at] : 0.f;
                const float sum = (acc[at] + acc[kRunMost + at]) + (acc[2 * kRunMost + at] + acc[3 * kRunMost + at]);
                p.mass[out + at] = fmaf(p.keep, before, sum);
            }
        }
    } else if (warp < (kEpilogue + kProducer) / 32) {
        // ------------------------------------------------------------ operands
        // tiles in the order of their products: T = stage * tiles + tile, two of them on their way
        const int t0 = tid - kEpilogue, total = stages * tiles;
        constexpr int S = W::kKStages;
        bool ok = true;
        auto free_stage = [&](int T) {
            return T < S || mbar_wait(&k_empty[T % S], (T / S - 1) & 1, p.status, abort_flag);
        };
        if constexpr (k4) {
            auto load = [&](Raw<D> &x, int T) {
                if (T >= total) return;
                const int st = T / tiles, t = T - st * tiles;
                load_raw<D>(x, p, layer_of(st), head_of(st), min(row0 + t * kTile + t0, last));
            };
            Raw<D> raw[2];
            load(raw[0], 0);
            load(raw[1], 1);
            for (int T = 0; ok && T < total; T += 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!ok || T + h >= total) break;
                    ok = free_stage(T + h);
                    if (!ok) break;
                    store_raw<D>(raw[h], k_base + h * W::kKBytes, t0);  // (two stages: h is the tile's)
                    fence_proxy_async_smem();
                    mbar_arrive(&k_full[h]);
                    load(raw[h], T + h + 2);
                }
            }
        } else {
            // tile T + 2 is sent for before tile T is handed over
            auto send = [&](int T) {
                if (T < total) {
                    ok = ok && free_stage(T);
                    const int st = T / tiles, t = T - st * tiles;
                    if (ok)
                        copy_tile<D>(p, layer_of(st), head_of(st), row0 + t * kTile, last,
                                     k_base + T % S * W::kKBytes, t0);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            send(0);
            send(1);
            for (int T = 0; ok && T < total; ++T) {
                send(T + 2);
                if (!ok) break;
                asm volatile("cp.async.wait_group 2;" ::: "memory");
                fence_proxy_async_smem();
                mbar_arrive(&k_full[T % S]);
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
    } else if (lane == 0) {
        // ------------------------------------------------------------ products
        const uint32_t id = k4 ? idesc_f16_f32(kTile, (uint32_t)N) : idesc_bf16_f32(kTile, (uint32_t)N, 0, 0);
        constexpr int S = W::kKStages;
        // (descriptors as a fixed one and offsets: formed anew, the eight of a tile took 1,000 clocks)
        const uint32_t k_lo = sw128_desc_lo(k_base, 16), q_lo = sw128_desc_lo(q_base, 16);
        const uint32_t hi = sw128_desc_hi(1024), half_q = (uint32_t)N * 128 >> 4;
        int T = 0;
        bool ok = true;
        for (int st = 0; ok && st < stages; ++st) {
            ok = mbar_wait(q_full, st & 1, p.status, abort_flag);
            for (int t = 0; ok && t < tiles; ++t, ++T) {
                const int k = T % S, b = T & 1;
                ok = mbar_wait(&k_full[k], (T / S) & 1, p.status, abort_flag) &&
                     (T < 2 || mbar_wait(&s_empty[b], ((T >> 1) - 1) & 1, p.status, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + b * (tmem_cols / 2), lo_k = k_lo + k * (W::kKBytes >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    tc_mma_ss(d, desc_join(lo_k + (kk >> 2) * (kTile * 128 >> 4) + (kk & 3) * 2, hi),
                              desc_join(q_lo + (kk >> 2) * half_q + (kk & 3) * 2, hi), id, kk > 0 ? 1u : 0u);
                tc_commit(&s_full[b]);
                tc_commit(&k_empty[k]);
            }
        }
        // nothing of this block's is in flight when its memory goes
        tc_commit(idle);
        mbar_drain(idle, 0);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kWinThreads / 32 - 1) tmem_dealloc(tmem, (uint32_t)tmem_cols);
}

template <int D, bool k4>
sonic_status_t launch(Params &p, cudaStream_t stream) {
    const int64_t rows = (int64_t)std::max(p.max_q_len, 1) * p.G;
    const bool window = rows > kStepRows;
    const int64_t units = (int64_t)p.unit_layers * p.B * p.unit_heads, max_len = std::max(p.max_len, 1);
    const int64_t resident = (int64_t)device_sm_count() * (window ? 1 : 2);
    const int64_t even = (units * max_len + 2 * resident - 1) / (2 * resident);
    p.run = (int32_t)std::min<int64_t>(kRunMost, (even + kTile - 1) / kTile * kTile);
    p.runs = (int32_t)((max_len + p.run - 1) / p.run);
    if (units * p.runs > 0x7fffffffLL) return SONIC_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(units * p.runs));
    cudaError_t e;
    if (!window) {
        const bool sum = p.sum_layers * p.sum_heads > 1;
        auto kern = rows <= 8 ? (sum ? mass_step_kernel<D, k4, 1, true> : mass_step_kernel<D, k4, 1, false>)
                              : (sum ? mass_step_kernel<D, k4, 2, true> : mass_step_kernel<D, k4, 2, false>);
        e = launch_pdl(kern, grid, kThreads, 0, stream, 1, p);
    } else {
        const int N = (int)std::min<int64_t>(kWindowRows, (rows + 31) / 32 * 32);
        int cols = 32;
        while (cols < 2 * N) cols *= 2;
        // (more than half of tensor memory: no second block on the SM, which would wait for it)
        const int smem = std::max(win_layout<D, k4>(N).total + 1024, cols > 256 ? 120 * 1024 : 0);
        auto kern = mass_window_kernel<D, k4>;
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 std::max(win_layout<D, k4>(kWindowRows).total + 1024, 120 * 1024));
        if (e == cudaSuccess) e = launch_pdl(kern, grid, kWinThreads, smem, stream, 1, p, N, cols);
    }
    return e == cudaSuccess ? SONIC_OK : SONIC_ERR_CUDA;
}

}  // namespace
}  // namespace sonic

using namespace sonic;

extern "C" sonic_status_t sonic_key_mass(const uint16_t *q, const uint16_t *K,
                                         const sonic_kv4_cache *cache, const float *lse,
                                         const int32_t *lens, float *mass,
                                         const sonic_key_mass_args *a, sonic_stream_t stream_) {
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (a == nullptr || a->batch < 0 || a->n_layers < 1 || a->n_heads_kv < 1 || a->n_heads_q < 1 ||
        a->n_heads_q % a->n_heads_kv != 0 || a->max_len < 0 || a->max_q_len < 0 ||
        a->total_kv_rows < 0 || a->total_q_rows < 0)
        return SONIC_ERR_INVALID_ARGUMENT;
    if ((a->mass_layers != 1 && a->mass_layers != a->n_layers) ||
        (a->mass_heads != 1 && a->mass_heads != a->n_heads_kv))
        return SONIC_ERR_INVALID_ARGUMENT;
    const int D = a->head_dim;
    if (D != 64 && D != 128) return SONIC_ERR_UNSUPPORTED;
    if (a->batch == 0 || a->total_kv_rows == 0) return SONIC_OK;  // no entry to write
    if (q == nullptr || lse == nullptr || lens == nullptr || mass == nullptr || a->kv_start == nullptr ||
        (K == nullptr) == (cache == nullptr))
        return SONIC_ERR_INVALID_ARGUMENT;
    if ((a->q_len == nullptr) != (a->q_start == nullptr) || !aligned16(q) ||
        (a->n_layers > 1 && a->q_layer_stride % 8 != 0))
        return SONIC_ERR_INVALID_ARGUMENT;
    if (K != nullptr) {
        if (!aligned16(K) || (a->n_layers > 1 && a->kv_layer_stride % 8 != 0))
            return SONIC_ERR_INVALID_ARGUMENT;
    } else {
        const sonic_status_t st = check_kv4(cache, a->n_layers, D, false);
        if (st != SONIC_OK) return st;
        if (cache->rows != a->total_kv_rows) return SONIC_ERR_INVALID_ARGUMENT;
    }
    if (a->total_kv_rows > kMostRows ||
        (int64_t)std::max(a->max_q_len, 1) * (a->n_heads_q / a->n_heads_kv) > 0x7fffffffLL)
        return SONIC_ERR_UNSUPPORTED;
    Params p{};
    p.q = q;
    p.K = K;
    if (cache != nullptr) {
        p.kc = cache->k_codes;
        p.ks = cache->k_scales;
        p.codes_ls = cache->codes_layer_bytes;
        p.scales_ls = cache->scales_layer_bytes;
    }
    p.lse = lse;
    p.prev = a->prev;
    p.mass = mass;
    p.lens = lens;
    p.kv_start = a->kv_start;
    p.q_start = a->q_start;
    p.q_len = a->q_len;
    p.status = a->status;
    p.B = a->batch;
    p.Hq = a->n_heads_q;
    p.Hkv = a->n_heads_kv;
    p.G = a->n_heads_q / a->n_heads_kv;
    p.rows = a->total_kv_rows;
    p.q_rows = a->total_q_rows;
    p.max_len = a->max_len;
    p.max_q_len = a->q_len != nullptr ? a->max_q_len : 1;
    p.unit_layers = a->mass_layers;
    p.sum_layers = a->mass_layers == a->n_layers ? 1 : a->n_layers;
    p.unit_heads = a->mass_heads;
    p.sum_heads = a->mass_heads == a->n_heads_kv ? 1 : a->n_heads_kv;
    p.kv_ls = a->kv_layer_stride;
    p.q_ls = a->q_layer_stride;
    p.scale = a->softmax_scale > 0.f ? a->softmax_scale : 1.0f / sqrtf((float)D);
    p.keep = a->prev != nullptr ? a->keep : 0.f;
    if (K != nullptr) return D == 128 ? launch<128, false>(p, stream) : launch<64, false>(p, stream);
    return D == 128 ? launch<128, true>(p, stream) : launch<64, true>(p, stream);
}
