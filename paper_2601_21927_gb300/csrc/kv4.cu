// Four-bit rows of a KV cache: packed from bf16 rows (sonic_kv4_store, sonic_kv4_compact) and
// unpacked again (sonic_kv4_load).  The format is in kv4_dev.cuh.
//
// Both directions are streams: 2 bytes of bf16 and 0.5625 of codes and scales a value, a few
// instructions each, so HBM bounds them.  A thread takes one 16-value block (32 bytes of bf16,
// 8 of codes, one scale).  Consecutive threads take the blocks of one head's row and then the
// same head's next rows: the 32 scale bytes of a warp (four rows at D = 128) then fill one
// 32-byte sector and its codes 256 consecutive bytes, while the bf16 side stays in runs of D * 2
// bytes.
#include <algorithm>

#include "kv4_dev.cuh"
#include "sonic_host.h"

namespace sonic {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // blocks per thread, their loads all issued before the first store

struct RowParams {
    const uint16_t *K, *V;   // store: source; load: destination
    uint8_t *kc, *ks, *vc, *vs;
    const int32_t *src_row, *dst_row;  // NULL: row j
    const int32_t *live;               // NULL, or negative where entry j is skipped
    const int32_t *n_valid;            // device row count, NULL: n_rows
    int32_t *status;
    int32_t n_rows, Hkv, n_layers;
    int32_t src_total, dst_total;      // rows there are on either side
    int64_t kv_ls;                     // elements between layers of K and V
    int64_t codes_ls, scales_ls;       // bytes between layers
    int32_t cache_rows;
    bool wide32;  // every row of K and V starts on 32 bytes
};

// 32 bytes: in one access where every row starts on 32 bytes, else in two.  (Two 16-byte stores of
// a warp each fill half of their sectors: unpacking ran at 4.7 TB/s with L2 at 63 %.)
__device__ __forceinline__ void load32(uint32_t (&w)[8], const void *p, bool whole) {
    if (whole) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]),
                       "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
    } else {
        const uint4 a = static_cast<const uint4 *>(p)[0], b = static_cast<const uint4 *>(p)[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
}
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8], bool whole) {
    if (whole) {
        st_global_v8(p, w);
    } else {
        static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// One pass over (layer, head, K or V) x (row, block).  kStore: bf16 to four bits.
template <int D, bool kStore>
__global__ void __launch_bounds__(kThreads) kv4_rows_kernel(const RowParams p) {
    constexpr int kBlocks = D / 16;  // per row and head
    pdl_wait();
    pdl_trigger();
    const int n = p.n_valid != nullptr ? min(*p.n_valid, p.n_rows) : p.n_rows;
    const int64_t items = (int64_t)n * kBlocks;
    const int64_t i0 = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
    if (i0 >= items) return;
    // this thread's blocks: the same for every layer and head
    int src[kUnroll], dst[kUnroll];
    const int blk = threadIdx.x % kBlocks;  // (kThreads is a multiple of kBlocks)
    const bool tell = blk == 0 && blockIdx.y == 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = i0 + u * kThreads;
        src[u] = -1;
        dst[u] = 0;
        if (i < items) {
            const int j = (int)(i / kBlocks);
            src[u] = p.src_row != nullptr ? p.src_row[j] : j;
            dst[u] = p.dst_row != nullptr ? p.dst_row[j] : j;
            if (p.live != nullptr && p.live[j] < 0) src[u] = -1;
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        if (src[u] == -1) continue;  // no source, or a free row
        if (src[u] < 0 || src[u] >= p.src_total) {
            if (tell) set_status(p.status, SONIC_ERR_INVALID_ARGUMENT);
            src[u] = -1;
        } else if (dst[u] < 0 || dst[u] >= p.dst_total) {
            if (tell) set_status(p.status, SONIC_ERR_CAPACITY);
            src[u] = -1;
        }
    }
    const int combos = p.n_layers * p.Hkv * 2;
    for (int y = blockIdx.y; y < combos; y += gridDim.y) {
        const bool is_v = y & 1;
        const int head = (y >> 1) % p.Hkv, layer = (y >> 1) / p.Hkv;
        uint16_t *wide = const_cast<uint16_t *>(is_v ? p.V : p.K) + layer * p.kv_ls + head * D + blk * 16;
        uint8_t *codes = (is_v ? p.vc : p.kc) + layer * p.codes_ls +
                         (int64_t)head * p.cache_rows * (D / 2) + blk * 8;
        uint8_t *scales = (is_v ? p.vs : p.ks) + layer * p.scales_ls +
                          (int64_t)head * p.cache_rows * kBlocks + blk;
        const int64_t wide_row = (int64_t)p.Hkv * D;
        if (kStore) {
            uint32_t x[kUnroll][8];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (src[u] >= 0) load32(x[u], wide + src[u] * wide_row, p.wide32);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (src[u] < 0) continue;
                uint32_t top = kv4_top(x[u]);
                if (top > 0x7F80u) {  // a NaN is stored as zero
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if ((x[u][e] & 0x7FFFu) > 0x7F80u) x[u][e] &= 0xFFFF0000u;
                        if ((x[u][e] & 0x7FFF0000u) > 0x7F800000u) x[u][e] &= 0xFFFFu;
                    }
                    top = kv4_top(x[u]);
                }
                const uint32_t sb = kv4_scale(__uint_as_float(top << 16));
                float inv;
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(kv4_scale_value(sb)));
                if (sb == 0) inv = 0.f;
                *reinterpret_cast<uint2 *>(codes + (int64_t)dst[u] * (D / 2)) =
                    make_uint2(kv4_encode8(x[u], inv), kv4_encode8(x[u] + 4, inv));
                scales[(int64_t)dst[u] * kBlocks] = (uint8_t)sb;
            }
        } else {
            uint2 c[kUnroll];
            uint32_t sb[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (src[u] >= 0) {
                    c[u] = ld_once8(codes + (int64_t)src[u] * (D / 2));
                    sb[u] = scales[(int64_t)src[u] * kBlocks];
                }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (src[u] < 0) continue;
                const uint32_t s2 = kv4_scale_f16x2(sb[u]);
                uint32_t o[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t r[4];
                    kv4_decode4(h == 0 ? c[u].x : c[u].y, r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t m = mul_f16x2(r[e], s2);  // exact, and so in bf16
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&m));
                        o[4 * h + e] = pack_bf16x2(f.x, f.y);
                    }
                }
                store32(wide + dst[u] * wide_row, o, p.wide32);
            }
        }
    }
}

template <bool kStore>
cudaError_t launch_rows(int D, const RowParams &p, cudaStream_t stream) {
    const int64_t items = (int64_t)p.n_rows * (D / 16);
    const int64_t x = (items + kThreads * kUnroll - 1) / (kThreads * kUnroll);
    const int combos = p.n_layers * p.Hkv * 2;
    // one slice per (layer, head, K or V) until there are some 32 blocks per SM
    const int64_t want = std::max<int64_t>(1, (32LL * device_sm_count() + x - 1) / x);
    const dim3 grid((unsigned)x, (unsigned)std::min<int64_t>(std::min<int64_t>(combos, 65535), want));
    auto kern = D == 128 ? kv4_rows_kernel<128, kStore> : kv4_rows_kernel<64, kStore>;
    return launch_pdl(kern, grid, kThreads, 0, stream, 1, p);
}

sonic_status_t check_shape(int n_layers, int hkv, int D, int64_t kv_ls) {
    if (n_layers < 1 || hkv < 1) return SONIC_ERR_INVALID_ARGUMENT;
    if (D != 64 && D != 128) return SONIC_ERR_UNSUPPORTED;
    if ((int64_t)n_layers * hkv * 2 > 0x7fffffffLL) return SONIC_ERR_UNSUPPORTED;
    if (n_layers > 1 && (kv_ls <= 0 || kv_ls % 8 != 0)) return SONIC_ERR_INVALID_ARGUMENT;
    return SONIC_OK;
}

RowParams row_params(const uint16_t *K, const uint16_t *V, const sonic_kv4_cache *c, int n_layers,
                     int hkv, int64_t kv_ls, int32_t *status) {
    RowParams p{};
    p.K = K;
    p.V = V;
    p.kc = c->k_codes;
    p.ks = c->k_scales;
    p.vc = c->v_codes;
    p.vs = c->v_scales;
    p.status = status;
    p.Hkv = hkv;
    p.n_layers = n_layers;
    p.kv_ls = kv_ls;
    p.codes_ls = c->codes_layer_bytes;
    p.scales_ls = c->scales_layer_bytes;
    p.cache_rows = c->rows;
    p.wide32 = ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) |
                 (n_layers > 1 ? (uintptr_t)kv_ls * 2 : 0)) & 31) == 0;
    return p;
}

template <bool kStore>
sonic_status_t move_rows(const uint16_t *K, const uint16_t *V, const sonic_kv4_cache *c,
                         const sonic_kv4_rows_args *a, cudaStream_t stream) {
    if (a == nullptr || c == nullptr || a->n_rows < 0) return SONIC_ERR_INVALID_ARGUMENT;
    sonic_status_t st = check_shape(a->n_layers, a->n_heads_kv, a->head_dim, a->kv_layer_stride);
    if (st != SONIC_OK) return st;
    if (a->n_rows == 0) return SONIC_OK;
    if (K == nullptr || V == nullptr || a->total_rows < 0) return SONIC_ERR_INVALID_ARGUMENT;
    if (!aligned16(K) || !aligned16(V)) return SONIC_ERR_INVALID_ARGUMENT;
    st = check_kv4(c, a->n_layers, a->head_dim, true);
    if (st != SONIC_OK) return st;
    RowParams p = row_params(K, V, c, a->n_layers, a->n_heads_kv, a->kv_layer_stride, a->status);
    p.src_row = a->src_row;
    p.dst_row = a->dst_row;
    p.live = a->live;
    p.n_rows = a->n_rows;
    p.src_total = kStore ? a->total_rows : c->rows;
    p.dst_total = kStore ? c->rows : a->total_rows;
    return launch_rows<kStore>(a->head_dim, p, stream) == cudaSuccess ? SONIC_OK : SONIC_ERR_CUDA;
}

}  // namespace

sonic_status_t check_kv4(const sonic_kv4_cache *c, int n_layers, int D, bool with_v) {
    if (c == nullptr || c->rows < 0) return SONIC_ERR_INVALID_ARGUMENT;
    if (c->rows == 0) return SONIC_OK;  // no row of it is touched
    if (c->k_codes == nullptr || c->k_scales == nullptr || !aligned16(c->k_codes) ||
        !aligned16(c->k_scales))
        return SONIC_ERR_INVALID_ARGUMENT;
    if (with_v && (c->v_codes == nullptr || c->v_scales == nullptr || !aligned16(c->v_codes) ||
                   !aligned16(c->v_scales)))
        return SONIC_ERR_INVALID_ARGUMENT;
    if (n_layers > 1 && (c->codes_layer_bytes <= 0 || c->codes_layer_bytes % 16 != 0 ||
                         c->scales_layer_bytes <= 0 || c->scales_layer_bytes % (D / 16) != 0))
        return SONIC_ERR_INVALID_ARGUMENT;
    return SONIC_OK;
}

}  // namespace sonic

using namespace sonic;

extern "C" sonic_status_t sonic_kv4_store(const uint16_t *K, const uint16_t *V,
                                          const sonic_kv4_cache *cache,
                                          const sonic_kv4_rows_args *a, sonic_stream_t stream) {
    return move_rows<true>(K, V, cache, a, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" sonic_status_t sonic_kv4_load(const sonic_kv4_cache *cache, uint16_t *K, uint16_t *V,
                                         const sonic_kv4_rows_args *a, sonic_stream_t stream) {
    return move_rows<false>(K, V, cache, a, reinterpret_cast<cudaStream_t>(stream));
}

namespace {

// The retention scan's arguments: it takes no part in how rows are stored.
sonic_compact_args scan_args(const sonic_kv4_cache *c, const sonic_kv4_compact_args *a) {
    sonic_compact_args s{};
    s.batch = a->batch;
    s.n_layers = a->n_layers;
    s.k_start = a->k_start;
    s.k_len = a->k_len;
    s.reserve = a->reserve;
    s.out_capacity_rows = c->rows;
    s.ret_len = a->ret_len;
    s.src_idx = a->src_idx;
    s.out_role = a->out_role;
    s.out_seg = a->out_seg;
    s.status = a->status;
    s.workspace = a->workspace;
    s.workspace_bytes = a->workspace_bytes;
    s.total_rows = a->total_rows;
    return s;
}

// Whether an output lies over an input: the scan's blocks write some while others still read.
bool outputs_over_inputs(const int32_t *seg_id, const uint8_t *role, const int32_t *offsets, const sonic_kv4_cache *c,
                         const sonic_kv4_compact_args *a) {
    const size_t word = sizeof(int32_t), per_seq = (size_t)a->batch * word;
    const size_t total = (size_t)a->total_rows, rows = (size_t)c->rows;
    const struct {
        const void *at;
        size_t bytes;
    } in[] = {{a->k_start, per_seq}, {a->k_len, per_seq}, {a->reserve, per_seq}, {role, total}, {seg_id, total * word}},
      out[] = {{offsets, per_seq + word}, {a->ret_len, per_seq}, {a->src_idx, rows * word}, {a->out_role, rows},
               {a->out_seg, rows * word}};
    for (const auto &o : out)
        for (const auto &i : in)
            if (overlap(o.at, o.bytes, i.at, i.bytes)) return true;
    return false;
}

}  // namespace

extern "C" size_t sonic_kv4_compact_workspace_size(const sonic_kv4_cache *c,
                                                   const sonic_kv4_compact_args *a) {
    if (c == nullptr || a == nullptr) return 0;
    const sonic_compact_args s = scan_args(c, a);
    return sonic_compact_workspace_size(&s);
}

extern "C" sonic_status_t sonic_kv4_compact(const uint16_t *K, const uint16_t *V,
                                            const int32_t *seg_id, const uint8_t *role,
                                            const sonic_kv4_cache *c, int32_t *offsets,
                                            const sonic_kv4_compact_args *a,
                                            sonic_stream_t stream_) {
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (a == nullptr || c == nullptr || offsets == nullptr || a->batch < 0)
        return SONIC_ERR_INVALID_ARGUMENT;
    sonic_status_t st = check_shape(a->n_layers, a->n_heads_kv, a->head_dim, a->kv_layer_stride);
    if (st != SONIC_OK) return st;
    if (a->batch == 0)
        return cudaMemsetAsync(offsets, 0, sizeof(int32_t), stream) == cudaSuccess ? SONIC_OK
                                                                                   : SONIC_ERR_CUDA;
    if (K == nullptr || V == nullptr || role == nullptr || a->k_start == nullptr ||
        a->k_len == nullptr || !aligned16(K) || !aligned16(V) || a->total_rows <= 0)
        return SONIC_ERR_INVALID_ARGUMENT;
    st = check_kv4(c, a->n_layers, a->head_dim, true);
    if (st != SONIC_OK) return st;
    if (a->batch > 65535) return SONIC_ERR_UNSUPPORTED;
    const sonic_compact_args s = scan_args(c, a);
    st = check_scan_workspace(&s);
    if (st != SONIC_OK) return st;
    if (outputs_over_inputs(seg_id, role, offsets, c, a)) return SONIC_ERR_INVALID_ARGUMENT;
    int32_t *src_idx = nullptr;
    if (launch_keep_scan(seg_id, role, offsets, &s, &src_idx, stream) != cudaSuccess)
        return SONIC_ERR_CUDA;
    if (c->rows == 0) return SONIC_OK;
    RowParams p = row_params(K, V, c, a->n_layers, a->n_heads_kv, a->kv_layer_stride, a->status);
    p.src_row = src_idx;
    p.n_valid = offsets + a->batch;
    p.n_rows = c->rows;
    p.src_total = a->total_rows;
    p.dst_total = c->rows;
    return launch_rows<true>(a->head_dim, p, stream) == cudaSuccess ? SONIC_OK : SONIC_ERR_CUDA;
}
