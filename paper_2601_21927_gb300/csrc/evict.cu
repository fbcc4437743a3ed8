// Eviction from a cache by accumulated attention weight (sonic_evict_kv).
//
// Sequence b keeps n_b = min(len, max(budget, protected)) rows: the protected ones and those of
// the largest mass, ties to the lower row, in their order.  No host round trip:
//   evict_select  a block per (sequence, choice): the largest key of which at least n_b rows have
//                 as much or more, by bisection over the bits of the masses (as ordered 32-bit
//                 keys in shared memory up to kSmemKeys rows; longer sequences read them again
//                 for each step) until few are left, then the rows above it and the first of those equal to it,
//                 placed by one ordered scan;
//   evict_move    the rows of every part: 16-byte pieces (8 or 4 where alignment asks), four
//                 per thread in flight.
// In small calls a select block counts the protected rows of its own and of the earlier
// sequences itself (role bytes, 16 a load); in others two launches before it do:
//   evict_count   a block per sequence: its protected rows and n_b;
//   evict_offsets one block: offsets and the capacity check.
// Protected rows have the largest key of all, so they need no list of their own.  The bisection
// counts four keys per 16-byte read of shared memory and settles two bits a step; histograms by
// shared-memory atomics took 44 us for 256 choices of up to 12,146 rows, whose weights crowd a few
// exponents (28 layers by head, 896 choices: 72 us of 315 now, the move 243 at 6.9 TB/s).  256 threads
// a block: with 1,024 the 16 steps' fixed part alone was 100 instructions for each of 32 warps (388 us).
// The rows moved outweigh the rest (4 bytes of mass against 512 of K and V at D = 128, once per
// choice), so HBM bounds a call of many layers, and the launches a call of one.
#include <algorithm>

#include "sonic_dev.cuh"
#include "sonic_host.h"

namespace sonic {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// Keys left that a block compares with one another instead of halving on: 64 where keys are in shared memory
// (evict of 28 layers by head 315 us; 322 without, 370 with 256: more shared memory, a block less on each
// SM), more where each step reads a long sequence again (sequences of 60,000 and 13,978 bf16 rows, 4 layers of 4 heads
// x 128, each choosing, 40 % kept: 427 us with 256, 441 with 64, 527 without; 347 with its loads eight at a time).
constexpr int kFewHeld = 64, kFewLong = kThreads;
// calls in which every select block counts for itself: role bytes read by all of them
constexpr int64_t kSelfCount = 1 << 25;
constexpr int kSmemKeys = 48 * 1024;
constexpr int kPerThread = 4;  // consecutive rows a thread places at a time
constexpr int kLoads = 8;
// (loops over a sequence's rows step at most kThreads * kLoads past its end in 32 bits)
constexpr int kMostRows = 0x7fffffff - 2 * kThreads * kLoads;
constexpr uint32_t kProtected = 0xFFFFFFFFu;
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;

struct Part {
    const uint8_t *src;
    uint8_t *dst;
    int64_t src_layer, src_head, src_row, dst_layer, dst_head, dst_row;
    int32_t pieces;  // per row and head, `width` bytes each
    int32_t width;
    int32_t heads;   // 1: all KV heads move as one row
};

struct Params {
    const float *mass;
    const int32_t *lens, *kv_start, *budget, *reserve;
    const uint8_t *role;
    int32_t *offsets, *out_len, *src_idx;
    float *out_mass;
    uint8_t *out_role;
    int32_t *kept;  // [B] rows kept
    int32_t *status;
    int32_t B, rows, max_len, recent, out_rows, n_layers, mass_layers, mass_heads, smem_keys;
    uint32_t keep_roles;
    Part parts[4];
};

__device__ __forceinline__ int seq_len(const Params &p, int b) {
    const int len = p.lens[b], start = p.kv_start[b];
    return len < 0 || len > p.max_len || start < 0 || (int64_t)start + len > p.rows ? 0 : len;
}

__device__ __forceinline__ int warp_inclusive_scan(int v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Protected rows of sequence b, this thread's share (lane `lane` of `lanes`, >= 16).
__device__ __forceinline__ int count_protected(const Params &p, int b, int len, int lane, int lanes) {
    const int older = max(0, len - p.recent);  // rows that only their role protects
    int n = lane == 0 ? len - older : 0;
    for (uint32_t roles = p.keep_roles; roles != 0; roles &= roles - 1)
        n += count_equal(p.role + p.kv_start[b], older, (uint8_t)(__ffs(roles) - 1), lane, lanes);
    return n;
}

__device__ __forceinline__ int rows_kept(const Params &p, int b, int len, int protect) {
    return min(len, max(p.budget[b], protect));
}

__device__ __forceinline__ int rows_reserved(const Params &p, int b) {
    return p.reserve != nullptr ? max(0, p.reserve[b]) : 0;
}

// Sum over the block, to every thread.
__device__ __forceinline__ long long block_sum(long long v, long long *part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += part[w];
    return v;
}

__global__ void __launch_bounds__(kThreads) evict_count_kernel(const Params p) {
    __shared__ long long part[kWarps];
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x, len = seq_len(p, b);
    if (threadIdx.x == 0 && len != p.lens[b]) set_status(p.status, SONIC_ERR_INVALID_ARGUMENT);
    const int n = (int)block_sum(count_protected(p, b, len, threadIdx.x, kThreads), part);
    if (threadIdx.x == 0) {
        p.kept[b] = rows_kept(p, b, len, n);
        if (p.out_len != nullptr) p.out_len[b] = p.kept[b];
    }
}

// (past 2^31 - 1 rows the offsets stop there; nothing is written from out_rows on)
__device__ __forceinline__ int32_t clip_offset(long long v) { return (int32_t)min(v, 0x7fffffffLL); }

__global__ void __launch_bounds__(kThreads) evict_offsets_kernel(const Params p) {
    __shared__ long long part[kWarps];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (p.B + kThreads - 1) / kThreads;
    const int b0 = min(p.B, tid * run), b1 = min(p.B, b0 + run);
    auto size = [&](int b) { return (long long)p.kept[b] + rows_reserved(p, b); };
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += size(b);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) part[warp] = incl;
    __syncthreads();
    long long at = incl - mine, sum = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) at += part[w];
        sum += part[w];
    }
    for (int b = b0; b < b1; ++b) {
        p.offsets[b] = clip_offset(at);
        at += size(b);
    }
    if (tid == 0) {
        p.offsets[p.B] = clip_offset(sum);
        if (sum > p.out_rows) set_status(p.status, SONIC_ERR_CAPACITY);
    }
}

// Masses as keys whose unsigned order is theirs: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float m) {
    uint32_t u = __float_as_uint(m);
    if (m != m) u = 0xFF800000u;
    if (m == 0.f) u = 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}

// kSelf: this block counts the protected rows of its own and the earlier sequences.
template <bool kSelf>
__global__ void __launch_bounds__(kThreads, 4) evict_select_kernel(const Params p) {
    extern __shared__ __align__(16) uint32_t s_key[];
    __shared__ int part[kWarps];
    __shared__ long long sums[kWarps];
    __shared__ int s_count[2][3], s_found, s_ties;
    __shared__ uint32_t s_few[kFewHeld], s_edge;
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = (int)(blockIdx.x % p.B);
    const int64_t choice = blockIdx.x / p.B;  // (layer, head) of mass
    const int len = seq_len(p, b), start = p.kv_start[b];
    const float *mass = p.mass + choice * p.rows + start;
    const bool held = len <= p.smem_keys;
    const uint8_t *role_of = p.role + start;
    const bool by_role = p.keep_roles != 0;
    // (both loads before the choice: a branch between them would have them wait for each other)
    auto make_key = [&](int t) {
        const float m = mass[t];
        const uint32_t r = by_role ? role_of[t] : 32;
        const bool stays = t >= len - p.recent || (r < 32 && (p.keep_roles >> r & 1));
        return stays ? kProtected : key_of(m);
    };
    auto key_at = [&](int t) {
        const uint32_t k = make_key(min(t, len - 1));
        return t < len ? k : 0;
    };
    if (held) {
        // eight rows' loads on their way at a time (one by one, a sequence of 12,146 rows took 20 us)
        for (int t0 = tid; t0 < ((len + 3) & ~3); t0 += kThreads * kLoads) {
            uint32_t k[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k[i] = key_at(t0 + i * kThreads);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (t0 + i * kThreads < ((len + 3) & ~3)) s_key[t0 + i * kThreads] = k[i];
        }
    }
    int kept;
    int64_t base;
    if (kSelf) {
        kept = rows_kept(p, b, len, (int)block_sum(count_protected(p, b, len, tid, kThreads), sums));
        // the sequences before this one, a warp each
        long long before = 0;
        for (int i = warp; i < b; i += kWarps) {
            const int li = seq_len(p, i);
            int n = count_protected(p, i, li, lane, 32);
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) before += (long long)rows_kept(p, i, li, n) + rows_reserved(p, i);
        }
        base = clip_offset(block_sum(before, sums));
        if (tid == 0 && choice == 0) {
            if (len != p.lens[b]) set_status(p.status, SONIC_ERR_INVALID_ARGUMENT);
            p.offsets[b] = (int32_t)base;
            if (p.out_len != nullptr) p.out_len[b] = kept;
            if (b == p.B - 1) {
                const long long sum = base + kept + rows_reserved(p, b);
                p.offsets[p.B] = clip_offset(sum);
                if (sum > p.out_rows) set_status(p.status, SONIC_ERR_CAPACITY);
            }
        }
    } else {
        kept = p.kept[b];
        base = p.offsets[b];
    }
    int32_t *src_idx = p.src_idx + choice * p.out_rows;
    float *out_mass = p.out_mass != nullptr ? p.out_mass + choice * p.out_rows : nullptr;
    uint8_t *out_role = p.out_role != nullptr ? p.out_role + choice * p.out_rows : nullptr;
    const bool all = kept == len;
    uint32_t edge = 0;  // rows with a larger key are kept,
    int ties = len;     // and the first so many of those with this one
    if (!all && kept > 0) {
        // every key once, and some 0, which no row has
        auto each_key = [&](auto take) {
            if (held) {
                const uint4 *k4 = reinterpret_cast<const uint4 *>(s_key);
                for (int t = tid; t < (len + 3) / 4; t += kThreads) {
                    const uint4 k = k4[t];
                    take(k.x), take(k.y), take(k.z), take(k.w);
                }
            } else {
                for (int t0 = tid; t0 < len; t0 += kThreads * kLoads) {
                    uint32_t k[kLoads];
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) k[i] = key_at(t0 + i * kThreads);
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) take(k[i]);
                }
            }
        };
        // rows whose key is at least c[0] < c[1] < c[2]
        auto count = [&](const uint32_t (&c)[3], int (&n)[3]) {
            n[0] = n[1] = n[2] = 0;
            auto add = [&](uint32_t k) {
                n[0] += k >= c[0];
                n[1] += k >= c[1];
                n[2] += k >= c[2];
            };
            each_key(add);
        };
        if (tid < 3) s_count[0][tid] = 0;
        if (tid == 3) {
            s_found = s_ties = 0;
            s_edge = kProtected;
        }
        __syncthreads();
        const int few_most = held ? kFewHeld : kFewLong;
        uint32_t *few_keys = held ? s_few : s_key;  // (not held: smem_keys is kSmemKeys, and free)
        // The kept-th largest key lies in the bracket edge .. edge + 2^lo - 1: `above` rows, fewer than are
        // kept, have larger keys, and `reach`, at least as many, have those of the bracket or larger.
        int above = 0, reach = len, lo = 32, step = 0;
#pragma unroll 1
        for (; lo > 0 && reach != kept && reach - above > few_most; step ^= 1) {
            lo -= 2;
            const uint32_t c[3] = {edge | 1u << lo, edge | 2u << lo, edge | 3u << lo};
            int n[3];
            count(c, n);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                n[i] = __reduce_add_sync(0xffffffffu, n[i]);
                if (lane == 0) atomicAdd(&s_count[step][i], n[i]);
            }
            if (tid < 3) s_count[step ^ 1][tid] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const int got = s_count[step][i];
                if (got >= kept) {
                    edge = c[i];
                    reach = got;
                }
            }
#pragma unroll
            for (int i = 2; i >= 0; --i)
                if (s_count[step][i] < kept) above = s_count[step][i];
            __syncthreads();  // (the counts are cleared two steps on)
        }
        if (reach == kept) {
            --edge;  // (edge > 0: all rows have 0 or more, and not all are kept)
            ties = 0;
        } else if (lo == 0) {
            ties = kept - above;
        } else {
            // few keys are left: each counts those among them that are larger
            const uint32_t span = lo == 32 ? 0xFFFFFFFFu : (1u << lo) - 1;
            auto collect = [&](uint32_t k) {
                if (k - edge > span || k == 0) return;
                const int i = atomicAdd(&s_found, 1);
                if (i < few_most) few_keys[i] = k;
            };
            each_key(collect);
            __syncthreads();
            const int few = reach - above, want = kept - above;
            if (tid < few) {
                const uint32_t k = few_keys[tid];
                int larger = 0, equal = 0;
#pragma unroll 4
                for (int i = 0; i < few; ++i) {
                    larger += few_keys[i] > k;
                    equal += few_keys[i] == k;
                }
                if (larger < want && want <= larger + equal) {  // (by all that have this key)
                    s_edge = k;
                    s_ties = want - larger;
                }
            }
            __syncthreads();
            edge = s_edge;
            ties = s_ties;
        }
    }
    // the kept rows in order: counts of rows above the edge and equal to it, 16 bits each (at most
    // kThreads * kPerThread of them a pass)
    int above_run = 0, equal_run = 0;
    for (int t0 = 0; t0 < len && kept > 0; t0 += kThreads * kPerThread) {
        const int t = t0 + tid * kPerThread;
        uint32_t key[kPerThread];
        float m[kPerThread];
        uint8_t role[kPerThread];
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {  // all loads ahead of the scan
            const bool in = t + i < len;
            const int at = min(t + i, len - 1);
            key[i] = !in || all ? 0 : held ? s_key[at] : make_key(at);
            m[i] = out_mass != nullptr ? mass[at] : 0.f;
            role[i] = out_role != nullptr ? role_of[at] : 0;
        }
        int above[kPerThread], equal[kPerThread], mine = 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            above[i] = t + i < len && !all && key[i] > edge;
            equal[i] = t + i < len && (all || key[i] == edge);
            mine += above[i] | equal[i] << 16;
        }
        const int incl = warp_inclusive_scan(mine);
        __syncthreads();
        if (lane == 31) part[warp] = incl;
        __syncthreads();
        // (each warp scans the warps' counts)
        const int each = lane < kWarps ? part[lane] : 0, upto = warp_inclusive_scan(each);
        const int total = __shfl_sync(0xffffffffu, upto, kWarps - 1);
        const int before = incl - mine + __shfl_sync(0xffffffffu, upto - each, warp);
        int a = above_run + (before & 0xFFFF), e = equal_run + (before >> 16);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int64_t o = base + a + min(e, ties);
            if ((above[i] || (equal[i] && e < ties)) && o < p.out_rows) {
                src_idx[o] = start + t + i;
                if (out_mass != nullptr) out_mass[o] = m[i];
                if (out_role != nullptr) out_role[o] = role[i];
            }
            a += above[i];
            e += equal[i];
        }
        above_run += total & 0xFFFF;
        equal_run += total >> 16;
    }
    const int res = rows_reserved(p, b);
    for (int i = tid; i < res; i += kThreads) {
        const int64_t o = base + kept + i;
        if (o >= p.out_rows) break;
        src_idx[o] = -1;
        if (out_role != nullptr) out_role[o] = SONIC_ROLE_BODY;
    }
}

template <typename Vec>
__device__ __forceinline__ void move_part(const Params &p, const Part &q) {
    const int n = min(p.offsets[p.B], p.out_rows);
    const int64_t items = (int64_t)n * q.pieces;
    const int64_t i0 = (int64_t)blockIdx.x * (kMoveThreads * kMoveUnroll) + threadIdx.x;
    if (i0 >= items) return;
    int row[kMoveUnroll], piece[kMoveUnroll];
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u) {
        const int64_t i = i0 + u * kMoveThreads;
        row[u] = i < items ? (int)(i / q.pieces) : -1;
        piece[u] = (int)(i - (int64_t)row[u] * q.pieces) * (int)sizeof(Vec);
    }
    const int combos = p.n_layers * q.heads;
    for (int y = blockIdx.y; y < combos; y += gridDim.y) {
        const int layer = y / q.heads, head = y % q.heads;
        const int64_t choice = (int64_t)(p.mass_layers > 1 ? layer : 0) * p.mass_heads +
                               (p.mass_heads > 1 ? head : 0);
        const int32_t *idx = p.src_idx + choice * p.out_rows;
        const uint8_t *src = q.src + layer * q.src_layer + head * q.src_head;
        uint8_t *dst = q.dst + layer * q.dst_layer + head * q.dst_head;
        int from[kMoveUnroll];
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u) from[u] = row[u] >= 0 ? idx[row[u]] : -1;
        Vec v[kMoveUnroll];
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u)
            if (from[u] >= 0)
                v[u] = *reinterpret_cast<const Vec *>(src + from[u] * q.src_row + piece[u]);
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u)
            if (from[u] >= 0) *reinterpret_cast<Vec *>(dst + row[u] * q.dst_row + piece[u]) = v[u];
    }
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const Params p) {
    pdl_wait();
    pdl_trigger();
    const Part &q = p.parts[blockIdx.z];
    if (q.width == 16)
        move_part<uint4>(p, q);
    else if (q.width == 8)
        move_part<uint2>(p, q);
    else
        move_part<uint32_t>(p, q);
}

// Whether an output lies over an input.  A block writes offsets, out_len and the rows that it chose while
// others still read the lengths, starts, budgets and masses.
bool outputs_over_inputs(const float *mass, const int32_t *lens, const int32_t *offsets, const sonic_evict_args *a) {
    const size_t word = sizeof(int32_t), per_seq = (size_t)a->batch * word;
    const size_t maps = (size_t)a->mass_layers * a->mass_heads;
    const size_t in_rows = (size_t)a->total_kv_rows, out_rows = maps * a->out_rows;
    const struct {
        const void *at;
        size_t bytes;
    } in[] = {{lens, per_seq}, {a->kv_start, per_seq}, {a->budget, per_seq}, {a->reserve, per_seq},
              {mass, maps * in_rows * word}, {a->role, in_rows}},
      out[] = {{offsets, per_seq + word}, {a->out_len, per_seq}, {a->src_idx, out_rows * word},
               {a->out_mass, out_rows * word}, {a->out_role, out_rows}};
    for (const auto &o : out)
        for (const auto &i : in)
            if (overlap(o.at, o.bytes, i.at, i.bytes)) return true;
    for (int i = 0; i < a->n_parts; ++i)  // (a part moved onto itself; regions may interleave by their strides)
        if (a->parts[i].src == a->parts[i].dst && a->parts[i].src != nullptr) return true;
    return false;
}

size_t kept_bytes(const sonic_evict_args *a) {
    return round_up((size_t)a->batch * sizeof(int32_t), 256);
}

}  // namespace
}  // namespace sonic

using namespace sonic;

extern "C" size_t sonic_evict_workspace_size(const sonic_evict_args *a) {
    if (a == nullptr || a->batch <= 0 || a->out_rows < 0 || a->mass_layers < 1 || a->mass_heads < 1)
        return 0;
    // rows kept per sequence, then (if the caller gives no src_idx) the source rows
    size_t n = kept_bytes(a);
    if (a->src_idx == nullptr)
        n += (size_t)a->mass_layers * a->mass_heads * a->out_rows * sizeof(int32_t);
    return n;
}

extern "C" sonic_status_t sonic_evict_kv(const float *mass, const int32_t *lens, int32_t *offsets,
                                         const sonic_evict_args *a, sonic_stream_t stream_) {
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (a == nullptr || offsets == nullptr || a->batch < 0 || a->n_layers < 1 || a->n_heads_kv < 1 ||
        a->max_len < 0 || a->total_kv_rows < 0 || a->recent < 0 || a->out_rows < 0 || a->n_parts < 0 ||
        a->n_parts > 4 || (a->mass_layers != 1 && a->mass_layers != a->n_layers) ||
        (a->mass_heads != 1 && a->mass_heads != a->n_heads_kv))
        return SONIC_ERR_INVALID_ARGUMENT;
    if (a->batch == 0)
        return cudaMemsetAsync(offsets, 0, sizeof(int32_t), stream) == cudaSuccess ? SONIC_OK
                                                                                   : SONIC_ERR_CUDA;
    if ((mass == nullptr && a->total_kv_rows > 0) || lens == nullptr || a->kv_start == nullptr || a->budget == nullptr ||
        ((a->keep_roles != 0 || a->out_role != nullptr) && a->role == nullptr && a->total_kv_rows > 0))
        return SONIC_ERR_INVALID_ARGUMENT;
    const int64_t choices = (int64_t)a->mass_layers * a->mass_heads;
    if (a->batch > 65535 || choices * a->batch > 0x7fffffffLL ||
        (int64_t)a->n_layers * a->n_heads_kv > 0x7fffffffLL || a->total_kv_rows > kMostRows)
        return SONIC_ERR_UNSUPPORTED;
    Params p{};
    int64_t blocks = 0;
    for (int i = 0; i < a->n_parts; ++i) {
        const sonic_evict_part &s = a->parts[i];
        if (s.bytes <= 0 || (s.src == nullptr && a->total_kv_rows > 0) ||
            (s.dst == nullptr && a->out_rows > 0))
            return SONIC_ERR_INVALID_ARGUMENT;
        Part &q = p.parts[i];
        q = Part{static_cast<const uint8_t *>(s.src), static_cast<uint8_t *>(s.dst),
                 s.src_layer, s.src_head, s.src_row, s.dst_layer, s.dst_head, s.dst_row, 0, 0,
                 a->n_heads_kv};
        // one choice for all heads, and these side by side: whole rows move
        int64_t bytes = s.bytes;
        if (a->mass_heads == 1 && s.src_head == s.bytes && s.dst_head == s.bytes &&
            bytes * a->n_heads_kv <= 0x7fffffffLL) {
            q.heads = 1;
            bytes *= a->n_heads_kv;
        }
        const uint64_t all = (uint64_t)bytes | (uint64_t)reinterpret_cast<uintptr_t>(s.src) |
                             (uint64_t)reinterpret_cast<uintptr_t>(s.dst) | (uint64_t)s.src_layer |
                             (uint64_t)s.src_head | (uint64_t)s.src_row | (uint64_t)s.dst_layer |
                             (uint64_t)s.dst_head | (uint64_t)s.dst_row;
        if (all & 3) return SONIC_ERR_INVALID_ARGUMENT;
        q.width = all & 7 ? 4 : all & 15 ? 8 : 16;
        q.pieces = (int32_t)(bytes / q.width);
        blocks = std::max(blocks, ((int64_t)a->out_rows * q.pieces + kMoveThreads * kMoveUnroll - 1) /
                                      (kMoveThreads * kMoveUnroll));
    }
    if (blocks > 0x7fffffffLL) return SONIC_ERR_UNSUPPORTED;
    const size_t need = sonic_evict_workspace_size(a);
    if (a->workspace == nullptr || a->workspace_bytes < need) return SONIC_ERR_WORKSPACE;
    if (!aligned16(a->workspace) || outputs_over_inputs(mass, lens, offsets, a)) return SONIC_ERR_INVALID_ARGUMENT;
    char *ws = static_cast<char *>(a->workspace);
    p.mass = mass;
    p.lens = lens;
    p.kv_start = a->kv_start;
    p.budget = a->budget;
    p.reserve = a->reserve;
    p.role = a->role;
    p.offsets = offsets;
    p.out_len = a->out_len;
    p.kept = reinterpret_cast<int32_t *>(ws);
    p.src_idx = a->src_idx != nullptr ? a->src_idx : reinterpret_cast<int32_t *>(ws + kept_bytes(a));
    p.out_mass = a->out_mass;
    p.out_role = a->out_role;
    p.status = a->status;
    p.B = a->batch;
    p.rows = a->total_kv_rows;
    p.max_len = a->max_len;
    p.recent = a->recent;
    p.out_rows = a->out_rows;
    p.n_layers = a->n_layers;
    p.mass_layers = a->mass_layers;
    p.mass_heads = a->mass_heads;
    p.keep_roles = a->keep_roles;
    p.smem_keys = (std::min(std::max(a->max_len, 1), kSmemKeys) + 3) & ~3;

    // Each block for itself while that is less than the launches it saves (two of 3 us each on
    // the host; counting costs 1 us where all blocks together read some 30 MB of role bytes).
    const bool self = (int64_t)std::min<int64_t>(p.rows, (int64_t)a->batch * a->max_len) * a->batch *
                              choices / 2 + choices * a->batch * a->batch * 16 <= kSelfCount;
    cudaError_t e = cudaSuccess;
    if (!self) {
        e = launch_pdl(evict_count_kernel, dim3(a->batch), kThreads, 0, stream, 1, p);
        if (e == cudaSuccess) e = launch_pdl(evict_offsets_kernel, dim3(1), kThreads, 0, stream, 1, p);
    }
    const auto select = self ? evict_select_kernel<true> : evict_select_kernel<false>;
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(select, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSmemKeys * (int)sizeof(uint32_t));
    if (e == cudaSuccess)
        e = launch_pdl(select, dim3((unsigned)(choices * a->batch)), kThreads,
                       p.smem_keys * sizeof(uint32_t), stream, 1, p);
    if (e == cudaSuccess && blocks > 0) {
        const int64_t combos = (int64_t)a->n_layers * a->n_heads_kv;
        const int64_t want = std::max<int64_t>(1, (32LL * device_sm_count() + blocks - 1) / blocks);
        const dim3 grid((unsigned)blocks, (unsigned)std::min<int64_t>(std::min<int64_t>(combos, 65535), want),
                        (unsigned)a->n_parts);
        e = launch_pdl(evict_move_kernel, grid, kMoveThreads, 0, stream, 1, p);
    }
    return e == cudaSuccess ? SONIC_OK : SONIC_ERR_CUDA;
}
