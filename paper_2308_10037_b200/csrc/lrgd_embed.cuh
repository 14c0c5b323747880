// Rows of a token table and the table's gradient.
//
//   lookup:    out[t,:] = scale * table[id_t,:]                                          (an id outside [0, V): zeros)
//   gradient:  grad[v,:] (+)= scale * sum over { t : id_t = v } of dout[t,:]            in fp32, v in [0, V), v != padding id
//
// The gradient sorts the positions t by their token (stable, so that a token's positions stay in order), then adds up runs of
// equal tokens: every row of the gradient is written by one thread per column, in a fixed order, without atomics on data.
#pragma once
#include "lrgd_route.cuh"

namespace lrgd {

// ---- lookup --------------------------------------------------------------------------------------------
constexpr int kEmbedThreads = 256;

struct EmbedParams {
    const void* table;
    long long ld_table;
    const void* ids;
    long long T;
    long long V;
    int n;
    float scale;
    void* out;
    long long ld_out;
    int* status;
};

template <class Id>
__device__ __forceinline__ long long load_id(const void* ids, long long t) {
    return static_cast<long long>(__ldg(static_cast<const Id*>(ids) + t));
}

// a value already in registers
__device__ __forceinline__ float load_local(const float* p) { return *p; }
__device__ __forceinline__ float load_local(const unsigned short* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }

// One warp takes one piece of one row: up to 128 vectors of VEC elements (four per lane, all loaded before the first store).
template <class E, int VEC, class Id>
__global__ void __launch_bounds__(kEmbedThreads) k_embed(const __grid_constant__ EmbedParams p) {
    struct alignas(sizeof(E) * VEC) Vec { E v[VEC]; };
    const int lane = threadIdx.x & 31;
    const int vecs = (p.n + VEC - 1) / VEC;
    const int first = blockIdx.y * 128 + lane;
    const long long warps = static_cast<long long>(gridDim.x) * (kEmbedThreads / 32);
    for (long long t = static_cast<long long>(blockIdx.x) * (kEmbedThreads / 32) + (threadIdx.x >> 5); t < p.T; t += warps) {
        const long long id = load_id<Id>(p.ids, t);
        const bool known = id >= 0 && id < p.V;
        const Vec* src = reinterpret_cast<const Vec*>(static_cast<const E*>(p.table) + (known ? id : 0) * p.ld_table);
        Vec* dst = reinterpret_cast<Vec*>(static_cast<E*>(p.out) + t * p.ld_out);
        Vec x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = first + 32 * j;
            if (i < vecs && known) x[j] = src[i];
            else x[j] = Vec{};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = first + 32 * j;
#pragma unroll
            for (int c = 0; c < VEC; ++c) store_from_float(&x[j].v[c], known ? load_local(&x[j].v[c]) * p.scale : 0.0f);
            if (i < vecs) dst[i] = x[j];
        }
        if (!known && first == 0) atomicExch(p.status, -4);          // LR_ERR_VALUE: an id outside the table
    }
}

// ---- positions sorted by token -------------------------------------------------------------------------
// One cluster of eight CTAs sorts: every pass orders by eight bits of the token, least significant first.  A CTA owns a contiguous
// eighth of the positions; the CTAs exchange their 256 counts through distributed shared memory, so a pass needs two cluster
// barriers and no launch of its own.  The other CTAs of the launch write the zeros of the gradient meanwhile.
constexpr int kSortThreads = 1024;
constexpr int kSortCtas = 8;
constexpr int kSortItems = 4;                       // positions per thread and tile
constexpr int kSortWarps = kSortThreads / 32;

struct SortParams {
    const void* ids;
    unsigned int T;
    long long V;               // also the key of positions without a gradient (padding, ids outside the table): sorted last
    long long padding;
    unsigned int* key[2];      // [T] each; pass i writes buffer i & 1
    unsigned int* pos[2];
    int passes;
    int* status;
    float* zero;               // nullable: floats to be cleared
    long long zero_count;
};

__device__ __forceinline__ unsigned int cluster_load_u32(const unsigned int* local, int rank) {
    uint32_t addr, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <class Id>
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) k_token_sort(const __grid_constant__ SortParams p) {
    __shared__ unsigned int count[kSortWarps][256];
    __shared__ unsigned int hist[256], base[256], scan[8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.x >= kSortCtas) {
        const long long threads = static_cast<long long>(gridDim.x - kSortCtas) * kSortThreads;
        const long long me = static_cast<long long>(blockIdx.x - kSortCtas) * kSortThreads + tid;
        const long long head = min(p.zero_count, static_cast<long long>((16 - (reinterpret_cast<uintptr_t>(p.zero) & 15)) & 15) / 4);
        const long long quads = (p.zero_count - head) / 4;
        float4* z = reinterpret_cast<float4*>(p.zero + head);
        for (long long i = me; i < quads; i += threads) z[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (me < head) p.zero[me] = 0.f;
        if (me < p.zero_count - head - quads * 4) p.zero[head + quads * 4 + me] = 0.f;
        return;
    }
    const int rank = blockIdx.x;
    const unsigned int per = (p.T + kSortCtas - 1) / kSortCtas;
    const unsigned int lo = min(p.T, per * rank), hi = min(p.T, lo + per);
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = 8 * pass;
        const unsigned int* kin = p.key[(pass + 1) & 1];
        const unsigned int* pin = p.pos[(pass + 1) & 1];
        unsigned int* kout = p.key[pass & 1];
        unsigned int* pout = p.pos[pass & 1];
        auto key_at = [&](unsigned int i) -> unsigned int {
            if (pass > 0) return __ldcg(kin + i);
            const long long id = load_id<Id>(p.ids, i);
            return id < 0 || id >= p.V || id == p.padding ? static_cast<unsigned int>(p.V) : static_cast<unsigned int>(id);
        };
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (unsigned int i = lo + tid; i < hi; i += kSortThreads) {
            if (pass == 0) {
                const long long id = load_id<Id>(p.ids, i);
                if ((id < 0 || id >= p.V) && id != p.padding) atomicExch(p.status, -4);     // LR_ERR_VALUE
            }
            atomicAdd(&hist[(key_at(i) >> shift) & 255u], 1u);
        }
        cluster_barrier();
        // first place of this CTA's elements of digit `tid`: all smaller digits, then the same digit of the CTAs before this one
        unsigned int total = 0, before = 0;
        if (tid < 256) {
#pragma unroll
            for (int r = 0; r < kSortCtas; ++r) {
                const unsigned int h = cluster_load_u32(&hist[tid], r);
                if (r < rank) before += h;
                total += h;
            }
        }
        unsigned int inc = total;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned int o = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += o;
        }
        if (tid < 256 && lane == 31) scan[warp] = inc;
        __syncthreads();
        if (tid < 256) {
            unsigned int add = 0;
            for (int w = 0; w < warp; ++w) add += scan[w];
            base[tid] = add + inc - total + before;
        }
        // tiles of 4096 positions; a warp ranks 128 consecutive ones, 32 at a time
        for (unsigned int tile = lo; tile < hi; tile += kSortThreads * kSortItems) {
            __syncthreads();
            for (int i = tid; i < kSortWarps * 256; i += kSortThreads) (&count[0][0])[i] = 0;
            __syncthreads();
            unsigned int key[kSortItems], rnk[kSortItems];
            const unsigned int mine = tile + warp * 32 * kSortItems + lane;
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) key[j] = mine + 32 * j < hi ? key_at(mine + 32 * j) : 0u;
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const bool in = mine + 32 * j < hi;
                const unsigned int digit = in ? (key[j] >> shift) & 255u : 256u;
                const unsigned int same = __match_any_sync(0xffffffffu, digit);
                const unsigned int earlier = __popc(same & ((1u << lane) - 1u));
                const unsigned int had = in ? count[warp][digit] : 0u;
                rnk[j] = had + earlier;
                __syncwarp();
                if (in && earlier == 0) count[warp][digit] = had + __popc(same);
                __syncwarp();
            }
            __syncthreads();
            if (tid < 256) {
                unsigned int run = base[tid];
                for (int w = 0; w < kSortWarps; ++w) {
                    const unsigned int c = count[w][tid];
                    count[w][tid] = run;
                    run += c;
                }
                base[tid] = run;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const unsigned int i = mine + 32 * j;
                if (i < hi) {
                    const unsigned int dst = count[warp][(key[j] >> shift) & 255u] + rnk[j];
                    kout[dst] = key[j];
                    pout[dst] = pass > 0 ? __ldcg(pin + i) : i;
                }
            }
        }
        __threadfence();
        cluster_barrier();          // the next pass reads what the other CTAs placed, and clears the counts they have read
    }
}

// ---- sums over runs of equal tokens --------------------------------------------------------------------
// The sorted positions are cut into chunks of R.  A run that starts in a chunk and ends no later than the chunk after it is
// summed whole by the CTA of its first chunk.  A longer run is cut at the chunk borders: every chunk leaves the sum of its piece in
// the scratch (slot 2c+1 for the piece the run starts with, 2c for the others) and k_run_join adds the pieces in order.  So no
// CTA adds more than 2R rows, however often a token stands, and the order of the additions follows from the ids alone.
constexpr int kRunThreads = 128;
constexpr int kRunMaxR = 64;

struct RunParams {
    const unsigned int* key;
    const unsigned int* pos;
    unsigned int T;
    unsigned int V;
    int R;
    const void* dout;
    long long ld;
    int n;
    float scale;
    int accumulate;
    float* grad;               // [V][n]
    float* piece;              // [2 * chunks][n]
    unsigned int* split;       // [chunks] token of the long run that starts in the chunk, V if none
};

// Columns a thread owns: with VEC > 1 one vector, with VEC == 1 four single columns, kRunThreads apart.
template <class E, int VEC>
struct RunCols {
    static constexpr int kCols = VEC > 1 ? VEC : 4;
    static constexpr int kSlice = kRunThreads * kCols;
    struct alignas(sizeof(E) * VEC) Vec { E v[VEC]; };
    int col;
    int n;
    __device__ RunCols(int slice, int n_) : col(slice * kSlice + threadIdx.x * VEC), n(n_) {}
    __device__ bool any() const { return col < n; }
    __device__ void load(const E* row, float (&x)[kCols]) const {
        if constexpr (VEC > 1) {
            const Vec v = __ldcs_vec(reinterpret_cast<const Vec*>(row + col));
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = load_local(&v.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = col + i * kRunThreads < n ? load_as_float(row + col + i * kRunThreads) : 0.0f;
        }
    }
    __device__ static Vec __ldcs_vec(const Vec* q) {
        Vec v;
        *reinterpret_cast<uint4*>(&v) = __ldcs(reinterpret_cast<const uint4*>(q));
        return v;
    }
    // dst row (fp32): dst = a * x, or dst += a * x
    __device__ void store(float* row, const float (&x)[kCols], float a, bool add) const {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                float4* q = reinterpret_cast<float4*>(row + col + i);
                float4 o = make_float4(a * x[i], a * x[i + 1], a * x[i + 2], a * x[i + 3]);
                if (add) {
                    const float4 h = *q;
                    o.x += h.x; o.y += h.y; o.z += h.z; o.w += h.w;
                }
                *q = o;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = col + i * kRunThreads;
                if (c < n) row[c] = add ? row[c] + a * x[i] : a * x[i];
            }
        }
    }
    // fp32 row of the scratch added to x
    __device__ void add_piece(const float* row, float (&x)[kCols]) const {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 h = *reinterpret_cast<const float4*>(row + col + i);
                x[i] += h.x; x[i + 1] += h.y; x[i + 2] += h.z; x[i + 3] += h.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i * kRunThreads < n) x[i] += row[col + i * kRunThreads];
        }
    }
};

template <class E, int VEC>
__global__ void __launch_bounds__(kRunThreads) k_run_sum(const __grid_constant__ RunParams p) {
    // keys of [c*R - R, c*R + 2R], one more on the right to see where a run ends there; positions of [c*R, c*R + 2R)
    __shared__ unsigned int key[3 * kRunMaxR + 1];
    __shared__ unsigned int pos[2 * kRunMaxR];
    __shared__ int first_start, last_start, head_end, last_end;
    const int tid = threadIdx.x, R = p.R;
    const long long c0 = static_cast<long long>(blockIdx.x) * R;
    constexpr unsigned int kNone = 0xffffffffu;         // outside [0, T): no token has this key
    for (int i = tid; i < 3 * R + 1; i += kRunThreads) {
        const long long q = c0 - R + i;
        key[i] = q >= 0 && q < p.T ? p.key[q] : kNone;
    }
    for (int i = tid; i < 2 * R; i += kRunThreads) pos[i] = c0 + i < p.T ? p.pos[c0 + i] : 0u;
    if (tid == 0) { first_start = R; last_start = -1; head_end = R; last_end = 2 * R + 1; }
    __syncthreads();
    const unsigned int* k = key + R;                     // k[i]: token at position c0 + i
    for (int i = tid; i < R; i += kRunThreads) {
        if (k[i] < p.V && k[i] != k[i - 1]) { atomicMin(&first_start, i); atomicMax(&last_start, i); }
        if (k[i] != k[0]) atomicMin(&head_end, i);
    }
    __syncthreads();
    const int ls = last_start;
    if (ls >= 0)
        for (int i = ls + 1 + tid; i <= 2 * R; i += kRunThreads)
            if (k[i] != k[ls]) atomicMin(&last_end, i);  // end of the last run that starts here; 2R + 1: beyond the next chunk
    __syncthreads();
    const RunCols<E, VEC> cols(blockIdx.y, p.n);
    const bool long_start = ls >= 0 && last_end > 2 * R;
    if (blockIdx.y == 0 && tid == 0) p.split[blockIdx.x] = long_start ? k[ls] : p.V;
    if (!cols.any()) return;
    const E* dout = static_cast<const E*>(p.dout);
    constexpr int kCols = RunCols<E, VEC>::kCols;
    float acc[kCols];
    auto sum_range = [&](int a, int z, auto&& flush) {   // flush(i) after the row of position c0 + i when a run ends there
        constexpr int U = VEC > 4 ? 4 : 8;
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[j] = 0.0f;
        for (int i = a; i < z; i += U) {
            float x[U][kCols];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u < z) cols.load(dout + static_cast<long long>(pos[i + u]) * p.ld, x[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u < z) {
#pragma unroll
                    for (int j = 0; j < kCols; ++j) acc[j] += x[u][j];
                    flush(i + u);
                }
            }
        }
    };
    // a run that comes from before this chunk: one of more than two chunks leaves its piece, a shorter one is its first chunk's
    if (k[0] < p.V && k[0] == k[-1]) {
        const int e = head_end;
        // it started in the chunk before and ends here exactly when the position before that chunk's end differs somewhere in
        // [-R, 0) and it does not reach past this chunk
        bool from_previous = k[-R] != k[0];
        if (!from_previous) from_previous = blockIdx.x == 1 || p.key[c0 - R - 1] != k[0];
        const bool ends_here = e < R || k[R] != k[0];
        if (!(from_previous && ends_here)) {
            sum_range(0, e, [](int) {});
            cols.store(p.piece + static_cast<long long>(2 * blockIdx.x) * p.n, acc, 1.0f, false);
        }
    }
    if (ls < 0) return;
    const int whole_end = long_start ? ls : last_end;    // everything in [first_start, whole_end) belongs to runs summed here
    sum_range(first_start, whole_end, [&](int i) {
        if (k[i + 1] != k[i]) {
            cols.store(p.grad + static_cast<long long>(k[i]) * p.n, acc, p.scale, p.accumulate != 0);
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] = 0.0f;
        }
    });
    if (long_start) {
        sum_range(ls, R, [](int) {});
        cols.store(p.piece + static_cast<long long>(2 * blockIdx.x + 1) * p.n, acc, 1.0f, false);
    }
}

template <class E, int VEC>
__global__ void __launch_bounds__(kRunThreads) k_run_join(const __grid_constant__ RunParams p) {
    const unsigned int v = p.split[blockIdx.x];
    if (v >= p.V) return;
    const RunCols<E, VEC> cols(blockIdx.y, p.n);
    if (!cols.any()) return;
    constexpr int kCols = RunCols<E, VEC>::kCols;
    float acc[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] = 0.0f;
    cols.add_piece(p.piece + (2ll * blockIdx.x + 1) * p.n, acc);
    const long long chunks = (static_cast<long long>(p.T) + p.R - 1) / p.R;
    for (long long c = blockIdx.x + 1ll; c < chunks && p.key[c * p.R] == v; ++c) cols.add_piece(p.piece + 2 * c * p.n, acc);
    cols.store(p.grad + static_cast<long long>(v) * p.n, acc, p.scale, p.accumulate != 0);
}

}  // namespace lrgd
