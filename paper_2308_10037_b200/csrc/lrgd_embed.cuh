// Rows of a token table and the table's gradient.
//
//   lookup:    out[t,:] = scale * table[id_t,:]                                          (an id outside [0, V): zeros)
//   gradient:  grad[v,:] (+)= scale * sum over { t : id_t = v } of dout[t,:]            in fp32, v in [0, V), v != padding id
//
// The gradient sorts the positions t by their token (stable, so that a token's positions stay in order), then adds up runs of
// equal tokens: every row of the gradient is written by one thread per column, in a fixed order, without atomics on data.
#pragma once
#include <type_traits>

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

// One warp takes one piece of one row: up to 128 vectors of VEC elements (four per lane, all loaded before the first store).  HBM-bound:
// 40009 tokens of 1024 fp32 columns 36 us, 6.0 TB/s of rows read once and written; a decoding step's 16 rows 2.4 us.
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
// One cluster of eight CTAs sorts: every pass orders by nine bits of the token, least significant first (two passes for up to 2^18
// tokens).  A CTA owns a contiguous eighth of the positions; the CTAs exchange their 512 counts through distributed shared
// memory, so a pass needs two cluster barriers and no launch of its own.  Up to kSortSolo positions one CTA does all passes alone,
// without barriers between CTAs.  The other CTAs of the launch clear the first rows of the gradient meanwhile (as many as the
// time of the sort allows).
constexpr int kSortThreads = 1024;
constexpr int kSortCtas = 8;
constexpr int kSortItems = 4;                       // positions per thread and tile, at most
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortBits = 9;
constexpr int kSortBins = 1 << kSortBits;
constexpr unsigned int kSortSolo = 2048;

struct SortParams {
    const void* ids;
    unsigned int T;
    long long V;               // also the key of positions without a gradient (padding, ids outside the table): sorted last
    long long padding;
    uint2* place[2];           // [T] each: token and position; pass i writes buffer i & 1
    int passes;
    int* status;
    unsigned int* present;     // nullable: one bit per token that has a position
    unsigned int* long_runs;   // set to 0: k_run_sum counts there
    float* zero;               // floats to be cleared
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
// Zeros by `threads` threads, 16 bytes at a time; `me` numbers them.
__device__ __forceinline__ void clear_floats(float* z, long long count, long long me, long long threads) {
    const long long head = min(count, static_cast<long long>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / 4);
    const long long quads = (count - head) / 4;
    float4* q = reinterpret_cast<float4*>(z + head);
    for (long long i = me; i < quads; i += threads) q[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (me < head) z[me] = 0.f;
    if (me < count - head - quads * 4) z[head + quads * 4 + me] = 0.f;
}

// What another CTA of the cluster has placed: from L2, and not before the barrier that this follows.
__device__ __forceinline__ uint2 load_placed(const uint2* p) {
    uint2 v;
    asm volatile("ld.global.cg.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
// Lanes whose digit is the same (all 32 lanes call it; `digit` has kSortBits + 1 bits): one ballot per bit.
__device__ __forceinline__ unsigned int lanes_alike(unsigned int digit) {
    unsigned int same = 0xffffffffu;
#pragma unroll
    for (int b = 0; b <= kSortBits; ++b) {
        const bool bit = (digit >> b) & 1u;
        const unsigned int with = __ballot_sync(0xffffffffu, bit);
        same &= bit ? with : ~with;
    }
    return same;
}

template <class Id>
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) k_token_sort(const __grid_constant__ SortParams p) {
    __shared__ unsigned short count[kSortWarps][kSortBins];      // of a tile: at most 4096
    __shared__ unsigned int hist[kSortBins], base[kSortBins], scan[kSortBins / 32];
    __shared__ unsigned short half[2][kSortBins];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_release();                      // the kernels after this one wait for its end on the device
    if (blockIdx.x >= kSortCtas) {
        clear_floats(p.zero, p.zero_count, static_cast<long long>(blockIdx.x - kSortCtas) * kSortThreads + tid,
                     static_cast<long long>(gridDim.x - kSortCtas) * kSortThreads);
        return;
    }
    const int rank = blockIdx.x;
    const bool solo = p.T <= kSortSolo;
    if (rank == 0 && tid == 0) *p.long_runs = 0;
    if (p.present) {
        const long long words = (p.V + 31) / 32;
        for (long long i = rank * kSortThreads + tid; i < words; i += kSortThreads * kSortCtas) p.present[i] = 0;
        cluster_barrier();
    }
    if (solo && rank > 0) return;
    const unsigned int per = solo ? p.T : (p.T + kSortCtas - 1) / kSortCtas;
    const unsigned int lo = min(p.T, per * rank), hi = min(p.T, lo + per);
    const unsigned int items = min(static_cast<unsigned int>(kSortItems), (per + kSortThreads - 1) / kSortThreads);
    auto token_key = [&](unsigned int i) -> unsigned int {
        const long long id = load_id<Id>(p.ids, i);
        return id < 0 || id >= p.V || id == p.padding ? static_cast<unsigned int>(p.V) : static_cast<unsigned int>(id);
    };
    for (unsigned int i = lo + tid; i < hi; i += kSortThreads) {
        const long long id = load_id<Id>(p.ids, i);
        if (id < 0 || id >= p.V) atomicExch(p.status, -4);      // LR_ERR_VALUE, also where padding_id (then no row of the table) says the same
        const unsigned int k = token_key(i);
        if (p.present && k < p.V) atomicOr(p.present + (k >> 5), 1u << (k & 31));
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = kSortBits * pass;
        const uint2* from = p.place[(pass + 1) & 1];
        uint2* to = p.place[pass & 1];
        auto place_at = [&](unsigned int i) -> uint2 { return pass > 0 ? load_placed(from + i) : make_uint2(token_key(i), i); };
        auto digit_of = [&](unsigned int key) { return (key >> shift) & (kSortBins - 1u); };
        // first place of this CTA's elements of digit `tid` (threads below kSortBins): all smaller digits, then the same digit of
        // the CTAs before this one.  Every thread calls it.
        auto digit_base = [&](unsigned int total, unsigned int before) {
            unsigned int inc = total;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const unsigned int o = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += o;
            }
            if (tid < kSortBins && lane == 31) scan[warp] = inc;
            __syncthreads();
            if (tid < kSortBins) {
                unsigned int add = 0;
#pragma unroll
                for (int w = 0; w < kSortBins / 32; ++w) add += w < warp ? scan[w] : 0u;
                base[tid] = add + inc - total + before;
            }
        };
        if (!solo) {
            if (tid < kSortBins) hist[tid] = 0;
            __syncthreads();
            for (unsigned int i = lo + tid; i < hi; i += kSortThreads) atomicAdd(&hist[digit_of(place_at(i).x)], 1u);
            cluster_barrier();
            unsigned int total = 0, before = 0;
            if (tid < kSortBins) {
#pragma unroll
                for (int r = 0; r < kSortCtas; ++r) {
                    const unsigned int h = cluster_load_u32(&hist[tid], r);
                    if (r < rank) before += h;
                    total += h;
                }
            }
            digit_base(total, before);
        }
        // tiles of up to 4096 positions; a warp ranks 32 * items consecutive ones, 32 at a time
        for (unsigned int tile = lo; tile < hi; tile += kSortThreads * items) {
            uint2 place[kSortItems];
            unsigned int rnk[kSortItems];
            const unsigned int mine = tile + warp * 32 * items + lane;
            auto in = [&](int j) { return j < items && mine + 32 * j < hi; };
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) place[j] = in(j) ? place_at(mine + 32 * j) : make_uint2(0u, 0u);
            __syncthreads();                        // the tile before this one is done with count
#pragma unroll
            for (int i = 0; i < kSortBins / 64; ++i) reinterpret_cast<uint32_t*>(count[warp])[i * 32 + lane] = 0;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (j < items) {
                    const unsigned int digit = in(j) ? digit_of(place[j].x) : kSortBins;
                    const unsigned int same = lanes_alike(digit);
                    const unsigned int earlier = __popc(same & ((1u << lane) - 1u));
                    const unsigned int had = in(j) ? count[warp][digit] : 0u;
                    rnk[j] = had + earlier;
                    __syncwarp();
                    if (in(j) && earlier == 0) count[warp][digit] = static_cast<unsigned short>(had + __popc(same));
                    __syncwarp();
                }
            }
            __syncthreads();
            // how many of the same digit the warps before have: two threads per digit add up sixteen warps each
            const int d = tid & (kSortBins - 1), part = tid / kSortBins;
            unsigned int sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps / 2; ++w) {
                const unsigned int c = count[part * (kSortWarps / 2) + w][d];
                count[part * (kSortWarps / 2) + w][d] = static_cast<unsigned short>(sum);
                sum += c;
            }
            half[part][d] = static_cast<unsigned short>(sum);
            __syncthreads();
            if (solo) {
                digit_base(tid < kSortBins ? half[0][d] + half[1][d] : 0u, 0u);
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (in(j)) {
                    const unsigned int digit = digit_of(place[j].x);
                    const unsigned int dst = base[digit] + (warp >= kSortWarps / 2 ? half[0][digit] : 0u) + count[warp][digit] + rnk[j];
                    to[dst] = place[j];
                }
            }
            if (tile + kSortThreads * items < hi) {
                __syncthreads();
                if (part == 0) base[d] += half[0][d] + half[1][d];
            }
        }
        if (solo) __syncthreads();                  // (one CTA: its own stores are visible to it)
        else cluster_barrier();                     // the next pass reads what the other CTAs placed, and clears the counts they have read
    }
}

// ---- sums over runs of equal tokens --------------------------------------------------------------------
// The sorted positions are cut into chunks of R.  A run that starts in a chunk and ends no later than the chunk after it is
// summed whole by the CTA of its first chunk.  A longer run is cut at the chunk borders: every chunk leaves the sum of its piece in
// the scratch (slot 2c+1 for the piece the run starts with, 2c for the others) and k_run_join adds the pieces in a fixed order.  So
// no CTA adds more than 2R rows, however often a token stands, and the order of the additions follows from the ids alone.
// 32768 tokens into 65536 x 1024 (bfloat16 rows): 75 us in all, 336 MB at 4.5 TB/s; the sort takes about 25 of them, the sums 31, the
// join 8 to 13.  Chunks of 64 with four rows in flight took 72 us for the sums alone (too few loads under way).
// Further CTAs of both kernels clear the rows of tokens that do not occur (all but the ones cleared during the sort): the join is
// a few CTAs' work and leaves the memory idle otherwise.
constexpr int kRunThreads = 128;
constexpr int kRunMaxR = 32;
constexpr int kRunAhead = 8;                        // rows loaded before the first of them is added

struct RunParams {
    const uint2* place;        // sorted: token and position
    unsigned int T;
    unsigned int V;
    int R;
    int chunks;
    int slices;                // column slices
    const void* dout;
    long long ld;
    int n;
    float scale;
    float* grad;               // [V][n]
    float* piece;              // [2 * chunks][n]
    unsigned int* long_runs;   // [1 + chunks / 2 + 1]: their number, then the chunks they start in
    const unsigned int* present;
    // rows of tokens that do not occur: [clear[0], clear[1]) is cleared beside the sums, [clear[1], V) beside the join
    long long clear[2];
    int clear_rows;            // rows per clearing CTA
    int joiners;               // CTAs of k_run_join per column slice
};

// Columns a thread owns: with VEC > 1 one 16-byte vector, with VEC == 1 two single columns, kRunThreads apart.
template <class E, int VEC>
struct RunCols {
    static constexpr int kCols = VEC > 1 ? VEC : 2;
    static constexpr int kSlice = kRunThreads * kCols;
    using Raw = typename std::conditional<(VEC > 1), uint4, float2>::type;
    int col;
    int n;
    __device__ RunCols(int slice, int n_, int thread) : col(slice * kSlice + thread * VEC), n(n_) {}
    __device__ bool any() const { return col < n; }
    __device__ Raw load(const E* row) const {
        if constexpr (VEC > 1) {
            return __ldcs(reinterpret_cast<const uint4*>(row + col));
        } else {
            return make_float2(load_as_float(row + col), col + kRunThreads < n ? load_as_float(row + col + kRunThreads) : 0.0f);
        }
    }
    __device__ static void add(float (&acc)[kCols], const Raw& x) {
        if constexpr (VEC == 1) {
            acc[0] += x.x;
            acc[1] += x.y;
        } else if constexpr (sizeof(E) == 4) {
            acc[0] += __uint_as_float(x.x); acc[1] += __uint_as_float(x.y); acc[2] += __uint_as_float(x.z); acc[3] += __uint_as_float(x.w);
        } else {
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[2 * i] += __uint_as_float(w[i] << 16);
                acc[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // fp32 row: = a * x + held
    __device__ void store(float* row, const float (&x)[kCols], float a, const float (&held)[kCols]) const {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4)
                *reinterpret_cast<float4*>(row + col + i) = make_float4(a * x[i] + held[i], a * x[i + 1] + held[i + 1], a * x[i + 2] + held[i + 2], a * x[i + 3] + held[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (col + i * kRunThreads < n) row[col + i * kRunThreads] = a * x[i] + held[i];
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
            for (int i = 0; i < 2; ++i)
                if (col + i * kRunThreads < n) x[i] += row[col + i * kRunThreads];
        }
    }
};

// CTA `index` of those that clear rows [from, to): its clear_rows of them, where no token points there.  The bits of 32 rows are
// taken into a register at once, so that the stores of one row do not wait for the look at the next.
__device__ __forceinline__ void clear_absent_rows(const RunParams& p, long long from, long long to, long long index) {
    const long long r0 = from + index * p.clear_rows, r1 = min(to, r0 + p.clear_rows);
    if (p.n >= kRunThreads) {
        const int group = threadIdx.x / kRunThreads, groups = blockDim.x / kRunThreads, t = threadIdx.x % kRunThreads;
        const bool whole = p.n % 4 == 0 && (reinterpret_cast<uintptr_t>(p.grad) & 15) == 0;
        const int quads = p.n / 4;
        for (long long v0 = r0 & ~31ll; v0 < r1; v0 += 32) {
            const uint32_t here = p.present[v0 >> 5];
#pragma unroll 4
            for (int k = group; k < 32; k += groups) {
                const long long v = v0 + k;
                if (v < r0 || v >= r1 || ((here >> k) & 1u)) continue;
                float* row = p.grad + v * p.n;
                if (whole) {
                    for (int i = t; i < quads; i += kRunThreads) reinterpret_cast<float4*>(row)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                } else {
                    for (int i = t; i < p.n; i += kRunThreads) row[i] = 0.f;
                }
            }
        }
    } else if (r1 > r0) {                                // narrow rows: several at a time
        const int count = static_cast<int>(r1 - r0) * p.n;
        for (int i = threadIdx.x; i < count; i += blockDim.x) {
            const long long v = r0 + i / p.n;
            if (!((p.present[v >> 5] >> (v & 31)) & 1u)) p.grad[r0 * p.n + i] = 0.f;
        }
    }
}

template <class E, int VEC, bool ADD>
__global__ void __launch_bounds__(kRunThreads) k_run_sum(const __grid_constant__ RunParams p) {
    // keys of [c*R - R, c*R + 2R], one more on the right to see where a run ends there; positions of [c*R, c*R + 2R)
    __shared__ unsigned int key[3 * kRunMaxR + 1];
    __shared__ unsigned int pos[2 * kRunMaxR];
    __shared__ int first_start, last_start, head_end, last_end;
    const int tid = threadIdx.x, R = p.R;
    grid_dependency_release();
    grid_dependency_wait();                              // the sort, and the rows it clears
    const int chunk = blockIdx.x / p.slices;
    if (chunk >= p.chunks) {
        clear_absent_rows(p, p.clear[0], p.clear[1], static_cast<long long>(blockIdx.x) - p.chunks * p.slices);
        return;
    }
    const int slice = blockIdx.x - chunk * p.slices;
    const long long c0 = static_cast<long long>(chunk) * R;
    constexpr unsigned int kNone = 0xffffffffu;         // outside [0, T): no token has this key
    for (int i = tid; i < 3 * R + 1; i += kRunThreads) {
        const long long q = c0 - R + i;
        const uint2 at = q >= 0 && q < p.T ? p.place[q] : make_uint2(kNone, 0u);
        key[i] = at.x;
        if (i >= R && i < 3 * R) pos[i - R] = at.y;
    }
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
    const RunCols<E, VEC> cols(slice, p.n, tid);
    const bool long_start = ls >= 0 && last_end > 2 * R;
    if (long_start && slice == 0 && tid == 0) p.long_runs[1 + atomicAdd(p.long_runs, 1u)] = chunk;   // (their order does not matter)
    if (!cols.any()) return;
    const E* dout = static_cast<const E*>(p.dout);
    using Cols = RunCols<E, VEC>;
    float acc[Cols::kCols], none[Cols::kCols];
#pragma unroll
    for (int j = 0; j < Cols::kCols; ++j) none[j] = 0.0f;
    // Rows [a, z) of the chunk, a few loaded ahead; WHOLE: a run that ends is written to the gradient (what the row holds is
    // fetched with the rows, so that no addition waits for it), otherwise all of them are one sum.
    auto sum_range = [&](int a, int z, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value, HELD = WHOLE && ADD;
        constexpr int U = HELD && VEC > 4 ? kRunAhead / 2 : kRunAhead;
#pragma unroll
        for (int j = 0; j < Cols::kCols; ++j) acc[j] = 0.0f;
        for (int i = a; i < z; i += U) {
            typename Cols::Raw x[U];
            float held[HELD ? U : 1][Cols::kCols];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u < z) {
                    x[u] = cols.load(dout + static_cast<long long>(pos[i + u]) * p.ld);
                    if constexpr (HELD) {
#pragma unroll
                        for (int j = 0; j < Cols::kCols; ++j) held[u][j] = 0.0f;
                        if (k[i + u + 1] != k[i + u]) cols.add_piece(p.grad + static_cast<long long>(k[i + u]) * p.n, held[u]);
                    }
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u < z) {
                    Cols::add(acc, x[u]);
                    if (WHOLE && k[i + u + 1] != k[i + u]) {
                        cols.store(p.grad + static_cast<long long>(k[i + u]) * p.n, acc, p.scale, HELD ? held[HELD ? u : 0] : none);
#pragma unroll
                        for (int j = 0; j < Cols::kCols; ++j) acc[j] = 0.0f;
                    }
                }
            }
        }
    };
    // a run that comes from before this chunk: one of more than two chunks leaves its piece, a shorter one is its first chunk's
    if (k[0] < p.V && k[0] == k[-1]) {
        // it started in the chunk before when a position of that chunk, or the one just before it, holds another token
        bool from_previous = k[-R] != k[0];
        if (!from_previous) from_previous = chunk == 1 || p.place[c0 - R - 1].x != k[0];
        const bool ends_here = head_end < R || k[R] != k[0];
        if (!(from_previous && ends_here)) {
            sum_range(0, head_end, std::false_type{});
            cols.store(p.piece + 2ll * chunk * p.n, acc, 1.0f, none);
        }
    }
    if (ls < 0) return;
    const int whole_end = long_start ? ls : last_end;    // everything in [first_start, whole_end) belongs to runs summed here
    sum_range(first_start, whole_end, std::true_type{});
    if (long_start) {
        sum_range(ls, R, std::false_type{});
        cols.store(p.piece + (2ll * chunk + 1) * p.n, acc, 1.0f, none);
    }
}

// Long runs: eight groups of threads take every eighth piece of a run, the eight sums are added in turn.
constexpr int kJoinGroups = 8;

template <class E, int VEC, bool ADD>
__global__ void __launch_bounds__(kRunThreads* kJoinGroups) k_run_join(const __grid_constant__ RunParams p) {
    using Cols = RunCols<E, VEC>;
    __shared__ float sums[kJoinGroups - 1][Cols::kCols][kRunThreads];
    __shared__ int last_chunk;
    const int tid = threadIdx.x % kRunThreads, group = threadIdx.x / kRunThreads;
    grid_dependency_wait();
    const int joiners = p.joiners * p.slices;
    if (static_cast<int>(blockIdx.x) >= joiners) {
        clear_absent_rows(p, p.clear[1], p.V, static_cast<long long>(blockIdx.x) - joiners);
        return;
    }
    const Cols cols(blockIdx.x % p.slices, p.n, tid);
    const unsigned int runs = *p.long_runs;
    for (unsigned int r = blockIdx.x / p.slices; r < runs; r += p.joiners) {
        const int chunk = static_cast<int>(p.long_runs[1 + r]);
        const unsigned int v = p.place[static_cast<long long>(chunk + 1) * p.R].x;      // the run covers the chunk after its first
        // how far it goes: the first chunk whose first position holds another token
        if (threadIdx.x == 0) last_chunk = p.chunks;
        __syncthreads();
        for (int c = chunk + 1 + threadIdx.x; c < last_chunk; c += kRunThreads * kJoinGroups)
            if (p.place[static_cast<long long>(c) * p.R].x != v) { atomicMin(&last_chunk, c); break; }
        __syncthreads();
        const int end = last_chunk;
        float acc[Cols::kCols];
#pragma unroll
        for (int j = 0; j < Cols::kCols; ++j) acc[j] = 0.0f;
        if (cols.any()) {
            if (group == 0) cols.add_piece(p.piece + (2ll * chunk + 1) * p.n, acc);
#pragma unroll 4
            for (int c = chunk + 1 + group; c < end; c += kJoinGroups) cols.add_piece(p.piece + 2ll * c * p.n, acc);
        }
        if (group > 0)
#pragma unroll
            for (int j = 0; j < Cols::kCols; ++j) sums[group - 1][j][tid] = acc[j];
        __syncthreads();
        if (group == 0 && cols.any()) {
#pragma unroll
            for (int g = 0; g < kJoinGroups - 1; ++g)
#pragma unroll
                for (int j = 0; j < Cols::kCols; ++j) acc[j] += sums[g][j][tid];
            float* row = p.grad + static_cast<long long>(v) * p.n;
            float held[Cols::kCols];
#pragma unroll
            for (int j = 0; j < Cols::kCols; ++j) held[j] = 0.0f;
            if (ADD) cols.add_piece(row, held);
            cols.store(row, acc, p.scale, held);
        }
        __syncthreads();
    }
}

}  // namespace lrgd
