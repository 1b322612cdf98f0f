// cache.hip -- rows of per-beam states and of a paged cache around a decoding step, on
// gfx950: states of the chosen beams (resispec_beam_reorder, resispec_beam_reorder_paged),
// pages and slots of new rows (resispec_plan_cache), accepted paths of verified trees
// (resispec_accepted_path) and their rows' places in the cache (resispec_commit_path).
// Declared in resispec.h.

#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>
#include <type_traits>

#include "resispec.h"

namespace {

// Vectors of 16 bytes at any address: rows need not be a multiple of 16 bytes long, nor start
// on one, and gfx950 loads and stores such vectors in one instruction.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

template <typename T>
struct Any;
template <>
struct Any<u32x4> {
    using type = u32x4_any;
};
template <>
struct Any<u32x2> {
    using type = u32x2_any;
};
template <>
struct Any<uint8_t> {
    using type = uint8_t;
};
template <typename T>
__device__ __forceinline__ T load_at(const uint8_t* p) {
    return *reinterpret_cast<const typename Any<T>::type*>(p);
}
template <typename T>
__device__ __forceinline__ void store_at(uint8_t* p, T v) {
    *reinterpret_cast<typename Any<T>::type*>(p) = v;
}

__device__ __forceinline__ int uniform_i(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---------------------------------------------------------------- reorder ----

// States move for all beams of a sequence at once.  A lane owns a column, 16 bytes (or one)
// at one place of every beam's state: it loads the new value of each beam and then stores
// them, so a move in place needs no second buffer and no wait between workgroups.  A wave
// takes a piece, positions that lie one after another, and its addresses are scalar.
struct ReorderParams {
    const uint8_t* src;
    uint8_t* dst;
    rs_rows s, d;
    const int32_t* parent;           // [B][K]
    const int32_t* lengths;          // [B] or NULL
    const int32_t *src_table, *dst_table;
    int64_t src_table_stride, dst_table_stride;
    int32_t max_pages;               // entries of a table's row
    int32_t W, K, G;                 // workgroups a sequence
    int32_t step, per_page;          // positions a piece, pieces a page
    int32_t* status;
};

constexpr int kReorderBlock = 256, kReorderWaves = kReorderBlock / 64;
constexpr int64_t kPieceBytes = 4096;

template <int KMAX, typename T, bool PAGED>
__global__ void __launch_bounds__(kReorderBlock) rs_reorder_kernel(const ReorderParams P) {
    const int b = blockIdx.x / P.G, g = blockIdx.x % P.G;
    const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
    const int32_t* parent = P.parent + (int64_t)b * P.K;
    const int S = (int)P.s.positions;
    const int64_t room = PAGED ? (int64_t)P.max_pages * S : S;
    const int64_t len = P.lengths ? P.lengths[b] : S;
    const int mine = lane < P.K ? parent[lane] : -1;
    const bool bad = __ballot(mine < -1 || mine >= P.W) != 0 || len < 0 || len > room;
    const int32_t* from_table = PAGED ? P.src_table + (int64_t)b * P.W * P.src_table_stride : nullptr;
    const int32_t* to_table = PAGED ? P.dst_table + (int64_t)b * P.K * P.dst_table_stride : nullptr;
    if (g == 0 && P.status) {
        int st = bad ? RS_SEQ_BAD_PARAM : RS_SEQ_OK;
        if (PAGED && !bad) {
            // every page that the sequence's rows are moved from or to
            const int used = (int)((len + S - 1) / S);
            bool out = false;
            for (int e = threadIdx.x; e < used; e += kReorderBlock)
                for (int k = 0; k < P.K; ++k) {
                    const int w = parent[k];
                    if (w < 0) continue;
                    out |= (uint32_t)from_table[w * P.src_table_stride + e] >= (uint32_t)P.s.pages;
                    out |= (uint32_t)to_table[k * P.dst_table_stride + e] >= (uint32_t)P.d.pages;
                }
            if (__syncthreads_or(out)) st = RS_SEQ_BAD_PAGE;
        }
        if (threadIdx.x == 0) P.status[b] = st;
    }
    if (bad || len == 0) return;
    const uint32_t full = (uint32_t)(len / S), rest = (uint32_t)(len % S);
    const uint32_t nq = full * P.per_page + (rest + P.step - 1) / P.step;
    const uint32_t inner = (uint32_t)P.s.inner, pieces = (uint32_t)P.s.outer * inner * nq;
    for (uint32_t piece = g * kReorderWaves + wave; piece < pieces; piece += P.G * kReorderWaves) {
        const uint32_t q = piece % nq, oi = piece / nq, i = oi % inner, o = oi / inner;
        const uint32_t page = q / P.per_page, t = (q % P.per_page) * P.step;
        const uint32_t end = min(t + P.step, page < full ? (uint32_t)S : rest);
        const int64_t bytes = (int64_t)(end - t) * P.s.row_bytes;
        const int64_t from0 = o * P.s.outer_stride + i * P.s.inner_stride + t * P.s.position_stride;
        const int64_t to0 = o * P.d.outer_stride + i * P.d.inner_stride + t * P.d.position_stride;
        const uint8_t* from[KMAX];
        uint8_t* to[KMAX];
#pragma unroll
        for (int k = 0; k < KMAX; ++k) {
            from[k] = nullptr;
            to[k] = nullptr;
            if (k >= P.K) continue;
            const int w = parent[k];
            if (w < 0) continue;
            int64_t f, d;
            if (PAGED) {
                f = from_table[w * P.src_table_stride + page];
                d = to_table[k * P.dst_table_stride + page];
                if ((uint64_t)f >= (uint64_t)P.s.pages || (uint64_t)d >= (uint64_t)P.d.pages) continue;
            } else {
                f = (int64_t)b * P.W + w;
                d = (int64_t)b * P.K + k;
            }
            const uint8_t* x = P.src + from0 + f * P.s.page_stride;
            uint8_t* y = P.dst + to0 + d * P.d.page_stride;
            if (x == y) continue;       // where it is
            from[k] = x;
            to[k] = y;
        }
        const int64_t whole = bytes / (int64_t)sizeof(T) * (int64_t)sizeof(T);
        for (int64_t c = lane * (int64_t)sizeof(T); c < whole; c += 64 * sizeof(T)) {
            T v[KMAX];
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (from[k]) v[k] = load_at<T>(from[k] + c);
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (from[k]) store_at<T>(to[k] + c, v[k]);
        }
        if (whole + lane < bytes) {
            const int64_t c = whole + lane;
            uint8_t v[KMAX];
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (from[k]) v[k] = from[k][c];
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (from[k]) to[k][c] = v[k];
        }
    }
}

// ------------------------------------------------------------------- plan ----

struct PlanParams {
    const int32_t *kept, *added, *held;
    int32_t R, page_size;
    int32_t* table;
    int64_t table_stride;
    int32_t max_pages;
    int32_t* free_pages;
    const int32_t* free_count;
    int32_t num_pages;
    int32_t *out_held, *out_free_count, *out_starts;
    int32_t T;
    int32_t *slots, *positions, *requests, *status;
};

constexpr int kPlanBlock = 1024;

// The sum over a workgroup's threads up to each, in order, and the whole sum.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t (&part)[kPlanBlock / 64], int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(v, d);
        if (lane >= d) v += x;
    }
    __syncthreads();
    if (lane == 63) part[wave] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < kPlanBlock / 64; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    return v + before;
}

// The slot, position and request of new row t.
__device__ __forceinline__ void plan_row(const PlanParams& P, const int32_t* starts, int t) {
    int slot = -1, position = -1, request = -1;
    if (P.R > 0 && t < starts[P.R]) {
        int lo = 0, hi = P.R;           // starts[lo] <= t < starts[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        const int64_t k = P.kept[lo], n = P.added[lo], want = (k + n + P.page_size - 1) / P.page_size;
        // granted: it holds what it wants, and its rows fit
        if (P.out_held[lo] == want && starts[lo] + n <= P.T) {
            const int p = (int)(k + t - starts[lo]);
            const int page = P.table[lo * P.table_stride + p / P.page_size];
            position = p;
            request = lo;
            if ((uint32_t)page < (uint32_t)P.num_pages) slot = page * P.page_size + p % P.page_size;
            else if (P.status) P.status[lo] = RS_SEQ_BAD_PAGE;
        }
    }
    P.slots[t] = slot;
    if (P.positions) P.positions[t] = position;
    if (P.requests) P.requests[t] = request;
}

// One workgroup, 1024 requests at a time, in two passes: the first has the running sums of
// rows and gives pages back, the second takes pages.  ROWS: it does the new rows as well.
template <bool ROWS>
__global__ void __launch_bounds__(kPlanBlock) rs_plan_kernel(const PlanParams P) {
    __shared__ int64_t part[kPlanBlock / 64];
    __shared__ int32_t released, taken;
    const int tid = threadIdx.x;
    const int count = P.free_count[0];
    const bool count_ok = count >= 0 && count <= P.num_pages;
    if (tid == 0) released = taken = 0;

    struct Request {
        int32_t held, want, give, need, status;
        int64_t first;
    };
    int64_t rows = 0, given = 0;        // before this tile
    int64_t given_before = 0;           // this request's place among the pages given back
    auto look = [&](int r, Request& q) {
        q = {0, 0, 0, 0, RS_SEQ_OK, 0};
        int64_t n = 0;
        if (r < P.R) {
            const int64_t k = P.kept[r];
            n = P.added[r];
            q.held = P.held[r];
            if (k < 0 || n < 0 || q.held < 0 || q.held > P.max_pages || k + n > (int64_t)P.max_pages * P.page_size) {
                q.status = RS_SEQ_BAD_PARAM;
                n = 0;
            } else {
                q.want = (int32_t)((k + n + P.page_size - 1) / P.page_size);
            }
        }
        int64_t total;
        const int64_t upto = rows + block_scan(n, part, total);
        rows += total;
        q.first = upto - n;
        if (q.status == RS_SEQ_OK && n > 0 && upto > P.T) q.status = RS_SEQ_NO_ROOM;
        if (q.status == RS_SEQ_OK) {
            q.give = max(q.held - q.want, 0);
            q.need = max(q.want - q.held, 0);
            if (!count_ok && (q.give || q.need)) q.status = RS_SEQ_BAD_PARAM;
        }
        if (q.status != RS_SEQ_OK) q.give = q.need = 0;
        const int64_t gives = given + block_scan(q.give, part, total);
        given += total;
        given_before = gives - q.give;
        if (q.give && count + gives > P.num_pages) {
            q.status = RS_SEQ_BAD_PARAM;
            q.give = 0;
        }
    };
    Request q;
    const int tiles = (P.R + kPlanBlock - 1) / kPlanBlock;
    for (int i = 0; i < tiles; ++i) {
        const int r = i * kPlanBlock + tid;
        look(r, q);
        for (int j = 0; j < q.give; ++j)
            P.free_pages[count + given_before + j] = P.table[r * P.table_stride + q.want + j];
        if (q.give) atomicAdd(&released, q.give);
    }
    __syncthreads();
    const int avail = count + released;
    const int64_t all_rows = rows;
    int64_t needed = 0;
    rows = given = 0;
    for (int i = 0; i < tiles; ++i) {
        const int r = i * kPlanBlock + tid;
        if (tiles > 1) look(r, q);
        int64_t total;
        const int64_t upto = needed + block_scan(q.need, part, total);
        needed += total;
        if (q.need && upto > avail) {
            q.status = RS_SEQ_NO_ROOM;
            q.need = 0;
        }
        for (int j = 0; j < q.need; ++j)
            P.table[r * P.table_stride + q.held + j] = P.free_pages[avail - 1 - (upto - q.need + j)];
        if (q.need) atomicAdd(&taken, q.need);
        if (r < P.R) {
            P.out_held[r] = q.status == RS_SEQ_OK ? q.want : q.held;
            P.out_starts[r] = (int32_t)min(q.first, (int64_t)INT_MAX);
            if (P.status) P.status[r] = q.status;
        }
    }
    __syncthreads();
    if (tid == 0) {
        P.out_starts[P.R] = (int32_t)min(all_rows, (int64_t)INT_MAX);
        P.out_free_count[0] = avail - taken;
    }
    if (ROWS) {
        __syncthreads();
        for (int t = tid; t < P.T; t += kPlanBlock) plan_row(P, P.out_starts, t);
    }
}

__global__ void __launch_bounds__(256) rs_plan_rows_kernel(const PlanParams P) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < P.T) plan_row(P, P.out_starts, (int)t);
}

// ------------------------------------------------------------------- path ----

// One workgroup a sequence.  A node of level d carries the tokens if its token is the d-th and
// its parent carries those before: one step over the nodes for each accepted token, with the
// levels of the nodes that do, and the parents, in LDS.
__global__ void rs_path_nodes_kernel(const int32_t* __restrict__ parent, const int32_t* __restrict__ node_token,
                                     const int32_t* __restrict__ tokens, const int32_t* __restrict__ accepted_len,
                                     int32_t N, int32_t max_depth, int32_t* __restrict__ path, int32_t* status) {
    extern __shared__ uint16_t tree[];      // [N] levels + 1 (0: carries none), [N] parents
    __shared__ int32_t last;
    uint16_t *level = tree, *up = tree + N;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x, width = max_depth + 1;
    parent += b * N;
    node_token += b * N;
    tokens += b * width;
    path += b * width;
    const int len = accepted_len[b];
    int st = len < -1 || len > max_depth ? RS_SEQ_DEPTH_EXCEEDED : RS_SEQ_OK;
    bool bad = false;
    for (int n = tid; n < N; n += blockDim.x) {
        const int p = parent[n];
        bad |= n == 0 ? p != -1 : p < 0 || p >= n;
        up[n] = (uint16_t)p;
        level[n] = n == 0;
    }
    if (tid == 0) last = N;
    if (__syncthreads_or(bad) && st == RS_SEQ_OK) st = RS_SEQ_BAD_TREE;
    int on = 0;                             // entries of the path
    if (st == RS_SEQ_OK && len >= 0 && len < N) {
        for (int d = 1; d <= len; ++d) {
            const int x = tokens[d - 1];
            for (int n = tid; n < N; n += blockDim.x)
                if (n > 0 && level[up[n]] == d && node_token[n] == x) level[n] = (uint16_t)(d + 1);
            __syncthreads();
        }
        for (int n = tid; n < N; n += blockDim.x)
            if (level[n] == len + 1) {
                atomicMin(&last, n);
                break;
            }
        __syncthreads();
        if (last < N) on = len + 1;
    }
    if (st == RS_SEQ_OK && len >= 0 && on == 0) st = RS_SEQ_BAD_TREE;
    for (int i = on + tid; i < width; i += blockDim.x) path[i] = -1;
    if (tid == 0) {
        int n = last;
        for (int i = on - 1; i >= 0; --i) {
            path[i] = n;
            n = up[n];
        }
        if (status) status[b] = st;
    }
}

// ----------------------------------------------------------------- commit ----

struct CommitParams {
    uint8_t* cache;
    rs_rows c;
    const int32_t *slots, *path;
    const uint8_t* source;               // NULL: the cache
    rs_rows s;
    int32_t N, depth, G;                 // workgroups a sequence
    int32_t* status;
};

constexpr int kCommitBlock = 256, kCommitWaves = kCommitBlock / 64, kCommitRows = 64;

// A lane owns a column of 16 bytes (or one) of all rows of a path, as in the reorder.  Paths
// ascend, so path[j] >= j: the slot that row i goes to, slots[i], is the source of none after
// it, and the rows are moved in order, eight loaded before they are stored.
__global__ void __launch_bounds__(kCommitBlock) rs_commit_kernel(const CommitParams P) {
    __shared__ int64_t from[kCommitRows], to[kCommitRows];
    __shared__ int32_t count;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6);
    const int b = blockIdx.x / P.G, g = blockIdx.x % P.G;
    const int32_t* path = P.path + (int64_t)b * P.depth;
    const int32_t* slots = P.slots + (int64_t)b * P.N;
    const uint32_t room = (uint32_t)(P.c.pages * P.c.positions), page = (uint32_t)P.c.positions;
    if (tid == 0) count = P.depth;
    __syncthreads();
    for (int i = tid; i < P.depth; i += kCommitBlock)
        if (path[i] == -1) {
            atomicMin(&count, i);
            break;
        }
    __syncthreads();
    const int n = count;
    bool order = false, out = false;
    for (int i = tid; i < n; i += kCommitBlock) {
        const int x = path[i];
        if (x < i || x >= P.N || (i > 0 && x <= path[i - 1])) order = true;
        else out |= (uint32_t)slots[i] >= room || (!P.source && (uint32_t)slots[x] >= room);
    }
    const bool wrong = __syncthreads_or(order), outside = __syncthreads_or(out);
    if (g == 0 && tid == 0 && P.status) P.status[b] = wrong ? RS_SEQ_BAD_TREE : outside ? RS_SEQ_BAD_PAGE : RS_SEQ_OK;
    if (wrong || outside) return;
    const uint32_t inner = (uint32_t)P.c.inner, pieces = (uint32_t)P.c.outer * inner;
    const int64_t bytes = P.c.row_bytes, whole = bytes & ~(int64_t)15;
    const uint8_t* source = P.source ? P.source : P.cache;
    const rs_rows& s = P.source ? P.s : P.c;
    for (int first = 0; first < n; first += kCommitRows) {
        const int rows = min(n - first, kCommitRows);
        __syncthreads();
        if (tid < rows) {
            const int x = path[first + tid];
            const uint32_t slot = (uint32_t)slots[first + tid];
            to[tid] = slot / page * P.c.page_stride + slot % page * P.c.position_stride;
            if (P.source) {
                from[tid] = b * P.s.page_stride + x * P.s.position_stride;
            } else {
                const uint32_t was = (uint32_t)slots[x];
                from[tid] = was / page * P.c.page_stride + was % page * P.c.position_stride;
            }
        }
        __syncthreads();
        for (uint32_t piece = g * kCommitWaves + wave; piece < pieces; piece += P.G * kCommitWaves) {
            const uint32_t o = piece / inner, i = piece % inner;
            const uint8_t* x = source + o * s.outer_stride + i * s.inner_stride;
            uint8_t* y = P.cache + o * P.c.outer_stride + i * P.c.inner_stride;
            auto move = [&](auto zero, int64_t c) {
                using T = decltype(zero);
                for (int r = 0; r < rows; r += 8) {
                    T v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (r + j < rows) v[j] = load_at<T>(x + from[r + j] + c);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (r + j < rows) store_at<T>(y + to[r + j] + c, v[j]);
                }
            };
            for (int64_t c = lane * 16; c < whole; c += 64 * 16) move(u32x4{}, c);
            if (whole + lane < bytes) move(uint8_t{}, whole + lane);
        }
    }
}

// ------------------------------------------------------------------- host ----

// Whether a layout's numbers can be worked with: no size below 1, strides that do not go back.
bool layout_ok(const rs_rows* r) {
    return r && r->outer >= 1 && r->pages >= 1 && r->inner >= 1 && r->positions >= 1 && r->row_bytes >= 1 &&
           r->outer_stride >= 0 && r->page_stride >= 0 && r->inner_stride >= 0 && r->position_stride >= 0;
}
bool same_layout(const rs_rows& a, const rs_rows& b) {
    return a.outer == b.outer && a.pages == b.pages && a.inner == b.inner && a.positions == b.positions &&
           a.row_bytes == b.row_bytes && a.outer_stride == b.outer_stride && a.page_stride == b.page_stride &&
           a.inner_stride == b.inner_stride && a.position_stride == b.position_stride;
}
// outer * inner * n < 2^31, without passing 64 bits
bool counts_fit(const rs_rows& r, int64_t n) {
    const int64_t most = INT_MAX;
    return n <= most && r.outer <= most && r.inner <= most && r.outer * r.inner <= most && r.outer * r.inner * n <= most;
}

// Workgroups a sequence: enough for the batch to fill the chip some times over, and no more
// than there are pieces for.
int32_t groups_for(int64_t pieces, int32_t B, int waves) {
    constexpr int64_t kWorkgroups = 4096;
    const int64_t most = (pieces + waves - 1) / waves, share = (kWorkgroups + B - 1) / B;
    return (int32_t)(most < share ? most : share);
}

rs_status reorder(const void* src, const rs_rows* src_rows, const int32_t* src_table, int64_t src_table_stride,
                  void* dst, const rs_rows* dst_rows, const int32_t* dst_table, int64_t dst_table_stride,
                  int32_t max_pages, const int32_t* parent, const int32_t* lengths, int32_t B, int32_t W, int32_t K,
                  int32_t* out_status, void* stream, bool paged) {
    if (B < 0 || W <= 0 || K <= 0 || !layout_ok(src_rows) || !layout_ok(dst_rows)) return RS_ERR_INVALID_ARG;
    if (src_rows->outer != dst_rows->outer || src_rows->inner != dst_rows->inner ||
        src_rows->positions != dst_rows->positions || src_rows->row_bytes != dst_rows->row_bytes)
        return RS_ERR_INVALID_ARG;
    if (W > RS_MAX_CANDIDATES || K > RS_MAX_CANDIDATES) return RS_ERR_UNSUPPORTED;
    if (B == 0) return RS_OK;
    if (!src || !dst || !parent) return RS_ERR_INVALID_ARG;
    if (paged) {
        if (!src_table || !dst_table || !lengths || max_pages <= 0 || src_table_stride < max_pages ||
            dst_table_stride < max_pages)
            return RS_ERR_INVALID_ARG;
    } else {
        if (src_rows->pages != (int64_t)B * W || dst_rows->pages != (int64_t)B * K) return RS_ERR_INVALID_ARG;
    }
    if (src == dst && (W != K || !same_layout(*src_rows, *dst_rows))) return RS_ERR_INVALID_ARG;
    if (src_rows->positions > INT_MAX) return RS_ERR_UNSUPPORTED;
    const int64_t longest = src_rows->positions * (paged ? max_pages : 1);
    if ((paged && src_rows->positions > INT_MAX / max_pages) || !counts_fit(*src_rows, longest)) return RS_ERR_UNSUPPORTED;
    ReorderParams P{};
    P.src = static_cast<const uint8_t*>(src);
    P.dst = static_cast<uint8_t*>(dst);
    P.s = *src_rows;
    P.d = *dst_rows;
    P.parent = parent;
    P.lengths = lengths;
    P.src_table = src_table;
    P.dst_table = dst_table;
    P.src_table_stride = src_table_stride;
    P.dst_table_stride = dst_table_stride;
    P.max_pages = max_pages;
    P.W = W;
    P.K = K;
    P.status = out_status;
    // positions that lie one after another in both are one piece
    const int64_t row = src_rows->row_bytes, S = src_rows->positions;
    P.step = 1;
    if (src_rows->position_stride == row && dst_rows->position_stride == row) {
        const int64_t n = (kPieceBytes + row - 1) / row;
        P.step = (int32_t)(n < S ? n : S);
    }
    P.per_page = (int32_t)((S + P.step - 1) / P.step);
    P.G = groups_for(src_rows->outer * src_rows->inner * P.per_page * (paged ? max_pages : 1), B, kReorderWaves);
    if ((int64_t)P.G * B > INT_MAX / kReorderBlock) return RS_ERR_UNSUPPORTED;
    auto launch = [&](auto kmax, auto zero, auto pages) {
        hipLaunchKernelGGL((rs_reorder_kernel<kmax(), decltype(zero), pages()>), dim3((unsigned)P.G * B),
                           dim3(kReorderBlock), 0, (hipStream_t)stream, P);
        return hipGetLastError();
    };
    auto by_beams = [&](auto pages) {
        using std::integral_constant;
        if (K <= 4) return launch(integral_constant<int, 4>(), u32x4{}, pages);
        if (K <= 8) return launch(integral_constant<int, 8>(), u32x4{}, pages);
        if (K <= 16) return launch(integral_constant<int, 16>(), u32x4{}, pages);
        return launch(integral_constant<int, 64>(), u32x2{}, pages);
    };
    const hipError_t e = paged ? by_beams(std::true_type()) : by_beams(std::false_type());
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // namespace

extern "C" {

rs_status resispec_beam_reorder(const void* src, const rs_rows* src_rows, void* dst, const rs_rows* dst_rows,
                                const int32_t* parent, const int32_t* lengths, int32_t B, int32_t W, int32_t K,
                                int32_t* out_status, void* stream) {
    return reorder(src, src_rows, nullptr, 0, dst, dst_rows, nullptr, 0, 1, parent, lengths, B, W, K, out_status, stream,
                   false);
}

rs_status resispec_beam_reorder_paged(const void* src, const rs_rows* src_rows, const int32_t* src_table,
                                      int64_t src_table_stride, void* dst, const rs_rows* dst_rows,
                                      const int32_t* dst_table, int64_t dst_table_stride, int32_t max_pages,
                                      const int32_t* parent, const int32_t* lengths, int32_t B, int32_t W, int32_t K,
                                      int32_t* out_status, void* stream) {
    return reorder(src, src_rows, src_table, src_table_stride, dst, dst_rows, dst_table, dst_table_stride, max_pages,
                   parent, lengths, B, W, K, out_status, stream, true);
}

rs_status resispec_plan_cache(const int32_t* kept, const int32_t* added, const int32_t* held, int32_t R,
                              int32_t page_size, int32_t* block_table, int64_t table_stride, int32_t max_pages,
                              int32_t* free_pages, const int32_t* free_count, int32_t num_pages, int32_t* out_held,
                              int32_t* out_free_count, int32_t* out_starts, int32_t T, int32_t* out_slots,
                              int32_t* out_positions, int32_t* out_requests, int32_t* out_status, void* stream) {
    if (R < 0 || T < 0 || page_size <= 0 || num_pages <= 0 || max_pages <= 0 || table_stride < max_pages)
        return RS_ERR_INVALID_ARG;
    if (!free_pages || !free_count || !out_free_count || !out_starts || (T > 0 && !out_slots)) return RS_ERR_INVALID_ARG;
    if (R > 0 && (!kept || !added || !held || !block_table || !out_held)) return RS_ERR_INVALID_ARG;
    if ((int64_t)num_pages * page_size > INT_MAX || (int64_t)max_pages * page_size > INT_MAX) return RS_ERR_UNSUPPORTED;
    PlanParams P{kept, added, held, R, page_size, block_table, table_stride, max_pages, free_pages, free_count, num_pages,
                 out_held, out_free_count, out_starts, T, out_slots, out_positions, out_requests, out_status};
    constexpr int32_t kRowsAlone = 2048;
    if (T <= kRowsAlone) {
        hipLaunchKernelGGL(rs_plan_kernel<true>, dim3(1), dim3(kPlanBlock), 0, (hipStream_t)stream, P);
        return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
    }
    hipLaunchKernelGGL(rs_plan_kernel<false>, dim3(1), dim3(kPlanBlock), 0, (hipStream_t)stream, P);
    if (hipGetLastError() != hipSuccess) return RS_ERR_HIP;
    hipLaunchKernelGGL(rs_plan_rows_kernel, dim3((unsigned)(((int64_t)T + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       P);
    return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_accepted_path(const int32_t* parent, const int32_t* node_token, const int32_t* tokens,
                                 const int32_t* accepted_len, int32_t B, int32_t N, int32_t max_depth,
                                 int32_t* out_path, int32_t* out_status, void* stream) {
    if (B < 0 || N <= 0 || max_depth < 0 || max_depth == INT_MAX) return RS_ERR_INVALID_ARG;
    if (N > RS_MAX_PATH_NODES) return RS_ERR_UNSUPPORTED;
    if (B == 0) return RS_OK;
    if (!parent || !node_token || !tokens || !accepted_len || !out_path) return RS_ERR_INVALID_ARG;
    const int block = N <= 64 ? 64 : N <= 1024 ? 256 : 1024;
    hipLaunchKernelGGL(rs_path_nodes_kernel, dim3((unsigned)B), dim3(block), (size_t)N * 4, (hipStream_t)stream, parent,
                       node_token, tokens, accepted_len, N, max_depth, out_path, out_status);
    return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_commit_path(void* cache, const rs_rows* cache_rows, const int32_t* slots, const int32_t* path,
                               const void* source, const rs_rows* source_rows, int32_t B, int32_t N, int32_t depth,
                               int32_t* out_status, void* stream) {
    if (B < 0 || N <= 0 || depth <= 0 || !layout_ok(cache_rows)) return RS_ERR_INVALID_ARG;
    if (source) {
        if (!layout_ok(source_rows) || source_rows->outer != cache_rows->outer || source_rows->inner != cache_rows->inner ||
            source_rows->row_bytes != cache_rows->row_bytes || source_rows->pages != B || source_rows->positions != N)
            return RS_ERR_INVALID_ARG;
    }
    if (N > RS_MAX_PATH_NODES || depth > RS_MAX_PATH_NODES) return RS_ERR_UNSUPPORTED;
    if (cache_rows->pages > INT_MAX || cache_rows->positions > INT_MAX ||
        cache_rows->pages * cache_rows->positions > INT_MAX || !counts_fit(*cache_rows, 1))
        return RS_ERR_UNSUPPORTED;
    if (B == 0) return RS_OK;
    if (!cache || !slots || !path) return RS_ERR_INVALID_ARG;
    CommitParams P{};
    P.cache = static_cast<uint8_t*>(cache);
    P.c = *cache_rows;
    P.slots = slots;
    P.path = path;
    P.source = static_cast<const uint8_t*>(source);
    if (source) P.s = *source_rows;
    P.N = N;
    P.depth = depth;
    P.status = out_status;
    P.G = groups_for(cache_rows->outer * cache_rows->inner, B, kCommitWaves);
    if ((int64_t)P.G * B > INT_MAX / kCommitBlock) return RS_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(rs_commit_kernel, dim3((unsigned)P.G * B), dim3(kCommitBlock), 0, (hipStream_t)stream, P);
    return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
