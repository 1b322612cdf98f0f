// cache.hip -- rows of per-beam states and of a paged cache around a decoding step, on
// gfx950: states of the chosen beams (resispec_beam_reorder, resispec_beam_reorder_paged),
// pages and slots of new rows (resispec_plan_cache), accepted paths of verified trees
// (resispec_accepted_path) and their rows' places in the cache (resispec_commit_path).
// Declared in resispec.h.

#include "common.h"
#include "share.h"

#include <algorithm>
#include <climits>

namespace {

// Vectors of 16 bytes at any address: rows need not be a multiple of 16 bytes long, nor start
// on one, and gfx950 loads and stores such vectors in one instruction.
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
// In registers: a byte has one of its own (four to a register wait for one another).
template <typename T>
using Held = std::conditional_t<sizeof(T) == 1, uint32_t, T>;
// By the address, in global memory: an address that has been through lanes is one of any memory
// to the compiler.
template <typename T>
__device__ __forceinline__ T load_at(int64_t at, uint32_t c) {
    using G = const __attribute__((address_space(1))) uint8_t;
    return *(const __attribute__((address_space(1))) typename Any<T>::type*)((G*)at + c);
}
// Rows are stored past the caches, which they would only fill: 40 states of 492 KB 39 us with
// ordinary stores and 25 with these, 1024 paths in rows of 1000 bytes 36 and 27.  Loads stay
// ordinary: beams of one parent, and the ends of rows, share lines.
template <typename T>
__device__ __forceinline__ void store_at(int64_t at, uint32_t c, T v) {
    using G = __attribute__((address_space(1))) uint8_t;
    auto* p = (__attribute__((address_space(1))) typename Any<T>::type*)((G*)at + c);
    if constexpr (sizeof(T) == 1) *p = v;
    else __builtin_nontemporal_store(v, p);
}

// Waits for the wave's loads, here and once.  Loads that may or may not have been made leave the
// compiler to wait before every store for all that came before it, the stores among them: 32
// beams of 3 KB 13.7 us, with this wait and bytes in registers of their own 7.1,
// 64 of 200 KB in 24 layers 166 and 97.  (vmcnt 0, the other counters as they are.)
__device__ __forceinline__ void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

__device__ __forceinline__ int uniform_i(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t readlane_i64(int64_t v, int l) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, l);
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | lo);
}

// ---------------------------------------------------------------- reorder ----

// States move for all beams of a sequence at once.  A lane owns columns, 16 bytes at one place
// of every beam's state: it loads the new value of each beam and then stores them, so a move in
// place needs no second buffer and no wait between workgroups.  A wave takes a piece, bytes that
// lie one after another.
// Arguments are kept short: a launch with 160 bytes of them takes the host 3.5 us, with 16 2.9.
struct Strides {
    int64_t outer, page, inner, position;
};
Strides strides_of(const rs_rows& r) { return {r.outer_stride, r.page_stride, r.inner_stride, r.position_stride}; }

struct ReorderParams {
    const uint8_t* src;
    uint8_t* dst;
    Strides s, d;
    const int32_t* parent;           // [B][K]
    const int32_t* lengths;          // [B] or NULL
    const int32_t *src_table, *dst_table;
    int64_t src_table_stride, dst_table_stride;
    int64_t row;                     // bytes
    uint32_t outer, inner, S;        // positions of a state, or of a page
    uint32_t src_pages, dst_pages;
    int32_t max_pages;               // entries of a table's row
    int32_t W, K, G;                 // workgroups a sequence
    int32_t together;                // positions lie one after another
    int32_t pieces;                  // a page has so many (together), or a row
    int32_t* status;
};

constexpr int kReorderBlock = 256, kReorderWaves = kReorderBlock / 64;

// A piece is a column a lane.  (With two or four 1 x 4 states of 32 KB 5.8 us instead of 3.8, 32 x
// 4 of 2 MB 114 and 88, the largest alike.)  40 states of 492 KB: 24 us, 6.0 TB/s; 256 of 2.1 MB in
// pages of 16 rows: 184 us, 4.7 TB/s, a copy's rate: HBM bounds it.
template <int KMAX, typename T, bool PAGED>
__global__ void __launch_bounds__(kReorderBlock) rs_reorder_kernel(const ReorderParams P) {
    constexpr int64_t kPiece = 64 * sizeof(T);
    const int b = blockIdx.x / P.G, g = blockIdx.x % P.G;
    const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
    const int32_t* parent = P.parent + (int64_t)b * P.K;
    const int S = (int)P.S;
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
            const uint32_t used = (uint32_t)((len + S - 1) / S);
            bool out = false;
            each_entry(used, (uint32_t)P.K, threadIdx.x, kReorderBlock, [&](uint32_t k, uint32_t e) {
                const int w = parent[k];
                if (w < 0) return;
                out |= (uint32_t)from_table[w * P.src_table_stride + e] >= P.src_pages;
                out |= (uint32_t)to_table[k * P.dst_table_stride + e] >= P.dst_pages;
            });
            if (__syncthreads_or(out)) st = RS_SEQ_BAD_PAGE;
        }
        if (threadIdx.x == 0) P.status[b] = st;
    }
    if (bad || len == 0) return;
    const uint32_t full = (uint32_t)(len / S), rest = (uint32_t)(len % S), each = (uint32_t)P.pieces;
    const int64_t row = P.row;
    const uint32_t nq = P.together ? full * each + (uint32_t)((rest * row + kPiece - 1) / kPiece) : (uint32_t)len * each;
    const uint32_t inner = P.inner, all = P.outer * inner * nq;
    for (uint32_t piece = g * kReorderWaves + wave; piece < all; piece += P.G * kReorderWaves) {
        // quotients are computed in vector registers
        const uint32_t oi = uniform_i(piece / nq), q = piece - oi * nq, o = uniform_i(oi / inner), i = oi - o * inner;
        uint32_t page = uniform_i(q / each), t = 0;
        const int64_t first = (q - page * each) * kPiece;
        int64_t bytes = row - first;
        if (P.together) {
            bytes = (page < full ? S : rest) * row - first;
        } else {
            const uint32_t p = uniform_i(page / (uint32_t)S);
            t = page - p * (uint32_t)S;
            page = p;
        }
        bytes = min(bytes, kPiece);
        // lane k has beam k's addresses
        int64_t from = o * P.s.outer + i * P.s.inner + t * P.s.position + first;
        int64_t to = o * P.d.outer + i * P.d.inner + t * P.d.position + first;
        bool moves = mine >= 0;
        if (moves) {
            int64_t f = (int64_t)b * P.W + mine, d = (int64_t)b * P.K + lane;
            if (PAGED) {
                f = from_table[mine * P.src_table_stride + page];
                d = to_table[lane * P.dst_table_stride + page];
                moves = (uint32_t)f < P.src_pages && (uint32_t)d < P.dst_pages;
            }
            from += reinterpret_cast<int64_t>(P.src) + f * P.s.page;
            to += reinterpret_cast<int64_t>(P.dst) + d * P.d.page;
        }
        const uint64_t on = __ballot(moves && from != to);      // equal: where it is
        auto move = [&](auto zero, uint32_t c) {
            using E = decltype(zero);
            Held<E> v[KMAX];
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (on >> k & 1) v[k] = load_at<E>(readlane_i64(from, k), c);
            wait_for_loads();
#pragma unroll
            for (int k = 0; k < KMAX; ++k)
                if (on >> k & 1) store_at<E>(readlane_i64(to, k), c, (E)v[k]);
        };
        // columns, and bytes at a run's end
        const uint32_t whole = (uint32_t)bytes / sizeof(T) * sizeof(T), c = lane * sizeof(T);
        if (c < whole) move(T{}, c);
        if (whole + lane < bytes) move(uint8_t{}, whole + lane);
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
    int32_t later;                   // out_held and out_free_count are left to rs_plan_tell_kernel
};

// The sum over a workgroup's threads up to each, in order, and the whole sum.  Whole numbers in
// fp64, exact to 2^53.  Two calls in a row need different halves of `part`.
template <int BLOCK>
__device__ __forceinline__ int64_t block_scan(int64_t v, double (&part)[BLOCK / 64], int64_t& total) {
    const int lane = threadIdx.x & 63;
    const double x = wave_incl_scan((double)v, lane);
    if constexpr (BLOCK == 64) {
        total = (int64_t)readlane_d(x, 63);
        return (int64_t)x;
    } else {
        const int wave = uniform_i(threadIdx.x >> 6);
        if (lane == 63) part[wave] = x;
        __syncthreads();
        double before = 0.0, all = 0.0;
#pragma unroll 4
        for (int w = 0; w < BLOCK / 64; ++w) {
            before += w < wave ? part[w] : 0.0;
            all += part[w];
        }
        total = (int64_t)all;
        return (int64_t)(x + before);
    }
}

// The first of n running sums above x (there is one).
template <typename Sums>
__device__ __forceinline__ int first_above(const Sums& upto, int n, int x) {
    int lo = 0;
    for (int step = 1 << (31 - __builtin_clz(n)); step; step >>= 1)
        if (lo + step <= n && upto[lo + step - 1] <= x) lo += step;
    return lo;
}

struct NewRow {
    int slot, position, request;
};
__device__ __forceinline__ void put_row(const PlanParams& P, int t, const NewRow& x) {
    P.slots[t] = x.slot;
    if (P.positions) P.positions[t] = x.position;
    if (P.requests) P.requests[t] = x.request;
}
// The place in a page of position p: entry p / page_size of the request's row, and the rest.
__device__ __forceinline__ int slot_in(const PlanParams& P, int page, uint32_t rest) {
    return (uint32_t)page < (uint32_t)P.num_pages ? (int)((uint32_t)page * (uint32_t)P.page_size + rest) : -1;
}

// A request's numbers, and its places in the running sums over those before it.
struct Request {
    int32_t kept, added, held, want, give, need, status;
    int64_t first;                       // rows before it
    int64_t gives, needs;                // pages given back, and taken, up to it
};

// The rules, for the BLOCK requests of a tile.
template <int BLOCK>
struct Plan {
    const PlanParams& P;
    double (&part)[3][BLOCK / 64];
    const int count;                     // free pages
    int64_t rows = 0, given = 0, needed = 0;   // before this tile

    __device__ __forceinline__ void look(int r, Request& q) {
        q = {0, 0, 0, 0, 0, 0, RS_SEQ_OK, 0, 0, 0};
        const bool count_ok = count >= 0 && count <= P.num_pages;
        if (r < P.R) {
            q.kept = P.kept[r];
            q.added = P.added[r];
            q.held = P.held[r];
            const int64_t n = (int64_t)q.kept + q.added;
            if (q.kept < 0 || q.added < 0 || q.held < 0 || q.held > P.max_pages || n > (int64_t)P.max_pages * P.page_size) {
                q.status = RS_SEQ_BAD_PARAM;
                q.added = 0;
            } else {
                q.want = (int32_t)(((uint32_t)n + (uint32_t)P.page_size - 1) / (uint32_t)P.page_size);
            }
        }
        int64_t total;
        const int64_t upto = rows + block_scan<BLOCK>(q.added, part[0], total);
        rows += total;
        q.first = upto - q.added;
        if (q.status == RS_SEQ_OK && q.added > 0 && upto > P.T) q.status = RS_SEQ_NO_ROOM;
        if (q.status == RS_SEQ_OK) {
            q.give = max(q.held - q.want, 0);
            q.need = max(q.want - q.held, 0);
            if (!count_ok && (q.give || q.need)) q.status = RS_SEQ_BAD_PARAM;
        }
        if (q.status != RS_SEQ_OK) q.give = q.need = 0;
        // requests that are refused here are the last that would give: what is given has no gaps
        q.gives = given + block_scan<BLOCK>(q.give, part[1], total);
        given += total;
        if (q.give && count + q.gives > P.num_pages) {
            q.status = RS_SEQ_BAD_PARAM;
            q.give = 0;
        }
    }
    // what is there to be taken, once all of that has been given back; likewise without gaps
    __device__ __forceinline__ void take(Request& q, int avail) {
        int64_t total;
        q.needs = needed + block_scan<BLOCK>(q.need, part[2], total);
        needed += total;
        if (q.need && q.needs > avail) {
            q.status = RS_SEQ_NO_ROOM;
            q.need = 0;
        }
    }
    static __device__ __forceinline__ int holds(const Request& q) { return q.status == RS_SEQ_OK ? q.want : q.held; }
};

// A step of up to BLOCK requests in one launch.  Every workgroup works out the running sums for
// itself, and then everything from the inputs alone: pages that are given back and taken again
// are found where their giver has them.  So no workgroup waits for another: some do the rows,
// some the pages that are taken, or given back, some the requests' numbers, and a thread looks
// up whose the next one is.  With several workgroups the outputs must not be inputs.
constexpr int kTakers = 8, kGivers = 4, kTellers = 4;
template <int BLOCK>
__global__ void __launch_bounds__(BLOCK) rs_plan_step_kernel(const PlanParams P) {
    __shared__ double part[3][BLOCK / 64];
    __shared__ int32_t end[BLOCK], first[BLOCK], kept[BLOCK];        // rows
    __shared__ int32_t gives[BLOCK], give_at[BLOCK];                 // pages given back up to it, where they are
    __shared__ int32_t needs[BLOCK], held[BLOCK], want[BLOCK];
    __shared__ int32_t touched[BLOCK], touch_at[BLOCK], wrong[BLOCK];
    __shared__ int32_t released, taken;
    const int tid = threadIdx.x;
    const int count = P.free_count[0];
    if (tid == 0) released = taken = 0;
    __syncthreads();
    Plan<BLOCK> plan{P, part, count};
    Request q;
    plan.look(tid, q);
    if (q.give) atomicAdd(&released, q.give);
    __syncthreads();
    const int avail = count + released;
    plan.take(q, avail);
    if (q.need) atomicAdd(&taken, q.need);
    const bool granted = q.status == RS_SEQ_OK;
    const int64_t rows = plan.rows;
    end[tid] = (int32_t)min(q.first + q.added, (int64_t)INT_MAX);
    first[tid] = granted ? (int32_t)q.first : -1;
    kept[tid] = q.kept;
    gives[tid] = (int32_t)min(q.gives, (int64_t)INT_MAX);
    give_at[tid] = q.want - (int32_t)(q.gives - q.give);
    needs[tid] = (int32_t)min(q.needs, (int64_t)INT_MAX);
    held[tid] = q.held;
    want[tid] = q.want;
    __syncthreads();
    const int F = released, A = taken;
    // page number x of those given back, and of those taken
    auto given_page = [&](int x) {
        const int r = first_above(gives, BLOCK, x);
        return P.table[r * P.table_stride + give_at[r] + x];
    };
    auto taken_page = [&](int x) {
        const int at = avail - 1 - x;
        return at < count ? P.free_pages[at] : given_page(at - count);
    };
    auto page_of = [&](int r, int e) {
        return e < held[r] ? P.table[r * P.table_stride + e] : taken_page(needs[r] - want[r] + e);
    };
    // the jobs' first workgroups and how many they have
    const bool alone = gridDim.x == 1;
    const int nrows = alone ? 1 : (int)gridDim.x - kTakers - kGivers - kTellers;
    auto job = [&](int from, int groups, int n, auto&& body) {
        if (alone) from = 0, groups = 1;
        const int g = (int)blockIdx.x - from;
        if (g < 0 || g >= groups) return;
        for (uint32_t x = g * BLOCK + tid; x < (uint32_t)n; x += groups * BLOCK) body((int)x);
    };
    job(nrows + kTakers, kGivers, F, [&](int x) { P.free_pages[count + x] = given_page(x); });
    job(nrows, kTakers, A, [&](int x) {
        const int r = first_above(needs, BLOCK, x);
        P.table[r * P.table_stride + x - needs[r] + want[r]] = taken_page(x);
    });
    job(0, nrows, P.T, [&](int t) {
        NewRow x = {-1, -1, -1};
        if (t < rows) {
            const int r = first_above(end, BLOCK, t);
            if (first[r] >= 0) {
                const uint32_t p = (uint32_t)kept[r] + (uint32_t)(t - first[r]), e = p / (uint32_t)P.page_size;
                x = {slot_in(P, page_of(r, (int)e), p - e * (uint32_t)P.page_size), (int)p, r};
            }
        }
        put_row(P, t, x);
    });
    const int teller = alone ? 0 : (int)blockIdx.x - nrows - kTakers - kGivers, tellers = alone ? 1 : kTellers;
    if (teller < 0) return;
    // every page that the new rows of this workgroup's requests lie in is looked at
    const int own = BLOCK / tellers, r0 = teller * own;
    const bool mine = tid >= r0 && tid < r0 + own && tid < P.R;
    if (P.status) {
        // from the page with position `kept` on
        const int from = granted && q.added ? (int)((uint32_t)q.kept / (uint32_t)P.page_size) : q.want;
        const int n = mine && granted ? q.want - from : 0;
        int64_t all;
        __syncthreads();
        const int64_t upto = block_scan<BLOCK>(n, part[0], all);
        touched[tid] = (int32_t)upto;
        touch_at[tid] = from - (int32_t)(upto - n);
        wrong[tid] = 0;
        __syncthreads();
        each_of(all, tid, BLOCK, [&](int64_t x) {
            const int r = first_above(touched, BLOCK, (int)x);
            if ((uint32_t)page_of(r, touch_at[r] + (int)x) >= (uint32_t)P.num_pages) wrong[r] = 1;
        });
        __syncthreads();
        if (mine) P.status[tid] = granted && wrong[tid] ? RS_SEQ_BAD_PAGE : q.status;
    }
    if (mine) P.out_starts[tid] = (int32_t)min(q.first, (int64_t)INT_MAX);
    if (mine && !P.later) P.out_held[tid] = plan.holds(q);
    if (teller == 0 && tid == 0) {
        P.out_starts[P.R] = (int32_t)min(rows, (int64_t)INT_MAX);
        if (!P.later) P.out_free_count[0] = avail - A;
    }
}

// What the requests hold then, and how many pages are free, where these are inputs of the step:
// they may change only when every workgroup has read them.
template <int BLOCK>
__global__ void __launch_bounds__(BLOCK) rs_plan_tell_kernel(const PlanParams P) {
    __shared__ double part[3][BLOCK / 64];
    __shared__ int32_t released, taken;
    const int tid = threadIdx.x, count = P.free_count[0];
    if (tid == 0) released = taken = 0;
    __syncthreads();
    Plan<BLOCK> plan{P, part, count};
    Request q;
    plan.look(tid, q);
    if (q.give) atomicAdd(&released, q.give);
    __syncthreads();
    const int avail = count + released;
    plan.take(q, avail);
    if (q.need) atomicAdd(&taken, q.need);
    __syncthreads();
    if (tid < P.R) P.out_held[tid] = plan.holds(q);
    if (tid == 0) P.out_free_count[0] = avail - taken;
}

// More than 1024 requests: one workgroup, 1024 at a time, in two passes (the first gives pages
// back, the second takes them), and the new rows in a launch of their own.  3000 requests of 33
// rows: 35 and 7 us.
constexpr int kPlanBlock = 1024;
__global__ void __launch_bounds__(kPlanBlock) rs_plan_kernel(const PlanParams P) {
    __shared__ double part[3][kPlanBlock / 64];
    __shared__ int32_t upto_s[kPlanBlock], at_s[kPlanBlock];
    __shared__ int32_t released, taken, in_tile;
    const int tid = threadIdx.x;
    const int count = P.free_count[0];
    if (tid == 0) released = taken = in_tile = 0;
    __syncthreads();
    // body(r, entry, i) for pages i = 0 .. of the tile's requests, `mine` from entry `at` of
    // request r's row on; upto: mine and those before
    auto pages = [&](int tile, int mine, int upto, int at, auto&& body) {
        if (!__syncthreads_or(mine)) return;
        upto_s[tid] = upto;
        at_s[tid] = at - (upto - mine);
        if (mine) atomicMax(&in_tile, upto);
        __syncthreads();
        const int all = in_tile;
        each_of(all, tid, kPlanBlock, [&](int64_t i) {
            const int x = first_above(upto_s, kPlanBlock, (int)i);
            body(tile * kPlanBlock + x, at_s[x] + (int)i, (int)i);
        });
        __syncthreads();
        if (tid == 0) in_tile = 0;
        __syncthreads();
    };
    Plan<kPlanBlock> plan{P, part, count};
    Request q;
    const int tiles = blocks_of(P.R, kPlanBlock);
    for (int i = 0; i < tiles; ++i) {
        const int64_t base = plan.given;
        plan.look(i * kPlanBlock + tid, q);
        if (q.give) atomicAdd(&released, q.give);
        pages(i, q.give, (int)min(q.gives - base, (int64_t)INT_MAX), q.want, [&](int r, int e, int x) {
            P.free_pages[count + base + x] = P.table[r * P.table_stride + e];
        });
    }
    __syncthreads();
    const int avail = count + released;
    const int64_t rows = plan.rows;
    plan.rows = plan.given = 0;
    for (int i = 0; i < tiles; ++i) {
        const int r = i * kPlanBlock + tid;
        const int64_t base = plan.needed;
        plan.look(r, q);
        plan.take(q, avail);
        if (q.need) atomicAdd(&taken, q.need);
        pages(i, q.need, (int)min(q.needs - base, (int64_t)INT_MAX), q.held, [&](int r, int e, int x) {
            P.table[r * P.table_stride + e] = P.free_pages[avail - 1 - (base + x)];
        });
        if (r < P.R) {
            P.out_held[r] = plan.holds(q);
            P.out_starts[r] = (int32_t)min(q.first, (int64_t)INT_MAX);
            if (P.status) P.status[r] = q.status;
        }
        __syncthreads();
    }
    __syncthreads();
    if (tid == 0) {
        P.out_starts[P.R] = (int32_t)min(rows, (int64_t)INT_MAX);
        P.out_free_count[0] = avail - taken;
    }
}

// A row a thread, with the running sums of up to kStarts requests in LDS.
constexpr int kStarts = 4096;
__global__ void __launch_bounds__(256) rs_plan_rows_kernel(const PlanParams P) {
    __shared__ int32_t ends[kStarts];
    const bool held = P.R <= kStarts;
    if (held) {
        for (int r = threadIdx.x; r < P.R; r += 256) ends[r] = P.out_starts[r + 1];
        __syncthreads();
    }
    const int64_t t64 = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t64 >= P.T) return;
    const int t = (int)t64;
    NewRow x = {-1, -1, -1};
    if (t < P.out_starts[P.R]) {
        const int r = held ? first_above(ends, P.R, t) : first_above(P.out_starts + 1, P.R, t);
        const int k = P.kept[r], n = P.added[r], first = P.out_starts[r];
        const int want = (int)(((uint32_t)k + (uint32_t)n + (uint32_t)P.page_size - 1) / (uint32_t)P.page_size);
        // granted: it holds what it wants, and its rows fit
        if (P.out_held[r] == want && (int64_t)first + n <= P.T) {
            const uint32_t p = (uint32_t)k + (uint32_t)(t - first), e = p / (uint32_t)P.page_size;
            x = {slot_in(P, P.table[r * P.table_stride + e], p - e * (uint32_t)P.page_size), (int)p, r};
            if (x.slot < 0 && P.status) P.status[r] = RS_SEQ_BAD_PAGE;
        }
    }
    put_row(P, t, x);
}

// ------------------------------------------------------------------- path ----

// Trees of up to 64 nodes, a wave a sequence: lane n has node n, and the nodes of a level that
// carry the tokens are bits of a mask.  All loads are on their way at once, so a call is a launch
// and one latency: 1 tree of 26 nodes 1.8 us, 1024 of 60 nodes 4.7 (6.2 by the kernel below).
constexpr int kPathWaves = 4;
__global__ void __launch_bounds__(kPathWaves * 64) rs_path_wave_kernel(
    const int32_t* __restrict__ parent, const int32_t* __restrict__ node_token, const int32_t* __restrict__ tokens,
    const int32_t* __restrict__ accepted_len, int32_t B, int32_t N, int32_t max_depth, int32_t* __restrict__ path,
    int32_t* status) {
    const int lane = threadIdx.x & 63;
    const int64_t b = (int64_t)blockIdx.x * kPathWaves + uniform_i(threadIdx.x >> 6), width = max_depth + 1;
    if (b >= B) return;
    const int len = accepted_len[b];
    const int up = lane < N ? parent[b * N + lane] : 0, token = lane < N ? node_token[b * N + lane] : 0;
    const int wanted = lane < max_depth ? tokens[b * width + lane] : 0;      // there are at most 63 levels
    int st = len < -1 || len > max_depth ? RS_SEQ_DEPTH_EXCEEDED : RS_SEQ_OK;
    const bool bad = lane < N && (lane == 0 ? up != -1 : up < 0 || up >= lane);
    if (__ballot(bad) && st == RS_SEQ_OK) st = RS_SEQ_BAD_TREE;
    uint64_t level = st == RS_SEQ_OK && len >= 0 && len < N ? 1 : 0;
    for (int d = 0; d < len && level; ++d)
        level = __ballot(lane > 0 && lane < N && (level >> (up & 63) & 1) && token == __builtin_amdgcn_readlane(wanted, d));
    if (st == RS_SEQ_OK && len >= 0 && !level) st = RS_SEQ_BAD_TREE;
    const int on = level ? len + 1 : 0;
    int mine = -1, n = level ? __builtin_ctzll(level) : 0;
    for (int i = on - 1; i >= 0; --i) {
        if (lane == i) mine = n;
        n = __builtin_amdgcn_readlane(up, n & 63);
    }
    for (int64_t i = lane; i < width; i += 64) path[b * width + i] = i < 64 ? mine : -1;
    if (lane == 0 && status) status[b] = st;
}

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
    each_of(width, on + tid, blockDim.x, [&](int64_t i) { path[i] = -1; });
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
    const uint8_t* source;               // the cache, or rows elsewhere
    Strides c, s;
    const int32_t *slots, *path;
    int32_t* status;
    uint32_t outer, inner, bytes;        // of a row
    uint32_t page, room;                 // slots of a page, and of the cache
    int32_t N, depth, G;                 // workgroups a sequence
    bool within;                         // the source is the cache
};

constexpr int kCommitBlock = 256, kCommitWaves = kCommitBlock / 64;

// A lane owns a column of 16 bytes (or one) of all rows of a path, as in the reorder.  Paths
// ascend, so path[j] >= j: the slot that row i goes to, slots[i], is the source of none after
// it, and the rows are moved in order, eight loaded before they are stored.  Lane i has row i's
// places, 64 at a time; no wave waits for another.  1024 paths of four rows of 16 x 1000 bytes:
// 26 us, 131 MB, 5.0 TB/s, a copy's rate: HBM bounds it.
__global__ void __launch_bounds__(kCommitBlock) rs_commit_kernel(const CommitParams P) {
    const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
    const int b = blockIdx.x / P.G, g = blockIdx.x % P.G;
    const int32_t* path = P.path + (int64_t)b * P.depth;
    const int32_t* slots = P.slots + (int64_t)b * P.N;
    const uint32_t room = P.room, page = P.page;
    // the rows of entries first .. first + 63: how many, and whether they can be moved
    int64_t from = 0, to = 0;
    int before = -1;                     // the entry before these
    int start = 0;                       // the first row that moves
    bool wrong = false, outside = false;
    auto look = [&](int first) {
        const int i = first + lane;
        const int x = i < P.depth ? path[i] : -1;
        const uint32_t slot = i < P.N ? (uint32_t)slots[i] : 0xffffffffu;
        const uint64_t ends = __ballot(x == -1);
        const int n = ends ? __builtin_ctzll(ends) : 64;
        const int last = __shfl_up(x, 1);
        const bool on = lane < n;
        const bool order = on && (x < i || x >= P.N || x <= (lane == 0 ? before : last));
        bool out = on && !order && slot >= room;
        from = to = 0;
        if (on && !order && !out) {
            to = slot / page * P.c.page + slot % page * P.c.position;
            if (!P.within) {
                from = b * P.s.page + x * P.s.position;
            } else {
                const uint32_t was = (uint32_t)slots[x];
                out = was >= room;
                from = was / page * P.c.page + was % page * P.c.position;
            }
        }
        wrong |= __ballot(order) != 0;
        outside |= __ballot(out) != 0;
        before = n == 64 ? __builtin_amdgcn_readlane(x, 63) : before;
        // rows that are where they belong are the path's first
        start = !P.within ? 0 : __popcll(__ballot(on && x == i));
        return n;
    };
    int n = look(0);
    if (n == 64 && P.depth > 64) {       // the whole path is looked at before anything is moved
        for (int first = 64, m = n; first < P.depth && m == 64; first += 64) m = look(first);
        before = -1;
        n = look(0);
    }
    if (g == 0 && threadIdx.x == 0 && P.status)
        P.status[b] = wrong ? RS_SEQ_BAD_TREE : outside ? RS_SEQ_BAD_PAGE : RS_SEQ_OK;
    if (wrong || outside) return;
    const uint32_t inner = P.inner, pieces = P.outer * inner;
    const uint32_t bytes = P.bytes, whole = bytes & ~15u;
    auto move_all = [&]() {
        for (uint32_t piece = g * kCommitWaves + wave; piece < pieces; piece += P.G * kCommitWaves) {
            const uint32_t o = uniform_i(piece / inner), i = piece - o * inner;
            const int64_t x = reinterpret_cast<int64_t>(P.source) + o * P.s.outer + i * P.s.inner;
            const int64_t y = reinterpret_cast<int64_t>(P.cache) + o * P.c.outer + i * P.c.inner;
            auto move = [&](auto zero, uint32_t c) {
                using T = decltype(zero);
                for (int r = start; r < n; r += 8) {
                    Held<T> v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (r + j < n) v[j] = load_at<T>(x + readlane_i64(from, r + j), c);
                    wait_for_loads();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (r + j < n) store_at<T>(y + readlane_i64(to, r + j), c, (T)v[j]);
                }
            };
            // what is left of a row: its last 16 bytes once more where they come from elsewhere
            const uint32_t tail = bytes - whole;
            const bool again = !P.within && tail && whole;
            for (uint32_t c = lane * 16; c < whole + (again ? 16 : 0); c += 64 * 16)
                move(u32x4{}, c < whole ? c : bytes - 16);
            if (!again && lane < tail) move(uint8_t{}, whole + lane);
        }
    };
    move_all();
    for (int first = 64; n == 64 && first < P.depth; first += 64) {
        n = look(first);
        move_all();
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
    constexpr int64_t kWorkgroups = 8192;
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
    // in place the beams are the same ones; with tables each side names its own rows
    if (src == dst && ((!paged && W != K) || !same_layout(*src_rows, *dst_rows))) return RS_ERR_INVALID_ARG;
    if (src_rows->positions > INT_MAX || src_rows->row_bytes > LLONG_MAX / src_rows->positions) return RS_ERR_UNSUPPORTED;
    const int64_t longest = src_rows->positions * (paged ? max_pages : 1);
    if ((paged && src_rows->positions > INT_MAX / max_pages) || !counts_fit(*src_rows, longest)) return RS_ERR_UNSUPPORTED;
    ReorderParams P{};
    P.src = static_cast<const uint8_t*>(src);
    P.dst = static_cast<uint8_t*>(dst);
    P.s = strides_of(*src_rows);
    P.d = strides_of(*dst_rows);
    P.row = src_rows->row_bytes;
    P.outer = (uint32_t)src_rows->outer;
    P.inner = (uint32_t)src_rows->inner;
    P.S = (uint32_t)src_rows->positions;
    // a table's numbers do not reach further
    P.src_pages = (uint32_t)std::min(src_rows->pages, (int64_t)INT_MAX);
    P.dst_pages = (uint32_t)std::min(dst_rows->pages, (int64_t)INT_MAX);
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
    // positions that lie one after another in both are one run
    const int64_t row = src_rows->row_bytes, S = src_rows->positions;
    P.together = src_rows->position_stride == row && dst_rows->position_stride == row;
    auto launch = [&](auto kmax, auto zero, auto pages) -> rs_status {
        constexpr int64_t piece = 64 * sizeof(zero);
        const int64_t run = P.together ? S * row : row, runs = (P.together ? 1 : S) * (paged ? max_pages : 1);
        const int64_t each = (run + piece - 1) / piece;
        if (each > INT_MAX || runs > INT_MAX || !counts_fit(*src_rows, each * runs)) return RS_ERR_UNSUPPORTED;
        P.pieces = (int32_t)each;
        P.G = groups_for(src_rows->outer * src_rows->inner * each * runs, B, kReorderWaves);
        if ((int64_t)P.G * B > INT_MAX / kReorderBlock) return RS_ERR_UNSUPPORTED;
        hipLaunchKernelGGL((rs_reorder_kernel<kmax(), decltype(zero), pages()>), dim3((unsigned)P.G * B),
                           dim3(kReorderBlock), 0, (hipStream_t)stream, P);
        return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
    };
    auto by_beams = [&](auto pages) {
        // columns of 8 bytes where the new values of so many beams would not fit the registers
        using std::integral_constant;
        if (K <= 4) return launch(integral_constant<int, 4>(), u32x4{}, pages);
        if (K <= 8) return launch(integral_constant<int, 8>(), u32x4{}, pages);
        if (K <= 16) return launch(integral_constant<int, 16>(), u32x4{}, pages);
        if (K <= 32) return launch(integral_constant<int, 32>(), u32x2{}, pages);
        return launch(integral_constant<int, 64>(), u32x2{}, pages);
    };
    return paged ? by_beams(std::true_type()) : by_beams(std::false_type());
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
                 out_held, out_free_count, out_starts, T, out_slots, out_positions, out_requests, out_status, 0};
    // One workgroup for the smallest steps (1 request of 26 rows 3.6 us), and for small ones whose
    // outputs are inputs, which need a second launch otherwise.  Jobs side by side are quicker
    // elsewhere: 64 requests of 4 rows 7.7 us in one, 200 of 2 rows 10.2 and 5.9, 16 of 33 rows
    // 7.3 and 5.5, 256 of 33 rows 6.4, 1024 of 2 rows 16.7 and 9.6, 1024 with prompts and 93,000
    // rows 11.4, of which each is a chain of latencies: numbers, sums, a search, a page, a row.
    const bool in_place = out_held == held || out_free_count == free_count;
    auto step = [&](auto block, unsigned groups) {
        P.later = groups > 1 && in_place;
        hipLaunchKernelGGL(rs_plan_step_kernel<block()>, dim3(groups), dim3(block()), 0, (hipStream_t)stream, P);
        if (hipGetLastError() != hipSuccess) return RS_ERR_HIP;
        if constexpr (block() > 64) {
            if (!P.later) return RS_OK;
            hipLaunchKernelGGL(rs_plan_tell_kernel<block()>, dim3(1), dim3(block()), 0, (hipStream_t)stream, P);
            if (hipGetLastError() != hipSuccess) return RS_ERR_HIP;
        }
        return RS_OK;
    };
    using std::integral_constant;
    constexpr unsigned kPageGroups = kTakers + kGivers + kTellers;
    if (R <= 64 && T <= 64) return step(integral_constant<int, 64>(), 1);
    if (R <= 256 && T <= 512 && in_place) return step(integral_constant<int, 256>(), 1);
    if (R <= 256) return step(integral_constant<int, 256>(), std::min(((unsigned)T + 255) / 256, 1024u) + kPageGroups);
    if (R <= 1024)
        return step(integral_constant<int, 1024>(), std::max(1u, std::min(((unsigned)T + 1023) / 1024, 256u)) + kPageGroups);
    hipLaunchKernelGGL(rs_plan_kernel, dim3(1), dim3(kPlanBlock), 0, (hipStream_t)stream, P);
    if (hipGetLastError() != hipSuccess) return RS_ERR_HIP;
    if (T == 0) return RS_OK;
    hipLaunchKernelGGL(rs_plan_rows_kernel, dim3((unsigned)(((int64_t)T + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                       P);
    return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_accepted_path(const int32_t* parent, const int32_t* node_token, const int32_t* tokens,
                                 const int32_t* accepted_len, int32_t B, int32_t N, int32_t max_depth,
                                 int32_t* out_path, int32_t* out_status, void* stream) {
    if (B < 0 || N <= 0 || max_depth < 0 || max_depth == INT_MAX) return RS_ERR_INVALID_ARG;
    if (N > RS_MAX_PATH_NODES || B >= 1 << 22) return RS_ERR_UNSUPPORTED;     // less than 2^32 threads
    if (B == 0) return RS_OK;
    if (!parent || !node_token || !tokens || !accepted_len || !out_path) return RS_ERR_INVALID_ARG;
    if (N <= 64) {
        hipLaunchKernelGGL(rs_path_wave_kernel, dim3((unsigned)(((int64_t)B + kPathWaves - 1) / kPathWaves)),
                           dim3(kPathWaves * 64), 0, (hipStream_t)stream, parent, node_token, tokens, accepted_len, B, N,
                           max_depth, out_path, out_status);
        return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
    }
    const int block = N <= 1024 ? 256 : 1024;
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
    if (cache_rows->row_bytes > INT_MAX) return RS_ERR_UNSUPPORTED;
    if (B == 0) return RS_OK;
    if (!cache || !slots || !path) return RS_ERR_INVALID_ARG;
    CommitParams P{};
    P.cache = static_cast<uint8_t*>(cache);
    P.c = strides_of(*cache_rows);
    P.slots = slots;
    P.path = path;
    P.within = !source;
    P.source = source ? static_cast<const uint8_t*>(source) : P.cache;
    P.s = source ? strides_of(*source_rows) : P.c;
    P.outer = (uint32_t)cache_rows->outer;
    P.inner = (uint32_t)cache_rows->inner;
    P.bytes = (uint32_t)cache_rows->row_bytes;
    P.page = (uint32_t)cache_rows->positions;
    P.room = (uint32_t)(cache_rows->pages * cache_rows->positions);
    P.N = N;
    P.depth = depth;
    P.status = out_status;
    P.G = groups_for(cache_rows->outer * cache_rows->inner, B, kCommitWaves);
    if ((int64_t)P.G * B > INT_MAX / kCommitBlock) return RS_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(rs_commit_kernel, dim3((unsigned)P.G * B), dim3(kCommitBlock), 0, (hipStream_t)stream, P);
    return hipGetLastError() == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
