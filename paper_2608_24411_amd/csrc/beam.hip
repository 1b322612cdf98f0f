// beam.hip -- beam search's choice of the next beams from rows of logits on gfx950
// (resispec_beam_select).  Declared in resispec.h.

#include "common.h"

#include <climits>

namespace {

// Mathematics.  The score of token v after beam w is s_w + (l_v - m)/T - L, L = ln sum_j
// exp((l_j - m)/T): within a row the order is that of the logits, across rows the sums decide.
// Two launches.  The first reads the rows once, in chunks of 512 elements that any wave may
// take: a chunk leaves its maximum and the sum of its masses against that maximum.  The second,
// a workgroup a sequence, adds the chunks up and chooses: of all a sequence's elements in order
// the first k lie in the first k chunks, ordered by their maximum, then by place.  (If an
// element's chunk were behind k others, each of these would hold an element before it.)  So
// only k chunks are read again.

constexpr int kChunk = 512;              // elements of a chunk
constexpr int kRowsBlock = 256, kRowsWaves = kRowsBlock / 64;
constexpr int kMergeBlock = 1024, kMergeWaves = kMergeBlock / 64;

struct ChunkSum {
    double sum;                          // of 2^((l - max) c)
    float max;
    float pad;
};

struct BeamParams {
    const void* logits;
    int64_t stride;
    const float* scores;
    const uint8_t* ended;
    int32_t end_token;
    int32_t B, W, V, k;
    int32_t rows_per_entry;
    float temperature;
    const float* temperatures;
    int32_t nch, parts;                  // chunks a row, workgroups a row
    ChunkSum* chunks;                    // [B * W][nch]
    int32_t *parent, *token, *status;
    float* score;
    __device__ __forceinline__ float T(int64_t r) const {
        return temperatures ? temperatures[r / rows_per_entry] : temperature;
    }
    // whether row r is read: there is such a beam, and it goes on
    __device__ __forceinline__ bool live(int64_t r) const {
        return scores[r] > -INFINITY && !(ended && ended[r]);
    }
};

template <typename In, int VEC>
struct Chunk {
    using W = Vec<In, VEC>;
    static constexpr int UNR = kChunk / (64 * VEC), N = UNR * VEC;
    typename W::raw t[UNR];
    // Loads take no branch: what lies past the row reads its last elements, and is put right
    // when it is unpacked.
    __device__ __forceinline__ void load(const In* row, int c, int V) {
        const int j0 = c * kChunk + (threadIdx.x & 63) * VEC;
#pragma unroll
        for (int u = 0; u < UNR; ++u) t[u] = W::template load_full<false>(row, min(j0 + u * 64 * VEC, V - VEC));
    }
    __device__ __forceinline__ void unpack(int c, int V, float (&v)[N]) {
        const int j0 = c * kChunk + (threadIdx.x & 63) * VEC;
        if (c * kChunk + kChunk > V) {
#pragma unroll
            for (int u = 0; u < UNR; ++u) {
                const int j = j0 + u * 64 * VEC;
                if constexpr (VEC == 1) {
                    if (j >= V) t[u] = 0xff800000u;
                } else {
                    constexpr uint32_t FILL = sizeof(In) == 2 ? 0xff80ff80u : 0xff800000u;
                    if (j >= V) t[u] = make_uint4(FILL, FILL, FILL, FILL);
                    else if (j + VEC > V) t[u] = drop_front<(int)sizeof(In), FILL>(t[u], j + VEC - V);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < UNR; ++u) {
            float x[VEC];
            W::unpack(t[u], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[u * VEC + e] = x[e];
        }
    }
    // the place of value i of this lane in the row
    static __device__ __forceinline__ int at(int c, int i) {
        return c * kChunk + (i / VEC) * 64 * VEC + (threadIdx.x & 63) * VEC + i % VEC;
    }
};

template <typename In, int VEC>
__global__ void __launch_bounds__(kRowsBlock) rs_beam_rows_kernel(const BeamParams P) {
    using C = Chunk<In, VEC>;
    const int64_t r = blockIdx.x / P.parts;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!P.live(r)) return;
    const In* row = reinterpret_cast<const In*>(P.logits) + r * P.stride;
    const double c2 = uniform(1.4426950408889634 / (double)P.T(r));
    for (int c = (int)(blockIdx.x % P.parts) * kRowsWaves + wave; c < P.nch; c += P.parts * kRowsWaves) {
        C chunk;
        chunk.load(row, c, P.V);
        float v[C::N];
        chunk.unpack(c, P.V, v);
        float m = v[0];
#pragma unroll
        for (int i = 1; i < C::N; ++i) m = fmaxf(m, v[i]);
        m = wave_max(m);
        const float ref = m > -INFINITY ? m : 0.0f;
        double sum = 0.0;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < C::N; ++i) {
            bad |= !(v[i] < INFINITY);
            sum += exp2_64(((double)v[i] - (double)ref) * c2);
        }
        sum = wave_sum(sum);
        if (__ballot(bad)) sum = NAN;
        if (lane == 0) P.chunks[r * P.nch + c] = {sum, m, 0.0f};
    }
}

// One place of the order: a beam, and an element of its row or a chunk of it.
struct Place {
    double score;
    int32_t w;
    float l;
    int32_t j;
};
// Whether a comes before b: by score, beam, logit, place in the row.
__device__ __forceinline__ bool before(const Place& a, const Place& b) {
    if (a.w == b.w) return a.l > b.l || (a.l == b.l && a.j < b.j);
    return a.score > b.score || (a.score == b.score && a.w < b.w);
}
__device__ __forceinline__ Place shfl_xor(const Place& a, int d) {
    return {__shfl_xor(a.score, d), __shfl_xor(a.w, d), __shfl_xor(a.l, d), __shfl_xor(a.j, d)};
}
constexpr int kNoBeam = INT_MAX;
__device__ __forceinline__ Place nothing() { return {-INFINITY, kNoBeam, -INFINITY, INT_MAX}; }
__device__ __forceinline__ Place wave_first(Place a) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const Place b = shfl_xor(a, d);
        if (before(b, a)) a = b;
    }
    return a;
}

struct MergeSmem {
    double log_sum[RS_MAX_CANDIDATES];
    float max[RS_MAX_CANDIDATES], s[RS_MAX_CANDIDATES], T[RS_MAX_CANDIDATES];
    int32_t kind[RS_MAX_CANDIDATES];     // 0: no beam, 1: live, 2: ended
    int32_t status;
    Place place[2][kMergeWaves];
    Place chosen[RS_MAX_CANDIDATES];     // chunks
};

template <typename In, int VEC>
__global__ void __launch_bounds__(kMergeBlock) rs_beam_merge_kernel(const BeamParams P) {
    using C = Chunk<In, VEC>;
    __shared__ MergeSmem sm;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t b = blockIdx.x, r0 = b * P.W;
    const ChunkSum* chunks = P.chunks + r0 * P.nch;
    if (tid == 0) sm.status = RS_SEQ_OK;
    __syncthreads();
    for (int w = wave; w < P.W; w += kMergeWaves) {
        const float s = P.scores[r0 + w], T = P.T(r0 + w);
        int kind = s == -INFINITY ? 0 : P.ended && P.ended[r0 + w] ? 2 : 1;
        int st = RS_SEQ_OK;
        if (!(s < INFINITY)) st = RS_SEQ_BAD_PARAM;
        if (kind == 1 && !(T > 0.0f && T < INFINITY)) st = RS_SEQ_BAD_PARAM;
        float m = -INFINITY;
        double sum = 0.0;
        if (kind == 1 && st == RS_SEQ_OK) {
            for (int c = lane; c < P.nch; c += 64) m = fmaxf(m, chunks[w * P.nch + c].max);
            m = wave_max(m);
            const double c2 = 1.4426950408889634 / (double)T;
            for (int c = lane; c < P.nch; c += 64) {
                const ChunkSum x = chunks[w * P.nch + c];
                if (x.sum != 0.0) sum += x.sum * exp2_64(((double)x.max - (double)m) * c2);
            }
            sum = wave_sum(sum);
            if (!(m > -INFINITY && m < INFINITY && sum < INFINITY)) st = RS_SEQ_UNDERFLOW;
        }
        if (lane == 0) {
            sm.kind[w] = kind;
            sm.s[w] = s;
            sm.T[w] = T;
            sm.max[w] = m;
            sm.log_sum[w] = kind == 1 && st == RS_SEQ_OK ? log(sum) : 0.0;
            if (st != RS_SEQ_OK) atomicMax(&sm.status, st);
        }
    }
    __syncthreads();
    const int status = sm.status;
    if (status != RS_SEQ_OK) {
        for (int i = tid; i < P.k; i += kMergeBlock) {
            P.parent[b * P.k + i] = P.token[b * P.k + i] = -1;
            P.score[b * P.k + i] = NAN;
        }
        if (tid == 0 && P.status) P.status[b] = status;
        return;
    }
    auto score = [&](int w, float l) {
        if (sm.kind[w] == 2) return (double)sm.s[w];
        return (((double)l - (double)sm.max[w]) / (double)sm.T[w] - sm.log_sum[w]) + (double)sm.s[w];
    };
    // the first k chunks, one after another
    Place prev = {INFINITY, -1, INFINITY, -1};
    int nsel = 0;
    for (int i = 0; i < P.k; ++i) {
        Place best = nothing();
        for (int w = 0; w < P.W; ++w) {
            const int kind = sm.kind[w];
            if (kind == 0) continue;
            for (int c = tid; c < (kind == 2 ? 1 : P.nch); c += kMergeBlock) {
                const float l = kind == 2 ? 0.0f : chunks[w * P.nch + c].max;
                if (l == -INFINITY) continue;
                const Place x = {score(w, l), w, l, c};
                if (before(prev, x) && before(x, best)) best = x;
            }
        }
        best = wave_first(best);
        if (lane == 0) sm.place[i & 1][wave] = best;
        __syncthreads();
        best = sm.place[i & 1][0];
        for (int w = 1; w < kMergeWaves; ++w)
            if (before(sm.place[i & 1][w], best)) best = sm.place[i & 1][w];
        if (best.w == kNoBeam) break;
        if (tid == 0) sm.chosen[i] = best;
        prev = best;
        nsel = i + 1;
    }
    __syncthreads();
    // their elements, a wave up to four chunks, and the first k of those
    constexpr int kEach = RS_MAX_CANDIDATES / kMergeWaves;
    float v[kEach][C::N];
    Place head[kEach];
    auto first_of = [&](int q) {
        const int i = wave + q * kMergeWaves;
        head[q] = nothing();
        if (i >= nsel) return;
        const Place ch = sm.chosen[i];
        if (sm.kind[ch.w] == 2) {
            if (v[q][0] == 0.0f) head[q] = {ch.score, ch.w, 0.0f, P.end_token};
            return;
        }
        float l = -INFINITY;
        int at = INT_MAX;
#pragma unroll
        for (int e = 0; e < C::N; ++e)
            if (v[q][e] > l) {
                l = v[q][e];
                at = C::at(ch.j, e);
            }
        const float top = wave_max(l);
        if (top == -INFINITY) return;
        int j = l == top ? at : INT_MAX;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) j = min(j, __shfl_xor(j, d));
        head[q] = {score(ch.w, top), ch.w, top, j};
    };
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        const int i = wave + q * kMergeWaves;
        if (i < nsel) {
            const Place ch = sm.chosen[i];
            if (sm.kind[ch.w] == 2) {
                v[q][0] = 0.0f;
            } else {
                C chunk;
                chunk.load(reinterpret_cast<const In*>(P.logits) + (r0 + ch.w) * P.stride, ch.j, P.V);
                chunk.unpack(ch.j, P.V, v[q]);
            }
        }
        first_of(q);
    }
    int found = 0;
    for (int i = 0; i < P.k; ++i) {
        Place mine = head[0];
#pragma unroll
        for (int q = 1; q < kEach; ++q)
            if (before(head[q], mine)) mine = head[q];
        if (lane == 0) sm.place[i & 1][wave] = mine;
        __syncthreads();
        Place best = sm.place[i & 1][0];
        for (int w = 1; w < kMergeWaves; ++w)
            if (before(sm.place[i & 1][w], best)) best = sm.place[i & 1][w];
        if (best.w == kNoBeam) break;
        found = i + 1;
        if (tid == 0) {
            P.parent[b * P.k + i] = best.w;
            P.token[b * P.k + i] = best.j;
            P.score[b * P.k + i] = (float)best.score;
        }
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (head[q].w == best.w && head[q].j == best.j) {
                const Place ch = sm.chosen[wave + q * kMergeWaves];
                if (sm.kind[ch.w] == 2) {
                    v[q][0] = -INFINITY;
                } else {
#pragma unroll
                    for (int e = 0; e < C::N; ++e)
                        if (C::at(ch.j, e) == best.j) v[q][e] = -INFINITY;
                }
                first_of(q);
            }
    }
    for (int i = found + tid; i < P.k; i += kMergeBlock) {
        P.parent[b * P.k + i] = P.token[b * P.k + i] = -1;
        P.score[b * P.k + i] = -INFINITY;
    }
    if (tid == 0 && P.status) P.status[b] = RS_SEQ_OK;
}

// ------------------------------------------------------------------- host ----

int32_t chunks_of(int32_t V) { return (V + kChunk - 1) / kChunk; }

constexpr int32_t kMostRows = (1 << 23) - 1;

}  // namespace

extern "C" {

size_t resispec_beam_workspace_bytes(int32_t B, int32_t W, int32_t V) {
    if (B <= 0 || W <= 0 || V <= 0 || W > RS_MAX_CANDIDATES || V > RS_MAX_VOCAB) return 0;
    if ((int64_t)B * W > kMostRows) return 0;
    return (size_t)B * W * chunks_of(V) * sizeof(ChunkSum);
}

rs_status resispec_beam_select(const void* logits, int64_t row_stride, const float* scores, const uint8_t* ended,
                               int32_t end_token, int32_t B, int32_t W, int32_t V, int32_t k, const rs_filter* filter,
                               int32_t* out_parent, int32_t* out_token, float* out_score, int32_t* out_status,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!filter || filter->rows_per_entry < 1) return RS_ERR_INVALID_ARG;
    if (filter->logits_dtype != RS_F32 && filter->logits_dtype != RS_BF16) return RS_ERR_INVALID_ARG;
    if (!filter->temperatures && !(filter->temperature > 0.0f && std::isfinite(filter->temperature)))
        return RS_ERR_INVALID_ARG;
    if (filter->top_ks || filter->top_ps || filter->min_ps || filter->top_k != 0 || filter->top_p != 1.0f ||
        filter->min_p != 0.0f)
        return RS_ERR_INVALID_ARG;
    if (B < 0 || W <= 0 || V <= 0 || k <= 0 || (int64_t)W * V < k || row_stride < V) return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB || W > RS_MAX_CANDIDATES || k > RS_MAX_CANDIDATES || (int64_t)B * W > kMostRows)
        return RS_ERR_UNSUPPORTED;
    if (B == 0) return RS_OK;
    if (!logits || !scores || !out_parent || !out_token || !out_score) return RS_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < resispec_beam_workspace_bytes(B, W, V) ||
        reinterpret_cast<uintptr_t>(workspace) % 16)
        return RS_ERR_WORKSPACE;
    BeamParams P{};
    P.logits = logits;
    P.stride = row_stride;
    P.scores = scores;
    P.ended = ended;
    P.end_token = end_token;
    P.B = B;
    P.W = W;
    P.V = V;
    P.k = k;
    P.rows_per_entry = filter->rows_per_entry;
    P.temperature = filter->temperature;
    P.temperatures = filter->temperatures;
    P.nch = chunks_of(V);
    P.chunks = static_cast<ChunkSum*>(workspace);
    P.parent = out_parent;
    P.token = out_token;
    P.score = out_score;
    P.status = out_status;
    const int64_t R = (int64_t)B * W, most = (P.nch + kRowsWaves - 1) / kRowsWaves, share = (4096 + R - 1) / R;
    P.parts = (int32_t)(most < share ? most : share);
    const int64_t esz = filter->logits_dtype == RS_BF16 ? 2 : 4;
    RowLoads loads = row_loads(logits, logits, V, filter->logits_dtype);
    if (loads == kLoadsAligned && row_stride * esz % 16) loads = kLoadsAny;
    const hipError_t e = with_layout(filter->logits_dtype, loads, [&](auto in, auto vec, auto) {
        hipLaunchKernelGGL((rs_beam_rows_kernel<decltype(in), vec()>), dim3((unsigned)(R * P.parts)), dim3(kRowsBlock), 0,
                           (hipStream_t)stream, P);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((rs_beam_merge_kernel<decltype(in), vec()>), dim3((unsigned)B), dim3(kMergeBlock), 0,
                           (hipStream_t)stream, P);
        return hipGetLastError();
    });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
