// beam.hip -- beam search's choice of the next beams from rows of logits on gfx950
// (resispec_beam_select).  Declared in resispec.h.

#include "mass64.h"

#include <climits>

namespace {

// Mathematics.  The score of token v after beam w is s_w + (l_v - m)/T - L, L = ln sum_j
// exp((l_j - m)/T): within a row the order is that of the logits, across rows the sums decide.
// Two launches.  The first reads the rows once, in units of four chunks of 1024 elements that
// any wave may take: a chunk leaves its maximum, a unit the sum of its masses against its own.
// The second, a workgroup a sequence, adds the units up and chooses: the k largest maxima of
// chunks are k elements, so whatever is chosen is not below the last of them, and only chunks
// that reach so far, about k of a sequence's hundreds, are read again.
//
// Sums are of 32-bit masses (1024 rows of 151,936 bf16 49 us, at 6.35 TB/s; with exponentials in
// fp64 122).  A sum is off by 1.3e-6 of itself at most: an exponent x by 3 * 2^-24 of itself (difference, scale and
// product are rounded), so a mass by 0.693 of that and 2^-23, the mean of |x| by mass over a
// unit of 4096 elements whose maximum is at 0 is 8.1 at most, and three additions are in 32
// bits.  That is enough for a score, and for an order too unless two beams' scores are closer
// than the two errors: then the rows concerned are summed again in 64 bits and the order is
// decided by that.  Such a sum is off by 3.7e-14 of itself for its exponentials, 3 * 2^-53 |x| for
// their arguments (|x| 17 at most in the mean, by mass), and 2^-53 for each of its V / 1024 + 38
// additions at most, one after another: 7e-14 at 151,936 elements, 5e-13 at 2^22.

constexpr int kChunk = 1024;             // elements of a chunk
constexpr int kUnitChunks = 4;           // chunks of a unit
constexpr int kUnit = kChunk * kUnitChunks;
constexpr int kRowsBlock = 256, kRowsWaves = kRowsBlock / 64;
constexpr int kMergeBlock = 1024, kMergeWaves = kMergeBlock / 64;
// Scores this close are told apart by sums in 64 bits; besides, a score has its own rounding.
constexpr double kNear = 3.0e-6, kNearOf = 0x1p-50;

struct UnitSum {
    double sum;                          // of 2^((l - max) c)
    float max, pad;
};

// What both launches are given, and what the second is given besides.  Arguments are kept short:
// a launch with 160 bytes of them takes the host 3.5 us, with 16 2.9.
struct RowsParams {
    const void* logits;
    int64_t stride;
    const float* scores;
    const uint8_t* ended;
    const float* temperatures;
    UnitSum* sums;                       // [B * W][units]
    float* maxima;                       // [B * W][units * kUnitChunks], of the chunks
    float temperature;
    int32_t rows_per_entry;
    int32_t V, units, parts;             // units a row, workgroups a row
    __device__ __forceinline__ float T(int64_t r) const {
        return temperatures ? temperatures[r / rows_per_entry] : temperature;
    }
    // whether row r is read: there is such a beam, and it goes on
    __device__ __forceinline__ bool live(int64_t r) const {
        return scores[r] > -INFINITY && !(ended && ended[r]);
    }
};
struct BeamParams : RowsParams {
    int32_t W, k, end_token;
    uint32_t by_nch;                     // ceil(2^32 / chunks a row)
    int32_t *parent, *token, *status;
    float* score;
};

template <typename In, int VEC>
struct Chunk {
    using W = Vec<In, VEC>;
    static constexpr int UNR = kChunk / (64 * VEC), N = UNR * VEC;
    typename W::raw t[UNR];
    // Loads take no branch: what lies past the row reads its last elements, and settle() puts
    // it right, once.
    template <bool NT>
    __device__ __forceinline__ void load(const In* row, int c, int V) {
        const int j0 = c * kChunk + (threadIdx.x & 63) * VEC;
#pragma unroll
        for (int u = 0; u < UNR; ++u) t[u] = W::template load_full<NT>(row, min(j0 + u * 64 * VEC, V - VEC));
    }
    __device__ __forceinline__ void settle(int c, int V) {
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
    }
    __device__ __forceinline__ void unpack(float (&v)[N]) const {
#pragma unroll
        for (int u = 0; u < UNR; ++u) {
            float x[VEC];
            W::unpack(t[u], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[u * VEC + e] = x[e];
        }
    }
    // the place of a lane's value i in the row
    static __device__ __forceinline__ int place(int c, int lane, int i) {
        return c * kChunk + (i / VEC) * 64 * VEC + lane * VEC + i % VEC;
    }
    static __device__ __forceinline__ int at(int c, int i) { return place(c, threadIdx.x & 63, i); }
};

// The maxima over the wave of four values a lane: lanes q, q + 4, q + 8 .. get that of value q.
__device__ __forceinline__ float wave_max4(float a, float b, float c, float d) {
    const int lane = threadIdx.x & 63;
    const bool odd = lane & 1, high = lane & 2;
    const float ab = fmaxf(odd ? b : a, dpp_f<kDppXor1>(odd ? a : b));
    const float cd = fmaxf(odd ? d : c, dpp_f<kDppXor1>(odd ? c : d));
    float m = fmaxf(high ? cd : ab, dpp_f<kDppXor2>(high ? ab : cd));
    constexpr int kDppRowRor4 = 0x124, kDppRowRor8 = 0x128;
    m = fmaxf(m, dpp_f<kDppRowRor4>(m));
    m = fmaxf(m, dpp_f<kDppRowRor8>(m));
    m = fmaxf(m, __shfl_xor(m, 16));
    return fmaxf(m, __shfl_xor(m, 32));
}

// log2(e) / (T h), within 32 bits.
__device__ __forceinline__ float factor(float T, float h) {
    return (float)fmin(1.4426950408889634 / ((double)T * (double)h), (double)FLT_MAX);
}

template <typename In, int VEC>
__global__ void __launch_bounds__(kRowsBlock) rs_beam_rows_kernel(const RowsParams P) {
    using C = Chunk<In, VEC>;
    const int64_t r = blockIdx.x / P.parts;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!P.live(r)) return;
    const In* row = reinterpret_cast<const In*>(P.logits) + r * P.stride;
    // An exponent is (v - max) h times the factor for that h.  h is 1, but for temperatures above
    // 2^100, where differences that pass 32 bits have masses, and, next to a small maximum, below
    // 2^-100, where the factor passes them.  (Next to a large one only equal elements have any
    // mass there.)  Powers of 2 change no other result.
    const float T = P.T(r), h_far = T > 0x1p100f ? 0x1p-20f : 1.0f;
    const bool tiny = T < 0x1p-100f;
    const float c_far = factor(T, h_far), c_near = tiny ? factor(T, 0x1p64f) : 0.0f;
    for (int unit = (int)(blockIdx.x % P.parts) * kRowsWaves + wave; unit < P.units; unit += P.parts * kRowsWaves) {
        C chunk[kUnitChunks];
#pragma unroll
        for (int q = 0; q < kUnitChunks; ++q) chunk[q].template load<true>(row, unit * kUnitChunks + q, P.V);
        float top[kUnitChunks];
#pragma unroll
        for (int q = 0; q < kUnitChunks; ++q) {
            chunk[q].settle(unit * kUnitChunks + q, P.V);
            float v[C::N];
            chunk[q].unpack(v);
            top[q] = v[0];
#pragma unroll
            for (int i = 1; i < C::N; ++i) top[q] = fmaxf(top[q], v[i]);
        }
        const float each = wave_max4(top[0], top[1], top[2], top[3]);
        float m = fmaxf(each, dpp_f<kDppXor1>(each));
        m = uniform(fmaxf(m, dpp_f<kDppXor2>(m)));
        const float ref = m > -INFINITY ? m : 0.0f;
        const bool near = tiny && fabsf(ref) < 0x1p60f;
        const float h = near ? 0x1p64f : h_far, c = near ? c_near : c_far, ref_h = -ref * h;
        // a NaN or +inf makes the sum a NaN
        double sum = 0.0;
#pragma unroll
        for (int q = 0; q < kUnitChunks; ++q) {
            float v[C::N];
            chunk[q].unpack(v);
#pragma unroll
            for (int i = 0; i < C::N; ++i) v[i] = exp2_fast(fmaf(v[i], h, ref_h) * c);
#pragma unroll
            for (int i = 0; i < C::N; i += 8)
                sum += (double)(((v[i] + v[i + 1]) + (v[i + 2] + v[i + 3])) +
                                ((v[i + 4] + v[i + 5]) + (v[i + 6] + v[i + 7])));
        }
        sum = wave_sum(sum);
        if (lane < kUnitChunks) P.maxima[(r * P.units + unit) * kUnitChunks + lane] = each;
        if (lane == 0) P.sums[r * P.units + unit] = {sum, m, 0.0f};
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

constexpr int kBins = 512;               // of scores of chunks, from the best downwards
constexpr double kBinsPerUnit = 16.0;
constexpr int kChunkList = 512, kList = 1024;
constexpr int kHeld = 5;                 // maxima of chunks a thread holds
// what is listed besides: the errors of two sums and of their logarithms in 32 bits (2e-6 each),
// and the rounding of a distance in bins (8e-6 where bins are told apart)
constexpr double kSlack = 2.0 * kNear + 2.0e-5;

struct MergeSmem {
    double sum[RS_MAX_CANDIDATES], log_sum[RS_MAX_CANDIDATES];
    double top[RS_MAX_CANDIDATES];       // a beam's best continuation, by a 32-bit logarithm
    float max[RS_MAX_CANDIDATES], s[RS_MAX_CANDIDATES], T[RS_MAX_CANDIDATES];
    int32_t kind[RS_MAX_CANDIDATES];     // 0: no beam, 1: live, 2: ended
    int32_t status[RS_MAX_CANDIDATES];
    int32_t nchunks, nlist;
    uint32_t doubt[2];                   // beams to be summed in 64 bits
    double part[kMergeWaves];
    int32_t bin[kBins];
    union {
        Place list[kList];
        struct {
            Place place[2][kMergeWaves];
            Place chosen[RS_MAX_CANDIDATES], heads[RS_MAX_CANDIDATES];
        };
    };
    int32_t chunks[kChunkList];          // those to read again: beam * chunks a row + chunk
};

// Inclusive prefix sum over the 64 lanes, as wave_incl_scan.
template <int CTRL, int ROWMASK>
__device__ __forceinline__ int dpp_or_zero(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWMASK, 0xF, true);
}
__device__ __forceinline__ int wave_incl_scan_i(int v) {
    v += dpp_or_zero<kDppRowShr1, 0xF>(v);
    v += dpp_or_zero<kDppRowShr2, 0xF>(v);
    v += dpp_or_zero<kDppRowShr4, 0xF>(v);
    v += dpp_or_zero<kDppRowShr8, 0xF>(v);
    v += dpp_or_zero<kDppRowBcast15, 0xA>(v);
    v += dpp_or_zero<kDppRowBcast31, 0xC>(v);
    return v;
}

template <typename In, int VEC>
struct Merge {
    using C = Chunk<In, VEC>;
    using E = std::conditional_t<sizeof(In) == 2, uint16_t, float>;
    const BeamParams& P;
    MergeSmem& sm;
    const int64_t b, r0;
    const int tid, lane, wave, nch;
    const uint32_t by_nch;               // i / nch is the high half of i * by_nch for i < 2^18, nch <= 2^12

    __device__ __forceinline__ const In* row(int w) const {
        return reinterpret_cast<const In*>(P.logits) + (r0 + w) * P.stride;
    }
    __device__ __forceinline__ float chunk_max(int w, int c) const {
        return P.maxima[(r0 + w) * (int64_t)nch + c];
    }
    __device__ __forceinline__ double score(int w, float l) const {
        if (sm.kind[w] == 2) return (double)sm.s[w];
        return (((double)l - (double)sm.max[w]) / (double)sm.T[w] - sm.log_sum[w]) + (double)sm.s[w];
    }

    // Every beam's kind, maximum and sum, a wave a beam.
    __device__ __forceinline__ void sums() {
        for (int w = wave; w < P.W; w += kMergeWaves) {
            // asked for before it is known whether they are wanted
            const UnitSum* units = P.sums + (r0 + w) * P.units;
            const UnitSum x = lane < P.units ? units[lane] : UnitSum{0.0, -INFINITY, 0.0f};
            const float s = P.scores[r0 + w], T = P.T(r0 + w);
            const int kind = s == -INFINITY ? 0 : P.ended && P.ended[r0 + w] ? 2 : 1;
            int st = RS_SEQ_OK;
            if (!(s < INFINITY) || (kind == 1 && !(T > 0.0f && T < INFINITY))) st = RS_SEQ_BAD_PARAM;
            float m = -INFINITY;
            double sum = 1.0;
            if (kind == 1 && st == RS_SEQ_OK) {
                m = x.max;
                for (int u = lane + 64; u < P.units; u += 64) m = fmaxf(m, units[u].max);
                m = wave_max(m);
                sum = 0.0;
                const double c2 = 1.4426950408889634 / (double)T;
                auto add = [&](const UnitSum& y) {
                    if (y.sum != 0.0) sum += y.sum * exp2_64(((double)y.max - (double)m) * c2);
                };
                add(x);
                for (int u = lane + 64; u < P.units; u += 64) add(units[u]);
                sum = wave_sum(sum);
                if (!(m > -INFINITY && m < INFINITY && sum < INFINITY)) st = RS_SEQ_UNDERFLOW;
            }
            if (lane == 0) {
                sm.kind[w] = kind;
                sm.s[w] = s;
                sm.T[w] = T;
                sm.max[w] = m;
                sm.sum[w] = sum;
                sm.top[w] = (double)s - (double)(__builtin_amdgcn_logf((float)sum) * 0.693147181f);
                sm.status[w] = st;
            }
        }
    }

    // Row w's sum in 64 bits, by all threads.
    __device__ __forceinline__ void sum_again(int w) {
        const double c2 = 1.4426950408889634 / (double)sm.T[w], md = (double)sm.max[w];
        double sum = 0.0;
        for (int c = wave; c < nch && c * (int64_t)kChunk < P.V; c += kMergeWaves) {
            C chunk;
            chunk.template load<false>(row(w), c, P.V);
            chunk.settle(c, P.V);
            float v[C::N];
            chunk.unpack(v);
#pragma unroll
            for (int i = 0; i < C::N; ++i) sum += exp2_64(((double)v[i] - md) * c2);
        }
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) sm.part[wave] = sum;
        __syncthreads();
        if (tid == 0) {
            sum = 0.0;
            for (int i = 0; i < kMergeWaves; ++i) sum += sm.part[i];
            sm.log_sum[w] = log(sum);
        }
    }

    // A distance from the reference, in bins, counted in its bin.
    __device__ __forceinline__ void count(float d) { atomicAdd(&sm.bin[(int)fminf(fmaxf(d, 0.0f), kBins - 1)], 1); }

    // The bin in which the k-th counted lies, or the last one if there are fewer.  Every wave
    // looks for itself.
    __device__ __forceinline__ int bin_of_kth() const {
        constexpr int kLaneBins = kBins / 64;
        int n[kLaneBins], mine = 0;
#pragma unroll
        for (int i = 0; i < kLaneBins; ++i) mine += n[i] = sm.bin[lane * kLaneBins + i];
        int upto = wave_incl_scan_i(mine);
        const uint64_t reached = __ballot(upto >= P.k);
        int kth = kLaneBins - 1;
#pragma unroll
        for (int i = kLaneBins - 1; i >= 0; --i) {
            if (upto >= P.k) kth = i;
            upto -= n[i];
        }
        const int at = reached ? __builtin_ctzll(reached) : 63;
        return at * kLaneBins + __builtin_amdgcn_readlane(kth, at);
    }

    // body(w, l, j) for what the listed chunks hold within `far` of the reference.
    template <typename Body>
    __device__ __forceinline__ void each_listed(double reference, double far, Body&& body) {
        const int n = sm.nchunks;
        for (int i = wave; i < n; i += kMergeWaves) {
            const int id = __builtin_amdgcn_readfirstlane(sm.chunks[i]), w = id / nch, c = id - w * nch;
            if (sm.kind[w] == 2) {
                if (lane == 0) body(w, 0.0f, P.end_token);
                continue;
            }
            C chunk;
            chunk.template load<false>(row(w), c, P.V);
            // the row's least logit within reach, or one below it
            const double least = (reference - far - (double)sm.s[w] + sm.log_sum[w]) * (double)sm.T[w] + (double)sm.max[w];
            const float cut = fmaxf((float)(least - fabs(least) * 0x1p-23), -FLT_MAX);
            chunk.settle(c, P.V);
            float v[C::N];
            chunk.unpack(v);
            float top = v[0];
#pragma unroll
            for (int e = 1; e < C::N; ++e) top = fmaxf(top, v[e]);
            // Elements are read again: in registers each is a place of its own, and much code (the
            // choice of 64 of 32 beams 15.2 us where this takes 13.6).  Few lanes have any, mostly:
            // the wave takes one lane's elements after another's, else every lane its own (rows
            // without an order, 8 of 128,256: 620 us by the first way alone, 110 so).
            auto one = [&](int j) {
                float l[1];
                load_vec<E, 1>(reinterpret_cast<const E*>(row(w)), j, P.V, l);
                if (l[0] >= cut) body(w, l[0], j);
            };
            uint64_t hits = __ballot(top >= cut);
            if (__popcll(hits) <= 4) {
                for (; hits; hits &= hits - 1) {
                    const int j = C::place(c, __builtin_ctzll(hits), lane);
                    if (lane < C::N && j < P.V) one(j);
                }
            } else {
#pragma unroll 1
                for (int e = 0; e < C::N; ++e)
                    if (C::at(c, e) < P.V) one(C::at(c, e));
            }
        }
        __syncthreads();
    }
    __device__ __forceinline__ void list_listed(double reference, double far) {
        each_listed(reference, far, [&](int w, float l, int j) {
            const int at = atomicAdd(&sm.nlist, 1);
            if (at < kList) sm.list[at] = {0.0, w, l, j};
        });
    }

    // Lists every continuation that can be among the first k.  False where the lists are too
    // short for it: many equal elements, or large vocabularies with no order to speak of.
    // maxima: those of the chunks tid, tid + kMergeBlock ..
    __device__ __forceinline__ bool list(const float (&maxima)[kHeld]) {
        const int n = P.W * nch;
        // a score near the best: distances are from here
        const float high = wave_max(lane < P.W ? (float)sm.top[lane] : -INFINITY);
        const double reference = high > -INFINITY ? (double)high : 0.0, slack = kSlack + 4.0 * fabs(reference) * kNearOf;
        // how far the score of chunk i's first element is below it, in bins
        auto key = [&](int i, float l) {
            const int w = (int)__umulhi((uint32_t)i, by_nch), kind = sm.kind[w];
            if (kind == 0 || (kind == 2 && i != w * nch)) return INFINITY;
            const float below = (float)(reference - sm.top[w]);
            if (kind == 2) return fminf(below * (float)kBinsPerUnit, FLT_MAX);
            if (l == -INFINITY) return INFINITY;
            return fminf((below + (sm.max[w] - l) / sm.T[w]) * (float)kBinsPerUnit, FLT_MAX);
        };
        float held[kHeld];
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = tid + h * kMergeBlock;
            held[h] = i < n ? key(i, maxima[h]) : INFINITY;
            if (held[h] < INFINITY) count(held[h]);
        }
        auto later = [&](auto&& body) {
            for (int i = tid + kHeld * kMergeBlock; i < n; i += kMergeBlock) {
                const float d = key(i, P.maxima[r0 * nch + i]);
                if (d < INFINITY) body(i, d);
            }
        };
        later([&](int, float d) { count(d); });
        __syncthreads();
        int bin = bin_of_kth();
        // the last bin has no end, so all chunks are listed
        const bool all = bin == kBins - 1;
        const double far = all ? (double)INFINITY : (bin + 1) / kBinsPerUnit + slack;
        const float limit = all ? FLT_MAX : (float)((far + slack) * kBinsPerUnit);
        auto pick = [&](int i, float d) {
            if (!(d <= limit)) return;
            const int at = atomicAdd(&sm.nchunks, 1);
            if (at < kChunkList) sm.chunks[at] = i;
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h) pick(tid + h * kMergeBlock, held[h]);
        later(pick);
        __syncthreads();
        if (sm.nchunks > kChunkList) return false;
        if (!all) {
            list_listed(reference, far);
            if (sm.nlist <= kList) return true;
        }
        // finer, by the elements themselves
        const double bins_per_unit = all ? kBinsPerUnit : kBins / far;
        __syncthreads();
        for (int i = tid; i < kBins; i += kMergeBlock) sm.bin[i] = 0;
        if (tid == 0) sm.nlist = 0;
        __syncthreads();
        each_listed(reference, far, [&](int w, float l, int) {
            count((float)fmin((reference - score(w, l)) * bins_per_unit, (double)FLT_MAX));
        });
        __syncthreads();
        bin = bin_of_kth();
        list_listed(reference, bin < kBins - 1 ? (bin + 1) / bins_per_unit + slack : far);
        return sm.nlist <= kList;
    }

    __device__ __forceinline__ void put(int i, int w, int j, double s) const {
        P.parent[b * P.k + i] = w;
        P.token[b * P.k + i] = j;
        P.score[b * P.k + i] = (float)s;
    }

    // The listed continuations at their places in the order: 16 lanes count how many come before
    // one.  Beams are marked whose scores are too close to call.
    __device__ __forceinline__ void rank() {
        const int n = sm.nlist, sub = lane & 15;
        for (int i = tid; i < n; i += kMergeBlock) sm.list[i].score = score(sm.list[i].w, sm.list[i].l);
        __syncthreads();
        for (int i = tid >> 4; i < n; i += kMergeBlock / 16) {
            const Place mine = sm.list[i];
            int ahead = 0;
            uint64_t close = 0;
            for (int x = sub; x < n; x += 16) {
                const Place other = sm.list[x];
                ahead += before(other, mine);
                if (other.w != mine.w && fabs(other.score - mine.score) <= kNear + fabs(mine.score) * kNearOf)
                    close |= 1ull << other.w;
            }
            ahead += dpp_i<kDppXor1>(ahead);
            ahead += dpp_i<kDppXor2>(ahead);
            ahead += dpp_i<kDppHalfMirror>(ahead);
            ahead += dpp_i<kDppMirror>(ahead);
            if (ahead >= P.k) continue;
            if (sub == 0) put(ahead, mine.w, mine.j, mine.score);
            if (close) {
                close |= 1ull << mine.w;
                atomicOr(&sm.doubt[0], (uint32_t)close);
                atomicOr(&sm.doubt[1], (uint32_t)(close >> 32));
            }
        }
    }

    __device__ __forceinline__ Place first_of_all(Place mine, int parity) {
        if (lane == 0) sm.place[parity][wave] = mine;
        __syncthreads();
        Place best = sm.place[parity][0];
        for (int w = 1; w < kMergeWaves; ++w)
            if (before(sm.place[parity][w], best)) best = sm.place[parity][w];
        return best;
    }

    // The choice where lists do not do: the first k chunks by their maxima hold it (if an
    // element's chunk were behind k others, each of these would hold an element before it), and
    // one place is settled after another.  Sums in 64 bits have been taken.
    __device__ __forceinline__ int one_by_one() {
        Place prev = {INFINITY, -1, INFINITY, -1};
        int nsel = 0;
        for (int i = 0; i < P.k; ++i) {
            Place best = nothing();
            for (int w = 0; w < P.W; ++w) {
                const int kind = sm.kind[w];
                if (kind == 0) continue;
                for (int c = tid; c < (kind == 2 ? 1 : nch); c += kMergeBlock) {
                    const float l = kind == 2 ? 0.0f : chunk_max(w, c);
                    if (l == -INFINITY) continue;
                    const Place x = {score(w, l), w, l, c};
                    if (before(prev, x) && before(x, best)) best = x;
                }
            }
            best = first_of_all(wave_first(best), i & 1);
            if (best.w == kNoBeam) break;
            if (tid == 0) sm.chosen[i] = best;
            prev = best;
            nsel = i + 1;
        }
        // heads[i]: the first element of chunk i that has not been put out; by logit and place
        // within a chunk, so that each is found without a score
        for (int i = tid; i < nsel; i += kMergeBlock) sm.heads[i] = {0.0, 0, INFINITY, -1};
        __syncthreads();
        auto next = [&](int i) {
            const Place ch = sm.chosen[i], was = sm.heads[i];
            float l = -INFINITY;
            int at = INT_MAX;
            if (sm.kind[ch.w] == 2) {
                if (lane == 0 && was.l == INFINITY) {
                    l = 0.0f;
                    at = P.end_token;
                }
            } else {
                C chunk;
                chunk.template load<false>(row(ch.w), ch.j, P.V);
                chunk.settle(ch.j, P.V);
                float v[C::N];
                chunk.unpack(v);
#pragma unroll
                for (int e = 0; e < C::N; ++e) {
                    const int j = C::at(ch.j, e);
                    if ((v[e] < was.l || (v[e] == was.l && j > was.j)) && v[e] > l) {
                        l = v[e];
                        at = j;
                    }
                }
            }
            const float top = wave_max(l);
            int j = l == top && top > -INFINITY ? at : INT_MAX;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) j = min(j, __shfl_xor(j, d));
            if (lane == 0) sm.heads[i] = top > -INFINITY ? Place{score(ch.w, top), ch.w, top, j} : nothing();
        };
        int mine = wave;                 // the chunk whose head is to be found
        int found = 0;
        for (int i = 0;;) {
            // every chunk's first head, then that of the chunk whose head has been put out
            while (mine < nsel) {
                next(mine);
                mine = found == 0 && i == 0 ? mine + kMergeWaves : nsel;
            }
            __syncthreads();
            if (i == P.k) break;
            const Place head = lane < nsel ? sm.heads[lane] : nothing();
            const Place best = wave_first(head);
            if (best.w == kNoBeam) break;
            if (tid == 0) put(i, best.w, best.j, best.score);
            found = ++i;
            const int from = __builtin_ctzll(__ballot(lane < nsel && head.w == best.w && head.j == best.j));
            mine = from % kMergeWaves == wave ? from : nsel;
            __syncthreads();
        }
        return found;
    }

    __device__ __forceinline__ void run() {
        float maxima[kHeld];
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = tid + h * kMergeBlock;
            maxima[h] = i < P.W * nch ? P.maxima[r0 * nch + i] : -INFINITY;
        }
        for (int i = tid; i < kBins; i += kMergeBlock) sm.bin[i] = 0;
        if (tid == 0) {
            sm.nchunks = sm.nlist = 0;
            sm.doubt[0] = sm.doubt[1] = 0;
        }
        sums();
        __syncthreads();
        const int st = lane < P.W ? sm.status[lane] : RS_SEQ_OK;
        const int status = __ballot(st == RS_SEQ_BAD_PARAM) ? RS_SEQ_BAD_PARAM
                           : __ballot(st != RS_SEQ_OK)      ? RS_SEQ_UNDERFLOW
                                                            : RS_SEQ_OK;
        // the sums' logarithms, by one wave while the others look for what to read
        if (wave == kMergeWaves - 1 && lane < P.W) sm.log_sum[lane] = log(sm.sum[lane]);
        int found = 0;
        if (status == RS_SEQ_OK) {
            if (list(maxima)) {
                found = min(sm.nlist, P.k);
                rank();
                __syncthreads();
                const uint64_t doubt = (uint64_t)sm.doubt[1] << 32 | sm.doubt[0];
                if (doubt) {
                    for (int w = 0; w < P.W; ++w)
                        if ((doubt >> w & 1) && sm.kind[w] == 1) sum_again(w);
                    __syncthreads();
                    rank();
                }
            } else {
                for (int w = 0; w < P.W; ++w)
                    if (sm.kind[w] == 1) sum_again(w);
                __syncthreads();
                found = one_by_one();
            }
        }
        const float none = status == RS_SEQ_OK ? -INFINITY : NAN;
        for (int i = found + tid; i < P.k; i += kMergeBlock) put(i, -1, -1, none);
        if (tid == 0 && P.status) P.status[b] = status;
    }
};

template <typename In, int VEC>
__global__ void __launch_bounds__(kMergeBlock) rs_beam_merge_kernel(const BeamParams P) {
    __shared__ MergeSmem sm;
    const int tid = threadIdx.x;
    Merge<In, VEC> m{P, sm, (int64_t)blockIdx.x, (int64_t)blockIdx.x * P.W, tid, tid & 63,
                     __builtin_amdgcn_readfirstlane(tid >> 6), P.units * kUnitChunks, P.by_nch};
    m.run();
}

// ------------------------------------------------------------------- host ----

int32_t units_of(int32_t V) { return (V + kUnit - 1) / kUnit; }

// less than 2^32 threads a launch: of the rows' pass, and of the merge
constexpr int32_t kMostRows = (1 << 23) - 1, kMostSequences = (1 << 22) - 1;

}  // namespace

extern "C" {

size_t resispec_beam_workspace_bytes(int32_t B, int32_t W, int32_t V) {
    if (B <= 0 || W <= 0 || V <= 0 || W > RS_MAX_CANDIDATES || V > RS_MAX_VOCAB) return 0;
    if ((int64_t)B * W > kMostRows || B > kMostSequences) return 0;
    return (size_t)B * W * units_of(V) * (sizeof(UnitSum) + kUnitChunks * sizeof(float));
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
    if (V > RS_MAX_VOCAB || W > RS_MAX_CANDIDATES || k > RS_MAX_CANDIDATES || (int64_t)B * W > kMostRows ||
        B > kMostSequences)
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
    P.W = W;
    P.V = V;
    P.k = k;
    P.rows_per_entry = filter->rows_per_entry;
    P.temperature = filter->temperature;
    P.temperatures = filter->temperatures;
    P.units = units_of(V);
    P.by_nch = (uint32_t)(((uint64_t)1 << 32) / (P.units * kUnitChunks)) + 1;
    P.sums = static_cast<UnitSum*>(workspace);
    P.maxima = reinterpret_cast<float*>(P.sums + (int64_t)B * W * P.units);
    P.parent = out_parent;
    P.token = out_token;
    P.score = out_score;
    P.status = out_status;
    // a unit a wave, and less than 2^32 threads a launch
    const int64_t R = (int64_t)B * W, most = (P.units + kRowsWaves - 1) / kRowsWaves, share = kMostRows / R;
    P.parts = (int32_t)(most < share ? most : share);
    const int64_t esz = filter->logits_dtype == RS_BF16 ? 2 : 4;
    RowLoads loads = row_loads(logits, logits, V, filter->logits_dtype);
    if (loads == kLoadsAligned && row_stride * esz % 16) loads = kLoadsAny;
    const hipError_t e = with_layout(filter->logits_dtype, loads, [&](auto in, auto vec, auto) {
        hipLaunchKernelGGL((rs_beam_rows_kernel<decltype(in), vec()>), dim3((unsigned)(R * P.parts)), dim3(kRowsBlock), 0,
                           (hipStream_t)stream, static_cast<const RowsParams&>(P));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((rs_beam_merge_kernel<decltype(in), vec()>), dim3((unsigned)B), dim3(kMergeBlock), 0,
                           (hipStream_t)stream, P);
        return hipGetLastError();
    });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
