// sample.hip -- sampling from rows of logits on gfx950: draws under temperature, top-k,
// top-p and min-p from given uniforms (resispec_sample), rows cut to what these keep
// (resispec_filter_logits), and log-probabilities and ranks of given tokens
// (resispec_token_logprobs).  Declared in resispec.h.

#include "mass64.h"

#include <climits>

namespace {

// Mathematics.  A row's elements are ordered by logit, equal ones by index.  top-k, top-p and
// min-p each keep a prefix of that order, so what is kept is one cut: the lowest kept value
// and, among the elements equal to it, the last kept index.  Masses are w_j = 2^((l_j - m) c)
// with m the row's maximum and c = log2(e) / T, in fp64: a token or a cut is decided by the
// side of a border that a sum over the whole row falls on, and of 1e5 borders one lies within
// 1e-6 (what 32-bit exponentials give) of a draw now and then.
//
// What bounds the kernels.  A row is one workgroup's: a cut needs the row's sums before the
// next pass begins.  So a lone row runs at one compute unit's pace through its phases: 1 x
// 32,000 fp32 under top-p 30 us, 1 x 128,256 bf16 under top-k 50 23 us, where the bytes would
// take less than 0.1.  With many rows a filter is two reads and a write (33 x 32 rows of 128,256
// bf16 178 us, 837 MB, 4.7 TB/s, a copy's rate), one and a write where registers hold the row
// (rs_floor_kernel), a cut and its draws are two reads (1024 x 151,936 bf16 under top-p 138 us,
// 581 MB fetched, 4.2 TB/s), a log-probability is one (512 x 151,936 fp32, 20 tokens a row,
// 79-85 us, 311 MB, 3.7-4.0 TB/s).  Rows that are only read, without a pause, come at 6 to 7
// TB/s on this card, so the last two are not at the rate of memory, nor at that of the vector
// ALU (56 % and 43 % of the time).  A batch with a setting a row waits for its slowest rows:
// 256 x 151,936 fp32 101-110 us, where its rows under top-p alone, whose histogram takes an
// fp64 exponential an element, need 101 to 122 and the others 37 to 51.

constexpr int kRowSlots = 256;      // runs of chunks with sums of their own
constexpr int kBins = 2048;         // histogram bins of a search for a cut
// 16-byte loads a lane and chunk.  Four give rows in sequence more loads under way (one row's
// log-probability 16.0 -> 15.0 us) but cost registers, and slots of twice the length to draw
// from: 1024 bf16 rows under top-p 134 us with two and 142 with four, six draws from each of
// 64 rows 45 and 50.
constexpr int kUnrRow = 2;

// Bins of bf16 values, from the highest to the lowest: one for every value with 2^-38 < |l| <
// 1020, one for both zeros, one on each side of it for the values nearer to zero, one at each
// end for those outside (-inf in the last).  Unused: bin 0.
constexpr int kHalf = 6144, kValueBins = 2 * kHalf;
constexpr uint16_t kLoMag = (127 - 38) << 7, kTopMag = kHalf - 1;
constexpr int kTopBin = 1, kZeroBin = kHalf, kLastBin = kValueBins - 1;
constexpr int kGroups = kValueBins / 64, kLaneGroups = kGroups / 64;

// Other rows: bins of 1/128 of a logit, from 8 above a reference near the maximum to 24 below
// it (the first and last take what lies outside).
constexpr int kLinearBins = 4096;
constexpr float kBinsPerUnit = 128.0f, kRefBin = 1024.0f;
constexpr double kMassUnit = 0x1p-40;           // of the masses in them
// Elements that a search may leave to be sorted, and how many of them are sorted by counting.
constexpr int kSorted = 2048, kRanked = 384;
constexpr float kSampleBins = 64.0f;            // of a row's sample: bins a unit of logits

struct SParams {
    const void* logits;
    int64_t stride;                 // elements from row to row
    void* out;                      // filter
    int64_t out_stride;
    const float* u;                 // [R][k]
    int32_t R, V, k;
    int32_t rows_per_entry;
    float temperature, top_p, min_p;
    int32_t top_k;
    const float *temperatures, *top_ps, *min_ps;
    const int32_t* top_ks;
    const int32_t* tokens;          // token_logprobs, [R][k]
    int32_t *token, *kept, *status, *rank;
    float* logprob;
    int32_t G, nslots;
};

struct ReduceSmem {
    double red[2][kMaxWaves];
    int32_t redi[2][kMaxWaves];
    uint32_t redk[2][kMaxWaves];
    float redf[kMaxWaves];
};

struct RowSmem : ReduceSmem {
    union {
        float hist[kBins];            // search within a range of keys
        uint32_t count[kValueBins];   // how often each bf16 value occurs
        double table[kValueBins / 2]; // their masses, from the highest value of the row
        int32_t equal[kValueBins];    // indices of equal elements
        uint32_t sample[kBins];       // of the row's first elements
        uint64_t bins[kLinearBins];   // number or mass of the elements in a bin
        struct {
            uint64_t list[kSorted];   // elements: inverted key, index
            uint64_t sorted[kSorted];
            union {
                double running[kSorted];           // running sums of their masses
                float packed[kMaxWaves][128];      // elements whose masses are to be summed
            };
        };
    };
    // sums over groups of 64 bins while the cut is looked for, over slots after that
    union {
        double slot[kRowSlots];
        double group_sum[kGroups];
    };
    union {
        int32_t ties[kRowSlots];
        int32_t group_count[kGroups];
    };
    int32_t nlist;
    int32_t bin, limit;
};

// The sum of an integer over a wave, to every lane.
__device__ __forceinline__ int wave_sum_i(int v) {
    v += dpp_i<kDppXor1>(v);
    v += dpp_i<kDppXor2>(v);
    v += dpp_i<kDppHalfMirror>(v);
    v += dpp_i<kDppMirror>(v);
    return (__builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16)) +
           (__builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48));
}

// Ordered keys: a > b as floats exactly where key(a) > key(b); -0 and +0 share one.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}

// What is kept of a row: values above tau, and those equal to it up to index `limit`.
struct Cut {
    float tau;
    int32_t limit;
    __device__ __forceinline__ bool keeps(float l, int j) const { return l > tau || (l == tau && j <= limit); }
};

// The same before the ties' last index is looked for: the first `keep` of the `all` elements
// equal to tau are kept.
struct Ties {
    float tau;
    int32_t keep, all;
};

// Byte offsets into the counts of the bins of the two bf16 values in a word.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 bin_bytes(uint32_t word) {
    const u16x2 lo = {kLoMag, kLoMag}, top = {kTopMag, kTopMag}, eight = {8, 8}, four = {4, 4};
    const u16x2 half = {(uint16_t)(4 * kHalf), (uint16_t)(4 * kHalf)};
    const u16x2 mag = __builtin_bit_cast(u16x2, word & 0x7fff7fffu);
    const u16x2 far = __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, lo), top);
    const u16x2 t = __builtin_elementwise_max(far, __builtin_elementwise_min(mag, u16x2{1, 1}));
    const u16x2 neg = __builtin_bit_cast(u16x2, __builtin_bit_cast(i16x2, word) >> 15);
    // 4 kHalf - 4 t for positive values, 4 kHalf + 4 t for negative ones
    return t * ((neg & eight) - four) + half;
}
__device__ __forceinline__ float bin_value(int bin) {
    const int t = bin < kHalf ? kHalf - bin : bin - kHalf;
    if (t == 0) return 0.0f;
    return __uint_as_float((uint32_t)(t + kLoMag) << 16 | (bin > kHalf ? 0x80000000u : 0u));
}

template <typename In, int VEC, int BLOCK, typename Smem = RowSmem>
struct Row {
    using W = Vec<In, VEC>;
    static constexpr int UNR = kUnrRow;
    static constexpr int CHUNK = 64 * VEC * UNR;
    static constexpr int kWaves = BLOCK / 64;
    const In* row;
    int V, G, nslots;
    float m;       // the row's maximum
    double md, c;  // the reference of the masses, the maximum or near it; log2(e) / T
    double T;
    Smem& sm;

    __device__ __forceinline__ double mass(float l) const { return exp2_64(((double)l - md) * c); }

    // body(t, j): a vector of VEC elements from index j as loaded (-inf at and past V);
    // flush(slot) after a slot's last.  A wave's slots are the same in every pass.  NT: the
    // row's last use.  Two chunks of registers alternate.  Loads take no branch, so that the
    // wait before a chunk is for that chunk alone (with bounds checks around them the compiler
    // waits for the next one too: 128 x 5 rows of 128,256 took 60 us where they take 48): what
    // lies past the row reads the row's last elements and is put right in the last chunk, and
    // a wave's last step loads its chunk again.
    template <bool NT, typename Body, typename Flush>
    __device__ __forceinline__ void sweep_raw(Body&& body, Flush&& flush) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        typename W::raw a[UNR], b[UNR];
        auto load = [&](int s, int g, typename W::raw(&t)[UNR]) {
            const int j0 = (s * G + g) * CHUNK + lane * VEC;
#pragma unroll
            for (int u = 0; u < UNR; ++u) t[u] = W::template load_full<NT>(row, min(j0 + u * 64 * VEC, V - VEC));
        };
        auto process = [&](int s, int g, typename W::raw(&t)[UNR]) {
            const int c0 = (s * G + g) * CHUNK, j0 = c0 + lane * VEC;
            if (c0 + CHUNK > V) {
#pragma unroll
                for (int u = 0; u < UNR; ++u) cut_off(t[u], j0 + u * 64 * VEC);
            }
#pragma unroll
            for (int u = 0; u < UNR; ++u) body(t[u], j0 + u * 64 * VEC);
            if (g == G - 1) flush(s);
        };
        int s = wid, g = 0;
        if (s >= nslots) return;
        load(s, g, a);
        for (;;) {
            int s2 = g + 1 == G ? s + kWaves : s, g2 = g + 1 == G ? 0 : g + 1;
            bool more = s2 < nslots;
            load(more ? s2 : s, more ? g2 : g, b);
            process(s, g, a);
            if (!more) break;
            s = g2 + 1 == G ? s2 + kWaves : s2;
            g = g2 + 1 == G ? 0 : g2 + 1;
            more = s < nslots;
            load(more ? s : s2, more ? g : g2, a);
            process(s2, g2, b);
            if (!more) break;
        }
    }
    __device__ __forceinline__ static int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

    // A vector loaded from index min(j, V - VEC): its elements from j on, and -inf after them.
    __device__ __forceinline__ void cut_off(typename W::raw& t, int j) const {
        if constexpr (VEC == 1) {
            if (j >= V) t = 0xff800000u;
        } else {
            constexpr uint32_t FILL = sizeof(In) == 2 ? 0xff80ff80u : 0xff800000u;
            if (j >= V) t = make_uint4(FILL, FILL, FILL, FILL);
            else if (j + VEC > V) t = drop_front<(int)sizeof(In), FILL>(t, j + VEC - V);
        }
    }

    // The same with the elements as floats.
    template <bool NT, typename Body, typename Flush>
    __device__ __forceinline__ void sweep(Body&& body, Flush&& flush) const {
        sweep_raw<NT>([&](const typename W::raw& t, int j) {
            float v[VEC];
            W::unpack(t, v);
            body(v, j);
        }, flush);
    }

    // body(l, j), one element a load: for the rare passes, which would cost the others their
    // registers.
    template <typename Body>
    __device__ __forceinline__ void each(Body&& body) const {
        using E = std::conditional_t<sizeof(In) == 2, uint16_t, float>;
        for (int j = threadIdx.x; j < V; j += BLOCK) {
            float v[1];
            load_vec<E, 1>(reinterpret_cast<const E*>(row), j, V, v);
            body(v[0], j);
        }
    }

    // Sums over the workgroup in an order fixed by its size, to every thread.
    __device__ __forceinline__ void sum2(double& a, double& b, int& p, int& q) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        const double wa = wave_sum(a), wb = wave_sum(b);
        const int wp = wave_sum_i(p), wq = wave_sum_i(q);
        __syncthreads();
        if (lane == 0) {
            sm.red[0][wid] = wa;
            sm.red[1][wid] = wb;
            sm.redi[0][wid] = wp;
            sm.redi[1][wid] = wq;
        }
        __syncthreads();
        a = b = 0.0;
        p = q = 0;
        for (int w = 0; w < kWaves; ++w) {
            a += sm.red[0][w];
            b += sm.red[1][w];
            p += sm.redi[0][w];
            q += sm.redi[1][w];
        }
        a = uniform(a);
        b = uniform(b);
        p = __builtin_amdgcn_readfirstlane(p);
        q = __builtin_amdgcn_readfirstlane(q);
    }
    // Sums of masses in an order that does not depend on the workgroup's size: that of kMaxWaves
    // waves, of which a wave takes kParts, its own number and those kWaves apart.  Cuts follow
    // from them, and one on a border (a share of the mass to the last bit) would fall on
    // another side of it in another batch.
    static constexpr int kParts = kMaxWaves / kWaves;
    static_assert(kParts * kWaves == kMaxWaves, "whole parts");
    __device__ __forceinline__ double sum_parts(const double (&v)[kParts]) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
            const double t = wave_sum(v[q]);
            if (lane == 0) sm.red[0][wid + q * kWaves] = t;
        }
        __syncthreads();
        double a = 0.0;
        for (int w = 0; w < kMaxWaves; ++w) a += sm.red[0][w];
        return uniform(a);
    }
    // Sums of what body(l, a, b) adds to a and b over the row's elements, one a load.
    template <typename Body>
    __device__ __forceinline__ void sum_each(Body&& body, double& a, double& b) const {
        using E = std::conditional_t<sizeof(In) == 2, uint16_t, float>;
        const int lane = threadIdx.x & 63, wid = wave_id();
        __syncthreads();
#pragma unroll 1
        for (int q = 0; q < kParts; ++q) {
            double x = 0.0, y = 0.0;
            for (int j = threadIdx.x + q * BLOCK; j < V; j += kMaxWaves * 64) {
                float v[1];
                load_vec<E, 1>(reinterpret_cast<const E*>(row), j, V, v);
                body(v[0], x, y);
            }
            x = wave_sum(x);
            y = wave_sum(y);
            if (lane == 0) {
                sm.red[0][wid + q * kWaves] = x;
                sm.red[1][wid + q * kWaves] = y;
            }
        }
        __syncthreads();
        a = b = 0.0;
        for (int w = 0; w < kMaxWaves; ++w) {
            a += sm.red[0][w];
            b += sm.red[1][w];
        }
        a = uniform(a);
        b = uniform(b);
    }
    __device__ __forceinline__ float block_max(float v) const {
        v = wave_max(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sm.redf[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) v = fmaxf(v, sm.redf[w]);
        return uniform(v);
    }
    __device__ __forceinline__ void range(uint32_t& lo, uint32_t& hi) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        for (int o = 32; o; o >>= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
        }
        __syncthreads();
        if (lane == 0) {
            sm.redk[0][wid] = lo;
            sm.redk[1][wid] = hi;
        }
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            lo = min(lo, sm.redk[0][w]);
            hi = max(hi, sm.redk[1][w]);
        }
    }

    // Maximum and number of the row's finite elements; false where the row has a NaN, a
    // +inf or no finite element.
    __device__ __forceinline__ bool statistics(int& n) {
        float mx = -INFINITY;
        int cnt = 0, bad = 0;
        sweep<false>([&](const float(&v)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                mx = fmaxf(mx, v[e]);
                cnt += v[e] > -INFINITY;
                bad |= !(v[e] < INFINITY);
            }
        }, [](int) {});
        mx = block_max(mx);
        const bool any_bad = __syncthreads_or(bad);
        double x = 0.0, y = 0.0;
        int z = 0;
        sum2(x, y, cnt, z);
        n = cnt;
        m = mx;
        md = uniform((double)mx);
        return !any_bad && n > 0;
    }

    // The first histogram bin (bins run from the highest logits down) at which `before` plus
    // the bins' sum reaches `target`; the last bin with something in it where none does.
    __device__ __forceinline__ int crossing(double before, double target) const {
        constexpr int PER = kBins / 64;
        __syncthreads();
        if (threadIdx.x < 64) {
            const int lane = threadIdx.x;
            double own = 0.0;
            for (int i = 0; i < PER; ++i) own += (double)sm.hist[lane * PER + i];
            const double incl = before + wave_incl_scan(own, lane);
            const uint64_t some = __ballot(own > 0.0);
            const uint64_t hit = __ballot(own > 0.0 && incl >= target);
            const int L = hit ? __ffsll((unsigned long long)hit) - 1 : some ? 63 - __clzll((long long)some) : 0;
            if (lane == L) {
                double s = incl - own;
                int at = 0;
                for (int i = 0; i < PER; ++i) {
                    const double h = (double)sm.hist[lane * PER + i];
                    if (h > 0.0) {
                        at = lane * PER + i;
                        s += h;
                        if (s >= target) break;
                    }
                }
                sm.bin = at;
            }
        }
        __syncthreads();
        return sm.bin;
    }

    // The cut at which the order's prefix reaches `target`, its number of elements (MASS
    // false) or its mass, known to lie among the keys from lo to hi, with `above` of the
    // target's units above them.  Bins of a histogram narrow the range until one value is
    // left; the histogram's 32-bit sums, whose order is not fixed, only say where to look.  The
    // mass above a bin and the mass down to its end are summed in fp64 over the same elements
    // in the same order as the next bin's, so that each is the other to the last bit and one
    // bin alone has the target between the two, wherever the search began.  `total_mass`: of
    // the prefix, where wanted.
    template <bool MASS>
    __device__ __forceinline__ Ties select(double target, uint32_t lo, uint32_t hi, double above, bool want_mass,
                                           double& total_mass) const {
        const int tid = threadIdx.x;
        for (;;) {
            const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
            __syncthreads();
            for (int i = tid; i < kBins; i += BLOCK) sm.hist[i] = 0.0f;
            __syncthreads();
            each([&](float l, int) {
                const uint32_t k = key_of(l);
                if (l > -INFINITY && k >= lo && k <= hi)
                    unsafeAtomicAdd(&sm.hist[(hi - k) >> shift], MASS ? (float)mass(l) : 1.0f);
            });
            int bin = crossing(above, target);
            double a, end, mass_a, mass_end;
            int na, nin;
            uint32_t kmin, kmax;
            int turned = 0;   // which way the search has gone
            for (;;) {
                // what lies above the bin, what down to its end, and the range of the keys in it
                na = nin = 0;
                kmin = ~0u;
                kmax = 0u;
                sum_each([&](float l, double& up, double& upto) {
                    const uint32_t k = key_of(l);
                    if (!(l > -INFINITY) || k < lo) return;
                    const int b = k > hi ? -1 : (int)((hi - k) >> shift);
                    if (b > bin) return;
                    const double w = MASS || want_mass ? mass(l) : 0.0;
                    upto += w;
                    if (b < bin) {
                        ++na;
                        up += w;
                    } else {
                        ++nin;
                        kmin = min(kmin, k);
                        kmax = max(kmax, k);
                    }
                }, mass_a, mass_end);
                double none = 0.0, none2 = 0.0;
                sum2(none, none2, na, nin);
                range(kmin, kmax);
                a = MASS ? mass_a : (double)na;
                end = MASS ? mass_end : (double)na + (double)nin;
                // the 32-bit sums may have named a neighbour of the bin
                if (MASS && a >= target && turned <= 0) {
                    int b = bin - 1;
                    while (b > 0 && sm.hist[b] == 0.0f) --b;
                    if (b >= 0 && sm.hist[b] != 0.0f) {
                        bin = b;
                        turned = -1;
                        continue;
                    }
                }
                if (MASS && end < target && turned >= 0) {
                    int b = bin + 1;
                    while (b < kBins && sm.hist[b] == 0.0f) ++b;
                    if (b < kBins) {
                        bin = b;
                        turned = 1;
                        continue;
                    }
                }
                break;
            }
            above = a;
            lo = kmin;
            hi = kmax;
            if (lo >= hi) {
                // nin equal values: how many of them are kept
                const float tau = value_of(lo);
                const double w = mass(tau);
                const int keep = MASS ? ties_for(target - above, w, nin) : (int)(target - above);
                total_mass = mass_a + (double)keep * w;
                return {tau, keep, nin};
            }
        }
    }

    // How many of n elements of mass w reach `rest`.
    __device__ __forceinline__ static int ties_for(double rest, double w, int n) {
        const double t = w > 0.0 ? ceil(rest / w) : (double)n;
        return t < 1.0 ? 1 : t > (double)n ? n : (int)t;
    }

    // How often each bf16 value occurs, and the row's maximum.  Whether the counts say all
    // that a cut needs (values outside the bins' range, unless they have no mass, make the row
    // one for the search above); a NaN or a +inf sets `bad`.
    __device__ __forceinline__ bool count_values(bool& bad) {
        const int tid = threadIdx.x, lane = tid & 63, wid = wave_id();
        __syncthreads();   // few() may have left a wave reading the sample, which lies here
        for (int i = tid; i < kValueBins / 4; i += BLOCK) reinterpret_cast<uint4*>(sm.count)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        bool mine = false;
        sweep_raw<false>([&](const typename W::raw& t, int) {
            if constexpr (VEC == 8) {
                const uint32_t w[4] = {t.x, t.y, t.z, t.w};
                u16x2 at[4], most = {0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    at[q] = bin_bytes(w[q]);
                    most = __builtin_elementwise_max(most, at[q]);
                }
                char* base = reinterpret_cast<char*>(sm.count);
                auto add = [&](int byte) {
                    uint32_t* at = reinterpret_cast<uint32_t*>(base + byte);
                    __hip_atomic_fetch_add(at, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                };
                // the last bin's count is not used, and masked rows would crowd it; a negative
                // NaN is in it, a positive one and +inf make the top bin, and the row one for
                // the search
                if (__ballot(most.x == 4 * kLastBin || most.y == 4 * kLastBin) == 0) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        add(at[q].x);
                        add(at[q].y);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (at[q].x < 4 * kLastBin) add(at[q].x);
                        if (at[q].y < 4 * kLastBin) add(at[q].y);
                        mine |= w[q] > 0xff80ffffu || (w[q] & 0xffffu) > 0xff80u;
                    }
                }
            }
        }, [](int) {});
        bad = __syncthreads_or(mine);
        static_assert(kGroups % kWaves == 0, "as many groups a wave");
#pragma unroll 4
        for (int i = 0; i < kGroups / kWaves; ++i) {
            const int g = wid + i * kWaves, b = g * 64 + lane;
            const int n = wave_sum_i(b < kLastBin ? (int)sm.count[b] : 0);
            if (lane == 0) sm.group_count[g] = n;
        }
        __syncthreads();
        // the highest value: the first bin that is not empty
        int first = kValueBins;
#pragma unroll
        for (int q = kLaneGroups - 1; q >= 0; --q)
            if (sm.group_count[lane * kLaneGroups + q]) first = lane * kLaneGroups + q;
        const uint64_t some = __ballot(first < kValueBins);
        if (some) {
            const int g = __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)some) - 1);
            const uint64_t in = __ballot(g * 64 + lane < kLastBin && sm.count[g * 64 + lane]);
            first = g * 64 + __ffsll((unsigned long long)in) - 1;
        }
        first = __builtin_amdgcn_readfirstlane(first);
        m = uniform(bin_value(first));
        md = uniform((double)m);
        top = first;
        return first > kTopBin && first < kLastBin && (md + 1020.0) * c > 150.0 &&
               (sm.count[kZeroBin - 1] | sm.count[kZeroBin + 1]) == 0;
    }
    int top = 0;   // the bin of the row's highest value

    // The group of 64 bins in which a running sum over the groups reaches `target`, or the last
    // with anything in it; `base` is the sum before it, `base2` that of another array.
    // Every wave finds the same.
    template <typename A, typename B>
    __device__ __forceinline__ static int reach_group(const A* sums, const B* others, double target, double& base,
                                                      double& base2) {
        const int lane = threadIdx.x & 63;
        double a[kLaneGroups], b[kLaneGroups], own = 0.0, own2 = 0.0;
#pragma unroll
        for (int q = 0; q < kLaneGroups; ++q) {
            a[q] = (double)sums[lane * kLaneGroups + q];
            b[q] = (double)others[lane * kLaneGroups + q];
            own += a[q];
            own2 += b[q];
        }
        const double incl = base + wave_incl_scan(own, lane), incl2 = base2 + wave_incl_scan(own2, lane);
        const uint64_t hit = __ballot(own > 0.0 && incl >= target), some = __ballot(own > 0.0);
        const int L = hit ? __ffsll((unsigned long long)hit) - 1 : some ? 63 - __clzll((long long)some) : 0;
        double c = incl - own, c2 = incl2 - own2, at = c, at2 = c2;
        int g = lane * kLaneGroups;
        bool found = false;
#pragma unroll
        for (int q = 0; q < kLaneGroups; ++q) {
            if (a[q] > 0.0 && !found) {
                g = lane * kLaneGroups + q;
                at = c;
                at2 = c2;
                found = c + a[q] >= target;
            }
            c += a[q];
            c2 += b[q];
        }
        base = readlane_d(at, L);
        base2 = readlane_d(at2, L);
        return __builtin_amdgcn_readlane(g, L);
    }

    // The value at which the counts (BY_MASS: the masses) of the row's values reach `target`,
    // how many of the elements equal to it are kept, and the prefix's mass.
    template <bool BY_MASS>
    __device__ __forceinline__ Ties locate(double target, bool want_mass, double& prefix) const {
        const int lane = threadIdx.x & 63;
        double base = 0.0, base2 = 0.0;
        const int g = BY_MASS ? reach_group(sm.group_sum, sm.group_sum, target, base, base2)
                              : reach_group(sm.group_count, sm.group_sum, target, base, base2);
        const int b = g * 64 + lane;
        const int n = b < kLastBin ? (int)sm.count[b] : 0;
        const double w = n && (BY_MASS || want_mass) ? mass(bin_value(b)) : 0.0;
        const double in_m = (BY_MASS ? base : base2) + wave_incl_scan((double)n * w, lane);
        const double in = BY_MASS ? in_m : base + wave_incl_scan((double)n, lane);
        const bool real = n > 0 && (!BY_MASS || w > 0.0);
        const uint64_t over = __ballot(real && in >= target), any = __ballot(real);
        const int L = over ? __ffsll((unsigned long long)over) - 1 : any ? 63 - __clzll((long long)any) : 0;
        const double above_m = in_m - (double)n * w;
        const int keep = BY_MASS ? ties_for(target - above_m, w, n) : (int)(target - (in - (double)n));
        prefix = readlane_d(above_m + (double)keep * w, L);
        return {readlane_f(bin_value(b), L), __builtin_amdgcn_readlane(keep, L), __builtin_amdgcn_readlane(n, L)};
    }

    // The cut of top_k and top_p from the counts of a row's values.  Where it falls among the
    // values below all bins, the search ends it, whose histogram lies over the counts: nothing
    // reads those of a cut down there.  With min_p (`floored`) there is no such cut: its floor
    // is above -1020 (min_p is at least 2^-149, and count_values has seen 2^-150 there) and the
    // counts say what it keeps, so the elements below the bins need no order.
    __device__ __forceinline__ Ties cut_values(int top_k, double top_p, bool floored) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        const bool want_mass = top_p < 1.0;
        // lane i: the count of the wave's i-th group, and then its mass
        double held = 0.0;
        uint64_t some = __ballot(want_mass && lane < kGroups / kWaves && sm.group_count[wid + min(lane, kGroups / kWaves - 1) * kWaves]);
        for (; some; some &= some - 1) {
            const int i = __ffsll((unsigned long long)some) - 1, b = (wid + i * kWaves) * 64 + lane;
            const int n = b < kLastBin ? (int)sm.count[b] : 0;
            const double t = wave_sum(n ? (double)n * mass(bin_value(b)) : 0.0);
            if (lane == i) held = t;
        }
        if (lane < kGroups / kWaves) sm.group_sum[wid + lane * kWaves] = held;
        __syncthreads();
        int all = 0;
        double all_m = 0.0;
#pragma unroll
        for (int q = 0; q < kLaneGroups; ++q) {
            all += sm.group_count[lane * kLaneGroups + q];
            all_m += sm.group_sum[lane * kLaneGroups + q];
        }
        all = wave_sum_i(all);
        all_m = wave_sum(all_m);
        Ties cut{-INFINITY, 0, 0};
        if (top_k > all) {
            // into the last bin, which holds -inf too; it has no mass, so top_p cuts above it
            int below = 0, none = 0;
            double x = 0.0, y = 0.0;
            if (!want_mass && !floored) {
                each([&](float l, int) { below += l > -INFINITY && l <= bin_value(kLastBin); });
                sum2(x, y, below, none);
                if (all + below > top_k)
                    cut = select<false>((double)top_k, key_of(-INFINITY) + 1, key_of(bin_value(kLastBin)), (double)all,
                                        false, x);
            }
        } else if (top_k > 0) {
            cut = locate<false>((double)top_k, want_mass, all_m);
        }
        if (!want_mass) return cut;
        double prefix;
        return locate<true>(top_p * all_m, true, prefix);
    }

    // Number of the row's elements in the bins up to `bin`.
    __device__ __forceinline__ int count_to(int bin) const {
        const int lane = threadIdx.x & 63, g = bin / 64;
        int n = lane <= bin % 64 ? (int)sm.count[g * 64 + lane] : 0;
#pragma unroll
        for (int q = 0; q < kLaneGroups; ++q)
            if (lane * kLaneGroups + q < g) n += sm.group_count[lane * kLaneGroups + q];
        return wave_sum_i(n);
    }

    // How many elements a cut from the counts keeps; -1 where they do not say.
    __device__ __forceinline__ int count_kept(const Ties& cut) const {
        if (!(cut.tau > -INFINITY)) return -1;
        const int end = bin_bytes(__float_as_uint(cut.tau) >> 16).x / 4;
        return end == kLastBin ? -1 : count_to(end) - (cut.keep < cut.all ? cut.all - cut.keep : 0);
    }

    // The index of the keep-th element equal to tau.
    __device__ __forceinline__ int tie_limit(float tau, int keep) const {
        const int lane = threadIdx.x & 63;
        int cnt = 0;
        __syncthreads();
        sweep<false>([&](const float(&v)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) cnt += v[e] == tau;
        }, [&](int s) {
            const int n = wave_sum_i(cnt);
            if (lane == 0) sm.ties[s] = n;
            cnt = 0;
        });
        return tie_place(tau, keep);
    }

    // The same from the slots' numbers of such elements (sm.ties, which then holds how many of
    // them are kept).
    __device__ __forceinline__ int tie_place(float tau, int keep) const {
        const int lane = threadIdx.x & 63;
        constexpr int SPL = kRowSlots / 64;
        __syncthreads();
        if (threadIdx.x < 64) {
            int n[SPL], own = 0;
#pragma unroll
            for (int q = 0; q < SPL; ++q) {
                n[q] = SPL * lane + q < nslots ? sm.ties[SPL * lane + q] : 0;
                own += n[q];
            }
            int before = incl_scan(own) - own, slot = -1, left = 0;
#pragma unroll
            for (int q = 0; q < SPL; ++q) {
                const int kept = max(0, min(n[q], keep - before));
                if (before < keep && before + n[q] >= keep) {
                    slot = SPL * lane + q;
                    left = keep - before;
                }
                if (SPL * lane + q < nslots) sm.ties[SPL * lane + q] = kept;
                before += n[q];
            }
            const int L = __ffsll((unsigned long long)__ballot(slot >= 0)) - 1;
            slot = __builtin_amdgcn_readlane(slot, L);
            left = __builtin_amdgcn_readlane(left, L);
            int limit = -1;
            for (int q = slot * G * UNR; q < (slot + 1) * G * UNR && limit < 0; ++q) {
                const int j = q * 64 * VEC + lane * VEC;
                float v[VEC];
                load_vec<In, VEC>(row, j, V, v);
                int eq = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) eq += v[e] == tau;
                const int incl = incl_scan(eq);
                const uint64_t hit = __ballot(incl >= left);
                if (hit) {
                    int at = -1, c2 = incl - eq;
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (v[e] == tau && ++c2 == left) at = j + e;
                    limit = __builtin_amdgcn_readlane(at, __ffsll((unsigned long long)hit) - 1);
                }
                left -= __builtin_amdgcn_readlane(incl, 63);
            }
            if (lane == 0) sm.limit = limit;
        }
        __syncthreads();
        return sm.limit;
    }
    __device__ __forceinline__ static int incl_scan(int v) {
        const int lane = threadIdx.x & 63;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(v, o);
            if (lane >= o) v += x;
        }
        return v;
    }

    // The slots' sums of all masses, against the highest element of the row's sample; or, where
    // the row's maximum is far above it, against that.  False where the row has no
    // distribution.
    __device__ __forceinline__ bool slot_masses() {
        const int lane = threadIdx.x & 63;
        float v[kSampleLane];
        load_sample(v);
        float mx = sample_max(v);
        for (int attempt = 0;; ++attempt) {
            // a NaN or a +inf here shows in the pass too
            md = uniform(mx > -INFINITY && mx < INFINITY ? (double)mx : 0.0);
            double a = 0.0;
            int n = 0, bad = 0, none = 0;
            sweep<true>([&](const float(&t)[VEC], int) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    mx = fmaxf(mx, t[e]);
                    n += t[e] > -INFINITY;
                    bad |= !(t[e] < INFINITY);
                    a += mass(t[e]);
                }
            }, [&](int s) {
                const double t = wave_sum(a);
                if (lane == 0) sm.slot[s] = t;
                a = 0.0;
            });
            double x = 0.0, y = 0.0;
            sum2(x, y, n, none);
            finite = n;
            m = block_max(mx);
            const bool any_bad = __syncthreads_or(bad);
            if (any_bad || n == 0) return false;
            if (attempt == 1 || fabs((double)m - md) * c < 500.0) return true;
            mx = m;   // the next pass's reference
        }
    }
    int finite = 0;

    // ---- rows whose kept elements are few, or whose values are many

    // The row's sample: the first elements of eight slots spread over it, whatever the
    // workgroup's size, so that what is relative to it does not depend on that; 16 elements
    // for each lane of the first eight waves.  The first run begins the row: a vocabulary whose
    // likely tokens crowd there is over-counted, and few() gives up on it (below).
    static constexpr int kSampleSlots = 8, kSampleVecs = VEC == 4 ? 4 : 2;
    static constexpr int kSampleLane = kSampleVecs * VEC, kSample = kSampleSlots * 64 * kSampleLane;
    __device__ __forceinline__ void load_sample(float (&v)[kSampleLane]) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
#pragma unroll
        for (int e = 0; e < kSampleLane; ++e) v[e] = -INFINITY;
        if (wid < kSampleSlots) {
            const int j = (int)((uint32_t)wid * (uint32_t)nslots / kSampleSlots) * G * CHUNK + lane * VEC;
            typename W::raw t[kSampleVecs];
#pragma unroll
            for (int u = 0; u < kSampleVecs; ++u) t[u] = W::template load_full<false>(row, min(j + u * 64 * VEC, V - VEC));
#pragma unroll
            for (int u = 0; u < kSampleVecs; ++u) {
                float x[VEC];
                cut_off(t[u], j + u * 64 * VEC);
                W::unpack(t[u], x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u * VEC + e] = x[e];
            }
        }
    }

    // The sample, the highest of its elements (finite, or the answer is false) and their
    // histogram below it.
    __device__ __forceinline__ bool take_sample(float (&v)[kSampleLane], float& ref) const {
        const int tid = threadIdx.x;
        load_sample(v);
        __syncthreads();
        for (int i = tid; i < kBins / 4; i += BLOCK) reinterpret_cast<uint4*>(sm.sample)[i] = make_uint4(0, 0, 0, 0);
        ref = sample_max(v);
        if (!(ref > -INFINITY && ref < INFINITY)) return false;
#pragma unroll
        for (int e = 0; e < kSampleLane; ++e) {
            const int b = sample_bin(ref, v[e]);
            if (b < kBins - 1) atomicAdd(&sm.sample[b], 1u);
        }
        __syncthreads();
        return true;
    }
    // Bins below ref; what is above it is in the first, what is far below in the last.
    __device__ __forceinline__ static int sample_bin(float ref, float l) {
        return (int)fminf(fmaxf((ref - l) * kSampleBins, 0.0f), (float)(kBins - 1));
    }
    __device__ __forceinline__ float sample_max(const float (&v)[kSampleLane]) const {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < kSampleLane; ++e) mx = fmaxf(mx, v[e]);
        return block_max(mx);
    }

    // The bin up to which a histogram below the sample's maximum counts `rank` elements; the
    // last where it does not.  Every wave finds the same.
    __device__ __forceinline__ int sample_rank(const uint32_t* counts, float rank) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        constexpr int kSampleGroups = kBins / 64;
        static_assert(kSampleGroups <= 64 && kSampleGroups % kWaves == 0, "a lane a group");
#pragma unroll
        for (int i = 0; i < kSampleGroups / kWaves; ++i) {
            const int g = wid + i * kWaves, n = wave_sum_i((int)counts[g * 64 + lane]);
            if (lane == 0) sm.group_sum[g] = (double)n;
        }
        __syncthreads();
        const double own = lane < kSampleGroups ? sm.group_sum[lane] : 0.0, incl = wave_incl_scan(own, lane);
        const uint64_t hit = __ballot(incl >= (double)rank);
        if (!hit) return kBins - 1;
        const int g = __ffsll((unsigned long long)hit) - 1;
        const double in = readlane_d(incl - own, g) + wave_incl_scan((double)counts[g * 64 + lane], lane);
        return g * 64 + __ffsll((unsigned long long)__ballot(in >= (double)rank)) - 1;
    }
    // A threshold above which lie, going by the sample, `rank` of its elements; -inf where
    // there is none.
    __device__ __forceinline__ float threshold(float ref, float rank) const {
        const int at = sample_rank(sm.sample, rank);
        return at < kBins - 1 ? ref - (float)(at + 1) / kSampleBins : -INFINITY;
    }

    // Takes from the list those of its n elements that are not among its first `rank` for sure:
    // the bins' order is the elements'.  How many are left.
    __device__ __forceinline__ int trim(int n, int rank, float ref) const {
        const int tid = threadIdx.x;
        constexpr int kEach = kSorted / BLOCK;
        uint32_t* counts = reinterpret_cast<uint32_t*>(sm.sorted);
        __syncthreads();
        for (int i = tid; i < kBins / 4; i += BLOCK) reinterpret_cast<uint4*>(counts)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) sm.nlist = 0;
        __syncthreads();
        uint64_t x[kEach];
        int b[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int i = tid + q * BLOCK;
            b[q] = kBins;
            if (i >= n) continue;
            x[q] = sm.list[i];
            b[q] = sample_bin(ref, value_of(~(uint32_t)(x[q] >> 32)));
            atomicAdd(&counts[b[q]], 1u);
        }
        __syncthreads();
        const int last = sample_rank(counts, (float)rank);
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (b[q] <= last) sm.list[atomicAdd(&sm.nlist, 1)] = x[q];
        __syncthreads();
        return sm.nlist;
    }

    // Adds a vector's elements that are at least tau, if any, to the list.
    __device__ __forceinline__ void gather(const float (&v)[VEC], int j, float tau) const {
        uint64_t in[VEC], any = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            in[e] = __ballot(v[e] >= tau);
            any |= in[e];
        }
        if (any == 0) return;
        int n = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) n += __popcll(in[e]);
        int at = 0;
        if ((threadIdx.x & 63) == 0) at = atomicAdd(&sm.nlist, n);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (in[e] == 0) continue;
            const int i = at + __popcll(in[e] & __lanemask_lt());
            if (v[e] >= tau && i < kSorted) sm.list[i] = (uint64_t)~key_of(v[e]) << 32 | (uint32_t)(j + e);
            at += __popcll(in[e]);
        }
    }

    // Sums the masses of the elements marked, 64 at a time: they wait in the wave's part of
    // sm.packed until there are as many.  Where a few of a vector's lanes hold one, the
    // exponentials of the others would be computed for nothing (20 instructions each; packing
    // takes 6).  rest() sums what is left.
    struct Packed {
        float* held;
        int head = 0, tail = 0;
    };
    __device__ __forceinline__ Packed packed() const { return {sm.packed[wave_id()]}; }
    __device__ __forceinline__ void pack(const float (&v)[VEC], const bool (&in)[VEC], Packed& p, double& a) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint64_t some = __ballot(in[e]);
            if (some == 0) continue;
            if (in[e]) p.held[(p.tail + __popcll(some & __lanemask_lt())) & 127] = v[e];
            p.tail += __popcll(some);
            if (p.tail - p.head >= 64) {
                __builtin_amdgcn_wave_barrier();
                a += mass(p.held[(p.head + lane) & 127]);
                p.head += 64;
            }
        }
    }
    __device__ __forceinline__ void rest(Packed& p, double& a) const {
        const int lane = threadIdx.x & 63;
        __builtin_amdgcn_wave_barrier();
        if (lane < p.tail - p.head) a += mass(p.held[(p.head + lane) & 127]);
        p.head = p.tail;
    }

    // sm.list[0 .. n) into sm.sorted in ascending order, n <= kSorted; no two are equal.
    __device__ __forceinline__ void sort(int n) const {
        const int tid = threadIdx.x;
        __syncthreads();
        if (n <= kRanked) {
            // an element's place is the number of those below it, counted by four threads
            if (tid < 8 && tid < kSorted - n) sm.list[n + tid] = ~0ull;
            __syncthreads();
            for (int i = tid; i < 4 * n; i += BLOCK) {
                const uint64_t x = sm.list[i >> 2];
                int before = 0;
                for (int q = 2 * (i & 3); q < n; q += 8) {
                    const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(&sm.list[q]);
                    before += (y.x < x) + (y.y < x);
                }
                before += dpp_i<kDppXor1>(before);
                before += dpp_i<kDppXor2>(before);
                if ((i & 3) == 0) sm.sorted[before] = x;
            }
            __syncthreads();
            return;
        }
        const int size = n <= 1024 ? 1024 : 2048;
        for (int i = tid; i < size; i += BLOCK) sm.sorted[i] = i < n ? sm.list[i] : ~0ull;
        for (int k = 2; k <= size; k <<= 1)
            for (int j = k >> 1; j; j >>= 1) {
                __syncthreads();
                for (int p = tid; p < size / 2; p += BLOCK) {
                    const int a = 2 * p - (p & (j - 1)), b = a + j;
                    const uint64_t x = sm.sorted[a], y = sm.sorted[b];
                    if ((x > y) == ((a & k) == 0)) {
                        sm.sorted[a] = y;
                        sm.sorted[b] = x;
                    }
                }
            }
        __syncthreads();
    }
    __device__ __forceinline__ float sorted_value(int i) const { return value_of(~(uint32_t)(sm.sorted[i] >> 32)); }

    // Running sums of the masses of sm.sorted[0 .. n) into sm.running.
    __device__ __forceinline__ void prefix(int n) const {
        const int tid = threadIdx.x, lane = tid & 63, wid = wave_id();
        static_assert(BLOCK >= 512, "as many elements a thread in every workgroup");
        const int per = (n + 511) / 512;
        double own = 0.0;
        for (int q = 0; q < per; ++q)
            if (tid * per + q < n) own += mass(sorted_value(tid * per + q));
        const double incl = wave_incl_scan(own, lane);
        if (lane == 63) sm.red[0][wid] = incl;
        __syncthreads();
        double at = incl - own;
        for (int v = 0; v < wid; ++v) at += sm.red[0][v];
        for (int q = 0; q < per; ++q) {
            if (tid * per + q >= n) break;
            at += mass(sorted_value(tid * per + q));
            sm.running[tid * per + q] = at;
        }
        __syncthreads();
    }
    // The first i < n with sm.running[i] >= goal, n where there is none.
    __device__ __forceinline__ int reach_running(int n, double goal) const {
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (sm.running[mid] >= goal) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    }
    // How many of sm.sorted[0 .. n) are at least `floor`; one at least.
    __device__ __forceinline__ int above_floor(int n, float floor) const {
        int lo = 1, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (sorted_value(mid) >= floor) lo = mid + 1;
            else hi = mid;
        }
        return lo;
    }
    // Adds the masses of sm.sorted[0 .. n) to the slots' sums (CLEAR: which were none), as
    // whole numbers, so that their order does not count.  Each slot's unit goes by the largest
    // mass in it, which is between 2^51 and 2^52 of them (below the normal range, where the
    // exponent field is 0, a mass is a whole number of the smallest one): with one unit for
    // all, a slot of elements 2^-52 below the row's maximum would hold no mass, and a draw of
    // u = 0 would pass over them.
    template <bool CLEAR>
    __device__ __forceinline__ void add_to_slots(int n) const {
        const int tid = threadIdx.x;
        unsigned long long* sums = reinterpret_cast<unsigned long long*>(sm.running);
        int* field = reinterpret_cast<int*>(sums + kRowSlots);   // the largest mass's exponent field
        auto slot_of = [&](int i) { return (uint32_t)sm.sorted[i] / (uint32_t)(G * CHUNK); };
        __syncthreads();
        for (int i = tid; i < kRowSlots; i += BLOCK) {
            sums[i] = 0;
            field[i] = 0;
        }
        __syncthreads();
        double w[kSorted / BLOCK];
#pragma unroll
        for (int q = 0; q < kSorted / BLOCK; ++q) {
            const int i = tid + q * BLOCK;
            if (i >= n) break;
            w[q] = mass(sorted_value(i));
            atomicMax(&field[slot_of(i)], __double2hiint(w[q]) >> 20);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSorted / BLOCK; ++q) {
            const int i = tid + q * BLOCK;
            if (i >= n) break;
            const uint32_t at = slot_of(i);
            atomicAdd(&sums[at], (unsigned long long)(__builtin_ldexp(w[q], 1074 - field[at]) + 0.5));
        }
        __syncthreads();
        for (int i = tid; i < nslots; i += BLOCK)
            sm.slot[i] = (CLEAR ? 0.0 : sm.slot[i]) + __builtin_ldexp((double)sums[i], field[i] - 1074);
        __syncthreads();
    }

    // kTied: the cut's value is known, and how many of the elements equal to it are kept
    enum Search { kFound, kTied, kNone, kUnsettled };

    // The cut of top_k, with top_p and min_p or without, or of min_p alone, where it keeps few
    // elements, in one pass: a sample of the row gives a threshold with some more elements
    // above it, the pass lists those, and the sorted list is cut (min_p's needs no order).
    // Left unsettled where they are too many or too few.  slots: sm.slot holds what is kept.
    // 128,256 logits under top-k 50, 1 row and 512: bf16 draws 24 and 45 us (from the counts
    // of values 31 and 55), filtered rows 27 and 72 (30 and 89), fp32 draws 24 and 59 (the
    // search over keys takes 498 and 1360).  What is left to others for their number alone:
    // the threshold's margin passes kRoom from a top_k of about 560 on (V 32,000: 790), and
    // bf16 rows then take 40 and 68 us, fp32 rows under top_p too 545 and 1540.  For too few:
    // where likely tokens crowd into the first 1024, 41 and 77 us, and 513 and 1350.
    __device__ __forceinline__ Search few(int top_k, double top_p, double min_p, bool want_slots, Cut& cut,
                                          bool& slots, int& kept) {
        constexpr float kRoom = 0.5f * (float)kSorted;
        const float scale = (float)V / (float)kSample;
        if (VEC == 1 || scale < 2.0f || (float)top_k > kRoom) return kUnsettled;
        float v0[kSampleLane], ref;
        if (!take_sample(v0, ref)) return kUnsettled;
        // min_p's cut lies at or above its threshold below the sample's maximum (less what its
        // rounding may be); top_p after top_k needs all that top_k keeps
        float tau = -INFINITY;
        bool floored = false;
        if (min_p > 0.0 && (top_k == 0 || top_p == 1.0)) {
            tau = (float)((double)ref + T * log(min_p));
            tau -= 1e-6f * (fabsf(ref) + fabsf(tau));
            floored = true;
        }
        if (top_k > 0) {
            const float mean = (float)top_k / scale;
            const float t = threshold(ref, mean + 4.0f * sqrtf(mean) + 3.0f);
            floored = floored && tau >= t;
            tau = fmaxf(tau, t);
        }
        tau = uniform(tau);
        if (!(tau > -INFINITY)) return kUnsettled;
        int up = 0;   // elements above it, going by the sample
#pragma unroll
        for (int e = 0; e < kSampleLane; ++e) up += v0[e] >= tau;
        double x = 0.0, y = 0.0;
        int bad = 0;
        if (threadIdx.x == 0) sm.nlist = 0;
        sum2(x, y, up, bad);
        if ((float)up * scale > kRoom) return kUnsettled;
        sweep<true>([&](const float(&v)[VEC], int j) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) bad |= !(v[e] < INFINITY);
            gather(v, j, tau);
        }, [](int) {});
        if (__syncthreads_or(bad)) return kNone;
        int n = sm.nlist;
        if (n > kSorted || n < 1 || (n < top_k && !floored)) return kUnsettled;
        if (top_k == 0) {   // no order is needed
            uint32_t lo = ~0u, hi = 0u;
            for (int i = threadIdx.x; i < n; i += BLOCK) hi = max(hi, ~(uint32_t)(sm.list[i] >> 32));
            range(lo, hi);
            m = uniform(value_of(hi));
            md = uniform((double)m);
            cut = Cut{min_floor(min_p), INT_MAX};
            const uint32_t last = ~key_of(cut.tau);
            kept = bad = 0;
            for (int i = threadIdx.x; i < n; i += BLOCK) {
                const uint64_t e = sm.list[i];
                const bool in = (uint32_t)(e >> 32) <= last;
                kept += in;
                sm.sorted[i] = in ? e : (uint64_t)~key_of(-INFINITY) << 32 | (uint32_t)e;
            }
            sum2(x, y, kept, bad);
            slots = true;
            add_to_slots<true>(n);
            return kFound;
        }
        if (n > kRanked) n = trim(n, top_k, ref);
        sort(n);
        m = uniform(sorted_value(0));
        md = uniform((double)m);
        int keep = min(n, top_k);
        if (top_p < 1.0) {
            prefix(keep);
            keep = min(keep, reach_running(keep, top_p * sm.running[keep - 1]) + 1);
        }
        if (min_p > 0.0) keep = above_floor(keep, min_floor(min_p));
        cut = Cut{sorted_value(keep - 1), (int)(uint32_t)sm.sorted[keep - 1]};
        kept = keep;
        slots = want_slots;
        if (want_slots) add_to_slots<true>(keep);
        return kFound;
    }

    // The cut of top_p alone, or of a top_k that keeps many elements: a histogram over linear
    // bins below the maximum says which bin the cut falls into, and a second pass sums what
    // lies above the bin and lists what is in it.  Left unsettled where that is too much to be
    // sorted and not all one value (128,256 fp32 logits under top-p, 1 row and 512: 75 and
    // 154 us; the search over keys takes 451 and 1083), or the histogram's masses (whole numbers of 2^-40; sums of
    // floats take ten times as long in LDS) named a neighbour of the bin.  slots: sm.slot
    // holds what is kept.
    __device__ __forceinline__ Search search(int top_k, double top_p, double min_p, bool want_slots, Cut& cut,
                                             Ties& ties, bool& slots, int& kept) {
        const int tid = threadIdx.x, lane = tid & 63;
        const bool by_mass = top_k == 0;
        if (!by_mass && top_p < 1.0) return kUnsettled;
        float v0[kSampleLane];
        load_sample(v0);
        float ref = sample_max(v0);
        if (!(ref > -INFINITY && ref < INFINITY)) return kUnsettled;
        int bin = 0;
        double before = 0.0, target = 0.0;
        for (;;) {
            md = uniform((double)ref);
            __syncthreads();
            for (int i = tid; i < kLinearBins / 2; i += BLOCK) reinterpret_cast<ulonglong2*>(sm.bins)[i] = make_ulonglong2(0, 0);
            __syncthreads();
            float mx = -INFINITY;
            double a = 0.0, parts[kParts] = {};
            int n = 0, bad = 0;
            auto add = [&](float l, uint64_t q) {
                atomicAdd(reinterpret_cast<unsigned long long*>(&sm.bins[linear_bin(l, ref)]), (unsigned long long)q);
            };
            if (by_mass) {
                sweep<false>([&](const float(&v)[VEC], int) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        mx = fmaxf(mx, v[e]);
                        bad |= !(v[e] < INFINITY);
                        const double w = mass(v[e]);
                        a += w;
                        // the low bits of 2^52 + w 2^40 are the mass in its units
                        add(v[e], __double_as_longlong(fma(w, 1.0 / kMassUnit, 0x1p52)) & 0xfffffffffffffull);
                    }
                }, [&](int s) {
                    parts[s / kWaves % kParts == 0 ? 0 : kParts - 1] += a;
                    a = 0.0;
                });
            } else {
                sweep<false>([&](const float(&v)[VEC], int) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        mx = fmaxf(mx, v[e]);
                        bad |= !(v[e] < INFINITY);
                        n += v[e] > -INFINITY;
                        if (linear_bin(v[e], ref) < kLinearBins - 1) add(v[e], 1);
                    }
                }, [](int) {});
            }
            if (by_mass) {
                a = sum_parts(parts);
            } else {
                double y = 0.0;
                int none = 0;
                sum2(a, y, n, none);
            }
            m = block_max(mx);
            if (__syncthreads_or(bad)) return kNone;
            if (!by_mass) md = uniform((double)m);
            if (!by_mass && top_k >= n) {
                cut = Cut{-INFINITY, -1};
                slots = false;
                return kFound;
            }
            // the units' 52 bits hold masses below 2^12 (thousands of them in one bin pass its
            // 64 bits, and the bin found may be any: the second pass, which sums anew, says so)
            if (by_mass && ((double)m - md) * c > 10.0) {
                ref = m;
                continue;
            }
            target = by_mass ? top_p * a : (double)top_k;
            bin = reach(target, by_mass ? kMassUnit : 1.0, before);
            if (bin < 0) return kUnsettled;
            break;
        }
        __syncthreads();
        if (tid == 0) sm.nlist = 0;
        __syncthreads();
        double a = 0.0, y = 0.0;
        int above = 0, none = 0;
        Packed held = packed();
        sweep<true>([&](const float(&v)[VEC], int j) {
            float in[VEC];
            bool up[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int b = linear_bin(v[e], ref);
                in[e] = b == bin && v[e] > -INFINITY ? v[e] : -INFINITY;
                up[e] = by_mass && b < bin;
                above += up[e];
            }
            pack(v, up, held, a);
            gather(in, j, -FLT_MAX);
        }, [&](int s) {
            if (by_mass) {
                rest(held, a);
                const double t = wave_sum(a);
                if (lane == 0) sm.slot[s] = t;
                a = 0.0;
            }
        });
        sum2(a, y, above, none);
        const int n = sm.nlist;
        if (n < 1) return kUnsettled;
        double total = 0.0;
        if (by_mass) {
            for (int s = lane; s < nslots; s += 64) total += sm.slot[s];
            total = wave_sum(total);
            if (total >= target) return kUnsettled;
        }
        if (n > kSorted) {
            uint32_t lo = ~0u, hi = 0u;
            each([&](float l, int) {
                if (l > -INFINITY && linear_bin(l, ref) == bin) {
                    lo = min(lo, key_of(l));
                    hi = max(hi, key_of(l));
                }
            });
            range(lo, hi);
            if (lo != hi) return kUnsettled;
            const double w = mass(value_of(lo));
            if (by_mass && total + (double)n * w < target) return kUnsettled;
            ties = Ties{value_of(lo), by_mass ? ties_for(target - total, w, n) : top_k - (int)before, n};
            return kTied;
        }
        sort(n);
        int keep;
        if (by_mass) {
            prefix(n);
            keep = reach_running(n, target - total) + 1;
        } else {
            keep = top_k - (int)before;
        }
        if (keep < 1 || keep > n) return kUnsettled;
        cut = Cut{sorted_value(keep - 1), (int)(uint32_t)sm.sorted[keep - 1]};
        kept = by_mass ? keep + above : top_k;
        slots = want_slots && by_mass && !(min_p > 0.0 && min_floor(min_p) > cut.tau);
        if (slots) add_to_slots<false>(keep);
        return kFound;
    }
    __device__ __forceinline__ static int linear_bin(float l, float ref) {
        // 2^23 and a whole number: the number is in the low bits
        const float b = fmaf(ref - l, kBinsPerUnit, 0x1p23f + kRefBin);
        return (int)(__float_as_uint(fminf(fmaxf(b, 0x1p23f), 0x1p23f + (float)(kLinearBins - 1))) & (kLinearBins - 1));
    }

    // The bin of sm.bins in which their running sum, in `unit`s, reaches `target` and what lies
    // above it; -1 where it does not.
    __device__ __forceinline__ int reach(double target, double unit, double& before) const {
        const int lane = threadIdx.x & 63, wid = wave_id();
        constexpr int kLinearGroups = kLinearBins / 64;
        static_assert(kLinearGroups == 64, "a lane a group");
#pragma unroll
        for (int i = 0; i < kLinearGroups / kWaves; ++i) {
            const int g = wid + i * kWaves;
            const double t = wave_sum((double)sm.bins[g * 64 + lane]);
            if (lane == 0) sm.group_sum[g] = t * unit;
        }
        __syncthreads();
        const double own = sm.group_sum[lane], incl = wave_incl_scan(own, lane);
        const uint64_t hit = __ballot(own > 0.0 && incl >= target);
        if (!hit) return -1;
        const int g = __ffsll((unsigned long long)hit) - 1;
        const double h = (double)sm.bins[g * 64 + lane] * unit;
        const double inc = readlane_d(incl - own, g) + wave_incl_scan(h, lane);
        const uint64_t over = __ballot(h > 0.0 && inc >= target), any = __ballot(h > 0.0);
        const int L = over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll((long long)any);
        before = readlane_d(inc - h, L);
        return g * 64 + L;
    }

    // The lowest value of the row's type with mass at least min_p: l >= m + T ln(min_p).
    __device__ __forceinline__ float min_floor(double min_p) const {
        const double t = (double)m + T * log(min_p);
        float f = (float)t;
        if ((double)f < t) f = value_of(key_of(f) + 1);
        if (sizeof(In) == 2) {
            const uint32_t b = __float_as_uint(f);
            f = __uint_as_float((b & 0xffff0000u) + ((b & 0xffffu) && !(b >> 31) ? 0x10000u : 0u));
        }
        return f;
    }

    // The slots' sums of what a cut keeps, and how many elements that is: those of a list,
    // where they fit one; else from a table of the masses of the values above the cut.
    // `partial`: the elements equal to the cut's value are counted by slot instead.  False
    // where the table has no room for all values.
    __device__ __forceinline__ bool table_masses(const Ties& cut, bool partial, int& n) const {
        const int tid = threadIdx.x, lane = tid & 63;
        if constexpr (VEC == 8) {
            const int kept = count_kept(cut);
            const int end = bin_bytes(__float_as_uint(cut.tau) >> 16).x / 4;
            if (kept < 0 || end - top + 2 > kValueBins / 2) return false;
            const int all = kept + (partial ? cut.all - cut.keep : 0);
            n = kept;
            // words from the cut's up, as signed numbers, are the values above it if that is
            // not negative
            const int32_t tau_word = (int32_t)__float_as_uint(cut.tau) >> 16;
            __syncthreads();
            if (all <= kSorted && cut.tau > 0.0f) {
                if (tid == 0) sm.nlist = 0;
                for (int s = tid; s < nslots; s += BLOCK) sm.ties[s] = 0;
                __syncthreads();
                sweep_raw<true>([&](const typename W::raw& t, int j) {
                    i16x2 most = __builtin_bit_cast(i16x2, t.x);
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(i16x2, t.y));
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(i16x2, t.z));
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(i16x2, t.w));
                    if (__ballot(most.x >= tau_word || most.y >= tau_word) == 0) return;
                    float v[VEC];
                    W::unpack(t, v);
                    gather(v, j, cut.tau);
                }, [](int) {});
                __syncthreads();
                for (int i = tid; i < all; i += BLOCK) {
                    // a tie that may be dropped has no mass in the sums
                    const uint64_t x = sm.list[i];
                    const bool tie = partial && (uint32_t)(x >> 32) == ~key_of(cut.tau);
                    if (tie) atomicAdd(&sm.ties[(uint32_t)x / (uint32_t)(G * CHUNK)], 1);
                    sm.sorted[i] = tie ? (uint64_t)~key_of(-INFINITY) << 32 | (uint32_t)x : x;
                }
                add_to_slots<true>(all);
                return true;
            }
            for (int i = tid; i <= end - top + 1; i += BLOCK)
                sm.table[i] = i > end - top || (partial && i == end - top) ? 0.0 : mass(bin_value(top + i));
            __syncthreads();
            const char* base = reinterpret_cast<const char*>(sm.table) - top * 8;
            const uint16_t last = (uint16_t)(end * 4 + 4), at_cut = (uint16_t)(end * 4);
            const u16x2 lasts = {last, last};
            double a = 0.0;
            int ties = 0;
            sweep_raw<true>([&](const typename W::raw& t, int) {
                const uint32_t w[4] = {t.x, t.y, t.z, t.w};
                u16x2 at[4];
                u16x2 lowest = lasts;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    at[q] = __builtin_elementwise_min(bin_bytes(w[q]), lasts);
                    lowest = __builtin_elementwise_min(lowest, at[q]);
                }
                if (__ballot(lowest.x < last || lowest.y < last) == 0) return;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    a += *reinterpret_cast<const double*>(base + 2 * at[q].x);
                    a += *reinterpret_cast<const double*>(base + 2 * at[q].y);
                    if (partial) ties += (at[q].x == at_cut) + (at[q].y == at_cut);
                }
            }, [&](int s) {
                const double t = wave_sum(a);
                const int nt = partial ? wave_sum_i(ties) : 0;
                if (lane == 0) {
                    sm.slot[s] = t;
                    sm.ties[s] = nt;
                }
                a = 0.0;
                ties = 0;
            });
            __syncthreads();
            return true;
        }
        return false;
    }

    // Of the listed elements of a filtered row, all equal, the first `keep` stay; the others
    // become -inf.  Those of the slot that the last kept one is in are counted among each other.
    __device__ __forceinline__ void drop_ties(int keep, uint16_t* out) const {
        const int tid = threadIdx.x, lane = tid & 63;
        constexpr int SPL = kRowSlots / 64;
        int32_t* part = sm.equal + kListed;
        __syncthreads();
        const int n = sm.nlist;
        for (int s = tid; s < kRowSlots; s += BLOCK) sm.ties[s] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += BLOCK) atomicAdd(&sm.ties[sm.equal[i] / (G * CHUNK)], 1);
        __syncthreads();
        if (tid < 64) {
            int cnt[SPL], own = 0;
#pragma unroll
            for (int q = 0; q < SPL; ++q) own += cnt[q] = sm.ties[SPL * lane + q];
            int before = incl_scan(own) - own;
#pragma unroll
            for (int q = 0; q < SPL; ++q) {
                const int left = keep - before;      // -1: the slot's all stay
                sm.ties[SPL * lane + q] = left >= cnt[q] ? -1 : max(left, 0);
                before += cnt[q];
            }
            if (lane == 0) sm.nlist = 0;
        }
        __syncthreads();
        for (int i = tid; i < n; i += BLOCK) {
            const int j = sm.equal[i], left = sm.ties[j / (G * CHUNK)];
            if (left == 0) out[j] = 0xff80;
            else if (left > 0) part[atomicAdd(&sm.nlist, 1)] = j;
        }
        __syncthreads();
        const int m = sm.nlist;
        for (int i = tid; i < m; i += BLOCK) {
            const int j = part[i];
            int before = 0;
            for (int q = 0; q < m; ++q) before += part[q] < j;
            if (before >= sm.ties[j / (G * CHUNK)]) out[j] = 0xff80;
        }
    }
    static constexpr int kListed = 4096;

    // The token of uniform u: the first index at which the kept masses' running sum exceeds
    // u times their total.  One wave; every lane returns it, and its logit.
    __device__ __forceinline__ int draw(float u, double total, const Cut& cut, float& logit) const {
        const int lane = threadIdx.x & 63;
        constexpr int PER = kRowSlots / 64;
        const double thr = (double)u * total;
        double t[PER], own = 0.0;
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int s = PER * lane + q;
            t[q] = s < nslots ? sm.slot[s] : 0.0;
            own += t[q];
        }
        const double incl = wave_incl_scan(own, lane);
        const uint64_t hit = __ballot(own > 0.0 && incl > thr);
        const uint64_t some = __ballot(own > 0.0);
        const int L = hit ? __ffsll((unsigned long long)hit) - 1 : 63 - __clzll((long long)some);
        int slot = 0;
        double base = 0.0;
        {
            double c2 = incl - own;
            bool found = false;
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                if (t[q] > 0.0 && !found) {
                    slot = PER * lane + q;
                    base = c2;
                    found = c2 + t[q] > thr;
                }
                c2 += t[q];
            }
        }
        slot = __builtin_amdgcn_readlane(slot, L);
        base = readlane_d(base, L);
        int last = 0;
        float last_l = 0.0f;
        typename W::raw held[UNR];
        for (int q = 0; q < G * UNR; ++q) {
            if (q % UNR == 0) {
#pragma unroll
                for (int u = 0; u < UNR; ++u)
                    held[u] = W::template load_full<false>(row, min((slot * G * UNR + q + u) * 64 * VEC + lane * VEC, V - VEC));
            }
            const int j = (slot * G * UNR + q) * 64 * VEC + lane * VEC;
            typename W::raw x = held[0];
#pragma unroll
            for (int u = 0; u + 1 < UNR; ++u) held[u] = held[u + 1];
            cut_off(x, j);
            float v[VEC];
            W::unpack(x, v);
            double w[VEC], sum = 0.0;
            int at = -1;
            float l = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                w[e] = j + e < V && cut.keeps(v[e], j + e) ? mass(v[e]) : 0.0;
                sum += w[e];
                if (w[e] > 0.0) {
                    at = j + e;
                    l = v[e];
                }
            }
            const double inc = wave_incl_scan(sum, lane);
            const uint64_t positive = __ballot(at >= 0);
            const uint64_t over = __ballot(at >= 0 && base + inc > thr);
            if (over) {
                const int H = __ffsll((unsigned long long)over) - 1;
                double c2 = base + (inc - sum);
                bool found = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    c2 += w[e];
                    if (w[e] > 0.0 && !found) {
                        at = j + e;
                        l = v[e];
                        found = c2 > thr;
                    }
                }
                logit = readlane_f(l, H);
                return __builtin_amdgcn_readlane(at, H);
            }
            if (positive) {
                const int H = 63 - __clzll((long long)positive);
                last = __builtin_amdgcn_readlane(at, H);
                last_l = readlane_f(l, H);
            }
            base += readlane_d(inc, 63);
        }
        logit = last_l;
        return last;
    }
};

// VEC logits to out[j ..), those past V left out.
template <typename In, int VEC>
__device__ __forceinline__ void store_vec(In* out, int j, int V, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        if (j >= V) return;
        if constexpr (sizeof(In) == 2) reinterpret_cast<uint16_t*>(out)[j] = (uint16_t)(__float_as_uint(v[0]) >> 16);
        else reinterpret_cast<float*>(out)[j] = v[0];
    } else if constexpr (sizeof(In) == 2) {
        u32x4 r;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            r[q] = (__float_as_uint(v[2 * q]) >> 16) | (__float_as_uint(v[2 * q + 1]) & 0xffff0000u);
        if (j + VEC <= V) *reinterpret_cast<u32x4_at2*>(out + j) = r;
        else
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j + e < V) reinterpret_cast<uint16_t*>(out)[j + e] = (uint16_t)(__float_as_uint(v[e]) >> 16);
    } else {
        u32x4 r;
#pragma unroll
        for (int q = 0; q < 4; ++q) r[q] = __float_as_uint(v[q]);
        if (j + VEC <= V) *reinterpret_cast<u32x4_at4*>(out + j) = r;
        else
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j + e < V) reinterpret_cast<float*>(out)[j + e] = v[e];
    }
}

// A vector's elements below tau (not zero) become -inf; whether one equals it.
__device__ __forceinline__ bool keep_from(uint4& t, float tau, uint16_t) {
    // bf16 words as signed numbers in the values' order: negative ones have their low bits
    // turned over
    const uint32_t b = __float_as_uint(tau) >> 16;
    const int16_t key = (int16_t)(b ^ (b & 0x8000u ? 0x7fffu : 0u));
    const i16x2 keys = {key, key}, below = {(int16_t)(key - 1), (int16_t)(key - 1)}, fifteen = {0x7fff, 0x7fff};
    u16x2 nearest = {0xffff, 0xffff};
    uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const i16x2 x = __builtin_bit_cast(i16x2, w[q]), k = x ^ ((x >> 15) & fifteen);
        const uint32_t m = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(below, k) >> 15);
        nearest = __builtin_elementwise_min(nearest, __builtin_bit_cast(u16x2, k ^ keys));
        w[q] = (w[q] & m) | (0xff80ff80u & ~m);
    }
    t = make_uint4(w[0], w[1], w[2], w[3]);
    return nearest.x == 0 || nearest.y == 0;
}
__device__ __forceinline__ bool keep_from(uint4& t, float tau, float) {
    bool tie = false;
    uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float v = __uint_as_float(w[q]);
        tie |= v == tau;
        w[q] = v >= tau ? w[q] : 0xff800000u;
    }
    t = make_uint4(w[0], w[1], w[2], w[3]);
    return tie;
}
__device__ __forceinline__ void store_raw(odd16* out, const uint4& t) {
    *reinterpret_cast<u32x4_at2*>(out) = u32x4{t.x, t.y, t.z, t.w};
}
__device__ __forceinline__ void store_raw(uint16_t* out, const uint4& t) { *reinterpret_cast<uint4*>(out) = t; }
__device__ __forceinline__ void store_raw(odd32* out, const uint4& t) {
    *reinterpret_cast<u32x4_at4*>(out) = u32x4{t.x, t.y, t.z, t.w};
}
__device__ __forceinline__ void store_raw(float* out, const uint4& t) { *reinterpret_cast<uint4*>(out) = t; }

// One workgroup a row: the cut, then the draws or the filtered row.  4 waves a SIMD: with
// room for 6 the compiler spills, and ran no faster.
template <typename In, int VEC, int BLOCK, bool FILTER>
__global__ void __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) rs_sample_kernel(const SParams P) {
    __shared__ RowSmem sm;
    constexpr int kWaves = BLOCK / 64;
    constexpr bool kCounts = VEC == 8;   // bf16 rows: counts of values
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r = blockIdx.x;
    const int64_t entry = r / P.rows_per_entry;
    const float T = P.temperatures ? P.temperatures[entry] : P.temperature;
    const float top_p = P.top_ps ? P.top_ps[entry] : P.top_p;
    const float min_p = P.min_ps ? P.min_ps[entry] : P.min_p;
    const int top_k = P.top_ks ? P.top_ks[entry] : P.top_k;
    Row<In, VEC, BLOCK> row{reinterpret_cast<const In*>(P.logits) + r * P.stride, P.V, P.G, P.nslots, 0.0f, 0.0,
                                 uniform(1.4426950408889634 / (double)T), uniform((double)T), sm};
    In* out = FILTER ? reinterpret_cast<In*>(P.out) + r * P.out_stride : nullptr;
    int status = RS_SEQ_OK;
    if (!(T > 0.0f && T < INFINITY && top_k >= 0 && top_p > 0.0f && top_p <= 1.0f && min_p >= 0.0f && min_p <= 1.0f))
        status = RS_SEQ_BAD_PARAM;
    if (!FILTER && status == RS_SEQ_OK) {
        const float u = tid < P.k ? P.u[r * P.k + tid] : 0.0f;
        if (__syncthreads_or(!(u >= 0.0f && u < 1.0f))) status = RS_SEQ_BAD_UNIFORM;
    }
    // ---- the cut: from the counts of the row's values, which are at hand then; by the search
    // over linear bins; or by the one over ranges of keys, which settles every row
    const bool filters = top_k > 0 || top_p < 1.0f || min_p > 0.0f;
    Ties ties{-INFINITY, 0, 0};
    Cut cut{-INFINITY, -1};
    bool counts = false, settled = false, slots = false;
    int kept = -1;
    if (status == RS_SEQ_OK && (filters || FILTER)) {
        bool bad = false;
        auto found = Row<In, VEC, BLOCK>::kUnsettled;
        if (top_k > 0 || (!FILTER && min_p > 0.0f && top_p == 1.0f))
            found = row.few(top_k, (double)top_p, (double)min_p, !FILTER, cut, slots, kept);
        if constexpr (kCounts) {
            if (found == Row<In, VEC, BLOCK>::kUnsettled) {
                counts = row.count_values(bad);
                if (counts && filters) ties = row.cut_values(top_k, (double)top_p, min_p > 0.0f);
            }
        }
        if (bad || found == Row<In, VEC, BLOCK>::kNone) {
            status = RS_SEQ_UNDERFLOW;
        } else if (!counts) {
            int n = 0;
            const bool cuts = top_k > 0 || top_p < 1.0f;
            if constexpr (!kCounts)
                if (cuts && found == Row<In, VEC, BLOCK>::kUnsettled) found = row.search(top_k, (double)top_p, (double)min_p, !FILTER, cut, ties, slots, kept);
            if (found == Row<In, VEC, BLOCK>::kNone) status = RS_SEQ_UNDERFLOW;
            settled = found == Row<In, VEC, BLOCK>::kFound;
            const bool tied = found == Row<In, VEC, BLOCK>::kTied;
            if (!settled && !tied && status == RS_SEQ_OK && !row.statistics(n)) status = RS_SEQ_UNDERFLOW;
            if (!settled && !tied && status == RS_SEQ_OK && cuts) {
                const uint32_t lo = key_of(-INFINITY) + 1, hi = key_of(row.m);
                double mass = 0.0;
                const bool cuts_k = top_k > 0 && top_k < n;
                if (cuts_k) ties = row.template select<false>((double)top_k, lo, hi, 0.0, top_p < 1.0f, mass);
                if (top_p < 1.0f) {
                    if (!cuts_k) {
                        double none = 0.0;
                        row.sum_each([&](float l, double& a, double&) { a += row.mass(l); }, mass, none);
                    }
                    ties = row.template select<true>((double)top_p * mass, lo, hi, 0.0, false, mass);
                }
            }
        }
        if (settled) ties = Ties{uniform(cut.tau), 0, 0};
        else cut = Cut{ties.tau, ties.tau > -INFINITY ? INT_MAX : -1};
        if (status == RS_SEQ_OK && min_p > 0.0f) {
            const float f = row.min_floor((double)min_p);
            if (f > ties.tau) {
                ties = Ties{f, 0, 0};
                cut = Cut{f, INT_MAX};
                kept = -1;
            }
        }
    }
    // ---- no filter: the slots' sums against a reference near the maximum
    double total = 0.0;
    if (status == RS_SEQ_OK && !FILTER && !filters)
        if (!row.slot_masses()) status = RS_SEQ_UNDERFLOW;
    if (status != RS_SEQ_OK) {
        if (FILTER) {
            float inf[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) inf[e] = -INFINITY;
            for (int j = tid * VEC; j < P.V; j += BLOCK * VEC) store_vec<In, VEC>(out, j, P.V, inf);
        } else if (tid < P.k) {
            P.token[r * P.k + tid] = -1;
            if (P.logprob) P.logprob[r * P.k + tid] = NAN;
        }
        if (tid == 0) {
            if (P.kept) P.kept[r] = -1;
            if (P.status) P.status[r] = status;
        }
        return;
    }
    // ---- which of the elements equal to the cut's value are kept
    const bool partial = ties.keep < ties.all;
    if (FILTER) {
        // many ties: their last index is found first; few: all are written as kept, and the
        // rest taken back
        const bool listed = counts && partial && ties.all <= row.kListed;
        if constexpr (kCounts)
            if (counts && filters) kept = row.count_kept(ties);
        if (partial && !listed) cut.limit = row.tie_limit(ties.tau, ties.keep);
        __syncthreads();
        if (tid == 0) sm.nlist = 0;
        __syncthreads();
        int n = 0, none = 0;
        auto exactly = [&](const float(&v)[VEC], int j) {
            float w[VEC];
            bool tie = false;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool k = cut.keeps(v[e], j + e);
                w[e] = k ? v[e] : -INFINITY;
                n += k;
                tie |= v[e] == ties.tau;
            }
            store_vec<In, VEC>(out, j, P.V, w);
            if (listed && tie) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (v[e] == ties.tau) sm.equal[atomicAdd(&sm.nlist, 1)] = j + e;
            }
        };
        const bool known = kept >= 0;
        if (!known || ties.tau == 0.0f) {
            row.template sweep<true>(exactly, [](int) {});
            double x = 0.0, y = 0.0;
            row.sum2(x, y, n, none);
            n -= listed ? ties.all - ties.keep : 0;
            if (!known) kept = n;
        } else {
            // vectors without an element equal to the cut's value take a comparison each, of
            // the two bf16 values of a word at once
            const bool check = listed || cut.limit != INT_MAX;
            row.template sweep_raw<true>([&](const typename Vec<In, VEC>::raw& t, int j) {
                typename Vec<In, VEC>::raw w = t;
                bool tie = false;
                if constexpr (VEC == 1) {
                    const float v = __uint_as_float(t);
                    tie = v == ties.tau;
                    w = v >= ties.tau ? t : 0xff800000u;
                } else {
                    tie = keep_from(w, ties.tau, std::conditional_t<sizeof(In) == 2, uint16_t, float>());
                }
                if (check && __ballot(tie)) {
                    float v[VEC];
                    Vec<In, VEC>::unpack(t, v);
                    exactly(v, j);
                } else {
                    float v[VEC];
                    if constexpr (VEC != 1) {
                        if (j + VEC <= P.V) {
                            store_raw(out + j, w);
                            return;
                        }
                    }
                    Vec<In, VEC>::unpack(w, v);
                    store_vec<In, VEC>(out, j, P.V, v);
                }
            }, [](int) {});
            __syncthreads();
        }
        if (listed) row.drop_ties(ties.keep, reinterpret_cast<uint16_t*>(out));
    } else if (filters && !slots) {
        int n = 0, none = 0;
        if (counts && row.table_masses(ties, partial, n)) {
            if (partial) cut.limit = row.tie_place(ties.tau, ties.keep);
            const double w = row.mass(ties.tau);
            __syncthreads();
            if (partial && tid < P.nslots) sm.slot[tid] += (double)sm.ties[tid] * w;
            __syncthreads();
            kept = n;
        } else {
            if (partial) cut.limit = row.tie_limit(ties.tau, ties.keep);
            double a = 0.0;
            auto held = row.packed();
            __syncthreads();
            row.template sweep<true>([&](const float(&v)[VEC], int j) {
                bool in[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) n += in[e] = cut.keeps(v[e], j + e);
                row.pack(v, in, held, a);
            }, [&](int s) {
                row.rest(held, a);
                const double t = wave_sum(a);
                if (lane == 0) sm.slot[s] = t;
                a = 0.0;
            });
            double x = 0.0, y = 0.0;
            row.sum2(x, y, n, none);
            kept = n;
        }
    } else if (!filters) {
        kept = row.finite;
    }
    if (tid == 0) {
        if (P.kept) P.kept[r] = kept;
        if (P.status) P.status[r] = RS_SEQ_OK;
    }
    if (FILTER) return;
    // ---- the draws
    for (int s = lane; s < P.nslots; s += 64) total += sm.slot[s];
    total = wave_sum(total);
    for (int i = wid; i < P.k; i += kWaves) {
        float l;
        const int token = row.draw(P.u[r * P.k + i], total, cut, l);
        if (lane == 0) {
            P.token[r * P.k + i] = token;
            // not above 0, where the sums' last bits would say so
            if (P.logprob) P.logprob[r * P.k + i] = (float)fmin(((double)l - row.md) / (double)T - log(total), 0.0);
        }
    }
}

// Filtered rows under min-p alone, or under nothing, that fit the registers of a workgroup (64 of
// the 128 that a lane has at 4 waves a SIMD): the maximum alone decides, so that a row is read
// once, where the kernel above reads it again to write it.  1344 rows of 32,001 fp32 68 us
// (344 MB, 5.1 TB/s), by the kernel above 102; of 128,256 bf16, which take 16 waves, 151 and
// 200; one such row 15 and 23; no size measured from 8,000 up is slower.
constexpr int kHeldVecs = 16;   // of a lane
template <typename In, int VEC, int BLOCK>
__global__ void __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) rs_floor_kernel(const SParams P) {
    __shared__ ReduceSmem sm;
    constexpr int N = kHeldVecs;
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x;
    const int64_t entry = r / P.rows_per_entry;
    const float T = P.temperatures ? P.temperatures[entry] : P.temperature;
    const float min_p = P.min_ps ? P.min_ps[entry] : P.min_p;
    using RowT = Row<In, VEC, BLOCK, ReduceSmem>;
    RowT row{reinterpret_cast<const In*>(P.logits) + r * P.stride, P.V, P.G, P.nslots, 0.0f, 0.0, 0.0, uniform((double)T), sm};
    In* out = reinterpret_cast<In*>(P.out) + r * P.out_stride;
    int status = RS_SEQ_OK, n = 0, none = 0, bad = 0;
    if (!(T > 0.0f && T < INFINITY && min_p >= 0.0f && min_p <= 1.0f)) status = RS_SEQ_BAD_PARAM;
    typename Vec<In, VEC>::raw t[N];
    float mx = -INFINITY, floor = NAN;   // nothing is above a NaN
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * BLOCK * VEC < P.V) t[i] = Vec<In, VEC>::template load_full<true>(row.row, min((i * BLOCK + tid) * VEC, P.V - VEC));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * BLOCK * VEC >= P.V) continue;
        row.cut_off(t[i], (i * BLOCK + tid) * VEC);
        float v[VEC];
        Vec<In, VEC>::unpack(t[i], v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            mx = fmaxf(mx, v[e]);
            bad |= !(v[e] < INFINITY);
        }
    }
    row.m = row.block_max(mx);
    if ((__syncthreads_or(bad) || row.m == -INFINITY) && status == RS_SEQ_OK) status = RS_SEQ_UNDERFLOW;
    if (status == RS_SEQ_OK) floor = min_p > 0.0f ? fmaxf(row.min_floor((double)min_p), -FLT_MAX) : -FLT_MAX;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * BLOCK * VEC >= P.V) continue;
        const int j = (i * BLOCK + tid) * VEC;
        float v[VEC];
        Vec<In, VEC>::unpack(t[i], v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool in = v[e] >= floor;
            n += in;
            v[e] = in ? v[e] : -INFINITY;
        }
        store_vec<In, VEC>(out, j, P.V, v);
    }
    double x = 0.0, y = 0.0;
    row.sum2(x, y, n, none);
    if (tid == 0) {
        if (P.kept) P.kept[r] = status == RS_SEQ_OK ? n : -1;
        if (P.status) P.status[r] = status;
    }
}

// One workgroup a row, one pass: the sum of the row's masses against the highest element of its
// sample and of the tokens, in 32-bit exponentials (a log-probability is no border: its error
// is that of the sum, 1e-7 or so, and 1.6e-5 at most, where the row's maximum is 2^127 above
// both: the exponent, up to 128, is rounded three times).  That element's own term is exactly
// 1, and no token is above it, so no log-probability is above 0.  For every token, how many
// elements come before it in the order: only vectors with an element that is not below every
// token take the count, a step a token.  Where the sum overflows or the sample is masked, a
// second pass against the maximum.  640 rows of 128,256 bf16: 47 us, 164 MB at 3.5 TB/s.
template <typename In, int VEC, int BLOCK>
__global__ void __launch_bounds__(BLOCK) rs_logprob_kernel(const SParams P) {
    __shared__ ReduceSmem sm;
    __shared__ float token_logit[kMaxCand];
    __shared__ int32_t token_id[kMaxCand], token_rank[kMaxCand];
    __shared__ double slot[kRowSlots];
    const int tid = threadIdx.x, lane = tid & 63;
    using E = std::conditional_t<sizeof(In) == 2, uint16_t, float>;
    const int64_t r = blockIdx.x;
    const float T = P.temperatures ? P.temperatures[r / P.rows_per_entry] : P.temperature;
    using RowT = Row<In, VEC, BLOCK, ReduceSmem>;
    RowT row{reinterpret_cast<const In*>(P.logits) + r * P.stride, P.V, P.G, P.nslots, 0.0f, 0.0,
                                 uniform(1.4426950408889634 / (double)T), uniform((double)T), sm};
    int status = RS_SEQ_OK;
    if (!(T > 0.0f && T < INFINITY)) status = RS_SEQ_BAD_PARAM;
    const int x = tid < P.k ? P.tokens[r * P.k + tid] : -1;
    if (__syncthreads_or(x < -1 || x >= P.V) && status == RS_SEQ_OK) status = RS_SEQ_BAD_TOKEN;
    double total = 0.0;
    if (status == RS_SEQ_OK) {
        if (tid < P.k) {
            float l[1] = {INFINITY};
            if (x >= 0) load_vec<E, 1>(reinterpret_cast<const E*>(row.row), x, P.V, l);
            token_logit[tid] = l[0];
            token_id[tid] = x;
            token_rank[tid] = 0;
        }
        __syncthreads();
        // the tokens' lowest logit, and their highest
        float lowest = INFINITY, highest = -INFINITY;
        for (int i = 0; i < P.k; ++i) {
            const float l = token_logit[i];
            lowest = fminf(lowest, l);
            highest = fmaxf(highest, l < INFINITY ? l : -INFINITY);
        }
        lowest = uniform(P.rank ? lowest : INFINITY);
        float v0[RowT::kSampleLane];
        row.load_sample(v0);
        float ref = fmaxf(row.sample_max(v0), highest);
        if (!(ref > -INFINITY && ref < INFINITY)) ref = 0.0f;
        // c in two parts, both above zero: a -inf element's exponent is -inf, not a NaN
        float ch = (float)fmin(row.c, (double)FLT_MAX);
        if ((double)ch >= row.c) ch = __uint_as_float(__float_as_uint(ch) - 1);
        const float cl = fmaxf((float)fmin(row.c - (double)ch, (double)FLT_MAX), 0x1p-149f);
        int before = 0;   // lane i: token i's, of the wave's elements
        for (int attempt = 0;; ++attempt) {
            double a = 0.0;
            row.template sweep<true>([&](const float(&v)[VEC], int j) {
                float w[VEC];
                bool some = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = v[e] - ref;
                    w[e] = exp2_fast(fmaf(d, cl, d * ch));
                    some |= v[e] >= lowest;
                }
#pragma unroll
                for (int h = VEC / 2; h; h >>= 1)
#pragma unroll
                    for (int e = 0; e < h; ++e) w[e] += w[e + h];
                a += (double)w[0];
                if (attempt == 0 && __ballot(some)) {
                    for (int i = 0; i < P.k; ++i) {
                        const float l = token_logit[i];
                        const int id = token_id[i];
                        int n = 0;
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            n += __popcll(__ballot(v[e] > l || (v[e] == l && j + e < id)));
                        if (lane == i) before += n;
                    }
                }
            }, [&](int s) {
                const double t = wave_sum(a);
                if (lane == 0) slot[s] = t;
                a = 0.0;
            });
            __syncthreads();
            total = 0.0;
            for (int s = lane; s < P.nslots; s += 64) total += slot[s];
            total = uniform(wave_sum(total));
            row.md = (double)ref;
            if (total >= kLowSum && total < INFINITY) break;
            int n = 0;
            if (attempt == 1 || !row.statistics(n)) {
                status = RS_SEQ_UNDERFLOW;
                break;
            }
            ref = row.m;
        }
        if (before) atomicAdd(&token_rank[lane], before);
        __syncthreads();
    }
    if (tid == 0 && P.status) P.status[r] = status;
    if (tid < P.k) {
        float lp = NAN;
        int rank = -1;
        if (status == RS_SEQ_OK) {
            lp = x < 0 ? 0.0f : (float)(((double)token_logit[tid] - row.md) / row.T - log(total));
            rank = x < 0 ? 0 : token_rank[tid] + 1;
        }
        P.logprob[r * P.k + tid] = lp;
        if (P.rank) P.rank[r * P.k + tid] = rank;
    }
}

// ------------------------------------------------------------------- host ----

rs_status check_filter(const rs_filter* f) {
    if (!f || f->rows_per_entry < 1) return RS_ERR_INVALID_ARG;
    if (f->logits_dtype != RS_F32 && f->logits_dtype != RS_BF16) return RS_ERR_INVALID_ARG;
    if (!f->temperatures && !(f->temperature > 0.0f && std::isfinite(f->temperature))) return RS_ERR_INVALID_ARG;
    if (!f->top_ks && f->top_k < 0) return RS_ERR_INVALID_ARG;
    if (!f->top_ps && !(f->top_p > 0.0f && f->top_p <= 1.0f)) return RS_ERR_INVALID_ARG;
    if (!f->min_ps && !(f->min_p >= 0.0f && f->min_p <= 1.0f)) return RS_ERR_INVALID_ARG;
    return RS_OK;
}

SParams row_params(const void* logits, int64_t stride, int32_t R, int32_t V, const rs_filter* f) {
    SParams P{};
    P.logits = logits;
    P.stride = stride;
    P.R = R;
    P.V = V;
    P.rows_per_entry = f->rows_per_entry;
    P.temperature = f->temperature;
    P.top_k = f->top_k;
    P.top_p = f->top_p;
    P.min_p = f->min_p;
    P.temperatures = f->temperatures;
    P.top_ks = f->top_ks;
    P.top_ps = f->top_ps;
    P.min_ps = f->min_ps;
    return P;
}

// How rows that start `stride` elements apart are loaded (see row_loads).
RowLoads strided_loads(const void* p, int64_t stride, int32_t V, int dtype) {
    const int64_t esz = dtype == RS_BF16 ? 2 : 4;
    const RowLoads l = row_loads(p, p, V, dtype);
    return l == kLoadsAligned && stride * esz % 16 ? kLoadsAny : l;
}

// A workgroup a row, and less than 2^32 threads a launch.
constexpr int32_t kMaxRows = (1 << 23) - 1;

// The row of V elements in slots of G chunks.
template <int VEC>
void set_slots(SParams& P) {
    constexpr int64_t CHUNK = 64 * VEC * kUnrRow;
    const int64_t nch = ((int64_t)P.V + CHUNK - 1) / CHUNK;
    P.G = (int32_t)((nch + kRowSlots - 1) / kRowSlots);
    P.nslots = (int32_t)((nch + P.G - 1) / P.G);
}

// f(element type, elements a load) for the kernels' instance.
template <typename F>
auto with_rows(int dtype, RowLoads loads, F&& f) {
    return with_layout(dtype, loads, [&](auto in, auto vec, auto) { return f(in, vec); });
}

// Threads a row: 16 waves where every row has a CU to itself, 8 where there are more, so that a
// CU holds two rows or more (registers allow the draws two, the filter of bf16 rows three, the
// log-probabilities four).  128,256 bf16 logits, 16 waves and 8: 64 rows under top-p 44 and 48
// us, 256 rows 48 and 51, 300 rows 83 and 73, 768 rows 127 and 111; filtered 38 and 48, 46 and
// 52, 81 and 68, 145 and 131; log-probabilities 24 and 32, 25 and 33, 39 and 43, 70 and 57.
// Those alone would take 16 waves up to some 350 rows (400: 47 and 44); one rule for all costs
// them a tenth between.
constexpr int kCus = 256;
template <typename F>
auto with_block(int32_t R, F&& f) {
    using std::integral_constant;
    return R <= kCus ? f(integral_constant<int, 1024>()) : f(integral_constant<int, 512>());
}

}  // namespace

extern "C" {

rs_status resispec_sample(const void* logits, int64_t row_stride, const float* u, int32_t R, int32_t V, int32_t k,
                          const rs_filter* filter, int32_t* out_token, float* out_logprob, int32_t* out_kept,
                          int32_t* out_status, void* stream) {
    const rs_status fs = check_filter(filter);
    if (fs != RS_OK) return fs;
    if (R < 0 || V <= 0 || k <= 0 || row_stride < V) return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB || k > RS_MAX_CANDIDATES || R > kMaxRows) return RS_ERR_UNSUPPORTED;
    if (R == 0) return RS_OK;
    if (!logits || !u || !out_token) return RS_ERR_INVALID_ARG;
    SParams P = row_params(logits, row_stride, R, V, filter);
    P.u = u;
    P.k = k;
    P.token = out_token;
    P.logprob = out_logprob;
    P.kept = out_kept;
    P.status = out_status;
    const hipError_t e = with_rows(
        filter->logits_dtype, strided_loads(logits, row_stride, V, filter->logits_dtype), [&](auto in, auto vec) {
            set_slots<vec()>(P);
            return with_block(R, [&](auto block) {
                hipLaunchKernelGGL((rs_sample_kernel<decltype(in), vec(), block(), false>), dim3((unsigned)R), dim3(block()),
                                   0, (hipStream_t)stream, P);
                return hipGetLastError();
            });
        });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_filter_logits(const void* logits, int64_t row_stride, int32_t R, int32_t V,
                                 const rs_filter* filter, void* out, int64_t out_row_stride, int32_t* out_kept,
                                 int32_t* out_status, void* stream) {
    const rs_status fs = check_filter(filter);
    if (fs != RS_OK) return fs;
    if (R < 0 || V <= 0 || row_stride < V || out_row_stride < V) return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB || R > kMaxRows) return RS_ERR_UNSUPPORTED;
    if (R == 0) return RS_OK;
    if (!logits || !out) return RS_ERR_INVALID_ARG;
    SParams P = row_params(logits, row_stride, R, V, filter);
    P.out = out;
    P.out_stride = out_row_stride;
    P.kept = out_kept;
    P.status = out_status;
    const RowLoads in = strided_loads(logits, row_stride, V, filter->logits_dtype);
    const RowLoads to = strided_loads(out, out_row_stride, V, filter->logits_dtype);
    // only the numbers are known here: rows with arrays of top_k or top_p go the general way
    const bool floors = !filter->top_ks && filter->top_k == 0 && !filter->top_ps && filter->top_p == 1.0f;
    const hipError_t e = with_rows(filter->logits_dtype, in > to ? in : to, [&](auto in, auto vec) {
        set_slots<vec()>(P);
        if constexpr (vec() > 1)
            if (floors && V <= kHeldVecs * 1024 * vec())
                return with_block(V <= kHeldVecs * 512 * vec() ? R : 1, [&](auto block) {
                    hipLaunchKernelGGL((rs_floor_kernel<decltype(in), vec(), block()>), dim3((unsigned)R), dim3(block()), 0,
                                       (hipStream_t)stream, P);
                    return hipGetLastError();
                });
        return with_block(R, [&](auto block) {
            hipLaunchKernelGGL((rs_sample_kernel<decltype(in), vec(), block(), true>), dim3((unsigned)R),
                               dim3(block()), 0, (hipStream_t)stream, P);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_token_logprobs(const void* logits, int64_t row_stride, const int32_t* tokens, int32_t R, int32_t V,
                                  int32_t k, const rs_filter* filter, float* out_logprob, int32_t* out_rank,
                                  int32_t* out_status, void* stream) {
    const rs_status fs = check_filter(filter);
    if (fs != RS_OK) return fs;
    if (R < 0 || V <= 0 || k <= 0 || row_stride < V) return RS_ERR_INVALID_ARG;
    if (filter->top_ks || filter->top_ps || filter->min_ps || filter->top_k != 0 || filter->top_p != 1.0f ||
        filter->min_p != 0.0f)
        return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB || k > RS_MAX_CANDIDATES || R > kMaxRows) return RS_ERR_UNSUPPORTED;
    if (R == 0) return RS_OK;
    if (!logits || !tokens || !out_logprob) return RS_ERR_INVALID_ARG;
    SParams P = row_params(logits, row_stride, R, V, filter);
    P.tokens = tokens;
    P.k = k;
    P.logprob = out_logprob;
    P.rank = out_rank;
    P.status = out_status;
    const hipError_t e = with_rows(
        filter->logits_dtype, strided_loads(logits, row_stride, V, filter->logits_dtype), [&](auto in, auto vec) {
            set_slots<vec()>(P);
            return with_block(R, [&](auto block) {
                hipLaunchKernelGGL((rs_logprob_kernel<decltype(in), vec(), block()>), dim3((unsigned)R), dim3(block()),
                                   0, (hipStream_t)stream, P);
                return hipGetLastError();
            });
        });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
