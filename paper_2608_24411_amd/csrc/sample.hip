// sample.hip -- sampling from rows of logits on gfx950: draws under temperature, top-k,
// top-p and min-p from given uniforms (resispec_sample), rows cut to what these keep
// (resispec_filter_logits), and log-probabilities and ranks of given tokens
// (resispec_token_logprobs).  Declared in resispec.h.

#include "common.h"

#include <climits>

namespace {

// Mathematics.  A row's elements are ordered by logit, equal ones by index.  top-k, top-p and
// min-p each keep a prefix of that order, so what is kept is one cut: the lowest kept value
// and, among the elements equal to it, the last kept index.  Masses are w_j = 2^((l_j - m) c)
// with m the row's maximum and c = log2(e) / T, in fp64: a token or a cut is decided by the
// side of a border that a sum over the whole row falls on, and of 1e5 borders one lies within
// 1e-6 (what 32-bit exponentials give) of a draw now and then.

constexpr int kRowSlots = 256;      // runs of chunks with sums of their own
constexpr int kBins = 2048;         // histogram bins of a search for a cut
constexpr int kUnrRow = 4;          // 16-byte loads a lane and chunk

// Bins of bf16 values, from the highest to the lowest: one for every value with 2^-38 < |l| <
// 1020, one for those between (where both zeros are), one at each end for those outside
// (-inf in the last).  Unused: bin 0.
constexpr int kHalf = 6144, kValueBins = 2 * kHalf;
constexpr uint16_t kLoMag = (127 - 38) << 7, kTopMag = kHalf - 1;
constexpr int kTopBin = 1, kZeroBin = kHalf, kLastBin = kValueBins - 1;

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

struct RowSmem {
    union {
        float hist[kBins];            // search within a range of keys
        uint32_t count[kValueBins];   // how often each bf16 value occurs
        double table[kValueBins / 2]; // their masses, from the highest value of the row
        int32_t list[kValueBins];     // indices of equal elements
    };
    double slot[kRowSlots];
    int32_t ties[kRowSlots];
    double cut_above, cut_mass;       // what lies above the crossing bin, and the prefix's mass
    int32_t cut_bin, cut_keep, cut_all, nlist;
    double red[2][kMaxWaves];
    int32_t redi[2][kMaxWaves];
    uint32_t redk[2][kMaxWaves];
    float redf[kMaxWaves];
    int32_t bin, limit;
};

// Ordered keys: a > b as floats exactly where key(a) > key(b); -0 and +0 share one.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}

// 2^x for x <= 0 in fp64, zero below 2^-1074.  2^f = 1 + f g(f) on [-1/2, 1/2], g of degree 8
// interpolated at Chebyshev nodes: 3.7e-14 off at most, and exactly 1 at 0.
__device__ __forceinline__ double exp2_64(double x) {
    x = fmax(x, -1100.0);
    const double n = rint(x), f = x - n;
    double p = 0x1.b63880a30e9ffp-24;
    p = fma(p, f, 0x1.63d136366db24p-20);
    p = fma(p, f, 0x1.ffcb9515a8016p-17);
    p = fma(p, f, 0x1.4308ac85aa947p-13);
    p = fma(p, f, 0x1.5d87fe86fe88ep-10);
    p = fma(p, f, 0x1.3b2ab7181b755p-7);
    p = fma(p, f, 0x1.c6b08d7047e52p-5);
    p = fma(p, f, 0x1.ebfbdff823cedp-3);
    p = fma(p, f, 0x1.62e42fefa39efp-1);
    p = fma(p, f, 1.0);
    return __builtin_ldexp(p, (int)n);
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
    const u16x2 lo = {kLoMag, kLoMag}, top = {kTopMag, kTopMag};
    const u16x2 one = {(uint16_t)(kHalf + 1), (uint16_t)(kHalf + 1)};
    const u16x2 mag = __builtin_bit_cast(u16x2, word & 0x7fff7fffu);
    const u16x2 t = __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, lo), top);
    const u16x2 neg = __builtin_bit_cast(u16x2, __builtin_bit_cast(i16x2, word) >> 15);
    // kHalf - t for positive values, kHalf + t for negative ones
    return (~(t ^ neg) + neg + one) << 2;
}
__device__ __forceinline__ float bin_value(int bin) {
    const int t = bin < kHalf ? kHalf - bin : bin - kHalf;
    if (t == 0) return 0.0f;
    return __uint_as_float((uint32_t)(t + kLoMag) << 16 | (bin > kHalf ? 0x80000000u : 0u));
}

template <typename In, int VEC, int UNR, int BLOCK>
struct Row {
    using W = Vec<In, VEC>;
    static constexpr int CHUNK = 64 * VEC * UNR;
    static constexpr int kWaves = BLOCK / 64;
    static constexpr int PER = kValueBins / BLOCK;   // bins a thread
    const In* row;
    int V, G, nslots;
    float m;       // the row's maximum
    double md, c;  // the same, and log2(e) / T
    RowSmem& sm;

    __device__ __forceinline__ double mass(float l) const { return exp2_64(((double)l - md) * c); }

    // body(t, j): a vector of VEC elements from index j as loaded (-inf at and past V);
    // flush(slot) after a slot's last.  A wave's slots are the same in every pass.
    template <typename Body, typename Flush>
    __device__ __forceinline__ void sweep_raw(Body&& body, Flush&& flush) const {
        const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
        typename W::raw a[UNR], b[UNR];
        auto load = [&](int s, int g, typename W::raw(&t)[UNR]) {
            load_chunk<In, VEC, UNR, false, false>(row, row, (s * G + g) * CHUNK, V, t, t);
        };
        auto process = [&](int s, int g, typename W::raw(&t)[UNR]) {
            const int j0 = (s * G + g) * CHUNK + lane * VEC;
#pragma unroll
            for (int u = 0; u < UNR; ++u) {
                W::settle(t[u], row, j0 + u * 64 * VEC, V);
                body(t[u], j0 + u * 64 * VEC);
            }
            if (g == G - 1) flush(s);
        };
        int s = wid, g = 0;
        if (s >= nslots) return;
        load(s, g, a);
        for (;;) {
            int s2 = s, g2 = g + 1;
            if (g2 == G) { s2 += kWaves; g2 = 0; }
            if (s2 < nslots) load(s2, g2, b);
            process(s, g, a);
            if (s2 >= nslots) break;
            s = s2; g = g2 + 1;
            if (g == G) { s += kWaves; g = 0; }
            if (s < nslots) load(s, g, a);
            process(s2, g2, b);
            if (s >= nslots) break;
        }
    }

    // The same with the elements as floats.
    template <typename Body, typename Flush>
    __device__ __forceinline__ void sweep(Body&& body, Flush&& flush) const {
        sweep_raw([&](const typename W::raw& t, int j) {
            float v[VEC];
            W::unpack(t, v);
            body(v, j);
        }, flush);
    }

    // Sums over the workgroup in a fixed order, to every thread.
    __device__ __forceinline__ void sum2(double& a, double& b, int& p, int& q) const {
        const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
        const double wa = wave_sum(a), wb = wave_sum(b);
        const int wp = __reduce_add_sync(~0ull, p), wq = __reduce_add_sync(~0ull, q);
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
    }
    __device__ __forceinline__ void range(uint32_t& lo, uint32_t& hi) const {
        const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
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
        const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
        float mx = -INFINITY;
        int cnt = 0, bad = 0;
        sweep([&](const float(&v)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                mx = fmaxf(mx, v[e]);
                cnt += v[e] > -INFINITY;
                bad |= !(v[e] < INFINITY);
            }
        }, [](int) {});
        mx = wave_max(mx);
        __syncthreads();
        if (lane == 0) sm.redf[wid] = mx;
        const bool any_bad = __syncthreads_or(bad);
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, sm.redf[w]);
        double x = 0.0, y = 0.0;
        int z = 0;
        sum2(x, y, cnt, z);
        n = cnt;
        m = mx;
        md = (double)mx;
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
    // left; the mass above a bin is summed in fp64 in a fixed order, and the histogram's
    // 32-bit sums only say where to look.  `total_mass`: of the prefix, where wanted.
    template <bool MASS>
    __device__ __forceinline__ Ties select(double target, uint32_t lo, uint32_t hi, double above, bool want_mass,
                                           double& total_mass) const {
        const int tid = threadIdx.x;
        for (;;) {
            const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
            __syncthreads();
            for (int i = tid; i < kBins; i += BLOCK) sm.hist[i] = 0.0f;
            __syncthreads();
            sweep([&](const float(&v)[VEC], int) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const uint32_t k = key_of(v[e]);
                    if (v[e] > -INFINITY && k >= lo && k <= hi) {
                        const float w = MASS ? exp2_fast((v[e] - m) * (float)fmin(c, (double)FLT_MAX)) : 1.0f;
                        unsafeAtomicAdd(&sm.hist[(hi - k) >> shift], w);
                    }
                }
            }, [](int) {});
            int bin = crossing(above, target);
            double a, in, mass_a, mass_in;
            int na, nin;
            uint32_t kmin, kmax;
            int turned = 0;   // which way the search has gone
            for (;;) {
                // what lies above the bin, what in it, and the range of the keys in it
                mass_a = mass_in = 0.0;
                na = nin = 0;
                kmin = ~0u;
                kmax = 0u;
                sweep([&](const float(&v)[VEC], int) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if (!(v[e] > -INFINITY)) continue;
                        const uint32_t k = key_of(v[e]);
                        if (k < lo) continue;
                        const int b = k > hi ? -1 : (int)((hi - k) >> shift);
                        if (b > bin) continue;
                        const double w = MASS || want_mass ? mass(v[e]) : 0.0;
                        if (b < bin) {
                            ++na;
                            mass_a += w;
                        } else {
                            ++nin;
                            mass_in += w;
                            kmin = min(kmin, k);
                            kmax = max(kmax, k);
                        }
                    }
                }, [](int) {});
                sum2(mass_a, mass_in, na, nin);
                range(kmin, kmax);
                a = MASS ? mass_a : (double)na;
                in = MASS ? mass_in : (double)nin;
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
                if (MASS && a + in < target && turned >= 0) {
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
        const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
        for (int i = tid; i < kValueBins / 4; i += BLOCK) reinterpret_cast<uint4*>(sm.count)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        i16x2 pos = {0, 0};
        u16x2 neg = {0, 0};
        sweep_raw([&](const typename W::raw& t, int) {
            if constexpr (VEC == 8) {
                const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    pos = __builtin_elementwise_max(pos, __builtin_bit_cast(i16x2, w[q]));
                    neg = __builtin_elementwise_max(neg, __builtin_bit_cast(u16x2, w[q]));
                    const u16x2 at = bin_bytes(w[q]);
                    char* base = reinterpret_cast<char*>(sm.count);
                    __hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(base + at.x), 1u, __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_WORKGROUP);
                    __hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(base + at.y), 1u, __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_WORKGROUP);
                }
            }
        }, [](int) {});
        // positive words from 0x7f80 are +inf and NaN, negative ones past 0xff80 NaN
        const bool mine = pos.x >= 0x7f80 || pos.y >= 0x7f80 || neg.x > 0xff80 || neg.y > 0xff80;
        bad = __syncthreads_or(mine);
        // the highest value: the first bin that is not empty
        int first = kValueBins;
        for (int q = 0; q < PER / 4; ++q) {
            const uint4 n = reinterpret_cast<const uint4*>(sm.count)[tid * (PER / 4) + q];
            const int b = tid * PER + 4 * q;
            first = min(first, n.x ? b : n.y ? b + 1 : n.z ? b + 2 : n.w ? b + 3 : kValueBins);
        }
        for (int o = 32; o; o >>= 1) first = min(first, __shfl_xor(first, o));
        if (lane == 0) sm.redi[0][wid] = first;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) first = min(first, sm.redi[0][w]);
        m = bin_value(first);
        md = (double)m;
        top = first;
        if (!(first > kTopBin && first < kLastBin && (md + 1020.0) * c > 150.0)) return false;
        if (sm.count[kZeroBin] == 0) return true;
        bool small = false;   // nonzero values in the bin around zero
        sweep([&](const float(&v)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) small |= v[e] != 0.0f && fabsf(v[e]) <= 0x1p-38f;
        }, [](int) {});
        return !__syncthreads_or(small);
    }
    int top = 0;   // the bin of the row's highest value

    // The bin in which the counts (BY_MASS: the masses) of the row's values reach `target`,
    // from every thread's sums before and in its PER bins; into sm.cut_*.
    template <bool BY_MASS>
    __device__ __forceinline__ void locate(double target, double before_n, double before_m, double own_n, double own_m,
                                           bool want_mass) const {
        const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
        const double own = BY_MASS ? own_m : own_n;
        const uint64_t some = __ballot(own > 0.0);
        const uint64_t hit = __ballot(own > 0.0 && (BY_MASS ? before_m : before_n) + own >= target);
        __syncthreads();
        if (lane == 0) {
            sm.redi[0][wid] = hit ? wid * 64 + __ffsll((unsigned long long)hit) - 1 : BLOCK;
            sm.redi[1][wid] = some ? wid * 64 + 63 - __clzll((long long)some) : 0;
        }
        __syncthreads();
        int at = BLOCK, last = 0;
        for (int w = 0; w < kWaves; ++w) {
            at = min(at, sm.redi[0][w]);
            last = max(last, sm.redi[1][w]);
        }
        if (at == BLOCK) at = last;
        if (tid == at) {
            sm.cut_above = before_n;
            sm.cut_mass = before_m;
        }
        __syncthreads();
        if (wid == 0) {   // a lane for each of that thread's bins
            const double base_n = sm.cut_above, base_m = sm.cut_mass;
            const int b = at * PER + lane;
            const int n = lane < PER && b < kLastBin ? (int)sm.count[b] : 0;
            const double w = n && (BY_MASS || want_mass) ? mass(bin_value(b)) : 0.0;
            const double in_n = base_n + wave_incl_scan((double)n, lane);
            const double in_m = base_m + wave_incl_scan((double)n * w, lane);
            const bool real = n > 0 && (!BY_MASS || w > 0.0);
            const uint64_t over = __ballot(real && (BY_MASS ? in_m : in_n) >= target);
            const uint64_t any = __ballot(real);
            const int L = over ? __ffsll((unsigned long long)over) - 1 : any ? 63 - __clzll((long long)any) : 0;
            if (lane == L) {
                const double above_n = in_n - (double)n, above_m = in_m - (double)n * w;
                const int keep = BY_MASS ? ties_for(target - above_m, w, n) : (int)(target - above_n);
                sm.cut_bin = b;
                sm.cut_keep = keep;
                sm.cut_all = n;
                sm.cut_above = BY_MASS ? above_m : above_n;
                sm.cut_mass = above_m + (double)keep * w;
            }
        }
        __syncthreads();
    }

    // The cut of top_k and top_p from the counts of a row's values.  Where it falls among the
    // values below all bins, the search ends it.
    __device__ __forceinline__ Ties cut_values(int top_k, double top_p) const {
        const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
        const bool want_mass = top_p < 1.0;
        double own_n = 0.0, own_m = 0.0;
        for (int q = 0; q < PER / 4; ++q) {
            const uint4 n4 = reinterpret_cast<const uint4*>(sm.count)[tid * (PER / 4) + q];
            const uint32_t n[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int b = tid * PER + 4 * q + e;
                if (n[e] && b < kLastBin) {
                    own_n += (double)n[e];
                    if (want_mass) own_m += (double)n[e] * mass(bin_value(b));
                }
            }
        }
        const double in_n = wave_incl_scan(own_n, lane), in_m = wave_incl_scan(own_m, lane);
        __syncthreads();
        if (lane == 63) {
            sm.red[0][wid] = in_n;
            sm.red[1][wid] = in_m;
        }
        __syncthreads();
        double before_n = in_n - own_n, before_m = in_m - own_m, all_n = 0.0, all_m = 0.0;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wid) {
                before_n += sm.red[0][w];
                before_m += sm.red[1][w];
            }
            all_n += sm.red[0][w];
            all_m += sm.red[1][w];
        }
        Ties cut{-INFINITY, 0, 0};
        double mass_k = all_m;
        bool cut_k = top_k > 0;
        if (cut_k && (double)top_k > all_n) {
            // into the last bin, which holds -inf too
            int below = 0, none = 0;
            double x = 0.0, y = 0.0;
            sweep([&](const float(&v)[VEC], int) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) below += v[e] > -INFINITY && v[e] <= bin_value(kLastBin);
            }, [](int) {});
            sum2(x, y, below, none);
            cut_k = all_n + (double)below > (double)top_k;
            if (cut_k && !want_mass)   // top_p cuts above that bin, which has no mass
                cut = select<false>((double)top_k, key_of(-INFINITY) + 1, key_of(bin_value(kLastBin)), all_n, want_mass,
                                    mass_k);
        } else if (cut_k) {
            locate<false>((double)top_k, before_n, before_m, own_n, own_m, want_mass);
            cut = {bin_value(sm.cut_bin), sm.cut_keep, sm.cut_all};
            mass_k = sm.cut_mass;
        }
        if (top_p == 1.0) return cut;
        locate<true>(top_p * mass_k, before_n, before_m, own_n, own_m, true);
        return {bin_value(sm.cut_bin), sm.cut_keep, sm.cut_all};
    }

    // Number of the row's elements in the bins up to `bin`.
    __device__ __forceinline__ int count_to(int bin) const {
        int n = 0, none = 0;
        double x = 0.0, y = 0.0;
        for (int b = threadIdx.x; b <= bin; b += BLOCK) n += (int)sm.count[b];
        sum2(x, y, n, none);
        return n;
    }

    // The index of the keep-th element equal to tau.
    __device__ __forceinline__ int tie_limit(float tau, int keep) const {
        const int lane = threadIdx.x & 63;
        int cnt = 0;
        __syncthreads();
        sweep([&](const float(&v)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) cnt += v[e] == tau;
        }, [&](int s) {
            const int n = __reduce_add_sync(~0ull, cnt);
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

    // The slots' sums of all masses, against the highest of the waves' first elements; or, where
    // the row's maximum is far above it, against that.  False where the row has no
    // distribution.
    __device__ __forceinline__ bool slot_masses() {
        const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
        float v[VEC], mx = -INFINITY;
        load_vec<In, VEC>(row, wid * G * CHUNK + lane * VEC, V, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) mx = fmaxf(mx, v[e]);
        for (int attempt = 0;; ++attempt) {
            mx = wave_max(mx);
            __syncthreads();
            if (lane == 0) sm.redf[wid] = mx;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, sm.redf[w]);
            // a NaN or a +inf here shows in the pass too
            md = mx > -INFINITY && mx < INFINITY ? (double)mx : 0.0;
            double a = 0.0;
            int n = 0, bad = 0, none = 0;
            sweep([&](const float(&t)[VEC], int) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
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
            m = wave_max(mx);
            __syncthreads();
            if (lane == 0) sm.redf[wid] = m;
            const bool any_bad = __syncthreads_or(bad);
            for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sm.redf[w]);
            if (any_bad || n == 0) return false;
            if (attempt == 1 || fabs((double)m - md) * c < 500.0) return true;
            mx = m;
        }
    }
    int finite = 0;

    // The slots' sums of what a cut keeps, from a table of the masses of the values above it,
    // and how many elements that is.  `partial`: the elements equal to the cut's value are
    // counted by slot instead.  False where the table has no room for all values.
    __device__ __forceinline__ bool table_masses(const Ties& cut, bool partial, int& n) const {
        const int tid = threadIdx.x, lane = tid & 63;
        if constexpr (VEC == 8) {
            if (!(cut.tau > -INFINITY)) return false;
            int end = bin_bytes(__float_as_uint(cut.tau) >> 16).x / 4;
            if (end == kZeroBin && cut.tau > 0.0f) --end;   // the bin holds zeros, below the cut
            if (end == kLastBin || end - top + 2 > kValueBins / 2) return false;
            n = count_to(end) - (partial ? cut.all - cut.keep : 0);
            __syncthreads();
            for (int i = tid; i <= end - top + 1; i += BLOCK)
                sm.table[i] = i > end - top || (partial && i == end - top) ? 0.0 : mass(bin_value(top + i));
            __syncthreads();
            const char* base = reinterpret_cast<const char*>(sm.table) - top * 8;
            const uint16_t last = (uint16_t)(end * 4 + 4), at_cut = (uint16_t)(end * 4);
            const u16x2 lasts = {last, last};
            double a = 0.0;
            int ties = 0;
            sweep_raw([&](const typename W::raw& t, int) {
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
                const int nt = partial ? __reduce_add_sync(~0ull, ties) : 0;
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
    // become -inf.
    __device__ __forceinline__ void drop_ties(int keep, uint16_t* out) const {
        const int tid = threadIdx.x;
        __syncthreads();
        const int n = sm.nlist;
        for (int s = tid; s < kRowSlots; s += BLOCK) sm.ties[s] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += BLOCK) atomicAdd(&sm.ties[sm.list[i] / (G * CHUNK)], 1);
        __syncthreads();
        for (int i = tid; i < n; i += BLOCK) {
            const int j = sm.list[i], s = j / (G * CHUNK);
            int before = 0;
            for (int q = 0; q < s; ++q) before += sm.ties[q];
            if (before + sm.ties[s] > keep) {
                if (before < keep)
                    for (int q = 0; q < n; ++q) before += sm.list[q] < j && sm.list[q] / (G * CHUNK) == s;
                if (before >= keep) out[j] = 0xff80;
            }
        }
    }

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
        for (int q = slot * G * UNR; q < (slot + 1) * G * UNR; ++q) {
            const int j = q * 64 * VEC + lane * VEC;
            float v[VEC];
            load_vec<In, VEC>(row, j, V, v);
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

// One workgroup a row: the cut, then the draws or the filtered row.
template <typename In, int VEC, int UNR, int BLOCK, bool FILTER>
__global__ void __launch_bounds__(BLOCK) rs_sample_kernel(const SParams P) {
    __shared__ RowSmem sm;
    constexpr int kWaves = BLOCK / 64;
    constexpr bool kCounts = VEC == 8;   // bf16 rows: counts of values
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int64_t r = blockIdx.x;
    const int64_t entry = r / P.rows_per_entry;
    const float T = P.temperatures ? P.temperatures[entry] : P.temperature;
    const float top_p = P.top_ps ? P.top_ps[entry] : P.top_p;
    const float min_p = P.min_ps ? P.min_ps[entry] : P.min_p;
    const int top_k = P.top_ks ? P.top_ks[entry] : P.top_k;
    Row<In, VEC, UNR, BLOCK> row{reinterpret_cast<const In*>(P.logits) + r * P.stride, P.V, P.G, P.nslots, 0.0f, 0.0,
                                 1.4426950408889634 / (double)T, sm};
    In* out = FILTER ? reinterpret_cast<In*>(P.out) + r * P.out_stride : nullptr;
    int status = RS_SEQ_OK;
    if (!(T > 0.0f && T < INFINITY && top_k >= 0 && top_p > 0.0f && top_p <= 1.0f && min_p >= 0.0f && min_p <= 1.0f))
        status = RS_SEQ_BAD_PARAM;
    if (!FILTER && status == RS_SEQ_OK) {
        const float u = tid < P.k ? P.u[r * P.k + tid] : 0.0f;
        if (__syncthreads_or(!(u >= 0.0f && u < 1.0f))) status = RS_SEQ_BAD_UNIFORM;
    }
    // ---- the cut, and whether the counts of the row's values are at hand
    const bool filters = top_k > 0 || top_p < 1.0f || min_p > 0.0f;
    Ties ties{-INFINITY, 0, 0};
    bool counts = false;
    int kept = -1;
    if (status == RS_SEQ_OK && (filters || FILTER)) {
        bool bad = false;
        if constexpr (kCounts) {
            counts = row.count_values(bad);
            if (counts && filters) ties = row.cut_values(top_k, (double)top_p);
        }
        if (!counts) {
            int n = 0;
            if (bad || !row.statistics(n)) {
                status = RS_SEQ_UNDERFLOW;
            } else {
                const uint32_t lo = key_of(-INFINITY) + 1, hi = key_of(row.m);
                double mass = 0.0;
                const bool cuts_k = top_k > 0 && top_k < n;
                if (cuts_k) ties = row.template select<false>((double)top_k, lo, hi, 0.0, top_p < 1.0f, mass);
                if (top_p < 1.0f) {
                    if (!cuts_k) {
                        double a = 0.0, b = 0.0;
                        int x = 0, y = 0;
                        row.sweep([&](const float(&v)[VEC], int) {
#pragma unroll
                            for (int e = 0; e < VEC; ++e) a += row.mass(v[e]);
                        }, [](int) {});
                        row.sum2(a, b, x, y);
                        mass = a;
                    }
                    ties = row.template select<true>((double)top_p * mass, lo, hi, 0.0, false, mass);
                }
            }
        } else if (bad) {
            status = RS_SEQ_UNDERFLOW;
        }
        if (status == RS_SEQ_OK && min_p > 0.0f) {
            // w >= min_p where l >= m + T ln(min_p): the lowest value of the row's type that is
            const double t = row.md + (double)T * log((double)min_p);
            float f = (float)t;
            if ((double)f < t) f = value_of(key_of(f) + 1);
            if (kCounts) {
                const uint32_t b = __float_as_uint(f);
                f = __uint_as_float((b & 0xffff0000u) + ((b & 0xffffu) && !(b >> 31) ? 0x10000u : 0u));
            }
            if (f > ties.tau) ties = Ties{f, 0, 0};
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
    Cut cut{ties.tau, ties.tau > -INFINITY ? INT_MAX : -1};
    if (FILTER) {
        // many ties: their last index is found first; few: all are written as kept, and the
        // rest taken back
        constexpr int kListed = 4096;
        const bool listed = counts && partial && ties.all <= kListed;
        if (partial && !listed) cut.limit = row.tie_limit(ties.tau, ties.keep);
        __syncthreads();
        if (tid == 0) sm.nlist = 0;
        __syncthreads();
        int n = 0, none = 0;
        row.sweep([&](const float(&v)[VEC], int j) {
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
                    if (v[e] == ties.tau) sm.list[atomicAdd(&sm.nlist, 1)] = j + e;
            }
        }, [](int) {});
        double x = 0.0, y = 0.0;
        row.sum2(x, y, n, none);
        if (listed) {
            row.drop_ties(ties.keep, reinterpret_cast<uint16_t*>(out));
            n -= ties.all - ties.keep;
        }
        kept = n;
    } else if (filters) {
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
            row.sweep([&](const float(&v)[VEC], int j) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if (cut.keeps(v[e], j + e)) {
                        a += row.mass(v[e]);
                        ++n;
                    }
                }
            }, [&](int s) {
                const double t = wave_sum(a);
                if (lane == 0) sm.slot[s] = t;
                a = 0.0;
            });
            double x = 0.0, y = 0.0;
            row.sum2(x, y, n, none);
            kept = n;
        }
    } else {
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
            if (P.logprob) P.logprob[r * P.k + i] = (float)(((double)l - row.md) / (double)T - log(total));
        }
    }
}

// One workgroup a row: the sum of the row's masses against its maximum, and for every token
// how many elements come before it in the order.
template <typename In, int VEC, int UNR, int BLOCK>
__global__ void __launch_bounds__(BLOCK) rs_logprob_kernel(const SParams P) {
    __shared__ RowSmem sm;
    const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63;
    constexpr int kWaves = BLOCK / 64;
    const int64_t r = blockIdx.x;
    const float T = P.temperatures ? P.temperatures[r / P.rows_per_entry] : P.temperature;
    Row<In, VEC, UNR, BLOCK> row{reinterpret_cast<const In*>(P.logits) + r * P.stride, P.V, P.G, P.nslots, 0.0f, 0.0,
                                 1.4426950408889634 / (double)T, sm};
    int status = RS_SEQ_OK, n = 0;
    if (!(T > 0.0f && T < INFINITY)) status = RS_SEQ_BAD_PARAM;
    const int x = tid < P.k ? P.tokens[r * P.k + tid] : -1;
    if (__syncthreads_or(x < -1 || x >= P.V) && status == RS_SEQ_OK) status = RS_SEQ_BAD_TOKEN;
    if (status == RS_SEQ_OK && !row.statistics(n)) status = RS_SEQ_UNDERFLOW;
    if (tid == 0 && P.status) P.status[r] = status;
    if (status != RS_SEQ_OK) {
        if (tid < P.k) {
            if (P.logprob) P.logprob[r * P.k + tid] = NAN;
            if (P.rank) P.rank[r * P.k + tid] = -1;
        }
        return;
    }
    double a = 0.0, b = 0.0;
    int p = 0, q = 0;
    row.sweep([&](const float(&v)[VEC], int) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) a += row.mass(v[e]);
    }, [](int) {});
    row.sum2(a, b, p, q);
    for (int i = 0; i < P.k; ++i) {
        const int t = P.tokens[r * P.k + i];
        float l = 0.0f;
        int before = 0;
        if (t >= 0) {
            float v[1];
            load_vec<std::conditional_t<sizeof(In) == 2, uint16_t, float>, 1>(
                reinterpret_cast<const std::conditional_t<sizeof(In) == 2, uint16_t, float>*>(row.row), t, P.V, v);
            l = v[0];
            if (P.rank) {
                row.sweep([&](const float(&w)[VEC], int j) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) before += w[e] > l || (w[e] == l && j + e < t);
                }, [](int) {});
                double z = 0.0, z2 = 0.0;
                int none = 0;
                row.sum2(z, z2, before, none);
            }
        }
        if (tid == 0) {
            if (P.logprob) P.logprob[r * P.k + i] = t < 0 ? 0.0f : (float)(((double)l - row.md) / (double)T - log(a));
            if (P.rank) P.rank[r * P.k + i] = t < 0 ? 0 : before + 1;
        }
    }
    (void)wid;
    (void)lane;
    (void)kWaves;
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

constexpr int kRowBlock = 512;

}  // namespace

extern "C" {

rs_status resispec_sample(const void* logits, int64_t row_stride, const float* u, int32_t R, int32_t V, int32_t k,
                          const rs_filter* filter, int32_t* out_token, float* out_logprob, int32_t* out_kept,
                          int32_t* out_status, void* stream) {
    const rs_status fs = check_filter(filter);
    if (fs != RS_OK) return fs;
    if (R < 0 || V <= 0 || k <= 0 || row_stride < V) return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB || k > RS_MAX_CANDIDATES) return RS_ERR_UNSUPPORTED;
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
            hipLaunchKernelGGL((rs_sample_kernel<decltype(in), vec(), kUnrRow, kRowBlock, false>), dim3((unsigned)R),
                               dim3(kRowBlock), 0, (hipStream_t)stream, P);
            return hipGetLastError();
        });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

rs_status resispec_filter_logits(const void* logits, int64_t row_stride, int32_t R, int32_t V,
                                 const rs_filter* filter, void* out, int64_t out_row_stride, int32_t* out_kept,
                                 int32_t* out_status, void* stream) {
    const rs_status fs = check_filter(filter);
    if (fs != RS_OK) return fs;
    if (R < 0 || V <= 0 || row_stride < V || out_row_stride < V) return RS_ERR_INVALID_ARG;
    if (V > RS_MAX_VOCAB) return RS_ERR_UNSUPPORTED;
    if (R == 0) return RS_OK;
    if (!logits || !out) return RS_ERR_INVALID_ARG;
    SParams P = row_params(logits, row_stride, R, V, filter);
    P.out = out;
    P.out_stride = out_row_stride;
    P.kept = out_kept;
    P.status = out_status;
    const RowLoads in = strided_loads(logits, row_stride, V, filter->logits_dtype);
    const RowLoads to = strided_loads(out, out_row_stride, V, filter->logits_dtype);
    const hipError_t e = with_rows(filter->logits_dtype, in > to ? in : to, [&](auto in, auto vec) {
        set_slots<vec()>(P);
        hipLaunchKernelGGL((rs_sample_kernel<decltype(in), vec(), kUnrRow, kRowBlock, true>), dim3((unsigned)R),
                           dim3(kRowBlock), 0, (hipStream_t)stream, P);
        return hipGetLastError();
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
    if (V > RS_MAX_VOCAB || k > RS_MAX_CANDIDATES) return RS_ERR_UNSUPPORTED;
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
            hipLaunchKernelGGL((rs_logprob_kernel<decltype(in), vec(), kUnrRow, kRowBlock>), dim3((unsigned)R),
                               dim3(kRowBlock), 0, (hipStream_t)stream, P);
            return hipGetLastError();
        });
    return e == hipSuccess ? RS_OK : RS_ERR_HIP;
}

}  // extern "C"
