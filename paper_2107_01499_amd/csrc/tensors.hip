// Many tensors in one launch: the global gradient norm with its clipping factor, and the AdamW step (see bagua_hip.h).
//
// A plan cuts every tensor into tiles of 1024 elements, counted from the tensor's first one, and gives for every tile the
// tensor that it belongs to; a wave takes one row of 256 elements of a tile, one access of four elements per lane and array.
// Tensors need the alignment of their elements only: the accesses are declared so, and the hardware takes them at any address.
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

#include "batch.hpp"
#include "elements.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr int kTensorTile = 1024;
constexpr int kTileRows = kTensorTile / kRow;
// Rows of 256 elements that a wave (the whole workgroup) takes of a tile.  32 bits: the step is bound by memory, and one row streams
// fastest: 1 | 2 | 4 rows, 335 M elements, bf16 gradients and copies, 1524 | 1639 | 1644 us, 25.6 M fp32 113 | 115 | 118.  8 bits: bound by the
// vector ALU, of which a block's maximum and reciprocals take less where blocks share them (blocks_most): 1 | 2 rows, 335 M elements, bf16
// parameters 701 | 565 us, 5 M 26.6 | 12.2, 109 M with fp32 parameters and bf16 copies 298 | 278, 49 small tensors 16.8 | 3.7 (four rows
// gained nothing on two in long launches and lost in small ones, 4.0 | 5.5).
constexpr int share_rows(int bits) { return bits == 8 ? 2 : 1; }
// Waves of a long launch with 32-bit states that share a CU (see lds_for_residency): more of them only spread what is in flight over more
// pages.  0 (as many as fit) | 11 | 12 | 13 | 16 waves: 335 M elements, bf16 gradients and copies, 1480 .. 1523 | 1433 | 1429 .. 1437 | 1456 | 1440 ..
// 1449 us, fp32 1479 | 1473 | 1467 | 1480 | 1497, bf16 parameters 1183 | 1200 | 1154 | 1138 | 1137; 109 M, bf16 gradients and copies, 477 | 466 | 472 |
// 474 | 480; 25.6 M fp32 111.1 | 109.6 | 110.4 | 110.8 | 110.7.  Shorter launches lose: 5 M, bf16 gradients and copies, 24.8 -> 25.1, 1 M fp32 6.8 -> 7.1.
// With 8-bit states, which need the waves for their arithmetic, 16 lose 10 % and more.
inline size_t adamw_lds(size_t tiles, int param_type, int bits)
{
    if (bits != 32 || tiles < (static_cast<size_t>(1) << 24) / kTensorTile) return 0;
    return lds_for_residency(param_type == BAGUA_F32 ? 12 : 16);
}
// The norm: one workgroup on a CU, with the waves that keep 32 KB of loads in flight there.  More waves read no faster, and each group more
// is one more that has to be counted at the end, 13 ns apiece: 335 M fp32 elements, 2048 groups of 4 waves 215 us, 512 of 8 197, 512 of
// 4 191, 256 of 8 192; bf16, 256 groups of 8 142, of 16 100; 25.6 M bf16, 2048 groups of 4 32.3, 256 of 16 14.3.
constexpr unsigned kNormGroups = kCus;
static_assert(kNormGroups <= kArriveMost, "groups that can be counted");
constexpr unsigned norm_waves(int type) { return type == BAGUA_F32 ? 8 : 16; }
// Up to four tiles a wave, one group alone is faster than several that have to meet: 20 K elements in 30 tensors 4.5 -> 3.5 us, 5 K 4.3 ->
// 3.4; 41 K in 49 tensors (eight tiles a wave) 4.9 -> 6.8.
inline unsigned norm_groups(size_t tiles, unsigned waves)
{
    return tiles <= 4 * waves ? 1 : static_cast<unsigned>(std::min<size_t>((tiles + waves - 1) / waves, kNormGroups));
}

struct TensorEntry {
    uint64_t grad, param, m, v, m_scale, v_scale, copy, numel;
    uint32_t first_tile, index;
    float decay;
    uint32_t unused;
};
static_assert(sizeof(TensorEntry) == 80, "the table is a whole number of 16-byte words");

// The plan's workspace: [counters | partial sums of the norm | entries | tensor of every tile].
constexpr size_t kPartialsAt = kArriveBytes, kEntriesAt = kPartialsAt + kNormGroups * sizeof(double);
struct TensorPlanView {
    uint32_t* counter;
    double* partial;
    const TensorEntry* entry;
    const uint32_t* tile_tensor;
};
inline TensorPlanView tensor_plan_view(const bagua_tensor_plan_t* p)
{
    unsigned char* w = static_cast<unsigned char*>(p->workspace);
    return TensorPlanView{reinterpret_cast<uint32_t*>(w), reinterpret_cast<double*>(w + kPartialsAt),
                          reinterpret_cast<const TensorEntry*>(w + kEntriesAt),
                          reinterpret_cast<const uint32_t*>(w + kEntriesAt + static_cast<size_t>(p->tensors) * sizeof(TensorEntry))};
}

// ---------------------------------------------------------------- four elements of a row
// Four elements of a lane, from element e on, as they are in memory.  kFull: all are there.  kCut: a lane that reaches over the end makes
// the last access that does not, and moves what it gets into place: no load stands behind a test, or each would be waited for before
// the next.  What lanes beyond the end hold means nothing.  `left`: valid elements; kFew: fewer than four, one by one.
template <typename T>
struct Four {
    typedef T v __attribute__((ext_vector_type(4)));
    typedef T u __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
enum Edge { kFull, kCut, kFew };
template <Edge EDGE, typename T>
__device__ __forceinline__ typename Four<T>::v fetch(const T* x, int e, int left)
{
    if (EDGE == kFew) {
        const int last = left - 1;
        return typename Four<T>::v{x[min(e, last)], x[min(e + 1, last)], x[min(e + 2, last)], x[min(e + 3, last)]};
    }
    return __builtin_nontemporal_load(reinterpret_cast<const typename Four<T>::u*>(x + (EDGE == kFull ? e : min(e, left - 4))));
}
template <Edge EDGE, typename T>
__device__ __forceinline__ T in_place(T q, int e, int left)
{
    if (EDGE != kCut) return q;
    const int skip = e - min(e, left - 4);
    const T s = (skip & 2) != 0 ? T{q.z, q.w, q.w, q.w} : q;
    return (skip & 1) != 0 ? T{s.y, s.z, s.w, s.w} : s;
}
template <Edge EDGE, typename T>
__device__ __forceinline__ void put(T* x, int e, int left, typename Four<T>::v v)
{
    if (EDGE == kFull || e + 4 <= left) {
        __builtin_nontemporal_store(static_cast<typename Four<T>::u>(v), reinterpret_cast<typename Four<T>::u*>(x + e));
    } else {
        if (e + 0 < left) x[e + 0] = v.x;
        if (e + 1 < left) x[e + 1] = v.y;
        if (e + 2 < left) x[e + 2] = v.z;
    }
}
template <int TYPE>
__device__ __forceinline__ f4 widened(typename Four<typename Elem<TYPE>::one>::v q)
{
    typedef Elem<TYPE> E;
    return f4{E::widen(q.x), E::widen(q.y), E::widen(q.z), E::widen(q.w)};
}
template <int TYPE>
__device__ __forceinline__ typename Four<typename Elem<TYPE>::one>::v narrowed(f4 v)
{
    typedef Elem<TYPE> E;
    return {E::narrow(v.x), E::narrow(v.y), E::narrow(v.z), E::narrow(v.w)};
}
// ---------------------------------------------------------------- E4M3 codes with a scale
typedef float f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f4 widen_codes(uint32_t w, float scale)
{
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    return f4{lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale};
}
// Scale of a block whose largest finite magnitude is `most`, and its reciprocal; a block that is (nearly) zero has neither.
struct Scale {
    float scale, inverse;
};
// 1 / b, correctly rounded (compared with the division for every mantissa), for b and 1 / b from 2^-126 on
__device__ __forceinline__ float reciprocal_in_range(float b)
{
    const float y = __builtin_amdgcn_rcpf(b);
    return __builtin_fmaf(y, __builtin_fmaf(-b, y, 1.0f), y);
}
template <bool FAST>
__device__ __forceinline__ Scale scale_of(float most)
{
    const float s = most * static_cast<float>(1.0 / 448.0);
    if (s < 0x1p-126f) return Scale{0.0f, 0.0f};
    return Scale{s, FAST ? reciprocal_in_range(s) : 1.0f / s};
}
__device__ __forceinline__ uint32_t nearest_codes(f4 y)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y.x, y.y, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y.z, y.w, w, true));
}
// y >= 0 times 2^-120 has E4M3's exponent field in the low bits of fp32's own (and its subnormals where fp32 has them), so
// the bits above the 20 lowest are the code, and what lies below them is how far y is on the way to the next one.  Two codes at a time
// in the halves of a register; a code is not below 1 where the root is above 0 (its upper half is not zero then) and not above 126.
// What is not finite gets code 127, E4M3's NaN, by not_finite.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 upper_halves(uint32_t a, uint32_t b) { return __builtin_bit_cast(u16x2, __builtin_amdgcn_perm(b, a, 0x07060302u)); }
__device__ __forceinline__ uint32_t code_bits(float y, uint32_t random) { return __float_as_uint(y * 0x1p-120f) + (random >> 12); }
__device__ __forceinline__ u16x2 two_codes(uint32_t a, uint32_t b, float ra, float rb)
{
    u16x2 one = u16x2{1, 1};
    asm("" : "+v"(one));      // (a minimum with a constant 1 becomes a comparison and a selection for each half)
    const u16x2 least = __builtin_elementwise_min(upper_halves(__float_as_uint(ra), __float_as_uint(rb)), one);
    const u16x2 c = __builtin_elementwise_min(upper_halves(a, b) >> static_cast<uint16_t>(4), u16x2{126, 126});
    return __builtin_elementwise_max(c, least);
}
// 127 in the bytes of those of four that are not finite, 0 in the others
__device__ __forceinline__ uint32_t not_finite(f4 x)
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= fabsf(x[i]) < INFINITY ? 0u : 127u << (8 * i);
    return w;
}
__device__ __forceinline__ f4 finite(f4 x)   // 0 for those that are not
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fabsf(x[i]) < INFINITY ? x[i] : 0.0f;
    return x;
}

__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}
constexpr uint32_t kGolden = 0x9E3779B9u;
__device__ __forceinline__ uint32_t turned(uint32_t h, int by) { return by == 0 ? h : __builtin_amdgcn_alignbit(h, h, 32 - by); }
// ANY: also what is no number, whose lower half may be so full that the random bits carry out of it.
template <bool ANY>
__device__ __forceinline__ uint16_t random_bf16(float x, uint32_t random)
{
    const uint16_t h = static_cast<uint16_t>((__float_as_uint(x) + (random >> 16)) >> 16);
    return ANY && x != x ? 0x7fc0 : h;
}

// ---------------------------------------------------------------- AdamW
struct AdamArgs {
    const float* clip;
    float beta1, omb1, beta2, omb2, root, eps, rate, decay;   // root: 1/sqrt(1-beta2^t), rate: lr/(1-beta1^t), decay: lr*weight_decay
    uint32_t seed;
    bool in_range;             // see root_in_range
};

// The largest magnitude of four (of numbers among them), as the bits of a number that is not negative: these are ordered as the numbers are, and across
// lanes the integer maximum comes without the instructions that make a NaN quiet.
__device__ __forceinline__ uint32_t most_of(f4 x) { return __float_as_uint(fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w)))); }
// Of four roots: none is negative, and what is no number (also the root of what has left fp32 in its scaled form, see root_in_range) is above
// all numbers in this order, where fmaxf would pass over it.
__device__ __forceinline__ uint32_t most_of_roots(f4 x)
{
    return max(max(__float_as_uint(x.x), __float_as_uint(x.y)), max(__float_as_uint(x.z), __float_as_uint(x.w)));
}
struct OpMaxU { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };

// The largest of each of K blocks of 256 values, of which every lane holds one: that of block k in the 64 / K lanes from k * 64 / K on.
// Two blocks are put side by side, in the halves of a register, so that they cost what one does.
template <int K>
__device__ __forceinline__ uint32_t blocks_most(const uint32_t (&x)[K])
{
    static_assert(K == 1 || K == 2, "");
    const OpMaxU op;
    auto halves = [&](uint32_t a, uint32_t b) { const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false); return op(r[0], r[1]); };
    auto rows = [&](uint32_t a, uint32_t b) { const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false); return op(r[0], r[1]); };
    const uint32_t v = halves(x[0], x[K - 1]);
    return row16_reduce(rows(v, v), op);
}

// Square root and quotient, correctly rounded, in 10 and 9 instruction slots instead of the 20 and 14 that they take for operands of any
// size: the step with 8-bit states is bound by the vector ALU.  The operands are kept in a range that allows it: first moments times
// 2^64, second ones times 2^64, roots times 2^32, which is exact, and the products with what belongs to them (rate, scales) undo it.
//   root:      y = rsqrt, g = t*y and h = y/2 are a few units off; t - g*g is exact in a fused operation, and g + h * that rounds to the
//              root: compared with sqrtf for every mantissa and both parities of the exponent.  Zero stays zero, as the reciprocal root is
//              taken of something above it.
//   quotient:  with the correctly rounded reciprocal of b (reciprocal_in_range) the remainder of
//              a quotient that is a unit off at most is exact, and adding its product with the reciprocal rounds to the quotient.
constexpr float kFirstScale = 0x1p64f, kSecondScale = 0x1p64f, kRootScale = 0x1p32f;
__device__ __forceinline__ float root_in_range(float t)   // 0, or 2^-90 <= t < 2^126; infinity gives no number
{
    const float y = __builtin_amdgcn_rsqf(fmaxf(t, 0x1p-90f)), g = t * y;
    return __builtin_fmaf(__builtin_fmaf(-g, g, t), 0.5f * y, g);
}
__device__ __forceinline__ float quotient_in_range(float a, float b)   // 2^-40 <= b < 2^21; a = 0, or 2^-101 <= |a| <= 2^84
{
    const float y = reciprocal_in_range(b), q = a * y;
    return __builtin_fmaf(-__builtin_fmaf(b, q, -a), y, q);             // (the remainder's sign keeps that of a zero)
}
// Blocks that keep to the ranges: first moments up to 2^20, roots up to 2^10 (in their scaled forms).  A root that is no number does not; a second
// moment of 2^64 and more is one of these.
// Of the step's own factors: with these a first moment is 0 or 2^-101 and more in its scaled form, for its terms are 0 or at least 2^-9 * 2^-62 * beta1 (the
// smallest code and scale) and 2^-85 * (1 - beta1), and their difference a multiple of the smaller one's last place; and the scale is taken out of
// the rate without rounding.
constexpr float kMostFirst = 0x1p84f, kMostRoot = 0x1p42f;
inline bool in_range(float beta1, float omb1, float root, float eps, float rate)
{
    return (beta1 == 0.0f || beta1 >= 0x1p-6f) && omb1 >= 0x1p-15f && root <= 0x1p10f && eps >= 0x1p-40f && eps <= 1.0f &&
           (rate == 0.0f || std::fabs(rate) >= 0x1p-62f);
}

// The general form's first moments: those below 2^-60 are held times kFirstScale, as all of the other form are, for fp32 ends for them as well; their bits
// are set in `small`.  Where no end is near every operation rounds alike with and without a scale, so that a result does not show in
// which form it was found.
__device__ __forceinline__ f4 first_moments(uint32_t codes, float scale, f4 g, float beta1, float omb1, uint32_t& small)
{
    const f4 scaled = widen_codes(codes, scale * kFirstScale) * beta1 + g * (omb1 * kFirstScale);
    f4 m = widen_codes(codes, scale) * beta1 + g * omb1;
    small = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (fabsf(scaled[i]) < kFirstScale * 0x1p-60f) {
            small |= 1u << i;
            m[i] = scaled[i];
        }
    return m;
}
// x, times the reciprocal of kFirstScale where the bit in `small` is set.
__device__ __forceinline__ f4 unscaled(f4 x, uint32_t small)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (small & 1u << i) != 0 ? x[i] * (1.0f / kFirstScale) : x[i];
    return x;
}
// rate * m / b.  Of a small one by something smaller yet the quotient is formed as it is, or it would leave fp32 at the other end.  One element
// after another: side by side the divisions take more registers than the other form needs.
__device__ __forceinline__ f4 updates(f4 m, f4 b, float rate, uint32_t small)
{
    f4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool scaled = (small & 1u << i) != 0, as_is = b[i] < 0x1p-40f;
        u[i] = m[i] / (scaled && as_is ? b[i] * kFirstScale : b[i]) * (scaled && !as_is ? rate * (1.0f / kFirstScale) : rate);
        __builtin_amdgcn_sched_barrier(0);
    }
    return u;
}

// K rows of 256 elements of a tile.  G, P, C: types of gradient, parameter and copy (C < 0: none).  e0: the first element
// in its tensor; left: elements from there on.  FAST (8 bits): with the functions above; false, and nothing done, where a block does not
// keep to their ranges.  kAny: 8 bits without FAST, of any operands.
template <int G, int P, int C, int BITS, int K, Edge EDGE, bool FAST>
__device__ __forceinline__ bool adamw_share(const TensorEntry& d, size_t e0, int lane, int left, float factor, const AdamArgs& a)
{
    static_assert(BITS == 8 || !FAST, "");
    constexpr bool kAny = BITS == 8 && !FAST;
    constexpr float kFirst = FAST ? kFirstScale : 1.0f, kSecond = FAST ? kSecondScale : 1.0f, kRoot = FAST ? kRootScale : 1.0f;
    typedef typename Elem<P>::one param_t;
    typedef typename Elem<G>::one grad_t;
    typedef typename std::conditional<BITS == 8, uint8_t, float>::type state_t;
    param_t* pp = table_ptr<param_t>(d.param) + e0;
    const grad_t* gp = table_ptr<const grad_t>(d.grad) + e0;
    state_t *mp = table_ptr<state_t>(d.m) + e0, *vp = table_ptr<state_t>(d.v) + e0;
    float ms[K], vs[K];
    if constexpr (BITS == 8) {
        const float *msp = table_ptr<const float>(d.m_scale) + e0 / kRow, *vsp = table_ptr<const float>(d.v_scale) + e0 / kRow;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int block = EDGE == kFull || k * kRow < left ? k : 0;     // of a block that is not there: any
            ms[k] = msp[block];
            vs[k] = vsp[block];
        }
    }
    typename Four<param_t>::v qp[K];
    typename Four<grad_t>::v qg[K];
    typename Four<state_t>::v qm[K], qv[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = k * kRow + lane * 4;
        qm[k] = fetch<EDGE>(mp, e, left);
        qv[k] = fetch<EDGE>(vp, e, left);
        qg[k] = fetch<EDGE>(gp, e, left);
        qp[k] = fetch<EDGE>(pp, e, left);
    }
    f4 m[K], r[K];
    uint32_t small[K], m_most[K], r_most[K], over = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = k * kRow + lane * 4;
        const f4 g = widened<G>(in_place<EDGE>(qg[k], e, left)) * factor;
        f4 v;
        if constexpr (BITS == 8) {
            const uint32_t codes = __builtin_bit_cast(uint32_t, in_place<EDGE>(qm[k], e, left));
            m[k] = kAny ? first_moments(codes, ms[k], g, a.beta1, a.omb1, small[k]) : widen_codes(codes, ms[k] * kFirst);
            v = widen_codes(__builtin_bit_cast(uint32_t, in_place<EDGE>(qv[k], e, left)), vs[k]);
            v = v * v;
        } else {
            m[k] = in_place<EDGE>(qm[k], e, left);
            v = in_place<EDGE>(qv[k], e, left);
        }
        if constexpr (!kAny) m[k] = m[k] * a.beta1 + g * (a.omb1 * kFirst);
        v = v * a.beta2 + (g * g) * a.omb2;
        if constexpr (BITS == 32) {
            put<EDGE>(mp, e, left, m[k]);
            put<EDGE>(vp, e, left, v);
        }
        if constexpr (FAST) {
            v = v * kSecond;
            r[k] = f4{root_in_range(v.x), root_in_range(v.y), root_in_range(v.z), root_in_range(v.w)};
        } else {
            r[k] = f4{sqrtf(v.x), sqrtf(v.y), sqrtf(v.z), sqrtf(v.w)};
        }
        if constexpr (BITS == 8) {
            if (EDGE != kFull) {
                clear_absent(m[k], e, left);
                clear_absent(r[k], e, left);
            }
            m_most[k] = most_of(kAny ? finite(unscaled(m[k], small[k])) : m[k]);
            r_most[k] = most_of_roots(FAST ? r[k] : finite(r[k]));
            if (FAST) over |= static_cast<uint32_t>(m_most[k] > __float_as_uint(kMostFirst)) | static_cast<uint32_t>(r_most[k] > __float_as_uint(kMostRoot));
        }
    }
    if constexpr (FAST) {
#pragma unroll
        for (int k = 0; k < K; ++k) asm volatile("" : "+v"(qp[k]));     // have arrived with the others, and are not asked for only now
        if (__any(over != 0)) return false;
    }
    const float decay = d.decay * a.decay, root = a.root * (1.0f / kRoot), rate = a.rate * (1.0f / kFirst);
    const uint32_t random = (static_cast<uint32_t>(e0 / 4) + lane) * kGolden + mix(d.index * kGolden + a.seed);
    uint32_t h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = k * kRow + lane * 4;
        f4 p = widened<P>(in_place<EDGE>(qp[k], e, left));
        const f4 b = r[k] * root + a.eps;
        f4 u;       // times the rate
        if constexpr (kAny) u = updates(m[k], b, rate, small[k]);
        else if constexpr (FAST) u = f4{quotient_in_range(m[k].x, b.x), quotient_in_range(m[k].y, b.y), quotient_in_range(m[k].z, b.z), quotient_in_range(m[k].w, b.w)} * rate;
        else u = m[k] / b * rate;
        p = p - (u + p * decay);
        if (BITS == 8 || P == BAGUA_BF16) h[k] = mix(random + static_cast<uint32_t>(k) * (kRow / 4 * kGolden));
        if constexpr (P == BAGUA_BF16) {
            const uint32_t w = mix(h[k] + kGolden);
            // (FAST: it comes from codes and bf16 parameters alone, whose lower half is empty)
            put<EDGE>(pp, e, left, h4{random_bf16<!FAST>(p.x, turned(w, 0)), random_bf16<!FAST>(p.y, turned(w, 8)), random_bf16<!FAST>(p.z, turned(w, 16)),
                                      random_bf16<!FAST>(p.w, turned(w, 24))});
        } else {
            put<EDGE>(pp, e, left, p);
        }
        if constexpr (C >= 0) put<EDGE>(table_ptr<typename Elem<C>::one>(d.copy) + e0, e, left, narrowed<C>(p));
    }
    if constexpr (BITS == 8) {
        constexpr int kLanes = kWave / K;      // that have a block's largest value
        const Scale sm = scale_of<FAST>(__uint_as_float(blocks_most<K>(m_most)) * (1.0f / kFirst)), sv = scale_of<FAST>(__uint_as_float(blocks_most<K>(r_most)) * (1.0f / kRoot));
        const float im = sm.inverse * (1.0f / kFirst), iv = sv.inverse * (1.0f / kRoot);
        auto of_block = [&](float x, int k) { return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(__float_as_int(x), k * kLanes))); };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = k * kRow + lane * 4;
            const f4 y = r[k] * of_block(iv, k);
            const u16x2 lo = two_codes(code_bits(y.x, turned(h[k], 0)), code_bits(y.y, turned(h[k], 8)), r[k].x, r[k].y);
            const u16x2 hi = two_codes(code_bits(y.z, turned(h[k], 16)), code_bits(y.w, turned(h[k], 24)), r[k].z, r[k].w);
            f4 inverse = of_block(im, k);
            if constexpr (kAny) inverse = unscaled(inverse, small[k]);
            uint32_t mc = nearest_codes(m[k] * inverse);
            uint32_t vc = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x06040200u);
            if constexpr (kAny) {      // (of FAST roots are finite, and so are first moments but for NaN, which the conversion keeps)
                mc |= not_finite(m[k]);
                vc |= not_finite(r[k]);
            }
            put<EDGE>(mp, e, left, __builtin_bit_cast(Four<uint8_t>::v, mc));
            put<EDGE>(vp, e, left, __builtin_bit_cast(Four<uint8_t>::v, vc));
        }
        if (lane % kLanes == 0 && (EDGE == kFull || lane / kLanes * kRow < left)) {
            table_ptr<float>(d.m_scale)[e0 / kRow + lane / kLanes] = sm.scale;
            table_ptr<float>(d.v_scale)[e0 / kRow + lane / kLanes] = sv.scale;
        }
    }
    return true;
}

// A share with 8-bit states, block by block: rare, operands out of range, or a tensor's last one to three elements.  It reads for itself, keeps nothing in
// registers up to here (nor through the loop: the lane is hidden from the compiler, which would form all its addresses in front of it), and
// does with few.
template <int G, int P, int C>
__device__ __forceinline__ void adamw_blocks(const TensorEntry& d, size_t e0, int lane, int left, float factor, const AdamArgs& a)
{
    asm volatile("" ::: "memory");
    int at = 0;
#pragma unroll 1
    for (; at + kRow <= left; at += kRow) {
        int l = lane;
        asm volatile("" : "+v"(l));
        adamw_share<G, P, C, 8, 1, kFull, false>(d, e0 + at, l, kRow, factor, a);
    }
    if (left - at >= 4) adamw_share<G, P, C, 8, 1, kCut, false>(d, e0 + at, lane, left - at, factor, a);
    else if (left - at > 0) adamw_share<G, P, C, 8, 1, kFew, false>(d, e0 + at, lane, left - at, factor, a);
}

// The step (in the order and with the roundings of bagua_hip.h): m = beta1 m + (1 - beta1) g, v = beta2 v + (1 - beta2) g^2,
// p = (1 - lr decay) p - rate m / (root sqrt(v) + eps), every element by itself, read and written once; with 8 bits a wave holds whole
// blocks, so that the new scale of a block is an exchange among its lanes and the states are
// not read again.  A workgroup is one wave, which ends as soon as its own rows are written.  32-bit states: bound by memory, 335 M elements with bf16
// gradients and copies 1436 us, 6.5 TB/s, 25.6 M fp32 109 us, 6.5 TB/s.  8-bit states with fp32 parameters and bf16 copies: near the memory's rate and the
// vector ALU's, 109 M, 278 us, 6.3 TB/s.  With bf16 parameters and gradients: bound by the vector ALU, 335 M, 563 to 600 us, 5.6 to 6.0 TB/s, with
// the clock that this load leaves (1.9 of 2.4 GHz; for some calls after it begins 1.3, and up to 880 us).
template <int G, int P, int C, int BITS>
__global__ void __launch_bounds__(kWave)
k_adamw(const TensorEntry* __restrict__ entries, const uint32_t* __restrict__ tile_tensor, AdamArgs a)
{
    constexpr int K = share_rows(BITS), kElements = K * kRow, kShares = kTensorTile / kElements;     // of a share; of a tile
    const uint32_t tile = blockIdx.x / kShares;
    const TensorEntry d = entries[tile_tensor[tile]];
    const size_t e0 = static_cast<size_t>(tile - d.first_tile) * kTensorTile + blockIdx.x % kShares * kElements;
    if (e0 >= d.numel) return;
    float factor = 1.0f;
    if (a.clip) {
        if (!(fabsf(a.clip[0]) < INFINITY)) return;
        factor = a.clip[1];
    }
    const int lane = threadIdx.x;
    const size_t left = d.numel - e0;
    if constexpr (BITS == 8) {
        if (left >= static_cast<size_t>(kElements)) {
            if (a.in_range && adamw_share<G, P, C, BITS, K, kFull, true>(d, e0, lane, kElements, factor, a)) return;
            adamw_blocks<G, P, C>(d, e0, lane, kElements, factor, a);
        } else {
            if (left >= 4 && a.in_range && adamw_share<G, P, C, BITS, K, kCut, true>(d, e0, lane, static_cast<int>(left), factor, a)) return;
            adamw_blocks<G, P, C>(d, e0, lane, static_cast<int>(left), factor, a);
        }
    } else if (left >= static_cast<size_t>(kElements)) {
        adamw_share<G, P, C, BITS, K, kFull, false>(d, e0, lane, kElements, factor, a);
    } else if (left >= 4) {
        adamw_share<G, P, C, BITS, K, kCut, false>(d, e0, lane, static_cast<int>(left), factor, a);
    } else {
        adamw_share<G, P, C, BITS, 1, kFew, false>(d, e0, lane, static_cast<int>(left), factor, a);
    }
}

// ---------------------------------------------------------------- norm
// Squares are exact in 64 bits and their sum loses nothing that an fp32 result could show, whatever the order; 64-bit additions
// run at half the rate of fp32 ones, a twentieth of what the loads leave time for.  A wave takes every so many-th tile, and looks up the
// next one while the present one is on its way; the workgroup that finishes last adds the groups' sums in a fixed order.  Bound by memory:
// 335 M fp32 elements 192 us, 7.0 TB/s; 41 K in 49 tensors 5.1 us: the launch, the table's entry and then
// the elements, the groups' meeting.
template <int G>
__device__ __forceinline__ double add_squares(double sum, const typename Four<typename Elem<G>::one>::v (&q)[kTileRows], int lane, int left)
{
    double part[4] = {sum, 0.0, 0.0, 0.0};
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        f4 x = widened<G>(q[i]);
        if (left < kTensorTile) clear_absent(x, i * kRow + lane * 4, left);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double y = static_cast<double>(x[j]);
            part[j] = __builtin_fma(y, y, part[j]);
        }
    }
    return (part[0] + part[1]) + (part[2] + part[3]);
}
template <int G>
__global__ void __launch_bounds__(kWave * norm_waves(G))
k_grad_norm(TensorPlanView plan, uint32_t tiles, double scale, double max_norm, float* __restrict__ out)
{
    typedef typename Elem<G>::one one;
    constexpr unsigned kNormWaves = norm_waves(G);
    const int lane = threadIdx.x & 63, wave = wave_index();
    const uint32_t step = gridDim.x * kNormWaves;
    double sum = 0.0;
    uint32_t tile = blockIdx.x * kNormWaves + wave;
    if (tile < tiles) {
        TensorEntry d = plan.entry[plan.tile_tensor[tile]];
        for (;;) {
            const size_t e0 = static_cast<size_t>(tile - d.first_tile) * kTensorTile;
            const one* g = table_ptr<const one>(d.grad) + e0;
            const int left = static_cast<int>(min(d.numel - e0, static_cast<uint64_t>(kTensorTile)));
            typename Four<one>::v q[kTileRows];
            if (left == kTensorTile) {
#pragma unroll
                for (int i = 0; i < kTileRows; ++i) q[i] = fetch<kFull>(g, i * kRow + lane * 4, left);
            } else if (left >= 4) {
#pragma unroll
                for (int i = 0; i < kTileRows; ++i) q[i] = fetch<kCut>(g, i * kRow + lane * 4, left);
            } else {
#pragma unroll
                for (int i = 0; i < kTileRows; ++i) q[i] = fetch<kFew>(g, i * kRow + lane * 4, left);
            }
            tile += step;
            const bool more = tile < tiles;
            if (more) d = plan.entry[plan.tile_tensor[tile]];
            if (left >= 4 && left < kTensorTile) {
#pragma unroll
                for (int i = 0; i < kTileRows; ++i) q[i] = in_place<kCut>(q[i], i * kRow + lane * 4, left);
            }
            sum = add_squares<G>(sum, q, lane, left);
            if (!more) break;
        }
    }
    __shared__ double part[kNormWaves];
    __shared__ bool last;
    auto group_sum = [&](double x) {      // in thread 0
        x = wave_sum(x);
        if (lane == 0) part[wave] = x;
        __syncthreads();
        x = threadIdx.x < kNormWaves ? part[threadIdx.x] : 0.0;
        return wave == 0 ? wave_sum(x) : 0.0;
    };
    sum = group_sum(sum);
    if (gridDim.x > 1) {
        if (threadIdx.x == 0) publish(plan.partial + blockIdx.x, sum);
        if (!last_to_arrive(plan.counter, &last)) return;
        sum = 0.0;
        static_assert(kNormGroups <= kWave * kNormWaves, "a thread for every group");
        sum = threadIdx.x < gridDim.x ? plan.partial[threadIdx.x] : 0.0;
        sum = group_sum(sum);
    }
    if (threadIdx.x != 0) return;
    const double n = scale * sqrt(sum);
    const float norm = static_cast<float>(n);
    out[0] = norm;
    const double c = max_norm / (n + 1e-6);
    out[1] = fabsf(norm) < INFINITY ? static_cast<float>(scale * (c < 1.0 ? c : 1.0)) : 0.0f;
}

inline size_t tiles_of(size_t numel) { return numel / kTensorTile + (numel % kTensorTile != 0); }
constexpr size_t kMaxTiles = kMaxGrid / kTileRows;   // one launch of single-wave rows holds them

inline size_t tensor_plan_bytes(size_t T, size_t tiles)
{
    return (kEntriesAt + T * sizeof(TensorEntry) + tiles * sizeof(uint32_t) + 15) & ~static_cast<size_t>(15);
}

}  // namespace bagua

using namespace bagua;

extern "C" size_t bagua_tensor_plan_bytes(const size_t* numel, size_t T)
{
    if (!numel || T == 0 || T > 0xfffffff0u) return 0;
    size_t tiles = 0;
    for (size_t t = 0; t < T && tiles <= kMaxTiles; ++t) tiles += tiles_of(numel[t]);
    return tiles > kMaxTiles ? 0 : tensor_plan_bytes(T, tiles);
}

extern "C" int bagua_tensor_plan(const size_t* numel, size_t T, const void* const* grad, int grad_type, void* const* param,
                                 int param_type, void* const* m, void* const* v, int state_bits, float* const* m_scale,
                                 float* const* v_scale, void* const* copy, int copy_type, const float* decay, void* workspace,
                                 size_t workspace_bytes, bagua_tensor_plan_t* plan, void* stream)
{
    if (!numel || T == 0 || !grad || !workspace || !plan || !type_ok(grad_type)) return BAGUA_ERR_INVALID_ARG;
    if (param) {
        if (!m || !v || (state_bits != 8 && state_bits != 32)) return BAGUA_ERR_INVALID_ARG;
        if (param_type != BAGUA_F32 && param_type != BAGUA_BF16) return BAGUA_ERR_INVALID_ARG;
        if (param_type == BAGUA_BF16 && (copy || grad_type == BAGUA_F16)) return BAGUA_ERR_INVALID_ARG;
        if ((state_bits == 8) != (m_scale != nullptr) || (state_bits == 8) != (v_scale != nullptr)) return BAGUA_ERR_INVALID_ARG;
        if (copy && copy_type != BAGUA_BF16 && copy_type != BAGUA_F16) return BAGUA_ERR_INVALID_ARG;
    } else if (m || v || m_scale || v_scale || copy || decay || state_bits != 0) {
        return BAGUA_ERR_INVALID_ARG;
    }
    if (T > 0xfffffff0u) return BAGUA_ERR_UNSUPPORTED;
    size_t tiles = 0;
    for (size_t t = 0; t < T; ++t) {
        if (numel[t] / kTensorTile >= kMaxTiles || (tiles += tiles_of(numel[t])) > kMaxTiles) return BAGUA_ERR_UNSUPPORTED;
    }
    const size_t bytes = tensor_plan_bytes(T, tiles);
    if (workspace_bytes < bytes) return BAGUA_ERR_INVALID_ARG;
    if (!aligned16(workspace)) return BAGUA_ERR_ALIGNMENT;
    try {
        std::vector<unsigned char> host(bytes, 0);
        TensorEntry* entry = reinterpret_cast<TensorEntry*>(host.data() + kEntriesAt);
        uint32_t* tile_tensor = reinterpret_cast<uint32_t*>(entry + T);
        RangeList rl;
        rl.writes(workspace, bytes);
        uint32_t tile = 0;
        for (size_t t = 0; t < T; ++t) {
            const size_t n = numel[t];
            TensorEntry& d = entry[t];
            d.numel = n;
            d.first_tile = tile;
            d.index = static_cast<uint32_t>(t);
            d.decay = decay ? decay[t] : 1.0f;
            if (!(std::fabs(d.decay) < INFINITY)) return BAGUA_ERR_INVALID_ARG;
            for (size_t i = tiles_of(n); i > 0; --i) tile_tensor[tile++] = static_cast<uint32_t>(t);
            if (n == 0) continue;
            const size_t blocks = (n + kRow - 1) / kRow, state = state_bits / 8;
            if (!grad[t]) return BAGUA_ERR_INVALID_ARG;
            if (!aligned_to(grad[t], type_bytes(grad_type))) return BAGUA_ERR_ALIGNMENT;
            rl.reads(grad[t], n * type_bytes(grad_type));
            d.grad = reinterpret_cast<uintptr_t>(grad[t]);
            if (!param) continue;
            if (!param[t] || !m[t] || !v[t] || (m_scale && (!m_scale[t] || !v_scale[t])) || (copy && !copy[t])) return BAGUA_ERR_INVALID_ARG;
            if (!aligned_to(param[t], type_bytes(param_type)) || !aligned_to(m[t], state) || !aligned_to(v[t], state) ||
                (m_scale && (!aligned4(m_scale[t]) || !aligned4(v_scale[t]))) || (copy && !aligned2(copy[t])))
                return BAGUA_ERR_ALIGNMENT;
            rl.writes(param[t], n * type_bytes(param_type));
            rl.writes(m[t], n * state);
            rl.writes(v[t], n * state);
            d.param = reinterpret_cast<uintptr_t>(param[t]);
            d.m = reinterpret_cast<uintptr_t>(m[t]);
            d.v = reinterpret_cast<uintptr_t>(v[t]);
            if (m_scale) {
                rl.writes(m_scale[t], blocks * sizeof(float));
                rl.writes(v_scale[t], blocks * sizeof(float));
                d.m_scale = reinterpret_cast<uintptr_t>(m_scale[t]);
                d.v_scale = reinterpret_cast<uintptr_t>(v_scale[t]);
            }
            if (copy) {
                rl.writes(copy[t], n * type_bytes(copy_type));
                d.copy = reinterpret_cast<uintptr_t>(copy[t]);
            }
        }
        if (!rl.disjoint()) return BAGUA_ERR_INVALID_ARG;
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (hipMemcpyAsync(workspace, host.data(), bytes, hipMemcpyHostToDevice, s) != hipSuccess) return BAGUA_ERR_LAUNCH;
        if (hipStreamSynchronize(s) != hipSuccess) return BAGUA_ERR_LAUNCH;   // `host` dies at return
    } catch (const std::bad_alloc&) {
        return BAGUA_ERR_UNSUPPORTED;   // more tensors than the host has memory to list
    }
    *plan = bagua_tensor_plan_t{workspace, tiles, static_cast<uint32_t>(T), grad_type, param ? param_type : -1, copy ? copy_type : -1, state_bits};
    return BAGUA_OK;
}

static bool plan_ok(const bagua_tensor_plan_t* plan)
{
    return plan && plan->workspace && aligned16(plan->workspace) && plan->tensors != 0 && plan->tiles <= kMaxTiles && type_ok(plan->grad_type);
}

extern "C" int bagua_grad_norm(const bagua_tensor_plan_t* plan, double grad_scale, double max_norm, float* out, void* stream)
{
    if (!plan_ok(plan) || !out || !(grad_scale >= 0.0 && grad_scale < INFINITY) || !(max_norm >= 0.0)) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(out)) return BAGUA_ERR_ALIGNMENT;
    const unsigned waves = norm_waves(plan->grad_type);
    const dim3 grid(norm_groups(plan->tiles, waves)), block(kWave * waves);
    const TensorPlanView view = tensor_plan_view(plan);
    auto* kernel = plan->grad_type == BAGUA_F32 ? k_grad_norm<BAGUA_F32> : plan->grad_type == BAGUA_BF16 ? k_grad_norm<BAGUA_BF16> : k_grad_norm<BAGUA_F16>;
    launch_kernel(kernel, grid, block, 0, static_cast<hipStream_t>(stream), view, static_cast<uint32_t>(plan->tiles), grad_scale, max_norm, out);
    return launch_status();
}

namespace bagua {
typedef void (*AdamKernel)(const TensorEntry*, const uint32_t*, AdamArgs);

template <int G, int BITS>
AdamKernel pick_adamw(int param_type, int copy_type)
{
    if constexpr (G != BAGUA_F16)
        if (param_type == BAGUA_BF16) return k_adamw<G, BAGUA_BF16, -1, BITS>;
    return copy_type == BAGUA_BF16 ? k_adamw<G, BAGUA_F32, BAGUA_BF16, BITS>
           : copy_type == BAGUA_F16 ? k_adamw<G, BAGUA_F32, BAGUA_F16, BITS> : k_adamw<G, BAGUA_F32, -1, BITS>;
}
template <int BITS>
AdamKernel pick_adamw(int grad_type, int param_type, int copy_type)
{
    return grad_type == BAGUA_F32 ? pick_adamw<BAGUA_F32, BITS>(param_type, copy_type)
           : grad_type == BAGUA_BF16 ? pick_adamw<BAGUA_BF16, BITS>(param_type, copy_type) : pick_adamw<BAGUA_F16, BITS>(param_type, copy_type);
}
}  // namespace bagua

extern "C" int bagua_adamw_step(const bagua_tensor_plan_t* plan, uint64_t step, double lr, double beta1, double beta2, double eps,
                                double weight_decay, const float* clip, uint32_t seed, void* stream)
{
    if (!plan_ok(plan) || (plan->state_bits != 8 && plan->state_bits != 32) || step == 0) return BAGUA_ERR_INVALID_ARG;
    if (!(std::fabs(lr) < INFINITY) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0 && eps < INFINITY) ||
        !(std::fabs(weight_decay) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(clip)) return BAGUA_ERR_ALIGNMENT;
    if (plan->tiles == 0) return BAGUA_OK;
    const TensorPlanView view = tensor_plan_view(plan);
    const uint32_t groups = static_cast<uint32_t>(plan->tiles * (kTileRows / share_rows(plan->state_bits)));
    const double t = static_cast<double>(step);
    AdamArgs a{clip, static_cast<float>(beta1), static_cast<float>(1.0 - beta1), static_cast<float>(beta2), static_cast<float>(1.0 - beta2),
               static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(beta2, t))), static_cast<float>(eps),
               static_cast<float>(lr / (1.0 - std::pow(beta1, t))), static_cast<float>(lr * weight_decay), seed, false};
    a.in_range = in_range(a.beta1, a.omb1, a.root, a.eps, a.rate);
    const AdamKernel kernel = plan->state_bits == 32 ? pick_adamw<32>(plan->grad_type, plan->param_type, plan->copy_type)
                                                     : pick_adamw<8>(plan->grad_type, plan->param_type, plan->copy_type);
    launch_kernel(kernel, dim3(groups), dim3(kWave), adamw_lds(plan->tiles, plan->param_type, plan->state_bits), static_cast<hipStream_t>(stream), view.entry,
                  view.tile_tensor, a);
    return launch_status();
}
