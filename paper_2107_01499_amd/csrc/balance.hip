// Balance loss of a mixture of experts (see bagua_hip.h): statistics over all workers' tokens, loss, and gradient of the logits.
//
// A row of logits lies in L = 2^i lanes of a wave, VEC * NV elements in each, so that a wave holds 64 / L rows at a time; a row's
// maximum and sums are exchanges among those lanes.  The last lanes of a row that does not fill them read its last elements once
// more (in bounds, whatever the length): these are left out of the sums by a factor of 0, and where they are stored both lanes
// store the same bits.
#include <cmath>
#include <type_traits>

#include "batch.hpp"
#include "elements.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr unsigned kBalanceGroups = kCus;    // most workgroups of the forward pass: the last one adds up their sums
static_assert(kBalanceGroups <= kArriveMost, "groups that can be counted");
constexpr int kGradWaves = 4;
constexpr uint32_t kGradMostWaves = 65536;   // of a launch of the backward pass

struct Workers {
    const void* logits[BAGUA_MAX_WORKERS];
    const void* ids[BAGUA_MAX_WORKERS];      // of the backward pass: where the gradients go
    const uint8_t* mask[BAGUA_MAX_WORKERS];
    uint32_t tokens[BAGUA_MAX_WORKERS];
    uint32_t first_tile[BAGUA_MAX_WORKERS + 1];   // a tile: the rows, of one worker, that a wave has in flight together
    uint32_t k;
};

template <typename T, int N>
struct Raw;   // N elements as they are in memory, with the alignment of one
template <typename T>
struct Raw<T, 1> {
    typedef T v __attribute__((ext_vector_type(1), aligned(sizeof(T))));
};
template <typename T>
struct Raw<T, 4> {
    typedef T v __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <typename T>
struct Raw<T, 8> {
    typedef T v __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// op over the L lanes of a row, in every one of them.
template <int L, typename T, typename F>
__device__ __forceinline__ T lanes_reduce(T v, const F& op)
{
    if (L >= 2) v = op(v, dpp<kXor1>(v));
    if (L >= 4) v = op(v, dpp<kXor2>(v));
    if (L >= 8) v = op(v, dpp<kHalfMirror>(v));
    if (L >= 16) v = op(v, dpp<kMirror>(v));
    if (L >= 32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        v = op(__builtin_bit_cast(T, static_cast<uint32_t>(r[0])), __builtin_bit_cast(T, static_cast<uint32_t>(r[1])));
    }
    if (L >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        v = op(__builtin_bit_cast(T, static_cast<uint32_t>(r[0])), __builtin_bit_cast(T, static_cast<uint32_t>(r[1])));
    }
    return v;
}

// The largest over the L lanes of a row.  Numbers are ordered as integers once those below zero have their other bits turned, and the
// integer maximum takes another lane's value in the same instruction, where that of numbers takes three to make a NaN quiet.
struct OpMaxI { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return static_cast<uint32_t>(max(static_cast<int32_t>(a), static_cast<int32_t>(b))); } };
__device__ __forceinline__ uint32_t in_order(uint32_t bits) { return bits ^ (static_cast<uint32_t>(static_cast<int32_t>(bits) >> 31) & 0x7fffffffu); }
template <int L>
__device__ __forceinline__ float lanes_most(float x)
{
    if (L == 1) return x;
    return __uint_as_float(in_order(lanes_reduce<L>(in_order(__float_as_uint(x)), OpMaxI())));
}

constexpr int kRor1 = 0x121, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;   // lane l reads l + 1, ... of its row of 16, around its end
// The sum over the lanes that hold the same elements of different rows: l, l + L, l + 2 L, ...
template <int L>
__device__ __forceinline__ float rows_sum(float v)
{
    if (L <= 8) v = v + dpp<kRor8>(v);
    if (L <= 4) v = v + dpp<kRor4>(v);
    if (L <= 2) v = v + dpp<kRor2>(v);
    if (L <= 1) v = v + dpp<kRor1>(v);
    if (L <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (L <= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// What a lane holds of a row.
template <int TYPE, int VEC, int L, int NV>
struct Row {
    typedef typename Elem<TYPE>::one one;
    typedef typename Raw<one, VEC>::v raw;
    static constexpr int kRows = kWave / L;       // rows of a unit
    raw q[NV];

    // Elements of vector j of the lane: from at(j) on; slot(j): what it would be if the row filled the lanes.
    static __device__ __forceinline__ int slot(int j) { return (j * L + static_cast<int>(threadIdx.x % L)) * VEC; }
    static __device__ __forceinline__ int at(int j, int experts) { return min(slot(j), experts - VEC); }

    __device__ __forceinline__ void load(const one* row, int experts, bool there)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            q[j] = raw(0);
            if (there) q[j] = __builtin_nontemporal_load(reinterpret_cast<const raw*>(row + at(j, experts)));
        }
    }
    __device__ __forceinline__ void keep_if(bool there)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) q[j] = there ? q[j] : raw(0);
    }
    // The lane's elements as fp32, and the row's largest.
    __device__ __forceinline__ float largest(float (&x)[NV][VEC]) const
    {
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                x[j][i] = Elem<TYPE>::widen(q[j][i]);
                most = fmaxf(most, x[j][i]);
            }
        return lanes_most<L>(most);
    }
    // x = exp(x - most).  Not HUGE: log2(e) times both, and then the difference, in one fused operation; the rounding of the product with `most`
    // is the same factor on all of a row, which the sum takes out again as long as it is near 1.  HUGE: the difference first, which costs an
    // operation more, and is right whatever the magnitude.
    template <bool HUGE>
    static __device__ __forceinline__ void exponentials(float (&x)[NV][VEC], float most)
    {
        constexpr float kLog2e = 1.44269504088896340736f;
        const float top = most == -INFINITY ? 0.0f : most, shift = -top * kLog2e;   // (nothing but -infinity: all become 0)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                x[j][i] = __builtin_amdgcn_exp2f(HUGE ? (x[j][i] - top) * kLog2e : __builtin_fmaf(x[j][i], kLog2e, shift));
    }
    static __device__ __forceinline__ float reciprocal_sum(const float (&own)[NV][VEC], const float (&e)[NV][VEC])
    {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum = __builtin_fmaf(e[j][i], own[j][i], sum);
        sum = lanes_reduce<L>(sum, OpAddF());
        const float r = __builtin_amdgcn_rcpf(sum);
        return sum == 0.0f ? 0.0f : __builtin_fmaf(__builtin_fmaf(-sum, r, 1.0f), r, r);
    }
    static __device__ __forceinline__ void owned(int experts, float (&own)[NV][VEC])
    {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) own[j][i] = j < NV / 2 || at(j, experts) + i >= slot(j) ? 1.0f : 0.0f;   // (rows are longer than half the lanes)
    }
};

// exp(x - largest) of a wave's U times rows, without a branch between them that would keep their exchanges from filling each other's gaps.
template <typename R, int U, int NV, int VEC>
__device__ __forceinline__ void exponentials_of(float (&e)[U][NV][VEC], const float (&most)[U], bool may_be_huge)
{
    bool huge = false;
#pragma unroll
    for (int u = 0; u < U; ++u) huge |= fabsf(most[u]) > 0x1p20f;
    // up to 2^20 the shift is off by 2^-4 at most, half a unit of its last place: 4 % on all of a row.  Beyond 2^31 it would be off by more than 128,
    // and leave nothing but zeros or infinities of the row
    if (may_be_huge && __any(huge)) {
#pragma unroll
        for (int u = 0; u < U; ++u) R::template exponentials<true>(e[u], most[u]);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) R::template exponentials<false>(e[u], most[u]);
    }
}

// The workers' table with worker i in lane i: which worker has a tile is one comparison and a count of bits, and what belongs to it
// is read from its lane.  (From the arguments that is a chain of scalar loads, a new one for every worker that is passed over.)
struct LaneTable {
    uint32_t first_tile, tokens;
    uint64_t logits, other, mask;
    __device__ __forceinline__ explicit LaneTable(const Workers& ws)
    {
        const uint32_t i = threadIdx.x & (BAGUA_MAX_WORKERS - 1);
        first_tile = ws.first_tile[i];
        tokens = ws.tokens[i];
        logits = reinterpret_cast<uintptr_t>(ws.logits[i]);
        other = reinterpret_cast<uintptr_t>(ws.ids[i]);
        mask = reinterpret_cast<uintptr_t>(ws.mask[i]);
    }
    static __device__ __forceinline__ uint32_t of(uint32_t v, uint32_t w) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), static_cast<int>(w))); }
    static __device__ __forceinline__ uint64_t of(uint64_t v, uint32_t w)
    {
        return static_cast<uint64_t>(of(static_cast<uint32_t>(v >> 32), w)) << 32 | of(static_cast<uint32_t>(v), w);
    }
    // The last worker whose tiles begin at `tile` or before it (of workers without tokens, which begin there too, the one behind them).
    __device__ __forceinline__ uint32_t worker(uint32_t tile) const
    {
        return static_cast<uint32_t>(__popc(static_cast<uint32_t>(__ballot(first_tile <= tile)))) - 1u;
    }
};
static_assert(BAGUA_MAX_WORKERS == 32, "a worker for each lane of half a wave");

// A tile's rows: of one worker, from token t0 on; all of it wave-uniform.
struct Tile {
    uint64_t logits, other, mask;
    uint32_t t0, rows;         // rows: that exist, one at least
    bool there;                // false: beyond the last tile; its addresses are those of the last one, and can be read
};
template <int ROWS>
__device__ __forceinline__ Tile tile_of(const LaneTable& table, uint32_t tile, uint32_t tiles)
{
    Tile k;
    k.there = tile < tiles;
    tile = k.there ? tile : tiles - 1;
    const uint32_t w = table.worker(tile);
    k.t0 = (tile - LaneTable::of(table.first_tile, w)) * ROWS;
    k.rows = min(static_cast<uint32_t>(ROWS), LaneTable::of(table.tokens, w) - k.t0);
    k.logits = LaneTable::of(table.logits, w);
    k.other = LaneTable::of(table.other, w);
    k.mask = LaneTable::of(table.mask, w);
    return k;
}
// Whether a row of the tile counts, or an address to read instead where there is no mask or no such row.
__device__ __forceinline__ uint8_t flag_of(const Tile& k, uint32_t row)
{
    const uint8_t* p = k.mask ? table_ptr<const uint8_t>(k.mask) + k.t0 + min(row, k.rows - 1) : table_ptr<const uint8_t>(k.logits);
    return *p;
}
__device__ __forceinline__ bool counts_in(const Tile& k, uint32_t row, uint8_t flag) { return k.there && row < k.rows && (k.mask == 0 || flag != 0); }

struct BalanceOut {
    int32_t* counts;
    float *prob, *loss, *weight;
    double alpha;
    int experts, top_k;
};

// Loss and weights from the sums, by one workgroup; thread i has experts i, i + THREADS, ...  `part`: one double per wave.
template <int THREADS, typename COUNT, typename PROB>
__device__ __forceinline__ void balance_loss(const BalanceOut& o, int32_t tokens, const COUNT& count, const PROB& prob, double* part)
{
    const int waves = min(THREADS, o.experts + kWave - 1) / kWave;     // that have an expert: the others would take the time of these
    double sum = 0.0;
    if (wave_index() < waves) {
        const double n = tokens, scale = tokens > 0 ? o.alpha * o.experts / (static_cast<double>(o.top_k) * n * n) : 0.0;
        for (int e = threadIdx.x; e < o.experts; e += THREADS) {
            const double w = scale * count(e), p = prob(e);
            o.weight[e] = static_cast<float>(w);
            if (tokens > 0) sum += w * p;
        }
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x / kWave] = sum;
    }
    if (waves > 1) __syncthreads();
    if (threadIdx.x >= kWave) return;
    if (waves > 1) sum = wave_sum(static_cast<int>(threadIdx.x) < waves ? part[threadIdx.x] : 0.0);
    if (threadIdx.x == 0) o.loss[0] = static_cast<float>(sum);
}

constexpr int kSumFloats = 8192;   // of LDS for the waves' sums
// Rows of `experts` sums that fit there, of as many waves at a time.
__host__ __device__ constexpr int sum_rows(int waves, int experts)
{
    int rows = waves;
    while (rows > 1 && rows * experts > kSumFloats) rows /= 2;
    return rows;
}

// The forward pass: over the rows that count, the sums of softmax(row)[e] and how often expert e was chosen.  A wave takes one tile after another
// and keeps its sums in registers, a group joins its waves' in LDS, and the group that ends last adds up the groups' in a fixed order and forms
// the loss, so that one launch reads each logit and choice once and no sum depends on which group came first.  Bound by what comes before and
// after the loop, not by memory: 8 workers' 32768 rows of 64, bf16, 20.0 us, where the 41 MB are read in 6: the launch, the wait for the first rows
// and the meeting of 256 groups are 9 to 12.  Long ones (524288 x 256, bf16, 65 to 67 us, 4.5 TB/s) use half of the vector ALU's slots and two thirds of
// the memory's rate, with three waves on a SIMD: what bounds them is not shown.
// Dynamic LDS: float sums[sum_rows][experts], then uint32 counters[(experts + 1) << lg]: 2^lg copies of each, one of
// which a lane adds to, so that popular experts are not waited for.  Workspace: counters (last_to_arrive), then every workgroup's sums and counts.
template <int TYPE, int VEC, int L, int NV, int UNROLL, int WAVES>
__global__ void __launch_bounds__(kWave * WAVES)
k_balance_stats(Workers ws, size_t ld, size_t ids_ld, int id_bytes, uint32_t tiles, uint32_t per_k, int lg, uint32_t* workspace, BalanceOut o)
{
    typedef Row<TYPE, VEC, L, NV> R;
    constexpr int kThreads = kWave * WAVES;
    extern __shared__ float sums[];
    __shared__ double part[WAVES];
    __shared__ bool last;
    const int experts = o.experts, lane = threadIdx.x & 63, wave = wave_index(), rows_of_sums = sum_rows(WAVES, experts);
    uint32_t* counters = reinterpret_cast<uint32_t*>(sums + rows_of_sums * experts);
    const LaneTable table(ws);
    for (int i = threadIdx.x; i < (experts + 1) << lg; i += kThreads) counters[i] = 0;
    __syncthreads();

    float own[NV][VEC], acc[NV][VEC];
    R::owned(experts, own);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[j][i] = 0.0f;
    // A tile's choices are taken one after another, 64 at a time, whatever rows they belong to; kAhead times 64 are asked for with the rows.
    constexpr int kRows = UNROLL * R::kRows, kAhead = NV == 1 ? 2 : 1;
    const uint32_t waves = gridDim.x * WAVES, top = static_cast<uint32_t>(o.top_k), own_row = static_cast<uint32_t>(lane) / L;
    struct Choice {
        uint64_t id;
        uint8_t flag;
    };
    auto row_of = [&](uint32_t i) { return per_k ? __umulhi(i, per_k) : i; };
    auto choice = [&](const Tile& k, uint32_t i) {      // beyond the last one: the last
        i = min(i, k.rows * top - 1);
        const uint32_t r = row_of(i);
        const size_t at = (k.t0 + r) * ids_ld + (i - r * top);
        return Choice{id_bytes == 8 ? table_ptr<const uint64_t>(k.other)[at] : static_cast<uint64_t>(static_cast<int64_t>(table_ptr<const int32_t>(k.other)[at])),
                      flag_of(k, r)};
    };
    auto count = [&](const Tile& k, Choice c, uint32_t i) {
        if (c.id < static_cast<uint64_t>(experts) && counts_in(k, row_of(i), c.flag))
            atomicAdd(counters + (static_cast<uint32_t>(c.id) << lg) + (lane & ((1 << lg) - 1)), 1u);
    };
    R row[UNROLL];
    uint8_t flag[UNROLL];
    Choice ahead[kAhead];
    // No load stands behind a test of another one of the tile except the rows behind their flags, from a wave's second tile on.
    auto ask = [&](const Tile& k) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) flag[u] = flag_of(k, u * R::kRows + own_row);
#pragma unroll
        for (int s = 0; s < kAhead; ++s) ahead[s] = choice(k, s * kWave + lane);
    };
    bool counts[UNROLL];
    auto ask_rows = [&](const Tile& k) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t r = u * R::kRows + own_row;
            counts[u] = counts_in(k, r, flag[u]);
            row[u].load(table_ptr<const typename R::one>(k.logits) + (k.t0 + min(r, k.rows - 1)) * ld, experts, counts[u]);
        }
    };
    uint32_t tokens = 0, tile = blockIdx.x * WAVES + wave;
    if (tile < tiles) {
        Tile k = tile_of<kRows>(table, tile, tiles);
        ask(k);
        // The first tile's rows do not wait for their flags: those that do not count are read and dropped.  32768 x 128, bf16, 15.3 -> 14.5 us.
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            row[u].load(table_ptr<const typename R::one>(k.logits) + (k.t0 + min(u * R::kRows + own_row, k.rows - 1)) * ld, experts, true);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            counts[u] = counts_in(k, u * R::kRows + own_row, flag[u]);
            row[u].keep_if(counts[u]);
        }
        while (k.there) {
            // the present tile's rows arrive; the next one's flags and choices, and then its rows, are on their way while the present
            // one is worked on
            tile += waves;
            const Tile next = tile_of<kRows>(table, tile, tiles);
            float e[UNROLL][NV][VEC], most[UNROLL];
            bool counted[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                counted[u] = counts[u];
                most[u] = row[u].largest(e[u]);
                tokens += __popcll(__ballot(counts[u])) / L;
            }
#pragma unroll
            for (int s = 0; s < kAhead; ++s) count(k, ahead[s], s * kWave + lane);
            for (uint32_t i0 = kAhead * kWave; i0 < k.rows * top; i0 += kAhead * kWave) {
                Choice more[kAhead];
#pragma unroll
                for (int s = 0; s < kAhead; ++s) more[s] = choice(k, i0 + s * kWave + lane);
#pragma unroll
                for (int s = 0; s < kAhead; ++s) count(k, more[s], i0 + s * kWave + lane);
            }
            ask(next);
            exponentials_of<R>(e, most, TYPE != BAGUA_F16);
            ask_rows(next);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float inverse = R::reciprocal_sum(own, e[u]);
                inverse = counted[u] ? inverse : 0.0f;      // (rows that do not count were read as zeros)
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[j][i] = __builtin_fmaf(e[u][j][i], inverse, acc[j][i]);
            }
            k = next;
        }
    }
    if (lane == 0 && tokens) atomicAdd(counters + (experts << lg), tokens);

    // the rows of a wave, then the waves: as many as there is room for side by side, the others on top of them
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[j][i] = rows_sum<L>(acc[j][i]);
    float* mine = sums + wave % rows_of_sums * experts;
    for (int first = 0; first < WAVES; first += rows_of_sums) {
        if (wave >= first && wave < first + rows_of_sums && lane < L) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (own[j][i] != 0.0f) mine[R::at(j, experts) + i] = first == 0 ? acc[j][i] : mine[R::at(j, experts) + i] + acc[j][i];
        }
        __syncthreads();
    }
    auto wave_sums = [&](int e) {
        float s = sums[e];
#pragma unroll 4
        for (int r = 1; r < rows_of_sums; ++r) s += sums[r * experts + e];
        return s;
    };
    auto copies = [&](int e) {
        uint32_t c = 0;
#pragma unroll 8
        for (int r = 0; r < 1 << lg; ++r) c += counters[(e << lg) + r];
        return c;
    };
    auto finish = [&](auto&& count, auto&& prob) {       // by what the whole workgroup sees
        auto count_out = [&](int e) {
            const int32_t c = static_cast<int32_t>(count(e));
            o.counts[e] = c;
            return static_cast<double>(c);
        };
        auto prob_out = [&](int e) {
            const float p = prob(e);
            o.prob[e] = p;
            return static_cast<double>(p);
        };
        if (threadIdx.x == 0) o.counts[experts] = static_cast<int32_t>(count(experts));
        if (o.loss) {
            balance_loss<kThreads>(o, static_cast<int32_t>(count(experts)), count_out, prob_out, part);
        } else {
            for (int e = threadIdx.x; e < experts; e += kThreads) {
                count_out(e);
                prob_out(e);
            }
        }
    };
    if (gridDim.x == 1) {
        finish(copies, wave_sums);
        return;
    }

    // Pairs of a sum and a count, [group][experts], behind them those of the clusters of groups, and behind these the tokens of both.
    const uint32_t pair_rows = gridDim.x + clusters();
    uint64_t* pairs = reinterpret_cast<uint64_t*>(workspace + kArriveBytes / sizeof(uint32_t));
    uint32_t* pair_tokens = reinterpret_cast<uint32_t*>(pairs + static_cast<size_t>(pair_rows) * experts);
    auto publish_row = [&](uint32_t row, auto&& count, auto&& prob) {
        for (int e = threadIdx.x; e < experts; e += kThreads)
            publish(pairs + static_cast<size_t>(row) * experts + e, static_cast<uint64_t>(count(e)) << 32 | __float_as_uint(prob(e)));
        if (threadIdx.x == 0) publish(pair_tokens + row, static_cast<uint32_t>(count(experts)));
    };
    __shared__ double slice_sum[kThreads];
    __shared__ uint32_t slice_count[kThreads];
    int width = 1;                                          // threads of a slice, a power of two
    while (width < experts && width < kThreads) width *= 2;
    const uint32_t slices = kThreads / width, slice = threadIdx.x / width, column = threadIdx.x & (width - 1);
    // The sums over `n` rows of pairs, by as many threads per expert as there are, in a fixed order: in sums and counters.  One group does it
    // while the chip waits, so it takes few instructions (32-bit indexes, no more rows asked for than there are, no test where all are there) and
    // the lanes of one expert together first: with the loss left to the waves that have experts, 4096 x 64, bf16, 11.7 -> 10.0 us, 500 x 8 5.4 -> 5.0.
    auto together = [&](uint32_t row, uint32_t n) {
        static_assert(kThreads >= kBalanceGroups, "a thread for every row");
        uint32_t all = threadIdx.x < n ? pair_tokens[row + threadIdx.x] : 0;
        for (int e0 = 0; e0 < experts; e0 += width) {
            const int e = e0 + column;
            const uint32_t step = slices * experts, first = row * experts + min(e, experts - 1), last_one = first + (n - 1) * experts;
            uint32_t at = first + slice * experts, taken = 0;   // taken: rows, by all slices
            double s = 0.0;
            uint32_t c = 0;
            // N rows of a slice; without a test before a load, or each would be waited for
            auto add = [&](auto batch, auto all_there) {
                constexpr int N = decltype(batch)::value;
                uint64_t pair[N];
#pragma unroll
                for (int i = 0; i < N; ++i) pair[i] = pairs[decltype(all_there)::value ? at + i * step : min(at + i * step, last_one)];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (!decltype(all_there)::value && taken + i * slices + slice >= n) pair[i] = 0;
                    s += __uint_as_float(static_cast<uint32_t>(pair[i]));
                    c += static_cast<uint32_t>(pair[i] >> 32);
                }
                at += N * step;
                taken += N * slices;
            };
            while (taken + 16 * slices <= n) add(std::integral_constant<int, 16>(), std::true_type());
            if (taken + 4 * slices < n) add(std::integral_constant<int, 16>(), std::false_type());
            else if (taken + slices < n) add(std::integral_constant<int, 4>(), std::false_type());
            else if (taken < n) add(std::integral_constant<int, 1>(), std::false_type());
            for (int d = kWave / 2; d >= width; d /= 2) {
                s += __shfl_xor(s, d);
                c += __shfl_xor(c, d);
            }
            const uint32_t parts = kThreads / max(width, kWave), mine = threadIdx.x / max(width, kWave) * width + column;
            slice_sum[mine] = s;                                // (lanes of one expert have the same)
            slice_count[mine] = c;
            __syncthreads();
            if (slice == 0 && e < experts) {
#pragma unroll 4
                for (uint32_t i = 1; i < parts; ++i) {
                    s += slice_sum[i * width + column];
                    c += slice_count[i * width + column];
                }
                sums[e] = static_cast<float>(s);
                counters[e] = c;
            }
            if (e0 == 0 && threadIdx.x == 0) counters[experts] = 0;
            __syncthreads();
        }
        if (wave * kWave < static_cast<int>(n)) {
            all = lanes_reduce<kWave>(all, [](uint32_t a, uint32_t b) { return a + b; });
            if (lane == 0 && all) atomicAdd(counters + experts, all);
        }
        __syncthreads();
    };
    auto summed_count = [&](int e) { return counters[e]; };
    auto summed_prob = [&](int e) { return sums[e]; };
    publish_row(blockIdx.x, copies, wave_sums);
    // In two steps where one group would read too much: 250 K x 512, fp16, 73.5 -> 65 us, but 8 x 32768 x 64 20.8 -> 25.3, 524288 x 256 66.8 -> 67.1.
    if (experts <= 256 || gridDim.x <= kArriveDirect) {
        if (!last_to_arrive(workspace, &last)) return;
        together(0, gridDim.x);
    } else {
        if (!last_of_cluster(workspace, &last)) return;
        const uint32_t cluster = blockIdx.x / kArriveGroup;
        together(cluster * kArriveGroup, cluster_groups(cluster));
        publish_row(gridDim.x + cluster, summed_count, summed_prob);
        if (!last_cluster(workspace, &last)) return;
        together(gridDim.x, clusters());
    }
    finish(summed_count, summed_prob);
}

__global__ void __launch_bounds__(256)
k_balance_loss(const int32_t* __restrict__ counts, const float* __restrict__ prob, BalanceOut o)
{
    __shared__ double part[4];
    balance_loss<256>(o, counts[o.experts], [&](int e) { return static_cast<double>(counts[e]); },
                      [&](int e) { return static_cast<double>(prob[e]); }, part);
}

// The backward pass: with p the softmax of a row and w[e] = coefficient * count[e], the gradient is p[e] * (w[e] - sum of w[j] * p[j]), 0 in a
// row that does not count.  The probabilities are formed again from the logits, which costs no second reading: a row stays in its lanes from
// the one load to the one store, so the pass reads and writes each logit once.  Bound by memory: 524288 rows of 256, bf16, 85.1 us, 6.3 TB/s,
// where a copy of as many bytes takes 78; 4 x 4099 rows of 60, fp32, 4.6 us, of which all but 1 is launching.
template <int TYPE, int VEC, int L, int NV, int UNROLL>
__global__ void __launch_bounds__(kWave * kGradWaves, NV == 1 ? 7 : 1)
k_balance_grad(Workers ws, size_t ld, size_t ld_out, uint32_t tiles, int experts, const float* __restrict__ weight, const float* __restrict__ upstream)
{
    typedef Row<TYPE, VEC, L, NV> R;
    typedef typename R::one one;
    const LaneTable table(ws);
    const uint32_t waves = gridDim.x * kGradWaves;
    const float up = upstream ? upstream[0] : 1.0f;
    float own[NV][VEC], g[NV][VEC];
    R::owned(experts, own);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[j][i] = weight[R::at(j, experts) + i];
    const uint32_t own_row = (threadIdx.x & 63) / L;
    for (uint32_t tile = blockIdx.x * kGradWaves + wave_index(); tile < tiles; tile += waves) {
        const Tile k = tile_of<UNROLL * R::kRows>(table, tile, tiles);
        R row[UNROLL];
        uint8_t flag[UNROLL];
        bool counts[UNROLL];
        float e[UNROLL][NV][VEC], most[UNROLL];
        auto token = [&](int u) { return k.t0 + min(static_cast<uint32_t>(u) * R::kRows + own_row, k.rows - 1); };
        if (k.mask == 0) {                                      // nothing to wait for: 524288 x 256, bf16, 89.9 -> 85.1 us, 32768 x 128 6.1 -> 5.2
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                counts[u] = u * R::kRows + own_row < k.rows;
                row[u].load(table_ptr<const one>(k.logits) + token(u) * ld, experts, true);
            }
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) flag[u] = flag_of(k, u * R::kRows + own_row);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                counts[u] = counts_in(k, u * R::kRows + own_row, flag[u]);
                row[u].load(table_ptr<const one>(k.logits) + token(u) * ld, experts, counts[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) most[u] = row[u].largest(e[u]);
        exponentials_of<R>(e, most, TYPE != BAGUA_F16);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float dot = 0.0f;
            const float inverse = R::reciprocal_sum(own, e[u]);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) dot = __builtin_fmaf(e[u][j][i], g[j][i] * own[j][i], dot);
            // (rows that do not count were read as zeros, or do not exist and are not stored)
            const float scale = counts[u] ? inverse * up : 0.0f, shift = -(lanes_reduce<L>(dot, OpAddF()) * inverse) * scale;
            one* out = table_ptr<one>(k.other) + token(u) * ld_out;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                typename R::raw q;
#pragma unroll
                for (int i = 0; i < VEC; ++i) q[i] = Elem<TYPE>::narrow(e[u][j][i] * __builtin_fmaf(g[j][i], scale, shift));
                if (u * R::kRows + own_row < k.rows) __builtin_nontemporal_store(q, reinterpret_cast<typename R::raw*>(out + R::at(j, experts)));
            }
        }
    }
}

// Calls f with the layout of a row of `experts` elements: VEC, L, NV, and units that a wave has in flight together.
template <int VEC_, int L_, int NV_, int UNROLL_, int WAVES_ = 16>
struct Layout {
    static constexpr int VEC = VEC_, L = L_, NV = NV_, UNROLL = UNROLL_, WAVES = WAVES_, GRAD_UNROLL = NV_ == 1 ? 2 : 1;   // WAVES: of a workgroup of the forward pass
};
// The forward pass of 16-bit rows beyond 128 elements: twice the elements in half the lanes take half the exchanges (524288 x 256, bf16, 78 -> 67 us,
// 250 K x 512, fp16, 82 -> 72; 8 x 32768 x 64 loses, 21.8 -> 22.0).
template <int V, bool FORWARD, typename F>
inline void with_vectors(int experts, const F& f)
{
    if (experts < V) {
        if (experts <= 1) f(Layout<1, 1, 1, 4>());
        else if (experts <= 2) f(Layout<1, 2, 1, 4>());
        else if (experts <= 4) f(Layout<1, 4, 1, 4>());
        else f(Layout<1, 8, 1, 4>());
    } else if (experts <= V) f(Layout<V, 1, 1, 4>());
    else if (experts <= 2 * V) f(Layout<V, 2, 1, 4>());
    else if (experts <= 4 * V) f(Layout<V, 4, 1, 4>());
    else if (experts <= 8 * V) f(Layout<V, 8, 1, 4>());
    else if (experts <= 16 * V) f(Layout<V, 16, 1, 4>());
    else if (experts <= 32 * V) f(std::conditional_t<FORWARD && V == 8, Layout<V, 16, 2, 2>, Layout<V, 32, 1, 4>>());
    else if (experts <= 64 * V) f(std::conditional_t<FORWARD && V == 8, Layout<V, 32, 2, 2>, Layout<V, 64, 1, 4>>());
    else if (experts <= 128 * V) f(Layout<V, 64, 2, 2>());
    else if (experts <= 256 * V) f(Layout<V, 64, 4, 1, V == 8 ? 8 : 16>());
    else if constexpr (V == 4) f(Layout<V, 64, 8, 1, 8>());
}
// 16 bytes of a row in a lane: a wider vector of fp32 is two accesses that each leave out every other 16 bytes, and a store of half a
// line costs a whole one (gradient of 1 M rows of 64, fp32: eight elements 101.8 us, four 82).
template <bool FORWARD, typename F>
inline void with_layout(int dtype, int experts, const F& f)
{
    if (dtype == BAGUA_F32) with_vectors<4, FORWARD>(experts, [&](auto layout) { f(layout, std::integral_constant<int, BAGUA_F32>()); });
    else if (dtype == BAGUA_BF16) with_vectors<8, FORWARD>(experts, [&](auto layout) { f(layout, std::integral_constant<int, BAGUA_BF16>()); });
    else with_vectors<8, FORWARD>(experts, [&](auto layout) { f(layout, std::integral_constant<int, BAGUA_F16>()); });
}
// Arguments that both passes have, and the workers' table.
inline int balance_check(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts, Workers& ws)
{
    if (!logits || !tokens || !type_ok(dtype) || k < 1 || k > BAGUA_MAX_WORKERS || experts < 1 || ld < static_cast<size_t>(experts)) return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS || ld > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] && !logits[w]) return BAGUA_ERR_INVALID_ARG;
        if (tokens[w] > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    }
    ws = Workers{};
    ws.k = static_cast<uint32_t>(k);
    for (int w = 0; w < k; ++w) {
        ws.logits[w] = logits[w];
        ws.tokens[w] = static_cast<uint32_t>(tokens[w]);
    }
    return BAGUA_OK;
}
inline bool tiles_of(Workers& ws, int rows)
{
    uint64_t tiles = 0;
    for (uint32_t w = 0; w < ws.k; ++w) {
        ws.first_tile[w] = static_cast<uint32_t>(tiles);
        tiles += (ws.tokens[w] + static_cast<uint32_t>(rows) - 1) / static_cast<uint32_t>(rows);
        if (tiles > kMaxGrid) return false;
    }
    for (uint32_t w = ws.k; w <= BAGUA_MAX_WORKERS; ++w) ws.first_tile[w] = static_cast<uint32_t>(tiles);
    return true;
}
inline size_t matrix_bytes(size_t rows, size_t ld, size_t columns, size_t element) { return rows ? ((rows - 1) * ld + columns) * element : 0; }

}  // namespace bagua

using namespace bagua;

extern "C" size_t bagua_balance_workspace_bytes(int experts)
{
    if (experts < 1 || experts > BAGUA_MAX_EXPERTS) return 0;
    return kArriveBytes + (kBalanceGroups + kBalanceGroups / kArriveGroup) * (static_cast<size_t>(experts) * sizeof(uint64_t) + sizeof(uint32_t));
}

extern "C" int bagua_balance_stats(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts,
                                   const void* const* ids, int id_bytes, size_t ids_ld, int top_k, const uint8_t* const* mask,
                                   int32_t* counts, float* prob, double alpha, float* loss, float* weight, void* workspace,
                                   size_t workspace_bytes, void* stream)
{
    Workers ws;
    const int bad = balance_check(dtype, logits, ld, tokens, k, experts, ws);
    if (bad) return bad;
    if (!ids || (id_bytes != 4 && id_bytes != 8) || top_k < 1 || top_k > experts || ids_ld < static_cast<size_t>(top_k) || !counts || !prob ||
        !workspace || !loss != !weight || !(std::fabs(alpha) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (ids_ld > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    if (workspace_bytes < bagua_balance_workspace_bytes(experts)) return BAGUA_ERR_INVALID_ARG;
    size_t choices = 0;
    RangeCheck rc;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!ids[w] || (mask && !mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(logits[w], type_bytes(dtype)) || !aligned_to(ids[w], static_cast<size_t>(id_bytes))) return BAGUA_ERR_ALIGNMENT;
        choices += tokens[w] * static_cast<size_t>(top_k);
        rc.reads(logits[w], matrix_bytes(tokens[w], ld, static_cast<size_t>(experts), type_bytes(dtype)));
        rc.reads(ids[w], matrix_bytes(tokens[w], ids_ld, static_cast<size_t>(top_k), static_cast<size_t>(id_bytes)));
        if (mask) rc.reads(mask[w], tokens[w]);
        ws.ids[w] = ids[w];
        ws.mask[w] = mask ? mask[w] : nullptr;
    }
    if (choices > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    const size_t e = static_cast<size_t>(experts);
    rc.writes(counts, (e + 1) * sizeof(int32_t));
    rc.writes(prob, e * sizeof(float));
    rc.writes(loss, sizeof(float));
    rc.writes(weight, e * sizeof(float));
    rc.writes(workspace, bagua_balance_workspace_bytes(experts));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned16(workspace) || !aligned4(counts) || !aligned4(prob) || !aligned4(loss) || !aligned4(weight)) return BAGUA_ERR_ALIGNMENT;
    const BalanceOut out{counts, prob, loss, weight, alpha, experts, top_k};
    const uint32_t per_k = top_k == 1 ? 0 : static_cast<uint32_t>((0x100000000ull + static_cast<uint64_t>(top_k) - 1) / static_cast<uint64_t>(top_k));
    int lg = 3;                                             // copies of a counter: what fits 16 KiB, eight at most
    while (lg > 0 && ((e + 1) << lg) > 4096) --lg;
    int status = BAGUA_OK;
    with_layout<true>(dtype, experts, [&](auto layout, auto type) {
        typedef decltype(layout) Lay;
        auto launch = [&](auto chosen) -> int {
            typedef decltype(chosen) C;
            if (!tiles_of(ws, C::UNROLL * kWave / C::L)) return BAGUA_ERR_UNSUPPORTED;
            const uint32_t tiles = ws.first_tile[BAGUA_MAX_WORKERS];
            const dim3 grid(std::min<uint32_t>(std::max<uint32_t>((tiles + C::WAVES - 1) / C::WAVES, 1), kBalanceGroups)), block(kWave * C::WAVES);
            const size_t lds = (static_cast<size_t>(sum_rows(C::WAVES, experts)) * e + ((e + 1) << lg)) * sizeof(float);
            launch_kernel(k_balance_stats<decltype(type)::value, C::VEC, C::L, C::NV, C::UNROLL, C::WAVES>, grid, block, lds, static_cast<hipStream_t>(stream),
                          ws, ld, ids_ld, id_bytes, tiles, per_k, lg, static_cast<uint32_t*>(workspace), out);
            return launch_status();
        };
        // Rows of a wave at a time, 64 / L, in short launches one after another in different waves rather than together in one.  Together | apart:
        // 100 tokens of 8 experts 5.9 | 4.4 us, 1000 6.5 | 5.7, 32768 13.1 | 10.1; 1000 of 64 11.1 | 9.3, 4096 11.4 | 10.0; 1000 of 256 11.5 | 10.5.  Not where that would
        // make more than one group of one: 4096 of 8 8.6 | 9.8, 100 of 256 7.2 | 9.7.  The line of 512 units: 400 | 512 | 700 units gain (lose) 1.4 | 1.4 | 0.9 us with
        // 64 experts, 1.4 | 1.4 | (0.1) with 128, (0.4) | (0.4) | 0.6 with 256, 0.8 | 1.0 | (3.5) with 512; 8 experts gain 2.5 beyond it as well, up to 2048.
        size_t units = 0, tiles = 0;
        for (int w = 0; w < k; ++w) {
            units += (tokens[w] + kWave / Lay::L - 1) / (kWave / Lay::L);
            tiles += (tokens[w] + Lay::UNROLL * kWave / Lay::L - 1) / (Lay::UNROLL * kWave / Lay::L);
        }
        if (units <= Lay::WAVES || (tiles > Lay::WAVES && units <= 512)) status = launch(Layout<Lay::VEC, Lay::L, Lay::NV, 1, Lay::WAVES>());
        else status = launch(layout);
    });
    return status;
}

extern "C" int bagua_balance_loss(const int32_t* counts, const float* prob, int experts, int top_k, double alpha, float* loss, float* weight, void* stream)
{
    if (!counts || !prob || !loss || !weight || experts < 1 || top_k < 1 || top_k > experts || !(std::fabs(alpha) < INFINITY)) return BAGUA_ERR_INVALID_ARG;
    if (experts > BAGUA_MAX_EXPERTS) return BAGUA_ERR_UNSUPPORTED;
    const size_t e = static_cast<size_t>(experts);
    RangeCheck rc;
    rc.reads(counts, (e + 1) * sizeof(int32_t));
    rc.reads(prob, e * sizeof(float));
    rc.writes(loss, sizeof(float));
    rc.writes(weight, e * sizeof(float));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(counts) || !aligned4(prob) || !aligned4(loss) || !aligned4(weight)) return BAGUA_ERR_ALIGNMENT;
    const BalanceOut out{nullptr, nullptr, loss, weight, alpha, experts, top_k};
    launch_kernel(k_balance_loss, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream), counts, prob, out);
    return launch_status();
}

extern "C" int bagua_balance_grad(int dtype, const void* const* logits, size_t ld, const size_t* tokens, int k, int experts,
                                  const uint8_t* const* mask, const float* weight, const float* upstream, void* const* dlogits, size_t ld_out,
                                  void* stream)
{
    Workers ws;
    const int bad = balance_check(dtype, logits, ld, tokens, k, experts, ws);
    if (bad) return bad;
    if (!weight || !dlogits || ld_out < static_cast<size_t>(experts)) return BAGUA_ERR_INVALID_ARG;
    if (ld_out > static_cast<size_t>(1) << 40) return BAGUA_ERR_UNSUPPORTED;
    const size_t element = type_bytes(dtype), e = static_cast<size_t>(experts);
    RangeCheck rc;
    for (int w = 0; w < k; ++w) {
        if (tokens[w] == 0) continue;
        if (!dlogits[w] || (mask && !mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(logits[w], element) || !aligned_to(dlogits[w], element)) return BAGUA_ERR_ALIGNMENT;
        rc.reads(logits[w], matrix_bytes(tokens[w], ld, e, element));
        rc.writes(dlogits[w], matrix_bytes(tokens[w], ld_out, e, element));
        if (mask) rc.reads(mask[w], tokens[w]);
        ws.ids[w] = dlogits[w];
        ws.mask[w] = mask ? mask[w] : nullptr;
    }
    rc.reads(weight, e * sizeof(float));
    rc.reads(upstream, sizeof(float));
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned4(weight) || !aligned4(upstream)) return BAGUA_ERR_ALIGNMENT;
    int status = BAGUA_OK;
    with_layout<false>(dtype, experts, [&](auto layout, auto type) {
        typedef decltype(layout) Lay;
        if (!tiles_of(ws, Lay::GRAD_UNROLL * kWave / Lay::L)) {
            status = BAGUA_ERR_UNSUPPORTED;
            return;
        }
        const uint32_t tiles = ws.first_tile[BAGUA_MAX_WORKERS];
        if (tiles == 0) return;
        const uint32_t waves = std::min<uint32_t>(tiles, kGradMostWaves);
        const dim3 grid((waves + kGradWaves - 1) / kGradWaves), block(kWave * kGradWaves);
        launch_kernel(k_balance_grad<decltype(type)::value, Lay::VEC, Lay::L, Lay::NV, Lay::GRAD_UNROLL>, grid, block, 0, static_cast<hipStream_t>(stream), ws,
                      ld, ld_out, tiles, experts, weight, upstream);
        status = launch_status();
    });
    return status;
}
