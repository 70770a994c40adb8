// Distillation from a teacher's top logits, and its backward pass (see bagua_hip.h).
//
// A row of logits over the vocabulary is read once: every thread keeps the largest logit that it has met and the sums of exponentials relative to it,
// scaled anew when a larger one comes, and these are put together over the workgroup, or over the workgroups that share a row.  Sums are relative
// to a logit and not to 0, and the row's statistics are that logit and the sums, not their logarithm: x - largest is rounded where it is small.
#include <cmath>

#include "lists.hpp"
#include "rows.hpp"

#pragma clang fp contract(off)

namespace bagua {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr uint32_t kMostParts = kWave;        // of a row: a lane for each where they are put together

constexpr uint32_t kLessonFloats = 5;         // of a row, beside its parts

enum { kLogits = 0, kIds, kTeacher, kLabels, kMask, kLoss, kStats, kDistillLists };
enum { kUp = kLoss, kOut = kStats + 1, kDistillGradLists };      // of the backward pass; the others are the same

struct DistillArgs {
    size_t ld, ids_ld, teacher_ld, out_ld;
    uint32_t vocab, parts;
    int top, id_bytes, teacher_type, label_bytes;    // label_bytes: 0 for no labels
    int up_per_row;
    float temperature, to_log2, teacher_weight, label_weight;    // to_log2: log2(e) / temperature
    float* partial;                                  // [row][3 * parts + kLessonFloats], where a row has several parts
};

// What a row is taught: the teacher's entries, and the label.
template <int P>
struct Taught {
    const DistillArgs& a;
    const ListTile<P>& t;
    __device__ __forceinline__ int id(int j) const
    {
        const size_t at = t.t0 * a.ids_ld + static_cast<size_t>(j);
        const uint64_t v = a.id_bytes == 8 ? t.template ptr<const uint64_t>(kIds)[at] : static_cast<uint64_t>(static_cast<int64_t>(t.template ptr<const int32_t>(kIds)[at]));
        return v < a.vocab ? static_cast<int>(v) : -1;
    }
    // The teacher's logit, -infinity where the id is none.
    __device__ __forceinline__ float logit(int j, int id) const
    {
        const size_t at = t.t0 * a.teacher_ld + static_cast<size_t>(j);
        if (id < 0) return -INFINITY;
        if (a.teacher_type == BAGUA_F32) return t.template ptr<const float>(kTeacher)[at];
        const uint16_t v = t.template ptr<const uint16_t>(kTeacher)[at];
        return a.teacher_type == BAGUA_BF16 ? Elem<BAGUA_BF16>::widen(v) : Elem<BAGUA_F16>::widen(v);
    }
    __device__ __forceinline__ int label() const
    {
        if (a.label_bytes == 0) return -1;
        const uint64_t v = a.label_bytes == 8 ? t.template ptr<const uint64_t>(kLabels)[t.t0]
                                              : static_cast<uint64_t>(static_cast<int64_t>(t.template ptr<const int32_t>(kLabels)[t.t0]));
        return v < a.vocab ? static_cast<int>(v) : -1;
    }
    __device__ __forceinline__ bool counts() const { return !t.has(kMask) || t.template ptr<const uint8_t>(kMask)[t.t0] != 0; }
};

// The teacher's softmax over its entries, by a wave that has entry j in lane j % 64: its largest logit and the sum relative to it; no entry: sum 0.
struct TeacherSum {
    float most, sum;
    // exp((logit - most) / temperature), 0 for an entry that is none
    static __device__ __forceinline__ float term(float logit, float most, const DistillArgs& a) { return logit == -INFINITY ? 0.0f : expf((logit - most) / a.temperature); }
    template <int P>
    __device__ __forceinline__ TeacherSum(const Taught<P>& w, float first, int lane)
    {
        most = first;
        for (int j = lane + kWave; j < w.a.top; j += kWave) most = fmaxf(most, w.logit(j, w.id(j)));
        most = lanes_most<kWave>(most);
        sum = term(first, most, w.a);
        for (int j = lane + kWave; j < w.a.top; j += kWave) sum += term(w.logit(j, w.id(j)), most, w.a);
        sum = lanes_reduce<kWave>(sum, OpAddF());
    }
};

// The logits of a row as the kernels go through them: some that lie before the first aligned vector, vectors, and some behind the last.
template <int TYPE>
struct Span {
    typedef typename Elem<TYPE>::one one;
    static constexpr int VEC = TYPE == BAGUA_F32 ? 4 : 8;
    typedef one v __attribute__((ext_vector_type(VEC), aligned(sizeof(one))));
    uint32_t head, vectors, first, last;       // first, last: vectors of this part
    uint32_t from, to;                         // elements of this part
    __device__ __forceinline__ Span(const one* aligned_row, uint32_t vocab, uint32_t part, uint32_t parts)
    {
        head = min(vocab, (0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(aligned_row) / sizeof(one))) & (VEC - 1));
        vectors = (vocab - head) / VEC;
        const uint32_t each = (vectors + parts - 1) / parts;
        first = min(part * each, vectors);
        last = min(first + each, vectors);
        from = part == 0 ? 0 : head + first * VEC;
        to = part + 1 == parts ? vocab : head + last * VEC;
    }
    // The elements that lie in no vector: `thread` has one of them, or none (vocab)
    __device__ __forceinline__ uint32_t single(uint32_t thread, uint32_t vocab) const
    {
        if (thread < VEC) return thread < head && from == 0 ? thread : vocab;
        const uint32_t e = head + vectors * VEC + thread - VEC;
        return to == vocab && thread < 2 * VEC ? min(e, vocab) : vocab;
    }
};

// exp(d) from e = exp(d / T), where T is the whole number POWER: its square, third or fourth power, an operation or two instead of an exponential, which takes
// as long as four.  POWER 0: T is another number.
template <int POWER>
__device__ __forceinline__ float power_of(float e, float d)
{
    if (POWER == 1) return e;
    if (POWER == 2) return e * e;
    if (POWER == 3) return e * e * e;
    if (POWER == 4) return (e * e) * (e * e);
    return __builtin_amdgcn_exp2f(d * kLog2e);
}

// The largest logit and the sums relative to it, at the teacher's temperature and, unless POWER is 1, at temperature 1.
template <int POWER>
struct Running {
    static constexpr bool TWO = POWER != 1;
    float most = -INFINITY, sum = 0.0f, sum_1 = 0.0f;
    __device__ __forceinline__ void rise(float m, const DistillArgs& a)
    {
        const float up = fmaxf(most, m), d = most == up ? 0.0f : most - up;     // (both -infinity: stays)
        const float e = __builtin_amdgcn_exp2f(d * a.to_log2);
        sum *= e;
        if (TWO) sum_1 *= power_of<POWER>(e, d);
        most = up;
    }
    __device__ __forceinline__ void add(float x, float from, const DistillArgs& a)
    {
        const float d = x - from, e = __builtin_amdgcn_exp2f(d * a.to_log2);
        sum += e;
        if (POWER == 2) sum_1 = __builtin_fmaf(e, e, sum_1);
        else if (TWO) sum_1 += power_of<POWER>(e, d);
    }
    __device__ __forceinline__ float origin() const { return most == -INFINITY ? 0.0f : most; }
    // Put together over a wave, in every lane.
    __device__ __forceinline__ void together(const DistillArgs& a)
    {
        rise(lanes_most<kWave>(most), a);
        sum = lanes_reduce<kWave>(sum, OpAddF());
        sum_1 = TWO ? lanes_reduce<kWave>(sum_1, OpAddF()) : sum;
    }
};

// What a wave knows of the row's entries and label before it knows the row's sums.
//   the teacher's part / T^2 = sum q log q - sum q (x - origin) / T + (most - origin) / T + log(sum)     with the row's largest logit and sum,
// relative to the largest of the entries' own logits, so that nothing is rounded where it is large.
struct Lesson {
    float known, origin, at_label;      // the first two sums; NaN in at_label: no label
    bool entries;
};
template <int TYPE, int P>
__device__ __forceinline__ Lesson lesson_of(const Taught<P>& w, const typename Elem<TYPE>::one* row, int lane, int first_id, float first_teacher, float first_x, int label, float at_label)
{
    const DistillArgs& a = w.a;
    const TeacherSum teacher(w, first_teacher, lane);
    Lesson l{0.0f, -INFINITY, label >= 0 ? at_label : 0.0f, teacher.sum != 0.0f};
    const float log_sum = logf(teacher.sum);
    if (first_id >= 0 && first_teacher != -INFINITY) l.origin = first_x;
    for (int j = lane + kWave; j < a.top; j += kWave) {
        const int id = w.id(j);
        if (id >= 0) l.origin = fmaxf(l.origin, Elem<TYPE>::widen(row[id]));
    }
    l.origin = lanes_most<kWave>(l.origin);
    if (l.origin == -INFINITY) l.origin = 0.0f;
    auto entry = [&](int id, float y, float x) {
        const float term = TeacherSum::term(y, teacher.most, a);
        if (id < 0 || term == 0.0f) return;
        l.known += term / teacher.sum * (((y - teacher.most) / a.temperature - log_sum) - (x - l.origin) / a.temperature);
    };
    entry(first_id, first_teacher, first_x);
    for (int j = lane + kWave; j < a.top; j += kWave) {
        const int id = w.id(j);
        if (id >= 0) entry(id, w.logit(j, id), Elem<TYPE>::widen(row[id]));
    }
    l.known = lanes_reduce<kWave>(l.known, OpAddF());
    return l;
}
// Loss and statistics of a row, by one lane.
template <int POWER, int P>
__device__ __forceinline__ void finish(const Taught<P>& w, const Lesson& l, const Running<POWER>& r, bool label)
{
    const DistillArgs& a = w.a;
    float loss = 0.0f;
    // (a part of weight 0 adds nothing where it is infinite either)
    if (l.entries && a.teacher_weight != 0.0f)
        loss = a.teacher_weight * (a.temperature * a.temperature) * (r.most == -INFINITY ? INFINITY : l.known + ((r.most - l.origin) / a.temperature + logf(r.sum)));
    if (label && a.label_weight != 0.0f) loss += a.label_weight * (l.at_label == -INFINITY ? INFINITY : logf(r.sum_1) - (l.at_label - r.most));
    w.t.template ptr<float>(kLoss)[w.t.t0] = loss;
    float* stats = w.t.template ptr<float>(kStats) + static_cast<size_t>(w.t.t0) * 3;
    stats[0] = r.most;
    stats[1] = r.sum;
    stats[2] = a.label_bytes ? r.sum_1 : 0.0f;
}

// One workgroup for a row, or a part of one.
template <int TYPE, int POWER, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_distill(Lists<kDistillLists> ls, DistillArgs a)
{
    typedef typename Elem<TYPE>::one one;
    typedef Span<TYPE> S;
    constexpr int VEC = S::VEC, UNROLL = 4, WAVES = THREADS / kWave;
    __shared__ float of_wave[3][WAVES];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const uint32_t unit = blockIdx.x / a.parts, part = blockIdx.x - unit * a.parts;
    const ListTile<kDistillLists> t(ls, unit, 1);
    const Taught<kDistillLists> w{a, t};
    if (!w.counts()) {
        if (part == 0 && threadIdx.x < 3) {
            t.template ptr<float>(kStats)[static_cast<size_t>(t.t0) * 3 + threadIdx.x] = 0.0f;
            if (threadIdx.x == 0) t.template ptr<float>(kLoss)[t.t0] = 0.0f;
        }
        return;
    }
    const one* row = t.template ptr<const one>(kLogits) + static_cast<size_t>(t.t0) * a.ld;
    const S span(row, a.vocab, part, a.parts);
    const bool teaches = part == 0 && wave == 0;
    int id = -1, label = -1;
    float teacher = -INFINITY, at_id = 0.0f, at_label = 0.0f;
    if (teaches) {                                                // on their way while the row is read
        label = w.label();
        if (lane < a.top) {
            id = w.id(lane);
            teacher = w.logit(lane, id);
            if (id >= 0) at_id = Elem<TYPE>::widen(row[id]);
        }
        if (label >= 0) at_label = Elem<TYPE>::widen(row[label]);
    }
    Running<POWER> r;
    const uint32_t alone = span.single(threadIdx.x, a.vocab);
    if (alone < a.vocab) {
        const float x = Elem<TYPE>::widen(row[alone]);
        r.rise(x, a);
        r.add(x, r.origin(), a);
    }
    const typename S::v* from = reinterpret_cast<const typename S::v*>(row + span.head);
    // A wave's vectors: UNROLL at a time as long as all of them are there, then what is left.
    uint32_t base = span.first + static_cast<uint32_t>(wave) * kWave;
    for (; base + (UNROLL - 1) * THREADS + kWave <= span.last; base += UNROLL * THREADS) {
        typename S::v q[UNROLL];
        float x[UNROLL][VEC], most = -INFINITY;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) q[u] = __builtin_nontemporal_load(from + base + u * THREADS + lane);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) most = fmaxf(most, x[u][e] = Elem<TYPE>::widen(q[u][e]));
        r.rise(most, a);
        const float origin = r.origin();
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) r.add(x[u][e], origin, a);
    }
    if (base < span.last) {
        typename S::v q[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) q[u] = __builtin_nontemporal_load(from + min(base + u * THREADS + lane, span.last - 1));
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (base + u * THREADS >= span.last) break;
            const bool there = base + u * THREADS + lane < span.last;
            float x[VEC], most = -INFINITY;
#pragma unroll
            for (int e = 0; e < VEC; ++e) most = fmaxf(most, x[e] = there ? Elem<TYPE>::widen(q[u][e]) : -INFINITY);
            r.rise(most, a);
            const float origin = r.origin();
#pragma unroll
            for (int e = 0; e < VEC; ++e) r.add(x[e], origin, a);
        }
    }
    r.together(a);
    if (WAVES > 1) {
        if (lane == 0) of_wave[0][wave] = r.most, of_wave[1][wave] = r.sum, of_wave[2][wave] = r.sum_1;
        __syncthreads();
        if (wave != 0) return;
        r = Running<POWER>();
        if (lane < WAVES) r.most = of_wave[0][lane], r.sum = of_wave[1][lane], r.sum_1 = of_wave[2][lane];
        r.together(a);
    }
    Lesson l{};
    if (teaches) l = lesson_of<TYPE>(w, row, lane, id, teacher, at_id, label, at_label);
    if (lane != 0) return;
    if (a.parts == 1) {
        finish(w, l, r, label >= 0);
        return;
    }
    float* out = a.partial + static_cast<size_t>(unit) * (3 * a.parts + kLessonFloats);
    out[part] = r.most, out[a.parts + part] = r.sum, out[2 * a.parts + part] = r.sum_1;
    if (teaches) {
        out += 3 * a.parts;
        out[0] = l.known, out[1] = l.origin, out[2] = l.at_label, out[3] = l.entries ? 1.0f : 0.0f, out[4] = label >= 0 ? 1.0f : 0.0f;
    }
}

// Puts the parts of a row together: one wave for each row.
template <int POWER>
__global__ void __launch_bounds__(kWave)
k_distill_finish(Lists<kDistillLists> ls, DistillArgs a)
{
    const int lane = threadIdx.x & 63;
    const ListTile<kDistillLists> t(ls, blockIdx.x, 1);
    const Taught<kDistillLists> w{a, t};
    if (!w.counts()) return;
    const float *p = a.partial + static_cast<size_t>(blockIdx.x) * (3 * a.parts + kLessonFloats), *q = p + 3 * a.parts;
    const Lesson l{q[0], q[1], q[2], q[3] != 0.0f};
    const bool label = q[4] != 0.0f;
    Running<POWER> r;
    if (lane < static_cast<int>(a.parts)) r.most = p[lane], r.sum = p[a.parts + lane], r.sum_1 = p[2 * a.parts + lane];
    r.together(a);
    if (lane == 0) finish(w, l, r, label);
}

// The backward pass, one workgroup for a part of a row: factor * exp((x - largest) / temperature), and with labels the same at temperature 1, for every
// logit; the few that the teacher or the label names are written over when the others are out, each with all that its entries take from it.
// The gradient may lie where the logits are: a workgroup reads those of its part that are named before it writes any.
template <int TYPE, int POWER, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_distill_grad(Lists<kDistillGradLists> ls, DistillArgs a)
{
    typedef typename Elem<TYPE>::one one;
    typedef Span<TYPE> S;
    constexpr int VEC = S::VEC, UNROLL = 4;
    extern __shared__ float named[];
    int* named_id = reinterpret_cast<int*>(named);                       // [top + 1]: the teacher's entries and the label
    float *named_x = named + a.top + 1, *named_less = named + 2 * (a.top + 1);
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x / a.parts, part = blockIdx.x - unit * a.parts;
    const ListTile<kDistillGradLists> t(ls, unit, 1);
    const Taught<kDistillGradLists> w{a, t};
    const one* row = t.template ptr<const one>(kLogits) + static_cast<size_t>(t.t0) * a.ld;
    one* out = t.template ptr<one>(kOut) + static_cast<size_t>(t.t0) * a.out_ld;
    const S span(out, a.vocab, part, a.parts);
    const bool counts = w.counts();
    const int first_id = counts && lane < a.top ? w.id(lane) : -1, label = counts ? w.label() : -1;
    TeacherSum teacher(w, counts && lane < a.top ? w.logit(lane, first_id) : -INFINITY, counts ? lane : a.top);
    typename S::v* to = reinterpret_cast<typename S::v*>(out + span.head);
    const uint32_t alone = span.single(threadIdx.x, a.vocab);
    if (!counts || (teacher.sum == 0.0f && label < 0)) {                  // nothing to learn: the logits do not matter
        for (uint32_t i = span.first + threadIdx.x; i < span.last; i += THREADS) __builtin_nontemporal_store(typename S::v(0), to + i);
        if (alone < a.vocab) out[alone] = 0;
        return;
    }
    const float* stats = t.template ptr<const float>(kStats) + static_cast<size_t>(t.t0) * 3;
    const float up = !t.has(kUp) ? 1.0f : t.template ptr<const float>(kUp)[a.up_per_row ? t.t0 : 0];
    const float origin = stats[0] == -INFINITY ? 0.0f : stats[0];
    const float teach = teacher.sum == 0.0f ? 0.0f : up * (a.teacher_weight * a.temperature), tell = label < 0 ? 0.0f : up * a.label_weight;
    float factor = stats[1] == 0.0f ? 0.0f : teach / stats[1];
    const float factor_1 = stats[1] == 0.0f || a.label_bytes == 0 ? 0.0f : tell / stats[2];
    if (POWER == 1) factor += factor_1;                                   // both at temperature 1, or no labels
    for (int j = static_cast<int>(threadIdx.x); j <= a.top; j += THREADS) {
        const int id = j < a.top ? w.id(j) : label;
        const bool here = id >= 0 && static_cast<uint32_t>(id) >= span.from && static_cast<uint32_t>(id) < span.to;
        named_id[j] = here ? id : -1;
        named_x[j] = here ? Elem<TYPE>::widen(row[id]) : 0.0f;
        named_less[j] = j == a.top ? tell : teach == 0.0f ? 0.0f : teach * (TeacherSum::term(w.logit(j, id), teacher.most, a) / teacher.sum);
    }
    __syncthreads();
    auto value = [&](float x) {
        const float d = x - origin, e = __builtin_amdgcn_exp2f(d * a.to_log2);
        return POWER == 1 ? factor * e : __builtin_fmaf(factor_1, power_of<POWER>(e, d), factor * e);
    };
    const typename S::v* from = reinterpret_cast<const typename S::v*>(row + span.head);
    uint32_t base = span.first + static_cast<uint32_t>(wave_index()) * kWave;
    auto put = [&](uint32_t i, const typename S::v& q) {
        typename S::v o;
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = Elem<TYPE>::narrow(value(Elem<TYPE>::widen(q[e])));
        __builtin_nontemporal_store(o, to + i);
    };
    for (; base + (UNROLL - 1) * THREADS + kWave <= span.last; base += UNROLL * THREADS) {
        typename S::v q[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) q[u] = __builtin_nontemporal_load(from + base + u * THREADS + lane);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) put(base + u * THREADS + lane, q[u]);
    }
    if (base < span.last) {
        typename S::v q[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) q[u] = __builtin_nontemporal_load(from + min(base + u * THREADS + lane, span.last - 1));
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (base + u * THREADS + lane < span.last) put(base + u * THREADS + lane, q[u]);
    }
    if (alone < a.vocab) out[alone] = Elem<TYPE>::narrow(value(Elem<TYPE>::widen(row[alone])));
    pace_loads();                                                         // what is out cannot overtake what is written over it
    __syncthreads();
    for (int j = static_cast<int>(threadIdx.x); j <= a.top; j += THREADS) {
        const int id = named_id[j];
        if (id < 0) continue;
        float less = 0.0f;
        for (int i = 0; i <= a.top; ++i) less += named_id[i] == id ? named_less[i] : 0.0f;
        out[id] = Elem<TYPE>::narrow(value(named_x[j]) - less);
    }
}

constexpr uint32_t kDistillThreads = 256;
constexpr uint32_t kShortVocab = 4096;        // up to here a wave for each row

// Parts of a row: enough workgroups for the chip, and none shorter than is worth one.
inline uint32_t distill_parts(size_t rows, size_t vocab, size_t shortest, size_t longest)
{
    size_t parts = (vocab + longest - 1) / longest;
    const size_t wanted = rows ? (8 * static_cast<size_t>(kCus) + rows - 1) / rows : 1, most = (vocab + shortest - 1) / shortest;
    parts = std::max(parts, std::min(wanted, most));
    return static_cast<uint32_t>(std::max<size_t>(1, std::min<size_t>(parts, kMostParts)));
}
inline uint32_t loss_parts(size_t rows, size_t vocab) { return distill_parts(rows, vocab, 8192, static_cast<size_t>(1) << 40); }
inline uint32_t grad_parts(size_t rows, size_t vocab) { return distill_parts(rows, vocab, 8192, 32768); }

struct DistillCall {
    int dtype;
    const void* const* logits;
    size_t ld;
    const size_t* rows;
    int k;
    size_t vocab;
    const void* const* ids;
    int id_bytes;
    size_t ids_ld;
    int top, teacher_type;
    const void* const* teacher;
    size_t teacher_ld;
    const void* const* labels;
    int label_bytes;
    const uint8_t* const* mask;
    double temperature, teacher_weight, label_weight;
};

template <int P>
inline int distill_check(const DistillCall& c, Lists<P>& ls, DistillArgs& a, RangeCheck& rc, size_t& total, bool in_place)
{
    if (!c.logits || !c.rows || !type_ok(c.dtype) || c.k < 1 || c.k > BAGUA_MAX_WORKERS || c.vocab < 1 || c.ld < c.vocab || !c.ids || (c.id_bytes != 4 && c.id_bytes != 8) ||
        c.top < 1 || c.ids_ld < static_cast<size_t>(c.top) || !type_ok(c.teacher_type) || !c.teacher || c.teacher_ld < static_cast<size_t>(c.top) ||
        (c.labels && c.label_bytes != 4 && c.label_bytes != 8) || !(c.temperature > 0.0) || !(c.temperature < INFINITY) || !(std::fabs(c.teacher_weight) < INFINITY) || !(std::fabs(c.label_weight) < INFINITY))
        return BAGUA_ERR_INVALID_ARG;
    if (c.temperature < 0x1p-60 || c.temperature > 0x1p60) return BAGUA_ERR_UNSUPPORTED;
    if (c.vocab > BAGUA_MAX_VOCABULARY || c.top > BAGUA_MAX_TEACHER_ENTRIES || c.ld > kMostStride || c.ids_ld > kMostStride || c.teacher_ld > kMostStride) return BAGUA_ERR_UNSUPPORTED;
    const size_t element = type_bytes(c.dtype), top = static_cast<size_t>(c.top), id_size = static_cast<size_t>(c.id_bytes), label_size = static_cast<size_t>(c.label_bytes);
    total = 0;
    for (int w = 0; w < c.k; ++w) {
        const size_t n = c.rows[w];
        if (n > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
        if (n == 0) continue;
        if (!c.logits[w] || !c.ids[w] || !c.teacher[w] || (c.labels && !c.labels[w]) || (c.mask && !c.mask[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned_to(c.logits[w], element) || !aligned_to(c.ids[w], id_size) || !aligned_to(c.teacher[w], type_bytes(c.teacher_type)) ||
            (c.labels && !aligned_to(c.labels[w], label_size)))
            return BAGUA_ERR_ALIGNMENT;
        total += n;
        if (!in_place) rc.reads(c.logits[w], rows_bytes(n, c.ld, c.vocab, element));
        rc.reads(c.ids[w], rows_bytes(n, c.ids_ld, top, id_size));
        rc.reads(c.teacher[w], rows_bytes(n, c.teacher_ld, top, type_bytes(c.teacher_type)));
        if (c.labels) rc.reads(c.labels[w], n * label_size);
        if (c.mask) rc.reads(c.mask[w], n);
        ls.at[kLogits][w] = c.logits[w];
        ls.at[kIds][w] = c.ids[w];
        ls.at[kTeacher][w] = c.teacher[w];
        ls.at[kLabels][w] = c.labels ? c.labels[w] : nullptr;
        ls.at[kMask][w] = c.mask ? c.mask[w] : nullptr;
    }
    if (tiles_of(ls, c.rows, c.k, 1) > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    a = DistillArgs{};
    a.ld = c.ld, a.ids_ld = c.ids_ld, a.teacher_ld = c.teacher_ld;
    a.vocab = static_cast<uint32_t>(c.vocab);
    a.top = c.top, a.id_bytes = c.id_bytes, a.teacher_type = c.teacher_type, a.label_bytes = c.labels ? c.label_bytes : 0;
    a.temperature = static_cast<float>(c.temperature);
    a.to_log2 = static_cast<float>(1.44269504088896340736 / c.temperature);
    a.teacher_weight = static_cast<float>(c.teacher_weight);
    a.label_weight = static_cast<float>(c.label_weight);
    return BAGUA_OK;
}

// f with the type, what power of an exponential at the teacher's temperature is one at 1, and the threads of a workgroup.
template <typename F>
inline void with_distill(int dtype, bool labels, double temperature, size_t vocab, const F& f)
{
    auto of_type = [&](auto type) {
        auto of_power = [&](auto power) {
            if (vocab <= kShortVocab) f(type, power, std::integral_constant<int, kWave>());
            else f(type, power, std::integral_constant<int, kDistillThreads>());
        };
        if (!labels || temperature == 1.0) of_power(std::integral_constant<int, 1>());
        else if (temperature == 2.0) of_power(std::integral_constant<int, 2>());
        else if (temperature == 3.0) of_power(std::integral_constant<int, 3>());
        else if (temperature == 4.0) of_power(std::integral_constant<int, 4>());
        else of_power(std::integral_constant<int, 0>());
    };
    if (dtype == BAGUA_F32) of_type(std::integral_constant<int, BAGUA_F32>());
    else if (dtype == BAGUA_BF16) of_type(std::integral_constant<int, BAGUA_BF16>());
    else of_type(std::integral_constant<int, BAGUA_F16>());
}

}  // namespace bagua

using namespace bagua;

extern "C" size_t bagua_distill_workspace_bytes(size_t rows, size_t vocab)
{
    if (vocab < 1 || vocab > BAGUA_MAX_VOCABULARY || rows > kMaxGrid) return 0;
    const size_t parts = loss_parts(rows, vocab);
    return 16 + (parts > 1 ? (rows * (parts * 3 + kLessonFloats) * sizeof(float) + 15) / 16 * 16 : 0);
}

extern "C" int bagua_distill_loss(int dtype, const void* const* logits, size_t ld, const size_t* rows, int k, size_t vocab, const void* const* ids, int id_bytes,
                                  size_t ids_ld, int top, int teacher_type, const void* const* teacher, size_t teacher_ld, const void* const* labels,
                                  int label_bytes, const uint8_t* const* mask, double temperature, double teacher_weight, double label_weight,
                                  float* const* loss, float* const* stats, void* workspace, size_t workspace_bytes, void* stream)
{
    const DistillCall c{dtype, logits, ld, rows, k, vocab, ids, id_bytes, ids_ld, top, teacher_type, teacher, teacher_ld, labels, label_bytes, mask, temperature, teacher_weight, label_weight};
    Lists<kDistillLists> ls{};
    DistillArgs a;
    RangeCheck rc;
    size_t total;
    const int bad = distill_check(c, ls, a, rc, total, false);
    if (bad) return bad;
    if (!loss || !stats || !workspace) return BAGUA_ERR_INVALID_ARG;
    for (int w = 0; w < k; ++w) {
        if (rows[w] == 0) continue;
        if (!loss[w] || !stats[w]) return BAGUA_ERR_INVALID_ARG;
        if (!aligned4(loss[w]) || !aligned4(stats[w])) return BAGUA_ERR_ALIGNMENT;
        rc.writes(loss[w], rows[w] * sizeof(float));
        rc.writes(stats[w], rows[w] * 3 * sizeof(float));
        ls.at[kLoss][w] = loss[w];
        ls.at[kStats][w] = stats[w];
    }
    const size_t bytes = bagua_distill_workspace_bytes(total, vocab);
    if (workspace_bytes < bytes) return BAGUA_ERR_INVALID_ARG;
    rc.writes(workspace, bytes);
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (!aligned16(workspace)) return BAGUA_ERR_ALIGNMENT;
    if (total == 0) return BAGUA_OK;
    a.parts = loss_parts(total, vocab);
    a.partial = static_cast<float*>(workspace);
    if (total * a.parts > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int status = BAGUA_OK;
    with_distill(dtype, labels != nullptr, temperature, vocab, [&](auto type, auto power, auto threads) {
        constexpr int TYPE = decltype(type)::value, POWER = decltype(power)::value, THREADS = decltype(threads)::value;
        launch_kernel(k_distill<TYPE, POWER, THREADS>, dim3(static_cast<uint32_t>(total) * a.parts), dim3(THREADS), 0, s, ls, a);
        status = launch_status();
        if (status != BAGUA_OK || a.parts == 1) return;
        launch_kernel(k_distill_finish<POWER>, dim3(static_cast<uint32_t>(total)), dim3(kWave), 0, s, ls, a);
        status = launch_status();
    });
    return status;
}

extern "C" int bagua_distill_grad(int dtype, const void* const* logits, size_t ld, const size_t* rows, int k, size_t vocab, const void* const* ids, int id_bytes,
                                  size_t ids_ld, int top, int teacher_type, const void* const* teacher, size_t teacher_ld, const void* const* labels,
                                  int label_bytes, const uint8_t* const* mask, double temperature, double teacher_weight, double label_weight,
                                  const float* const* stats, const float* const* upstream, int upstream_per_row, void* const* dlogits, size_t ld_out, void* stream)
{
    const DistillCall c{dtype, logits, ld, rows, k, vocab, ids, id_bytes, ids_ld, top, teacher_type, teacher, teacher_ld, labels, label_bytes, mask, temperature, teacher_weight, label_weight};
    Lists<kDistillGradLists> ls{};
    DistillArgs a;
    RangeCheck rc;
    size_t total;
    const int bad = distill_check(c, ls, a, rc, total, true);
    if (bad) return bad;
    if (!stats || !dlogits || ld_out < vocab) return BAGUA_ERR_INVALID_ARG;
    if (ld_out > kMostStride) return BAGUA_ERR_UNSUPPORTED;
    const size_t element = type_bytes(dtype);
    for (int w = 0; w < k; ++w) {
        if (rows[w] == 0) continue;
        if (!stats[w] || !dlogits[w] || (upstream && !upstream[w])) return BAGUA_ERR_INVALID_ARG;
        if (!aligned4(stats[w]) || !aligned_to(dlogits[w], element) || (upstream && !aligned4(upstream[w]))) return BAGUA_ERR_ALIGNMENT;
        // the gradient may lie where the logits are, element upon element
        if (!(dlogits[w] == logits[w] && (ld == ld_out || rows[w] == 1))) rc.reads(logits[w], rows_bytes(rows[w], ld, vocab, element));
        rc.writes(dlogits[w], rows_bytes(rows[w], ld_out, vocab, element));
        rc.reads(stats[w], rows[w] * 3 * sizeof(float));
        if (upstream) rc.reads(upstream[w], (upstream_per_row ? rows[w] : 1) * sizeof(float));
        ls.at[kUp][w] = upstream ? upstream[w] : nullptr;
        ls.at[kStats][w] = stats[w];
        ls.at[kOut][w] = dlogits[w];
    }
    if (!rc.disjoint()) return BAGUA_ERR_INVALID_ARG;
    if (total == 0) return BAGUA_OK;
    a.out_ld = ld_out;
    a.up_per_row = upstream_per_row != 0;
    a.parts = grad_parts(total, vocab);
    if (total * a.parts > kMaxGrid) return BAGUA_ERR_UNSUPPORTED;
    int status = BAGUA_OK;
    with_distill(dtype, labels != nullptr, temperature, vocab, [&](auto type, auto power, auto threads) {
        constexpr int TYPE = decltype(type)::value, POWER = decltype(power)::value, THREADS = decltype(threads)::value;
        launch_kernel(k_distill_grad<TYPE, POWER, THREADS>, dim3(static_cast<uint32_t>(total) * a.parts), dim3(THREADS), static_cast<size_t>(top + 1) * 3 * sizeof(float),
                      static_cast<hipStream_t>(stream), ls, a);
        status = launch_status();
    });
    return status;
}
