// Log probabilities of symbols under rows of logits, with entropy and alternatives, and their gradient.
#pragma once

namespace pilc {

// Per row of logits x: M = max x, S = sum of e^(x - M), U = sum of (x - M) e^(x - M); lse = M + ln S, ln p of symbol t = x_t - lse,
// entropy = ln S - U / S, and the gradient of a logp + b entropy is a (1[j = t] - p_j) - b p_j (ln p_j + entropy).  A value
// takes 11 vector instructions for the gradient alone, 14 to 15 for the law of a long row with alternatives and 21 for law and
// gradient (counted), and two or four bytes: vector units and memory bound the kernels about alike.  So a value is read once, into
// registers, and gone through there: for M, for S and U, for the alternatives, for the gradient.

constexpr int kMaxTop = 32;

struct LogitsArgs {
    const void *x;
    const void *target;
    float *logp, *entropy, *lse;
    int32_t *top_sym;
    float *top_logp;
    const float *lse_in, *entropy_in, *up_logp, *up_entropy;
    float4 *law;  // of each row for k_logits_grad: its largest, total, log_total, entropy (see Law)
    void *grad;
    uint64_t stride, grad_stride;
    uint32_t rows, num_sym, top, target_type;
    uint32_t splits, span;  // a row goes into `splits` runs of `span` values, the last one maybe shorter
    float4 *part;           // of each run: its largest, sum, sum of products (see Law)
    uint64_t *part_top;     // and its `top` keys, best first, 0 where there are fewer
};

__device__ __forceinline__ int64_t target_of(const LogitsArgs &a, uint32_t row)
{
    return a.target_type == PILC_U8    ? (int64_t)((const uint8_t *)a.target)[row]
           : a.target_type == PILC_I32 ? (int64_t)((const int32_t *)a.target)[row]
                                       : ((const int64_t *)a.target)[row];
}

// Integers in the order of the values they are made of; of a key, the lower symbol's is the higher among equals.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);  // no -0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderNone = 0x007FFFFFu;  // of -inf
__device__ __forceinline__ uint64_t key_of(float x, uint32_t sym) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - sym); }
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order);
}

constexpr float kLn2 = 0.693147180559945309f;
// No 32-bit power of two is left here: what a power is multiplied with need not go on falling, and may not be -inf.
constexpr float kLeast = -200.0f;

// How exponentials of a row's values are taken: 2^(x log2 e - shift), one fused multiply-add and one power a value.  shift is
// the largest value times log2 e, rounded, so that all powers are the same factor 2^off too large, which is taken out of
// sums.  off is half a unit of shift at most: 1/16 where the largest value is under 2^20 in size, but 128, and 2^off no
// number, from 2^31 on.  Rows whose largest value lies further out than 2^20 have it subtracted first, which is an instruction more a
// value (4093 x 100003 bf16 with alternatives 162 us, all rows that way 168; training 65536 x 256 bf16 16.0 and 16.5, 16384 x 65536
// 744 and 745).
struct Scale {
    static constexpr float kFused = 0x1p20f;
    float center, shift, off;
    bool apart;

    __device__ explicit Scale(float m)
    {
        center = m == -kInf ? 0.0f : m;
        apart = !(fabsf(center) < kFused);
        shift = center * kLog2e;
        off = apart ? 0.0f : __builtin_fmaf(center, kLog2e, -shift);
    }
    template <bool kApart>
    __device__ float power(float x) const { return kApart ? (x - center) * kLog2e : __builtin_fmaf(x, kLog2e, -shift); }
    // f(std::bool_constant) with the way that this row's values go
    template <class F>
    __device__ void by_power(F f) const
    {
        if (apart)
            f(std::true_type());
        else
            f(std::false_type());
    }
};

// What is known of a row or of a part of it: its largest value, the sum of its values' powers 2^z, z = (x - max) log2 e, and
// the sum of z 2^z.
struct Tally {
    float max, total, inside;
};

// Both tallies' values together.  Where neither maximum is a number's (-inf twice) there is nothing to add.
__device__ __forceinline__ Tally both(Tally a, Tally b)
{
    const float max = fmaxf(a.max, b.max);
    const float da = fmaxf((a.max - max) * kLog2e, kLeast), db = fmaxf((b.max - max) * kLog2e, kLeast);
    const float fa = exp2_fast(da), fb = exp2_fast(db);
    return {max, a.total * fa + b.total * fb, (a.inside + da * a.total) * fa + (b.inside + db * b.total) * fb};
}

struct Law {
    float max, log_total, entropy, total;  // lse = max + log_total

    // An empty row: max -inf.  A NaN, or +inf less itself, in the sum: all NaN.
    __device__ explicit Law(Tally t) : max(t.max), total(t.total)
    {
        if (t.max == -kInf && t.total == 0.0f) {
            log_total = entropy = 0.0f;
            return;
        }
        log_total = logf(t.total);
        entropy = log_total - kLn2 * t.inside / t.total;
        if (!(log_total == log_total)) max = entropy = log_total;
    }
    __device__ float lse() const { return max + log_total; }
    __device__ float4 kept() const { return make_float4(max, total, log_total, entropy); }
    __device__ float logp(float x) const { return max == -kInf ? -kInf : (x - max) - log_total; }
};

// grad_j = -p_j (a + b (ln p_j + entropy)), a more at the target: with z the exponent of a value's power, which is 2^off too
// large, 2^z (from + slope z).
struct Descent {
    float from, slope;

    __device__ Descent(const Scale &scale, float total, float log_total, float entropy, float up, float up_entropy)
    {
        const float each = 1.0f / (exp2_fast(scale.off) * total);
        from = -(up + up_entropy * (entropy - log_total - kLn2 * scale.off)) * each;
        slope = -up_entropy * kLn2 * each;
    }
};

// Where a workgroup, or with kThreads 64 a wavefront by itself, puts side by side what may be among a row's best.
template <int kThreads>
struct PickRoom {
    static constexpr uint32_t kMost = kThreads < 256 ? 128 : 256;
    static constexpr uint32_t kMostPacks = kThreads < 256 ? 64 : 192;
    uint32_t best[kThreads];
    uint64_t picked[kMost], rounds[kThreads / 64];
    u32x4_t pack[kMostPacks];
    uint32_t column[kMostPacks];
    uint32_t count, packs;

    __device__ __forceinline__ void add(uint32_t order, uint32_t sym)
    {
        const uint32_t at = atomicAdd(&count, 1u);
        if (at < kMost) picked[at] = (uint64_t)order << 32 | (0xFFFFFFFFu - sym);
    }
};
template <int kThreads>
__device__ __forceinline__ void meet()
{
    if constexpr (kThreads > 64) {
        __syncthreads();
    } else {  // a wavefront's accesses to LDS are done in order: the compiler has to leave them in it
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// A row, or a run of it, in registers: kLanes lanes hold kPer packs of 16 bytes each.  A pack that would reach over the
// end begins earlier, and what another holds of it already is ruled out.  Rows need a pack's values at least.
template <class T, int kLanes, int kPer>
struct LogitsRow {
    static constexpr int kVec = 16 / sizeof(T);
    static constexpr int kThreads = kLanes > 256 ? kLanes : 256;
    static constexpr int kRows = kThreads / kLanes;  // that a workgroup has in hand
    static constexpr int kWithin = kLanes < 64 ? kLanes : 64, kWaves = kLanes > 64 ? kLanes / 64 : 1;
    static constexpr uint32_t kValues = kLanes * kPer * kVec;
    // Wavefronts a SIMD that registers are kept down to.  Two workgroups of 1024 instead of one, so that one's values are on
    // their way while the other is worked on: training 16384 x 65536 bf16 in 788 us instead of 842, 4000 x 33000 in 139
    // instead of 153.  Three wavefronts of 16 packs a lane and five of 8 are what their registers allow as they are (with two of
    // 16 asked for, 16384 x 32768 bf16 with 20 alternatives takes the same 221 us).
    static constexpr int kResident = kLanes == 1024 ? (kPer == 8 ? 8 : 4) : kPer == 16 ? 3 : kPer == 8 ? 5 : 1;

    uint32_t lane, row_in_block;

    __device__ LogitsRow() : lane(threadIdx.x % kLanes), row_in_block(kRows > 1 ? threadIdx.x / kLanes : 0) {}
    __device__ uint32_t place(int q, uint32_t begin) const { return begin + (q * kLanes + lane) * kVec; }
    __device__ uint32_t column(int q, uint32_t begin, uint32_t end) const { return min(place(q, begin), end - kVec); }
    __device__ int twice(int q, uint32_t begin, uint32_t end) const
    {
        return (int)min(place(q, begin) - column(q, begin, end), (uint32_t)kVec);
    }
    // Where column `column` of a row at p is, by way of the run's first place: the same for a workgroup's lanes, and what
    // is added to it fits 32 bits, so that a pack's address takes one register.
    template <class V>
    __device__ static V *address(V *p, uint32_t column, uint32_t begin, uint32_t end)
    {
        const uint32_t first = min(begin, end - kVec);
        using Byte = std::conditional_t<std::is_const_v<V>, const char, char>;
        return (V *)((Byte *)(p + first) + (uint32_t)((column - first) * (uint32_t)sizeof(T)));
    }
    __device__ void load(const T *p, uint32_t begin, uint32_t end, Raw<T> (&x)[kPer]) const
    {
#pragma unroll
        for (int q = 0; q < kPer; ++q) x[q] = Raw<T>::load(address(p, column(q, begin, end), begin, end));
    }
    // Packs that are gone through, for all lanes the same: those with values of the row in them, up to a whole group.  The others are
    // loaded, with the row's last values, and left alone.  bf16, us with these groups, with four in all, with whole rows and pack by
    // pack: training 16384 x 65536 782 779 770 789, 8000 x 100003 839 866 860 884, 4000 x 33000 136 157 157 126; laws
    // 16384 x 5000 33.5 34.3 38.4 32.5, 65536 x 256 9.3 9.9 9.4 9.3, 4093 x 100003 with 5 alternatives 182 184 191 176.
    static constexpr int kGroup = kLanes == 1024 ? 2 : kPer < 4 ? kPer : 4;
    __device__ int used(uint32_t begin, uint32_t end) const
    {
        return (int)((end - begin + kLanes * kVec * kGroup - 1) / (kLanes * kVec * kGroup)) * kGroup;
    }
    template <class F>
    __device__ static void for_used(int used, F f)
    {
#pragma unroll
        for (int g = 0; g < kPer; g += kGroup)
            if (g < used)
#pragma unroll
                for (int q = g; q < g + kGroup; ++q) f(q);
    }
    __device__ void rule_out(uint32_t begin, uint32_t end, Raw<T> (&x)[kPer]) const
    {
        const int whole = (int)((end - begin) / (kLanes * kVec));
        if (whole < kPer)
#pragma unroll
            for (int q = 0; q < kPer; ++q)
                if (q >= whole) x[q].rule_out(twice(q, begin, end));
    }
    // Neither what the values were widened to nor where the packs lie is kept for after: worked out again it takes no registers.
    __device__ void forget(Raw<T> (&x)[kPer])
    {
        asm volatile("" : "+v"(lane));
#pragma unroll
        for (int q = 0; q < kPer; ++q) x[q].forget();
    }
    // of each pack, and of all
    __device__ float largest(const Raw<T> (&x)[kPer], int used, float (&of)[kPer]) const
    {
        float m = -kInf;
        for_used(used, [&](int q) {
            of[q] = max3(x[q][0], x[q][1], x[q][2]);
            if constexpr (kVec == 8) of[q] = max3(of[q], max3(x[q][3], x[q][4], x[q][5]), x[q][6]);
            of[q] = max3(of[q], x[q][kVec - 1], of[q]);
            m = max3(m, of[q], m);
        });
        return m;
    }
    // The keys of the values whose order is `line` at least.  Packs with such values are put into LDS and looked through
    // there by all threads: to take them apart value by value in registers would be code for each of them.
    __device__ bool collect(const Raw<T> (&x)[kPer], const float (&of)[kPer], uint32_t begin, uint32_t end, int used, uint32_t line,
                            PickRoom<kLanes> &room) const
    {
        const float least = value_of((uint64_t)line << 32);
        for_used(used, [&](int q) {
            if (of[q] >= least) {
                const uint32_t at = atomicAdd(&room.packs, 1u);
                if (at < room.kMostPacks) room.pack[at] = x[q].bits, room.column[at] = column(q, begin, end);
            }
        });
        meet<kLanes>();
        const uint32_t packs = room.packs;
        if (packs > room.kMostPacks) return false;
        for (uint32_t i = threadIdx.x & (kLanes - 1); i < packs * kVec; i += kLanes) {
            const uint32_t order = order_of(widen(((const T *)&room.pack[i / kVec])[i % kVec]));
            if (order >= line) room.add(order, room.column[i / kVec] + i % kVec);
        }
        return true;
    }
    // f(order, symbol) for each of the lane's values
    template <class F>
    __device__ void each(Raw<T> (&x)[kPer], uint32_t begin, uint32_t end, int used, F f) const
    {
        for_used(used, [&](int q) {
            x[q].forget();
            const uint32_t column_q = column(q, begin, end);
#pragma unroll
            for (int k = 0; k < kVec; ++k) f(order_of(x[q][k]), column_q + k);
        });
    }
    // The same from memory, in little code
    template <class F>
    __device__ void again(const T *p, uint32_t begin, uint32_t end, F f) const
    {
#pragma unroll 1
        for (int q = 0; q < kPer; ++q)
#pragma unroll 1
            for (uint32_t j = place(q, begin); j < min(place(q, begin) + kVec, end); ++j) f(order_of(widen(p[j])), j);
    }
    // The row's tally in all its lanes; `room` holds 2 * kWaves, its halves are used in turn.
    __device__ Tally tally(const Raw<T> (&x)[kPer], int used, float own, Tally *room, int half) const
    {
        const float max = lanes_reduce<kWithin>(own, MaxFloat());
        const Scale scale(max);
        float total[2] = {0.0f, 0.0f}, inside[2] = {0.0f, 0.0f};
        scale.by_power([&](auto apart) {
            for_used(used, [&](int q) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float z = scale.power<apart.value>(x[q][k]), e = exp2_fast(z);
                    total[k & 1] += e;
                    inside[k & 1] = __builtin_fmaf(e, fmaxf(z, kLeast), inside[k & 1]);
                }
            });
        });
        // the largest value's power is 2^off to the last bit, and by itself makes a total of 1
        const float whole = lanes_reduce<kWithin>(total[0] + total[1], Sum()), first = exp2_fast(scale.off);
        Tally t = {max, whole / first, (lanes_reduce<kWithin>(inside[0] + inside[1], Sum()) - scale.off * whole) * __builtin_amdgcn_rcpf(first)};
        if constexpr (kWaves > 1) {
            room += half * kWaves;
            if ((threadIdx.x & 63) == 0) room[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)] = t;
            __syncthreads();
            t = room[threadIdx.x & (kWaves - 1)];
#pragma unroll
            for (int d = 1; d < kWaves; d *= 2) {
                const Tally o = {__shfl_xor(t.max, d, 64), __shfl_xor(t.total, d, 64), __shfl_xor(t.inside, d, 64)};
                t = both(t, o);
            }
        }
        return t;
    }
};

// The `top` best of what kThreads threads hold: a workgroup, or with 64 a wavefront by itself.  `best` is the highest order
// (see order_of) among the calling thread's values; `collect` puts the keys of all threads' values from an order on into
// `room`, or says that they are too many; `again` calls its argument with order and symbol of all of the thread's values, for
// the rare way below; `put` is called, once for each place in 0 .. top-1 and by some thread, with the place and the key that
// belongs there, or 0.
//
// The top-th best of the threads' best values has `top` values at least that are as good, and few more in what a model
// answers with; those are put side by side, and each one's place is the number of better ones.  The more threads stand
// for a row the fewer there are to look at: four wavefronts that each pick by themselves before they join take longer
// (16384 x 32768 bf16, 20 alternatives: 417 against 294 us).  Rows with many equal values may have too many of them:
// then the best that is worse than the last is looked for `top` times.
template <int kThreads, class Collect, class Again, class Put>
__device__ void pick_top(uint32_t top, int bits, uint32_t best, Collect collect, Again again, Put put, PickRoom<kThreads> &room)
{
    constexpr int kEach = kThreads / 64;
    const uint32_t thread = threadIdx.x & (kThreads - 1);
    meet<kThreads>();  // `room` may be in use from a row before
    if (kEach > 1) room.best[thread] = best;
    if (thread == 0) room.count = room.packs = 0;
    meet<kThreads>();
    // the highest order that `top` threads' best reach, bit by bit from the top; `bits` is what the type's values differ in
    uint32_t b[kEach] = {best}, line = 0;
    if (kEach > 1)
#pragma unroll
        for (int i = 0; i < kEach; ++i) b[i] = room.best[i * 64 + (threadIdx.x & 63)];
    for (int bit = 31; bit >= 32 - bits; --bit) {
        const uint32_t next = line | 1u << bit;
        uint32_t reach = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) reach += (uint32_t)__builtin_popcountll(__ballot(b[i] >= next));
        if (reach >= top) line = next;
    }
    line = max(line, kOrderNone + 1);  // -inf is no alternative
    const bool few = collect(line, room);
    meet<kThreads>();
    const uint32_t count = room.count;
    if (few && count <= room.kMost) {
        for (uint32_t i = thread; i < count; i += kThreads) {
            const uint64_t key = room.picked[i];
            uint32_t better = 0;
            for (uint32_t j = 0; j < count; ++j) better += room.picked[j] > key;
            if (better < top) put(better, key);
        }
        for (uint32_t i = count + thread; i < top; i += kThreads) put(i, (uint64_t)0);
        return;
    }
    uint64_t below = ~0ull;
    for (uint32_t i = 0; i < top; ++i) {
        uint64_t next = 0;
        if (best >= line)
            again([&](uint32_t order, uint32_t sym) {
                const uint64_t key = (uint64_t)order << 32 | (0xFFFFFFFFu - sym);
                if (order >= line && key < below && key > next) next = key;
            });
        below = block_reduce<kThreads / 64>(next, Max(), room.rounds);
        if (thread == 0) put(i, below);
    }
}
template <class T>
constexpr int kOrderBits = sizeof(T) == 4 ? 32 : __is_same(T, __bf16) ? 16 : 19;

__device__ __forceinline__ void put_alternative(const LogitsArgs &a, const Law &law, uint32_t row, uint32_t place, uint64_t key)
{
    const size_t at = (size_t)row * a.top + place;
    const bool none = !(law.max == law.max);  // NaN or +inf in the row
    a.top_sym[at] = key && !none ? (int32_t)(0xFFFFFFFFu - (uint32_t)key) : -1;
    a.top_logp[at] = none ? __builtin_nanf("") : key ? law.logp(value_of(key)) : -kInf;
}

// The gradient of one pack's values, the first of which is that of symbol `column` and goes to `to`; `up` more at the target.
template <bool kApart, class T>
__device__ __forceinline__ void put_gradient(const Raw<T> &x, T *to, uint32_t column, int twice, const Scale &scale, const Descent &d_of,
                                             bool in, int64_t t, float up, bool zeros)
{
    constexpr int kVec = 16 / sizeof(T);
    float d[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float z = fmaxf(scale.power<kApart>(x[i]), kLeast);
        d[i] = exp2_fast(z) * __builtin_fmaf(d_of.slope, z, d_of.from);
    }
    const uint32_t k = (uint32_t)t - column;
    if (in && k < (uint32_t)kVec)
#pragma unroll
        for (int i = 0; i < kVec; ++i) d[i] += i == (int)k ? up : 0.0f;
    if (zeros)
#pragma unroll
        for (int i = 0; i < kVec; ++i) d[i] = 0.0f;
    if (twice == 0) {
        Raw<T>::of(d).store(to);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i >= twice) to[i] = (T)d[i];
    }
}

// What k_logits does: the rows' laws, alternatives too, or (whole rows) their gradient from the same registers.
enum Task { kLaw, kPick, kTrainRows };

// A row, or a run of one, a workgroup or a part of it; a row that is one run is finished here.  Measured (whole calls):
// laws of 16384 x 32768 bf16 191 us (5.6 TB/s), of 65536 x 256 f32 12.4 (5.4); with alternatives 4093 x 100003 bf16 165 (5.0,
// with the joining kernel); with the gradient 16384 x 65536 bf16 747 (5.8), 65536 x 256 bf16 16.0 (4.3).
template <class T, int kLanes, int kPer, Task kTask>
__global__ __launch_bounds__((LogitsRow<T, kLanes, kPer>::kThreads), (LogitsRow<T, kLanes, kPer>::kResident)) void k_logits(LogitsArgs a)
{
    using Row = LogitsRow<T, kLanes, kPer>;
    constexpr int kVec = Row::kVec;
    constexpr bool kTrain = kTask == kTrainRows;
    __shared__ Tally room[2 * Row::kWaves];
    constexpr bool kPicks = kTask == kPick && kLanes >= 64;
    constexpr int kPickers = kPicks ? kLanes : 64;
    __shared__ PickRoom<kPickers> picked[kPicks ? Row::kRows : 1];
    Row r;
    const uint32_t splits = kTrain ? 1 : a.splits;
    const uint64_t items = (uint64_t)a.rows * splits, step = (uint64_t)gridDim.x * Row::kRows;
    uint64_t item = (uint64_t)blockIdx.x * Row::kRows + r.row_in_block;
    int half = 0;
    for (; item < items; item += step) {
        const uint32_t row = (uint32_t)(splits == 1 ? item : item / splits), begin = (uint32_t)(item - (uint64_t)row * splits) * a.span;
        const bool whole = splits == 1;
        // what comes with a row is asked for before its values: loads come back in order
        const int64_t t = a.target && whole ? target_of(a, row) : -1;
        const float up_given = kTrain ? a.up_logp[row] : 0.0f, up_entropy = kTrain && a.up_entropy ? a.up_entropy[row] : 0.0f;
        Raw<T> x[kPer];
        const uint32_t end = min(begin + a.span, a.num_sym);
        r.load((const T *)a.x + row * a.stride, begin, end, x);
        r.rule_out(begin, end, x);
        const int used = r.used(begin, end);
        float of[kPer];
        const float own = r.largest(x, used, of);
        r.forget(x);
        const Tally tally = r.tally(x, used, own, room, half);
        r.forget(x);
        half ^= 1;
        const Law law(tally);
        if (!whole) {
            if (r.lane == 0) a.part[item] = make_float4(tally.max, tally.total, tally.inside, 0.0f);
        } else {
            if (r.lane == 0) {
                if (a.entropy) a.entropy[row] = law.entropy;
                if (a.lse) a.lse[row] = law.lse();
                if (!kTrain && a.law) a.law[row] = law.kept();
                if (a.logp && (t < 0 || t >= (int64_t)a.num_sym)) a.logp[row] = t < 0 ? 0.0f : __builtin_nanf("");
            }
            const bool in = t >= 0 && t < (int64_t)a.num_sym;
            if (a.logp && in)
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    const uint32_t k = (uint32_t)t - r.column(q, begin, end);
                    if (k < (uint32_t)kVec && (int)k >= r.twice(q, begin, end)) {
                        a.logp[row] = law.logp(x[q].at(k));
                    }
                }
            if constexpr (kTrain) {
                const float up = t < 0 ? 0.0f : up_given;
                const Scale scale(tally.max);
                Descent d(scale, law.total, law.log_total, law.entropy, up, up_entropy);
                const bool zeros = (up == 0.0f && up_entropy == 0.0f) || law.max == -kInf;
                if (t >= (int64_t)a.num_sym || !(law.max == law.max)) d.from = __builtin_nanf("");
                T *grad = (T *)a.grad + row * a.grad_stride;
                r.forget(x);
                scale.by_power([&](auto apart) {
                    r.for_used(used, [&](int q) {
                        const uint32_t column = r.column(q, begin, end);
                        put_gradient<apart.value>(x[q], Row::address(grad, column, begin, end), column, r.twice(q, begin, end), scale, d, in, t, up, zeros);
                    });
                });
            }
        }
        if constexpr (kPicks) {
            pick_top<kLanes>(
                a.top, kOrderBits<T>, order_of(own), [&](uint32_t line, auto &to) { return r.collect(x, of, begin, end, used, line, to); },
                [&](auto f) { r.again((const T *)a.x + row * a.stride, begin, end, f); },
                [&](uint32_t place, uint64_t key) {
                    if (whole)
                        put_alternative(a, law, row, place, key);
                    else
                        a.part_top[item * a.top + place] = key;
                },
                picked[r.row_in_block]);
        } else if constexpr (kTask == kPick) {
            // few values a lane, in whole rows: the best that is worse than the last, `top` times
            uint64_t below = ~0ull;
            for (uint32_t i = 0; i < a.top; ++i) {
                uint64_t best = 0;
                r.each(x, begin, end, used, [&](uint32_t order, uint32_t sym) {
                    const uint64_t key = (uint64_t)order << 32 | (0xFFFFFFFFu - sym);
                    if (order > kOrderNone && key < below && key > best) best = key;
                });
                const uint32_t high = lanes_reduce<Row::kWithin>((uint32_t)(best >> 32), Max());
                const uint32_t low = lanes_reduce<Row::kWithin>(best >> 32 == high ? (uint32_t)best : 0u, Max());
                below = (uint64_t)high << 32 | low;
                if (below == 0) {  // no more
                    for (uint32_t j = i + r.lane; j < a.top; j += kLanes) put_alternative(a, law, row, j, 0);
                    break;
                }
                if (r.lane == 0) put_alternative(a, law, row, i, below);
            }
        }
    }
}

// The runs of a row put together by kThreads threads: a workgroup, or a wavefront.  A launch and a few trips to memory: 5.0 us
// for one row of 32 runs with 20 alternatives each, 7.3 for 4093 rows of 7 runs with 5.
template <int kThreads>
__global__ __launch_bounds__(256) void k_logits_join(LogitsArgs a, uint32_t type)
{
    constexpr uint32_t kRows = 256 / kThreads;
    constexpr int kHeld = 4;
    __shared__ PickRoom<kThreads> picked[kRows];
    __shared__ Tally room[4];
    const uint32_t thread = threadIdx.x & (kThreads - 1), which = threadIdx.x / kThreads;
    for (uint64_t row = (uint64_t)blockIdx.x * kRows + which; row < a.rows; row += (uint64_t)gridDim.x * kRows) {
        // the first keys are asked for with the rest, and kept
        const uint64_t *keys = a.part_top + row * a.splits * a.top;
        const uint32_t count = a.splits * a.top;
        uint64_t held[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) held[i] = i * kThreads + thread < count ? keys[i * kThreads + thread] : 0;
        Tally t = {-kInf, 0.0f, 0.0f};
        for (uint32_t s = thread; s < a.splits; s += kThreads) {
            const float4 p = a.part[row * a.splits + s];
            t = both(t, {p.x, p.y, p.z});
        }
        const auto over = [&](int lanes) {
            for (int d = 1; d < lanes; d *= 2) t = both(t, {__shfl_xor(t.max, d, 64), __shfl_xor(t.total, d, 64), __shfl_xor(t.inside, d, 64)});
        };
        over(64);
        if (kThreads > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = t;
            __syncthreads();
            t = room[threadIdx.x & 3];
            over(4);
        }
        const Law law(t);
        if (thread == 0) {
            if (a.entropy) a.entropy[row] = law.entropy;
            if (a.lse) a.lse[row] = law.lse();
            if (a.law) a.law[row] = law.kept();
            if (a.logp) {
                const int64_t target = target_of(a, (uint32_t)row);
                float at = 0.0f;
                if (target >= 0 && target < (int64_t)a.num_sym) {
                    const uint64_t i = row * a.stride + (uint64_t)target;
                    at = type == PILC_F32 ? ((const float *)a.x)[i] : type == PILC_BF16 ? widen(((const bf16_t *)a.x)[i]) : widen(((const f16_t *)a.x)[i]);
                }
                a.logp[row] = target < 0 ? 0.0f : target >= (int64_t)a.num_sym ? __builtin_nanf("") : law.logp(at);
            }
        }
        if (a.top) {
            uint32_t best = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) best = max(best, (uint32_t)(held[i] >> 32));
            for (uint32_t i = kHeld * kThreads + thread; i < count; i += kThreads) best = max(best, (uint32_t)(keys[i] >> 32));
            const auto again = [&](auto f) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i) f((uint32_t)(held[i] >> 32), 0xFFFFFFFFu - (uint32_t)held[i]);
                for (uint32_t i = kHeld * kThreads + thread; i < count; i += kThreads) f((uint32_t)(keys[i] >> 32), 0xFFFFFFFFu - (uint32_t)keys[i]);
            };
            const auto collect = [&](uint32_t line, auto &room) {
                again([&](uint32_t order, uint32_t sym) {
                    if (order >= line) room.add(order, sym);
                });
                return true;
            };
            pick_top<kThreads>(
                a.top, type == PILC_BF16 ? kOrderBits<bf16_t> : type == PILC_F16 ? kOrderBits<f16_t> : kOrderBits<float>, best, collect, again,
                [&](uint32_t place, uint64_t key) { put_alternative(a, law, (uint32_t)row, place, key); }, picked[which]);
        }
    }
}

// The gradient where a row's law is known: run by run, 16 KB at most, read once and written once.  Memory bounds it: 8190 x
// 50001 f16 275 us (5.9 TB/s).  A caller's law is an lse and an entropy; pilc_logprobs_train leaves largest value and total apart,
// as an lse of 32 bits has a 2^-24th of its size less to say about p.
template <class T, int kLanes, int kPer>
__global__ __launch_bounds__((LogitsRow<T, kLanes, kPer>::kThreads)) void k_logits_grad(LogitsArgs a)
{
    using Row = LogitsRow<T, kLanes, kPer>;
    const Row r;
    const uint64_t items = (uint64_t)a.rows * a.splits, step = (uint64_t)gridDim.x * Row::kRows;
    for (uint64_t item = (uint64_t)blockIdx.x * Row::kRows + r.row_in_block; item < items; item += step) {
        const uint32_t row = (uint32_t)(a.splits == 1 ? item : item / a.splits), begin = (uint32_t)(item - (uint64_t)row * a.splits) * a.span;
        const uint32_t end = min(begin + a.span, a.num_sym);
        const int64_t t = target_of(a, row);
        const float up = t < 0 ? 0.0f : a.up_logp[row], up_entropy = a.up_entropy ? a.up_entropy[row] : 0.0f;
        const float4 law = a.law ? a.law[row] : make_float4(a.lse_in[row], 1.0f, 0.0f, a.up_entropy ? a.entropy_in[row] : 0.0f);
        const bool zeros = (up == 0.0f && up_entropy == 0.0f) || law.x == -kInf;
        const Scale scale(law.x);
        Descent d(scale, law.y, law.z, law.w, up, up_entropy);
        if (t >= (int64_t)a.num_sym || !(law.x == law.x)) d.from = __builtin_nanf("");
        Raw<T> x[kPer];
        r.load((const T *)a.x + row * a.stride, begin, end, x);
        T *grad = (T *)a.grad + row * a.grad_stride;
        const bool in = t >= 0 && t < (int64_t)a.num_sym;
        scale.by_power([&](auto apart) {
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                const uint32_t column = r.column(q, begin, end);
                put_gradient<apart.value>(x[q], Row::address(grad, column, begin, end), column, r.twice(q, begin, end), scale, d, in, t, up, zeros);
            }
        });
    }
}

// Rows shorter than a pack: a thread a row.  kTrain: with the gradient; kGrad: the gradient by a law that is known.
template <class T, bool kTrain, bool kGrad>
__global__ __launch_bounds__(256) void k_logits_short(LogitsArgs a)
{
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < a.rows; i += gridDim.x * 256ull) {
        const uint32_t row = (uint32_t)i;
        const T *x = (const T *)a.x + row * a.stride;
        const int64_t t = a.target ? target_of(a, row) : -1;
        const bool in = t >= 0 && t < (int64_t)a.num_sym;
        float largest = -kInf;
        for (uint32_t j = 0; j < a.num_sym; ++j) largest = fmaxf(largest, widen(x[j]));
        const float known = kGrad ? a.lse_in[row] : largest, center = known == -kInf ? 0.0f : known;
        const auto power = [&](float v) { return (v - center) * kLog2e; };
        float up = 0.0f, up_entropy = 0.0f, total = 1.0f, log_total = 0.0f, entropy = 0.0f;
        if (kTrain || kGrad) {
            up = t < 0 ? 0.0f : a.up_logp[row];
            up_entropy = a.up_entropy ? a.up_entropy[row] : 0.0f;
        }
        bool zeros = up == 0.0f && up_entropy == 0.0f, spoilt = t >= (int64_t)a.num_sym;
        if constexpr (kGrad) {
            if (a.up_entropy) entropy = a.entropy_in[row];
            zeros |= known == -kInf;
            spoilt |= !(known == known);
        } else {
            Tally tally = {largest, 0.0f, 0.0f};
            float first = 0.0f, rest = 0.0f;  // the largest's power and the others', apart: a nearly certain symbol's ln p is the others'
            bool met = false;
            for (uint32_t j = 0; j < a.num_sym; ++j) {
                const float v = widen(x[j]), z = power(v), e = exp2_fast(z);
                const bool it = v == largest && !met;
                met |= it;
                it ? first = e : rest += e;
                tally.inside += e * fmaxf(z, kLeast);
            }
            tally.total = first + rest;
            Law law(tally);
            if (law.max > -kInf) law.log_total = log1pf(rest);
            if (a.entropy) a.entropy[row] = law.entropy;
            if (a.lse) a.lse[row] = law.lse();
            if (a.logp) a.logp[row] = t < 0 ? 0.0f : spoilt ? __builtin_nanf("") : law.logp(widen(x[t]));
            uint64_t below = ~0ull;
            for (uint32_t k = 0; k < a.top; ++k) {
                uint64_t best = 0;
                for (uint32_t j = 0; j < a.num_sym && k < a.num_sym; ++j) {
                    const uint64_t key = key_of(widen(x[j]), j);
                    if (key >> 32 > kOrderNone && key < below && key > best) best = key;
                }
                below = best;
                put_alternative(a, law, row, k, best);
            }
            total = law.total, log_total = law.log_total, entropy = law.entropy;
            zeros |= law.max == -kInf;
            spoilt |= !(law.max == law.max);
        }
        if constexpr (kTrain || kGrad) {
            float from = -(up + up_entropy * (entropy - log_total)) / total, slope = -up_entropy * kLn2 / total;
            if (spoilt) from = __builtin_nanf("");
            T *grad = (T *)a.grad + row * a.grad_stride;
            for (uint32_t j = 0; j < a.num_sym; ++j) {
                const float z = fmaxf(power(widen(x[j])), kLeast);
                float d = exp2_fast(z) * __builtin_fmaf(slope, z, from);
                if (in && (int64_t)j == t) d += up;
                grad[j] = (T)(zeros ? 0.0f : d);
            }
        }
    }
}

static bool logits_shape_ok(const pilc_logits_shape *s)
{
    return s && s->num_sym >= 1 && s->num_sym <= 0x7FFFFFFFu && s->stride >= s->num_sym && s->stride <= (1ull << 48) && s->dtype <= PILC_F16 &&
           s->target_type <= PILC_I64 && s->top <= (uint32_t)kMaxTop;
}

static bool logits_in_ok(const pilc_logits_shape *s, const void *logits, const void *target)
{
    const size_t target_bytes = s->target_type == PILC_U8 ? 1 : s->target_type == PILC_I32 ? 4 : 8;
    return logits && aligned_to(logits, value_bytes(s->dtype)) && aligned_to(target, target_bytes);
}

// How rows are gone through.  Rows of up to 64 KB, in the registers of a workgroup of 256, are one run; longer ones go in
// runs of 32 KB, of which more are on their way at a time (4093 x 100003 bf16 with 5 alternatives: 201 us, in runs of 64 KB 217).  With few rows
// runs are as much smaller as it takes to give every compute unit two.
struct LogitsPlan {
    uint32_t splits, span;
};
constexpr uint32_t kWholeRow = 64 << 10, kLongestRun = 32 << 10, kShortestRun = 8 << 10;
static LogitsPlan logits_plan(uint32_t rows, uint32_t num_sym, uint32_t value, uint32_t whole, uint32_t longest, uint32_t shortest)
{
    const uint32_t vec = 16 / value, needed = num_sym <= whole / value ? 1 : div_up(num_sym, longest / value), most = div_up(num_sym, shortest / value);
    const uint32_t wanted = div_up(2 * compute_units(), std::max(rows, 1u)), splits = std::max(needed, std::min(wanted, most));
    // many rows: full runs, so that only the last one has packs without values
    const uint32_t span = splits == needed ? (splits == 1 ? num_sym : longest / value) : div_up(div_up(num_sym, splits), vec) * vec;
    return {div_up(num_sym, span), span};
}
// Whether pilc_logprobs_train keeps whole rows in registers: up to 256 KB, those of a workgroup of 1024.  Few rows of over
// 32 KB keep more of the GPU busy in runs, which costs two launches more (bf16, us by rows and by runs: 16000 symbols 10.8
// and 11.0 for 16 rows; 50000 symbols 14.5 and 12.8 for 16, 16.9 and 17.9 for 128; 131072 symbols 24.5 and 20.2 for 64, 26.6
// and 26.6 for 128).
constexpr uint32_t kLongestRow = 256 << 10;
static bool train_by_row(uint32_t rows, uint32_t num_sym, uint32_t value)
{
    const uint64_t bytes = (uint64_t)num_sym * value;
    return bytes <= kLongestRow && (bytes <= (32u << 10) || rows >= compute_units() / 2);
}

// What the runs of split rows leave for the kernel that puts them together.
static size_t parts_bytes(const LogitsPlan &p, uint32_t rows, uint32_t top)
{
    return p.splits > 1 ? (size_t)rows * p.splits * (sizeof(float4) + sizeof(uint64_t) * top) : 0;
}
static size_t logits_workspace(const pilc_logits_shape &s)
{
    size_t most = 256;
    for (uint32_t value : {2u, 4u}) {  // whatever the type, so that a caller need not ask for each
        const LogitsPlan p = logits_plan(s.rows, s.num_sym, value, kWholeRow, kLongestRun, kShortestRun);
        // pilc_logprobs_train, where it goes two ways, keeps the rows' laws behind the parts
        const size_t kept = s.top == 0 && !train_by_row(s.rows, s.num_sym, value) ? sizeof(float4) * (size_t)s.rows : 0;
        most = std::max(most, parts_bytes(p, s.rows, s.top) + kept);
    }
    return most;
}

// Calls `go` with the lanes and packs a lane for runs of `bytes` bytes.  Alternatives of short rows are looked for by a whole
// wavefront where twice as many of its lanes as alternatives have values (20 alternatives: 65536 x 256 f32 104 us in
// groups of 16 lanes, 53 by 64; 32567 x 655 bf16 with 32 alternatives 304 and 47.  The line is a rough one:
// 65536 x 256 bf16 takes 104 with 20, below it, and by 64 lanes would take 57; with 5, above it, 40, and in groups 34).
//
// Whole rows of up to 16 KB are a wavefront's by itself, which has no other to wait for (16384 x 4096 bf16: 26 us, by
// workgroups 38; 30000 x 3000 f32: 61 and 82); runs of a split row, of which there are few, a workgroup's.
template <Task kTask, class Go>
static void logits_row(uint32_t bytes, uint32_t top, bool whole, Go go)
{
    using std::integral_constant;
    const auto with = [&](auto lanes, auto per) {
        if (bytes > (uint32_t)(lanes.value * per.value * 16)) return false;
        go(lanes, per);
        return true;
    };
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    const integral_constant<int, 8> eight;
    const integral_constant<int, 16> sixteen;
    const integral_constant<int, 64> wave;
    const integral_constant<int, 256> group;
    if constexpr (kTask == kPick)
        if (bytes >= 32 * top && (with(wave, one) || with(wave, two))) return;
    const bool done = with(integral_constant<int, 8>(), one) || with(integral_constant<int, 8>(), four) || with(integral_constant<int, 16>(), four) ||
                      with(integral_constant<int, 32>(), four) || with(wave, four) || (whole && (with(wave, eight) || with(wave, sixteen))) ||
                      with(group, two) || with(group, four) || with(group, eight) || with(group, sixteen);
    if constexpr (kTask == kTrainRows)
        if (!done) (void)(with(integral_constant<int, 1024>(), eight) || with(integral_constant<int, 1024>(), sixteen));
}

// A workgroup for each `rows` of the rows or runs: what one asks for early is no gain over what the others ask for
// beside it (65536 x 256 bf16, training: 17.6 us, with workgroups that go from row to row, the next one on its way, 19.1).
static uint32_t logits_blocks(uint64_t items, uint32_t rows) { return (uint32_t)std::min<uint64_t>((items + rows - 1) / rows, 1u << 21); }

template <class T, Task kTask>
static void launch_logits(const LogitsArgs &a, hipStream_t stream)
{
    if (a.num_sym < 16 / sizeof(T)) {
        k_logits_short<T, kTask == kTrainRows, false><<<(uint32_t)std::min<uint64_t>((a.rows + 255ull) / 256, 1u << 20), 256, 0, stream>>>(a);
        return;
    }
    logits_row<kTask>(a.span * (uint32_t)sizeof(T), a.top, a.splits == 1, [&](auto lanes, auto per) {
        using Row = LogitsRow<T, decltype(lanes)::value, decltype(per)::value>;
        const uint32_t blocks = logits_blocks((uint64_t)a.rows * a.splits, Row::kRows);
        k_logits<T, decltype(lanes)::value, decltype(per)::value, kTask><<<blocks, Row::kThreads, 0, stream>>>(a);
    });
}

// The law of each row; the runs of split rows are put together by a second kernel.
template <class T>
static void launch_law(LogitsArgs a, uint32_t type, void *workspace, hipStream_t stream)
{
    const LogitsPlan p = logits_plan(a.rows, a.num_sym, sizeof(T), kWholeRow, kLongestRun, kShortestRun);
    a.splits = p.splits, a.span = std::min(p.span, a.num_sym);
    a.part = (float4 *)workspace;
    a.part_top = (uint64_t *)(a.part + (size_t)a.rows * a.splits);
    if (a.top)
        launch_logits<T, kPick>(a, stream);
    else
        launch_logits<T, kLaw>(a, stream);
    if (a.splits == 1) return;
    // by wavefronts, or few rows with many keys or runs by workgroups (bf16, 131072 symbols, 20 alternatives: one row 12.4 and
    // 10.5 us, 64 rows 13.7 and 13.8; without alternatives one row 5.9 and 6.3)
    if (a.splits > (a.top ? 16u : 256u))
        k_logits_join<256><<<std::min(a.rows, 1u << 20), 256, 0, stream>>>(a, type);
    else
        k_logits_join<64><<<std::min(div_up(a.rows, 4), 1u << 20), 256, 0, stream>>>(a, type);
}

template <class T>
static void launch_grad(LogitsArgs a, hipStream_t stream)
{
    if (a.num_sym < 16 / sizeof(T)) {
        k_logits_short<T, false, true><<<(uint32_t)std::min<uint64_t>((a.rows + 255ull) / 256, 1u << 20), 256, 0, stream>>>(a);
        return;
    }
    constexpr uint32_t kRun = 16 << 10;
    const LogitsPlan p = logits_plan(a.rows, a.num_sym, sizeof(T), kRun, kRun, kShortestRun);
    a.splits = p.splits, a.span = std::min(p.span, a.num_sym);
    using std::integral_constant;
    const auto with = [&](auto lanes, auto per) {
        using Row = LogitsRow<T, decltype(lanes)::value, decltype(per)::value>;
        if (a.span > Row::kValues) return false;
        k_logits_grad<T, decltype(lanes)::value, decltype(per)::value>
            <<<logits_blocks((uint64_t)a.rows * a.splits, Row::kRows), Row::kThreads, 0, stream>>>(a);
        return true;
    };
    (void)(with(integral_constant<int, 8>(), integral_constant<int, 1>()) || with(integral_constant<int, 8>(), integral_constant<int, 4>()) ||
           with(integral_constant<int, 16>(), integral_constant<int, 4>()) || with(integral_constant<int, 32>(), integral_constant<int, 4>()) ||
           with(integral_constant<int, 64>(), integral_constant<int, 4>()) || with(integral_constant<int, 256>(), integral_constant<int, 2>()) ||
           with(integral_constant<int, 256>(), integral_constant<int, 4>()));
}

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_logprobs_workspace_size(const pilc_logits_shape *shape, size_t *workspace_bytes_host)
{
    if (!logits_shape_ok(shape) || !workspace_bytes_host) return PILC_E_ARG;
    *workspace_bytes_host = logits_workspace(*shape);
    return PILC_OK;
}

int pilc_logprobs(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, float *logp_dev, float *entropy_dev,
                  float *lse_dev, int32_t *top_sym_dev, float *top_logp_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!logits_shape_ok(shape)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || (logp_dev && !target_dev) || (shape->top && (!top_sym_dev || !top_logp_dev)) ||
        !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(top_sym_dev, 4) ||
        !aligned_to(top_logp_dev, 4) || !workspace_dev || !aligned_to(workspace_dev, 256))
        return PILC_E_ARG;
    if (workspace_bytes < logits_workspace(*shape)) return PILC_E_WORKSPACE;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.logp = logp_dev, a.entropy = entropy_dev, a.lse = lse_dev, a.top_sym = top_sym_dev;
    a.top_logp = top_logp_dev, a.stride = shape->stride, a.rows = shape->rows, a.num_sym = shape->num_sym, a.top = shape->top;
    a.target_type = shape->target_type;
    return by_type(shape->dtype,
                   [&](auto *t) { launch_law<std::remove_pointer_t<decltype(t)>>(a, shape->dtype, workspace_dev, (hipStream_t)hip_stream); });
}

int pilc_logprobs_grad(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, const float *lse_dev,
                       const float *entropy_dev, const float *up_logp_dev, const float *up_entropy_dev, void *grad_dev,
                       uint64_t grad_stride, void *hip_stream)
{
    if (!logits_shape_ok(shape) || grad_stride < shape->num_sym || grad_stride > (1ull << 48)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || !target_dev || !lse_dev || !up_logp_dev || (up_entropy_dev && !entropy_dev) ||
        !grad_dev || !aligned_to(grad_dev, value_bytes(shape->dtype)) || !aligned_to(lse_dev, 4) || !aligned_to(entropy_dev, 4) ||
        !aligned_to(up_logp_dev, 4) || !aligned_to(up_entropy_dev, 4) || (grad_dev == logits_dev && grad_stride != shape->stride))
        return PILC_E_ARG;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.lse_in = lse_dev, a.entropy_in = entropy_dev, a.up_logp = up_logp_dev;
    a.up_entropy = up_entropy_dev, a.grad = grad_dev, a.grad_stride = grad_stride, a.stride = shape->stride, a.rows = shape->rows;
    a.num_sym = shape->num_sym, a.target_type = shape->target_type;
    return by_type(shape->dtype, [&](auto *t) { launch_grad<std::remove_pointer_t<decltype(t)>>(a, (hipStream_t)hip_stream); });
}

int pilc_logprobs_train(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, const float *up_logp_dev,
                        const float *up_entropy_dev, float *logp_dev, float *entropy_dev, float *lse_dev, void *grad_dev,
                        uint64_t grad_stride, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!logits_shape_ok(shape) || shape->top != 0 || grad_stride < shape->num_sym || grad_stride > (1ull << 48)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || !target_dev || !up_logp_dev || !logp_dev || !grad_dev ||
        !aligned_to(grad_dev, value_bytes(shape->dtype)) || !aligned_to(up_logp_dev, 4) || !aligned_to(up_entropy_dev, 4) ||
        !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(lse_dev, 4) || !workspace_dev ||
        !aligned_to(workspace_dev, 256) || (grad_dev == logits_dev && grad_stride != shape->stride))
        return PILC_E_ARG;
    if (workspace_bytes < logits_workspace(*shape)) return PILC_E_WORKSPACE;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.up_logp = up_logp_dev, a.up_entropy = up_entropy_dev, a.logp = logp_dev;
    a.entropy = entropy_dev, a.lse = lse_dev, a.grad = grad_dev, a.grad_stride = grad_stride, a.stride = shape->stride;
    a.rows = shape->rows, a.num_sym = shape->num_sym, a.target_type = shape->target_type;
    const hipStream_t stream = (hipStream_t)hip_stream;
    return by_type(shape->dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (train_by_row(a.rows, a.num_sym, sizeof(T))) {
            a.splits = 1, a.span = a.num_sym;
            launch_logits<T, kTrainRows>(a, stream);
            return;
        }
        // too few rows to keep the GPU busy one a workgroup, or too long ones: the law first, then the gradient by it
        const LogitsPlan p = logits_plan(a.rows, a.num_sym, sizeof(T), kWholeRow, kLongestRun, kShortestRun);
        a.law = (float4 *)((char *)workspace_dev + parts_bytes(p, a.rows, 0));
        launch_law<T>(a, shape->dtype, workspace_dev, stream);
        launch_grad<T>(a, stream);
    });
}

}  // extern "C"
