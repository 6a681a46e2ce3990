// Attention over the latent cache (include/ag_latent.h): one row a token is key and value of every query head,
//     S = scale * Q . row,   O = softmax(S) . row[0 .. L)
// so that the rows of a tile serve all heads of all the query rows that see it.  Decode reads ctx * (L + R) * 2 bytes for 2 H ctx (2 L + R) operations: 242 a byte at
// 128 heads, where the matrix units and memory are about equally long; fewer heads are bound by memory, chunks of rows by the matrix units.
//
// A workgroup holds 128, 64 or 32 columns - (query row, head) pairs of one session, rows that follow each other - and walks 32-token tiles of its rows:
//     S^T (32 tokens x 32 columns) = rows . Q^T     O^T (L channels x 32 columns) += rows^T . P^T         on 32x32x16 bf16 MFMA
// Q^T stays in registers, O^T in fp32 accumulators: of 512 channels and 128 columns together 80 % of a CU's registers, so that one workgroup of four waves is
// all a CU holds and latency is hidden by order alone: the tile after the next is on its way, and the softmax of a tile runs beside the value product of the one
// before.  With 64 or 32 columns, waves share columns and divide the channels of O; each takes the scores again, which memory's pace leaves time for.  The matrix units
// run at the chip's power limit: on random numbers a loop of nothing but these products reaches 1630 TFLOP/s.
//
// One tile in LDS feeds both products: scores read it along a row (16 bytes a lane), values across rows, by transposing reads.  Tiles come in by direct
// global-to-LDS loads.
//
// Work is dealt in equal shares of key tiles, one a workgroup and CU: units (session, column tile) lie end to end, a share cuts them where it ends, and the
// pieces' partial (max, sum, O) go through the workspace and are merged in order by a second launch.
//
// Measured, L + R = 512 + 64, from card to card.  Eight chunks of 32 to 256 rows onto 2048 to 8192 tokens, 128 heads: 1440 to 1490 us, 1.25 to 1.29 PFLOP/s, 78 % of the
// products' own rate.  A decode step of 64 sessions of 1024 to 4096 tokens, 128 heads: 80 to 93 us, of which 17 are the merge of 82 MB (its 214 MB alone would take 43 at a
// copy's rate).  Four sessions of 20000 to 32768, 16 heads: 35 to 42 us, 3.0 to 3.6 TB/s.  One of 1000, 32 heads: 13 us, all of it latency.  128 + 64 channels, with
// the rules below as they were measured at 512 + 64: 560, 33, 20 and 9.8 us (at a product's or a copy's rate 401, 14, 8.5 and a launch).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "latent_internal.h"
#include "lds_dma.h"

namespace ag {
namespace latent {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTokens = 32;             // of a tile
constexpr int kStages = 4;              // tiles in LDS: the one whose values are taken, the one whose scores are, two on their way
constexpr int kMostShares = 256;
constexpr float kLog2e = 1.4426950408889634f;
// What a column's reference m may be exceeded by: a lane's 16 weights of a tile sum to at most this.  Weights are floating-point numbers, as exact at 2^40 as at 1.
// O is then below 2^41 x a context's tiles (2^26) x a channel: fp32 holds it for channels up to 2^60, which is the range that the header gives.
constexpr float kMostWeight = 1099511627776.0f;
constexpr float kLeastSum = 1.0f / kMostWeight;

// ---- how a batch is cut ----

// Columns of a tile: whole query rows' heads while they fit (m rows of `heads` columns), otherwise parts of one row's heads (nh tiles a row).
struct Cut {
    int cols, heads, m, nh;
    int lead;                   // what a unit costs beside its tiles, in tiles: its queries, its first tile, its output
    int whole;                  // a unit of so many tiles or fewer is not cut
    __host__ __device__ Cut(int cols_, int heads_, int lead_ = 0, int whole_ = 0)
        : cols(cols_), heads(heads_), m(heads_ < cols_ ? cols_ / heads_ : 1), nh((heads_ + cols_ - 1) / cols_), lead(lead_), whole(whole_) {}
};

// Work is counted in tiles of 32 keys for decode.  A chunk's column tile k counts the keys that its last row sees, P + min((k + 1) m, N), so that the
// sum over the tiles of a session has a closed form; shares are multiples of 32 of that.  A unit costs `lead` tiles on top.
template <bool kDecode> struct Counting { typedef uint32_t Cost; static constexpr int kTile = 1; };
template <> struct Counting<false> { typedef uint64_t Cost; static constexpr int kTile = kTokens; };

struct Lens { int prefix, n, row0; };   // of a session
template <bool kDecode>
__device__ __forceinline__ Lens lens_of(const AttnArgs& a, int s)
{
    if constexpr (kDecode) {
        const int ctx = a.ctx_lens[s];
        return Lens{ctx - 1, ctx > 0 ? 1 : 0, s};
    } else {
        return Lens{a.prefix_lens[s], max(a.new_lens[s], 0), a.cu_new[s]};
    }
}
// of column tiles 0 .. k - 1 of a session (all full), without the factor nh
__device__ __forceinline__ uint64_t cost_below(const Lens& x, const Cut& cut, uint64_t k)
{
    return k * ((uint64_t)x.prefix + (uint64_t)cut.lead * kTokens) + (uint64_t)cut.m * (k * (k + 1) / 2);
}
template <bool kDecode>
__device__ __forceinline__ typename Counting<kDecode>::Cost session_cost(const Lens& x, const Cut& cut)
{
    if (x.n <= 0) return 0;
    if constexpr (kDecode) return (uint32_t)cut.nh * (uint32_t)((x.prefix + kTokens) / kTokens + cut.lead);
    const uint64_t k = (x.n - 1) / cut.m;                              // tiles before the last
    return (uint64_t)cut.nh * (cost_below(x, cut, k) + x.prefix + x.n + (uint64_t)cut.lead * kTokens);
}

template <typename T>
__device__ __forceinline__ T scan64(T v)                               // inclusive, over the wave
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T up = __shfl_up(v, d);
        v += lane >= d ? up : 0;
    }
    return v;
}
__device__ __forceinline__ uint32_t from_lane(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int l) { return from_lane((uint32_t)v, l) | (uint64_t)from_lane((uint32_t)(v >> 32), l) << 32; }

// A unit: column tile k of session s, part hh of its heads.
struct Unit { int s, k, hh; Lens x; };

// Share w of `shares`: [begin, begin + len) of the batch's work, and the unit that begin lies in, `off` into it.  len 0: nothing.
template <bool kDecode>
struct Share {
    typedef typename Counting<kDecode>::Cost Cost;
    Cost begin, len, off, per, total;
    Unit u;
    __device__ __forceinline__ Share(const AttnArgs& a, const Cut& cut, int w, int shares, int least)
    {
        const int lane = threadIdx.x & 63;
        Cost incl = 0, units = 0;
        total = 0;
        for (int base = 0; base < a.batch; base += 64) {
            const Lens x = base + lane < a.batch ? lens_of<kDecode>(a, base + lane) : Lens{0, 0, 0};
            incl = scan64(session_cost<kDecode>(x, cut));
            total += from_lane(incl, 63);
            if constexpr (kDecode) units += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x.n > 0));
            else units += from_lane(scan64((uint32_t)((x.n + cut.m - 1) / cut.m)), 63);
        }
        // not less than `least` tiles, but for units that are smaller themselves (four prompts of 200 to 300 rows, 32 heads: 27.5 us, as long as only sessions were counted 38)
        constexpr Cost kT = Counting<kDecode>::kTile;
        units *= cut.nh;
        Cost floor = total / (units > 0 ? units : 1);
        floor = floor < (Cost)least * kT ? floor : (Cost)least * kT;
        per = (total + shares - 1) / shares;
        per = ((per < floor ? floor : per) + kT - 1) / kT * kT;
        per = per > 0 ? per : kT;
        begin = (Cost)w * per;
        len = begin < total ? (total - begin < per ? total - begin : per) : 0;
        off = 0;
        u = Unit{0, 0, 0, Lens{0, 0, 0}};
        if (len == 0) return;
        Cost run = 0;
        for (int base = 0;; base += 64) {                              // ends: begin < total
            if (a.batch > 64) incl = scan64(base + lane < a.batch ? session_cost<kDecode>(lens_of<kDecode>(a, base + lane), cut) : (Cost)0);
            const uint64_t past = __builtin_amdgcn_ballot_w64(run + incl > begin);
            if (past) {
                const int l = __builtin_ctzll(past);
                u.s = base + l;
                run += l ? from_lane(incl, l - 1) : 0;
                break;
            }
            run += from_lane(incl, 63);
        }
        u.x = lens_of<kDecode>(a, u.s);
        Cost y = begin - run;
        if constexpr (!kDecode) {
            int lo = 0, hi = (u.x.n - 1) / cut.m;                      // the last tile that starts at or before y
            while (lo < hi) {
                const int mid = lo + (hi - lo + 1) / 2;
                if ((uint64_t)cut.nh * cost_below(u.x, cut, mid) <= y) lo = mid;
                else hi = mid - 1;
            }
            u.k = lo;
            y -= (uint64_t)cut.nh * cost_below(u.x, cut, lo);
        }
        const Cost c = cost(cut);
        u.hh = (int)(y / c);
        off = y - (Cost)u.hh * c;
    }
    __device__ __forceinline__ int last_pos(const Cut& cut) const { return u.x.prefix + min((u.k + 1) * cut.m, u.x.n) - 1; }      // that the unit's last row sees
    __device__ __forceinline__ int tiles(const Cut& cut) const { return last_pos(cut) / kTokens + 1; }
    __device__ __forceinline__ Cost cost(const Cut& cut) const { return (kDecode ? (Cost)tiles(cut) : (Cost)last_pos(cut) + 1) + (Cost)cut.lead * Counting<kDecode>::kTile; }
    // tiles of the unit that lie before a cut at `y`
    __device__ __forceinline__ int tiles_before(const Cut& cut, Cost y) const
    {
        if (whole(cut)) return 2 * y > cost(cut) ? tiles(cut) : 0;
        return max((int)(y / Counting<kDecode>::kTile) - cut.lead, 0);
    }
    // A unit of a few tiles goes to the share that has more of it: its pieces would cost more than they save
    __device__ __forceinline__ bool whole(const Cut& cut) const { return tiles(cut) <= cut.whole; }
    // the unit after u, from its start
    __device__ __forceinline__ bool next(const AttnArgs& a, const Cut& cut)
    {
        off = 0;
        if (++u.hh < cut.nh) return true;
        u.hh = 0;
        if (++u.k * cut.m < u.x.n) return true;
        u.k = 0;
        do {
            if (++u.s >= a.batch) return false;
            u.x = lens_of<kDecode>(a, u.s);
        } while (u.x.n <= 0);
        return true;
    }
};

// ---- the workspace ----
// Records of the cuts: for share w's start, if it is the first that cuts its unit, the unit's first output row, its columns, and how many pieces it is in
// (otherwise 0).  Pieces: two places a share, 2 w for a unit that began in an earlier one, 2 w + 1 for the one that it leaves unfinished.
struct Record { int64_t row; int32_t cols, pieces; };
__host__ __device__ inline size_t ml_offset() { return kMostShares * sizeof(Record); }
__host__ __device__ inline size_t o_offset(int places, int cols) { return ml_offset() + (size_t)places * cols * 8; }
// O of a place: [32 columns][channel / 32][channel / 8 % 4][channel / 4 % 2][column][channel % 4]: a store writes 1 KiB in a run
__host__ __device__ inline size_t place_floats(int cols, int lat) { return (size_t)cols * lat; }

// ---- the kernel ----

template <int L, int R> struct Row {
    static constexpr int kRow = row_of(L, R), kBytes = kRow * 2, kBlocks = kRow / 64, kSteps = (L + R) / 16, kTile = kTokens * kBytes;
};
// Where a tile's 16-byte pieces stand in LDS: [token / 8][channel / 64][token % 8][8 pieces], piece c of token n at place c ^ turn(n): the tokens of a score operand
// and the four rows of a transposing read then lie in different banks.
__device__ __forceinline__ int turn_of(int n) { return (((n & 3) ^ ((n >> 3) & 1)) << 1) | ((n >> 2) & 1); }

__device__ __forceinline__ bf16x4 read_across(unsigned lds_addr)
{
    typedef __attribute__((address_space(3))) bf16x4* ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ptr)(uintptr_t)lds_addr);
}
__device__ __forceinline__ bf16x8 read_along(unsigned lds_addr)
{
    typedef const __attribute__((address_space(3))) bf16x8* ptr;
    return *(ptr)(uintptr_t)lds_addr;
}
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int kAhead = 4;               // operand reads run this many products ahead of their use (two measure alike)

// The products are written in assembly because the scores' accumulators have to be vector registers and O's accumulation registers: the compiler gives all matrix
// instructions of a kernel the same kind, and O^T fills that.  What the compiler keeps for its own matrix instructions is kept here by hand: two states between a vector
// instruction that may have moved an operand or an accumulator and the product; none between products into one accumulator; and nothing of a result is read before
// products_end(), 20 states after the last product (its 16 passes and four).  Operands come by the compiler's loads, whose arrival it waits for.
// tests/test_latent_asm.py and tests/test_latent_paths.py look for all of that in the code.
__device__ __forceinline__ void score_product_first(f32x16& s, const bf16x8& a, const bf16x8& b)
{
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void score_product(f32x16& s, const bf16x8& a, const bf16x8& b)
{
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void value_product(f32x16& o, const bf16x8& a, const bf16x8& b)
{
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(a), "v"(b));
}
// ... where the compiler may just have moved the accumulator, as it does behind the loop
__device__ __forceinline__ void value_product_moved(f32x16& o, const bf16x8& a, const bf16x8& b)
{
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(a), "v"(b));
}
__device__ __forceinline__ void products_end() { asm volatile("s_nop 15\n\ts_nop 3"); }
__device__ __forceinline__ void products_end(f32x16& s) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s)); }

struct Weights { bf16x8 k[2]; };        // of a tile, as the B operands of the two k-steps of the value product

__device__ __forceinline__ float add_pair(bf16x2 p, float sum)
{
    return __builtin_amdgcn_fdot2_f32_bf16(p, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, sum, false);
}

// Weights of a tile under m, and their sum as rounded.
__device__ __forceinline__ float weigh(const f32x16& s, float sl2, float m, Weights& p)
{
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bf16x2 w = {(__bf16)__builtin_amdgcn_exp2f(fmaf(s[2 * i], sl2, -m)), (__bf16)__builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], sl2, -m))};
        p.k[i >> 2][(2 * i) & 7] = w[0];
        p.k[i >> 2][(2 * i + 1) & 7] = w[1];
        sum = add_pair(w, sum);
    }
    return sum;
}

// The value product's operand i: k-step i / kCb, channel block i % kCb.  vb: the lane's places for slots 0..7 / 8..15 of a k-step (turn_of() differs by 2) and
// even / odd blocks (four pieces on).
template <int L, int R, int kCb>
__device__ __forceinline__ bf16x8 value_operand(const unsigned (&vb)[2][2], int i)
{
    const int kk = i / kCb, cb = i % kCb;
    const bf16x4 lo = read_across(vb[0][cb & 1] + (2 * kk) * (8 * Row<L, R>::kBytes) + (cb >> 1) * 1024);
    const bf16x4 hi = read_across(vb[1][cb & 1] + (2 * kk + 1) * (8 * Row<L, R>::kBytes) + (cb >> 1) * 1024);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A block of O is in accumulation registers here: the compiler would otherwise take all of it into vector registers at once, where it does not fit.
__device__ __forceinline__ void stays_put(f32x16& o) { asm volatile("" : "+a"(o)); }

// One iteration: the scores of tile t (kScores), then O += rows(t-1)^T . P(t-1) (kValues) beside the weights of tile t under m, which go to p_cur, and their sum to `sum`.
// The operands of both products are one stream, read kAhead products ahead.  between(j) runs behind score product j, mask(s) once the scores are there; without values
// the scores are all that comes of it.
template <int L, int R, int kCb, bool kScores, bool kValues, class Between, class Mask>
__device__ __forceinline__ void step(unsigned k0, unsigned v0, const bf16x8 (&qf)[Row<L, R>::kSteps], float sl2, float m, float& sum, f32x16& s, const Weights& p_prev,
                                     Weights& p_cur, f32x16 (&o)[kCb], Between between, Mask mask)
{
    constexpr int kNs = kScores ? Row<L, R>::kSteps : 0, kNv = kValues ? 2 * kCb : 0, kN = kNs + kNv;
    const unsigned kb[4] = {k0, k0 ^ 32, k0 ^ 64, k0 ^ 96}, vb[2][2] = {{v0, v0 ^ 64}, {v0 ^ 32, v0 ^ 96}};
    bf16x8 opnd[kAhead + 1];
    auto operand = [&](int j) { return j < kNs ? read_along(kb[j & 3] + (j >> 2) * 1024) : value_operand<L, R, kCb>(vb, j - kNs); };
#pragma unroll
    for (int j = 0; j < kAhead && j < kN; ++j) {
        opnd[j] = operand(j);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = 0; j < kNs; ++j) {
        if (j + kAhead < kN) opnd[(j + kAhead) % (kAhead + 1)] = operand(j + kAhead);
        if (j == 0) score_product_first(s, opnd[0], qf[0]);
        else score_product(s, opnd[j % (kAhead + 1)], qf[j]);
        between(j);
        __builtin_amdgcn_sched_barrier(0);
    }
    // The scores' wait: behind the first three value products where there are enough of them, seven states each
    constexpr int kWait = kScores && kNv >= 16 ? 3 : 0;
    if constexpr (kScores && kWait == 0) {
        products_end(s);
        mask(s);
    }
    if constexpr (kValues) {
        // a pair of scores goes through four links (scale, exp, round, sum), one a step, so that nothing in a step waits for anything else in it
        constexpr int kLinks = 8 + 2;
        float x0 = 0.f, x1 = 0.f, q0 = 0.f, q1 = 0.f;
        bf16x2 w = {(__bf16)0.f, (__bf16)0.f};
        sum = 0.f;
        auto scale = [&](int pair) {
            x0 = fmaf(s[2 * pair], sl2, -m);
            x1 = fmaf(s[2 * pair + 1], sl2, -m);
        };
        auto link = [&](int i) {
            if (i >= 2) sum = add_pair(w, sum);
            if (i >= 1 && i <= 8) {
                w = bf16x2{(__bf16)q0, (__bf16)q1};
                p_cur.k[(i - 1) >> 2][(2 * (i - 1)) & 7] = w[0];
                p_cur.k[(i - 1) >> 2][(2 * (i - 1) + 1) & 7] = w[1];
            }
            if (i < 8) {
                q0 = __builtin_amdgcn_exp2f(x0);
                q1 = __builtin_amdgcn_exp2f(x1);
            }
            if (i + 1 < 8) scale(i + 1);
        };
        if constexpr (kScores && kWait == 0) scale(0);
#pragma unroll
        for (int j = 0; j < kNv; ++j) {
            if (kNs + j + kAhead < kN) opnd[(kNs + j + kAhead) % (kAhead + 1)] = operand(kNs + j + kAhead);
            if (!kScores && j < kCb) value_product_moved(o[j], opnd[j % (kAhead + 1)], p_prev.k[0]);
            else value_product(o[j % kCb], opnd[(kNs + j) % (kAhead + 1)], p_prev.k[j / kCb]);
            if constexpr (kScores) {
                if (j < kWait) asm volatile("s_nop 6");
                if (j + 1 == kWait) {
                    asm volatile("" : "+v"(s));      // 21 states and two products after the last score product: the scores are there
                    mask(s);
                    scale(0);
                }
                if (j >= kWait) {
#pragma unroll
                    for (int i = 0; i < kLinks; ++i)
                        if (kWait + i * (kNv - kWait) / kLinks == j) link(i);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

template <int L, int R, int kSplit, bool kDecode>
__global__ __launch_bounds__(256, 1) void latent_kernel(AttnArgs a, int least, int lead, int uncut)
{
    typedef Row<L, R> Rw;
    constexpr int kCols = 128 / kSplit, kCb = L / 32 / kSplit, kRB = Rw::kBytes;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    int* const s_bad = reinterpret_cast<int*>(lds + kStages * Rw::kTile);         // rows that are not finite; a piece to be done again
    int* const s_again = s_bad + 1;
    const unsigned lds0 = lds_address(lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ct = wave / kSplit, part = wave % kSplit, n = lane & 31, hi = lane >> 5;
    const Cut cut(kCols, a.heads, lead, uncut);
    const int shares = gridDim.x;
    // shares that follow each other on one XCD: they read the same rows
    const int w = shares % 8 == 0 ? (blockIdx.x % 8) * (shares / 8) + blockIdx.x / 8 : blockIdx.x;
    Share<kDecode> sh(a, cut, w, shares, least);
    typedef typename Share<kDecode>::Cost Cost;
    constexpr Cost kT = Counting<kDecode>::kTile;

    if (tid == 0) {
        Record rec = {0, 0, 0};
        if (sh.len && sh.off && !sh.whole(cut) && sh.tiles_before(cut, sh.off) > 0) {
            const Cost u0 = sh.begin - sh.off, first = (u0 + (cut.lead + 1) * kT + sh.per - 1) / sh.per;       // the first share whose start cuts the unit
            if (first == (Cost)w) {
                rec.row = ((int64_t)sh.u.x.row0 + (int64_t)sh.u.k * cut.m) * a.heads + (int64_t)sh.u.hh * kCols;
                rec.cols = a.heads <= kCols ? min(cut.m, sh.u.x.n - sh.u.k * cut.m) * a.heads : min(kCols, a.heads - sh.u.hh * kCols);
                rec.pieces = (int)((u0 + sh.cost(cut) - 1) / sh.per) - w + 2;
            }
        }
        reinterpret_cast<Record*>(a.ws)[w] = rec;
        *s_bad = *s_again = 0;
    }

    // ---- the lane's places ----
    // loads: token lane / 8 of the wave's eight, piece lane % 8 of its place
    const uint32_t piece = (uint32_t)((lane & 7) ^ turn_of(wave * 8 + (lane >> 3))) * 16;
    // scores: token n of the tile, piece hi of a run of eight; piece 2 j + hi is 32 j further, by exclusive or (runs are 128 bytes, aligned)
    const unsigned k_lane = lds0 + (n >> 3) * (8 * kRB) + (n & 7) * 128 + (hi ^ turn_of(n)) * 16;
    // values: sixteen lanes read four tokens (row i / 4, four channels i % 4); tokens 16 kk + 4 hi + row, channels of the part's first block
    unsigned v_lane;
    {
        const int i = lane & 15, row = 4 * hi + (i >> 2), chunk = part * kCb * 4 + ((lane >> 4) & 1) * 2 + ((i >> 1) & 1);
        v_lane = lds0 + row * 128 + (chunk >> 3) * 1024 + ((chunk & 7) ^ turn_of(row)) * 16 + (i & 1) * 8;
    }

    const float sl2 = a.scale * kLog2e;
    const int ps = a.c.ps, shift = a.c.ps_shift;
    Cost left = sh.len;
    int done = 0;                        // tiles of this share so far
    while (left) {
        const int tiles = sh.tiles(cut);
        const Cost rest = sh.cost(cut) - sh.off;
        // the piece of the unit, counted from its far end: a share starts with the first keys of a unit, like the whole units that others take at that time
        const int from = sh.tiles_before(cut, sh.off), to = left >= rest ? tiles : sh.tiles_before(cut, sh.off + left), begin = tiles - to, end = tiles - from;
        if (begin < end) {
            // ---- the unit's columns ----
            const Unit& u = sh.u;
            const int first_row = u.k * cut.m, last = sh.last_pos(cut), qmin = u.x.prefix + first_row;
            const int cols = a.heads <= kCols ? min(cut.m, u.x.n - first_row) * a.heads : min(kCols, a.heads - u.hh * kCols);
            const int64_t base_row = ((int64_t)u.x.row0 + first_row) * a.heads + (int64_t)u.hh * kCols;
            const int col = min(ct * 32 + n, cols - 1);                   // columns beyond the tile repeat the last one
            const int qpos = a.heads <= kCols ? qmin + col / a.heads : qmin;

            // ---- pages: the ids of 64 at a time, a lane each ----
            const int32_t* const bt = a.bt + (int64_t)u.s * a.max_pages;
            int window = -1, ids = 0;
            auto page_of = [&](int pos) {
                const int p = pos >> shift;
                if (p >> 6 != window) {
                    window = p >> 6;
                    ids = bt[min(window * 64 + lane, last >> shift)];
                    AG_WAIT_VMCNT(0);            // here and not at the use, which would wait for the tiles on their way every time
                }
                return __builtin_amdgcn_readlane(ids, p & 63);
            };
            // The order of the tiles: a whole unit starts where `done` says and wraps round, so that workgroups that have done as much read the same keys at
            // the same time, and find them in their XCD's cache (chunks, eight at 128 heads 1489 us, from the start each 1531; a decode's keys have one reader)
            const int count = end - begin, start = begin + (kDecode || from != 0 || to != tiles || done % count * kTokens > qmin ? 0 : done % count);
            const int shown = (qmin + 1) / kTokens;      // tiles from here on have keys that some column does not see
            const bool split = !kDecode && cut.m > 1;    // ... and others do

            // The tiles in hand: values are taken of `before`, scores of `now`; `last_asked` is the latest requested, and left_to_ask are still to be.  Their stages go round
            // with them.  (Past the end of the order the last tile is read again, into stages that nothing reads: the loop has one shape.)
            int before = 0, now = 0, after = 0, last_asked = 0, left_to_ask = 0;
            unsigned st_before = 0, st_now = 0, st_after = 0, st_next = 0;
            // A request in six short parts, which go behind products one by one: address arithmetic is scalar and has no other wave to hide behind.  A run of the wave's eight
            // tokens an instruction follows; positions past the last one repeat that.
            struct { int at, room; int64_t row; const unsigned char* src; uint32_t off; } ask;
            auto plan = [&](int part) {
                if (part == 0) {
                    if (left_to_ask > 0) last_asked = last_asked + 1 == end ? begin : last_asked + 1;
                    --left_to_ask;
                } else if (part == 1) {
                    const int r0 = last_asked * kTokens + wave * 8;
                    ask.room = last - r0;
                    ask.at = min(r0, last);
                } else if (part == 2) {
                    ask.row = page_of(ask.at);
                } else if (part == 3) {
                    ask.row = ask.row * ps + (ask.at & (ps - 1));
                } else if (part == 4) {
                    ask.src = (const unsigned char*)a.c.pool + ask.row * kRB;
                } else {
                    ask.off = (uint32_t)min(lane >> 3, max(ask.room, 0)) * kRB + piece;
                }
            };
            constexpr int kParts = 6;
            auto request = [&](int b) { load_to_lds_from(ask.src + b * 128, ask.off, lds0 + st_next + wave * (8 * kRB) + b * 1024); };
            auto go_round = [&] {
                before = now;
                now = after;
                after = last_asked;
                const unsigned x = st_before;
                st_before = st_now;
                st_now = st_after;
                st_after = st_next;
                st_next = x;
            };
            auto request_all = [&] {
#pragma unroll
                for (int part = 0; part < kParts; ++part) plan(part);
#pragma unroll
                for (int b = 0; b < Rw::kBlocks; ++b) request(b);
                go_round();
            };
            auto request_first = [&] {
                AG_WAIT_VMCNT(0);
                barrier();                       // the last tiles have been read, and no request is on the way
                st_before = 0, st_now = Rw::kTile, st_after = 2 * Rw::kTile, st_next = 3 * Rw::kTile;
                left_to_ask = count;
                last_asked = start == begin ? end - 1 : start - 1;       // (the first plan() steps to `start`)
                request_all();
                request_all();
            };

            // ---- the queries, as B operands: column n, channels i * 16 + hi * 8 .. + 7 ----
            bf16x8 qf[Rw::kSteps];
            request_first();
            const __bf16* const q0 = (const __bf16*)a.q + base_row * (L + R);
            if constexpr (kSplit == 1) {
                const __bf16* qp = q0 + (int64_t)col * (L + R) + hi * 8;
#pragma unroll
                for (int i = 0; i < Rw::kSteps; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(qp + i * 16);
                AG_WAIT_VMCNT(0);
            } else {
                // By way of the stages that the first tiles do not take: waves that share columns read them once, in whole lines (16 bytes a lane out of 32 rows are 64
                // requests an instruction).  Where a row ends inside a run of 128 bytes, lanes past its end repeat its last half.
                static_assert(kSplit == 4 || kSplit == 2, "a stage for 32 columns, and two are free");
#pragma unroll
                for (int t = 0; t < 4 / kSplit; ++t) {
                    const unsigned dst = lds0 + (t + 1) * Rw::kTile + wave * (8 * kRB);
                    const int row = min(t * 32 + wave * 8 + (lane >> 3), cols - 1);
#pragma unroll
                    for (int b = 0; b < Rw::kBlocks; ++b) {
                        const uint32_t in = (b + 1) * 64 <= L + R ? piece : piece & 63;
                        load_to_lds_from(reinterpret_cast<const unsigned char*>(q0) + b * 128, (uint32_t)row * ((L + R) * 2) + in, dst + b * 1024);
                    }
                }
                AG_WAIT_VMCNT(0);
                barrier();
                const unsigned k0 = k_lane + (ct + 1) * Rw::kTile, kb[4] = {k0, k0 ^ 32, k0 ^ 64, k0 ^ 96};
#pragma unroll
                for (int i = 0; i < Rw::kSteps; ++i) qf[i] = read_along(kb[i & 3] + (i >> 2) * 1024);
                __builtin_amdgcn_s_waitcnt(0xC07F);         // lgkmcnt(0): they are read before the next barrier lets a request into their stages
            }

            // m is a reference that every weight of the column is taken under, the largest score of its first tile: weights may come out far above one, and only if they
            // leave what kMostWeight allows for (or nothing came out at all) the piece is done again, under the largest score of all its tiles.  O never has to be rescaled.
            // (Two passes more: scores that rise by 30 nats in a context's last quarter, 64 sessions' decode 81 -> 131 us, eight chunks 1442 -> 3520; by 20 nats no slower.)
            float m = -INFINITY, lsum;
            f32x16 o[kCb];
            bool wrong = false;                  // this column's weights
            Weights pa, pb;
            auto largest = [](const f32x16& s) {
                float x = s[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) x = fmaxf(x, s[e]);
                return x;
            };
            // Scores of the tile `now`, values of the one before
            auto iter = [&](auto scores, auto values, float& sum, f32x16& s) {
                AG_WAIT_VMCNT(Rw::kBlocks);
                barrier();                       // `now` is there, and every wave has taken the values of the tile two before
                // A weight of zero does not hide a NaN.  Rows that only some of the columns see are looked through, their scores being taken: what is not
                // finite in them becomes zero for the value product, and goes to the columns that see it afterwards.
                constexpr bool kValues = decltype(values)::value;
                bool bad = false;
                if (kValues && split && before >= shown) {
                    const int unseen = max(qmin + 1 - before * kTokens, 0);        // the first token that not all columns see
                    unsigned char* const tile = lds + st_before;
                    bool mine = false;
                    for (int x = tid; x < (kTokens - unseen) * (L / 8); x += 256) {
                        const int tok = unseen + x / (L / 8), c = x % (L / 8);
                        u32x4* const at = reinterpret_cast<u32x4*>(tile + (tok >> 3) * (8 * kRB) + (c >> 3) * 1024 + (tok & 7) * 128 + ((c & 7) ^ turn_of(tok)) * 16);
                        u32x4 v = *at;
                        uint32_t any = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t high = ((v[j] & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u;       // the halves whose exponent is all ones
                            any |= high;
                            v[j] &= ~((high << 1) - (high >> 15));
                        }
                        if (any) {
                            *at = v;
                            mine = true;
                        }
                    }
                    if (mine) *s_bad = 1;
                    __syncthreads();
                    bad = __builtin_amdgcn_readfirstlane(*s_bad) != 0;
                }
                auto between = [&](int j) {
                    if (j < kParts) plan(j);
#pragma unroll
                    for (int b = 0; b < Rw::kBlocks; ++b)
                        if (j == kParts + b * (Rw::kSteps - kParts) / Rw::kBlocks) request(b);
                };
                auto mask = [&](f32x16& s) {
                    if (now < shown) return;
                    const int key = now * kTokens + hi * 4;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = key + (e >> 2) * 8 + (e & 3) <= qpos ? s[e] : -INFINITY;
                };
                const unsigned k0 = k_lane + st_now, v0 = v_lane + st_before;
                step<L, R, kCb, decltype(scores)::value, kValues>(k0, v0, qf, sl2, m, sum, s, pa, pb, o, between, mask);
                if (bad) {
                    products_end();
#pragma unroll 1
                    for (int at = max(before * kTokens, qmin + 1); at <= min(before * kTokens + kTokens - 1, last); ++at) {
                        const int page = bt[at >> shift];
                        const uint16_t* const row = (const uint16_t*)a.c.pool + ((int64_t)page * ps + (at & (ps - 1))) * Rw::kRow + part * (kCb * 32) + hi * 4;
#pragma unroll
                        for (int cb = 0; cb < kCb; ++cb) {
                            stays_put(o[cb]);
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const bool odd = (row[cb * 32 + (e >> 2) * 8 + (e & 3)] & 0x7F80) == 0x7F80;
                                o[cb][e] = odd && at <= qpos ? __builtin_nanf("") : o[cb][e];
                            }
                            stays_put(o[cb]);
                        }
                    }
                    __syncthreads();
                    if (tid == 0) *s_bad = 0;
                    __syncthreads();
                }
                go_round();
            };
            constexpr std::true_type yes{};
            constexpr std::false_type no{};
            for (int attempt = 0;; ++attempt) {
                f32x16 s;
                float sum;
                if (attempt > 0) {                   // the largest scores first
                    request_first();
                    float most = -INFINITY;
#pragma unroll 1
                    for (int i = 0; i < count; ++i) {
                        iter(yes, no, sum, s);
                        most = fmaxf(most, largest(s));
                    }
                    most = fmaxf(most, __shfl_xor(most, 32)) * sl2;               // (scale > 0: maximum and scaling commute)
                    if (wrong) m = most == -INFINITY ? 0.f : most;
                    request_first();
                }
                iter(yes, no, sum, s);
                if (attempt == 0) {
                    m = largest(s);
                    m = fmaxf(m, __shfl_xor(m, 32)) * sl2;                         // the two lanes of a column share it
                    if (m == -INFINITY) m = 0.f;                                   // (no key seen yet: weights of zero)
                }
                lsum = weigh(s, sl2, m, pa);
                wrong = !(lsum <= kMostWeight);
#pragma unroll
                for (int cb = 0; cb < kCb; ++cb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
#pragma unroll 1
                for (int i = 1; i < count; ++i) {
                    iter(yes, yes, sum, s);
                    pa = pb;
                    lsum += sum;
                    wrong |= !(sum <= kMostWeight);
                }
                iter(no, yes, sum, s);
                AG_WAIT_VMCNT(0);                // the requests past the end write to LDS too: before rows of O do, and before the workgroup's LDS is another's
                done += count;
                products_end();
                lsum += __shfl_xor(lsum, 32);
                // (a column that sees no key of the piece has a sum of zero, and that is right)
                wrong |= lsum < kLeastSum && begin * kTokens <= qpos;
                wrong |= __shfl_xor((int)wrong, 32) != 0;
                if (attempt > 0) break;
                if (__builtin_amdgcn_ballot_w64(wrong) != 0 && lane == 0) *s_again = 1;
                __syncthreads();
                if (__builtin_amdgcn_readfirstlane(*s_again) == 0) break;
                __syncthreads();
                if (tid == 0) *s_again = 0;
            }
            if (lsum == 0.f) m = -INFINITY;

            if (from == 0 && to == tiles) {
                // by way of LDS, 16-byte pieces in a place that depends on the row, so that whole rows are stored (8-byte stores of the accumulators themselves, 32 rows an
                // instruction: four prompts of 500 to 700 rows at 128 heads 1201 -> 947 us)
                constexpr int kPieces = kCb * 4, kMask = kPieces < 8 ? kPieces - 1 : 7;      // of a row
                barrier();                       // the last tiles' values have been taken
                const float inv = 1.0f / lsum;
                unsigned char* const mine = lds + wave * (32 * kPieces * 16);
#pragma unroll
                for (int cb = 0; cb < kCb; ++cb) {
                    stays_put(o[cb]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16x4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (__bf16)(o[cb][q * 4 + i] * inv);
                        *reinterpret_cast<bf16x4*>(mine + (n * kPieces + ((cb * 4 + q) ^ (n & kMask))) * 16 + hi * 8) = v;
                    }
                }
                u32x4* const op = reinterpret_cast<u32x4*>((__bf16*)a.out + (base_row + ct * 32) * L + part * (kCb * 32));
#pragma unroll
                for (int i = 0; i < kPieces / 2; ++i) {
                    const int at = i * 64 + lane, row = at / kPieces, c = at % kPieces;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + (row * kPieces + (c ^ (row & kMask))) * 16);
                    if (ct * 32 + row < cols) __builtin_nontemporal_store(v, op + (int64_t)row * (L / 8) + c);
                }
            } else {
                const int place = 2 * w + (from == 0);
                unsigned char* const ws = (unsigned char*)a.ws;
                if (part == 0 && hi == 0)
                    reinterpret_cast<float2*>(ws + ml_offset())[(int64_t)place * kCols + ct * 32 + n] = make_float2(m, lsum);
                f32x4* const op = reinterpret_cast<f32x4*>(ws + o_offset(2 * shares, kCols)) + ((int64_t)place * kCols * L + ct * (32 * L)) / 4 + (part * kCb) * 256 + lane;
#pragma unroll
                for (int cb = 0; cb < kCb; ++cb) {
                    stays_put(o[cb]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f32x4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = o[cb][q * 4 + i];
                        op[(cb * 4 + q) * 64] = v;
                    }
                }
            }
        }
        if (left <= rest) break;
        left -= rest;
        if (!sh.next(a, cut)) break;
    }
    if constexpr (kDecode) {
        // sessions without a token: rows of zeros
        for (int s = blockIdx.x; s < a.batch; s += gridDim.x) {
            if (a.ctx_lens[s] > 0) continue;
            u32x4* const op = reinterpret_cast<u32x4*>((__bf16*)a.out + (int64_t)s * a.heads * L);
            for (int64_t i = tid; i < (int64_t)a.heads * (L / 8); i += 256) op[i] = u32x4{0, 0, 0, 0};
        }
    }
}

// Pieces of the units that shares cut, in order.  A workgroup finds those units among the records and takes slices of them, eight columns by 32 kQ channels: a lane has
// kQ times four channels of a column, a wave every fourth piece.  Bound by the caches that hold the pieces: 256 x 128 columns x 512 channels in fp32, 82 MB, take 17 us.
template <int kQ>
__global__ __launch_bounds__(256) void latent_merge_kernel(const unsigned char* ws, __bf16* out, int shares, int cols, int lat)
{
    __shared__ int s_cut[kMostShares];
    __shared__ int s_count[4];
    __shared__ float s_part[3][64][2 + 4 * kQ];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Record* const recs = reinterpret_cast<const Record*>(ws);
    {
        static_assert(kMostShares <= 256, "a thread a record");
        const bool cut = tid >= 1 && tid < shares && recs[tid < shares ? tid : 0].pieces > 0;
        const uint64_t those = __builtin_amdgcn_ballot_w64(cut);
        if (lane == 0) s_count[wave] = __builtin_popcountll(those);
        __syncthreads();
        int at = __builtin_popcountll(those & ((1ull << lane) - 1));
        for (int i = 0; i < wave; ++i) at += s_count[i];
        if (cut) s_cut[at] = tid;
        __syncthreads();
    }
    const int cuts = s_count[0] + s_count[1] + s_count[2] + s_count[3];
    const float2* const ml = reinterpret_cast<const float2*>(ws + ml_offset());
    const f32x4* const o = reinterpret_cast<const f32x4*>(ws + o_offset(2 * shares, cols));
    const int across = lat / (32 * kQ), slices = cols / 8 * across;
    for (int item = blockIdx.x; item < cuts * slices; item += gridDim.x) {
        const int w = s_cut[item / slices], slice = item % slices;
        const Record rec = recs[w];
        const int col = slice / across * 8 + (lane >> 3), quad0 = slice % across * (8 * kQ) + (lane & 7);
        const int64_t o0 = (col >> 5) * (8 * lat) + quad0 * 32 + (col & 31);
        float top = -INFINITY, l = 0.f;
        f32x4 sum[kQ];
#pragma unroll
        for (int q = 0; q < kQ; ++q) sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (col < rec.cols) {
            constexpr int kFlight = 4;           // pieces whose loads are in flight together
            for (int p0 = wave; p0 < rec.pieces; p0 += 4 * kFlight) {
                float2 x[kFlight];
                f32x4 v[kFlight][kQ];
#pragma unroll
                for (int j = 0; j < kFlight; ++j) {
                    const int p = p0 + 4 * j;
                    if (p >= rec.pieces) break;
                    const int64_t place = p == 0 ? 2 * (w - 1) + 1 : 2 * (w + p - 1);
                    x[j] = ml[place * cols + col];
#pragma unroll
                    for (int q = 0; q < kQ; ++q) v[j][q] = o[place * (cols * lat / 4) + o0 + q * 256];
                }
#pragma unroll
                for (int j = 0; j < kFlight; ++j) {
                    if (p0 + 4 * j >= rec.pieces) break;
                    const float t = fmaxf(top, x[j].x), f0 = top == -INFINITY ? 0.f : exp2f(top - t), f1 = x[j].x == -INFINITY ? 0.f : exp2f(x[j].x - t);
                    top = t;
                    l = l * f0 + x[j].y * f1;
#pragma unroll
                    for (int q = 0; q < kQ; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[q][e] = sum[q][e] * f0 + v[j][q][e] * f1;
                }
            }
        }
        __syncthreads();                         // the slice before has been read
        if (wave > 0) {
            float* const x = s_part[wave - 1][lane];
            x[0] = top;
            x[1] = l;
#pragma unroll
            for (int i = 0; i < 4 * kQ; ++i) x[2 + i] = sum[i >> 2][i & 3];
        }
        __syncthreads();
        if (wave > 0 || col >= rec.cols) continue;
        float most = top;
        for (int i = 0; i < 3; ++i) most = fmaxf(most, s_part[i][lane][0]);
        float f = top == -INFINITY ? 0.f : exp2f(top - most);
        l *= f;
#pragma unroll
        for (int i = 0; i < 4 * kQ; ++i) sum[i >> 2][i & 3] *= f;
        for (int j = 0; j < 3; ++j) {
            const float* const x = s_part[j][lane];
            f = x[0] == -INFINITY ? 0.f : exp2f(x[0] - most);
            l += x[1] * f;
#pragma unroll
            for (int i = 0; i < 4 * kQ; ++i) sum[i >> 2][i & 3] += x[2 + i] * f;
        }
        const float inv = 1.0f / l;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (__bf16)(sum[q][e] * inv);
            *reinterpret_cast<bf16x4*>(out + (rec.row + col) * lat + (quad0 + q * 8) * 4) = r;
        }
    }
}

// ---- the host's side ----

// Tiles of a share at least: what a piece writes and a merge reads back, the columns' O in fp32, is worth a few.  Decode, us, 2 / 4 / 8 tiles: one session of 1000 tokens,
// 32 heads 13.3 / 15.1 / 18.9; two of 10500 together, 128 heads 38.2 / 35.1 / 32.0.
constexpr int least_tiles(int cols) { return cols == 32 ? 2 : cols == 64 ? 4 : 8; }
// A unit of so many tiles or fewer is not cut: two shares' least ones (four prompts of 500 to 700 rows, 128 heads: 281 us, with every unit cut 291).
// Contexts of 512 tokens and less stay whole altogether where there are units for an eighth of the CUs, and nothing is merged: decode, us, cut / whole,
//                                                100 to 300 tokens    300 to 512    512
//     16 units (16 sessions, 16 heads)                 14.7 / 15.3     14.4 / 21.7    17.2 / 22.1
//     32 units (32 sessions, 16 heads)                 16.3 / 16.1     17.6 / 22.1    20.8 / 22.4
//     32 units (32 sessions, 32 heads)                 16.8 / 16.3     21.0 / 22.1    23.3 / 22.7
//     32 units ( 8 sessions, 128 heads)                16.0 / 15.6     20.8 / 22.0    22.1 / 22.4
//     48 units (48 sessions, 32 heads)                 19.6 / 16.3     23.6 / 22.5    24.8 / 23.0
//     64 units (16 sessions, 128 heads)                19.7 / 15.6     23.3 / 22.4    24.4 / 22.3
//     128 units (128 sessions, 128 heads)              35.7 / 23.1     40.8 / 40.8    42.2 / 42.2
// and of chunks, whose pieces have more columns: 100 rows behind 300, 128 heads 41.9 / 24.2; 8 sessions' 4 rows behind 200 to 400, 128 heads 29.3 / 20.1.
constexpr int kWholeTiles = 16;
int uncut_tiles(int64_t units, int64_t tiles, int cols, int cus)
{
    return tiles <= kWholeTiles && 8 * units >= cus ? kWholeTiles : 2 * least_tiles(cols);
}
constexpr int kMergeMost = 1024;        // workgroups of a merge

// As few columns as hold a session's: decode of 256 sessions of 1024 tokens, us, in 32 / 64 / 128 columns: 32 heads 66 / 73 / 93; 64 heads - / 77 / 91.
int columns(int64_t most) { return most <= 32 ? 32 : most <= 64 ? 64 : 128; }

// Shares of a launch whose units are at most `units` of `tiles` tiles: one for each at least, as far as there are CUs (256 sessions of 32 tokens, 128 heads: 27 us; by
// `least` alone 131).
int shares_of(int64_t units, int64_t tiles, int cols, int cus)
{
    const int64_t n = std::max<int64_t>(units, (units * tiles + least_tiles(cols) - 1) / least_tiles(cols));
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, cus));
}
// A unit's lead, measured in whole prompts of 500 to 700 rows at 128 heads, where a share has up to fifty: 4, 8, 12 tiles 356, 287, 287 us; where shares are smaller than
// that, less, so that none is left with a lead alone.
// Where no unit is cut and a share need have one at most, a lead beside which their tiles do not count, so that none has two: what units of 1 to 16 tiles
// differ by adds up to 128 x 7.5 tiles at most, and has to stay below half a unit; where units are fewer than shares, a share is shorter than a unit by a 256th
// of one, which has to be more than their tiles (20 rows behind 30 tokens, 32 heads: 10.4 us, by their tiles 14.9; 256 sessions of 2, 4, .. 512 tokens, 128 heads: 50.8, with a lead of
// 1024 tiles 55.5).
constexpr int kMostLead = 8, kOnlyLead = 8192;
int lead_of(int64_t units, int64_t tiles, int shares, int uncut)
{
    if (units <= shares && tiles <= uncut) return kOnlyLead;
    return (int)std::min<int64_t>(kMostLead, units * tiles / shares / 2);
}
int64_t units_of(bool decode, int batch, int total, const Cut& cut)
{
    return (decode ? (int64_t)batch : (int64_t)total / cut.m + batch) * cut.nh;
}
size_t bytes_of(int shares, int cols, int lat) { return o_offset(2 * shares, cols) + (size_t)2 * shares * place_floats(cols, lat) * 4; }

template <int L, int R, int kSplit, bool kDecode>
ag_status run(const AttnArgs& a, int64_t units, int shares, int lead, int uncut, hipStream_t st)
{
    static std::atomic<uint64_t> told{0};
    constexpr int kLds = kStages * Row<L, R>::kTile + 16;
    ag_status e = allow_dynamic_lds((const void*)latent_kernel<L, R, kSplit, kDecode>, kLds, told);
    if (e) return e;
    prof_before(st);
    hipLaunchKernelGGL((latent_kernel<L, R, kSplit, kDecode>), dim3(shares), dim3(256), kLds, st, a, least_tiles(128 / kSplit), lead, uncut);
    if (shares > 1 && (a.max_ctx - 1) / kTokens >= uncut) {
        constexpr int kCols = 128 / kSplit, kSlices = kCols / 8 * (L / 32);
        const int64_t cuts = std::min<int64_t>(shares - 1, units);
        // four channels a lane where the cut units have few columns between them, sixteen otherwise: decode, us, both ways, four sessions of 16 heads 35.8 and 42.2, 64 of
        // 128 heads 100.9 and 91.9
        if (cuts * kSlices <= kMergeMost) hipLaunchKernelGGL(latent_merge_kernel<1>, dim3(cuts * kSlices), dim3(256), 0, st, (const unsigned char*)a.ws, (__bf16*)a.out, shares, kCols, L);
        else hipLaunchKernelGGL(latent_merge_kernel<4>, dim3(std::min<int64_t>(cuts * kSlices / 4, kMergeMost)), dim3(256), 0, st, (const unsigned char*)a.ws, (__bf16*)a.out, shares, kCols, L);
    }
    prof_after(st);
    return hip_check(hipGetLastError(), "latent attention launch");
}
template <int L, int R>
ag_status run_columns(const AttnArgs& a, int cols, int64_t units, int shares, int lead, int uncut, hipStream_t st)
{
    if (a.ctx_lens) {
        if (cols == 32) return run<L, R, 4, true>(a, units, shares, lead, uncut, st);
        return cols == 64 ? run<L, R, 2, true>(a, units, shares, lead, uncut, st) : run<L, R, 1, true>(a, units, shares, lead, uncut, st);
    }
    if (cols == 32) return run<L, R, 4, false>(a, units, shares, lead, uncut, st);
    return cols == 64 ? run<L, R, 2, false>(a, units, shares, lead, uncut, st) : run<L, R, 1, false>(a, units, shares, lead, uncut, st);
}

}  // namespace

size_t attn_workspace(bool decode, int batch, int total, int heads, int lat, int max_ctx)
{
    const int64_t tiles = ((int64_t)max_ctx + kTokens - 1) / kTokens;
    size_t most = 0;
    for (int cols : {32, 64, 128}) {
        if (cols > columns((int64_t)total * heads)) break;             // (no session has more columns than all rows)
        const Cut cut(cols, heads);
        const int64_t units = units_of(decode, batch, total, cut);
        // sums of costs: 32 bits of tiles for decode, 64 of keys otherwise
        if ((double)units * (double)(tiles + kMostLead) >= (decode ? 2147483648.0 : 1.0e16)) return 0;
        most = std::max(most, bytes_of(shares_of(units, tiles, cols, kMostShares), cols, lat));
    }
    return most;
}

ag_status launch_attn(const AttnArgs& a, hipStream_t st)
{
    const bool decode = a.ctx_lens != nullptr;
    const int64_t tiles = ((int64_t)a.max_ctx + kTokens - 1) / kTokens;
    const int cus = std::min(stream_cus(st), kMostShares);
    int cols = columns(decode ? a.heads : (int64_t)a.max_new * a.heads), shares;
    int64_t units;
    // ... and fewer, down to 32, while CUs would go without a share: more units read the same rows, and more waves share a column's work.  Decode at 128 heads, us, in
    // 128 / 64 / 32 columns: two sessions of 5000 tokens 33.4 / 27.9 / 25.1 (45, 178, 256 shares); 256 of 128, a share each, 32.7 / 39.0 / 53.7.
    for (;; cols /= 2) {
        units = units_of(decode, a.batch, a.total, Cut(cols, a.heads));
        shares = shares_of(units, tiles, cols, cus);
        if (cols == 32 || shares >= cus) break;
    }
    const int uncut = uncut_tiles(units, tiles, cols, cus), lead = lead_of(units, tiles, shares, uncut);
    if (a.c.lat == 512) return a.c.rd == 64 ? run_columns<512, 64>(a, cols, units, shares, lead, uncut, st) : run_columns<512, 32>(a, cols, units, shares, lead, uncut, st);
    if (a.c.lat == 256) return a.c.rd == 64 ? run_columns<256, 64>(a, cols, units, shares, lead, uncut, st) : run_columns<256, 32>(a, cols, units, shares, lead, uncut, st);
    return a.c.rd == 64 ? run_columns<128, 64>(a, cols, units, shares, lead, uncut, st) : run_columns<128, 32>(a, cols, units, shares, lead, uncut, st);
}

}  // namespace latent
}  // namespace ag
