// Embedding of tokens and its partial gradients (rows of G).
//   out[t] = scale * E[id_t]             a zero row where id_t is outside [0, vocab)
//   G[p, v] = scale * sum of dout[t] over the tokens t of partition p with id_t = v, ascending in t
//
// The gradient writes all k * vocab rows of the table, most of them zeros, so it is bound by the write of G.  Tokens are
// put in order of (partition, id) by a radix sort that keeps equal keys in place; a row's tokens are then one run of the
// order, found by searching it, and are summed by whoever writes the row: no atomics on values, no clearing before.
// Rows with long runs (few ids, or the commonest one) would leave one wave with all the work: runs are first summed in
// pieces of 64 places of the order and those in groups of 16, so that a row of n tokens takes about n / 1024 + 160 steps.
#include "agc_dispatch.h"
#include "agc_operators.h"

namespace agc {

namespace {

constexpr int kBlock = 256;
constexpr int kMostBits = 11, kMostDigits = 1 << kMostBits;   // of a pass of the sort
constexpr int kSortTile = 1024;    // keys of one workgroup in a pass
constexpr int kFewTiles = 16;      // up to here a workgroup adds up the tiles' counts itself
constexpr int kPiece = 64;         // places of a piece
constexpr int kGroup = 16;         // pieces of a group

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct EmbedParts {
    int end[kMostParts];
    int k;
};

__device__ __forceinline__ float from_bf16(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t to_bf16(float v) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v); }

// Four values of a row of T (float or bfloat16 bits).  WHOLE: elements c .. c+3, one aligned load; else c + e * step, so
// that the lanes of a wave stay side by side, and the last element of the row in place of those behind it.
template <class T, bool WHOLE>
__device__ __forceinline__ f32x4 load4(const T* row, int c, int step, int width)
{
    f32x4 v;
    if constexpr (WHOLE && sizeof(T) == 4) {
        v = *reinterpret_cast<const f32x4*>(row + c);
    } else if constexpr (WHOLE) {
        const u32x2 u = *reinterpret_cast<const u32x2*>(row + c);
        v = f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                  __uint_as_float(u.y & 0xFFFF0000u)};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = min(c + e * step, width - 1);
            if constexpr (sizeof(T) == 4) v[e] = row[at];
            else v[e] = from_bf16(row[at]);
        }
    }
    return v;
}

// Past the caches: nothing that is written here is read here, and what is read stays (131072 x 1024 forward 109 us through
// them, 99 us so).
template <class T, bool WHOLE>
__device__ __forceinline__ void store4(T* row, int c, int step, int width, const f32x4& v)
{
    if constexpr (WHOLE && sizeof(T) == 4) {
        __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(row + c));
    } else if constexpr (WHOLE) {
        __builtin_nontemporal_store(u32x2{to_bf16(v.x) | (to_bf16(v.y) << 16), to_bf16(v.z) | (to_bf16(v.w) << 16)},
                                    reinterpret_cast<u32x2*>(row + c));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e * step < width) {
                if constexpr (sizeof(T) == 4) row[c + e * step] = v[e];
                else row[c + e * step] = (T)to_bf16(v[e]);
            }
    }
}

// ------------------------------------------------------------------ forward
// `lanes` (a power of two up to 64) lanes walk over one row.  Bound by memory: 131072 rows of 1024, binary32 to bfloat16,
// in 99 us, 4.8 TB/s of what has to move, the rate of a copy.
template <class TABLE, class OUT, class ID, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_embed(const TABLE* table, int64_t vocab, int dim, const ID* tokens, int64_t n,
                                                  float scale, OUT* out, int64_t ldo, int lanes)
{
    const int per = kBlock / lanes, mine = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
    for (int64_t t = (int64_t)blockIdx.x * per + mine; t < n; t += (int64_t)gridDim.x * per) {
        const int64_t id = (int64_t)tokens[t];
        const bool held = id >= 0 && id < vocab;
        const TABLE* row = table + (held ? id : 0) * dim;
#pragma unroll 4
        for (int c = WHOLE ? lane * 4 : lane; c < dim; c += lanes * 4) {
            f32x4 v = load4<TABLE, WHOLE>(row, c, lanes, dim);   // of row 0 at an empty place
            v = held ? v * scale : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            store4<OUT, WHOLE>(out + t * ldo, c, lanes, dim, v);
        }
    }
}

// ------------------------------------------------------------------ order of the tokens
// Radix sort, `bits` bits a pass: count the digits of every tile of keys, then move the keys.  Per pass two launches, or
// three above kFewTiles tiles.
struct SortArgs {
    int n, tiles, shift, bits;
    uint32_t* counts;      // [tile][digit]
    uint32_t* totals;      // [digit], above kFewTiles tiles
    const uint32_t *key_in, *place_in;
    uint32_t *key_out, *place_out;
};

// key = partition * vocab + id, or `none` (above all keys) at an empty place
template <class ID>
struct KeySource {
    const ID* tokens;
    int64_t vocab;
    uint32_t none;
    uint32_t* key;
    EmbedParts parts;
    __device__ __forceinline__ uint32_t operator()(int t) const
    {
        int lo = 0, hi = parts.k - 1;   // the first partition that ends after t
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (parts.end[mid] > t) hi = mid;
            else lo = mid + 1;
        }
        const int64_t id = (int64_t)tokens[t];
        const uint32_t k = id >= 0 && id < vocab ? (uint32_t)(lo * vocab + id) : none;
        key[t] = k;
        return k;
    }
};

struct SortedSource {
    const uint32_t* key;
    __device__ __forceinline__ uint32_t operator()(int t) const { return key[t]; }
};

template <class SOURCE>
__global__ __launch_bounds__(kBlock) void k_sort_count(const SortArgs a, const SOURCE source)
{
    __shared__ uint32_t bin[kMostDigits];
    const int digits = 1 << a.bits;
    for (int i = threadIdx.x; i < digits; i += kBlock) bin[i] = 0;
    __syncthreads();
    const int from = blockIdx.x * kSortTile, to = min(a.n, from + kSortTile);
    for (int i = from + threadIdx.x; i < to; i += kBlock) atomicAdd(&bin[(source(i) >> a.shift) & (digits - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += kBlock) a.counts[(int64_t)blockIdx.x * digits + i] = bin[i];
}

// counts[tile][digit] -> that digit's keys in the tiles before; totals[digit]
__global__ __launch_bounds__(64) void k_sort_tiles(const SortArgs a)
{
    const int digits = 1 << a.bits, digit = blockIdx.x * 64 + threadIdx.x;
    if (digit >= digits) return;
    uint32_t sum = 0;
    for (int t = 0; t < a.tiles; t += 16) {
        uint32_t here[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) here[e] = t + e < a.tiles ? a.counts[(int64_t)(t + e) * digits + digit] : 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if (t + e < a.tiles) a.counts[(int64_t)(t + e) * digits + digit] = sum;
            sum += here[e];
        }
    }
    a.totals[digit] = sum;
}

// All passes at once where the keys are one tile: keys and places stay in LDS, one launch in place of two or three a pass
// (57 tokens of 1776 ids in 9 partitions: 21 us for the whole gradient, then 16).
template <class SOURCE>
__global__ __launch_bounds__(kBlock) void k_sort_one_tile(const SortArgs a, int passes, const SOURCE source)
{
    __shared__ uint32_t next[4][kMostDigits];
    __shared__ uint32_t keys[kSortTile], places[kSortTile];
    __shared__ uint32_t carry[4];
    constexpr int kRounds = kSortTile / kBlock;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1 << a.bits;
    const int from = wave * (kSortTile / 4) + lane, per = digits > kBlock ? digits / kBlock : 1;
    uint32_t key[kRounds], place[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = from + r * 64;
        key[r] = i < a.n ? source(i) : 0;
        place[r] = (uint32_t)i;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * a.bits;
        for (int i = tid; i < 4 * digits; i += kBlock) next[i >> a.bits][i & (digits - 1)] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (from + r * 64 < a.n) atomicAdd(&next[wave][(key[r] >> shift) & (digits - 1)], 1u);
        __syncthreads();
        uint32_t sum = 0;
        for (int i = 0; i < per; ++i) {
            const int digit = tid * per + i;
            if (digit < digits) sum += (next[0][digit] + next[1][digit]) + (next[2][digit] + next[3][digit]);
        }
        uint32_t scan = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t add = __shfl_up(scan, d);
            if (lane >= d) scan += add;
        }
        if (lane == 63) carry[wave] = scan;
        __syncthreads();
        uint32_t at = scan - sum;
        for (int w = 0; w < wave; ++w) at += carry[w];
        for (int i = 0; i < per; ++i) {
            const int digit = tid * per + i;
            if (digit >= digits) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t here = next[w][digit];
                next[w][digit] = at;
                at += here;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const bool valid = from + r * 64 < a.n;
            const uint32_t digit = (key[r] >> shift) & (digits - 1);
            uint64_t same = __ballot(valid);   // the wave's lanes with my digit
            for (int b = 0; b < a.bits; ++b) {
                const uint64_t ones = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? ones : ~ones;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (valid) {
                const uint32_t to = next[wave][digit] + rank;
                keys[to] = key[r];
                places[to] = place[r];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (valid && rank == 0) next[wave][digit] += __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = from + r * 64;
            key[r] = i < a.n ? keys[i] : 0;
            place[r] = i < a.n ? places[i] : 0;
        }
        // the next pass clears `next` before its first barrier; nobody reads `keys` after this
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = from + r * 64;
        if (i < a.n) a.key_out[i] = key[r], a.place_out[i] = place[r];
    }
}

// Moves a tile's keys and places to where their digit puts them, equal digits in the order in which they lie.  Each
// wave takes a quarter of the tile, 64 keys at a time.  FIRST: the places are 0, 1, 2, ...
template <bool FIRST>
__global__ __launch_bounds__(kBlock) void k_sort_move(const SortArgs a)
{
    __shared__ uint32_t next[4][kMostDigits];
    __shared__ uint32_t carry[4];
    constexpr int kRounds = kSortTile / kBlock;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1 << a.bits;
    const int from = blockIdx.x * kSortTile + wave * (kSortTile / 4) + lane;
    uint32_t key[kRounds], place[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = from + r * 64;
        key[r] = i < a.n ? a.key_in[i] : 0;
        place[r] = (uint32_t)i;
        if (!FIRST && i < a.n) place[r] = a.place_in[i];
    }
    for (int i = tid; i < 4 * digits; i += kBlock) next[i >> a.bits][i & (digits - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (from + r * 64 < a.n) atomicAdd(&next[wave][(key[r] >> a.shift) & (digits - 1)], 1u);
    // `per` digits a thread: keys of the tiles before, and of all tiles
    constexpr int kMostPer = kMostDigits / kBlock;
    const int per = digits > kBlock ? digits / kBlock : 1;
    uint32_t before[kMostPer], all[kMostPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kMostPer; ++i) {
        before[i] = all[i] = 0;
        const int digit = tid * per + i;
        if (i >= per || digit >= digits) continue;
        if (a.tiles > kFewTiles) {
            before[i] = a.counts[(int64_t)blockIdx.x * digits + digit];
            all[i] = a.totals[digit];
        } else {
#pragma unroll
            for (int t = 0; t < kFewTiles; ++t) {
                const uint32_t c = t < a.tiles ? a.counts[t * digits + digit] : 0;
                all[i] += c;
                if (t < (int)blockIdx.x) before[i] += c;
            }
        }
        sum += all[i];
    }
    // what precedes my digits: the lanes before, then the waves before
    uint32_t scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t add = __shfl_up(scan, d);
        if (lane >= d) scan += add;
    }
    if (lane == 63) carry[wave] = scan;
    __syncthreads();
    uint32_t at = scan - sum;
    for (int w = 0; w < wave; ++w) at += carry[w];
#pragma unroll
    for (int i = 0; i < kMostPer; ++i) {
        const int digit = tid * per + i;
        if (i >= per || digit >= digits) continue;
        uint32_t go = at + before[i];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t here = next[w][digit];
            next[w][digit] = go;
            go += here;
        }
        at += all[i];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const bool valid = from + r * 64 < a.n;
        const uint32_t digit = (key[r] >> a.shift) & (digits - 1);
        uint64_t same = __ballot(valid);   // the wave's lanes with my digit
        for (int b = 0; b < a.bits; ++b) {
            const uint64_t ones = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? ones : ~ones;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (valid) {
            const uint32_t to = next[wave][digit] + rank;
            a.key_out[to] = key[r];
            a.place_out[to] = place[r];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (valid && rank == 0) next[wave][digit] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ------------------------------------------------------------------ sums
struct SumArgs {
    const uint32_t *key, *place;
    int n, dim;
    uint32_t none;
    int64_t ldd;         // of dout
    int64_t pitch;       // of the pieces' sums: dim, rounded up to the 256 columns of a wave
    float* pieces;       // sums of kPiece places of one key, at place / kPiece
    float* groups;       // sums of kGroup pieces of one key
};

// The four columns of a lane in strip `strip` of 256, and where a piece's sum holds them.
template <bool WHOLE>
__device__ __forceinline__ int first_column(int strip, int lane) { return strip * 256 + (WHOLE ? lane * 4 : lane); }
__device__ __forceinline__ int kept_column(int strip, int lane) { return strip * 256 + lane * 4; }

// Adds the tokens at places [from, to) of the order, four columns from c on; uniform over the wave.  64 places are
// fetched at once, a lane each, and DEEP rows are on their way together.
template <class T, bool WHOLE, int DEEP>
__device__ __forceinline__ f32x4 sum_tokens(const SumArgs& a, const T* dout, int from, int to, int c, int lane, f32x4 acc)
{
    const int col = c < a.dim ? c : 0;   // lanes behind the row add up something that nobody stores
    for (; from < to; from += 64) {
        const int count = to - from < 64 ? to - from : 64;
        const uint32_t spot = a.place[from + (lane < count ? lane : 0)];
        for (int i = 0; i < count; i += DEEP) {
            f32x4 v[DEEP];
#pragma unroll
            for (int e = 0; e < DEEP; ++e) {
                const int64_t t = (uint32_t)__builtin_amdgcn_readlane(spot, (i + e) & 63);   // behind `count`: the first again
                v[e] = load4<T, WHOLE>(dout + t * a.ldd, col, 64, a.dim);
            }
#pragma unroll
            for (int e = 0; e < DEEP; ++e)
                if (i + e < count) acc += v[e];
        }
    }
    return acc;
}

__device__ __forceinline__ f32x4 sum_rows(const float* rows, int64_t pitch, int from, int to, int c, f32x4 acc)
{
    for (int i = from; i < to; i += 8) {
        f32x4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const f32x4*>(rows + (int64_t)(i + e < to ? i + e : to - 1) * pitch + c);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < to) acc += v[e];
    }
    return acc;
}

// Sums of the pieces and groups that hold one key alone.  A wave takes a piece, a workgroup a group, 256 columns of it.
template <class T, bool WHOLE>
__global__ __launch_bounds__(kGroup * 64) void k_embed_pieces(const SumArgs a, const T* dout)
{
    __shared__ f32x4 part[kGroup][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = blockIdx.x, piece = group * kGroup + wave, first = piece * kPiece;
    const int c = first_column<WHOLE>(blockIdx.y, lane), kept = kept_column(blockIdx.y, lane);
    if (first + kPiece <= a.n) {
        const uint32_t key = a.key[first];
        if (key == a.key[first + kPiece - 1] && key != a.none) {
            const f32x4 sum = sum_tokens<T, WHOLE, 16>(a, dout, first, first + kPiece, c, lane, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
            *reinterpret_cast<f32x4*>(a.pieces + (int64_t)piece * a.pitch + kept) = sum;
            part[wave][lane] = sum;
        }
    }
    const int64_t end = (int64_t)(group + 1) * kGroup * kPiece;
    if (end > a.n || a.key[end - 1] != a.key[end - kGroup * kPiece] || a.key[end - 1] == a.none) return;
    __syncthreads();   // the whole workgroup or none of it comes here, with all its pieces summed
    if (wave == 0) {
        f32x4 sum = part[0][lane];
#pragma unroll
        for (int w = 1; w < kGroup; ++w) sum += part[w][lane];
        *reinterpret_cast<f32x4*>(a.groups + (int64_t)group * a.pitch + kept) = sum;
    }
}

// First place in [lo, hi) whose key is not below `what`; hi if none is.
__device__ __forceinline__ int lower_bound(const uint32_t* key, int lo, int hi, uint32_t what)
{
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (key[mid] < what) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// The same by a whole wave, 64 places at a time: three steps for 2^18 keys.
__device__ __forceinline__ int wave_lower_bound(const uint32_t* key, int lo, int hi, uint32_t what, int lane)
{
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && key[at] < what);   // a run of ones from lane 0 on
        const int n = __popcll(below);
        if (n == 0) return lo;
        const int top = lo + n * step;
        lo = lo + (n - 1) * step + 1;
        hi = top < hi ? top : hi;
    }
    return lo;
}

// Zeros by a whole wave, 16 bytes a lane between the ends.
__device__ __forceinline__ void zero_floats(float* at, int64_t count, int lane)
{
    int64_t head = (-(reinterpret_cast<uintptr_t>(at) >> 2)) & 3;
    head = head < count ? head : count;
    if (lane < head) at[lane] = 0.0f;
    at += head, count -= head;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t q = lane; q < count >> 2; q += 64) __builtin_nontemporal_store(zero, reinterpret_cast<f32x4*>(at) + q);
    if (lane < (count & 3)) at[(count & ~(int64_t)3) + lane] = 0.0f;
}

// Rows of G that nobody names: a wave takes `rows` (up to 64) consecutive rows and writes zeros to those whose run is
// empty (32 x 37604 rows of 30, a row at a time 95 us).
__device__ __forceinline__ void fill_rows(const SumArgs& a, int64_t vocab, int64_t total, float* G, int64_t ldg, int rows,
                                          int64_t wave, int lane)
{
    const int64_t first = wave * rows;
    if (first >= total) return;
    const int count = total - first < rows ? (int)(total - first) : rows;
    const int lo = wave_lower_bound(a.key, 0, a.n, (uint32_t)first, lane);
    const int hi = wave_lower_bound(a.key, lo, a.n, (uint32_t)(first + count), lane);
    uint64_t empty = ~0ull;
    if (lo < hi) {
        const int begin = lower_bound(a.key, lo, hi, (uint32_t)(first + lane));
        const int end = __shfl_down(begin, 1);
        empty = __ballot(begin == (lane < 63 ? end : hi));
    }
    // neighbouring empty rows of a partition are one stretch of G
    for (int r = 0; r < count;) {
        const uint64_t left = empty >> r;
        if (!(left & 1)) {
            if (left == 0) break;
            r += __builtin_ctzll(left);
            continue;
        }
        int len = ~left ? __builtin_ctzll(~left) : 64;
        len = len < count - r ? len : count - r;
        const int64_t p = (first + r) / vocab, v = first + r - p * vocab;
        if (len > vocab - v) len = (int)(vocab - v);
        zero_floats(G + p * ldg + v * a.dim, (int64_t)len * a.dim, lane);
        r += len;
    }
}

// Rows that somebody names: a wave takes kHeads places of the order and the runs that begin there, 256 columns of them.
constexpr int kHeads = 8;

template <class T, bool WHOLE>
__device__ __forceinline__ void sum_runs(const SumArgs& a, const T* dout, int64_t vocab, float scale, float* G, int64_t ldg,
                                         int64_t wave, int lane)
{
    const int across = (a.dim + 255) >> 8;
    const int64_t strip = wave / across;
    const int mine = (int)(wave - strip * across), c = first_column<WHOLE>(mine, lane), kept = kept_column(mine, lane);
    const int64_t first = strip * kHeads;
    if (first >= a.n) return;
    const int at = (int)first + lane;
    const uint32_t key = at < a.n ? a.key[at] : a.none;
    const uint32_t before = at > 0 && at <= a.n ? a.key[at - 1] : ~0u;
    const uint64_t heads = __ballot(key != before || at >= a.n);
    for (uint64_t left = heads & ((1ull << kHeads) - 1); left; left &= left - 1) {
        const int h = __builtin_ctzll(left);
        const uint32_t k = __builtin_amdgcn_readlane(key, h);
        if (k == a.none) return;   // empty places, or the end: nothing comes behind them
        const int from = (int)first + h;
        const uint64_t later = heads & ~((2ull << h) - 1);
        int to = (int)first + (later ? __builtin_ctzll(later) : 64);
        if (!later) to = wave_lower_bound(a.key, to < a.n ? to : a.n, a.n, k + 1, lane);
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const int p0 = (from + kPiece - 1) / kPiece, p1 = to / kPiece;   // whole pieces
        if (p0 < p1) {
            acc = sum_tokens<T, WHOLE, 8>(a, dout, from, p0 * kPiece, c, lane, acc);
            const int g0 = (p0 + kGroup - 1) / kGroup, g1 = p1 / kGroup;
            if (g0 < g1) {
                acc = sum_rows(a.pieces, a.pitch, p0, g0 * kGroup, kept, acc);
                acc = sum_rows(a.groups, a.pitch, g0, g1, kept, acc);
                acc = sum_rows(a.pieces, a.pitch, g1 * kGroup, p1, kept, acc);
            } else {
                acc = sum_rows(a.pieces, a.pitch, p0, p1, kept, acc);
            }
            acc = sum_tokens<T, WHOLE, 8>(a, dout, p1 * kPiece, to, c, lane, acc);
        } else {
            acc = sum_tokens<T, WHOLE, 8>(a, dout, from, to, c, lane, acc);
        }
        if (c >= a.dim) continue;
        const int64_t p = k / (uint32_t)vocab, v = k - p * vocab;
        store4<float, WHOLE>(G + p * ldg + v * a.dim, c, 64, a.dim, acc * scale);
    }
}

// All rows of G.  The first `sum_blocks` workgroups sum runs, which take longest, the others write zeros.  Bound by the
// write of G: 8 x 32000 x 768 in 156 us, 5.0 TB/s (a fill of 4 GiB: 6.9).
template <class T, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_embed_rows(const SumArgs a, const T* dout, int64_t vocab, int64_t total, float scale,
                                                       float* G, int64_t ldg, int rows, unsigned sum_blocks)
{
    const int lane = threadIdx.x & 63, sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned id = blockIdx.y * gridDim.x + blockIdx.x;
    if (id < sum_blocks) sum_runs<T, WHOLE>(a, dout, vocab, scale, G, ldg, (int64_t)id * 4 + sub, lane);
    else fill_rows(a, vocab, total, G, ldg, rows, (int64_t)(id - sum_blocks) * 4 + sub, lane);
}

template <class TABLE, class OUT, class ID>
hipError_t forward_as(const EmbedCall& c, hipStream_t stream)
{
    const TABLE* table = static_cast<const TABLE*>(c.table);
    OUT* out = static_cast<OUT*>(c.out);
    const ID* tokens = static_cast<const ID*>(c.tokens);
    const bool whole = c.dim % 4 == 0 && c.ld % 4 == 0 && reinterpret_cast<uintptr_t>(table) % (4 * sizeof(TABLE)) == 0 &&
                       reinterpret_cast<uintptr_t>(out) % (4 * sizeof(OUT)) == 0;
    int lanes = 1;
    while (lanes < 64 && lanes * 4 < c.dim) lanes *= 2;
    const int64_t blocks = (c.n + kBlock / lanes - 1) / (kBlock / lanes);
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
    if (whole)
        hipLaunchKernelGGL((k_embed<TABLE, OUT, ID, true>), grid, dim3(kBlock), 0, stream, table, c.vocab, c.dim, tokens, c.n,
                           c.scale, out, c.ld, lanes);
    else
        hipLaunchKernelGGL((k_embed<TABLE, OUT, ID, false>), grid, dim3(kBlock), 0, stream, table, c.vocab, c.dim, tokens, c.n,
                           c.scale, out, c.ld, lanes);
    return hipGetLastError();
}

template <class TABLE, class OUT>
hipError_t forward_with(const EmbedCall& c, hipStream_t stream)
{
    return c.wide_ids ? forward_as<TABLE, OUT, int64_t>(c, stream) : forward_as<TABLE, OUT, int32_t>(c, stream);
}

template <class T, bool WHOLE>
hipError_t sums_as(const EmbedCall& c, const SumArgs& a, hipStream_t stream)
{
    const T* dout = static_cast<const T*>(c.dout);
    const unsigned across = (unsigned)((c.dim + 255) / 256);
    if (a.n >= kPiece) {
        hipLaunchKernelGGL((k_embed_pieces<T, WHOLE>), dim3((a.n + kGroup * kPiece - 1) / (kGroup * kPiece), across),
                           dim3(kGroup * 64), 0, stream, a, dout);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t total = c.vocab * c.k_parts;
    int rows = 64;
    while (rows > 1 && total / rows < 8192) rows /= 2;
    const int64_t fills = (total + rows - 1) / rows, sums = (int64_t)((a.n + kHeads - 1) / kHeads) * across;
    const unsigned sum_blocks = (unsigned)((sums + 3) / 4);
    const FoldedGrid grid = folded_grid(sum_blocks + (fills + 3) / 4, kBlock);
    hipLaunchKernelGGL((k_embed_rows<T, WHOLE>), dim3(grid.x, grid.y), dim3(kBlock), 0, stream, a, dout, c.vocab, total, c.scale,
                       c.G, c.ldg, rows, sum_blocks);
    return hipGetLastError();
}

template <class T>
hipError_t sums_with(const EmbedCall& c, const SumArgs& a, hipStream_t stream)
{
    const bool whole = c.dim % 4 == 0 && c.ld % 4 == 0 && c.ldg % 4 == 0 &&
                       reinterpret_cast<uintptr_t>(c.dout) % (4 * sizeof(T)) == 0 && reinterpret_cast<uintptr_t>(c.G) % 16 == 0;
    return whole ? sums_as<T, true>(c, a, stream) : sums_as<T, false>(c, a, stream);
}

}  // namespace

// keys, places, twice | counts of the sort's tiles | totals | sums of pieces | of groups
int64_t embed_workspace_bytes(int64_t n, int64_t vocab, int dim, int k_parts)
{
    (void)vocab, (void)k_parts;
    const int64_t tiles = (n + kSortTile - 1) / kSortTile, pitch = round_up(dim, 256) * 4;
    return 4 * round_up(n * 4, 256) + round_up(tiles * kMostDigits * 4, 256) + kMostDigits * 4 + round_up(n / kPiece * pitch, 256) +
           round_up(n / (kPiece * kGroup) * pitch, 256) + 256;
}

hipError_t launch_embed_forward(const EmbedCall& c, hipStream_t stream)
{
    if (c.table_bf16)
        return c.value_bf16 ? forward_with<uint16_t, uint16_t>(c, stream) : forward_with<uint16_t, float>(c, stream);
    return c.value_bf16 ? forward_with<float, uint16_t>(c, stream) : forward_with<float, float>(c, stream);
}

hipError_t launch_embed_gradients(const EmbedCall& c, hipStream_t stream)
{
    const int n = (int)c.n, tiles = (n + kSortTile - 1) / kSortTile;
    char* room = c.workspace;
    auto take = [&](int64_t bytes) {
        char* p = room;
        room += round_up(bytes, 256);
        return p;
    };
    uint32_t *key[2], *place[2];
    for (int i = 0; i < 2; ++i) {
        key[i] = reinterpret_cast<uint32_t*>(take((int64_t)n * 4));
        place[i] = reinterpret_cast<uint32_t*>(take((int64_t)n * 4));
    }
    SortArgs order{};
    order.n = n, order.tiles = tiles;
    order.counts = reinterpret_cast<uint32_t*>(take((int64_t)tiles * kMostDigits * 4));
    order.totals = reinterpret_cast<uint32_t*>(take(kMostDigits * 4));
    SumArgs a{};
    a.n = n, a.dim = c.dim, a.ldd = c.ld, a.pitch = round_up(c.dim, 256);
    a.pieces = reinterpret_cast<float*>(take(n / kPiece * a.pitch * 4));
    a.groups = reinterpret_cast<float*>(take(n / (kPiece * kGroup) * a.pitch * 4));
    a.none = (uint32_t)(c.vocab * c.k_parts);
    int now = 0;
    if (n > 0) {
        EmbedParts parts{};
        parts.k = c.k_parts;
        for (int p = 0; p < c.k_parts; ++p) parts.end[p] = (int)c.part_end[p];
        int key_bits = 1;
        while ((a.none >> key_bits) != 0) ++key_bits;
        const int passes = (key_bits + kMostBits - 1) / kMostBits;
        order.bits = (key_bits + passes - 1) / passes;
        const dim3 grid(tiles), block(kBlock);
        if (tiles == 1) {
            order.key_out = key[1], order.place_out = place[1];
            if (c.wide_ids)
                hipLaunchKernelGGL(k_sort_one_tile<KeySource<int64_t>>, grid, block, 0, stream, order, passes,
                                   KeySource<int64_t>{static_cast<const int64_t*>(c.tokens), c.vocab, a.none, key[0], parts});
            else
                hipLaunchKernelGGL(k_sort_one_tile<KeySource<int32_t>>, grid, block, 0, stream, order, passes,
                                   KeySource<int32_t>{static_cast<const int32_t*>(c.tokens), c.vocab, a.none, key[0], parts});
            now = 1;
        }
        for (int pass = 0; tiles > 1 && pass < passes; ++pass, now ^= 1) {
            order.shift = pass * order.bits;
            order.key_in = key[now], order.place_in = place[now], order.key_out = key[now ^ 1], order.place_out = place[now ^ 1];
            if (pass > 0)
                hipLaunchKernelGGL(k_sort_count<SortedSource>, grid, block, 0, stream, order, SortedSource{key[now]});
            else if (c.wide_ids)
                hipLaunchKernelGGL(k_sort_count<KeySource<int64_t>>, grid, block, 0, stream, order,
                                   KeySource<int64_t>{static_cast<const int64_t*>(c.tokens), c.vocab, a.none, key[0], parts});
            else
                hipLaunchKernelGGL(k_sort_count<KeySource<int32_t>>, grid, block, 0, stream, order,
                                   KeySource<int32_t>{static_cast<const int32_t*>(c.tokens), c.vocab, a.none, key[0], parts});
            if (tiles > kFewTiles)
                hipLaunchKernelGGL(k_sort_tiles, dim3(((1 << order.bits) + 63) / 64), dim3(64), 0, stream, order);
            if (pass == 0) hipLaunchKernelGGL(k_sort_move<true>, grid, block, 0, stream, order);
            else hipLaunchKernelGGL(k_sort_move<false>, grid, block, 0, stream, order);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    a.key = key[now], a.place = place[now];
    return c.value_bf16 ? sums_with<uint16_t>(c, a, stream) : sums_with<float>(c, a, stream);
}

}  // namespace agc
