// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// The lookup is a copy of rows: bound by the write of the output and the read of the rows named.
// The gradient is the sum of the row atoms e_token dy^T.  The tokens are sorted (stably, so that equal ones keep their
// order), and each row of the table sums the run of its tokens: no atomics on values, one write per row.  Bound by the read of dy
// and the write of the gradient; from few tokens, by the latency of the launches.
#include <algorithm>
#include <cstring>

#include "element_types.h"

namespace atomo {

namespace {

constexpr int64_t MOST_GROUPS = 1 << 23;   // a grid has less than 2^32 threads

struct Tokens {
    const void* data;
    long long padding;
    int n, bytes;
};

// The row of a token, or -1 (padding), -2 (outside of the table).
__device__ inline int row_of(const Tokens& t, long long token, int rows)
{
    return token == t.padding ? -1 : token < 0 || token >= rows ? -2 : (int)token;
}

// Where keys come from: an array of them, or tokens of 4 or 8 bytes (which the loads of a round must not branch on).
enum { KEYS = 0, TOKENS4 = 4, TOKENS8 = 8 };

template <int SOURCE>
__device__ inline long long token_at(const Tokens& t, long long i)
{
    if constexpr (SOURCE == TOKENS8) return ((const long long*)t.data)[i];
    else return (long long)((const int*)t.data)[i];
}

__device__ inline long long token_at(const Tokens& t, long long i)
{
    return t.bytes == 8 ? token_at<TOKENS8>(t, i) : token_at<TOKENS4>(t, i);
}

// ---------------------------------------------------------------------------------------------
// Neighbouring columns of a row, VEC of them in a lane
// ---------------------------------------------------------------------------------------------

template <int VEC> struct Cols { float x[VEC]; };

template <int TYPE, int VEC, bool ONCE = false>
__device__ inline Cols<VEC> load_cols(const void* base, long long i)
{
    Cols<VEC> c;
    if constexpr (VEC == 1) {
        c.x[0] = load1<TYPE>(base, i);
    } else if constexpr (VEC == 8 && TYPE != ATOMO_F32) {
        const auto at = (const u16x8_any*)((const uint16_t*)base + i);
        const u16x8_any s = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
        for (int k = 0; k < 8; ++k) c.x[k] = Element<TYPE>::up(s[k]);
    } else if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
            const f32x4 v = load4<TYPE, ONCE>(base, i + 4 * q);
#pragma unroll
            for (int k = 0; k < 4; ++k) c.x[4 * q + k] = v[k];
        }
    } else {
        static_assert(VEC == 2, "");
        typedef typename Element<TYPE>::Stored two __attribute__((ext_vector_type(2), aligned(sizeof(typename Element<TYPE>::Stored))));
        const two s = *(const two*)((const typename Element<TYPE>::Stored*)base + i);
        c.x[0] = Element<TYPE>::up(s[0]);
        c.x[1] = Element<TYPE>::up(s[1]);
    }
    return c;
}

// ONCE: see element_types.h; only where the lanes of a wave fill whole lines.
template <int TYPE, int VEC, bool ONCE = false>
__device__ inline void store_cols(void* base, long long i, const Cols<VEC>& c)
{
    typedef typename Element<TYPE>::Stored Stored;
    if constexpr (VEC == 1) {
        store1<TYPE>(base, i, c.x[0]);
    } else if constexpr (VEC == 8 && TYPE != ATOMO_F32) {
        u16x8_any s;
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = Element<TYPE>::down(c.x[k]);
        if constexpr (ONCE) __builtin_nontemporal_store(s, (u16x8_any*)((uint16_t*)base + i));
        else *(u16x8_any*)((uint16_t*)base + i) = s;
    } else if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) store4<TYPE, ONCE>(base, i + 4 * q, f32x4{c.x[4 * q], c.x[4 * q + 1], c.x[4 * q + 2], c.x[4 * q + 3]});
    } else {
        typedef Stored two __attribute__((ext_vector_type(2), aligned(sizeof(Stored))));
        *(two*)((Stored*)base + i) = two{Element<TYPE>::down(c.x[0]), Element<TYPE>::down(c.x[1])};
    }
}

template <int VEC>
__device__ inline void add(Cols<VEC>& a, const Cols<VEC>& b)
{
#pragma unroll
    for (int k = 0; k < VEC; ++k) a.x[k] += b.x[k];
}

// ---------------------------------------------------------------------------------------------
// Lookup: lanes_x threads side by side on a row, ROWS rows of theirs on their way together
// ---------------------------------------------------------------------------------------------

// Sixteen bytes of the output per lane and store, whole lines per wave, which the caches need not keep (with eight columns per lane, fp32
// takes two stores of half a line each, and was slower past the caches than through them by a quarter).  Two rows of a thread on their way: 65,536
// rows of 2048 from bf16 to bf16 68 us, one row 100, four 66; to fp32 97, 163 and 106; from fp32 to bf16 89, 101 and 95.
constexpr int TWO_ROWS = 2, MANY_GROUPS = 4096;

template <int IN, int OUT, int ROWS>
__global__ __launch_bounds__(256) void embedding_rows(Tokens tokens, const void* table, long long ld, int rows, int cols,
                                                      float scale, void* out, long long ld_out, int lanes_x, int32_t* flags)
{
    constexpr int VEC = OUT == ATOMO_F32 ? 4 : 8;
    const int x = threadIdx.x % lanes_x, y = threadIdx.x / lanes_x, per = 256 / lanes_x;
    for (long long base = (long long)blockIdx.x * (per * ROWS) + y; base < tokens.n; base += (long long)gridDim.x * (per * ROWS)) {
        int row[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            row[u] = row_of(tokens, token_at(tokens, min(base + u * per, (long long)tokens.n - 1)), rows);
            if (row[u] == -2 && x == 0) flags[FLAG_TOKEN] = 1;
        }
        for (int col = x * VEC; col < cols; col += lanes_x * VEC) {
            if (col + VEC <= cols) {
                Cols<VEC> a[ROWS];
#pragma unroll
                for (int u = 0; u < ROWS; ++u) a[u] = load_cols<IN, VEC>(table, (long long)max(row[u], 0) * ld + col);
#pragma unroll
                for (int u = 0; u < ROWS; ++u) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) a[u].x[k] = row[u] >= 0 ? a[u].x[k] * scale : 0.0f;
                    if (base + u * per < tokens.n) store_cols<OUT, VEC, true>(out, (base + u * per) * ld_out + col, a[u]);
                }
            } else {
                for (int u = 0; u < ROWS && base + u * per < tokens.n; ++u)
                    for (int j = col; j < cols; ++j)
                        store1<OUT>(out, (base + u * per) * ld_out + j, row[u] >= 0 ? load1<IN>(table, row[u] * ld + j) * scale : 0.0f);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Sort
// ---------------------------------------------------------------------------------------------

// The key of a token: its row, or `rows` if it has none.
__device__ inline uint32_t key_of(const Tokens& t, long long token, int rows, int32_t* flags)
{
    const int row = row_of(t, token, rows);
    if (row == -2 && flags) flags[FLAG_TOKEN] = 1;
    return row < 0 ? (uint32_t)rows : (uint32_t)row;
}

// Up to RANKED tokens: the place of each is the number of those in front of it, by comparison with all.  One launch; n^2 comparisons.
// A workgroup has 32 tokens, one per lane of each half of its sixteen waves, and the halves share out the keys to compare with.
// (8192 tokens of 512 columns into 32,768 rows: 37 us for all of the gradient, 47 with the sort by digits; 12,288: 52, 49.)
constexpr int RANKED = 8192, RANK_TOKENS = 32;

template <int SOURCE>
__global__ __launch_bounds__(1024) void sort_by_rank(Tokens tokens, int rows, uint32_t* keys_out, uint32_t* from_out, int32_t* flags)
{
    __shared__ uint4 keys4[RANKED / 4];
    __shared__ int ranks[32][RANK_TOKENS];
    uint32_t* const keys = (uint32_t*)keys4;
    const int n = tokens.n, lane = threadIdx.x % RANK_TOKENS, part = threadIdx.x / RANK_TOKENS;
    const int blocks = (n + RANK_TOKENS - 1) / RANK_TOKENS, own = blockIdx.x;
    long long token[RANKED / 1024];
#pragma unroll
    for (int k = 0; k < RANKED / 1024; ++k) token[k] = token_at<SOURCE>(tokens, min(k * 1024 + (int)threadIdx.x, n - 1));
#pragma unroll
    for (int k = 0; k < RANKED / 1024; ++k) {
        const int i = k * 1024 + threadIdx.x;
        if (i < blocks * RANK_TOKENS) keys[i] = i < n ? key_of(tokens, token[k], rows, flags) : 0xffffffffu;
    }
    __syncthreads();
    const uint32_t key = keys[own * RANK_TOKENS + lane];
    int rank = 0;
    for (int b = part; b < blocks; b += 32) {
        const uint4* const other = keys4 + b * (RANK_TOKENS / 4);
        // (key, place) in front of (this key, this place); behind the own block equal keys are not
        const uint32_t limit = b < own ? key + 1 : key;          // (keys are below 2^31)
#pragma unroll
        for (int j = 0; j < RANK_TOKENS / 4; ++j) {
            const uint4 o = other[j];
            rank += (o.x < limit ? 1 : 0) + (o.y < limit ? 1 : 0) + (o.z < limit ? 1 : 0) + (o.w < limit ? 1 : 0);
        }
        if (b == own) {
            for (int j = 0; j < RANK_TOKENS; ++j) rank += keys[b * RANK_TOKENS + j] == key && j < lane ? 1 : 0;
        }
    }
    ranks[part][lane] = rank;
    __syncthreads();
    if (part == 0 && own * RANK_TOKENS + lane < n) {
        int to = 0;
#pragma unroll
        for (int p = 0; p < 32; ++p) to += ranks[p][lane];
        keys_out[to] = key;
        from_out[to] = (uint32_t)(own * RANK_TOKENS + lane);
    }
}

// More: least significant digit first, two launches per digit.  A workgroup of sixteen waves has a part of the keys; few parts, so that each
// can add up the counts of those in front of it by itself.  (That it counts the keys of all parts itself, in one launch, is no faster at
// 8193 tokens, and slower from 16,384 on: 42 and 40 us in all, 55 and 43 at 32,768.)
constexpr int MOST_BITS = 9, MOST_BINS = 1 << MOST_BITS;
constexpr int ROUNDS = 4;              // keys of a lane that are on their way at a time

struct Digit { int shift, bits; };

template <int SOURCE>
__device__ inline uint32_t key_at(const Tokens& t, const uint32_t* keys, long long i, int rows, int32_t* flags)
{
    if constexpr (SOURCE == KEYS) return keys[i];
    else return key_of(t, token_at<SOURCE>(t, i), rows, flags);
}

// counts[part][digit]
template <int SOURCE>
__global__ __launch_bounds__(1024) void sort_count(Tokens tokens, const uint32_t* keys, int rows, Digit d, int per, int* counts, int32_t* flags)
{
    __shared__ int hist[MOST_BINS];
    const int bins = 1 << d.bits;
    if ((int)threadIdx.x < bins) hist[threadIdx.x] = 0;
    __syncthreads();
    const long long first = (long long)blockIdx.x * per, end = min(first + per, (long long)tokens.n);
    for (long long base = first + threadIdx.x; base < end; base += 1024 * ROUNDS) {
        uint32_t key[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) key[r] = key_at<SOURCE>(tokens, keys, min(base + r * 1024, end - 1), rows, flags);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (base + r * 1024 < end) atomicAdd(&hist[key[r] >> d.shift & (bins - 1)], 1);
    }
    __syncthreads();
    if ((int)threadIdx.x < bins) counts[(long long)blockIdx.x * bins + threadIdx.x] = hist[threadIdx.x];
}

// Each wave takes a sixteenth of the part, 64 keys after the other: a key's place is that of its digit, plus what the waves in front and the
// keys in front of it have of the same digit.  Bound by the latency of its loads.
template <int SOURCE>
__global__ __launch_bounds__(1024) void sort_place(Tokens tokens, const uint32_t* keys, const uint32_t* from, int rows, Digit d, int per,
                                                   int parts, const int* counts, uint32_t* keys_out, uint32_t* from_out)
{
    __shared__ int at[16][MOST_BINS];
    __shared__ int before[MOST_BINS], totals[MOST_BINS];
    __shared__ int sums[8];
    const int bins = 1 << d.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long first = (long long)blockIdx.x * per + wave * (per / 16);
    const long long end = min(first + per / 16, (long long)tokens.n);
    uint32_t key[ROUNDS], source[ROUNDS];
    const auto load = [&](long long base, bool sources) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const long long i = min(base + r * 64 + lane, (long long)tokens.n - 1);   // (what is beyond the end is not looked at)
            key[r] = key_at<SOURCE>(tokens, keys, i, rows, nullptr);
            if (sources) source[r] = SOURCE == KEYS ? from[i] : (uint32_t)i;
        }
    };
    // how often each digit comes in the parts in front, and at all: a thread per digit and share of the parts
    const int digit = (int)threadIdx.x & (bins - 1), stride = 1024 >> d.bits;
    int in_front = 0, in_all = 0;
    for (int p = (int)threadIdx.x >> d.bits; p < parts; p += 16 * stride) {
        int c[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) c[q] = counts[((long long)min(p + q * stride, parts - 1) << d.bits) + digit];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int part = p + q * stride;
            in_all += part < parts ? c[q] : 0;
            in_front += part < (int)blockIdx.x ? c[q] : 0;
        }
    }
    load(first, true);
    for (int b = threadIdx.x; b < 16 * MOST_BINS; b += 1024) ((int*)at)[b] = 0;
    if (threadIdx.x < MOST_BINS) before[threadIdx.x] = totals[threadIdx.x] = 0;
    __syncthreads();
    if (in_all) {
        atomicAdd(&totals[digit], in_all);
        atomicAdd(&before[digit], in_front);
    }
    for (long long base = first; base < end; base += 64 * ROUNDS) {
        if (base > first) load(base, false);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (base + r * 64 + lane < end) atomicAdd(&at[wave][key[r] >> d.shift & (bins - 1)], 1);
    }
    __syncthreads();
    const int total = (int)threadIdx.x < bins ? totals[threadIdx.x] : 0;
    int sum = total;                                             // of the digits up to this one, first within the wave
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int other = __shfl_up(sum, s);
        if (lane >= s) sum += other;
    }
    if (wave < 8 && lane == 63) sums[wave] = sum;
    __syncthreads();
    if ((int)threadIdx.x < bins) {
        int place = before[threadIdx.x] + sum - total;
        for (int w = 0; w < wave; ++w) place += sums[w];
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const int c = at[w][threadIdx.x];
            at[w][threadIdx.x] = place;
            place += c;
        }
    }
    __syncthreads();
    for (long long base = first; base < end; base += 64 * ROUNDS) {
        if (per > 16 * 64 * ROUNDS) load(base, true);            // (else they are those from the beginning)
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const bool live = base + r * 64 + lane < end;
            const int digit = (int)(key[r] >> d.shift & (bins - 1));
            uint64_t same = __ballot(live);
            for (int b = 0; b < d.bits; ++b) {
                const uint64_t set = __ballot(digit >> b & 1);
                same &= (digit >> b & 1) ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            int to = 0;
            if (live) to = at[wave][digit] + rank;
            lanes_in_order();
            if (live && rank == 0) at[wave][digit] += __popcll(same);
            lanes_in_order();
            if (live) {
                keys_out[to] = key[r];
                from_out[to] = source[r];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------------------------

// Lanes of a wave lie side by side on the columns, VEC each.  The last lane moves back to where it ends with the columns: it then forms
// what its neighbour forms, and stores the same.  A tile of fewer than VEC columns is taken one column per lane.
// What is read once (dy) and what is written once (zeros, sums) goes past the caches: 32,768 tokens into 65,536 x 2048 175 -> 162 us.

struct Grad {
    void* data;
    long long ld;
    uint32_t rows;
    int cols;
    float scale;
};

// `before`: what the row held, if sums are added to it.  Lanes that overlap have all read that before one of them writes.
template <int OUT, int VEC>
__device__ inline Cols<VEC> load_before(const Grad& g, uint32_t row, int col)
{
    return load_cols<OUT, VEC>(g.data, (long long)row * g.ld + col);
}

template <int OUT, bool ACC, int VEC>
__device__ inline void write_sum(const Grad& g, uint32_t row, int col, Cols<VEC> sum, const Cols<VEC>& before)
{
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum.x[k] *= g.scale;
    if constexpr (ACC) {
        add(sum, before);
        lanes_in_order();
    }
    store_cols<OUT, VEC, VEC * sizeof(typename Element<OUT>::Stored) <= 16>(g.data, (long long)row * g.ld + col, sum);
}

// Sums of the runs of equal keys among `length` sorted tokens, by one wave: runs that lie within the piece are written, the
// others go into `heads` (the run has begun in front of the piece) and `tails` (it begins here and does not end), one row per piece each.
struct Pieces {
    const uint32_t* keys;
    const uint32_t* from;
    int n, length;
    float* heads;
    float* tails;
    long long ld;
    uint32_t* notes;                   // of each piece: what its last run does, and the run's key behind it
};

// The last run of a piece ends in it; begins in it and goes on; fills it, having begun in front of it, and goes on.
enum : uint32_t { ENDS = 0, BEGINS = 1, PASSES = 2 };

constexpr int AHEAD = 8;               // rows on their way at a time

template <int IN, int OUT, int VEC, bool ACC>
__device__ void sum_piece(const Pieces& s, int piece, bool noting, const void* dy, long long ld_dy, int col, bool mine, const Grad& g)
{
    const int lane = threadIdx.x & 63, first = piece * s.length;
    const int here = min(s.length, s.n - first);
    const uint32_t key = lane < here ? s.keys[first + lane] : g.rows;
    const uint32_t from = lane < here ? s.from[first + lane] : 0;
    const uint32_t in_front = first > 0 ? s.keys[first - 1] : g.rows, behind = s.n - first > s.length ? s.keys[first + s.length] : g.rows;
    const int count = __popcll(__ballot(key < g.rows));          // (those of no row stand behind all others)
    if (count == 0) {
        if (noting && lane == 0) s.notes[2 * piece] = ENDS;
        return;
    }
    const bool begun = in_front == (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
    const bool goes_on = count == s.length && behind == (uint32_t)__builtin_amdgcn_readlane((int)key, count - 1);
    const uint32_t next = (uint32_t)__shfl_down((int)key, 1);
    const uint64_t ends = __ballot(lane < count && (lane == count - 1 || key != next));
    if (noting && lane == 0) {
        s.notes[2 * piece] = !goes_on ? ENDS : begun && ends == 1ull << (count - 1) ? PASSES : BEGINS;
        s.notes[2 * piece + 1] = behind;
    }
    Cols<VEC> sum = {};
    bool in_first = true;
    for (int i = 0; i < count; i += AHEAD) {
        Cols<VEC> x[AHEAD], before[ACC ? AHEAD : 1];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i + u < count) {
                const long long row = (long long)(uint32_t)__builtin_amdgcn_readlane((int)from, i + u);
                const uint32_t to = (uint32_t)__builtin_amdgcn_readlane((int)key, i + u);
                if (mine) {
                    x[u] = load_cols<IN, VEC, true>(dy, row * ld_dy + col);
                    if constexpr (ACC) {
                        if (ends >> (i + u) & 1) before[u] = load_before<OUT, VEC>(g, to, col);
                    }
                }
            }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i + u < count) {
                if (mine) add(sum, x[u]);
                if (ends >> (i + u) & 1) {
                    const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, i + u);
                    if (mine) {
                        if (in_first && begun) store_cols<ATOMO_F32, VEC>(s.heads, piece * s.ld + col, sum);
                        else if (i + u == count - 1 && goes_on) store_cols<ATOMO_F32, VEC>(s.tails, piece * s.ld + col, sum);
                        else write_sum<OUT, ACC, VEC>(g, row, col, sum, before[ACC ? u : 0]);
                    }
                    in_first = false;
                    sum = Cols<VEC>{};
                }
            }
    }
}

// How many of the sorted keys are below `key`: 64 probes at a time.
__device__ inline int keys_below(const uint32_t* keys, int n, uint32_t key)
{
    int lo = 0, left = n;
    while (left > 0) {
        const int step = (left + 63) / 64;
        const long long at = (long long)((threadIdx.x & 63) + 1) * step - 1;
        const int passed = __popcll(__ballot(at < left && keys[lo + at] < key));
        lo += passed * step;
        left = min(step - 1, left - passed * step);
    }
    return lo;
}

constexpr int ZERO_ROWS = 256;         // most rows of a workgroup that writes zeros

// Zeros in those of the rows [first, end) that are not named, a wave per row.
template <int OUT>
__device__ inline void write_zeros(const uint8_t* named, uint32_t first, uint32_t end, const Grad& g)
{
    constexpr int VEC = OUT == ATOMO_F32 ? 4 : 8;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const Cols<VEC> zero = {};
    for (uint32_t r = first + wave; r < end; r += 4) {
        if (named[r - first]) continue;
        for (int col = lane * VEC; col < g.cols; col += 64 * VEC) {
            if (col + VEC <= g.cols) store_cols<OUT, VEC, true>(g.data, (long long)r * g.ld + col, zero);
            else for (int j = col; j < g.cols; ++j) store1<OUT>(g.data, (long long)r * g.ld + j, 0.0f);
        }
    }
}

// Zeros for those of `per` rows that no token names.
template <int OUT>
__device__ void zero_rows(const uint32_t* keys, int n, uint32_t first, int per, const Grad& g)
{
    __shared__ int bounds[2];
    __shared__ uint8_t named[ZERO_ROWS];
    const uint32_t end = min(first + (uint32_t)per, g.rows);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wave < 2) {
        const int at = keys_below(keys, n, wave ? end : first);
        if (lane == 0) bounds[wave] = at;
    }
    __syncthreads();
    const int hi = bounds[1];
    if ((int)threadIdx.x < (int)(end - first)) {
        const uint32_t row = first + threadIdx.x;
        int lo = bounds[0], up = hi;
        while (lo < up) {
            const int mid = lo + (up - lo) / 2;
            if (keys[mid] < row) lo = mid + 1;
            else up = mid;
        }
        named[threadIdx.x] = lo < hi && keys[lo] == row;
    }
    __syncthreads();
    write_zeros<OUT>(named, first, end, g);
}

// Waves of the first workgroups take a piece and a tile of columns each; the workgroups behind them write the zeros.  (On a stream of their
// own beside the sort, with a byte per row for what the tokens name, they made no difference beyond 3 %, and needed a second stream.)
template <int IN, int OUT, int VEC, bool ACC>
__global__ __launch_bounds__(256) void sum_pieces(Pieces s, const void* dy, long long ld_dy, Grad g, int pieces, int tiles, unsigned groups, int zero_per)
{
    if (blockIdx.x >= groups) {
        for (unsigned long long b = blockIdx.x - groups; b * zero_per < g.rows; b += gridDim.x - groups) {
            zero_rows<OUT>(s.keys, s.n, (uint32_t)(b * zero_per), zero_per, g);
            __syncthreads();
        }
        return;
    }
    const int lane = threadIdx.x & 63;
    for (long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); w < (long long)pieces * tiles; w += (long long)groups * 4) {
        const int piece = __builtin_amdgcn_readfirstlane((int)(w / tiles)), tile = __builtin_amdgcn_readfirstlane((int)(w % tiles));
        const int first = tile * (64 * VEC), left = g.cols - first;
        if (left >= VEC) sum_piece<IN, OUT, VEC, ACC>(s, piece, tile == 0, dy, ld_dy, min(first + lane * VEC, g.cols - VEC), lane * VEC < left, g);
        else sum_piece<IN, OUT, 1, ACC>(s, piece, tile == 0, dy, ld_dy, first + lane, lane < left, g);
    }
}

// Runs over several pieces: the tail of the piece in which a run begins, and the heads of those behind it up to its end.  A
// workgroup looks after JOINED pieces and 256 columns; a wave adds up to SHORT rows by itself, longer runs are shared out among the
// sixteen.  Bound by latency: the notes, then the rows, then the store (found by searching the keys instead, the ends took ten loads one
// after the other: 16 - 24 us).
constexpr int SHORT = 16, JOINED = 16;

// The sum of rows [k, end), sixteen of them on their way at a time.
template <int VEC>
__device__ inline void add_rows(Cols<VEC>& sum, const float* rows, long long ld, int k, int end, int col)
{
    for (; k < end; k += 2 * AHEAD) {
        Cols<VEC> x[2 * AHEAD];
#pragma unroll
        for (int u = 0; u < 2 * AHEAD; ++u)
            if (k + u < end) x[u] = load_cols<ATOMO_F32, VEC>(rows, (k + u) * ld + col);
#pragma unroll
        for (int u = 0; u < 2 * AHEAD; ++u)
            if (k + u < end) add(sum, x[u]);
    }
}

template <int OUT, int VEC, bool ACC>
__device__ void join_tile(const Pieces& s, int pieces, int base, int col, bool mine, const Grad& g)
{
    __shared__ Cols<VEC> part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // lane k: the note of piece base + k; a run that begins in one ends in the first behind it that is not passed
    const int piece = base + lane;
    const uint32_t note = piece < pieces ? s.notes[2 * piece] : ENDS;
    const uint32_t key = piece < pieces ? s.notes[2 * piece + 1] : 0;
    const uint64_t stops = __ballot(note != PASSES);
    const uint64_t behind = lane < 63 ? stops >> (lane + 1) : 0;
    const int last = behind ? piece + 1 + __builtin_ctzll(behind) : piece + 64;   // (beyond these 64: further below)
    const uint64_t runs = __ballot(lane < JOINED && note == BEGINS), longer = __ballot(last - piece > SHORT);
    int turn = 0;
    for (uint64_t left = runs & ~longer; left; left &= left - 1, ++turn) {
        const int at = __builtin_ctzll(left);
        const int p = base + at, q = __builtin_amdgcn_readlane(last, at);
        const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, at);
        if (turn % 16 != wave || !mine) continue;
        Cols<VEC> before = {}, sum;
        if constexpr (ACC) before = load_before<OUT, VEC>(g, row, col);
        sum = load_cols<ATOMO_F32, VEC>(s.tails, p * s.ld + col);
        add_rows(sum, s.heads, s.ld, p + 1, q + 1, col);
        write_sum<OUT, ACC, VEC>(g, row, col, sum, before);
    }
    for (uint64_t left = runs & longer; left; left &= left - 1) {
        const int at = __builtin_ctzll(left);
        const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, at);
        const int p = base + at;
        int q = __builtin_amdgcn_readlane(last, at);
        if (!(stops >> at >> 1)) {                               // 256 notes at a time
            for (q = base + 64;; q += 256) {
                uint32_t more[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) more[k] = q + k * 64 + lane < pieces ? s.notes[2 * (q + k * 64 + lane)] : ENDS;
                uint64_t stop[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) stop[k] = __ballot(more[k] != PASSES);
                const int k = stop[0] ? 0 : stop[1] ? 1 : stop[2] ? 2 : 3;
                const uint64_t found = k == 0 ? stop[0] : k == 1 ? stop[1] : k == 2 ? stop[2] : stop[3];
                if (!found) continue;
                q += k * 64 + __builtin_ctzll(found);
                break;
            }
        }
        const int share = (q - p + 15) / 16;
        const int k0 = p + 1 + wave * share, k1 = min(k0 + share, q + 1);
        Cols<VEC> sum = {}, before = {};
        if (mine) add_rows(sum, s.heads, s.ld, k0, k1, col);
        part[wave][lane] = sum;
        if (wave == 0 && mine) {
            if constexpr (ACC) before = load_before<OUT, VEC>(g, row, col);
            sum = load_cols<ATOMO_F32, VEC>(s.tails, p * s.ld + col);
        }
        __syncthreads();
        if (wave == 0 && mine) {
#pragma unroll
            for (int w = 0; w < 16; ++w) add(sum, part[w][lane]);
            write_sum<OUT, ACC, VEC>(g, row, col, sum, before);
        }
        __syncthreads();
    }
}

template <int OUT, bool ACC>
__global__ __launch_bounds__(1024) void join_pieces(Pieces s, Grad g, int pieces)
{
    const int lane = threadIdx.x & 63;
    for (int tile = blockIdx.y; tile * 256 < g.cols; tile += gridDim.y) {
        const int first = tile * 256, left = g.cols - first;
        if (left >= 4) join_tile<OUT, 4, ACC>(s, pieces, (int)blockIdx.x * JOINED, min(first + lane * 4, g.cols - 4), lane * 4 < left, g);
        else join_tile<OUT, 1, ACC>(s, pieces, (int)blockIdx.x * JOINED, first + lane, lane < left, g);
    }
}

// ---------------------------------------------------------------------------------------------
// Few tokens: one launch.  Every workgroup reads them all; the one of the first place of a token finds the others by comparison, a quarter of
// the list per wave, and adds up their rows.  Up to FEW_GROUPS workgroups: 1024 tokens x 2048 columns 17 us, by pieces 20; 1024 x 4096 31, 22.
// ---------------------------------------------------------------------------------------------

constexpr int FEW = 2048, FEW_GROUPS = 4096;

// Keys of the tokens first, first + step, ..., all loaded before one is looked at; `rows` from `end` on.
__device__ inline void keys_of_few(const Tokens& tokens, int first, int step, int end, int rows, uint32_t (&keys)[FEW / 256])
{
    long long token[FEW / 256] = {};
    const auto load = [&](auto source) {
#pragma unroll
        for (int b = 0; b < FEW / 256; ++b)
            if (b * 256 < tokens.n) token[b] = token_at<source>(tokens, min(first + b * step, tokens.n - 1));
    };
    if (tokens.bytes == 8) load(std::integral_constant<int, TOKENS8>());
    else load(std::integral_constant<int, TOKENS4>());
#pragma unroll
    for (int b = 0; b < FEW / 256; ++b) keys[b] = first + b * step < end ? key_of(tokens, token[b], rows, nullptr) : (uint32_t)rows;
}

template <int IN, int OUT, int VEC, bool ACC>
__device__ void sum_few(const Tokens& tokens, const void* dy, long long ld_dy, int own, int col, bool mine, const Grad& g, int32_t* flags)
{
    __shared__ Cols<VEC> part[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = tokens.n;
    const int share = (n + 255) / 256 * 64, first = wave * share;            // places of this wave
    uint32_t keys[FEW / 256];
    keys_of_few(tokens, first + lane, 64, min(first + share, n), (int)g.rows, keys);
    const uint32_t key = key_of(tokens, token_at(tokens, own), (int)g.rows, flags);
    if (key == g.rows) return;
    uint64_t same[FEW / 256];
    bool seen = false;
#pragma unroll
    for (int b = 0; b < FEW / 256; ++b) {
        same[b] = b * 256 < n ? __ballot(keys[b] == key) : 0;
        if (same[b] && first + b * 64 + __builtin_ctzll(same[b]) < own) seen = true;
    }
    if (__syncthreads_or(seen)) return;
    Cols<VEC> sum = {}, before = {};
    if (ACC && wave == 0 && mine) before = load_before<OUT, VEC>(g, key, col);
#pragma unroll
    for (int b = 0; b < FEW / 256; ++b) {
        uint64_t left = same[b];
        while (left) {
            Cols<VEC> x[AHEAD];
            int count = 0;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (left) {
                    const long long row = first + b * 64 + __builtin_ctzll(left);
                    left &= left - 1;
                    if (mine) x[u] = load_cols<IN, VEC>(dy, row * ld_dy + col);
                    count = u + 1;
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (u < count && mine) add(sum, x[u]);
        }
    }
    if (wave > 0) part[wave - 1][lane] = sum;
    __syncthreads();
    if (wave == 0 && mine) {
#pragma unroll
        for (int w = 0; w < 3; ++w) add(sum, part[w][lane]);
        write_sum<OUT, ACC, VEC>(g, key, col, sum, before);
    }
}

template <int IN, int OUT, int VEC, bool ACC>
__global__ __launch_bounds__(256) void grad_of_few(Tokens tokens, const void* dy, long long ld_dy, Grad g, int tiles, unsigned groups, int zero_per, int32_t* flags)
{
    const int lane = threadIdx.x & 63;
    if (blockIdx.x < groups) {
        for (unsigned w = blockIdx.x; w < (unsigned)tokens.n * (unsigned)tiles; w += groups) {
            const int own = (int)(w / tiles), tile = (int)(w % tiles);
            const int first = tile * (64 * VEC), left = g.cols - first;
            if (left >= VEC) sum_few<IN, OUT, VEC, ACC>(tokens, dy, ld_dy, own, min(first + lane * VEC, g.cols - VEC), lane * VEC < left, g, flags);
            else sum_few<IN, OUT, 1, ACC>(tokens, dy, ld_dy, own, first + lane, lane < left, g, flags);
            __syncthreads();
        }
        return;
    }
    __shared__ uint8_t named[ZERO_ROWS];
    for (unsigned long long b = blockIdx.x - groups; b * zero_per < g.rows; b += gridDim.x - groups) {
        const uint32_t first = (uint32_t)(b * zero_per), end = min(first + (uint32_t)zero_per, g.rows);
        named[threadIdx.x] = 0;
        __syncthreads();
        uint32_t keys[FEW / 256];
        keys_of_few(tokens, threadIdx.x, 256, tokens.n, (int)g.rows, keys);
#pragma unroll
        for (int q = 0; q < FEW / 256; ++q)
            if (keys[q] >= first && keys[q] < end) named[keys[q] - first] = 1;
        __syncthreads();
        write_zeros<OUT>(named, first, end, g);
        __syncthreads();
    }
}

struct Layout {
    uint32_t* keys[2];
    uint32_t* from[2];
    int* counts;
    int passes, bits, parts, per;      // passes == 0: by rank
    float* heads;
    float* tails;
    long long ld;                      // of a row of those
    int pieces, length;
    uint32_t* notes;
    size_t bytes;
};

Layout layout_of(void* base, int64_t n, int64_t rows, int cols)
{
    Layout l = {};
    const int bits = 64 - __builtin_clzll((unsigned long long)rows);             // of keys 0 .. rows
    l.passes = n <= RANKED ? 0 : (bits + MOST_BITS - 1) / MOST_BITS;
    l.bits = l.passes ? (bits + l.passes - 1) / l.passes : 0;
    // as few rounds of a workgroup's waves as 64 parts allow, whose counts it adds up in passing
    const int64_t parts = n <= 1 << 20 ? 64 : 256;
    l.per = (int)std::max<int64_t>(1024, (n + parts * 1024 - 1) / (parts * 1024) * 1024);
    l.parts = (int)((n + l.per - 1) / l.per);
    // long pieces write fewer rows that have to be joined, short ones make more waves: 64 tokens from 4096 waves on
    const int64_t tiles = (cols + 511) / 512;
    l.length = 64;
    while (l.length > 16 && (n + l.length - 1) / l.length * tiles < 4096) l.length /= 2;
    l.pieces = (int)((n + l.length - 1) / l.length);
    l.ld = ((long long)cols + 3) / 4 * 4;
    Carver c(base);
    for (int k = 0; k < 2; ++k) {
        l.keys[k] = c.take<uint32_t>(n);
        l.from[k] = c.take<uint32_t>(n);
    }
    l.counts = c.take<int>((size_t)l.parts << l.bits);
    l.heads = c.take<float>(l.pieces * l.ld);
    l.tails = c.take<float>(l.pieces * l.ld);
    l.notes = c.take<uint32_t>(2 * (size_t)l.pieces);
    l.bytes = c.off;
    return l;
}

// Calls f with where keys come from.  (Kernels are launched by name: for a call through a pointer the host sanitizer reads what lies in
// front of the kernel's handle, and the optimizer then drops the launch as undefined.)
template <typename F>
void with_source(const Tokens& t, bool sorted, F&& f)
{
    if (sorted) f(std::integral_constant<int, KEYS>());
    else if (t.bytes == 8) f(std::integral_constant<int, TOKENS8>());
    else f(std::integral_constant<int, TOKENS4>());
}

Tokens tokens_of(const atomo_tokens& t) { return Tokens{t.data, (long long)t.padding, (int)t.n, t.bytes}; }

}  // namespace

size_t embedding_workspace_bytes(int64_t n_tokens, int64_t rows, int32_t cols) { return layout_of(nullptr, n_tokens, rows, cols).bytes; }

int embedding(atomo_ctx* ctx, const atomo_rows& table, const atomo_tokens& tokens, float scale, const atomo_rows& out, hipStream_t stream)
{
    if (tokens.n == 0) return ATOMO_OK;
    int lanes_x = 1;
    while (lanes_x < 256 && lanes_x * (out.type == ATOMO_F32 ? 4 : 8) < table.cols) lanes_x *= 2;
    const int per = 256 / lanes_x;
    const bool many = tokens.n / per >= MANY_GROUPS;             // (else workgroups are what there is too little of)
    const int64_t each = many ? per * TWO_ROWS : per;
    const unsigned grid = (unsigned)std::min<int64_t>(MOST_GROUPS, (tokens.n + each - 1) / each);
    ProfScope ps(ctx, ATOMO_K_EMBEDDING, stream);
    with_type(table.type, [&](auto in) {
        with_type(out.type, [&](auto ty) {
            const auto launch = [&](auto rows) {
                embedding_rows<in, ty, rows><<<grid, 256, 0, stream>>>(tokens_of(tokens), table.data, table.ld, (int)table.rows, table.cols,
                                                                      scale, out.data, out.ld, lanes_x, ctx->d_flags);
            };
            if (many) launch(std::integral_constant<int, TWO_ROWS>());
            else launch(std::integral_constant<int, 1>());
        });
    });
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

int embedding_grad(atomo_ctx* ctx, const atomo_tokens& tokens, const atomo_rows& dy, float scale, const atomo_rows& grad,
                   bool accumulate, hipStream_t stream)
{
    if (tokens.n == 0 && accumulate) return ATOMO_OK;
    const int64_t few_tiles = (grad.cols - 1) / (dy.type == ATOMO_F32 ? 256 : 512) + 1;
    const bool few = tokens.n <= FEW && tokens.n * few_tiles <= FEW_GROUPS;
    const int rc = few ? ATOMO_OK : workspace_for_stream(ctx, layout_of(nullptr, tokens.n, grad.rows, grad.cols).bytes, stream);
    if (rc != ATOMO_OK) return rc;
    const Layout l = few ? Layout{} : layout_of(ctx->ws, tokens.n, grad.rows, grad.cols);
    const Tokens t = tokens_of(tokens);
    const Grad g = {grad.data, (long long)grad.ld, (uint32_t)grad.rows, grad.cols, scale};
    // workgroups that write zeros: at least four rows each, at most 128 KiB, and a thousand workgroups where there are as many rows
    // (849 rows of 192 columns, bf16, in four workgroups of 256 rows: 14.0 us, now 7.1)
    const int64_t row_bytes = (int64_t)grad.cols * type_bytes(grad.type);
    const int zero_per = (int)std::max<int64_t>(4, std::min<int64_t>(ZERO_ROWS, std::min<int64_t>((128 << 10) / row_bytes, grad.rows / 1024)));
    const unsigned zeros = accumulate ? 0 : (unsigned)std::min<int64_t>(MOST_GROUPS / 2, (grad.rows + zero_per - 1) / zero_per);
    ProfScope ps(ctx, ATOMO_K_EMBEDDING, stream);
    int at = 0;
    if (!few && l.passes == 0) {
        with_source(t, false, [&](auto source) {
            sort_by_rank<source><<<(t.n + RANK_TOKENS - 1) / RANK_TOKENS, 1024, 0, stream>>>(t, (int)grad.rows, l.keys[0], l.from[0], ctx->d_flags);
        });
    }
    for (int p = 0; p < l.passes; ++p) {
        const Digit d = {p * l.bits, l.bits};
        with_source(t, p > 0, [&](auto source) {
            sort_count<source><<<l.parts, 1024, 0, stream>>>(t, l.keys[at], (int)grad.rows, d, l.per, l.counts, ctx->d_flags);
            sort_place<source><<<l.parts, 1024, 0, stream>>>(t, l.keys[at], l.from[at], (int)grad.rows, d, l.per, l.parts, l.counts,
                                                             l.keys[1 - at], l.from[1 - at]);
        });
        at = 1 - at;
    }
    const Pieces pieces = {l.keys[at], l.from[at], t.n, l.length, l.heads, l.tails, l.ld, l.notes};
    with_type(dy.type, [&](auto in) {
        with_type(grad.type, [&](auto ty) {
            const auto launch = [&](auto vec, auto acc) {
                const int tiles = (grad.cols - 1) / (64 * vec) + 1;
                if (few) {
                    const unsigned groups = (unsigned)std::min<int64_t>(MOST_GROUPS / 2, tokens.n * tiles);
                    grad_of_few<in, ty, vec, acc><<<groups + zeros, 256, 0, stream>>>(t, dy.data, dy.ld, g, tiles, groups, zero_per, ctx->d_flags);
                } else {
                    const unsigned groups = (unsigned)std::min<int64_t>(MOST_GROUPS / 2, ((int64_t)l.pieces * tiles + 3) / 4);
                    sum_pieces<in, ty, vec, acc><<<groups + zeros, 256, 0, stream>>>(pieces, dy.data, dy.ld, g, l.pieces, tiles, groups, zero_per);
                }
            };
            // few columns: as many lanes as there are, with less each
            constexpr int WIDE = in == ATOMO_F32 ? 4 : 8, NARROW = in == ATOMO_F32 ? 1 : 2;
            const auto launch_vec = [&](auto acc) {
                if (grad.cols <= 64 * NARROW) launch(std::integral_constant<int, NARROW>(), acc);
                else launch(std::integral_constant<int, WIDE>(), acc);
            };
            if (accumulate) launch_vec(std::true_type());
            else launch_vec(std::false_type());
        });
    });
    if (!few) {
        const dim3 grid((unsigned)((l.pieces + JOINED - 1) / JOINED), (unsigned)std::min(256, (grad.cols - 1) / 256 + 1));
        with_type(grad.type, [&](auto ty) {
            if (accumulate) join_pieces<ty, true><<<grid, 1024, 0, stream>>>(pieces, g, l.pieces);
            else join_pieces<ty, false><<<grid, 1024, 0, stream>>>(pieces, g, l.pieces);
        });
    }
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

}  // namespace atomo
