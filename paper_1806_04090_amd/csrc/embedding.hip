// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// The lookup is a copy of rows: bound by the write of the output and the read of the rows named.
// The gradient is the sum of the row atoms e_token dy^T.  The tokens are sorted (stably, so that equal ones keep their
// order), and each row of the table sums the run of its tokens: no atomics on values, one write per row.  Bound by the read of dy
// and the write of the gradient.
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

__device__ inline long long token_at(const Tokens& t, long long i)
{
    return t.bytes == 8 ? ((const long long*)t.data)[i] : (long long)((const int*)t.data)[i];
}

// The row of a token, or -1 (padding), -2 (outside of the table).
__device__ inline int row_of(const Tokens& t, long long i, int rows)
{
    const long long token = token_at(t, i);
    return token == t.padding ? -1 : token < 0 || token >= rows ? -2 : (int)token;
}

// ---------------------------------------------------------------------------------------------
// Lookup: lanes_x threads side by side on a row, eight elements each
// ---------------------------------------------------------------------------------------------

template <int IN, int OUT>
__global__ __launch_bounds__(256) void embedding_rows(Tokens tokens, const void* table, long long ld, int rows, int cols,
                                                      float scale, void* out, long long ld_out, int lanes_x, int32_t* flags)
{
    const int x = threadIdx.x % lanes_x, y = threadIdx.x / lanes_x, per = 256 / lanes_x;
    for (long long t = (long long)blockIdx.x * per + y; t < tokens.n; t += (long long)gridDim.x * per) {
        const int row = row_of(tokens, t, rows);
        if (row == -2 && x == 0) flags[FLAG_TOKEN] = 1;
        for (int col = x * 8; col < cols; col += lanes_x * 8) {
            if (col + 8 <= cols) {
                f32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
                if (row >= 0) {
                    a = load4<IN>(table, row * ld + col) * scale;
                    b = load4<IN>(table, row * ld + col + 4) * scale;
                }
                store4<OUT>(out, t * ld_out + col, a);
                store4<OUT>(out, t * ld_out + col + 4, b);
            } else {
                for (int j = col; j < cols; ++j) store1<OUT>(out, t * ld_out + j, row >= 0 ? load1<IN>(table, row * ld + j) * scale : 0.0f);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Sort: least significant digit first, three launches per digit
// ---------------------------------------------------------------------------------------------

constexpr int MOST_BINS = 1024, MOST_PARTS = 512;

struct Digit { int shift, bits; };

// Keys of the first pass come from the tokens themselves: their rows, `rows` for those that have none.
__device__ inline uint32_t key_at(const Tokens& t, const uint32_t* keys, int i, int rows, int32_t* flags)
{
    if (keys) return keys[i];
    const int row = row_of(t, i, rows);
    if (row == -2 && flags) flags[FLAG_TOKEN] = 1;
    return row < 0 ? (uint32_t)rows : (uint32_t)row;
}

// counts[digit][part]
__global__ __launch_bounds__(256) void sort_count(Tokens tokens, const uint32_t* keys, int rows, Digit d, int per, int* counts, int32_t* flags)
{
    __shared__ int hist[MOST_BINS];
    const int bins = 1 << d.bits;
    for (int b = threadIdx.x; b < bins; b += 256) hist[b] = 0;
    __syncthreads();
    const long long first = (long long)blockIdx.x * per;
    for (int i = threadIdx.x; i < per && first + i < tokens.n; i += 256)
        atomicAdd(&hist[key_at(tokens, keys, (int)(first + i), rows, flags) >> d.shift & (bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += 256) counts[(long long)b * gridDim.x + blockIdx.x] = hist[b];
}

// One wave per digit: counts in front of each part, and the total.
__global__ __launch_bounds__(64) void sort_sums(int* counts, int parts, int* totals)
{
    int* const c = counts + (long long)blockIdx.x * parts;
    int before = 0;
    for (int base = 0; base < parts; base += 64) {
        const int i = base + (int)threadIdx.x;
        const int own = i < parts ? c[i] : 0;
        int sum = own;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(sum, s);
            if ((int)threadIdx.x >= s) sum += other;
        }
        if (i < parts) c[i] = before + sum - own;
        before += __shfl(sum, 63);
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// Each wave takes a quarter of the part, 64 keys after the other: a key's place is that of its digit, plus what the waves in front and the
// keys in front of it have of the same digit.
__global__ __launch_bounds__(256) void sort_place(Tokens tokens, const uint32_t* keys, const uint32_t* from, int rows, Digit d, int per,
                                                  const int* counts, const int* totals, uint32_t* keys_out, uint32_t* from_out)
{
    __shared__ int at[4][MOST_BINS];
    __shared__ int sums[256];
    const int bins = 1 << d.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < bins; b += 256)
        for (int w = 0; w < 4; ++w) at[w][b] = 0;
    __syncthreads();
    const long long first = (long long)blockIdx.x * per + wave * (per / 4);
    const long long end = min(first + per / 4, (long long)tokens.n);
    for (long long i = first + lane; i < end; i += 64)
        atomicAdd(&at[wave][key_at(tokens, keys, (int)i, rows, nullptr) >> d.shift & (bins - 1)], 1);
    // places of the digits: sums over the totals in front
    const int share = (bins + 255) / 256;
    int own = 0;
    for (int k = 0; k < share; ++k) {
        const int b = threadIdx.x * share + k;
        if (b < bins) own += totals[b];
    }
    sums[threadIdx.x] = own;
    __syncthreads();
    for (int s = 1; s < 256; s <<= 1) {
        const int other = (int)threadIdx.x >= s ? sums[threadIdx.x - s] : 0;
        __syncthreads();
        sums[threadIdx.x] += other;
        __syncthreads();
    }
    int place = sums[threadIdx.x] - own;
    for (int k = 0; k < share; ++k) {
        const int b = threadIdx.x * share + k;
        if (b < bins) {
            int p = place + counts[(long long)b * gridDim.x + blockIdx.x];
            place += totals[b];
            for (int w = 0; w < 4; ++w) {
                const int n = at[w][b];
                at[w][b] = p;
                p += n;
            }
        }
    }
    __syncthreads();
    for (long long base = first; base < end; base += 64) {
        const long long i = base + lane;
        const bool live = i < end;
        const uint32_t key = live ? key_at(tokens, keys, (int)i, rows, nullptr) : 0;
        const uint32_t source = live ? (from ? from[i] : (uint32_t)i) : 0;
        const int digit = (int)(key >> d.shift & (bins - 1));
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
            keys_out[to] = key;
            from_out[to] = source;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------------------------

// Lanes of a wave lie side by side on the columns, VEC each.  The last lane moves back to where it ends with the columns: it then forms
// what its neighbour forms, and stores the same.  A tile of fewer than VEC columns is taken one column per lane.
template <int VEC> struct Cols { float x[VEC]; };

template <int TYPE, int VEC>
__device__ inline Cols<VEC> load_cols(const void* base, long long i)
{
    Cols<VEC> c;
    if constexpr (VEC == 1) {
        c.x[0] = load1<TYPE>(base, i);
    } else if constexpr (VEC == 8 && TYPE != ATOMO_F32) {
        typedef uint16_t eight __attribute__((ext_vector_type(8), aligned(2)));
        const eight s = *(const eight*)((const uint16_t*)base + i);
#pragma unroll
        for (int k = 0; k < 8; ++k) c.x[k] = Element<TYPE>::up(s[k]);
    } else if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
            const f32x4 v = load4<TYPE>(base, i + 4 * q);
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

template <int TYPE, int VEC>
__device__ inline void store_cols(void* base, long long i, const Cols<VEC>& c)
{
    typedef typename Element<TYPE>::Stored Stored;
    if constexpr (VEC == 1) {
        store1<TYPE>(base, i, c.x[0]);
    } else if constexpr (VEC == 8 && TYPE != ATOMO_F32) {
        typedef uint16_t eight __attribute__((ext_vector_type(8), aligned(2)));
        eight s;
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = Element<TYPE>::down(c.x[k]);
        *(eight*)((uint16_t*)base + i) = s;
    } else if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) store4<TYPE>(base, i + 4 * q, f32x4{c.x[4 * q], c.x[4 * q + 1], c.x[4 * q + 2], c.x[4 * q + 3]});
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

// The gradient, and what of it a call writes.
struct Grad {
    void* data;
    long long ld;
    uint32_t rows;
    int cols;
    float scale;
    int accumulate;
};

template <int OUT, int VEC>
__device__ inline void write_sum(const Grad& g, uint32_t row, int col, Cols<VEC> sum)
{
    const long long at = (long long)row * g.ld + col;
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum.x[k] *= g.scale;
    if (g.accumulate) {
        add(sum, load_cols<OUT, VEC>(g.data, at));
        lanes_in_order();                                        // (lanes that overlap have all read before one writes)
    }
    store_cols<OUT, VEC>(g.data, at, sum);
}

// Sums of the runs of equal keys among PIECE sorted tokens, by one wave: runs that lie within the piece are written, the
// others go into `heads` (the run has begun in front of the piece) and `tails` (it begins here and does not end), one row per piece each.
struct Pieces {
    const uint32_t* keys;
    const uint32_t* from;
    int n, length;
    float* heads;
    float* tails;
    long long ld;
};

constexpr int AHEAD = 8;               // rows on their way at a time

template <int IN, int OUT, int VEC>
__device__ void sum_piece(const Pieces& s, int piece, const void* dy, long long ld_dy, int col, bool mine, const Grad& g)
{
    const int lane = threadIdx.x & 63, first = piece * s.length;
    const int here = min(s.length, s.n - first);
    const uint32_t key = lane < here ? s.keys[first + lane] : g.rows;
    const uint32_t from = lane < here ? s.from[first + lane] : 0;
    const int count = __popcll(__ballot(key < g.rows));          // (those of no row stand behind all others)
    if (count == 0) return;
    const bool begun = first > 0 && s.keys[first - 1] == (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
    const uint32_t last = (uint32_t)__builtin_amdgcn_readlane((int)key, count - 1);
    const bool goes_on = count == s.length && first + count < s.n && s.keys[first + count] == last;
    const uint32_t next = (uint32_t)__shfl_down((int)key, 1);
    const uint64_t ends = __ballot(lane < count && (lane == count - 1 || key != next));
    Cols<VEC> sum = {};
    bool in_first = true;
    for (int i = 0; i < count; i += AHEAD) {
        Cols<VEC> x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i + u < count) {
                const long long row = (long long)(uint32_t)__builtin_amdgcn_readlane((int)from, i + u);
                if (mine) x[u] = load_cols<IN, VEC>(dy, row * ld_dy + col);
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
                        else write_sum<OUT, VEC>(g, row, col, sum);
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
            const int mid = (lo + up) / 2;
            if (keys[mid] < row) lo = mid + 1;
            else up = mid;
        }
        named[threadIdx.x] = lo < hi && keys[lo] == row;
    }
    __syncthreads();
    constexpr int VEC = OUT == ATOMO_F32 ? 4 : 8;
    const Cols<VEC> zero = {};
    for (uint32_t r = first + wave; r < end; r += 4) {
        if (named[r - first]) continue;
        for (int col = lane * VEC; col < g.cols; col += 64 * VEC) {
            if (col + VEC <= g.cols) store_cols<OUT, VEC>(g.data, (long long)r * g.ld + col, zero);
            else for (int j = col; j < g.cols; ++j) store1<OUT>(g.data, (long long)r * g.ld + j, 0.0f);
        }
    }
}

// Waves of the first workgroups take a piece and a tile of columns each; the workgroups behind them write the zeros.
template <int IN, int OUT, int VEC>
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
        if (left >= VEC) sum_piece<IN, OUT, VEC>(s, piece, dy, ld_dy, min(first + lane * VEC, g.cols - VEC), lane * VEC < left, g);
        else sum_piece<IN, OUT, 1>(s, piece, dy, ld_dy, first + lane, lane < left, g);
    }
}

// Runs over several pieces: the tail of the piece in which a run begins, and the heads of those behind it up to its end.  A
// workgroup looks after 64 pieces and 256 columns; a wave adds up to SHORT rows by itself, longer runs are shared out among the sixteen.
constexpr int SHORT = 16;

template <int OUT, int VEC>
__device__ void join_tile(const Pieces& s, int pieces, int base, int col, bool mine, const Grad& g)
{
    __shared__ Cols<VEC> part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // this lane's piece: where the run that begins there ends
    const int piece = base + lane;
    int last = 0;
    uint32_t key = g.rows;
    const long long end = (long long)(piece + 1) * s.length;
    if (piece < pieces && end < s.n) {
        key = s.keys[end - 1];
        const bool begins = s.keys[end - s.length] != key || piece == 0 || s.keys[end - s.length - 1] != key;
        if (key < g.rows && begins && s.keys[end] == key) {
            int step = 1;                                        // the last piece whose first key is this one
            last = piece + 1;
            while (last + step < pieces && s.keys[(long long)(last + step) * s.length] == key) {
                last += step;
                step *= 2;
            }
            for (; step > 0; step /= 2)
                if (last + step < pieces && s.keys[(long long)(last + step) * s.length] == key) last += step;
        }
    }
    const uint64_t runs = __ballot(last > 0), longer = __ballot(last - piece > SHORT && last > 0);
    int turn = 0;
    for (uint64_t left = runs & ~longer; left; left &= left - 1, ++turn) {
        const int at = __builtin_ctzll(left);
        const int p = base + at, q = __builtin_amdgcn_readlane(last, at);
        const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, at);
        if (turn % 16 != wave || !mine) continue;
        Cols<VEC> sum = load_cols<ATOMO_F32, VEC>(s.tails, p * s.ld + col);
#pragma unroll 4
        for (int k = p + 1; k <= q; ++k) add(sum, load_cols<ATOMO_F32, VEC>(s.heads, k * s.ld + col));
        write_sum<OUT, VEC>(g, row, col, sum);
    }
    for (uint64_t left = longer; left; left &= left - 1) {
        const int at = __builtin_ctzll(left);
        const int p = base + at, q = __builtin_amdgcn_readlane(last, at), share = (q - p + 15) / 16;
        const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, at);
        const int k0 = p + 1 + wave * share, k1 = min(k0 + share, q + 1);
        Cols<VEC> sum = {};
        if (mine) {
#pragma unroll 8
            for (int k = k0; k < k1; ++k) add(sum, load_cols<ATOMO_F32, VEC>(s.heads, k * s.ld + col));
        }
        part[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && mine) {
            sum = load_cols<ATOMO_F32, VEC>(s.tails, p * s.ld + col);
#pragma unroll
            for (int w = 0; w < 16; ++w) add(sum, part[w][lane]);
            write_sum<OUT, VEC>(g, row, col, sum);
        }
        __syncthreads();
    }
}

template <int OUT>
__global__ __launch_bounds__(1024) void join_pieces(Pieces s, Grad g, int pieces)
{
    const int lane = threadIdx.x & 63;
    for (int tile = blockIdx.y; tile * 256 < g.cols; tile += gridDim.y) {
        const int first = tile * 256, left = g.cols - first;
        if (left >= 4) join_tile<OUT, 4>(s, pieces, (int)blockIdx.x * 64, min(first + lane * 4, g.cols - 4), lane * 4 < left, g);
        else join_tile<OUT, 1>(s, pieces, (int)blockIdx.x * 64, first + lane, lane < left, g);
    }
}

struct Layout {
    uint32_t* keys[2];
    uint32_t* from[2];
    int* counts;
    int* totals;
    int passes, bits, parts, per;
    float* heads;
    float* tails;
    long long ld;                      // of a row of those
    int pieces, length;
    size_t bytes;
};

Layout layout_of(void* base, int64_t n, int64_t rows, int cols)
{
    Layout l = {};
    const int bits = 64 - __builtin_clzll((unsigned long long)rows);             // of keys 0 .. rows
    l.passes = (bits + 9) / 10;
    l.bits = (bits + l.passes - 1) / l.passes;
    l.per = (int)std::max<int64_t>(1024, (n + MOST_PARTS * 256 - 1) / (MOST_PARTS * 256) * 256);
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
    l.totals = c.take<int>((size_t)1 << l.bits);
    l.heads = c.take<float>(l.pieces * l.ld);
    l.tails = c.take<float>(l.pieces * l.ld);
    l.bytes = c.off;
    return l;
}

Tokens tokens_of(const atomo_tokens& t) { return Tokens{t.data, (long long)t.padding, (int)t.n, t.bytes}; }

}  // namespace

size_t embedding_workspace_bytes(int64_t n_tokens, int64_t rows, int32_t cols) { return layout_of(nullptr, n_tokens, rows, cols).bytes; }

int embedding(atomo_ctx* ctx, const atomo_rows& table, const atomo_tokens& tokens, float scale, const atomo_rows& out, hipStream_t stream)
{
    if (tokens.n == 0) return ATOMO_OK;
    int lanes_x = 1;
    while (lanes_x < 256 && lanes_x * 8 < table.cols) lanes_x *= 2;
    const int per = 256 / lanes_x;
    const unsigned grid = (unsigned)std::min<int64_t>(MOST_GROUPS, (tokens.n + per - 1) / per);
    ProfScope ps(ctx, ATOMO_K_EMBEDDING, stream);
    with_type(table.type, [&](auto in) {
        with_type(out.type, [&](auto ty) {
            embedding_rows<in, ty><<<grid, 256, 0, stream>>>(tokens_of(tokens), table.data, table.ld, (int)table.rows, table.cols, scale,
                                                            out.data, out.ld, lanes_x, ctx->d_flags);
        });
    });
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

int embedding_grad(atomo_ctx* ctx, const atomo_tokens& tokens, const atomo_rows& dy, float scale, const atomo_rows& grad,
                   bool accumulate, hipStream_t stream)
{
    if (tokens.n == 0 && accumulate) return ATOMO_OK;
    const int rc = workspace_for_stream(ctx, layout_of(nullptr, tokens.n, grad.rows, grad.cols).bytes, stream);
    if (rc != ATOMO_OK) return rc;
    const Layout l = layout_of(ctx->ws, tokens.n, grad.rows, grad.cols);
    const Tokens t = tokens_of(tokens);
    ProfScope ps(ctx, ATOMO_K_EMBEDDING, stream);
    int at = 0;
    if (tokens.n > 0) {
        for (int p = 0; p < l.passes; ++p) {
            const Digit d = {p * l.bits, l.bits};
            const uint32_t* keys = p ? l.keys[at] : nullptr;
            sort_count<<<l.parts, 256, 0, stream>>>(t, keys, (int)grad.rows, d, l.per, l.counts, ctx->d_flags);
            sort_sums<<<1 << l.bits, 64, 0, stream>>>(l.counts, l.parts, l.totals);
            sort_place<<<l.parts, 256, 0, stream>>>(t, keys, p ? l.from[at] : nullptr, (int)grad.rows, d, l.per, l.counts, l.totals,
                                                    l.keys[1 - at], l.from[1 - at]);
            at = 1 - at;
        }
    }
    const Pieces pieces = {l.keys[at], l.from[at], t.n, l.length, l.heads, l.tails, l.ld};
    const Grad g = {grad.data, (long long)grad.ld, (uint32_t)grad.rows, grad.cols, scale, accumulate ? 1 : 0};
    with_type(dy.type, [&](auto in) {
        with_type(grad.type, [&](auto ty) {
            const auto launch = [&](auto vec) {
                const int tiles = (grad.cols - 1) / (64 * vec) + 1;
                const unsigned groups = (unsigned)std::min<int64_t>(MOST_GROUPS / 2, ((int64_t)l.pieces * tiles + 3) / 4);
                const int64_t row_bytes = (int64_t)grad.cols * type_bytes(grad.type);
                const int zero_per = (int)std::min<int64_t>(ZERO_ROWS, std::max<int64_t>(4, (128 << 10) / row_bytes));
                const unsigned zeros = accumulate ? 0 : (unsigned)std::min<int64_t>(MOST_GROUPS / 2, (grad.rows + zero_per - 1) / zero_per);
                sum_pieces<in, ty, vec><<<groups + zeros, 256, 0, stream>>>(pieces, dy.data, dy.ld, g, l.pieces, tiles, groups, zero_per);
            };
            // few columns: as many lanes as there are, with less each
            constexpr int WIDE = in == ATOMO_F32 ? 4 : 8, NARROW = in == ATOMO_F32 ? 1 : 2;
            if (grad.cols <= 64 * NARROW) launch(std::integral_constant<int, NARROW>());
            else launch(std::integral_constant<int, WIDE>());
        });
    });
    if (l.pieces > 1) {
        const dim3 grid((unsigned)((l.pieces + 63) / 64), (unsigned)std::min(256, (grad.cols - 1) / 256 + 1));
        with_type(grad.type, [&](auto ty) { join_pieces<ty><<<grid, 1024, 0, stream>>>(pieces, g, l.pieces); });
    }
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

}  // namespace atomo
