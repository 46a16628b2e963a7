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

__device__ inline int lower_bound(const uint32_t* keys, int n, uint32_t key)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// A wave per row and 256 columns.
template <int IN, int OUT>
__global__ __launch_bounds__(64) void sum_rows(const uint32_t* keys, const uint32_t* from, int n, const void* dy, long long ld_dy,
                                               uint32_t rows, int cols, float scale, void* grad, long long ld, int accumulate)
{
  for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x)
   for (int col = blockIdx.y * 256 + threadIdx.x * 4; col < cols; col += gridDim.y * 256) {
    const int lo = lower_bound(keys, n, row), hi = lower_bound(keys, n, row + 1);
    if (accumulate && lo == hi) continue;
    if (col + 4 <= cols) {
        f32x4 sum = {0, 0, 0, 0};
        for (int i = lo; i < hi; ++i) sum += load4<IN>(dy, from[i] * ld_dy + col);
        sum *= scale;
        if (accumulate) sum += load4<OUT>(grad, row * ld + col);
        store4<OUT>(grad, row * ld + col, sum);
    } else {
        for (int j = col; j < cols; ++j) {
            float sum = 0.0f;
            for (int i = lo; i < hi; ++i) sum += load1<IN>(dy, from[i] * ld_dy + j);
            sum *= scale;
            if (accumulate) sum += load1<OUT>(grad, row * ld + j);
            store1<OUT>(grad, row * ld + j, sum);
        }
    }
   }
}

struct Layout {
    uint32_t* keys[2];
    uint32_t* from[2];
    int* counts;
    int* totals;
    int passes, bits, parts, per;
    size_t bytes;
};

Layout layout_of(void* base, int64_t n, int64_t rows)
{
    Layout l = {};
    const int bits = 64 - __builtin_clzll((unsigned long long)rows);             // of keys 0 .. rows
    l.passes = (bits + 9) / 10;
    l.bits = (bits + l.passes - 1) / l.passes;
    l.per = (int)std::max<int64_t>(1024, (n + MOST_PARTS * 256 - 1) / (MOST_PARTS * 256) * 256);
    l.parts = (int)((n + l.per - 1) / l.per);
    Carver c(base);
    for (int k = 0; k < 2; ++k) {
        l.keys[k] = c.take<uint32_t>(n);
        l.from[k] = c.take<uint32_t>(n);
    }
    l.counts = c.take<int>((size_t)l.parts << l.bits);
    l.totals = c.take<int>((size_t)1 << l.bits);
    l.bytes = c.off;
    return l;
}

Tokens tokens_of(const atomo_tokens& t) { return Tokens{t.data, (long long)t.padding, (int)t.n, t.bytes}; }

}  // namespace

size_t embedding_workspace_bytes(int64_t n_tokens, int64_t rows, int32_t) { return layout_of(nullptr, n_tokens, rows).bytes; }

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
    const int rc = workspace_for_stream(ctx, layout_of(nullptr, tokens.n, grad.rows).bytes, stream);
    if (rc != ATOMO_OK) return rc;
    const Layout l = layout_of(ctx->ws, tokens.n, grad.rows);
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
    const dim3 grid((unsigned)std::min<int64_t>(MOST_GROUPS, grad.rows), (unsigned)std::min((grad.cols - 1) / 256 + 1, 65535));
    with_type(dy.type, [&](auto in) {
        with_type(grad.type, [&](auto ty) {
            sum_rows<in, ty><<<grid, 64, 0, stream>>>(l.keys[at], l.from[at], t.n, dy.data, dy.ld, (uint32_t)grad.rows, grad.cols, scale, grad.data, grad.ld,
                                                      accumulate ? 1 : 0);
        });
    });
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

}  // namespace atomo
