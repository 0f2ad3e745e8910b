// kv_extend.cu -- mp_kv_extend: a step's block table, lengths, positions and slots from the requests' new tokens.
//
// Who gets which block is a matter of prefix sums over the requests: of their rows, of the blocks that done requests give
// back, and of the blocks that the others need.  One CTA takes them (a thread a strip of requests) and writes what there
// is one of for each request; rows (position, slot, and the table's entry where a row opens a block) need no more than
// their request's sums, so in large steps a second kernel has them, a thread a row.
#include <algorithm>

#include "kv_attend.cuh"

namespace mp {
namespace {

constexpr int kThreads = 1024, kRowThreads = 256;
// Rows up to which the first kernel writes them too, a warp a request.
constexpr int64_t kFewRows = 4096;

struct ExtendArgs {
    mp_kv_blocks b;
    mp_kv_extension x;
    int32_t* had;       // [n_seqs] tokens that a request held
    int64_t* before;    // [n_seqs] blocks that the requests before it need
    int64_t* top;       // height of the stack after the pushes
};

__device__ __forceinline__ int blocks_of(int tokens, int block) { return (tokens + block - 1) / block; }

// Sum over the threads before this one; total: over all.
__device__ int64_t scan(int64_t mine, int64_t* smem, int64_t& total) {
    const int lane = threadIdx.x % 32, wid = threadIdx.x / 32;
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    __syncthreads();  // smem's last use
    if (lane == 31) smem[wid] = sum;
    __syncthreads();
    int64_t w = smem[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, w, o);
        if (lane >= o) w += y;
    }
    total = __shfl_sync(~0u, w, 31);
    const int64_t base = __shfl_sync(~0u, w, wid) - __shfl_sync(~0u, sum, 31);
    return base + sum - mine;
}

struct Request {
    int len, n;
    bool sound, done;  // sound: what it asks for can be answered, if there are blocks
};
__device__ __forceinline__ Request request(const ExtendArgs& a, int b) {
    Request r;
    r.len = a.x.lens[b];
    const int n = a.x.n_new[b];
    r.done = n < 0, r.n = max(n, 0);
    r.sound = r.len >= 0 && r.len <= a.x.max_len && r.n <= a.x.max_tokens && (int64_t)r.len + r.n <= a.x.max_len;
    return r;
}
__device__ __forceinline__ int need_of(const ExtendArgs& a, const Request& r) {
    return r.done ? 0 : blocks_of(r.len + r.n, a.b.block_tokens) - blocks_of(r.len, a.b.block_tokens);
}

// Row `row` of a request that got its blocks: its i-th new token.
__device__ __forceinline__ void write_row(const ExtendArgs& a, int b, int len, int64_t before, int64_t top, int i, int64_t row) {
    const int block = a.b.block_tokens, at = len + i, col = at / block, slot = at - col * block;
    const int have = blocks_of(len, block);
    int32_t* const entry = a.b.table + (int64_t)b * a.b.max_blocks + col;
    int page;
    if (a.b.first != nullptr) page = a.b.first[b] + col;
    else if (col < have) page = *entry;
    else page = a.b.free[top - 1 - (before + col - have)];
    if (col >= have && slot == 0) *entry = page;
    a.x.positions[row] = at;
    a.x.slots[row] = (int64_t)page * block + slot;
}
__device__ __forceinline__ void skip_row(const ExtendArgs& a, int64_t row) { a.x.positions[row] = -1, a.x.slots[row] = -1; }

template <bool kRows>
__global__ void __launch_bounds__(kThreads) k_kv_extend(ExtendArgs a) {
    __shared__ int64_t smem[32];
    __shared__ unsigned long long pushed, popped;
    const int tid = threadIdx.x, lane = tid % 32, B = a.b.n_seqs;
    after_previous();
    let_next_begin();
    const bool pool = a.b.first == nullptr;
    const int64_t n_free = pool ? *a.x.n_free : 0;
    const bool stack = n_free >= 0 && n_free <= a.b.n_blocks;  // else no request is answered
    if (tid == 0) pushed = popped = 0;
    const int strip = (B + kThreads - 1) / kThreads;
    // rows, and blocks that come back
    int64_t rows = 0, back = 0, total;
    for (int i = 0; i < strip; ++i) {
        const int b = tid * strip + i;
        if (b >= B) break;
        const Request r = request(a, b);
        rows += r.n;
        if (pool && r.done && r.sound) back += blocks_of(r.len, a.b.block_tokens);
    }
    const int64_t row0 = scan(rows, smem, total);
    if (tid == 0) a.x.token_ptr[B] = total;
    const int64_t back0 = scan(back, smem, total);
    // a request's rows have to be there; done requests push their blocks as long as the stack has room
    int64_t need = 0;
    rows = row0, back = back0;
    for (int i = 0; i < strip; ++i) {
        const int b = tid * strip + i;
        if (b >= B) break;
        const Request r = request(a, b);
        if (pool && r.done && r.sound && stack) {
            back += blocks_of(r.len, a.b.block_tokens);
            if (n_free + back <= a.b.n_blocks) atomicMax(&pushed, (unsigned long long)back);
        }
        rows += r.n;
        if (r.sound && rows <= a.x.n_tokens) need += need_of(a, r);
    }
    const int64_t need0 = scan(need, smem, total);
    __syncthreads();
    const int64_t top = n_free + (int64_t)pushed;
    if (tid == 0) *a.top = top;
    rows = row0, back = back0, need = need0;
    for (int i = 0; i < strip; ++i) {
        const int b = tid * strip + i;
        const unsigned there = __ballot_sync(~0u, b < B);
        if (!there) break;
        Request r = {};
        int status = MP_EINVAL, take = 0;
        int64_t from = back;
        if (b < B) {
            r = request(a, b);
            take = r.sound && rows + r.n <= a.x.n_tokens ? need_of(a, r) : 0;
            a.x.token_ptr[b] = rows;
            a.had[b] = r.len, a.before[b] = need;
            if (r.sound && stack && (r.done || rows + r.n <= a.x.n_tokens)) {
                status = MP_OK;
                if (r.done) {
                    if (pool) {
                        back += blocks_of(r.len, a.b.block_tokens);
                        if (n_free + back > a.b.n_blocks) status = MP_EINVAL;
                    }
                } else if (pool) {
                    if (take > 0) {
                        if (need + take > top) status = MP_ENOMEM;
                        else atomicMax(&popped, (unsigned long long)(need + take));
                    }
                } else {
                    const int blocks = blocks_of(r.len + r.n, a.b.block_tokens);
                    if (a.b.first[b] < 0 || (int64_t)a.b.first[b] + blocks > a.b.n_blocks) status = MP_EINVAL;
                    else if (blocks > a.b.room[b]) status = MP_ENOMEM;
                }
            }
            const bool part = status == MP_OK && !r.done;
            a.x.seq_status[b] = status;
            a.x.step_lens[b] = part ? r.len + r.n : -1;
            a.x.lens_out[b] = status != MP_OK ? r.len : r.done ? 0 : r.len + r.n;
        }
        // the blocks of done requests, a warp a request
        unsigned gone = __ballot_sync(~0u, b < B && pool && r.done && status == MP_OK);
        for (; gone; gone &= gone - 1) {
            const int l = __ffs(gone) - 1;
            const int who = __shfl_sync(~0u, b, l), n = blocks_of(__shfl_sync(~0u, r.len, l), a.b.block_tokens);
            const int64_t to = n_free + __shfl_sync(~0u, from, l);
            for (int j = lane; j < n; j += 32) a.b.free[to + j] = a.b.table[(int64_t)who * a.b.max_blocks + j];
        }
        rows += r.n, need += take;
    }
    __syncthreads();
    if (tid == 0 && pool) *a.x.n_free_out = (int32_t)(stack ? top - (int64_t)popped : n_free);
    if (!kRows) return;
    // rows: a lane those of its request where there are few, else the warp those of one request after another
    rows = row0;
    for (int i = 0; i < strip; ++i) {
        const int b = tid * strip + i;
        if (!__any_sync(~0u, b < B)) break;
        const int n = b < B ? max(a.x.n_new[b], 0) : 0;
        const bool part = b < B && a.x.step_lens[b] >= 0;
        const int len = b < B ? a.had[b] : 0;
        const int64_t before = b < B ? a.before[b] : 0;
        if (!__any_sync(~0u, n > 2)) {
            for (int k = 0; k < n; ++k) {
                if (rows + k >= a.x.n_tokens) break;
                if (part) write_row(a, b, len, before, top, k, rows + k);
                else skip_row(a, rows + k);
            }
        } else {
            for (unsigned left = __ballot_sync(~0u, n > 0); left; left &= left - 1) {
                const int l = __ffs(left) - 1;
                const int who = __shfl_sync(~0u, b, l), many = __shfl_sync(~0u, n, l), held = __shfl_sync(~0u, len, l);
                const int64_t at = __shfl_sync(~0u, rows, l), since = __shfl_sync(~0u, before, l);
                const bool takes = __shfl_sync(~0u, (int)part, l);
                for (int k = lane; k < many && at + k < a.x.n_tokens; k += 32) {
                    if (takes) write_row(a, who, held, since, top, k, at + k);
                    else skip_row(a, at + k);
                }
            }
        }
        rows += n;
    }
}

__global__ void __launch_bounds__(kRowThreads) k_kv_extend_rows(ExtendArgs a) {
    after_previous();
    let_next_begin();
    const int64_t past = min(a.x.n_tokens, a.x.token_ptr[a.b.n_seqs]), top = *a.top;
    for (int64_t row = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; row < past; row += (int64_t)gridDim.x * kRowThreads) {
        int lo = 0, hi = a.b.n_seqs;  // the last request that begins at or before the row
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.x.token_ptr[mid] <= row) lo = mid;
            else hi = mid;
        }
        if (a.x.step_lens[lo] >= 0) write_row(a, lo, a.had[lo], a.before[lo], top, (int)(row - a.x.token_ptr[lo]), row);
        else skip_row(a, row);
    }
}

}  // namespace

size_t kv_extend_workspace_bytes(const mp_kv_blocks& b) {
    return align_up(sizeof(int64_t)) + align_up(sizeof(int64_t) * (size_t)b.n_seqs) + align_up(sizeof(int32_t) * (size_t)b.n_seqs);
}

cudaError_t launch_kv_extend(const mp_kv_blocks& b, const mp_kv_extension& x, void* workspace, cudaStream_t stream) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    ExtendArgs a;
    a.b = b, a.x = x;
    a.top = reinterpret_cast<int64_t*>(ws);
    a.before = reinterpret_cast<int64_t*>(ws + align_up(sizeof(int64_t)));
    a.had = reinterpret_cast<int32_t*>(ws + align_up(sizeof(int64_t)) + align_up(sizeof(int64_t) * (size_t)b.n_seqs));
    if (x.n_tokens <= kFewRows) return launch_close(k_kv_extend<true>, 1, kThreads, 0, stream, a);
    cudaError_t e = launch_close(k_kv_extend<false>, 1, kThreads, 0, stream, a);
    if (e != cudaSuccess) return e;
    const int64_t ctas = std::min<int64_t>((x.n_tokens + kRowThreads - 1) / kRowThreads, kSms * 8);
    return launch_close(k_kv_extend_rows, (int)ctas, kRowThreads, 0, stream, a);
}

}  // namespace mp
