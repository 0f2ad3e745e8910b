// kv_extend.cu -- mp_kv_extend: a step's block table, lengths, positions and slots from the requests' new tokens.
//
// Who gets which block is a matter of prefix sums over the requests: of their rows, of the blocks that done requests give
// back, and of the blocks that the others need.  One CTA takes them (a thread a strip of requests) and writes what there
// is one of for each request; rows (position, slot, and the table's entry where a row opens a block) need no more than
// their request's sums, so in large steps a second kernel has them, a thread a row.
//
// Measured (GPU time): 64 requests with a token each 6 us, 509 requests of which 484 get 125,000 tokens and 25 end 14 us: trips to
// memory one after another (lengths, the ended requests' table rows, then sums, tables and stacks for the rows).
#include <algorithm>

#include "kv_attend.cuh"

namespace mp {
namespace {

constexpr int kThreads = 1024, kRowThreads = 256;
// Rows up to which the first kernel writes them too, a warp a request; the second launch costs 2 us.
constexpr int64_t kFewRows = 4096;

struct ExtendArgs {
    mp_kv_blocks b;
    mp_kv_extension x;
    int32_t* had;       // [n_seqs] tokens that a request held
    int64_t* before;    // [n_seqs] blocks that the requests before it need
    int64_t* top;       // height of the stack after the pushes
};

__device__ __forceinline__ int blocks_of(int tokens, int block) { return (tokens + block - 1) / block; }

// Rows, and blocks that come back and are needed.
struct Sums {
    int64_t rows, back, need;
    __device__ __forceinline__ void add(const Sums& x) { rows += x.rows, back += x.back, need += x.need; }
};
__device__ __forceinline__ Sums shuffled(const Sums& x, int lane) {
    return {__shfl_sync(~0u, x.rows, lane), __shfl_sync(~0u, x.back, lane), __shfl_sync(~0u, x.need, lane)};
}
__device__ __forceinline__ Sums scan_warp(Sums x) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums y = {__shfl_up_sync(~0u, x.rows, o), __shfl_up_sync(~0u, x.back, o), __shfl_up_sync(~0u, x.need, o)};
        if (lane >= o) x.add(y);
    }
    return x;
}
// Sums over the threads before this one; total: over all.
__device__ Sums scan(const Sums& mine, Sums* smem, Sums& total) {
    const int lane = threadIdx.x % 32, wid = threadIdx.x / 32;
    const Sums x = scan_warp(mine);
    __syncthreads();  // smem's last use
    if (lane == 31) smem[wid] = x;
    __syncthreads();
    const Sums w = scan_warp(smem[lane]);
    total = shuffled(w, 31);
    Sums base = shuffled(w, wid);
    const Sums last = shuffled(x, 31);
    return {base.rows - last.rows + x.rows - mine.rows, base.back - last.back + x.back - mine.back,
            base.need - last.need + x.need - mine.need};
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
    // one that ends may have held more than the others may
    const int64_t most = r.done ? min((int64_t)a.b.max_blocks * a.b.block_tokens, (int64_t)1 << 28) : a.x.max_len;
    r.sound = r.len >= 0 && r.n <= a.x.max_tokens && (int64_t)r.len + r.n <= most;
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

// Blocks of a request that ends, and where on the stack they go; a warp pushes them.
struct Ended {
    int32_t b, blocks, to;
};
__device__ __forceinline__ void push(const ExtendArgs& a, const Ended& e) {
#pragma unroll 4
    for (int j = threadIdx.x % 32; j < e.blocks; j += 32) a.b.free[e.to + j] = a.b.table[(int64_t)e.b * a.b.max_blocks + j];
}

template <bool kRows>
__global__ void __launch_bounds__(kThreads) k_kv_extend(ExtendArgs a) {
    __shared__ Sums smem[32];
    __shared__ unsigned long long pushed, popped;
    __shared__ Ended ended[kThreads];
    __shared__ int n_ended;
    const int tid = threadIdx.x, lane = tid % 32, B = a.b.n_seqs;
    after_previous();
    let_next_begin();
    const int strip = (B + kThreads - 1) / kThreads;
    Request held = {};
    if (strip == 1 && tid < B) held = request(a, tid);  // read once where a thread has one request
    auto of = [&](int b) { return strip == 1 ? held : request(a, b); };
    const bool pool = a.b.first == nullptr;
    const int64_t n_free = pool ? *a.x.n_free : 0;
    const bool stack = n_free >= 0 && n_free <= a.b.n_blocks;  // else no request is answered
    // what a request adds, if its rows are there
    auto sums_of = [&](const Request& r) {
        Sums x = {r.n, 0, 0};
        if (pool && stack && r.done && r.sound) x.back = blocks_of(r.len, a.b.block_tokens);
        if (r.sound) x.need = need_of(a, r);
        return x;
    };
    Sums mine = {}, total;
    for (int b = tid * strip; b < min((tid + 1) * strip, B); ++b) mine.add(sums_of(of(b)));
    Sums from0 = scan(mine, smem, total);
    if (tid == 0) a.x.token_ptr[B] = total.rows;
    if (total.rows > a.x.n_tokens) {  // requests whose rows are not there need nothing
        mine = {};
        int64_t rows = from0.rows;
        for (int b = tid * strip; b < min((tid + 1) * strip, B); ++b) {
            const Request r = of(b);
            rows += r.n;
            if (rows <= a.x.n_tokens) mine.need += sums_of(r).need;
        }
        Sums needs;
        from0.need = scan(mine, smem, needs).need, total.need = needs.need;
    }
    // done requests push their blocks as long as the stack has room for them
    if (tid == 0) pushed = n_free + total.back <= a.b.n_blocks ? total.back : 0, popped = 0, n_ended = 0;
    __syncthreads();
    if (n_free + total.back > a.b.n_blocks) {
        int64_t back = from0.back;
        for (int b = tid * strip; b < min((tid + 1) * strip, B); ++b) {
            back += sums_of(of(b)).back;
            if (n_free + back <= a.b.n_blocks) atomicMax(&pushed, (unsigned long long)back);
        }
        __syncthreads();
    }
    const int64_t top = n_free + (int64_t)pushed;
    const bool enough = total.need <= top;
    if (tid == 0) {
        *a.top = top;
        if (enough) popped = total.need;
    }
    int64_t rows = from0.rows, back = from0.back, need = from0.need;
    for (int i = 0; i < strip; ++i) {
        const int b = tid * strip + i;
        const unsigned there = __ballot_sync(~0u, b < B);
        if (!there) break;
        Request r = {};
        int status = MP_EINVAL, take = 0;
        int64_t from = back;
        if (b < B) {
            r = of(b);
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
                        else if (!enough) atomicMax(&popped, (unsigned long long)(need + take));
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
        // the blocks of done requests, a warp a request: all at once where a thread has one request
        const bool gone = b < B && pool && r.done && status == MP_OK && r.len > 0;
        if (strip == 1) {
            if (gone) ended[atomicAdd(&n_ended, 1)] = {b, blocks_of(r.len, a.b.block_tokens), (int32_t)(n_free + from)};
        } else {
            for (unsigned left = __ballot_sync(~0u, gone); left; left &= left - 1) {
                const int l = __ffs(left) - 1;
                push(a, {__shfl_sync(~0u, b, l), blocks_of(__shfl_sync(~0u, r.len, l), a.b.block_tokens),
                         (int32_t)(n_free + __shfl_sync(~0u, from, l))});
            }
        }
        rows += r.n, need += take;
    }
    if (strip == 1) {
        __syncthreads();
        for (int i = tid / 32; i < n_ended; i += kThreads / 32) push(a, ended[i]);
    }
    __syncthreads();
    if (tid == 0 && pool) *a.x.n_free_out = (int32_t)(stack ? top - (int64_t)popped : n_free);
    if (!kRows) return;
    // rows: a lane those of its request where there are few, else the warp those of one request after another
    rows = from0.rows;
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

// The last request that begins at or before the row; the lanes of a warp have rows in a row.  A search among 32 requests a
// step finds the first lane's; the others' are mostly among the 32 after it.
__device__ __forceinline__ int request_of(const ExtendArgs& a, int64_t row, int64_t past) {
    const int lane = threadIdx.x % 32, B = a.b.n_seqs;
    const int64_t* const ptr = a.x.token_ptr;
    int lo = 0, span = B;  // among lo, ..., lo + span - 1
    if (row - lane + 31 < past) {  // every lane has one
        const int64_t first = __shfl_sync(~0u, row, 0);
        while (span > 1) {
            const int step = (span + 31) / 32, at = lo + lane * step;
            const int before = __popc(__ballot_sync(~0u, at < lo + span && ptr[min(at, B - 1)] <= first));
            const int next = lo + (before - 1) * step;
            span = min(step, lo + span - next), lo = next;
        }
        const int64_t begins = ptr[min(lo + 1 + lane, B)];  // of the 32 after it
        if (lo + 33 > B || __shfl_sync(~0u, begins, 31) > __shfl_sync(~0u, row, 31)) {
            int more = 0;  // how many of them begin at or before the row
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const int64_t x = __shfl_sync(~0u, begins, more + o - 1);
                if (lo + more + o < B && x <= row) more += o;
            }
            return lo + more;
        }
        span = B - lo;
    }
    while (span > 1) {
        const int half = span / 2;
        if (ptr[lo + half] <= row) lo += half, span -= half;
        else span = half;
    }
    return lo;
}

__global__ void __launch_bounds__(kRowThreads) k_kv_extend_rows(ExtendArgs a) {
    after_previous();
    let_next_begin();
    const int64_t past = min(a.x.n_tokens, a.x.token_ptr[a.b.n_seqs]), top = *a.top;
    for (int64_t row = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; row < past; row += (int64_t)gridDim.x * kRowThreads) {
        const int lo = request_of(a, row, past);
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
