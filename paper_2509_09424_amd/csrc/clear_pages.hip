// Tokens and pages of a cache after a step: the path of drafted tokens that is accepted, its tokens moved together, and sequences forked.
//
// All three are bound by a call's latency or by memory; codes are moved as they are wherever the scale of their block of 16 stays the same.  A call takes the caches of many
// layers, which share lengths and tables.
#include "clear.h"

#define CACHES_PER_LAUNCH 32
struct CacheList {
    KvView kv[CACHES_PER_LAUNCH];  // 56 bytes each, as arguments of a kernel
};

// A wave to a sequence, a lane to a token: from token 0 on, the first later token whose parent is the node and which is what was sampled there.  Every step goes to a later
// token, so it ends.
__global__ __launch_bounds__(256) void k_clear_accept(ensi_clear_accept_args a) {
    const int lane = threadIdx.x % 64, seq = blockIdx.x * 4 + threadIdx.x / 64;
    if (seq >= a.seqs) return;
    const int64_t b0 = a.begin[seq], b1 = a.begin[seq + 1];
    const bool fits = b0 >= 0 && b1 >= b0 && b1 <= a.tokens && b1 - b0 <= a.max_new;
    const int n = fits ? (int)(b1 - b0) : 0;
    int parent = lane - 1, token = -1, sampled = -1;
    if (lane < n) {
        if (a.parents) parent = a.parents[b0 + lane];
        token = a.drafted[b0 + lane];
        sampled = a.sampled[b0 + lane];
    }
    int node = 0, count = 0, mine = -1, following = -1;
    while (count < n) {
        if (lane == count) mine = node;
        count++;
        following = __shfl(sampled, node);
        const u64 fit = __ballot(lane < n && lane > node && parent == node && token == following && following >= 0);
        if (!fit) break;
        node = __ffsll((unsigned long long)fit) - 1;
    }
    if (lane < a.max_new) a.path[seq * a.path_stride + lane] = mine;
    if (lane == 0) {
        a.count[seq] = count;
        a.following[seq] = following;
    }
}

// A wave: one sequence, one head of one cache, keys and values side by side.  Lane j looks after the j-th accepted token.  Blocks of 16 places are filled one after the other, each read
// whole before it is written; tokens only move towards the front, so what a later block needs is not overwritten by then.  A chain of latencies (path, page, scale, codes) decides:
// 64 sequences in 30 caches of 5 heads take 9600 waves, little more than the card holds at once.
template <int ITEMS>
__global__ __launch_bounds__(256) void k_clear_keep(CacheList list, ensi_clear_keep_args a, int caches, int heads) {
    const int lane = threadIdx.x % 64, seq = blockIdx.y;
    const int slot = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64), head = slot % heads;
    if (slot >= caches * heads) return;
    const KvView kv = list.kv[slot / heads];
    if (head >= kv.heads) return;
    const int dim = kv.dim, chunks = dim / 16;
    const SeqPart part = seq_part(a.s, seq, kv.page, 1 << 30, kv.status, lane == 0);  // (a workgroup's waves may have different caches)
    const int count = a.count[seq];
    if (part.count == 0 && count == 0) return;
    int from = lane < min(max(count, 0), a.s.max_new) ? a.path[seq * a.path_stride + lane] : INT32_MAX;
    const int before = __shfl_up(from, 1);
    // ascending, among the new tokens
    const bool wrong = lane < count && (from < 0 || from >= part.count || (lane > 0 && from <= before));
    if (count < 0 || count > part.count || __any(wrong)) {
        if (lane == 0) atomicOr(kv.status, ENSI_KV_BAD_TREE);
        return;
    }
    const u64 moves = __ballot(lane < count && from != lane);
    if (!moves) return;
    const int first = __ffsll((unsigned long long)moves) - 1;  // tokens before it stay where they are
    const auto block_of = [&](int place) -> int64_t {  // of 16 rows; -1: its page is outside the cache
        const int page = a.s.table[seq * a.s.table_stride + place / kv.page];
        if (page < 0 || page >= kv.pages) return -1;
        return (((int64_t)page * kv.heads + head) * kv.page + place % kv.page) / KV_BLOCK;
    };
    // the lane's token: the block that it lies in (a cache has fewer than 2^31) with its scales; and lane b's, the b-th block that tokens come to (5 at most)
    const int block0 = (part.ctx + first) / KV_BLOCK, block1 = (part.ctx + count - 1) / KV_BLOCK;
    int src = 0, dst = 0;
    bool good = true;
    float scale[2] = {0, 0}, was[2] = {0, 0};
    if (lane >= first && lane < count) {
        const int64_t block = block_of(part.ctx + from);
        good = block >= 0;
        if (good) {
            src = (int)block;
            scale[0] = kv.ks[block];
            scale[1] = kv.vs[block];
        }
    }
    if (lane <= block1 - block0) {
        const int64_t block = block_of((block0 + lane) * KV_BLOCK);
        good = good && block >= 0;
        if (block >= 0) {
            dst = (int)block;
            was[0] = kv.ks[block];
            was[1] = kv.vs[block];
        }
    }
    if (!__all(good)) {  // all or nothing
        if (lane == 0) atomicOr(kv.status, ENSI_KV_BAD_PAGE);
        return;
    }
    const int line = (part.ctx + from) % KV_BLOCK;  // of its block
    for (int b = block0; b <= block1; b++) {
        const int start = b * KV_BLOCK, j0 = max(first, start - part.ctx), j1 = min(count, start + KV_BLOCK - part.ctx);  // tokens that arrive in the block
        const int stay = max(0, part.ctx + first - start);                                                               // of its tokens
        const int64_t block = __builtin_amdgcn_readlane(dst, b - block0);
        float old[2], most[2];
#pragma unroll
        for (int c = 0; c < 2; c++) {
            old[c] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, was[c]), b - block0));
            most[c] = lane >= j0 && lane < j1 ? scale[c] : stay > 0 ? old[c] : 0.0f;
#pragma unroll
            for (int k = 1; k < 64; k *= 2) most[c] = fmaxf(most[c], __shfl_xor(most[c], k));
        }
        // chunks of 16 codes: of the tokens that arrive, and of those that stay where their scale grows
        const int arrive = (j1 - j0) * chunks, kept = stay > 0 && (old[0] != most[0] || old[1] != most[1]) ? stay * chunks : 0;
        u32x4 w[2][ITEMS];
        float ratio[2][ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int item = lane + 64 * i, j = (j0 + item / chunks) & 63;
            const int64_t at = __shfl(src, j);
            const int from_line = __shfl(line, j);
            const int64_t row = item < arrive ? at * KV_BLOCK + from_line : block * KV_BLOCK + (item - arrive) / chunks;
            const int64_t byte = row * dim + 16 * ((item < arrive ? item : item - arrive) % chunks);
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const float s = __shfl(scale[c], j), mine = item < arrive ? s : old[c];
                ratio[c][i] = mine == most[c] ? 1.0f : mine / most[c];
                if (item < arrive + kept) w[c][i] = *(const u32x4 *)((c ? kv.v : kv.k) + byte);
            }
        }
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int item = lane + 64 * i;
            const int row = item < arrive ? part.ctx + j0 - start + item / chunks : (item - arrive) / chunks;
            const int64_t byte = (block * KV_BLOCK + row) * dim + 16 * ((item < arrive ? item : item - arrive) % chunks);
#pragma unroll
            for (int c = 0; c < 2; c++) {
                if (ratio[c][i] != 1.0f)
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const u32 u = w[c][i][k];
                        const float f = ratio[c][i];
                        w[c][i][k] = to_e4m3(__builtin_amdgcn_cvt_f32_fp8(u, 0) * f, __builtin_amdgcn_cvt_f32_fp8(u, 1) * f, __builtin_amdgcn_cvt_f32_fp8(u, 2) * f, __builtin_amdgcn_cvt_f32_fp8(u, 3) * f);
                    }
                if (item < arrive + kept) *(u32x4 *)((c ? kv.v : kv.k) + byte) = w[c][i];
            }
        }
        if (lane == 0 && old[0] != most[0]) kv.ks[block] = most[0];
        if (lane == 0 && old[1] != most[1]) kv.vs[block] = most[1];
    }
}

// A workgroup: one row, one head of one cache.  The begun page's blocks in use are copied, 16 bytes to a thread at a time and eight of them under way; one workgroup of a row writes its table.
__global__ __launch_bounds__(256) void k_clear_fork(CacheList list, ensi_clear_fork_args a, int pages, int first) {
    const KvView kv = list.kv[blockIdx.z];
    const int row = blockIdx.y, head = blockIdx.x, t = threadIdx.x;
    if (head >= kv.heads) return;
    const bool writes = first && head == 0 && blockIdx.z == 0;
    const int source = a.source[row], fresh = a.fresh[row];
    int length = 0, error = 0;
    if (source < 0 || source >= a.seqs) error = ENSI_KV_BAD_LENGTH;
    if (!error) {
        length = a.lengths[source];
        if (length < 0 || length > (int64_t)a.table_width * kv.page) error = ENSI_KV_BAD_LENGTH;
    }
    const int full = error ? 0 : length / kv.page, rest = error ? 0 : length % kv.page;
    int begun = -1;
    if (!error && rest) {
        begun = a.table[source * a.table_stride + full];
        if (begun < 0 || begun >= pages || fresh < 0 || fresh >= pages) error = ENSI_KV_BAD_PAGE;
    }
    if (!error && fresh >= pages) error = ENSI_KV_BAD_PAGE;
    // a page that an earlier row has been given
    bool twice = false;
    if (fresh >= 0)
        for (int i = t; i < row; i += 256) twice |= a.fresh[i] == fresh;
    if (__syncthreads_or(twice) && !error) error = ENSI_KV_BAD_PAGE;
    if (error && t == 0) atomicOr(kv.status, error);
    if (writes) {
        for (int i = t; i < a.table_width; i += 256) a.table_out[row * a.out_stride + i] = error ? -1 : i < full ? a.table[source * a.table_stride + i] : i == full ? max(fresh, -1) : -1;
        if (t == 0) a.lengths_out[row] = error ? 0 : length;
    }
    if (error || !rest || begun == fresh) return;
    const int blocks = (rest + KV_BLOCK - 1) / KV_BLOCK, chunks = blocks * kv.dim;  // of 16 bytes, in keys and in values
    const int64_t from = ((int64_t)begun * kv.heads + head) * kv.page, to = ((int64_t)fresh * kv.heads + head) * kv.page;
    const u32x4 *k_from = (const u32x4 *)(kv.k + from * kv.dim), *v_from = (const u32x4 *)(kv.v + from * kv.dim);
    u32x4 *k_to = (u32x4 *)(kv.k + to * kv.dim), *v_to = (u32x4 *)(kv.v + to * kv.dim);
    constexpr int AHEAD = 4;
    for (int i = t; i < chunks; i += 256 * AHEAD) {
        u32x4 k[AHEAD], v[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; e++)
            if (i + 256 * e < chunks) {
                k[e] = k_from[i + 256 * e];
                v[e] = v_from[i + 256 * e];
            }
#pragma unroll
        for (int e = 0; e < AHEAD; e++)
            if (i + 256 * e < chunks) {
                k_to[i + 256 * e] = k[e];
                v_to[i + 256 * e] = v[e];
            }
    }
    for (int i = t; i < blocks; i += 256) {
        kv.ks[to / KV_BLOCK + i] = kv.ks[from / KV_BLOCK + i];
        kv.vs[to / KV_BLOCK + i] = kv.vs[from / KV_BLOCK + i];
    }
}

void launch_clear_accept(ensi_ctx *ctx, const ensi_clear_accept_args &a, hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_accept", st);
    hipLaunchKernelGGL(k_clear_accept, dim3((a.seqs + 3) / 4), dim3(256), 0, st, a);
}

// `go` for every group of caches that a kernel's arguments hold
template <class GO>
static void for_caches(const ensi_kv *const *kv, int caches, const GO &go) {
    for (int at = 0; at < caches; at += CACHES_PER_LAUNCH) {
        CacheList list;
        const int n = min(caches - at, CACHES_PER_LAUNCH);
        int heads = 0, dim = 0;
        for (int i = 0; i < CACHES_PER_LAUNCH; i++) {
            list.kv[i] = kv[at + (i < n ? i : 0)]->view;
            heads = max(heads, list.kv[i].heads);
            dim = max(dim, list.kv[i].dim);
        }
        go(list, n, heads, dim, at == 0);
    }
}

void launch_clear_keep(ensi_ctx *ctx, const ensi_kv *const *kv, int caches, const ensi_clear_keep_args &a, hipStream_t st) {
    for_caches(kv, caches, [&](const CacheList &list, int n, int heads, int dim, bool) {
        ScopedTimer timer(ctx, "k_clear_keep", st);
        const dim3 grid((n * heads + 3) / 4, a.s.seqs);
        // 16 rows of a block, moved or rounded again, dim / 16 chunks each
        if (dim <= 64) hipLaunchKernelGGL(k_clear_keep<1>, grid, dim3(256), 0, st, list, a, n, heads);
        else if (dim <= 128) hipLaunchKernelGGL(k_clear_keep<2>, grid, dim3(256), 0, st, list, a, n, heads);
        else hipLaunchKernelGGL(k_clear_keep<4>, grid, dim3(256), 0, st, list, a, n, heads);
    });
}

void launch_clear_fork(ensi_ctx *ctx, const ensi_kv *const *kv, int caches, const ensi_clear_fork_args &a, hipStream_t st) {
    int pages = INT32_MAX;
    for (int i = 0; i < caches; i++) pages = min(pages, kv[i]->view.pages);
    for_caches(kv, caches, [&](const CacheList &list, int n, int heads, int, bool first) {
        ScopedTimer timer(ctx, "k_clear_fork", st);
        hipLaunchKernelGGL(k_clear_fork, dim3(heads, a.rows, n), dim3(256), 0, st, list, a, pages, first ? 1 : 0);
    });
}
