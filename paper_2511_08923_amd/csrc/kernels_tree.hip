// A tree of drafted tokens: positions and ancestors from the parents, and the path that verification accepts.
//
// Sequence b's tree is rows [row_start[b], row_start[b + 1]) of the packed arrays, at most 256; a row's parent is the index, within
// the tree, of a row that comes before it, or -1.  Both kernels take a workgroup per sequence and a tree in LDS; they are bound by
// their launch and by dependent steps: a trip to memory for row_start, one for the rows, then LDS (one tree of 16 rows 3.1 and 2.9 us, 64 trees of
// up to 64 rows 4.7 and 4.2).
#include "span_device.h"

namespace {

// Rows of sequence b that lie within the arrays, whatever row_start says.
__device__ inline void rows_within(const int32_t *row_start, int n_rows, int b, int &s, int &e) {
    s = min(max(row_start[b], 0), n_rows);
    e = min(max(row_start[b + 1], s), n_rows);
}

// The end of the rows from s on that no sequence but b has a range of (s itself, where one has): asked by a whole workgroup.
__device__ inline int end_of_free(const int32_t *row_start, int n_rows, int b, int s, int e) {
    __shared__ int end;
    if (threadIdx.x == 0) end = e;
    __syncthreads();
    const int B = gridDim.x;
    for (int x = threadIdx.x; x < B; x += 256) {
        int s1;
        const int m = tree_range(row_start, n_rows, TIDAR_MAX_TREE, x, s1);
        if (x != b && m > 0 && s1 + m > s) atomicMin(&end, max(s1, s));
    }
    __syncthreads();
    return end;
}

// A row's bits are its own and its parent's.  Every row starts with its own bit and its parent as the row to look up next; each
// step adds that row's bits and goes on to the row that that one would look up, which is twice as far: eight steps for 256.
__global__ __launch_bounds__(256) void tree_plan_kernel(const int32_t *__restrict__ prefix_len, const int32_t *__restrict__ row_start,
                                                        int n_rows, const int32_t *__restrict__ parent, int32_t *__restrict__ pos,
                                                        uint32_t *__restrict__ ancestors) {
    __shared__ uint32_t bits[TIDAR_MAX_TREE][kTreeWords + 1];
    __shared__ int up[TIDAR_MAX_TREE];
    const int b = blockIdx.x, i = threadIdx.x, L = prefix_len[b];
    int s, e;
    rows_within(row_start, n_rows, b, s, e);
    const int n = e - s;
    const bool here = i < n, taken = tree_taken(row_start, n_rows, TIDAR_MAX_TREE, b, s, n, i & 63, 64);
    const bool mine = row_start[b] == s && row_start[b + 1] == e && n <= TIDAR_MAX_TREE && !taken;       // (the same in all threads)
    bool bad = !mine || L < 0 || L > (1 << 30);
    int p = -1;
    if (!bad && here) {
        p = parent[s + i];
        bad = p < -1 || p >= i;
    }
    if (__syncthreads_or(bad)) {
        if (!mine) e = end_of_free(row_start, n_rows, b, s, e);          // (other workgroups write the others' rows)
        for (int r = s + i; r < e; r += 256) pos[r] = -1;
        for (size_t w = (size_t)s * kTreeWords + i; w < (size_t)e * kTreeWords; w += 256) ancestors[w] = 0;
        return;
    }
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) bits[i][w] = (i >> 5) == w ? 1u << (i & 31) : 0u;
    up[i] = p;
    while (__syncthreads_or(p >= 0)) {
        uint32_t x[kTreeWords] = {};
        int next = -1;
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < kTreeWords; ++w) x[w] = bits[p][w];
            next = up[p];
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) bits[i][w] |= x[w];
        up[i] = p = next;
    }
    if (!here) return;
    int depth = -1;
    u32x4 lo, hi;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) {
        const uint32_t x = bits[i][w];
        depth += __popc(x);
        (w < 4 ? lo : hi)[w & 3] = x;
    }
    pos[s + i] = L + depth;
    u32x4 *dst = (u32x4 *)(ancestors + (size_t)(s + i) * kTreeWords);
    dst[0] = lo;
    dst[1] = hi;
}

struct AcceptArgs {
    const int32_t *prefix_len, *row_start, *parent, *tokens, *choice, *page_table;
    int n_rows, vocab, pages_per_seq, n_pages, max_path;
    int32_t *new_len, *accepted_len, *accepted_rows, *accepted_tokens, *next_token;
};

// Every row that was drafted as its parent's choice offers itself to the parent, the lowest wins; the path is then followed from row
// 0, one LDS read a token.
__global__ __launch_bounds__(256) void tree_accept_kernel(AcceptArgs a) {
    __shared__ int child[TIDAR_MAX_TREE], token[TIDAR_MAX_TREE], said[TIDAR_MAX_TREE], path[TIDAR_MAX_TREE];
    const int b = blockIdx.x, i = threadIdx.x, L = a.prefix_len[b];
    int s, e;
    rows_within(a.row_start, a.n_rows, b, s, e);
    const int n = e - s;
    const bool here = i < n;
    bool bad = a.row_start[b] != s || a.row_start[b + 1] != e || n < 1 || n > TIDAR_MAX_TREE || L < 0;
    bad = tree_taken(a.row_start, a.n_rows, TIDAR_MAX_TREE, b, s, n, i, 256) || bad;        // (a wave's share of them: the workgroup asks together below)
    int p = -1;
    child[i] = TIDAR_MAX_TREE;
    if (!bad && here) {
        p = a.parent[s + i];
        token[i] = a.tokens[s + i];
        said[i] = a.choice[s + i];
        bad = p < -1 || p >= i;
    }
    if (!__syncthreads_or(bad)) {
        if (p >= 0 && token[i] == said[p]) atomicMin(&child[p], i);
        __syncthreads();
        int len = 0, at = 0, next = -1;
        bool ok = (unsigned)token[0] < (unsigned)a.vocab;
        for (int cur = 0; cur < TIDAR_MAX_TREE && len < a.max_path; cur = child[cur]) {      // (every thread; no row twice: children come later)
            next = said[cur];
            ok = ok && (unsigned)next < (unsigned)a.vocab;
            at = cur;
            if (i == 0) path[len] = at;
            ++len;
        }
        if (ok && (long long)L + len > (long long)a.pages_per_seq * 16) ok = false;
        if (ok) {                                        // the pages that the path goes into, at most 17
            const int u = (L >> 4) + i;
            const bool odd = u <= (L + len - 1) >> 4 && (unsigned)a.page_table[(size_t)b * a.pages_per_seq + u] >= (unsigned)a.n_pages;
            ok = !__syncthreads_or(odd);
        }
        if (ok) {
            __syncthreads();
            for (int j = i; j < a.max_path; j += 256) {
                a.accepted_rows[(size_t)b * a.max_path + j] = j < len ? path[j] : -1;
                a.accepted_tokens[(size_t)b * a.max_path + j] = j < len ? token[path[j]] : -1;
            }
            if (i == 0) {
                a.new_len[b] = L + len;
                a.accepted_len[b] = len;
                a.next_token[b] = next;
            }
            return;
        }
    }
    for (int j = i; j < a.max_path; j += 256) {
        a.accepted_rows[(size_t)b * a.max_path + j] = -1;
        a.accepted_tokens[(size_t)b * a.max_path + j] = -1;
    }
    if (i == 0) {
        a.new_len[b] = L;
        a.accepted_len[b] = 0;
        a.next_token[b] = -1;
    }
}

}  // namespace

void launch_tree_plan(int batch, const int32_t *prefix_len, const int32_t *row_start, int n_rows, const int32_t *parent,
                      int32_t *pos, uint32_t *ancestors, hipStream_t st) {
    tree_plan_kernel<<<batch, 256, 0, st>>>(prefix_len, row_start, n_rows, parent, pos, ancestors);
}

void launch_tree_accept(int batch, const int32_t *prefix_len, const int32_t *row_start, int n_rows, const int32_t *parent,
                        const int32_t *tokens, const int32_t *choice, int vocab, const int32_t *page_table, int pages_per_seq,
                        int n_pages, int max_path, int32_t *new_len, int32_t *accepted_len, int32_t *accepted_rows,
                        int32_t *accepted_tokens, int32_t *next_token, hipStream_t st) {
    const AcceptArgs a = {prefix_len, row_start, parent, tokens, choice, page_table, n_rows, vocab, pages_per_seq, n_pages, max_path,
                          new_len, accepted_len, accepted_rows, accepted_tokens, next_token};
    tree_accept_kernel<<<batch, 256, 0, st>>>(a);
}
