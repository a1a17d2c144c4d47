// The drafted tokens that the model agrees with: the path through the tree, and its rows of K and V moved
// together behind the cached ones (see reform_tree_accept in reform.h).
//
// One lane per node: a step down the path is a ballot over the nodes that are children of the current one
// and carry the wanted token, so the whole walk is some ten instructions per accepted token.  Every
// workgroup (one per cache stream: layer, sequence, KV head, K or V) walks for itself, which is cheaper than
// a launch that walks once.  The path ascends (a child comes after its parent), so path_m >= m, and rows moved
// in ascending order of m never overwrite one that is still to be read: a pass of the workgroup reads its rows
// into registers, waits for all of its waves, and stores.
//
// Bound: latency (three dependent loads, the walk, one row copy): 12 sequences of 32 nodes, 8 heads of 128 3.8 us.
#include "common.h"

namespace reform {

constexpr int kAcceptThreads = 256;

__global__ __launch_bounds__(kAcceptThreads) void tree_accept(AcceptParams p)
{
    __shared__ int rows[64];
    __shared__ int found;                                // length of the path
    const int lane = threadIdx.x & 63;
    const bool moves = p.k != nullptr;
    const int streams = moves ? 2 * p.n_kv * p.n_layers : 1;
    const int seq = blockIdx.x / streams, stream = blockIdx.x % streams;
    const int len = p.cache_len[seq];
    int nodes = p.n_nodes;
    if (p.node_count) nodes = min(max(p.node_count[seq], 0), p.n_nodes);
    const bool valid = nodes > 0 && len >= 0 && len <= p.capacity - nodes;
    if (threadIdx.x < 64) {
        const size_t at = (size_t)seq * p.n_nodes + min(lane, p.n_nodes - 1);
        const int target = p.target[at];
        int up = -1, token = 0;
        if (lane < nodes) {
            up = p.parent ? p.parent[at] : lane - 1;
            token = p.drafted[at];
        }
        int cur = 0, n = 0;
        if (valid) {
            if (lane == 0) rows[0] = 0;
            for (n = 1; n < nodes; ++n) {                // at most nodes - 1 steps down
                const int want = __builtin_amdgcn_readlane(target, cur);
                const unsigned long long fits = __builtin_amdgcn_ballot_w64(lane > cur && lane < nodes && up == cur && token == want);
                if (fits == 0ull) break;
                cur = __builtin_ctzll(fits);
                if (lane == 0) rows[n] = cur;
            }
        }
        const int following = __builtin_amdgcn_readlane(target, cur);
        if (lane == 0) found = n;
        if (stream == 0 && lane == 0) {
            if (p.accepted) p.accepted[seq] = n;
            if (p.next_token) p.next_token[seq] = valid ? following : -1;
            if (p.new_len) p.new_len[seq] = len + n;
        }
    }
    __syncthreads();
    const int n = found;
    if (stream == 0 && p.path && threadIdx.x < p.n_nodes)
        p.path[(size_t)seq * p.n_nodes + threadIdx.x] = threadIdx.x < n ? rows[threadIdx.x] : -1;
    if (!moves) return;
    const int half = stream & 1, head = (stream >> 1) % p.n_kv, layer = (stream >> 1) / p.n_kv;
    char *base = (char *)(half ? p.v : p.k) + (size_t)layer * p.layer_bytes + (size_t)seq * p.seq_bytes +
                 (size_t)head * p.head_bytes + (size_t)max(len, 0) * p.row_bytes;
    const int per_row = p.row_bytes / 16, total = n * per_row;
    for (int t0 = 0; t0 < total; t0 += 4 * kAcceptThreads) {
        v4u held[4];
        int from[4], to[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + i * kAcceptThreads + (int)threadIdx.x;
            from[i] = to[i] = 0;
            if (t < total) {
                const int m = t / per_row;
                from[i] = rows[m];
                to[i] = m;
                if (from[i] != m) held[i] = *(const v4u *)(base + (size_t)from[i] * p.row_bytes + (t % per_row) * 16);
            }
        }
        __syncthreads();                                 // all rows of the pass are read
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + i * kAcceptThreads + (int)threadIdx.x;
            if (from[i] != to[i]) *(v4u *)(base + (size_t)to[i] * p.row_bytes + (t % per_row) * 16) = held[i];
        }
    }
}

hipError_t tree_accept_launch(const AcceptParams &p, hipStream_t st)
{
    if (p.n_seq == 0) return hipSuccess;
    const unsigned streams = p.k ? 2u * p.n_kv * p.n_layers : 1u;
    hipLaunchKernelGGL(tree_accept, dim3(streams * p.n_seq), dim3(kAcceptThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace reform
