// The operators of include/tessel_block_ops.h: what their kernels are handed, and the launches that the host side calls.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/tessel_block_ops.h"

namespace tessel {

// A tile of an attention launch: `rows` tokens of one sequence that starts at token `begin` and has `length`, tile number `tile`
// of it.  length < 0: -length tokens from `begin` on that belong to no sequence.
struct AttendTile {
    int32_t begin, length, tile, tiles;
};
constexpr int kAttendRows = 128;
constexpr int kAttendThreads = 256, kDkvThreads = 512;   // of a workgroup over queries, over keys
constexpr int kJoinRows = 8;                             // that a workgroup joins of its splits

struct AttendLaunch {
    tessel_attention a;
    const AttendTile *tiles;
    int32_t  num_tiles;
    int32_t  splits;             // workgroups that share a tile's keys (forward, dq) or queries (dk, dv) among them
    int64_t  tokens;
    float   *parts;              // their sums, where there are several: [splits][2 dk, dv][heads][tokens][dim] in 32 bits (one for o, dq)
    float   *tops;               // forward: [splits][heads][tokens][2], a query's largest score and its sum of exponentials
    float   *delta;              // [heads][tokens]
};

int attend_splits(int64_t longest, int64_t total, int resident, double step, double bytes);
int launch_attend(const AttendLaunch &l, void *stream);
int launch_attend_dq(const AttendLaunch &l, void *stream);
int launch_attend_dkv(const AttendLaunch &l, void *stream);

int launch_norm(const tessel_residual_norm &a, void *stream);
int norm_parts(const tessel_residual_norm &a);
int launch_norm_backward(const tessel_residual_norm &a, float *parts, void *stream);

int launch_store(const tessel_checkpoint &c, const tessel_rows &x, void *stream);
int launch_restore(const tessel_checkpoint &c, const tessel_rows &x, void *stream);
int launch_gated(int act, const tessel_rows &g, const tessel_rows &u, const tessel_rows &a, const tessel_checkpoint &kg,
                 const tessel_checkpoint &ku, void *stream);
int launch_gated_backward(int act, const tessel_rows &da, const tessel_checkpoint &kg, const tessel_checkpoint &ku,
                          const tessel_rows &dg, const tessel_rows &du, const tessel_rows &a, void *stream);

constexpr int kWeightThreads = 512;
int64_t weight_tiles(const tessel_weight_grad &a);
int weight_parts(const tessel_weight_grad &a);
int launch_weight_gradient(const tessel_weight_grad &a, float *parts, void *stream);

}  // namespace tessel
