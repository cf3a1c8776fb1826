// Scales of groups of consecutive weights of a row: S = root mean square of the group, Z = W / S, and what goes with them.
//   scale             S[r, g] = sqrt(sum W^2 / count),  Z = W / S  (0 where S = 0)
//   unscale           Wq = S Zq
//   unscale backward  dZq = S dWq,  dS = sum over the group of dWq Zq
//   scale backward    dW = dZ / S + Z / count (dS - sum over the group of dZ Z / S)   (0 where S = 0)
// Bound by memory: every weight is read once and written once.  LPG lanes take a group and hold it in registers between the
// sum and the result (up to NV pieces of VEC weights a lane; NV = 0: longer groups are read again, from the cache).  Sums are
// float64: squares of float32 cannot overflow in it, and the order of the lanes does not show in the result's 24 bits.
// 4096 x 4096 in groups of 128: scale 25.5 us (5.3 TB/s), unscale 24.5 (5.5), unscale backward 33 (6.2), scale backward 39 (5.3), where a large
// copy reaches 5.2.  At 1000 x 512 each takes 3 to 4 us, and what bounds a call is its launch.
#include "layers.h"

namespace idkm {

template <int OP, int VEC, int LPG, int NV>
__global__ __launch_bounds__(256) void k_group_scale(const ScaleArgs a) {
    struct alignas(4 * VEC) Piece { float v[VEC]; };
    const int lane = threadIdx.x & (LPG - 1);
    const int64_t units = a.rows * a.groups;
    const int64_t step = (int64_t)gridDim.x * (256 / LPG);
    // every lane of a wavefront goes round equally often, so that all take part in the exchanges
    const int64_t rounds = (units + step - 1) / step;
    int64_t u = (int64_t)blockIdx.x * (256 / LPG) + threadIdx.x / LPG;
    for (int64_t round = 0; round < rounds; ++round, u += step) {
        const bool there = u < units;
        const int64_t r = there ? u / a.groups : 0, g = there ? u - r * a.groups : 0;
        const int64_t c0 = g * a.group;
        const int count = there ? (int)min(a.group, a.cols - c0) : 0;
        const int64_t at = r * a.cols + c0;
        const int pieces = count / VEC;  // VEC = 4 only where it divides
        float s = 0.f, ds = 0.f;
        if (OP != SCALE_FWD && there) s = a.S[u];
        if (OP == SCALE_BWD && there && a.dS) ds = a.dS[u];
        double sum = 0.0;
        // x, y of one piece: SCALE_FWD W; UNSCALE_FWD Zq; UNSCALE_BWD dWq, Zq; SCALE_BWD dZ, Z
        constexpr bool TWO = OP == UNSCALE_BWD || OP == SCALE_BWD;
        constexpr int HELD = NV > 0 ? NV : 1;
        Piece x[HELD], y[HELD];
        auto load = [&](int i, Piece& px, Piece& py) {
            px = *reinterpret_cast<const Piece*>(a.x + at + (int64_t)i * VEC);
            if (TWO) py = *reinterpret_cast<const Piece*>(a.y + at + (int64_t)i * VEC);
        };
        auto add = [&](const Piece& px, const Piece& py) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += (double)px.v[e] * (double)(TWO ? py.v[e] : px.v[e]);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int h = 0; h < NV; ++h)
                if (h * LPG + lane < pieces) load(h * LPG + lane, x[h], y[h]);
#pragma unroll
            for (int h = 0; h < NV; ++h)
                if (OP != UNSCALE_FWD && h * LPG + lane < pieces) add(x[h], y[h]);
        } else if (OP != UNSCALE_FWD) {
            for (int i = lane; i < pieces; i += LPG) {
                load(i, x[0], y[0]);
                add(x[0], y[0]);
            }
        }
        if (OP != UNSCALE_FWD) {
#pragma unroll
            for (int o = LPG / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, LPG);
        }
        float inner = 0.f;
        if (OP == SCALE_FWD) {
            s = (float)sqrt(sum / (double)count);
            if (there && lane == 0) a.s_out[u] = s;
        } else if (OP == UNSCALE_BWD) {
            if (there && lane == 0) a.s_out[u] = (float)sum;
        } else if (OP == SCALE_BWD) {
            inner = (float)(((double)ds - sum / (double)s) / (double)count);
        }
        const bool none = s == 0.f;
        auto store = [&](int i, const Piece& px, const Piece& py) {
            Piece o;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (OP == SCALE_FWD) o.v[e] = none ? 0.f : px.v[e] / s;
                if (OP == UNSCALE_FWD || OP == UNSCALE_BWD) o.v[e] = s * px.v[e];
                if (OP == SCALE_BWD) o.v[e] = none ? 0.f : px.v[e] / s + py.v[e] * inner;
            }
            *reinterpret_cast<Piece*>(a.out + at + (int64_t)i * VEC) = o;
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int h = 0; h < NV; ++h)
                if (h * LPG + lane < pieces) store(h * LPG + lane, x[h], y[h]);
        } else {
            for (int i = lane; i < pieces; i += LPG) {
                load(i, x[0], y[0]);
                store(i, x[0], y[0]);
            }
        }
    }
}

template <int OP, int VEC, int LPG, int NV>
static void launch(const ScaleArgs& a, hipStream_t s) {
    const int64_t wg = (a.rows * a.groups + 256 / LPG - 1) / (256 / LPG);
    hipLaunchKernelGGL((k_group_scale<OP, VEC, LPG, NV>), dim3((unsigned)(wg < 8192 ? wg : 8192)), dim3(256), 0, s, a);
}

template <int OP, int VEC>
static void launch_for_group(const ScaleArgs& a, hipStream_t s) {
    const int64_t pieces = a.group / VEC + (a.group % VEC != 0);
    if (pieces <= 8) launch<OP, VEC, 8, 1>(a, s);
    else if (pieces <= 16) launch<OP, VEC, 16, 1>(a, s);
    else if (pieces <= 32) launch<OP, VEC, 32, 1>(a, s);
    else if (pieces <= 64) launch<OP, VEC, 64, 1>(a, s);
    else if (pieces <= 256) launch<OP, VEC, 64, 4>(a, s);
    else launch<OP, VEC, 64, 0>(a, s);
}

template <int OP>
static void launch_op(const ScaleArgs& a, hipStream_t s) {
    const uintptr_t any = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.out);
    if (a.cols % 4 == 0 && a.group % 4 == 0 && any % 16 == 0) launch_for_group<OP, 4>(a, s);
    else launch_for_group<OP, 1>(a, s);
}

void launch_group_scale(int op, const ScaleArgs& a, hipStream_t s) {
    switch (op) {
        case SCALE_FWD: launch_op<SCALE_FWD>(a, s); break;
        case UNSCALE_FWD: launch_op<UNSCALE_FWD>(a, s); break;
        case UNSCALE_BWD: launch_op<UNSCALE_BWD>(a, s); break;
        default: launch_op<SCALE_BWD>(a, s); break;
    }
}

}  // namespace idkm
