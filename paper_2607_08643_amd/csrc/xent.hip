// Softmax cross entropy of a large vocabulary from hidden states H [T][D] and
// head weights V [N][D], and its gradient, without keeping the T x N logits:
//   z = H V^T,  lse = log sum exp(z),  loss = lse - z_target,
//   d = g (exp(z - lse) - onehot),  dH = d V,  dV = d^T H.
//
// loss: one matrix product whose tiles are reduced where they are made: per
// token and tile the largest logit and the sum of exponentials against it, and
// the target's logit; a second launch joins a token's tiles. 2 T N D
// operations, D-deep; V is read once.
//
// gradient: the vocabulary in pieces of `vp` words. Per piece the logits are
// made again and leave the tile as d in bf16 (the workspace holds one piece; for
// a dV of 32 bits in two bf16 parts, which its product takes one after the other);
// two further products read them: dV's rows of the piece, and the piece's
// contribution to dH, added in fp32 over the pieces in order.
//
// Bound by the matrix cores from some hundred tokens on: 4096 tokens of 151936
// words, 4096 inputs: logits 4.5 ms (1.14 PFLOP/s), dH 3.9 (1.31), dV 4.5 (1.13; the
// whole gradient 12.8, with a dV of 32 bits 17.7); the loss alone of 2000 tokens 2.25
// ms a pass (1.11; 2.37 in a profiled run). One token's loss is one reading of V: 247
// us, 5.0 TB/s.
//
// Tokens without a loss are taken out first: the rows that have one are copied
// next to each other (padded with zeros to whole tiles and to a multiple of
// 64 inputs), and every product runs over those alone.
#include "vocab_product.h"

namespace bsq {
namespace {

// A token's tiles joined: TOK tokens a block, XT / TOK threads each over the
// tiles, their pairs then joined in order. (One block of 16 threads a token took
// 22 us for 594 tiles, with any number of tokens.)
template <int TOK>
__global__ __launch_bounds__(XT) void xent_join_kernel(const XArgs a, int tiles)
{
    constexpr int PARTS = XT / TOK;
    __shared__ float s_m[PARTS][TOK + 1], s_s[PARTS][TOK + 1];
    const int tok = threadIdx.x % TOK, part = threadIdx.x / TOK;
    const int64_t m = int64_t(blockIdx.x) * TOK + tok;
    const int row = m < a.T ? a.pos[m] : -1;
    float mx = -__builtin_inff(), s = 0.0f;
    if (row >= 0)
#pragma unroll 4
        for (int q = part; q < tiles; q += PARTS) {
            const float2 v = a.stat[int64_t(q) * a.Tp + row];
            join_stats(mx, s, v.x, v.y);
        }
    s_m[part][tok] = mx;
    s_s[part][tok] = s;
#pragma unroll
    for (int h = PARTS / 2; h > 0; h >>= 1) {
        __syncthreads();
        if (part < h) {
            join_stats(mx, s, s_m[part + h][tok], s_s[part + h][tok]);
            s_m[part][tok] = mx;
            s_s[part][tok] = s;
        }
    }
    if (part != 0 || m >= a.T) return;
    // (of the loss only the smaller terms are rounded: mx is often near z)
    a.lse_out[m] = row >= 0 ? mx + logf(s) : 0.0f;
    a.loss_out[m] = row >= 0 ? (mx - a.ztgt[row]) + logf(s) : 0.0f;
}

}  // namespace

size_t xent_ws_bytes(bool grad, int64_t T, int64_t N, int64_t D) { return xent_layout(grad, T, N, D).total; }

hipError_t launch_xent_loss(const XentCall &c, hipStream_t st)
{
    const XLayout l = xent_layout(false, c.T, c.N, c.D);
    XArgs a = xent_args(c, l, c.ws);
    a.ztgt = reinterpret_cast<float *>(static_cast<char *>(c.ws) + l.ztgt);
    a.stat = reinterpret_cast<float2 *>(static_cast<char *>(c.ws) + l.stat);
    a.loss_out = c.loss;
    a.lse_out = c.lse;
    const hipError_t e = launch_stats<EPI_STATS>(a, l, st);
    if (e != hipSuccess) return e;
    // few tokens: a block each; else eight, whose pairs lie next to each other
    if (c.T < 512) hipLaunchKernelGGL((xent_join_kernel<1>), dim3(unsigned(c.T)), dim3(XT), 0, st, a, int(l.tiles));
    else hipLaunchKernelGGL((xent_join_kernel<8>), dim3(unsigned((c.T + 7) / 8)), dim3(XT), 0, st, a, int(l.tiles));
    return hipGetLastError();
}

hipError_t launch_xent_grad(const XentCall &c, hipStream_t st)
{
    const XLayout l = xent_layout(true, c.T, c.N, c.D);
    const XArgs a = xent_args(c, l, c.ws);
    return launch_grad<false>(c, l, a, false, st, [&](const XArgs &piece) { return launch_tokens<EPI_PROB>(piece, piece.vp, 1, st); });
}

}  // namespace bsq
