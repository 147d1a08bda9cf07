// The residual stream, backward; residual.cuh has what both directions share.
//
// With xhat the standardised r, g = dh * A (A the norm's weight) and rho the reciprocal deviation:
//   d = dr + rho * (g - mean(g) - xhat * mean(g xhat)),     dx = alpha * d            (mean(g) with a mean in the norm only)
// With yhat the standardised y, e = gate * post_weight * d:   dy = rho_y * (e - mean(e) - yhat * mean(e yhat)); without a post norm
// dy = gate * d.  Rows are standardised before they are multiplied by anything: rho^2 and rho^3 leave the range of 32 bits long before rho
// does (rows beyond 1e12, and rows of zeros, which fill up a short batch, behind an eps below 2e-26).  Sums over tokens, per channel:
//   A: dh * xhat -> dweight        B: dh -> dbias
//   S: d * yhat (d * y without a post norm)       N: d             (N only behind a post norm)
//   dgate = post_weight * S + post_bias * N,  dpost_weight = gate * S,  dpost_bias = gate * N      (dgate = S without a post norm)
// A thread keeps them for its channels over a segment of tokens; segments' sums go to the workspace and residual_sums_kernel
// adds them up in order.  A row takes two rounds of sums over its threads, three behind a post norm: sum x (and sum y); sum x^2, sum g,
// sum g x (and sum y^2); sum e, sum e yhat.
#pragma once

#include <type_traits>

#include "residual.cuh"

namespace avggt {

constexpr int kBackwardThreads = 512;   // of an SM, as the launch bounds have them

struct ResidualBackArgs {
  const char *dh, *dr, *r, *y;
  char *dx, *dy;
  int64_t dhs, drs, rs, ys, dxs, dys;
  const float *weight, *gate, *post_weight, *post_bias;
  float *dweight, *dbias, *dgate;     // written directly where a segment holds whole groups and they are grouped
  float* partials;                    // [segments][4][channels]: A, B, S, N
  int n_tokens, channels, per_group;
  int norm, post, weight_grouped, gate_grouped;
  float eps, post_eps, alpha, one, inv_c;
  int segments;
  int parts;                          // > 0: a group is cut into that many segments; 0: segments of `groups` whole groups
  int groups;
  int smem_sums;                      // grouped gate behind a post norm, segments of whole groups: gate * S and gate * N in shared memory
  int stages;
};

// The kernels of 16-bit streams (residual_backward_narrow.cu) and of 32-bit ones (residual_backward_wide.cu), which are compiled apart: they
// are many.  type: of the stream, of the branch.
cudaError_t residual_backward_narrow(const ResidualBackArgs& a, int type, int layout, cudaStream_t st);
cudaError_t residual_backward_wide(const ResidualBackArgs& a, int type, int layout, cudaStream_t st);

namespace {

// R rows go through together, as in the forward kernel; they are read again from their stage where they are needed, which leaves the
// registers to the sums and parameters.  A batch ends where a group does.  30 frames of 1,024 channels in bf16 (507 MB): 82 us, 6.2 TB/s,
// and 6 us for the sums over segments; with a post norm and the stream in 32 bits (2,048 channels, 619 MB) 116 us and 10: there the latency of
// the exchanges among a row's eight warps, two blocks of them on an SM, bounds it.  Of the 112 variants 42 spill registers: a warp's rows
// behind a post norm (up to 236 bytes a thread stored), rows above 4,096 channels (48 to 180) and rows of single channels (24 to 92, above
// 4,096 channels 428 to 944).  The two above do not.
template <typename TR, typename TB, int LAY, bool BLOCK, int THREADS, int RUNS, int R, bool POST>
__global__ void __launch_bounds__(THREADS, kBackwardThreads / THREADS) residual_backward_kernel(const __grid_constant__ ResidualBackArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float scratch[BLOCK ? 2 * 4 * R * 32 : 1];
  int turn = 0;
  const Channels<LAY, BLOCK, RUNS> ch(a.channels);
  const int segment = BLOCK ? blockIdx.x : blockIdx.x * kWarpRows + (threadIdx.x >> 5);
  using StagedR = Staged<TR, LAY, THREADS, RUNS>;
  using StagedB = Staged<TB, LAY, THREADS, RUNS>;
  constexpr int kRowWarps = BLOCK ? THREADS / 32 : 1;
  constexpr uint32_t rb = StagedR::kBytes, bb = StagedB::kBytes, row_bytes = 2 * rb + 2 * bb, stage_bytes = R * row_bytes;
  const uint32_t ring = a.stages * stage_bytes;
  // behind the pipeline: [2][RUNS * 8][threads], each thread's own
  float* gated = reinterpret_cast<float*>(smem + (LAY > 2 ? ring : 0)) + threadIdx.x;
  const auto clear = [&](unsigned char* p, int rows) {
    StagedR::clear(p, rows, row_bytes);
    StagedR::clear(p + rb, rows, row_bytes);
    StagedB::clear(p + 2 * rb, rows, row_bytes);
    StagedB::clear(p + 2 * rb + bb, rows, row_bytes);
  };
  if constexpr (LAY > 2) clear(smem, a.stages * R);
  grid_dependency_wait();
  grid_launch_dependents();
  if (segment >= a.segments) return;                   // a whole warp (BLOCK: never)
  // tokens [t0, t1) of the segment, in groups
  int t0, t1, group;
  if (a.parts > 0) {
    group = segment / a.parts;
    const int part = segment - group * a.parts;
    const int64_t g0 = static_cast<int64_t>(group) * a.per_group;
    const int64_t g1 = g0 + a.per_group < a.n_tokens ? g0 + a.per_group : a.n_tokens;
    t0 = static_cast<int>(g0 + (g1 - g0) * part / a.parts);
    t1 = static_cast<int>(g0 + (g1 - g0) * (part + 1) / a.parts);
  } else {
    group = segment * a.groups;
    t0 = group * a.per_group;
    const int64_t end = t0 + static_cast<int64_t>(a.groups) * a.per_group;
    t1 = end < a.n_tokens ? static_cast<int>(end) : a.n_tokens;
  }
  const char* r = a.r + t0 * a.rs + ch.first * static_cast<int64_t>(sizeof(TR));
  const char* dr = a.dr + t0 * a.drs + ch.first * static_cast<int64_t>(sizeof(TR));
  const char* dh = a.dh + t0 * a.dhs + ch.first * static_cast<int64_t>(sizeof(TB));
  const char* y = a.y + t0 * a.ys + ch.first * static_cast<int64_t>(sizeof(TB));
  char* dx = a.dx + t0 * a.dxs + ch.first * static_cast<int64_t>(sizeof(TR));
  char* dy = a.dy + t0 * a.dys + ch.first * static_cast<int64_t>(sizeof(TB));
  const bool through_norm = a.dh != nullptr, behind = a.dr != nullptr, branch = a.y != nullptr;
  int ahead = t0;
  int64_t ahead_group_end = a.parts > 0 ? t1 : static_cast<int64_t>(group + 1) * a.per_group;
  const auto fetch = [&](uint32_t at) {
    at += smem_u32(smem);
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (ahead < t1 && (j == 0 || ahead < ahead_group_end)) {
        if (j == 0 && ahead >= ahead_group_end) ahead_group_end += a.per_group;
        ++ahead;
        if (through_norm) {
          StagedR::fetch(at + j * row_bytes, r, ch);
          StagedB::fetch(at + j * row_bytes + 2 * rb, dh, ch);
          r += a.rs;
          dh += a.dhs;
        }
        if (behind) {
          StagedR::fetch(at + j * row_bytes + rb, dr, ch);
          dr += a.drs;
        }
        if (branch) {
          StagedB::fetch(at + j * row_bytes + 2 * rb + bb, y, ch);
          y += a.ys;
        }
      } else {                                           // the batch is short: rows of zeros
        clear(smem + (at - smem_u32(smem)) + j * row_bytes, 1);
      }
    copy_async_commit();
  };
  if constexpr (LAY > 2)
    for (int s = 0; s < a.stages - 1; ++s) fetch(s * stage_bytes);

  float sA[RUNS][kRun], sB[RUNS][kRun], sS[RUNS][kRun], sN[RUNS][kRun];
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < kRun; ++e) sA[i][e] = sB[i][e] = sS[i][e] = sN[i][e] = 0.f;
  if (a.smem_sums)
#pragma unroll
    for (int e = 0; e < 2 * RUNS * kRun; ++e) gated[e * blockDim.x] = 0.f;

  float A[RUNS][kRun], E[RUNS][kRun];                  // the norm's weight; the gate (behind a post norm times its weight)
  const auto read_params = [&]() {
    const int64_t row = static_cast<int64_t>(group) * a.channels;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      ch.read_param(A[i], a.weight ? a.weight + (a.weight_grouped ? row : 0) : nullptr, i, 1.f - a.one);
      if (a.one != 0.f) add_each<kRun>(A[i], a.one);   // beside the row's channels dh is zero
      ch.read_param(E[i], a.gate ? a.gate + (a.gate_grouped ? row : 0) : nullptr, i, 1.f);
      if constexpr (POST) {
        float pw[kRun];
        ch.read_param(pw, a.post_weight, i, 1.f);
        multiply<kRun>(E[i], E[i], pw);
      }
    }
  };
  // a whole group is done: what belongs to it is finished
  const auto finish_group = [&]() {
    const int64_t at = static_cast<int64_t>(group) * a.channels;
    const auto out = [&](float* row) { return reinterpret_cast<char*>(row + at + ch.first); };
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      if (a.weight_grouped) {
        if (a.dweight) ch.template write<float>(sA[i], out(a.dweight), i);
        if (a.dbias) ch.template write<float>(sB[i], out(a.dbias), i);
#pragma unroll
        for (int e = 0; e < kRun; ++e) sA[i][e] = sB[i][e] = 0.f;
      }
      if (a.gate_grouped) {
        if constexpr (POST) {
          float pw[kRun], pb[kRun], gate[kRun];
          ch.read_param(pw, a.post_weight, i, 1.f);
          ch.read_param(pb, a.post_bias, i, 0.f);
          ch.read_param(gate, a.gate ? a.gate + at : nullptr, i, 1.f);
          if (a.smem_sums)
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
              float& s = gated[(i * kRun + e) * blockDim.x];
              float& n = gated[((RUNS + i) * kRun + e) * blockDim.x];
              s = fmaf(gate[e], sS[i][e], s);
              n = fmaf(gate[e], sN[i][e], n);
            }
#pragma unroll
          for (int e = 0; e < kRun; ++e) sS[i][e] = fmaf(sS[i][e], pw[e], sN[i][e] * pb[e]);
        }
        if (a.dgate) ch.template write<float>(sS[i], out(a.dgate), i);
#pragma unroll
        for (int e = 0; e < kRun; ++e) sS[i][e] = sN[i][e] = 0.f;
      }
    }
  };
  read_params();
  int64_t group_end = a.parts > 0 ? t1 : static_cast<int64_t>(group + 1) * a.per_group;

  const bool r_mean = through_norm && a.norm == AVGGT_NORM_LAYER, y_mean = POST && a.post == AVGGT_NORM_LAYER;
  // The sums that the means are made of join the last exchange of the batch before (its data has to be there by then: with two stages it
  // has had time to arrive only behind a post norm, whose batches have an exchange more).
  const bool early = LAY > 2 && (r_mean || y_mean) && (POST || a.stages > 2);
  float next_mean[R], next_y_m[R];
#pragma unroll
  for (int j = 0; j < R; ++j) next_mean[j] = next_y_m[j] = 0.f;
  uint32_t at = 0, last = ring - stage_bytes;            // this batch's stage, and the one before, which is used up
  for (int row = t0; row < t1;) {
    if (row >= group_end) {                              // the next group (a.parts == 0)
      finish_group();
      ++group;
      group_end += a.per_group;
      read_params();
    }
    int n = t1 - row < R ? t1 - row : R;                 // rows of this batch; the others count as zeros
    if (group_end - row < n) n = static_cast<int>(group_end - row);
    Run<TR, kRun> rq[R][RUNS], drq[R][RUNS];             // where there is no pipeline
    Run<TB, kRun> dhq[R][RUNS], yq[R][RUNS];
    const unsigned char* stage = smem + at;
    if constexpr (LAY > 2) {
      if (!early || row == t0) wait_stages(a.stages);
      fetch(last);
      last = at;
      at = at + stage_bytes == ring ? 0 : at + stage_bytes;
    } else {
#pragma unroll
      for (int j = 0; j < R; ++j) {
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          if (through_norm && j < n) {
            ch.read(rq[j][i], r, i);
            ch.read(dhq[j][i], dh, i);
          } else {
            rq[j][i].zero();
            dhq[j][i].zero();
          }
          if (behind && j < n) ch.read(drq[j][i], dr, i); else drq[j][i].zero();
          if (branch && j < n) ch.read(yq[j][i], y, i); else yq[j][i].zero();
        }
        if (j < n) {
          r += a.rs;
          dh += a.dhs;
          dr += a.drs;
          y += a.ys;
        }
      }
    }
    // row j of an array, zero behind the batch's rows and where the call has no such array
    const auto get = [&](auto& kept, int j, uint32_t array, float (&v)[RUNS][kRun]) {
      using Q = typename std::remove_reference<decltype(kept[0][0])>::type;
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        if constexpr (LAY > 2) {
          Q q;
          using S = typename std::conditional<std::is_same<Q, Run<TR, kRun>>::value, StagedR, StagedB>::type;
          S::take(q, stage + (j * row_bytes + array), i);
          q.values(v[i]);
        } else {
          kept[j][i].values(v[i]);
        }
      }
    };
    // a row of the next batch, which is in its stage by then
    const auto sum_of_next = [&](int j, uint32_t array, auto& kind) {
      using Q = typename std::remove_reference<decltype(kind[0][0])>::type;
      using S = typename std::conditional<std::is_same<Q, Run<TR, kRun>>::value, StagedR, StagedB>::type;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        Q q;
        float v[kRun];
        S::take(q, smem + at + (j * row_bytes + array), i);
        q.values(v);
        sum += sum_of<kRun>(v);
      }
      return sum;
    };
    const auto get_r = [&](int j, float (&v)[RUNS][kRun]) { get(rq, j, 0, v); };
    const auto get_dr = [&](int j, float (&v)[RUNS][kRun]) { get(drq, j, rb, v); };
    const auto get_dh = [&](int j, float (&v)[RUNS][kRun]) { get(dhq, j, 2 * rb, v); };
    const auto get_y = [&](int j, float (&v)[RUNS][kRun]) { get(yq, j, 2 * rb + bb, v); };

    float mean[R], y_m[R], rstd[R], y_rstd[R], pull[R], shift[R];          // pull, shift: -mean(g xhat) and -mean(g)
#pragma unroll
    for (int j = 0; j < R; ++j) {
      mean[j] = next_mean[j];
      y_m[j] = next_y_m[j];
      rstd[j] = y_rstd[j] = pull[j] = shift[j] = 0.f;
    }
    if ((r_mean || y_mean) && (!early || row == t0)) {
      float sums[POST ? 2 * R : R];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float v[RUNS][kRun];
        get_r(j, v);
        sums[j] = sum_all<RUNS>(v);
        if constexpr (POST) {
          get_y(j, v);
          sums[R + j] = sum_all<RUNS>(v);
        }
      }
      row_sums<kRowWarps, 4 * R>(sums, scratch, turn);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (r_mean) mean[j] = sums[j] * a.inv_c;
        if (POST && y_mean) y_m[j] = sums[POST ? R + j : j] * a.inv_c;
      }
    }
    float more[4 * R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float x[RUNS][kRun], t[RUNS][kRun], g[RUNS][kRun];
      get_r(j, x);
      ch.centre(x, mean[j]);
      get_dh(j, t);
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        multiply<kRun>(g[i], t[i], A[i]);
        accumulate<kRun>(sB[i], t[i]);
      }
      more[4 * j] = dot_all<RUNS>(x, x);
      more[4 * j + 1] = sum_all<RUNS>(g);
      more[4 * j + 2] = dot_all<RUNS>(g, x);
      more[4 * j + 3] = 0.f;
      if constexpr (POST) {
        get_y(j, x);
        ch.centre(x, y_m[j]);
        more[4 * j + 3] = dot_all<RUNS>(x, x);
      }
    }
    if (!POST && early) {
      wait_stages(a.stages);
#pragma unroll
      for (int j = 0; j < R; ++j) more[4 * j + 3] = sum_of_next(j, 0, rq);
    }
    row_sums<kRowWarps, 4 * R>(more, scratch, turn);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (!POST && early) next_mean[j] = more[4 * j + 3] * a.inv_c;
      if (POST) y_rstd[j] = rsqrtf(more[4 * j + 3] * a.inv_c + a.post_eps);
      rstd[j] = rsqrtf(more[4 * j] * a.inv_c + a.eps);
      if (r_mean) shift[j] = -more[4 * j + 1] * a.inv_c;
      pull[j] = -rstd[j] * (more[4 * j + 2] * a.inv_c);
    }
    float dots[LAY > 2 ? 4 * R : 2 * R], e[POST ? R : 1][RUNS][kRun];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float d[RUNS][kRun], yv[RUNS][kRun];
      get_dr(j, d);
      if (through_norm) {
        float x[RUNS][kRun], t[RUNS][kRun];
        get_r(j, x);
        ch.centre(x, mean[j]);
        get_dh(j, t);
        const uint64_t rr = pack_f32x2(rstd[j], rstd[j]), pp = pack_f32x2(pull[j], pull[j]), ss = pack_f32x2(shift[j], shift[j]);
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
          for (int k = 0; k < kRun; k += 2) {
            const uint64_t xhat = mul_f32x2(two(x[i] + k), rr), tt = two(t[i] + k);
            put_two(fma_f32x2(tt, xhat, two(sA[i] + k)), sA[i] + k);
            put_two(fma_f32x2(fma_f32x2(xhat, pp, fma_f32x2(tt, two(A[i] + k), ss)), rr, two(d[i] + k)), d[i] + k);
          }
      }
      if (a.dx && j < n) {
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          float out[kRun];
#pragma unroll
          for (int k = 0; k < kRun; ++k) out[k] = d[i][k];
          scale_each<kRun>(out, a.alpha);
          ch.template write<TR>(out, dx, i);
        }
        dx += a.dxs;
      }
      get_y(j, yv);
      if constexpr (POST) {
        ch.centre(yv, y_m[j]);
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          scale_each<kRun>(yv[i], y_rstd[j]);
          accumulate_products<kRun>(sS[i], d[i], yv[i]);
          accumulate<kRun>(sN[i], d[i]);
          multiply<kRun>(e[j][i], d[i], E[i]);
        }
        dots[2 * j] = sum_all<RUNS>(e[j]);
        dots[2 * j + 1] = dot_all<RUNS>(e[j], yv);
      } else {
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          accumulate_products<kRun>(sS[i], d[i], yv[i]);
          multiply<kRun>(d[i], d[i], E[i]);
        }
        if (a.dy && j < n) {
#pragma unroll
          for (int i = 0; i < RUNS; ++i) ch.template write<TB>(d[i], dy, i);
          dy += a.dys;
        }
      }
    }
    if constexpr (POST) {
      if constexpr (LAY > 2) {
        if (early) wait_stages(a.stages);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          dots[2 * R + j] = early && r_mean ? sum_of_next(j, 0, rq) : 0.f;
          dots[3 * R + j] = early && y_mean ? sum_of_next(j, 2 * rb + bb, yq) : 0.f;
        }
      }
      row_sums<kRowWarps, 4 * R>(dots, scratch, turn);
      if constexpr (LAY > 2) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          next_mean[j] = dots[2 * R + j] * a.inv_c;
          next_y_m[j] = dots[3 * R + j] * a.inv_c;
        }
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (!a.dy || j >= n) continue;
        const float back = y_mean ? -dots[2 * j] * a.inv_c : 0.f, dot = -dots[2 * j + 1] * a.inv_c;      // -mean(e), -mean(e yhat)
        const uint64_t mm = pack_f32x2(back, back), qq = pack_f32x2(dot, dot), rr = pack_f32x2(y_rstd[j], y_rstd[j]);
        float yv[RUNS][kRun];
        get_y(j, yv);
        ch.centre(yv, y_m[j]);
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
#pragma unroll
          for (int k = 0; k < kRun; k += 2)
            put_two(mul_f32x2(fma_f32x2(mul_f32x2(two(yv[i] + k), rr), qq, add_f32x2(two(e[j][i] + k), mm)), rr), e[j][i] + k);
          ch.template write<TB>(e[j][i], dy, i);
        }
        dy += a.dys;
      }
    }
    row += n;
  }
  if (a.parts == 0) finish_group();
  if (a.partials == nullptr) return;
  char* out = reinterpret_cast<char*>(a.partials + static_cast<int64_t>(segment) * 4 * a.channels + ch.first);
  const int64_t apart = static_cast<int64_t>(a.channels) * 4;
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    if (a.smem_sums)
#pragma unroll
      for (int e = 0; e < kRun; ++e) {
        sS[i][e] = gated[(i * kRun + e) * blockDim.x];
        sN[i][e] = gated[((RUNS + i) * kRun + e) * blockDim.x];
      }
    ch.template write<float>(sA[i], out, i);
    ch.template write<float>(sB[i], out + apart, i);
    ch.template write<float>(sS[i], out + 2 * apart, i);
    ch.template write<float>(sN[i], out + 3 * apart, i);
  }
}

template <typename TR, typename TB, int LAY, bool BLOCK, int THREADS, int RUNS, int R>
cudaError_t launch_backward_rows(ResidualBackArgs a, unsigned threads, cudaStream_t st) {
  constexpr int stage = LAY > 2 ? THREADS * R * RUNS * 2 * kRun * static_cast<int>(sizeof(TR) + sizeof(TB)) : 0;
  const int sums = a.smem_sums ? static_cast<int>(threads) * 2 * RUNS * kRun * 4 : 0;
  if constexpr (2 * stage > kMostSmem) {                 // wide rows of 32 bits on both sides: no room for a pipeline
    return launch_backward_rows<TR, TB, 2, true, 512, RUNS, R>(a, threads, st);
  } else {
    if (LAY > 2 && 2 * stage + sums > kMostSmem)         // nor for one with wide rows' sums behind it
      return launch_backward_rows<TR, TB, 2, true, 512, RUNS, R>(a, threads, st);
    const int per_sm = kBackwardThreads / static_cast<int>(threads);
    a.stages = per_sm * (3 * stage + sums + kSmemPerBlock) <= kSmemPerSm ? 3 : 2;
    const int64_t blocks = BLOCK ? a.segments : (a.segments + kWarpRows - 1) / kWarpRows;
    const int smem = a.stages * stage + sums;
    return a.post == AVGGT_NORM_NONE
               ? launch_with_smem<residual_backward_kernel<TR, TB, LAY, BLOCK, THREADS, RUNS, R, false>>(blocks, threads, smem, st, a)
               : launch_with_smem<residual_backward_kernel<TR, TB, LAY, BLOCK, THREADS, RUNS, R, true>>(blocks, threads, smem, st, a);
  }
}

template <typename TR, typename TB, int LAY>
cudaError_t launch_backward_of(const ResidualBackArgs& a, cudaStream_t st) {
  const unsigned threads = threads_of(a.channels);
  if (runs_of(a.channels) == 2) return launch_backward_rows<TR, TB, LAY, true, 512, 2, 1>(a, threads, st);
  if constexpr (LAY > 2) {            // a stage is laid out for the variant's THREADS
    if (a.channels <= kSpan) return launch_backward_rows<TR, TB, LAY, false, kWarpThreads, 1, 2>(a, kWarpThreads, st);
    if (threads <= 128) return launch_backward_rows<TR, TB, LAY, true, 128, 1, 2>(a, threads, st);
    if (threads <= 256) return launch_backward_rows<TR, TB, LAY, true, 256, 1, 2>(a, threads, st);
  }
  return launch_backward_rows<TR, TB, LAY, true, 512, 1, 2>(a, threads, st);
}

template <typename TR, typename TB>
cudaError_t backward_of(const ResidualBackArgs& a, int layout, cudaStream_t st) {
  constexpr int kBest = sizeof(TR) == 2 && sizeof(TB) == 2 ? 16 : 8;
  return layout == kBest ? launch_backward_of<TR, TB, kBest>(a, st)
         : layout == 4   ? launch_backward_of<TR, TB, 4>(a, st)
                         : launch_backward_of<TR, TB, 2>(a, st);
}

}  // namespace

}  // namespace avggt
