// The residual stream, forward; residual.cuh has what both directions share.
#pragma once

#include "residual.cuh"

namespace avggt {

constexpr int kForwardThreads = 512;   // of an SM, as the launch bounds have them

struct ResidualArgs {
  const char *x, *y;
  char *r, *h;
  int64_t xs, ys, rs, hs;            // in bytes, as all strides below
  const float *weight, *bias, *gate, *post_weight, *post_bias;
  int n_tokens, channels, per_group;
  int norm, post, weight_grouped, gate_grouped;
  float eps, post_eps, alpha, one, inv_c;
  int stages;
};

// The kernels of 16-bit streams (residual_forward_narrow.cu) and of 32-bit ones (residual_forward_wide.cu), which are compiled apart: they
// are many.  type: of the stream, of the branch.
cudaError_t residual_forward_narrow(const ResidualArgs& a, int type, int layout, int sm_count, cudaStream_t st);
cudaError_t residual_forward_wide(const ResidualArgs& a, int type, int layout, int sm_count, cudaStream_t st);

namespace {

// TR, TB: types of the residual stream and of the branch.  A row is a warp's (BLOCK false) or that of a block of at most THREADS.
// R: rows that go through together, so that their sums share exchanges and barriers and there is work while one waits.  Parameters stay
// in registers (read for every row, their loads alone took 70% of what the cache passes); a grouped one is read again where a
// group begins.  HBM bounds it: 100 frames of 1,024 channels (1.13 GB) 197 us, in a loop of calls 204, where two copies side by side take 195.
// Of the 120 variants 16 spill registers, 8 to 116 bytes a thread: rows of single channels, and above 4,096 channels behind a post norm.
template <typename TR, typename TB, int LAY, bool BLOCK, int THREADS, int RUNS, int R, bool POST>
__global__ void __launch_bounds__(THREADS, kForwardThreads / THREADS) residual_norm_kernel(const __grid_constant__ ResidualArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float scratch[BLOCK ? 2 * R * 32 : 1];
  int turn = 0;
  const Channels<LAY, BLOCK, RUNS> ch(a.channels);
  const int64_t mine = BLOCK ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * kWarpRows + (threadIdx.x >> 5);
  const int64_t all = BLOCK ? gridDim.x : static_cast<int64_t>(gridDim.x) * kWarpRows;
  const int64_t batches = (static_cast<int64_t>(a.n_tokens) + R - 1) / R;
  const int row0 = static_cast<int>(batches * mine / all) * R;
  const int64_t past = batches * (mine + 1) / all * R;
  const int row1 = past < a.n_tokens ? static_cast<int>(past) : a.n_tokens;
  const char* x = a.x + row0 * a.xs + ch.first * static_cast<int64_t>(sizeof(TR));
  const char* y = a.y + row0 * a.ys + ch.first * static_cast<int64_t>(sizeof(TB));
  char* r = a.r + row0 * a.rs + ch.first * static_cast<int64_t>(sizeof(TR));
  char* h = a.h + row0 * a.hs + ch.first * static_cast<int64_t>(sizeof(TB));
  const bool branch = a.y != nullptr;
  using StagedR = Staged<TR, LAY, THREADS, RUNS>;
  using StagedB = Staged<TB, LAY, THREADS, RUNS>;
  constexpr int kRowWarps = BLOCK ? THREADS / 32 : 1;
  constexpr uint32_t xb = StagedR::kBytes, row_bytes = xb + StagedB::kBytes, stage_bytes = R * row_bytes;
  const uint32_t ring = a.stages * stage_bytes;
  if constexpr (LAY > 2) {
    StagedR::clear(smem, a.stages * R, row_bytes);
    StagedB::clear(smem + xb, a.stages * R, row_bytes);
  }
  grid_dependency_wait();
  grid_launch_dependents();

  int to_fetch = row1 - row0;
  const auto fetch = [&](uint32_t at) {
    at += smem_u32(smem);
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (to_fetch > 0) {
        --to_fetch;
        StagedR::fetch(at + i * row_bytes, x, ch);
        x += a.xs;
        if (branch) {
          StagedB::fetch(at + i * row_bytes + xb, y, ch);
          y += a.ys;
        }
      }
    copy_async_commit();
  };
  if constexpr (LAY > 2)
    for (int s = 0; s < a.stages - 1; ++s) fetch(s * stage_bytes);
  uint32_t at = 0, last = ring - stage_bytes;            // these rows' stage, and the one before, which is used up

  float w[RUNS][kRun], b[RUNS][kRun], g[RUNS][kRun], gb[RUNS][kRun];     // gb: of the bias behind the branch's norm
  const auto read_weight = [&](int64_t offset) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      ch.read_param(w[i], a.weight ? a.weight + offset : nullptr, i, 1.f - a.one);
      ch.read_param(b[i], a.bias ? a.bias + offset : nullptr, i, 0.f);
      if (a.one != 0.f) add_each<kRun>(w[i], a.one);
    }
  };
  const auto read_gate = [&](int64_t offset) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      ch.read_param(g[i], a.gate ? a.gate + offset : nullptr, i, 1.f);
      if constexpr (POST) {
        float pw[kRun];
        ch.read_param(gb[i], a.post_bias, i, 0.f);
        ch.read_param(pw, a.post_weight, i, 1.f);
        multiply<kRun>(gb[i], gb[i], g[i]);
        multiply<kRun>(g[i], g[i], pw);
      }
    }
  };
  int64_t weight_end = INT64_MAX, gate_end = INT64_MAX;  // the first row of the next group
  if (a.weight_grouped) weight_end = row0;
  else read_weight(0);
  if (a.gate_grouped) gate_end = row0;
  else read_gate(0);

  for (int row = row0; row < row1; row += R) {
    float v[R][RUNS][kRun];
    Run<TR, kRun> xq[R][RUNS];
    Run<TB, kRun> yq[R][RUNS];
    if constexpr (LAY > 2) {
      wait_stages(a.stages);
#pragma unroll
      for (int j = 0; j < R; ++j)                        // rows behind the last one: whatever the stage holds, never written
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          StagedR::take(xq[j][i], smem + at + j * row_bytes, i);
          if (branch) StagedB::take(yq[j][i], smem + at + j * row_bytes + xb, i);
        }
      fetch(last);
      last = at;
      at = at + stage_bytes == ring ? 0 : at + stage_bytes;
    } else {
#pragma unroll
      for (int j = 0; j < R; ++j) {
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          if (row + j < row1) {
            ch.read(xq[j][i], x, i);
            if (branch) ch.read(yq[j][i], y, i);
          } else {
            xq[j][i].zero();
            yq[j][i].zero();
          }
        }
        x += a.xs;
        y += a.ys;
      }
    }
    float s[R];
    if (branch) {
#pragma unroll
      for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < RUNS; ++i) yq[j][i].values(v[j][i]);
      if constexpr (POST) {
        if (a.post == AVGGT_NORM_LAYER) {
#pragma unroll
          for (int j = 0; j < R; ++j) s[j] = sum_all<RUNS>(v[j]);
          row_sums<kRowWarps, R>(s, scratch, turn);
#pragma unroll
          for (int j = 0; j < R; ++j) ch.centre(v[j], s[j] * a.inv_c);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) s[j] = dot_all<RUNS>(v[j], v[j]);
        row_sums<kRowWarps, R>(s, scratch, turn);
#pragma unroll
        for (int j = 0; j < R; ++j) s[j] = rsqrtf(s[j] * a.inv_c + a.post_eps);
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (row + j >= gate_end && row + j < row1) {
          const int64_t group = (row + j) / a.per_group;
          gate_end = (group + 1) * a.per_group;
          read_gate(group * a.channels);
        }
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          float xv[kRun];
          xq[j][i].values(xv);
          if constexpr (POST) {
            scale_each<kRun>(v[j][i], s[j]);
            affine_each<kRun>(v[j][i], g[i], gb[i]);
          } else {
            multiply<kRun>(v[j][i], v[j][i], g[i]);
          }
          const uint64_t alpha = pack_f32x2(a.alpha, a.alpha);
#pragma unroll
          for (int e = 0; e < kRun; e += 2) put_two(fma_f32x2(two(xv + e), alpha, two(v[j][i] + e)), v[j][i] + e);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          xq[j][i].values(v[j][i]);
          scale_each<kRun>(v[j][i], a.alpha);
        }
    }
    if (a.r != nullptr)
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (row + j < row1)
#pragma unroll
          for (int i = 0; i < RUNS; ++i) ch.template write<TR>(v[j][i], r, i);
        r += a.rs;
      }
    if (a.h == nullptr) continue;
    if (a.norm == AVGGT_NORM_LAYER) {
#pragma unroll
      for (int j = 0; j < R; ++j) s[j] = sum_all<RUNS>(v[j]);
      row_sums<kRowWarps, R>(s, scratch, turn);
#pragma unroll
      for (int j = 0; j < R; ++j) ch.centre(v[j], s[j] * a.inv_c);
    }
#pragma unroll
    for (int j = 0; j < R; ++j) s[j] = dot_all<RUNS>(v[j], v[j]);
    row_sums<kRowWarps, R>(s, scratch, turn);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (row + j >= weight_end && row + j < row1) {
        const int64_t group = (row + j) / a.per_group;
        weight_end = (group + 1) * a.per_group;
        read_weight(group * a.channels);
      }
      const float rstd = rsqrtf(s[j] * a.inv_c + a.eps);
      if (row + j < row1)
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          scale_each<kRun>(v[j][i], rstd);
          affine_each<kRun>(v[j][i], w[i], b[i]);
          ch.template write<TB>(v[j][i], h, i);
        }
      h += a.hs;
    }
  }
}

template <typename TR, typename TB, int LAY, bool BLOCK, int THREADS, int RUNS, int R>
cudaError_t launch_forward_rows(ResidualArgs a, unsigned threads, int sm_count, cudaStream_t st) {
  const int stage = LAY > 2 ? THREADS * R * RUNS * kRun * static_cast<int>(sizeof(TR) + sizeof(TB)) : 0;
  constexpr int kRoom = kForwardThreads >= 2 * THREADS ? kForwardThreads / THREADS * THREADS : THREADS;   // threads, by the launch bounds
  int per_sm = kRoom / static_cast<int>(threads);
  a.stages = per_sm * (3 * stage + kSmemPerBlock) <= kSmemPerSm ? 3 : 2;
  const int fit = kSmemPerSm / (a.stages * stage + kSmemPerBlock);
  if (fit < per_sm) per_sm = fit;
  const int64_t batches = (static_cast<int64_t>(a.n_tokens) + R - 1) / R;
  int64_t blocks = BLOCK ? batches : (batches + kWarpRows - 1) / kWarpRows;
  if (blocks > static_cast<int64_t>(sm_count) * per_sm) blocks = static_cast<int64_t>(sm_count) * per_sm;
  return a.post == AVGGT_NORM_NONE
             ? launch_with_smem<residual_norm_kernel<TR, TB, LAY, BLOCK, THREADS, RUNS, R, false>>(blocks, threads, a.stages * stage, st, a)
             : launch_with_smem<residual_norm_kernel<TR, TB, LAY, BLOCK, THREADS, RUNS, R, true>>(blocks, threads, a.stages * stage, st, a);
}

template <typename TR, typename TB, int LAY>
cudaError_t launch_forward_of(const ResidualArgs& a, int sm_count, cudaStream_t st) {
  const unsigned threads = threads_of(a.channels);
  if (runs_of(a.channels) == 2) return launch_forward_rows<TR, TB, LAY, true, 512, 2, 1>(a, threads, sm_count, st);
  if constexpr (LAY > 2) {            // a stage is laid out for the variant's THREADS
    if (a.channels <= kSpan) return launch_forward_rows<TR, TB, LAY, false, kWarpThreads, 1, 2>(a, kWarpThreads, sm_count, st);
    if (threads <= 128) return launch_forward_rows<TR, TB, LAY, true, 128, 1, 2>(a, threads, sm_count, st);
    if (threads <= 256) return launch_forward_rows<TR, TB, LAY, true, 256, 1, 2>(a, threads, sm_count, st);
  }
  return launch_forward_rows<TR, TB, LAY, true, 512, 1, (LAY > 2 ? 2 : 4)>(a, threads, sm_count, st);
}

template <typename TR, typename TB>
cudaError_t forward_of(const ResidualArgs& a, int layout, int sm_count, cudaStream_t st) {
  constexpr int kBest = sizeof(TR) == 2 && sizeof(TB) == 2 ? 16 : 8;
  return layout == kBest ? launch_forward_of<TR, TB, kBest>(a, sm_count, st)
         : layout == 4   ? launch_forward_of<TR, TB, 4>(a, sm_count, st)
                         : launch_forward_of<TR, TB, 2>(a, sm_count, st);
}

}  // namespace

}  // namespace avggt
