// The paged key-value cache: rows written into pages (RoPE on the way), one token's attention over them, and eviction by the
// attention's accumulated weights.  A page holds page_rows rows of every key head, K and V step-tiled (formulas: header of the
// C ABI), so a 64-byte column of 16 keys, or 16 dims of a step's values, is again a contiguous 1 KB matrix-core fragment.
#include <algorithm>

#include "kernels.h"
#include "paged_plan.h"

namespace amph {

__device__ __forceinline__ float paged_exp2(float x) { return __builtin_amdgcn_exp2f(x); }   // arguments <= 0: no rescue of tiny results
constexpr int BUF_RAW = 0x00020000;                    // word 3 of a buffer descriptor: plain bytes
__device__ __forceinline__ uint4 ldb16_stream(__amdgpu_buffer_rsrc_t r, int at) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 2);            // (2: non-temporal)
  return make_uint4(v.x, v.y, v.z, v.w);
}
constexpr float PAGED_LOWEST = -3.402823466e38f;       // of a running maximum: no finite score is below it, and -inf - it is -inf

// Inclusive sum over the lanes of a wave, inside the vector ALU: shifts within rows of 16, then the rows' last lanes passed on.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast:31 into rows 2 and 3
  return v;
}

__device__ __forceinline__ int paged_len(const PagedSeqs &s, int b) {
  return paged_rows(s.kv_len[b], s.n_valid ? paged_new(s.n_new, s.n_valid[b]) : s.n_new, s.cap);
}

// =====================================================================================================
// amph_paged_attn
//   S^T[key, q] = K[key, :] . Q[q, :],   O^T[d, q] += V^T[d, keys] . P^T[keys, q]
// on the matrix cores as in the verification attention (the accumulator of a score tile is the second product's operand), with
// the G query heads of a key head as the columns.  Bound by the cache's bytes: every row is read once, for all its query heads.
// =====================================================================================================
template <typename T, int DH, int NQB>
struct PA {
  static constexpr int PER = Elem<T>::PER;
  static constexpr int KSTEP = 4 * PER;            // keys per step
  static constexpr int NT = KSTEP / 16;            // S^T tiles per step
  static constexpr int DSTEPS = DH / (4 * PER);    // 64-byte pieces of a K/Q row
  static constexpr int DB = DH / 16;               // 16-row blocks of O^T
  static constexpr int NQ = NQB * 16;              // queries per workgroup
  static constexpr int OPITCH = DH + 4;            // floats
  static constexpr int PART = NQ * DH + 2 * NQ;    // floats of one partial: O, then m, then l (-1: a bad page)
};

template <int N> struct Rows { static constexpr int value = N; };

// ALONE: a workgroup for every walk (one key head's query group of one sequence).  Otherwise the walks' key steps are dealt out
// in equal pieces (paged_plan.h) and k_paged_fold joins what was cut.
template <typename T, int DH, int NQB, bool ALONE>
__global__ __launch_bounds__(256, 2) void k_paged_attn(const PagedAttnArgs a) {
  using C = PA<T, DH, NQB>;
  constexpr int PER = C::PER, KSTEP = C::KSTEP, NT = C::NT, DSTEPS = C::DSTEPS, DB = C::DB, NQ = C::NQ;
  __shared__ __align__(16) float sm_o[PAGED_WAVES][NQ][C::OPITCH];
  __shared__ float sm_m[PAGED_WAVES][NQ], sm_l[PAGED_WAVES][NQ];
  __shared__ int sm_len[ALONE ? 1 : PAGED_MAX_SEQ], sm_sum[PAGED_WAVES], sm_at[2];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r16 = lane & 15;
  const int n_seq = a.seqs.n_seq, G = a.group, n_qg = a.n_qg, U = a.walks;
  const int psteps = a.c.page_rows / KSTEP;            // key steps of a page
  const float scale = 1.4426950408889634f * rsqrtf((float)DH);
  const float NEG_INF = -__builtin_huge_valf();

  // ---- the key steps [s, s + n) of one walk
  auto walk = [&](int b, int u, int L, int s, int n, bool whole, int place) {
    // this wave's steps are s + wave + 4 i, i < n_w; lane l finds where step 64 * block + l begins (bytes into the pages)
    const int32_t *row_table = a.c.table + (size_t)b * a.c.table_pages;
    const int n_w = (n - wave + PAGED_WAVES - 1) / PAGED_WAVES;
    auto step_of = [&](int i0) { return max(min(s + wave + PAGED_WAVES * min(i0 + lane, n_w - 1), s + n - 1), 0); };   // (idle waves: any of the walk's)
    int id = row_table[step_of(0) / psteps];           // asked for ahead of all else
    const int h = u / n_qg, q_base = (u - h * n_qg) * NQ, live_q = min(G - q_base, NQ);
    const T *qb0 = (const T *)a.q + (size_t)b * a.ld_q + ((size_t)h * G + q_base) * DH;
    uint4 Qf[NQB][DSTEPS];                             // queries as B fragments: lane = query r16 of block qb
    #pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      const int qi = qb * 16 + r16;
      #pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds)              // padding queries repeat query 0; nothing of theirs is stored
        Qf[qb][ds] = ldg16(qb0 + (size_t)(qi < live_q ? qi : 0) * DH + ds * (4 * PER) + g * PER);
    }
    unsigned char *Kh = (unsigned char *)a.c.k + (size_t)h * a.c.head_stride * sizeof(T);
    unsigned char *Vh = (unsigned char *)a.c.v + (size_t)h * a.c.head_stride * sizeof(T);
    const int lane_at = r16 * 64 + g * 16;
    float *score = a.scores ? a.scores + ((size_t)b * a.n_heads + (size_t)h * G + q_base) * a.seqs.cap : nullptr;

    f32x4 O[NQB][DB];
    float m_run[NQB], l_run[NQB];
    #pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      m_run[qb] = PAGED_LOWEST; l_run[qb] = 0.f;
      #pragma unroll
      for (int db = 0; db < DB; ++db) O[qb][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    bool bad = false;

    unsigned long long where = 0;
    auto look_up = [&](int i0) {
      const int st = step_of(i0), pg = st / psteps;
      if ((unsigned)id >= (unsigned)a.c.n_pages) { bad = n_w > 0; id = 0; }
      where = ((unsigned long long)id * a.c.page_stride + (unsigned long long)(st - pg * psteps) * (KSTEP * DH)) * sizeof(T);
    };
    auto step_base = [&](int i) -> size_t {            // (uniform)
      const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)where, i & 63);
      const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(where >> 32), i & 63);
      return ((size_t)hi << 32) | lo;
    };
    uint4 Kf[NT][DSTEPS], Vf[DB];
    // A step's fragments through a buffer of its bytes; of no bytes where there is no further step: such loads fetch nothing, and the
    // loop needs no branch around them.
    auto load_k = [&](size_t at, bool live) {
      const auto r = __builtin_amdgcn_make_buffer_rsrc(Kh + at, 0, live ? NT * DSTEPS * 1024 : 0, BUF_RAW);
      #pragma unroll
      for (int t = 0; t < NT; ++t)
        #pragma unroll
        for (int ds = 0; ds < DSTEPS; ++ds) Kf[t][ds] = ldb16_stream(r, lane_at + (t * DSTEPS + ds) * 1024);
    };
    auto load_v = [&](size_t at, bool live) {
      const auto r = __builtin_amdgcn_make_buffer_rsrc(Vh + at, 0, live ? DB * 1024 : 0, BUF_RAW);
      #pragma unroll
      for (int db = 0; db < DB; ++db) Vf[db] = ldb16_stream(r, lane_at + db * 1024);
    };
    // scores of step i: keys key0 + g * PER + j, query r16 of every block
    auto scores = [&](int i, float (&sv)[NQB][PER]) {
      #pragma unroll
      for (int qb = 0; qb < NQB; ++qb)
        #pragma unroll
        for (int t = 0; t < NT; ++t) {
          f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
          #pragma unroll
          for (int ds = 0; ds < DSTEPS; ++ds) acc = mma16<T>(Kf[t][ds], Qf[qb][ds], acc);
          #pragma unroll
          for (int c = 0; c < 4; ++c) sv[qb][t * 4 + c] = acc[c] * scale;
        }
    };
    // the running maximum, and the step's probabilities
    auto softmax = [&](int i, float (&sv)[NQB][PER], float (&pv)[NQB][PER]) {
      const int key0 = (s + wave + PAGED_WAVES * i) * KSTEP;
      #pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        if (key0 + KSTEP > L) {
          #pragma unroll
          for (int j = 0; j < PER; ++j) if (key0 + g * PER + j >= L) sv[qb][j] = NEG_INF;
        }
        float mx = sv[qb][0], ls = 0.f;
        #pragma unroll
        for (int j = 1; j < PER; ++j) mx = fmaxf(mx, sv[qb][j]);
        const float mn = fmaxf(m_run[qb], lanes_xor32(lanes_xor16(mx, MaxF()), MaxF()));
        if (__any(mn > m_run[qb])) {                   // the running maximum rarely moves after the first steps
          const float corr = paged_exp2(m_run[qb] - mn);
          l_run[qb] *= corr;
          #pragma unroll
          for (int db = 0; db < DB; ++db) O[qb][db] *= corr;
          m_run[qb] = mn;
        }
        #pragma unroll
        for (int j = 0; j < PER; ++j) { pv[qb][j] = paged_exp2(sv[qb][j] - mn); ls += pv[qb][j]; }
        l_run[qb] += ls;
      }
    };
    // for the weights (cap is a multiple of the step: rows behind the last have their place)
    auto keep_scores = [&](int i, const float (&sv)[NQB][PER]) {
      #pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        if (qb * 16 + r16 >= live_q) continue;
        float *to = score + (size_t)(qb * 16 + r16) * a.seqs.cap + (s + wave + PAGED_WAVES * i) * KSTEP + g * PER;
        #pragma unroll
        for (int j = 0; j < PER; j += 4)
          *reinterpret_cast<float4 *>(to + j) = make_float4(sv[qb][j], sv[qb][j + 1], sv[qb][j + 2], sv[qb][j + 3]);
      }
    };
    auto values = [&](int i, const float (&pv)[NQB][PER]) {
      const int key0 = (s + wave + PAGED_WAVES * i) * KSTEP;
      if (key0 + KSTEP > L) {                          // rows behind the last may hold anything, NaN too: 0 * V has to be 0
        const int in = L - key0 - g * PER;             // elements of the lane's pieces that are rows
        unsigned keep[4];
        #pragma unroll
        for (int w = 0; w < 4; ++w)
          keep[w] = sizeof(T) == 4 ? (in > w ? ~0u : 0u) : (in > 2 * w ? 0xffffu : 0u) | (in > 2 * w + 1 ? 0xffff0000u : 0u);
        #pragma unroll
        for (int db = 0; db < DB; ++db) { Vf[db].x &= keep[0]; Vf[db].y &= keep[1]; Vf[db].z &= keep[2]; Vf[db].w &= keep[3]; }
      }
      #pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        if constexpr (sizeof(T) == 2) {
          // P in two operands, 16 bits: its upper half as it is, and what that leaves out, which is not negative, nor zero (an infinite value
          // times zero would be NaN; 2^-100 of a finite one is nothing)
          float rest[PER];
          unsigned hi[PER / 2];
          #pragma unroll
          for (int j = 0; j < PER; ++j) rest[j] = fmaxf(pv[qb][j] - __uint_as_float(__float_as_uint(pv[qb][j]) & 0xffff0000u), 7.8886091e-31f);
          #pragma unroll
          for (int j = 0; j < PER / 2; ++j) hi[j] = __builtin_amdgcn_perm(__float_as_uint(pv[qb][2 * j + 1]), __float_as_uint(pv[qb][2 * j]), 0x07060302u);
          const uint4 Pf = make_uint4(hi[0], hi[1], hi[PER / 2 - 2], hi[PER / 2 - 1]), Rf = pack16<T>(rest);
          #pragma unroll
          for (int db = 0; db < DB; ++db) O[qb][db] = mma16<T>(Vf[db], Pf, O[qb][db]);
          #pragma unroll
          for (int db = 0; db < DB; ++db) O[qb][db] = mma16<T>(Vf[db], Rf, O[qb][db]);
        } else {
          const uint4 Pf = pack16<T>(pv[qb]);
          #pragma unroll
          for (int db = 0; db < DB; ++db) O[qb][db] = mma16<T>(Vf[db], Pf, O[qb][db]);
        }
      }
    };

    if (n_w > 0) {
      // One register set: a step's keys are asked for when the scores of the step before are done, its values when the products
      // before are.  The other waves of the SIMD cover what is left of the latency.
      look_up(0);
      size_t at = step_base(0);
      load_k(at, true);
      load_v(at, true);
      #pragma unroll 1
      for (int i = 0; i < n_w; ++i) {
        const bool more = i + 1 < n_w;
        if (more && ((i + 1) & 63) == 0) { id = row_table[step_of(i + 1) / psteps]; look_up(i + 1); }
        at = step_base(i + 1);
        float sv[NQB][PER], pv[NQB][PER];
        scores(i, sv);
        load_k(at, more);
        softmax(i, sv, pv);
        values(i, pv);
        load_v(at, more);
        if (score) keep_scores(i, sv);                 // (behind the loads, which would otherwise wait for the stores)
      }
    }
    const bool wave_bad = __any(bad);

    // ---- lane groups hold partial sums of l for the same query; then waves -> workgroup through LDS
    __syncthreads();                                   // the walk before has read its sums
    #pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      const float l = lanes_xor32(lanes_xor16(l_run[qb], AddF()), AddF());
      if (qb * 16 + r16 < live_q) {
        if (g == 0) { sm_m[wave][qb * 16 + r16] = m_run[qb]; sm_l[wave][qb * 16 + r16] = wave_bad ? -1.f : l; }
        #pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(&sm_o[wave][qb * 16 + r16][db * 16 + g * 4]) = O[qb][db];
      }
    }
    __syncthreads();
    const bool any_bad = sm_l[0][0] < 0.f || sm_l[1][0] < 0.f || sm_l[2][0] < 0.f || sm_l[3][0] < 0.f;
    if (any_bad && tid == 0) atomicOr(a.dev_status, (unsigned)AMPH_DEV_BAD_PAGE);
    float *part = whole ? nullptr : a.partials + (size_t)place * C::PART;
    for (int idx = tid; idx < live_q * (DH / 4); idx += 256) {        // 4 dims of one query
      const int q = idx / (DH / 4), d4 = (idx % (DH / 4)) * 4;
      float mw = sm_m[0][q], l = 0.f;
      #pragma unroll
      for (int w = 1; w < PAGED_WAVES; ++w) mw = fmaxf(mw, sm_m[w][q]);
      f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
      #pragma unroll
      for (int w = 0; w < PAGED_WAVES; ++w) {
        const float f = paged_exp2(sm_m[w][q] - mw);
        o += *reinterpret_cast<const f32x4 *>(&sm_o[w][q][d4]) * f;
        l += sm_l[w][q] * f;
      }
      if (any_bad) l = -1.f;
      const size_t head = (size_t)b * a.n_heads + (size_t)h * G + q_base + q;
      if (whole) {
        const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
        const float r[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        if (!any_bad) store4<T>((T *)a.out + head * DH + d4, r);
        if (score && d4 == 0) a.stats[head] = make_float2(mw, l);
      } else {
        *reinterpret_cast<f32x4 *>(part + (size_t)q * DH + d4) = o;
        if (d4 == 0) { part[NQ * DH + q] = mw; part[NQ * DH + NQ + q] = l; }
      }
    }
    if constexpr (ALONE) {
      // ---- a workgroup that has all query heads of the key head adds up the weights itself, from the scores that it left (eight sequences of 500 rows,
      // 32 and 8 heads: 10.4 us, with a launch for it 14.2)
      if (!score || n_qg > 1 || any_bad) return;       // (whole workgroup)
      __syncthreads();                                 // sums are read, scores are written
      if (tid < live_q) {
        float mw = sm_m[0][tid], l = 0.f;
        #pragma unroll
        for (int w = 1; w < PAGED_WAVES; ++w) mw = fmaxf(mw, sm_m[w][tid]);
        #pragma unroll
        for (int w = 0; w < PAGED_WAVES; ++w) l += sm_l[w][tid] * paged_exp2(sm_m[w][tid] - mw);
        sm_m[0][tid] = mw;
        sm_l[0][tid] = l > 0.f || l != l ? 1.0f / l : 0.f;
      }
      __syncthreads();
      const size_t w_at = ((size_t)b * a.c.n_kv + h) * a.c.table_pages * a.c.page_rows;
      for (int row = tid * 4; row < L; row += 4 * 256) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        #pragma unroll 4
        for (int q = 0; q < live_q; ++q) {
          const float4 v = *reinterpret_cast<const float4 *>(score + (size_t)q * a.seqs.cap + row);
          const float mw = sm_m[0][q], inv = sm_l[0][q];
          acc[0] += paged_exp2(v.x - mw) * inv; acc[1] += paged_exp2(v.y - mw) * inv;
          acc[2] += paged_exp2(v.z - mw) * inv; acc[3] += paged_exp2(v.w - mw) * inv;
        }
        #pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row + i < L) a.weights_out[w_at + row + i] = (a.weights_in ? a.weights_in[w_at + row + i] : 0.f) + acc[i];
      }
    }
  };

  if constexpr (ALONE) {
    const int b = blockIdx.x / U, u = blockIdx.x % U, L = paged_len(a.seqs, b);
    if (L < 0) {                                       // (whole workgroup)
      if (tid == 0 && u == 0) atomicOr(a.dev_status, (unsigned)AMPH_DEV_KV_OVERFLOW);
      return;
    }
    walk(b, u, L, 0, (L + KSTEP - 1) / KSTEP, true, 0);
    return;
  }

  // ---- the sequences' lengths, the steps before each, and the sequence and walk that this piece begins in.  Up to 64 sequences every
  // wave finds that by itself, a sequence a lane, without a barrier (one sequence of 1025 rows, 32 heads: 9.0 us against 9.4 the other way);
  // beyond, thread t has sequences 4 t .. 4 t + 3.
  const bool few = n_seq <= WAVE;
  int all, L_lane = 0, b, at;
  long long first, last;
  if (few) {
    if (lane < n_seq) L_lane = paged_len(a.seqs, lane);
    const int st = L_lane > 0 ? (L_lane + KSTEP - 1) / KSTEP : 0, upto = wave_scan(st), before = upto - st;
    all = __builtin_amdgcn_readlane(upto, WAVE - 1);
    const PagedDeal pieces = paged_deal((long long)all * U);
    first = pieces.begin(blockIdx.x);
    last = pieces.begin(blockIdx.x + 1);
    if (blockIdx.x == 0 && wave == 0 && lane < n_seq) {
      a.plan[lane] = before;
      a.plan[n_seq + 1 + lane] = L_lane;
      if (L_lane < 0) atomicOr(a.dev_status, (unsigned)AMPH_DEV_KV_OVERFLOW);
    }
    const long long off = first - (long long)before * U;
    const uint64_t here = __ballot(off >= 0 && off < (long long)st * U);
    b = here ? __builtin_ctzll(here) : 0;
    at = __builtin_amdgcn_readlane((int)off, b);
  } else {
    constexpr int PT = PAGED_MAX_SEQ / 256;
    int st[PT], sum = 0;
    bool over = false;
    #pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int bi = tid * PT + i;
      int L = 0;
      if (bi < n_seq) {
        L = paged_len(a.seqs, bi);
        sm_len[bi] = L;
        over |= L < 0;
      }
      st[i] = L > 0 ? (L + KSTEP - 1) / KSTEP : 0;
      sum += st[i];
    }
    const int upto = wave_scan(sum);
    if (lane == WAVE - 1) sm_sum[wave] = upto;
    if (blockIdx.x == 0 && over) atomicOr(a.dev_status, (unsigned)AMPH_DEV_KV_OVERFLOW);
    __syncthreads();
    int before = upto - sum;
    all = 0;
    #pragma unroll
    for (int w = 0; w < PAGED_WAVES; ++w) { before += w < wave ? sm_sum[w] : 0; all += sm_sum[w]; }
    const PagedDeal pieces = paged_deal((long long)all * U);
    first = pieces.begin(blockIdx.x);
    last = pieces.begin(blockIdx.x + 1);
    #pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int bi = tid * PT + i;
      if (bi < n_seq) {
        if (blockIdx.x == 0) { a.plan[bi] = before; a.plan[n_seq + 1 + bi] = sm_len[bi]; }
        const long long off = first - (long long)before * U;
        if (off >= 0 && off < (long long)st[i] * U) { sm_at[0] = bi; sm_at[1] = (int)off; }
      }
      before += st[i];
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(sm_at[0]);
    at = __builtin_amdgcn_readfirstlane(sm_at[1]);
  }
  const long long total = (long long)all * U;
  if (blockIdx.x == 0 && tid == 0) a.plan[n_seq] = all;
  if (first >= total) return;                          // (whole workgroup; what b and at are then is not looked at)
  auto len_of = [&](int i) { return few ? __builtin_amdgcn_readlane(L_lane, i) : __builtin_amdgcn_readfirstlane(sm_len[i]); };
  int L = len_of(b), left = __builtin_amdgcn_readfirstlane((int)(min(last, total) - first));
  int u = at / ((L + KSTEP - 1) / KSTEP), s = at - u * ((L + KSTEP - 1) / KSTEP);
  bool head_of_piece = true;
  while (left > 0) {
    const int steps = (L + KSTEP - 1) / KSTEP, n = min(steps - s, left);
    walk(b, u, L, s, n, n == steps, 2 * blockIdx.x + (head_of_piece ? 0 : 1));
    head_of_piece = false;
    left -= n;
    s = 0;
    if (++u == U) {
      u = 0;
      while (left > 0 && (L = len_of(++b)) <= 0) {}    // (steps are left: so is a sequence that has them)
    }
  }
}

// Joins the walks that were cut: out = sum_i O_i 2^(m_i - m) / sum_i l_i 2^(m_i - m) over a walk's pieces; writes zeros for a
// sequence without rows; and, where weights are asked for, adds every row's probabilities up from the scores that the walks left.
// Workgroups [0, n_seq * n_heads): a query's output each; those behind: 1024 rows of one key head each.
constexpr int PAGED_WROWS = 1024;

template <typename T, int DH, int NQB>
__global__ __launch_bounds__(256) void k_paged_fold(const PagedAttnArgs a, bool alone, int row_wgs) {
  using C = PA<T, DH, NQB>;
  constexpr int KSTEP = C::KSTEP, NQ = C::NQ, LPQ = DH / 4, NG = 256 / LPQ;
  __shared__ __align__(16) float sm_o[NG][DH];
  __shared__ float sm_m[NG], sm_l[NG];
  __shared__ float2 sm_ml[8];
  const int tid = threadIdx.x, n_seq = a.seqs.n_seq, G = a.group, n_qg = a.n_qg, U = a.walks;
  const int outs = alone ? 0 : n_seq * a.n_heads;
  const int item = (int)blockIdx.x - outs;
  const int bh = item < 0 ? blockIdx.x : item / row_wgs;                       // (sequence, head) or (sequence, key head)
  const int b = item < 0 ? bh / a.n_heads : bh / a.c.n_kv;
  const int L = alone ? paged_len(a.seqs, b) : a.plan[n_seq + 1 + b];
  if (L < 0) return;
  const int steps = (L + KSTEP - 1) / KSTEP;
  const int pre = alone ? 0 : a.plan[b];
  const PagedDeal pieces = alone ? PagedDeal{1, 0} : paged_deal((long long)a.plan[n_seq] * U);

  if (item < 0) {
    const int head = bh % a.n_heads, h = head / G, q = head % G, d4 = (tid % LPQ) * 4, grp = tid / LPQ;
    T *dst = (T *)a.out + (size_t)bh * DH + d4;
    if (L == 0) {
      const float z[4] = {0.f, 0.f, 0.f, 0.f};
      if (grp == 0) store4<T>(dst, z);
      return;
    }
    const PagedWalk wk = paged_walk((long long)pre * U + (long long)(h * n_qg + q / NQ) * steps, steps, pieces);
    if (wk.w0 == wk.w1) return;                        // one workgroup had the whole walk and wrote its output
    const int np = wk.w1 - wk.w0 + 1, qi = q % NQ;
    // the chain of round trips is what this costs: four pieces a thread are asked for at once
    constexpr int FU = 4;
    float m = PAGED_LOWEST, l = 0.f;
    f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
    bool bad = false;
    for (int i0 = grp; i0 < np; i0 += NG * FU) {
      float ms[FU], ls[FU];
      f32x4 os[FU];
      #pragma unroll
      for (int k = 0; k < FU; ++k) {
        const float *p = a.partials + (size_t)wk.place(wk.w0 + min(i0 + k * NG, np - 1)) * C::PART;
        ms[k] = p[NQ * DH + qi];
        ls[k] = p[NQ * DH + NQ + qi];
        os[k] = *reinterpret_cast<const f32x4 *>(p + (size_t)qi * DH + d4);
      }
      #pragma unroll
      for (int k = 0; k < FU; ++k) {
        if (i0 + k * NG >= np) continue;
        bad |= ls[k] < 0.f;
        const float mn = fmaxf(m, ms[k]), f0 = paged_exp2(m - mn), f1 = paged_exp2(ms[k] - mn);
        o = o * f0 + os[k] * f1;
        l = l * f0 + ls[k] * f1;
        m = mn;
      }
    }
    *reinterpret_cast<f32x4 *>(&sm_o[grp][d4]) = o;
    if (d4 == 0) { sm_m[grp] = m; sm_l[grp] = l; }
    if (__syncthreads_or(bad)) return;
    if (grp != 0) return;
    float mt = PAGED_LOWEST, lt = 0.f;
    f32x4 ot = (f32x4){0.f, 0.f, 0.f, 0.f};
    #pragma unroll
    for (int k = 0; k < NG; ++k) mt = fmaxf(mt, sm_m[k]);
    #pragma unroll
    for (int k = 0; k < NG; ++k) {
      const float f = paged_exp2(sm_m[k] - mt);
      ot += *reinterpret_cast<const f32x4 *>(&sm_o[k][d4]) * f;
      lt += sm_l[k] * f;
    }
    const float inv = lt > 0.f || lt != lt ? 1.0f / lt : 0.f;
    const float r[4] = {ot[0] * inv, ot[1] * inv, ot[2] * inv, ot[3] * inv};
    store4<T>(dst, r);
    return;
  }

  // ---- weights of rows [row0, row0 + 1024) of key head h: thread t has four of them
  const int h = bh % a.c.n_kv, row0 = (item % row_wgs) * PAGED_WROWS, row = row0 + tid * 4;
  if (row0 >= L) return;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  bool bad = false;
  constexpr int QB = 8;                                // queries at a time: their scores are asked for, then 32 lanes find each one's sum
  for (int qa = 0; qa < G; qa += QB) {
    const float *sc = a.scores + ((size_t)b * a.n_heads + (size_t)h * G + qa) * a.seqs.cap + min(row, a.seqs.cap - 4);
    float4 v[QB];
    #pragma unroll
    for (int i = 0; i < QB; ++i) v[i] = *reinterpret_cast<const float4 *>(sc + (size_t)min(i, G - 1 - qa) * a.seqs.cap);
    const int q = qa + tid / 32, t32 = tid & 31;
    float m = PAGED_LOWEST, l = 0.f;
    if (q < G) {
      const PagedWalk wk = alone ? PagedWalk{0, 0, true}
                                 : paged_walk((long long)pre * U + (long long)(h * n_qg + q / NQ) * steps, steps, pieces);
      if (wk.w0 == wk.w1) {
        const float2 st = a.stats[(size_t)b * a.n_heads + h * G + q];
        if (t32 == 0) { m = st.x; l = st.y; bad |= l < 0.f; }
      } else {
        for (int i = t32; i <= wk.w1 - wk.w0; i += 32) {
          const float *p = a.partials + (size_t)wk.place(wk.w0 + i) * C::PART + NQ * DH + q % NQ;
          const float mi = p[0], li = p[NQ], mn = fmaxf(m, mi);
          bad |= li < 0.f;
          l = l * paged_exp2(m - mn) + li * paged_exp2(mi - mn);
          m = mn;
        }
      }
    }
    #pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float mo = __shfl_xor(m, o), lo = __shfl_xor(l, o), mn = fmaxf(m, mo);
      l = l * paged_exp2(m - mn) + lo * paged_exp2(mo - mn);
      m = mn;
    }
    __syncthreads();
    if (t32 == 0) sm_ml[tid / 32] = make_float2(m, l > 0.f || l != l ? 1.0f / l : 0.f);
    if (__syncthreads_or(bad)) return;
    #pragma unroll
    for (int i = 0; i < QB; ++i) {
      if (qa + i >= G) continue;
      const float2 ml = sm_ml[i];
      acc[0] += paged_exp2(v[i].x - ml.x) * ml.y; acc[1] += paged_exp2(v[i].y - ml.x) * ml.y;
      acc[2] += paged_exp2(v[i].z - ml.x) * ml.y; acc[3] += paged_exp2(v[i].w - ml.x) * ml.y;
    }
  }
  const size_t at = (size_t)bh * a.c.table_pages * a.c.page_rows + row;
  #pragma unroll
  for (int i = 0; i < 4; ++i)
    if (row + i < L) a.weights_out[at + i] = (a.weights_in ? a.weights_in[at + i] : 0.f) + acc[i];
}

// Blocks of 16 query heads that a workgroup has of a key head's group: two where there are more than 16 (32 heads on a key head of 128 dims, 269 MB
// of bf16 cache: 46 us, with one block, and the keys read twice, 63; 64 dims 26 and 45).  Four are no faster for more (64 heads 68 and 69 us,
// 128 heads 110 and 103): one wave a SIMD is left.
int paged_query_blocks(int group) { return group > 16 ? 2 : 1; }

// A workgroup for every walk saves the launch of a fold, but a compute unit takes in some 60 GB/s, and unequal lengths are not evened out.  So:
// while the longest walk that the bound allows has few steps, more of them where there are walks for half of the compute units.  Measured (us;
// 32 query heads, bf16, 128 dims, alone / cut and joined): 32 walks of 512 rows 9.1 / 10.3, 768 10.9 / 10.4, 1024 13.3 / 11.2; 128 walks of 512
// 10.4 / 14.4, 1024 16.0 / 18.6, 1536 22.1 / 23.7; 256 walks of 1024 23.3 / 28.5, 2048 43.3 / 48.2 (there the bound says too little about
// lengths that differ).  Eight waves instead of four were no faster (32 walks of 1024 rows 13.8, 512 walks of 256 16.1 against 13.5).
static bool paged_alone(const PagedAttnArgs &a, int walks, int kstep) { return a.seqs.cap <= (walks >= 128 ? 8 : 4) * PAGED_WAVES * kstep; }

size_t paged_attn_ws_bytes(int n_seq, int n_heads, int n_kv, int d_h, int cap, bool weights, PagedAttnArgs *a, unsigned char *ws) {
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at = (at + n + 255) / 256 * 256; return ws ? ws + o : nullptr; };
  const int nq = 16 * paged_query_blocks(n_heads / n_kv);
  unsigned char *plan = take((size_t)(2 * n_seq + 1) * 4), *stats = take((size_t)n_seq * n_heads * 8);
  unsigned char *part = take((size_t)2 * PAGED_WGS * (nq * d_h + 2 * nq) * 4);
  unsigned char *scores = weights ? take((size_t)n_seq * n_heads * cap * 4) : nullptr;
  if (a) { a->plan = (int32_t *)plan; a->stats = (float2 *)stats; a->partials = (float *)part; a->scores = (float *)scores; }
  return at;
}

template <typename T, int DH, int NQB>
static hipError_t paged_attn_shape(hipStream_t st, PagedAttnArgs a) {
  using C = PA<T, DH, NQB>;
  a.group = a.n_heads / a.c.n_kv;
  a.n_qg = (a.group + C::NQ - 1) / C::NQ;
  a.walks = a.c.n_kv * a.n_qg;
  const int walks = a.seqs.n_seq * a.walks;
  const bool alone = paged_alone(a, walks, C::KSTEP), weights = a.weights_out != nullptr;
  if (alone)
    hipLaunchKernelGGL((k_paged_attn<T, DH, NQB, true>), dim3(walks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_paged_attn<T, DH, NQB, false>), dim3(PAGED_WGS), dim3(256), 0, st, a);
  const int row_wgs = weights && !(alone && a.n_qg == 1) ? (a.seqs.cap + PAGED_WROWS - 1) / PAGED_WROWS : 0;
  const unsigned grid = (alone ? 0 : a.seqs.n_seq * a.n_heads) + a.seqs.n_seq * a.c.n_kv * row_wgs;
  if (grid)
    hipLaunchKernelGGL((k_paged_fold<T, DH, NQB>), dim3(grid), dim3(256), 0, st, a, alone, std::max(row_wgs, 1));
  return hipGetLastError();
}

template <typename T>
hipError_t launch_paged_attn(hipStream_t st, const PagedAttnArgs &a, int d_h) {
  const int nqb = paged_query_blocks(a.n_heads / a.c.n_kv);
  if (d_h == 128) return nqb == 2 ? paged_attn_shape<T, 128, 2>(st, a) : paged_attn_shape<T, 128, 1>(st, a);
  return nqb == 2 ? paged_attn_shape<T, 64, 2>(st, a) : paged_attn_shape<T, 64, 1>(st, a);
}
template hipError_t launch_paged_attn<float>(hipStream_t, const PagedAttnArgs &, int);
template hipError_t launch_paged_attn<bf16_t>(hipStream_t, const PagedAttnArgs &, int);

// =====================================================================================================
// amph_paged_append
// A workgroup has one key step's rows of one sequence (those of them that are new) for some of the heads: first the rows' cosines
// and sines into LDS, then a wave takes head after head.  A step's values are turned round in registers, so that runs of rows are
// written at once; a few rows, as of a decoding step, and the ends among a lane's rows element by element.
// =====================================================================================================
// Sine and cosine of an angle in turns: the nearest quarter turn is taken off in 64 bits, what is left, up to half a quarter, goes through
// the Taylor polynomials (their next terms are 2e-9 and 2.5e-8 there), and the quarters swap and negate the two.
__device__ __forceinline__ void sincos_turns(double turns, float *sn, float *cs) {
  const double quarters = turns * 4.0, n = rint(quarters);
  const float x = (float)(quarters - n) * 1.57079632679f, x2 = x * x;
  const float s = x + x * x2 * (-1.0f / 6 + x2 * (1.0f / 120 + x2 * (-1.0f / 5040 + x2 * (1.0f / 362880))));
  const float c = 1.0f + x2 * (-0.5f + x2 * (1.0f / 24 + x2 * (-1.0f / 720 + x2 * (1.0f / 40320))));
  const int q = (int)(n - 4.0 * floor(n * 0.25));
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  *sn = q & 2 ? -a : a;
  *cs = (q + 1) & 2 ? -b : b;
}
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_paged_append(const PagedAppendArgs a, const PagedRope rope) {
  constexpr int PER = Elem<T>::PER, KSTEP = 4 * PER, HALF = DH / 2, LPR = HALF / PER, RPP = WAVE / LPR;   // LPR lanes: a row's pairs
  typedef T frag __attribute__((ext_vector_type(PER)));
  __shared__ __align__(16) float sm_c[KSTEP][HALF + 4], sm_s[KSTEP][HALF + 4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, b = blockIdx.y;
  const int len = a.seqs.kv_len[b], fresh = a.seqs.n_valid ? paged_new(a.seqs.n_new, a.seqs.n_valid[b]) : a.seqs.n_new;
  const int L = paged_rows(len, fresh, a.seqs.cap);
  if (L < 0) {                                         // (whole workgroup)
    if (tid == 0 && blockIdx.x == 0 && blockIdx.z == 0) atomicOr(a.dev_status, (unsigned)AMPH_DEV_KV_OVERFLOW);
    return;
  }
  const int step = len / KSTEP + blockIdx.x, row0 = max(step * KSTEP, len), row1 = min((step + 1) * KSTEP, L), live = row1 - row0;
  if (live <= 0) return;
  const int psteps = a.c.page_rows / KSTEP, pg = step / psteps;
  const int id = a.c.table[(size_t)b * a.c.table_pages + pg];
  if ((unsigned)id >= (unsigned)a.c.n_pages) {
    if (tid == 0) atomicOr(a.dev_status, (unsigned)AMPH_DEV_BAD_PAGE);
    return;
  }
  const int j0 = row0 - len, k0 = row0 - step * KSTEP;             // the first row among the new ones, and in its step
  const size_t new0 = (size_t)b * a.seqs.n_new + j0;
  for (int t = tid; t < live * HALF; t += 256) {
    const int r = t / HALF, i = t % HALF;
    // turns, in 64 bits: of a far position's angle 32 bits would leave a few places; then what is left of the last whole turn
    float sn, cs;
    sincos_turns((double)(a.pos ? a.pos[new0 + r] : row0 + r) * rope.turns[i], &sn, &cs);
    sm_c[r][i] = cs;
    sm_s[r][i] = sn;
  }
  __syncthreads();
  const size_t page = (size_t)id * a.c.page_stride + (size_t)(step - pg * psteps) * (KSTEP * DH);
  const int n_rot = (a.q ? a.n_heads : 0) + a.c.n_kv, n_units = n_rot + a.c.n_kv;
  for (int unit = blockIdx.z * 4 + wave; unit < n_units; unit += gridDim.z * 4) {
    const bool is_q = unit < n_rot - a.c.n_kv, is_v = unit >= n_rot;
    const int h = is_v ? unit - n_rot : is_q ? unit : unit - (n_rot - a.c.n_kv);
    if (!is_v) {
      const T *src = (const T *)(is_q ? a.q : a.k) + new0 * (is_q ? a.ld_q : a.ld_k) + (size_t)h * DH;
      const size_t ld = is_q ? a.ld_q : a.ld_k;
      T *dst = is_q ? (T *)a.q_out + (new0 * a.n_heads + h) * DH : (T *)a.c.k + page + (size_t)h * a.c.head_stride;
      const int p = (lane % LPR) * PER, r0 = lane / LPR;
      auto pass = [&](auto tag) {                      // N x RPP rows, all asked for before the first is used; past the last one: that again
        constexpr int N = decltype(tag)::value;
        frag lo[N], hi[N];
        #pragma unroll
        for (int i = 0; i < N; ++i) {
          const T *at = src + (size_t)min(r0 + i * RPP, live - 1) * ld + p;
          lo[i] = __builtin_nontemporal_load(reinterpret_cast<const frag *>(at));
          hi[i] = __builtin_nontemporal_load(reinterpret_cast<const frag *>(at + HALF));
        }
        #pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = r0 + i * RPP;
          if (r >= live) continue;
          float cs[PER], sn[PER];
          #pragma unroll
          for (int e = 0; e < PER; e += 4) { load4<float>(&sm_c[r][p + e], cs + e); load4<float>(&sm_s[r][p + e], sn + e); }
          frag x, y;
          #pragma unroll
          for (int e = 0; e < PER; ++e) {
            const float u = Elem<T>::to_f32(lo[i][e]), v = Elem<T>::to_f32(hi[i][e]);
            x[e] = Elem<T>::from_f32(u * cs[e] - v * sn[e]);
            y[e] = Elem<T>::from_f32(v * cs[e] + u * sn[e]);
          }
          T *to = is_q ? dst + (size_t)r * a.n_heads * DH : dst;
          *reinterpret_cast<frag *>(to + (is_q ? p : (int)k_tiled_index<T>(k0 + r, p, DH))) = x;
          *reinterpret_cast<frag *>(to + (is_q ? HALF + p : (int)k_tiled_index<T>(k0 + r, HALF + p, DH))) = y;
        }
      };
      if (live <= RPP) pass(Rows<1>{}); else pass(Rows<KSTEP / RPP>{});
      if (!is_q && lane < live) {
        const size_t at = ((size_t)b * a.c.n_kv + h) * a.c.table_pages * a.c.page_rows + row0 + lane;
        if (a.weights) a.weights[at] = 0.f;
        if (a.row_pos) a.row_pos[at] = a.pos ? a.pos[new0 + lane] : row0 + lane;
      }
    } else {
      const T *src = (const T *)a.v + new0 * a.ld_v + (size_t)h * DH;
      T *dst = (T *)a.c.v + page + (size_t)h * a.c.head_stride;
      // all rows are asked for before the first is stored (past the last one: that again)
      auto few = [&](auto tag) {
        constexpr int N = decltype(tag)::value;
        T x[N][DH / WAVE];
        #pragma unroll
        for (int r = 0; r < N; ++r)
          #pragma unroll
          for (int c = 0; c < DH / WAVE; ++c) x[r][c] = src[(size_t)min(r, live - 1) * a.ld_v + c * WAVE + lane];
        #pragma unroll
        for (int r = 0; r < N; ++r) {
          if (r >= live) break;
          #pragma unroll
          for (int c = 0; c < DH / WAVE; ++c) dst[v_tiled_index<T>(k0 + r, c * WAVE + lane, DH)] = x[r][c];
        }
      };
      if (live == 1) {
        few(Rows<1>{});
      } else if (live <= 4) {
        few(Rows<4>{});
      } else {
        constexpr int UN = DH / 16, LPV = DH / PER;    // a lane has UN adjacent rows of the step, PER adjacent dims of each
        typedef T run __attribute__((ext_vector_type(UN)));
        const int li = lane % LPV, first = (lane / LPV) * UN;
        frag x[UN];
        #pragma unroll
        for (int j = 0; j < UN; ++j) {
          const int r = min(max(first + j - k0, 0), live - 1);
          x[j] = __builtin_nontemporal_load(reinterpret_cast<const frag *>(src + (size_t)r * a.ld_v + li * PER));
        }
        if (first >= k0 && first + UN <= k0 + live) {
          #pragma unroll
          for (int e = 0; e < PER; ++e) {
            run y;
            #pragma unroll
            for (int j = 0; j < UN; ++j) y[j] = x[j][e];
            *reinterpret_cast<run *>(dst + v_tiled_index<T>(first, li * PER + e, DH)) = y;
          }
        } else {                                       // an end of the new rows lies among the lane's: one by one
          #pragma unroll
          for (int j = 0; j < UN; ++j) {
            if (first + j < k0 || first + j >= k0 + live) continue;
            #pragma unroll
            for (int e = 0; e < PER; ++e) dst[v_tiled_index<T>(first + j, li * PER + e, DH)] = x[j][e];
          }
        }
      }
    }
  }
}

template <typename T>
hipError_t launch_paged_append(hipStream_t st, const PagedAppendArgs &a, const PagedRope &rope, int d_h) {
  constexpr int KSTEP = 4 * Elem<T>::PER;
  const int steps = (a.seqs.n_new + KSTEP - 2) / KSTEP + 1, units = (a.q ? a.n_heads : 0) + 2 * a.c.n_kv;
  // Heads are spread over workgroups, as many for every wave.  Twelve waves are resident on each of 256 compute units; beyond, one head each would start anew for the rest, and
  // with unequal prompts part of the grid is idle.  Measured (us, heads a wave: 128 dims, bf16): four prompts of 256 to 1024 rows, 32 heads and as many key
  // heads, 1: 31.2, 2: 34.6, 3: 27.5, 4: 31.1, 6: 34.5; two of 1340 rows, 32 and 8 heads, 1: 22.1, 2: 18.5, 3: 19.9; one of 512 rows, 32 and
  // 32 heads, 1: 10.0, 2: 11.6.
  const long long all = (long long)steps * a.seqs.n_seq * units;
  const int m = (int)std::min<long long>(units, std::max<long long>(all / 4096, all > 12 * 256 ? 2 : 1)), z = (units + 4 * m - 1) / (4 * m);
  const dim3 grid(steps, a.seqs.n_seq, z);
  if (d_h == 128) hipLaunchKernelGGL((k_paged_append<T, 128>), grid, dim3(256), 0, st, a, rope);
  else hipLaunchKernelGGL((k_paged_append<T, 64>), grid, dim3(256), 0, st, a, rope);
  return hipGetLastError();
}
template hipError_t launch_paged_append<float>(hipStream_t, const PagedAppendArgs &, const PagedRope &, int);
template hipError_t launch_paged_append<bf16_t>(hipStream_t, const PagedAppendArgs &, const PagedRope &, int);

// =====================================================================================================
// amph_paged_evict
// k_evict: one workgroup for every (layer, sequence, key head).  A row's key is its weight as an ordered integer, all ones for the
//   newest rows.  The smallest kept key is found by counting: the range from the smallest to the largest key in 2048 bins, then
//   the bin that holds it the same way (spread over the range, the counters are hit by few lanes at once, however close the
//   exponents are).  Then the rows in their order: of equal keys the lowest are kept, the i-th kept row behind the budget gets the
//   i-th dropped place below it.  A step that drops one row (a cache at its budget) needs only the smallest key.
// The keys and values of the moved rows: by the same workgroup where few can move, or k_evict_move with a wave for every 16 moves.  Sources lie behind the budget and destinations below it, so no order is needed.
// =====================================================================================================
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}
struct MinU { __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return min(a, b); } };
struct MaxU { __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); } };
struct AddI { __device__ __forceinline__ int operator()(int a, int b) const { return a + b; } };

// Rows s[m] -> d[m] of one head for the 16 moves i0 .. i0 + 15 (of n), by one wave: lane = 16 moves x 4; a quarter of a 64-byte column
// of the keys, every fourth dim of the values.
template <typename T, int DH>
__device__ __forceinline__ void evict_move_rows(const PagedPages &c, const int32_t *row_table, size_t base, const int2 *moves, int i0, int n) {
  constexpr int PIECE = 64 / (int)sizeof(T), SEGS = DH / PIECE;
  const int lane = threadIdx.x & 63, m = lane & 15, sub = lane >> 4;
  const bool in = i0 + m < n;
  const int2 mv = moves[min(i0 + m, n - 1)];
  const int d = mv.x, s = mv.y, dp = d / c.page_rows, sp = s / c.page_rows, dr = d - dp * c.page_rows, sr = s - sp * c.page_rows;
  const size_t dpage = base + (size_t)row_table[dp] * c.page_stride, spage = base + (size_t)row_table[sp] * c.page_stride;
  T *K = (T *)c.k, *V = (T *)c.v;
  uint4 k[SEGS];
  #pragma unroll
  for (int p = 0; p < SEGS; ++p) k[p] = ldg16(K + spage + k_tiled_index<T>(sr, p * PIECE + sub * (PIECE / 4), DH));
  constexpr int UN = 16;
  #pragma unroll
  for (int c0 = 0; c0 < DH; c0 += 4 * UN) {
    T v[UN];
    #pragma unroll
    for (int e = 0; e < UN; ++e) if (c0 + e * 4 < DH) v[e] = V[spage + v_tiled_index<T>(sr, c0 + e * 4 + sub, DH)];
    if (in) {
      #pragma unroll
      for (int e = 0; e < UN; ++e) if (c0 + e * 4 < DH) V[dpage + v_tiled_index<T>(dr, c0 + e * 4 + sub, DH)] = v[e];
    }
  }
  if (in) {
    #pragma unroll
    for (int p = 0; p < SEGS; ++p) stg16(K + dpage + k_tiled_index<T>(dr, p * PIECE + sub * (PIECE / 4), DH), k[p]);
  }
}

// NT threads.  Rows are dealt in order to waves, groups, lanes, J to a lane; RPT > 0: a lane keeps the keys of its RPT rows in registers
// (cap <= NT * RPT; up to 16 rows their weights and positions too), 0: they are computed anew where they are needed.
template <typename T, int DH, int NT, int RPT>
__global__ __launch_bounds__(NT) void k_evict(const PagedEvictArgs a) {
  constexpr int NW = NT / WAVE, BINS = 2048, FEW = 64;
  constexpr bool HELD = RPT > 0, WHOLE = HELD && RPT <= 16;
  constexpr int J = HELD && RPT < 8 ? RPT : 8, GROUPS = HELD ? RPT / J : 1;
  typedef float fj __attribute__((ext_vector_type(J), aligned(4)));
  typedef int ij __attribute__((ext_vector_type(J), aligned(4)));
  extern __shared__ __align__(16) int sm_hole[];       // [most] places below the budget, ascending; [most] moves where they are made here (WHOLE)
  __shared__ int hist[BINS];
  __shared__ __align__(16) int sm_new[NW], sm_a[NW], sm_b[NW], sm_c[NW], sm_d[NW], sm_e[NW], sm_f[NW], sm_eq[NW];
  static_assert(NW <= 16, "a row of lanes has a value of every wave");
  __shared__ int sm_pick[3], sm_few;
  __shared__ unsigned sm_key[FEW];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, unit = blockIdx.x;
  const int h = unit % a.c.n_kv, b = (unit / a.c.n_kv) % a.seqs.n_seq, layer = unit / (a.c.n_kv * a.seqs.n_seq);
  const size_t at = (size_t)unit * a.c.table_pages * a.c.page_rows;
  const float *w = a.weights_in + at;
  const int32_t *pos = a.pos_in + at, *row_table = a.c.table + (size_t)b * a.c.table_pages;
  float *w_out = a.weights_out + at;
  int32_t *pos_out = a.pos_out + at;
  const int len = a.seqs.kv_len[b], R = paged_len(a.seqs, b), budget = a.budget;
  const int groups = HELD ? GROUPS : (max(R, 0) + NT * J - 1) / (NT * J);
  auto row_of = [&](int g) { return (wave * groups + g) * (WAVE * J) + lane * J; };
  auto load = [&](int g, fj &x, ij &p) {               // (J rows lie in cap places or behind them, as cap is a multiple of J)
    const int r = min(row_of(g), a.seqs.cap - J);
    x = *reinterpret_cast<const fj *>(w + r);
    p = *reinterpret_cast<const ij *>(pos + r);
  };
  fj wr[WHOLE ? GROUPS : 1];
  ij pr[WHOLE ? GROUPS : 1];
  const int live_groups = R <= 0 ? 0 : min(groups, (R - 1 - wave * groups * WAVE * J + WAVE * J) / (WAVE * J));      // (may be negative)
  if constexpr (WHOLE) {
    #pragma unroll
    for (int g = 0; g < GROUPS; ++g) if (g < live_groups) load(g, wr[g], pr[g]);
  }
  bool bad = R < 0;
  for (int i = tid; i < (max(R, 0) + a.c.page_rows - 1) / a.c.page_rows; i += NT) bad |= (unsigned)row_table[i] >= (unsigned)a.c.n_pages;
  auto lines = [&](auto f) {                           // f(g, first row of the lane, J weights, J positions)
    auto one = [&](int g) {
      fj x;
      ij p;
      load(g, x, p);
      f(g, row_of(g), x, p);
    };
    if constexpr (WHOLE) {
      #pragma unroll
      for (int g = 0; g < GROUPS; ++g) if (g < live_groups) f(g, row_of(g), wr[g], pr[g]);
    } else if constexpr (HELD) {
      #pragma unroll
      for (int g = 0; g < GROUPS; ++g) if (g < live_groups) one(g);
    } else {
      for (int g = 0; g < live_groups; ++g) one(g);
    }
  };
  // op over the waves' values, in every lane
  auto across = [&](const int *sm, auto op, auto none) {
    auto v = (lane & 15) < NW ? (decltype(none))sm[lane & 15] : none;
    v = op(v, lanes_ror<8>(v));
    v = op(v, lanes_ror<4>(v));
    v = op(v, lanes_ror<2>(v));
    return op(v, lanes_ror<1>(v));
  };
  int newest = INT32_MIN;
  lines([&](int, int row, const fj &, const ij &p) {
    #pragma unroll
    for (int j = 0; j < J; ++j) newest = row + j < R ? max(newest, p[j]) : newest;
  });
  newest = wave_max(newest);
  if (lane == 0) sm_new[wave] = newest;
  bad = __syncthreads_or(bad);
  if (h == 0 && layer == 0 && tid == 0) {              // one thread of the sequence
    const int now = bad ? len : min(R, budget);        // nothing changes for a sequence that is not sound
    if (a.kv_len_out) a.kv_len_out[b] = now; else a.new_len[b] = now;
    if (bad) atomicOr(a.dev_status, (unsigned)(R < 0 ? AMPH_DEV_KV_OVERFLOW : AMPH_DEV_BAD_PAGE));
  }
  if (!bad && (a.weights_in != a.weights_out || a.pos_in != a.pos_out))               // elsewhere: all places first, then what moves
    lines([&](int, int row, const fj &x, const ij &p) {
      const int end = min(R, budget);
      if (row + J <= end) {
        *reinterpret_cast<fj *>(w_out + row) = x;
        *reinterpret_cast<ij *>(pos_out + row) = p;
      } else {
        #pragma unroll
        for (int j = 0; j < J; ++j) if (row + j < end) { w_out[row + j] = x[j]; pos_out[row + j] = p[j]; }
      }
    });
  if (bad || R <= budget) {
    if (!a.fused && tid == 0) a.n_moves[unit] = 0;
    return;
  }
  newest = across(sm_new, MaxI(), (int)INT32_MIN);
  const long long safe_from = (long long)newest - a.recent;           // positions above it are kept first
  auto key_of = [&](float x, int p) -> unsigned { return (long long)p > safe_from ? 0xffffffffu : rank_key(x); };
  typedef unsigned uj __attribute__((ext_vector_type(J)));
  uj kr[GROUPS];
  auto line_keys = [&](int row, const fj &x, const ij &p, uj &k) {     // places behind the last row have the lowest key, as NaN has
    #pragma unroll
    for (int j = 0; j < J; ++j) k[j] = row + j < R ? key_of(x[j], p[j]) : 0u;
  };
  if constexpr (HELD) lines([&](int g, int row, const fj &x, const ij &p) { line_keys(row, x, p, kr[g]); });
  auto keys = [&](auto f) {                            // f(g, first row, J keys)
    if constexpr (HELD) {
      #pragma unroll
      for (int g = 0; g < GROUPS; ++g) if (g < live_groups) f(g, row_of(g), kr[g]);
    } else {
      lines([&](int g, int row, const fj &x, const ij &p) { uj k; line_keys(row, x, p, k); f(g, row, k); });
    }
  };
  // a sum over the waves before this one, and over all
  auto before = [&](const int *sm, int &all) {
    const int v = lane < NW ? sm[lane] : 0, s = wave_scan(v);
    all = __builtin_amdgcn_readlane(s, WAVE - 1);
    return __builtin_amdgcn_readlane(s, wave) - __builtin_amdgcn_readlane(v, wave);
  };
  int2 *moves = a.moves + (size_t)unit * a.most;
  int2 *fused_moves = reinterpret_cast<int2 *>(sm_hole + (a.most + 1) / 2 * 2);      // (WHOLE)
  const size_t base = (size_t)layer * a.c.layer_stride + (size_t)h * a.c.head_stride;

  if (R == budget + 1) {
    // ---- the smallest key goes, the last row of that key
    unsigned least = 0xffffffffu;
    keys([&](int, int row, const uj &k) {
      #pragma unroll
      for (int j = 0; j < J; ++j) least = row + j < R ? min(least, k[j]) : least;
    });
    least = wave_fold(least, MinU());
    int gone = -1;                                     // the wave's: waves have their rows in order, so the last one of the least key counts
    keys([&](int, int row, const uj &k) {
      #pragma unroll
      for (int j = 0; j < J; ++j) gone = row + j < R && k[j] == least ? row + j : gone;
    });
    gone = wave_max(gone);
    if (lane == 0) { sm_b[wave] = (int)least; sm_c[wave] = gone; }
    __syncthreads();
    least = 0xffffffffu;
    #pragma unroll
    for (int i = 0; i < NW; ++i)
      if (sm_c[i] >= 0 && (unsigned)sm_b[i] <= least) { least = (unsigned)sm_b[i]; gone = sm_c[i]; }
    const int2 one = make_int2(gone, budget);
    if (tid == 0 && a.fused && gone < budget) { w_out[gone] = w[budget]; pos_out[gone] = pos[budget]; }
    if (!a.fused) {
      if (tid == 0) { moves[0] = one; a.n_moves[unit] = gone < budget; }
    } else if (wave == 0 && gone < budget) {
      evict_move_rows<T, DH>(a.c, row_table, base, &one, 0, 1);
    }
    return;
  }

  // ---- the smallest kept key: `want` of the keys in [lo, hi] are kept.  Weights are hardly ever negative, and often zero: the positive ones
  // are a range of their own (many zeros would wait for one counter, and lie far from the smallest other weight)
  constexpr unsigned ZERO = 0x80000000u;
  unsigned lo = 0xffffffffu, hi = 0u;
  for (int i = tid; i < BINS; i += NT) hist[i] = 0;
  if (tid == 0) sm_few = 0;
  int over_zero = 0, safe = 0;                         // rows above zero, and newest ones
  keys([&](int, int, const uj &k) {
    #pragma unroll
    for (int j = 0; j < J; ++j) {
      const bool fixed = k[j] == 0xffffffffu, over = k[j] > ZERO;
      over_zero += over ? 1 : 0;
      safe += fixed ? 1 : 0;
      lo = over ? min(lo, k[j]) : lo;
      hi = fixed ? hi : max(hi, k[j]);
    }
  });
  over_zero = wave_fold(over_zero, AddI());
  safe = wave_fold(safe, AddI());
  lo = wave_fold(lo, MinU());
  hi = wave_fold(hi, MaxU());
  if (lane == 0) { sm_a[wave] = safe; sm_b[wave] = (int)lo; sm_c[wave] = (int)hi; sm_e[wave] = over_zero; }
  __syncthreads();
  safe = across(sm_a, AddI(), 0);
  over_zero = across(sm_e, AddI(), 0);
  lo = across(sm_b, MinU(), 0xffffffffu);
  hi = across(sm_c, MaxU(), 0u);
  int want = budget - safe;
  bool all_equal = false;                              // all keys from lo on are kept
  bool search = true;
  if (want <= 0) { lo = 0xffffffffu; want = budget; search = false; }
  else if (over_zero < budget) {                       // zero weights, negative ones or NaN are kept too
    int some = 0;                                      // rows of any key but the lowest
    lo = 0xffffffffu;
    hi = ZERO;
    keys([&](int, int, const uj &k) {
      #pragma unroll
      for (int j = 0; j < J; ++j) { some += k[j] != 0u ? 1 : 0; lo = k[j] ? min(lo, k[j]) : lo; }
    });
    some = wave_fold(some, AddI());
    lo = wave_fold(lo, MinU());
    if (lane == 0) { sm_d[wave] = some; sm_f[wave] = (int)lo; }
    __syncthreads();
    some = across(sm_d, AddI(), 0);
    lo = across(sm_f, MinU(), 0xffffffffu);
    if (some < budget) { lo = 0u; want = budget - some; search = false; }
    else { want = budget - over_zero; search = lo != ZERO; }
  }
  if (search) {
    for (;;) {
      const unsigned span = hi - lo;
      const int shift = span >> 11 ? 21 - __clz(span) : 0;             // (bins: span >> shift < 2048)
      keys([&](int, int, const uj &k) {
        #pragma unroll
        for (int j = 0; j < J; ++j) if (k[j] - lo <= span) atomicAdd(&hist[(k[j] - lo) >> shift], 1);
      });
      __syncthreads();
      // from the top, thread t has PB bins; the bin at which the count reaches `want`
      constexpr int PB = BINS / NT;
      int c[PB], mine = 0;
      #pragma unroll
      for (int i = 0; i < PB; ++i) { c[i] = hist[BINS - 1 - (tid * PB + i)]; mine += c[i]; }
      int upto = wave_scan(mine);
      if (lane == WAVE - 1) sm_new[wave] = upto;
      __syncthreads();
      #pragma unroll
      for (int i = 0; i < PB; ++i) hist[BINS - 1 - (tid * PB + i)] = 0;
      int all;
      upto += before(sm_new, all);
      int above = upto - mine;
      if (upto >= want && above < want) {
        #pragma unroll
        for (int i = 0; i < PB; ++i) {
          if (above < want && above + c[i] >= want) { sm_pick[0] = BINS - 1 - (tid * PB + i); sm_pick[1] = want - above; sm_pick[2] = c[i]; above = want; }
          else if (above < want) above += c[i];
        }
      }
      __syncthreads();
      lo += (unsigned)sm_pick[0] << shift;
      hi = min(hi, lo + ((1u << shift) - 1));
      want = sm_pick[1];
      const int in_bin = sm_pick[2];
      all_equal = in_bin == want;
      if (shift == 0 || all_equal) break;
      if (in_bin <= FEW) {
        // ---- few keys left: one wave ranks them; the want-th largest, and how many are larger
        const unsigned few_span = hi - lo;
        keys([&](int, int, const uj &k) {
          #pragma unroll
          for (int j = 0; j < J; ++j) if (k[j] - lo <= few_span) sm_key[atomicAdd(&sm_few, 1)] = k[j];
        });
        __syncthreads();
        if (wave == 0) {
          const unsigned own = lane < in_bin ? sm_key[lane] : 0u;      // (in the order they came: only their values count)
          int larger = 0, same = 0;
          for (int s = 0; s < in_bin; ++s) {
            const unsigned o = (unsigned)__builtin_amdgcn_readlane((int)own, s);
            larger += o > own ? 1 : 0;
            same += o == own ? 1 : 0;
          }
          if (lane < in_bin && larger < want && larger + same >= want) {       // (lanes of the same key write the same)
            sm_pick[0] = (int)own;
            sm_pick[1] = want - larger;
            sm_pick[2] = same;
          }
        }
        __syncthreads();
        lo = (unsigned)sm_pick[0];
        want = sm_pick[1];
        all_equal = sm_pick[2] == want;
        break;
      }
    }
  }
  // ---- kept: all keys above lo, and of those that are lo the first `want`; then the places below the budget and the rows behind it
  const unsigned from_key = lo;
  int eq = 0;
  if (!all_equal) {
    keys([&](int, int row, const uj &k) {
      #pragma unroll
      for (int j = 0; j < J; ++j) eq += k[j] == from_key && row + j < R ? 1 : 0;
    });
    eq = wave_fold(eq, AddI());
    if (lane == 0) sm_eq[wave] = eq;
    __syncthreads();
    int all;
    eq = before(sm_eq, all);
  }
  const int eq_before = eq;
  // the J rows that a lane keeps, as bits; all lanes, groups in order (eq: the equal keys before the group)
  auto kept = [&](int row, const uj &k) {
    unsigned keep = 0;
    if (all_equal) {                                   // (lo is not the lowest key, which has no bin)
      #pragma unroll
      for (int j = 0; j < J; ++j) keep |= (k[j] >= from_key ? 1u : 0u) << j;
    } else {
      unsigned same = 0;
      #pragma unroll
      for (int j = 0; j < J; ++j) {
        keep |= (k[j] > from_key ? 1u : 0u) << j;
        same |= (k[j] == from_key && row + j < R ? 1u : 0u) << j;      // (the lowest key is also that of places that are no rows)
      }
      const int mine = __popc(same), upto = wave_scan(mine);
      int left = want - eq - (upto - mine);            // of the lane's equal keys, so many are kept: its first
      #pragma unroll
      for (int j = 0; j < J; ++j) if (same >> j & 1u) { if (left > 0) keep |= 1u << j; --left; }
      eq += __builtin_amdgcn_readlane(upto, WAVE - 1);
    }
    return keep;
  };
  auto below = [&](int row) { return row >= budget ? 0u : budget - row >= J ? (1u << J) - 1 : (1u << (budget - row)) - 1; };
  unsigned bits[GROUPS];                               // (HELD: found once)
  int n_hole = 0, n_from = 0;
  keys([&](int g, int row, const uj &k) {
    const unsigned keep = kept(row, k), lt = below(row);
    if constexpr (HELD) bits[g] = keep;
    n_hole += __popc(~keep & lt);
    n_from += __popc(keep & ~lt);
  });
  n_hole = wave_fold(n_hole, AddI());
  n_from = wave_fold(n_from, AddI());
  if (lane == 0) { sm_a[wave] = n_hole; sm_c[wave] = n_from; }         // (read by all: a barrier of the search or of the equal keys is behind)
  __syncthreads();
  int total;
  n_hole = before(sm_a, total);
  n_from = before(sm_c, total);
  const int from0 = n_from;
  auto listed = [&](auto f) {                          // f(bits of the lane's kept rows, its first row)
    eq = eq_before;
    if constexpr (HELD) {
      #pragma unroll
      for (int g = 0; g < GROUPS; ++g) if (g < live_groups) f(bits[g], row_of(g));
    } else {
      keys([&](int, int row, const uj &k) { f(kept(row, k), row); });
    }
  };
  listed([&](unsigned keep, int row) {
    unsigned m = ~keep & below(row);
    const int mine = __popc(m), upto = wave_scan(mine);
    for (int i = n_hole + upto - mine; m; m &= m - 1, ++i) {
      const int r = row + __builtin_ctz(m);
      if constexpr (WHOLE) sm_hole[i] = r; else moves[i].x = r;
    }
    n_hole += __builtin_amdgcn_readlane(upto, WAVE - 1);
  });
  __syncthreads();
  n_from = from0;
  listed([&](unsigned keep, int row) {
    unsigned m = keep & ~below(row);
    const int mine = __popc(m), upto = wave_scan(mine);
    for (int i = n_from + upto - mine; m; m &= m - 1, ++i) {
      const int r = row + __builtin_ctz(m);
      if constexpr (WHOLE) {
        const int2 mv = make_int2(sm_hole[i], r);
        if (a.fused) fused_moves[i] = mv; else moves[i] = mv;
      } else {
        moves[i].y = r;
      }
    }
    n_from += __builtin_amdgcn_readlane(upto, WAVE - 1);
  });
  if (!a.fused) {                                      // k_evict_move makes them
    if (tid == 0) a.n_moves[unit] = total;
    return;
  }
  __syncthreads();
  for (int i = tid; i < total; i += NT) {              // (rows behind the budget, which nobody writes, to places below it)
    int2 mv;
    if constexpr (WHOLE) mv = fused_moves[i]; else mv = moves[i];
    w_out[mv.x] = w[mv.y];
    pos_out[mv.x] = pos[mv.y];
  }
  for (int i0 = wave * 16; i0 < total; i0 += NW * 16) {
    if constexpr (WHOLE) evict_move_rows<T, DH>(a.c, row_table, base, fused_moves, i0, total);
    else evict_move_rows<T, DH>(a.c, row_table, base, moves, i0, total);
  }
}

constexpr int EVICT_MOVES = 16;                        // moves of a workgroup, which is a wave

// Many moves.  Bound by HBM: a value row's dims lie 64 bytes apart, each among the same dim of its step's other rows, so the lines of every
// step that a row leaves or enters move.  8191 -> 2048 rows in 16 heads of 128 dims (1640 moves each, 27 MB of rows in 51 MB of lines):
// 14.8 us; in workgroups of four waves 16.6 (416 of them on 256 compute units); whole steps through LDS, where the rows change places, 16.8
// and 18.0 us (a wave for all dims, and for a quarter).
template <typename T, int DH>
__global__ __launch_bounds__(WAVE) void k_evict_move(const PagedEvictArgs a, int32_t *kv_len_out) {
  const int lane = threadIdx.x, unit = blockIdx.x;
  const int h = unit % a.c.n_kv, b = (unit / a.c.n_kv) % a.seqs.n_seq, layer = unit / (a.c.n_kv * a.seqs.n_seq);
  if (!a.kv_len_out && h == 0 && layer == 0 && blockIdx.y == 0 && lane == 0) kv_len_out[b] = a.new_len[b];
  if (a.fused) return;
  const int n = a.n_moves[unit];
  const size_t base = (size_t)layer * a.c.layer_stride + (size_t)h * a.c.head_stride;
  const int2 *moves = a.moves + (size_t)unit * a.most;
  const size_t at = (size_t)unit * a.c.table_pages * a.c.page_rows;
  for (int i0 = blockIdx.y * EVICT_MOVES; i0 < n; i0 += gridDim.y * EVICT_MOVES) {
    if (lane < EVICT_MOVES && i0 + lane < n) {
      const int2 mv = moves[i0 + lane];
      a.weights_out[at + mv.x] = a.weights_in[at + mv.y];
      a.pos_out[at + mv.x] = a.pos_in[at + mv.y];
    }
    evict_move_rows<T, DH>(a.c, a.c.table + (size_t)b * a.c.table_pages, base, moves, i0, n);
  }
}

// Up to so many moves a head the workgroup that chose them makes them itself: a cache that is held to a budget drops a row or a few a step, and has
// up to a page more than the budget.  Measured (us, 16 heads of 128 dims): one move 5.6 in all; 112 moves 10.6, by a launch of their own some 11.4;
// 212 moves 12.0 and 11.4.
constexpr int EVICT_FUSED = 256;

size_t paged_evict_ws_bytes(int n_layers, int n_seq, int n_kv, int cap, int budget, PagedEvictArgs *a, unsigned char *ws) {
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at = (at + n + 255) / 256 * 256; return ws ? ws + o : nullptr; };
  const size_t units = (size_t)n_layers * n_seq * n_kv;
  const int most = budget ? std::max(std::min(budget, cap - budget), 1) : cap / 2;       // (budget 0: whatever it will be)
  unsigned char *len = take((size_t)n_seq * 4), *n_moves = take(units * 4), *moves = take(units * most * 8);
  if (a) { a->new_len = (int32_t *)len; a->n_moves = (int32_t *)n_moves; a->moves = (int2 *)moves; a->most = most; }
  return at;
}

template <typename T, int DH>
static hipError_t paged_evict_shape(hipStream_t st, PagedEvictArgs a, int n_layers) {
  const unsigned units = (unsigned)n_layers * a.seqs.n_seq * a.c.n_kv;
  int32_t *const len_out = a.kv_len_out;
  const bool same_len = len_out == a.seqs.kv_len;      // other workgroups may still read it: a launch behind this one writes it
  if (same_len) a.kv_len_out = nullptr;
  a.fused = a.most <= EVICT_FUSED;
  const int cap = a.seqs.cap;
  const size_t lds = (size_t)a.most * (a.fused ? 12 : 4) + 8;
  #define EVICT(NT, RPT) hipLaunchKernelGGL((k_evict<T, DH, NT, RPT>), dim3(units), dim3(NT), RPT && RPT <= 16 ? lds : 0, st, a)
  // Threads by the rows that a sequence may have: what one workgroup holds in registers.  (512 threads instead of 256 up to 2048 rows: 256 heads that drop
  // a row each 5.5 us against 5.8, but 2048 of them 21.0 against 16.7; instead of 1024 up to 8192 rows 13.1 and 12.9.)
  if (cap <= 512) EVICT(256, 2);
  else if (cap <= 2048) EVICT(256, 8);
  else if (cap <= 8192) EVICT(1024, 8);
  else if (cap <= 16384) EVICT(1024, 16);
  else if (cap <= 32768) EVICT(1024, 32);
  else if (cap <= 65536) EVICT(1024, 64);
  else EVICT(1024, 0);
  #undef EVICT
  if (!a.fused)
    hipLaunchKernelGGL((k_evict_move<T, DH>), dim3(units, std::min((a.most + EVICT_MOVES - 1) / EVICT_MOVES, 65535)), dim3(WAVE), 0, st, a, len_out);
  else if (same_len)
    hipLaunchKernelGGL((k_evict_move<T, DH>), dim3(a.seqs.n_seq * a.c.n_kv), dim3(WAVE), 0, st, a, len_out);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_paged_evict(hipStream_t st, const PagedEvictArgs &a, int n_layers, int d_h) {
  return d_h == 128 ? paged_evict_shape<T, 128>(st, a, n_layers) : paged_evict_shape<T, 64>(st, a, n_layers);
}
template hipError_t launch_paged_evict<float>(hipStream_t, const PagedEvictArgs &, int, int);
template hipError_t launch_paged_evict<bf16_t>(hipStream_t, const PagedEvictArgs &, int, int);

}  // namespace amph
