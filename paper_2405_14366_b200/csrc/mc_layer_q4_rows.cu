// Rows into and out of a layer held in 4 bits.
//   layer_q4_append_kernel  rows behind the cached tokens: complete pages are quantised, the others stay 16-bit
//   layer_q4_read_kernel    code * scale + zero of a range of tokens, as 16-bit rows
// 512 bytes of 16-bit rows and 160 of codes and parameters per (token, kv head) are what they cannot do without: 107 us each for
// 8 x 4096 tokens of 32 heads.  Reading takes 127 us; writing 153 (bfloat16 176: no mixed-precision subtraction), with no unit at its limit
// (61 % of the issue slots, ALU 41 %, memory 52 %): 1500 instructions per page of K or V in 16 warps an SM, whose latencies show.
// Keys with a channel whose scale is subnormal take the exact code for the whole page: 307 us if every page has one; values for four rows:
// 233 us if every eighth row is next to zero.  A warp takes one (page, kv head) -- of K or V when it writes -- with all its loads in flight at once; neighbouring warps
// take neighbouring heads, whose parts of a row are next to each other.
#include <algorithm>

#include "mc_kernels.h"
#include "mc_layer.h"
#include "mc_layer_q4.cuh"
#include "mc_layer_q4.h"

namespace mc {

constexpr int kLrThreads = 256;
constexpr int kLrWarps = kLrThreads / 32;

struct Q4RowParams {
  Geom g;
  unsigned char* codes[2];  // K, V
  unsigned char* meta[2];
  char* res[2];
  int32_t* status;
  char* rows[2];  // the caller's K and V rows
  long long stride[2];
  const int32_t* row_offsets;
  const int32_t* begin;
  int n_rows;
};

// Rows of sequence b: [first, first + count) of the caller's arrays.
__device__ __forceinline__ void rows_of(const Q4RowParams& p, int b, int& first, int& count, int& bad) {
  const int r0 = p.row_offsets[b], r1 = p.row_offsets[b + 1];
  const bool ok = r0 >= 0 && r1 >= r0 && r1 <= p.n_rows;
  bad |= ok ? 0 : 1;
  first = ok ? r0 : 0;
  count = ok ? r1 - r0 : 0;
}
__device__ __forceinline__ int len_of(const Q4RowParams& p, int b, int& bad) {
  const int n = __ldcg(p.g.seq_lens + b);
  if (n < 0 || n > p.g.max_seq_len) bad = 1;
  return min(max(n, 0), p.g.max_seq_len);
}
// The pool slot of (sequence, page slot, kv head); -1 (flagged) if there is no such page.
__device__ __forceinline__ long long tile_of(const Q4RowParams& p, int b, int slot, int head) {
  const int page = checked_page(p.g, b, slot, p.status);
  return page < 0 ? -1 : (long long)page * p.g.n_kv_heads + head;
}

// Item counts to their prefix.  True: an offset is out of range or falls, and the call does nothing (offsets that rise are
// what bounds the items of the batch by the rows that there are).
__device__ __forceinline__ bool all_rows_bad(const Q4RowParams& p, int* pre, int bad, int bad_rows) {
  const bool none = __syncthreads_or(bad_rows) != 0;
  if ((bad || bad_rows) && blockIdx.x == 0) atomicOr(p.status, MC_FLAG_BAD_METADATA);
  if (!none) scan_counts(pre, p.g.batch);
  return none;
}

struct AppendItem {
  int n, first, count;  // cached tokens, the sequence's rows
};

// An item is a page that the call completes, or -- where it completes none -- the rows of the begun page.  The first
// item of a sequence also leaves the rows behind its last complete page in the begun page's place, after the warp has read
// what was there.  A warp keeps the page that it works on in shared memory and the next one, on its way, in registers.
struct AppendWork {
  int b, head, tensor, slot;
  bool page, first;  // a page to quantise; the sequence's first item
};

template <int DT>
__global__ void __launch_bounds__(kLrThreads, 2) layer_q4_append_kernel(const __grid_constant__ Q4RowParams p) {
  grid_dep_launch();
  extern __shared__ __align__(16) unsigned char tile_smem[];  // [warps][8 KB]
  __shared__ int pre_s[kMaxLayerBatch + 1];
  __shared__ AppendItem seq_s[kMaxLayerBatch];
  const int tid = threadIdx.x, lane = tid & 31, H = p.g.n_kv_heads;
  int bad = 0, bad_rows = 0;
  grid_dep_wait();  // (the offsets and lengths may be what the kernel ahead has written)
  for (int b = tid; b < p.g.batch; b += kLrThreads) {
    AppendItem s;
    int no_len = 0;
    s.n = len_of(p, b, no_len);
    rows_of(p, b, s.first, s.count, bad_rows);
    if (no_len) s.count = 0;  // (rows would land on cached ones)
    bad |= no_len;
    seq_s[b] = s;
    pre_s[b + 1] = s.count == 0 ? 0 : max((s.n + s.count) / kLqPage - s.n / kLqPage, 1);
  }
  if (all_rows_bad(p, pre_s, bad, bad_rows)) return;
  unsigned char* tile = tile_smem + (tid >> 5) * kLqResBytes;
  const int ch = lane & 15, half = lane >> 4;  // loading: half a warp has a row, a lane 16 bytes of it
  // A warp has columns (K or V, kv head) that do not change, and every `step`-th page: as many pages as there are warps for all
  // columns at a time (or, with more columns than warps, one, and several columns).
  const int pages = pre_s[p.g.batch], columns = 2 * H, warps = gridDim.x * kLrWarps, gw = blockIdx.x * kLrWarps + (tid >> 5);
  const int step = max(warps / columns, 1), pg0 = warps >= columns ? gw / columns : 0;
  int column = warps >= columns ? gw % columns : gw, pg = pg0, b_at = 0;
  if (pg0 >= step) column = columns;  // (a warp left over)
  AppendWork w;
  auto next = [&]() {  // the warp's next item into w; false behind the last one
    while (column < columns && pg >= pages) {
      column += warps >= columns ? columns : warps;
      pg = pg0;
      b_at = 0;
    }
    if (column >= columns) return false;
    while (pg >= pre_s[b_at + 1]) ++b_at;
    const AppendItem s = seq_s[b_at];
    w.b = b_at;
    w.tensor = column >= H ? 1 : 0;
    w.head = column - w.tensor * H;
    w.slot = s.n / kLqPage + pg - pre_s[b_at];
    w.page = w.slot < (s.n + s.count) / kLqPage;
    w.first = pg == pre_s[b_at];
    pg += step;
    return true;
  };
  auto row_at = [&](const AppendWork& w, const AppendItem& s, int t) -> const char* {  // token t: already in the begun page, or new
    return t < s.n ? p.res[w.tensor] + (((long long)w.b * H + w.head) * kLqPage + (t & (kLqPage - 1))) * kRowBytes
                   : p.rows[w.tensor] + (long long)w.head * kRowBytes + (long long)(s.first + t - s.n) * p.stride[w.tensor] * 2;
  };
  uint4 v[kLqPage / 2];
  auto fetch = [&](const AppendWork& w) {
    if (!w.page) return;
    const AppendItem s = seq_s[w.b];
    const int t0 = w.slot * kLqPage + half;
    if (t0 - half >= s.n) {  // all rows new: one address, a stride
      const char* src = row_at(w, s, t0) + 16 * ch;
      const long long two = p.stride[w.tensor] * 4;
#pragma unroll
      for (int k = 0; k < kLqPage / 2; ++k, src += two) v[k] = *reinterpret_cast<const uint4*>(src);
    } else {
#pragma unroll
      for (int k = 0; k < kLqPage / 2; ++k) v[k] = *reinterpret_cast<const uint4*>(row_at(w, s, t0 + 2 * k) + 16 * ch);
    }
  };

  bool more = next();
  if (more) fetch(w);
  while (more) {
    const AppendWork cur = w;
    if (cur.page) {
#pragma unroll
      for (int k = 0; k < kLqPage / 2; ++k) *reinterpret_cast<uint4*>(tile + (2 * k + half) * kRowBytes + 16 * ch) = v[k];
    }
    __syncwarp();
    more = next();
    if (more) fetch(w);
    if (cur.page) {
      const long long at = tile_of(p, cur.b, cur.slot, cur.head);
      if (at >= 0)
        lq_quantise<DT>(cur.tensor == 0, [&](int t) { return *reinterpret_cast<const uint4*>(tile + t * kRowBytes + 16 * ch); },
                        p.codes[cur.tensor] + at * kLqCodeBytes, p.meta[cur.tensor] + at * kLqMetaBytes);
    }
    if (cur.first) {
      const AppendItem s = seq_s[cur.b];
      const int t1 = s.n + s.count;
      char* res = p.res[cur.tensor] + ((long long)cur.b * H + cur.head) * kLqResBytes + 16 * ch;
      for (int t = max(t1 / kLqPage * kLqPage, s.n) + half; t < t1; t += 2)
        *reinterpret_cast<uint4*>(res + (t & (kLqPage - 1)) * kRowBytes) = *reinterpret_cast<const uint4*>(row_at(cur, s, t) + 16 * ch);
    }
    __syncwarp();  // (the tile has been read)
  }
}

// code * scale + zero of two channels.  Binary16: one packed FMA, rounded once; bfloat16: in binary32, then rounded.
template <int DT>
__device__ __forceinline__ uint32_t lq_value(uint32_t code, uint32_t m0, uint32_t m1) {
  if (DT == MC_F16) {
    const uint32_t s = __byte_perm(m0, m1, 0x5410), z = __byte_perm(m0, m1, 0x7632);
    __half2 v = __hfma2(*reinterpret_cast<__half2*>(&code), *reinterpret_cast<const __half2*>(&s), *reinterpret_cast<const __half2*>(&z));
    const __half2 most = __half2half2(__ushort_as_half((unsigned short)0x7BFF));
    v = __hmin2(__hmax2(v, __hneg2(most)), most);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  const float2 c = Elem<MC_F16>::unpack(code), a = Elem<MC_F16>::unpack(m0), b = Elem<MC_F16>::unpack(m1);
  return Elem<DT>::pack(fmaf(c.x, a.x, a.y), fmaf(c.y, b.x, b.y));
}
// Codes of bytes `i` of a word (channels 2i, 2i + 1) as two integers of binary16: the low one's unit in the mantissa of 1024,
// the high one's in that of 64.
__device__ __forceinline__ uint32_t lq_code_pair(uint32_t w, int i) {
  uint32_t b = (__byte_perm(w, 0, 0x0 | i | (0x4 << 4) | (i << 8) | (0x4 << 12)) & 0x00F0000Fu) | 0x54006400u;
  const uint32_t base = 0x54006400u;
  const __half2 v = __hsub2(*reinterpret_cast<__half2*>(&b), *reinterpret_cast<const __half2*>(&base));
  return *reinterpret_cast<const uint32_t*>(&v);
}

struct ReadItem {
  int n, begin, first, count;
};

// An item is a page of which tokens are wanted, of one kv head, K and V: half a warp has a row, a lane 8 channels.
template <int DT>
__global__ void __launch_bounds__(kLrThreads, 3) layer_q4_read_kernel(const __grid_constant__ Q4RowParams p) {
  grid_dep_launch();
  __shared__ int pre_s[kMaxLayerBatch + 1];
  __shared__ ReadItem seq_s[kMaxLayerBatch];
  const int tid = threadIdx.x, lane = tid & 31, H = p.g.n_kv_heads;
  const int ch = lane & 15, half = lane >> 4;
  int bad = 0, bad_rows = 0;
  grid_dep_wait();
  for (int b = tid; b < p.g.batch; b += kLrThreads) {
    ReadItem s;
    s.n = len_of(p, b, bad);
    rows_of(p, b, s.first, s.count, bad_rows);
    s.begin = p.begin ? p.begin[b] : 0;
    if (s.begin < 0) {
      bad = 1;
      s.begin = s.count = 0;
    }
    s.count = min(s.count, max(s.n - s.begin, 0));  // (n - begin: both at most 2^31 - 1 and not negative)
    seq_s[b] = s;
    pre_s[b + 1] = s.count == 0 ? 0 : (s.begin + s.count - 1) / kLqPage - s.begin / kLqPage + 1;
  }
  if (all_rows_bad(p, pre_s, bad, bad_rows)) return;
  const long long items = (long long)pre_s[p.g.batch] * H;
  const long long step = (long long)gridDim.x * kLrWarps;
  for (long long i = (long long)blockIdx.x * kLrWarps + (tid >> 5); i < items; i += step) {
    const int pg = (int)(i / H), head = (int)(i - (long long)pg * H);
    const int b = seq_of_item(pre_s, p.g.batch, pg);
    const ReadItem s = seq_s[b];
    const int slot = s.begin / kLqPage + pg - pre_s[b];
    const int t_page = slot * kLqPage;
    const int t0 = max(s.begin, t_page), t1 = min(s.begin + s.count, t_page + kLqPage);
    const bool full = t_page + kLqPage <= s.n;
    const long long tile = full ? tile_of(p, b, slot, head) : 0;
    if (tile < 0) continue;
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
      char* rows = p.rows[tensor] + (long long)head * kRowBytes + 16 * ch;
      const long long pitch = p.stride[tensor] * 2;
      if (full) {
        const uint32_t* codes = reinterpret_cast<const uint32_t*>(p.codes[tensor] + tile * kLqCodeBytes) + lane;
        const unsigned char* meta = p.meta[tensor] + tile * kLqMetaBytes;
        uint32_t w[16], m[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = codes[32 * k];  // row 2k + half
        if (tensor == 0) {
          *reinterpret_cast<uint4*>(m) = *reinterpret_cast<const uint4*>(meta + 32 * ch);
          *reinterpret_cast<uint4*>(m + 4) = *reinterpret_cast<const uint4*>(meta + 32 * ch + 16);
        } else {
#pragma unroll
          for (int k = 0; k < 16; ++k) m[k] = *reinterpret_cast<const uint32_t*>(meta + 16 * (2 * k + half) + 4 * (ch >> 2));
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int t = t_page + 2 * k + half;
          uint32_t v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t c = lq_code_pair(w[k], j);
            v[j] = tensor == 0 ? lq_value<DT>(c, m[2 * j], m[2 * j + 1]) : lq_value<DT>(c, m[k], m[k]);
          }
          if (t >= t0 && t < t1) st_stream16(rows + (long long)(s.first + t - s.begin) * pitch, make_uint4(v[0], v[1], v[2], v[3]));
        }
      } else {
        const char* res = p.res[tensor] + ((long long)b * H + head) * kLqResBytes + 16 * ch;
        for (int t = t0 + half; t < t1; t += 2)
          *reinterpret_cast<uint4*>(rows + (long long)(s.first + t - s.begin) * pitch) =
              *reinterpret_cast<const uint4*>(res + (long long)(t & (kLqPage - 1)) * kRowBytes);
      }
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------
static Q4RowParams row_params(const Geom& g, const mc_layer_q4_cache* layer, void* k, void* v, const Q4RowArgs& rows) {
  Q4RowParams p;
  p.g = g;
  p.codes[0] = (unsigned char*)layer->k_codes;
  p.codes[1] = (unsigned char*)layer->v_codes;
  p.meta[0] = (unsigned char*)layer->k_meta;
  p.meta[1] = (unsigned char*)layer->v_meta;
  p.res[0] = (char*)layer->res_k;
  p.res[1] = (char*)layer->res_v;
  p.status = layer->status;
  p.rows[0] = (char*)k;
  p.rows[1] = (char*)v;
  p.stride[0] = rows.k_stride;
  p.stride[1] = rows.v_stride;
  p.row_offsets = rows.row_offsets;
  p.begin = rows.begin;
  p.n_rows = rows.n_rows;
  return p;
}
// CTAs for n_rows rows, whose pages are not known here: each sequence may add a page at both ends.
static int row_ctas(const mc_batch* bt, int n_rows, int per_page, int most) {
  const long long items = ((long long)n_rows / kLqPage + 2LL * bt->batch) * per_page;
  return (int)std::max<long long>(1, std::min<long long>((items + kLrWarps - 1) / kLrWarps, most));
}

mc_status launch_layer_q4_append(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer, const void* k,
                                 const void* v, const Q4RowArgs& rows, cudaStream_t stream) {
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  auto* kernel = cfg->dtype == MC_F16 ? layer_q4_append_kernel<MC_F16> : layer_q4_append_kernel<MC_BF16>;
  MC_CUDA_CHECK(allow_smem(kernel, kLrWarps * kLqResBytes));
  MC_CUDA_CHECK(launch_pdl(kernel, dim3(row_ctas(bt, rows.n_rows, 2 * cfg->n_kv_heads, 2 * n_sm)), dim3(kLrThreads), kLrWarps * kLqResBytes,
                           stream, row_params(g, layer, const_cast<void*>(k), const_cast<void*>(v), rows)));
  return MC_OK;
}

mc_status launch_layer_q4_read(const mc_config* cfg, const mc_batch* bt, const Geom& g, const mc_layer_q4_cache* layer, void* k, void* v,
                               const Q4RowArgs& rows, cudaStream_t stream) {
  int n_sm = 0;
  if (mc_status st = sm_count(&n_sm)) return st;
  auto* kernel = cfg->dtype == MC_F16 ? layer_q4_read_kernel<MC_F16> : layer_q4_read_kernel<MC_BF16>;
  MC_CUDA_CHECK(launch_pdl(kernel, dim3(row_ctas(bt, rows.n_rows, cfg->n_kv_heads, 3 * n_sm)), dim3(kLrThreads), 0, stream,
                           row_params(g, layer, k, v, rows)));
  return MC_OK;
}

}  // namespace mc
