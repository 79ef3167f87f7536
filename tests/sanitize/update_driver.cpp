// Drives the host code of the row norm, the gradient norm, clipping and the Adam update through the C ABI for the
// sanitizer build (test infrastructure): launch tables of every size, lists in and out of order, overlaps.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "aecct.h"

#define EXPECT(x, st) do { aecct_status s_ = (x); if (s_ != (st)) { std::printf("FAIL %s:%d %s -> %d, expected %d\n", __FILE__, __LINE__, #x, (int)s_, (int)(st)); return 1; } } while (0)

typedef std::vector<aecct_tensor> List;

// n tensors of count(i) values of type(i): back to back from an odd place, or apart, ascending or not
static List make_list(std::vector<unsigned char> &mem, int n, int kind, bool apart, bool down, int type) {
  List l(n);
  size_t off = 4;
  mem.resize((size_t)n * 5000 * 4 + 4096);
  for (int i = 0; i < n; ++i) {
    const int k = down ? n - 1 - i : i;
    const int64_t count = kind == 0 ? 1 : kind == 1 ? (i * 37) % 4999 : (i % 3 ? 0 : 1025);
    const int t = type < 3 ? type : k % 3;
    off = (off + 3) / 4 * 4;
    l[k] = aecct_tensor{mem.data() + off, count, t};
    off += (size_t)count * (t == AECCT_F32 ? 4 : 2) + (apart ? 64 : 0);
  }
  return l;
}

int main() {
  int64_t step = 0;
  float norm = 0;
  for (int n : {0, 1, 2, 23, 24, 25, 56, 57, 96, 97, 160, 161, 400})
    for (int kind = 0; kind < 3; ++kind)
      for (int variant = 0; variant < 4; ++variant)
        for (int type = 0; type < 4; ++type) {
          std::vector<unsigned char> mem[5];
          const bool apart = variant & 1, down = variant & 2;
          const List g = make_list(mem[0], n, kind, apart, down, type), o = make_list(mem[1], n, kind, apart, down, 0),
                     p = make_list(mem[2], n, kind, apart, down, 0), m = make_list(mem[3], n, kind, apart, down, 0),
                     v = make_list(mem[4], n, kind, apart, down, 0);
          size_t need = 0;
          EXPECT(aecct_update_workspace_size(n, &need), AECCT_OK);
          std::vector<unsigned char> ws(need);
          EXPECT(aecct_grad_norm(g.data(), n, &norm, ws.data(), need, nullptr), AECCT_OK);
          EXPECT(aecct_grad_norm(g.data(), n, &norm, ws.data(), need - 1, nullptr), AECCT_ERR_WORKSPACE_TOO_SMALL);
          EXPECT(aecct_grad_clip(g.data(), nullptr, n, 1.0, &norm, ws.data(), need, nullptr), AECCT_OK);
          EXPECT(aecct_grad_clip(g.data(), o.data(), n, 1.0, &norm, ws.data(), need, nullptr), AECCT_OK);
          aecct_adam_options opt{1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, nullptr};
          EXPECT(aecct_adam_step(p.data(), m.data(), v.data(), g.data(), nullptr, n, &opt, &step, &norm, ws.data(), need, nullptr), AECCT_OK);
          EXPECT(aecct_adam_step(p.data(), m.data(), v.data(), g.data(), o.data(), n, &opt, &step, nullptr, ws.data(), need, nullptr), AECCT_OK);
          opt.max_norm = 0;
          EXPECT(aecct_adam_step(p.data(), m.data(), v.data(), g.data(), nullptr, n, &opt, &step, nullptr, ws.data(), need, nullptr), AECCT_OK);
          bool any = false;
          for (const auto &t : p) any = any || t.count;
          if (any) EXPECT(aecct_adam_step(p.data(), p.data(), v.data(), g.data(), nullptr, n, &opt, &step, nullptr, ws.data(), need, nullptr), AECCT_ERR_INVALID_ARG);
        }
  for (int64_t d : {1, 31, 32, 100, 512, 2048, 5000, 16384, 30000, 65536})
    for (int type = 0; type < 3; ++type)
      for (int64_t rows : {0, 1, 3, 70}) {
        std::vector<float> x(rows * d + 1), r(rows * d + 1), y(rows * d + 1), h(rows * d + 1), gain(d), dgain(d), alpha(rows * (d / 32 + 1) + 1);
        std::vector<int8_t> codes(rows * d + 1);
        aecct_rms_norm_args a{};
        a.rows = rows; a.d = d; a.type = type; a.gain_type = AECCT_F32; a.eps = 1e-5f; a.code_type = AECCT_CODE_I8; a.group = 32;
        a.x = x.data(); a.ldx = d; a.res = r.data(); a.ldres = d; a.gain = gain.data(); a.h = h.data(); a.ldh = d; a.y = y.data(); a.ldy = d;
        a.codes = codes.data(); a.ldcodes = d; a.alpha = alpha.data();
        EXPECT(aecct_rms_norm(&a, nullptr), AECCT_OK);
        a.ldx = (int64_t)1 << 62;
        if (rows) EXPECT(aecct_rms_norm(&a, nullptr), AECCT_ERR_INVALID_ARG);
        aecct_rms_norm_grad_args b{};
        b.rows = rows; b.d = d; b.type = type; b.gain_type = AECCT_F32; b.eps = 1e-5f;
        b.h = h.data(); b.ldh = d; b.dy = y.data(); b.lddy = d; b.dres = r.data(); b.lddres = d; b.gain = gain.data(); b.dh = x.data(); b.lddh = d; b.dgain = dgain.data();
        size_t need = 0;
        EXPECT(aecct_rms_norm_grad_workspace_size(rows, d, &need), AECCT_OK);
        std::vector<unsigned char> ws(need);
        EXPECT(aecct_rms_norm_grad(&b, ws.data(), need, nullptr), AECCT_OK);
      }
  std::printf("update driver ok\n");
  return 0;
}
