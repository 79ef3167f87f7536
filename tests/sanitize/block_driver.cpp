// Drives the host code of linear maps, their gradients, dropout and cross attention through the C ABI for the sanitizer build
// (test infrastructure): plans and workspaces of every size class, type and layout.  The addresses are never read.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "aecct.h"

#define EXPECT(x, st) do { aecct_status s_ = (x); if (s_ != (st)) { std::printf("FAIL %s:%d %s -> %d, expected %d\n", __FILE__, __LINE__, #x, (int)s_, (int)(st)); return 1; } } while (0)

static char *at(int i) { return (char *)((uintptr_t)0x7000000000ull + ((uintptr_t)i << 44)); }

int main() {
  const int64_t sizes[] = {0, 1, 4, 5, 64, 129, 1000, 4096, 70001};
  for (int64_t rows : sizes)
    for (int64_t in : sizes)
      for (int64_t out : sizes) {
        if (!in || !out) continue;
        for (int kind = 0; kind < 5; ++kind)
          for (int pad : {0, 3, 8})
            for (int turned = 0; turned < 2; ++turned) {
              aecct_linear_map_args a{};
              a.rows = rows, a.in = in, a.out = out, a.w_turned = turned, a.act = kind % 4;
              a.type = a.y_type = kind < 3 ? kind : pad ? AECCT_F32 : AECCT_BF16;
              a.code_type = kind < 3 ? AECCT_CODE_NONE : kind - 2;
              a.x = at(0) + (pad == 3 ? 4 : 0), a.ldx = in + pad, a.w = at(1), a.ldw = (turned ? in : out) + pad;
              if (kind >= 3) a.alpha = (float *)at(2), a.scale = (float *)at(3);
              a.bias = (float *)at(4), a.res = at(5), a.ldres = out + pad, a.z = at(6), a.ldz = out, a.y = at(7), a.ldy = out + pad;
              size_t need = 1;
              EXPECT(aecct_linear_map_workspace_size(&a, &need), AECCT_OK);
              EXPECT(aecct_linear_map(&a, need ? at(8) : nullptr, need, nullptr), AECCT_OK);
              if (need && rows) EXPECT(aecct_linear_map(&a, at(8), need - 1, nullptr), AECCT_ERR_WORKSPACE_TOO_SMALL);
              if (kind >= 3) continue;
              for (int want = 1; want < 8; ++want) {
                aecct_linear_map_grad_args g{};
                g.rows = rows, g.in = in, g.out = out, g.type = kind, g.act = pad ? AECCT_ACT_GELU : AECCT_ACT_NONE, g.w_turned = turned;
                g.dw_type = want % 2 ? AECCT_F32 : kind;
                g.x = at(0), g.ldx = in + pad, g.w = at(1), g.ldw = (turned ? in : out) + pad, g.dy = at(2), g.lddy = out + pad;
                if (pad) g.z = at(3), g.ldz = out + pad;
                if (want & 1) g.dx = at(4), g.lddx = in;
                if (want & 2) g.dw = at(5), g.lddw = out;
                if (want & 4) g.dbias = (float *)at(6);
                EXPECT(aecct_linear_map_grad_workspace_size(&g, &need), AECCT_OK);
                EXPECT(aecct_linear_map_grad(&g, need ? at(8) : nullptr, need, nullptr), AECCT_OK);
                if (need) EXPECT(aecct_linear_map_grad(&g, at(8), need - 1, nullptr), AECCT_ERR_WORKSPACE_TOO_SMALL);
              }
            }
      }
  for (int64_t rows : sizes)
    for (int64_t d : sizes) {
      if (!d) continue;
      for (int type = 0; type < 3; ++type)
        for (int pad : {0, 1, 8}) {
          aecct_dropout_args a{};
          a.rows = rows, a.d = d, a.type = type, a.p = 0.1, a.seed = ~0ull, a.offset = 1, a.x = at(0), a.ldx = d + pad, a.res = at(1);
          a.ldres = d, a.y = at(2), a.ldy = d + pad;
          EXPECT(aecct_dropout(&a, nullptr), AECCT_OK);
        }
    }
  const int64_t lengths[] = {0, 1, 31, 64, 300, 2111, 100000};
  for (int64_t batch : {0, 1, 3, 200})
    for (int64_t queries : lengths)
      for (int64_t keys : lengths)
        for (int kv : {1, 8})
          for (int group : {1, 5})
            for (int d : {1, 16, 33, 100, 128, 200, 256})
              for (int type = 0; type < 3; ++type)
                for (int masked = 0; masked < 2; ++masked) {
                  const int heads = kv * group, pad = d % 2 ? 3 : 0;
                  auto box = [&](int i, int64_t n, int h) {
                    return aecct_heads{at(i), n * h * (d + pad), (int64_t)h * (d + pad), d + pad};
                  };
                  aecct_cross_attention_args a{};
                  a.batch = batch, a.queries = queries, a.keys = keys, a.heads = heads, a.kv_heads = kv, a.d = d, a.type = type, a.scale = 0.5f;
                  a.q = box(0, queries, heads), a.k = box(1, keys, kv), a.v = box(2, keys, kv), a.o = box(3, queries, heads);
                  a.lse = (float *)at(4), a.lengths = (int32_t *)at(5);
                  if (masked) a.mask = (uint8_t *)at(6), a.ldmask = keys;
                  size_t need = 0;
                  if (batch * queries * heads >= (int64_t)1 << 28) {
                    EXPECT(aecct_cross_attention_workspace_size(&a, &need), AECCT_ERR_UNSUPPORTED);
                    EXPECT(aecct_cross_attention(&a, at(12), ~(size_t)0 >> 1, nullptr), AECCT_ERR_UNSUPPORTED);
                    continue;
                  }
                  EXPECT(aecct_cross_attention_workspace_size(&a, &need), AECCT_OK);
                  EXPECT(aecct_cross_attention(&a, need ? at(12) : nullptr, need, nullptr), AECCT_OK);
                  aecct_cross_attention_grad_args g{};
                  g.batch = batch, g.queries = queries, g.keys = keys, g.heads = heads, g.kv_heads = kv, g.d = d, g.type = type, g.scale = 0.5f;
                  g.q = a.q, g.k = a.k, g.v = a.v, g.o = a.o, g.dout = box(7, queries, heads), g.lse = a.lse, g.lengths = a.lengths;
                  g.mask = a.mask, g.ldmask = a.ldmask;
                  g.dq = box(8, queries, heads), g.dk = box(9, keys, kv), g.dv = box(10, keys, kv);
                  EXPECT(aecct_cross_attention_grad_workspace_size(&g, &need), AECCT_OK);
                  EXPECT(aecct_cross_attention_grad(&g, need ? at(12) : nullptr, need, nullptr), AECCT_OK);
                  if (need && batch) EXPECT(aecct_cross_attention_grad(&g, at(12), need - 1, nullptr), AECCT_ERR_WORKSPACE_TOO_SMALL);
                }
  std::printf("block driver ok\n");
  return 0;
}
