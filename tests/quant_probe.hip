// What the entry points of normalised heads and of the 8-bit cache refuse, and how attention over that cache is planned, on a machine without a GPU:
// the runtime functions of launch_probe.hip, which print a line per launch.
#define main launch_probe_main
#include "launch_probe.hip"
#undef main

// quant_probe CASE bf16 hidden heads kv_heads head_dim B L max_rows cap
//   plan      rows in a tile, key splits, keys of a split of a list of `cap` entries
//   q|k|v     K splits, rows in row tiles and splits of the rows behind them of the projections of `cap` rows
//   scratch   floats of scratch that the GEMMs ask for, and of what attention over codes may use
//   all rows  attention, write and read of all tokens (no list)
//   refresh   dyllm_qkv_refresh_normed with one of its weights at an address that is no multiple of 16 bytes, weight by weight
//   step      dyllm_layer_step_quant likewise
int main(int argc, char **argv) {
  if (argc != 11) return 2;
  int v[9];
  for (int i = 0; i < 9; ++i) v[i] = atoi(argv[2 + i]);
  const std::string what = argv[1];
  const int H = v[2], Hkv = v[3], dh = v[4], B = v[5], L = v[6], cap = v[8];
  dyllm_layer_cfg cfg{};
  cfg.dtype = v[0] ? DYLLM_BF16 : DYLLM_F32;
  cfg.hidden = v[1]; cfg.n_heads = H; cfg.n_kv_heads = Hkv; cfg.head_dim = dh; cfg.ffn_dim = 256;
  cfg.max_batch = B; cfg.max_seq = L; cfg.max_rows = v[7]; cfg.rms_eps = 1e-5f; cfg.rope_theta = 1e4f;
  dyllm_ctx *ctx = nullptr;
  if (dyllm_create(&cfg, &ctx) != DYLLM_OK) return 3;
  alignas(16) static char mem[32][64];  // addresses that nothing follows
  int n = 0;
  auto any = [&]() { return (void *)mem[n++]; };
  dyllm_quant_cache quant{any(), any(), (float *)any(), (float *)any(), DYLLM_E4M3};
  dyllm_layer_cache cache{};
  cache.c = any(); cache.out = any();
  const dyllm_index_list in{(int32_t *)any(), (int32_t *)any(), cap};
  dyllm_index_list out{(int32_t *)any(), (int32_t *)any(), cap};
  void *x = any(), *y = any(), *z = any();
  if (what == "plan") {
    AttnArgs a{};
    a.rows = rows_of(&in, B); a.offsets = in.offsets; a.B = B; a.L = L; a.H = H; a.Hkv = Hkv; a.dh = dh;
    attention_quant_plan(dt(ctx), ctx->quant_part_elems, &a);
    printf("%d %d %d\n", a.bq, a.splits, a.chunk);
    return 0;
  }
  if (what == "q|k|v") {
    const mm::GemmPlan p = mm::plan_on_host(mm::raw_plan_args(ctx->dq + 2 * ctx->dkv, cfg.hidden, ctx->part_elems, true, 32), cap);
    printf("%d %d %d\n", p.sk, p.row_hi, p.sk_tail);
    return 0;
  }
  if (what == "scratch") {
    printf("%zu %zu\n", ctx->part_elems, ctx->quant_part_elems);
    return 0;
  }
  if (what == "all rows") {
    printf("attention %d\n", dyllm_partial_attention_quant(ctx, x, &quant, nullptr, nullptr, B, L, y, nullptr));
    printf("write %d\n", dyllm_quant_write(ctx, x, y, nullptr, B, L, &quant, nullptr));
    printf("read %d\n", dyllm_quant_read(ctx, &quant, nullptr, B, L, y, z, nullptr));
    return 0;
  }
  const bool step = what == "step";
  if (!step && what != "refresh") return 4;
  const char *names[] = {"wq", "wk", "wv", "bq", "bk", "bv", "g_attn", "wo", "w_gate", "w_up", "w_down", "g_ffn"};
  for (int i = -1; i < (step ? 12 : 7); ++i) {
    dyllm_layer_weights w{x, x, x, x, x, x, x, x, x, x, x, x};
    const void **at[] = {&w.wq, &w.wk, &w.wv, &w.bq, &w.bk, &w.bv, &w.g_attn, &w.wo, &w.w_gate, &w.w_up, &w.w_down, &w.g_ffn};
    if (i >= 0) *at[i] = (char *)x + 4;
    const int rc = step ? dyllm_layer_step_quant(ctx, &w, nullptr, nullptr, &cache, &quant, nullptr, y, &in, B, L, 0.5f, &out, nullptr, nullptr)
                        : dyllm_qkv_refresh_normed(ctx, &w, nullptr, nullptr, y, &in, B, L, nullptr, &quant, z, nullptr);
    printf("%s %d\n", i < 0 ? "none" : names[i], rc);
  }
  return 0;
}
