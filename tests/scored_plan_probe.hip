// How attention with masked and reshaped scores is planned, on a machine without a GPU: the runtime functions of launch_probe.hip.
#define main launch_probe_main
#include "launch_probe.hip"
#undef main

// A call a line on standard input:
//   bf16 heads kv_heads head_dim pages lists lengths B L cap max_batch max_seq max_rows
// (pages: over pages of L tokens a request at most; lists: with a row list of `cap` places, else all B * L tokens; lengths: a length for every
// sequence; max_*: of the context), and a line for each on standard output:
//   rows of a tile, most splits, whether the last workgroup merges, whether copies go past the L2, whether a launch merges, tiles * kv_heads at most,
//   workgroups that pieces are made for, elements of the scratch for partial rows, rows that the merge's launch has room for, counters
int main() {
  int v[13];
  dyllm_layer_cfg made{};
  dyllm_ctx *ctx = nullptr;
  for (;;) {
    for (int &x : v)
      if (scanf("%d", &x) != 1) return 0;
    dyllm_layer_cfg cfg{};
    cfg.hidden = 256; cfg.ffn_dim = 256; cfg.rms_eps = 1e-5f; cfg.rope_theta = 1e4f;
    cfg.dtype = v[0] ? DYLLM_BF16 : DYLLM_F32; cfg.n_heads = v[1]; cfg.n_kv_heads = v[2]; cfg.head_dim = v[3];
    cfg.max_batch = v[10]; cfg.max_seq = v[11]; cfg.max_rows = v[12];
    if (!ctx || memcmp(&cfg, &made, sizeof(cfg))) {  // (the one of the line before, where that is the same)
      if (ctx) dyllm_destroy(ctx);
      ctx = nullptr;
      if (dyllm_create(&cfg, &ctx) != DYLLM_OK) return 3;
      made = cfg;
    }
    ScoredAttn a = scored_args(ctx, nullptr, nullptr, nullptr);
    int32_t some = 0;
    a.pages.table = v[4] ? &some : nullptr;
    a.offsets = v[5] ? &some : nullptr;
    a.kv_len = v[6] ? &some : nullptr;
    a.B = v[7]; a.L = v[8]; a.cap = v[5] ? v[9] : v[7] * v[8];
    scored_plan(dt(ctx), &a);
    const long g = a.H / a.Hkv, tiles = a.offsets ? (a.cap * g + a.bq - 1) / a.bq + a.B : a.B * ((a.L * g + a.bq - 1) / a.bq);
    printf("%d %d %d %d %d %ld %d %zu %d %d\n", a.bq, a.splits, a.fused, a.once, a.n_split != nullptr, tiles * a.Hkv, a.target, a.part_elems, a.split_rows,
           ARRIVE_WORDS);
  }
}
