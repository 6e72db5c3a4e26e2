// What the entry points of requests over pages and of masked scores refuse, and how attention is planned, on a machine without a GPU: the runtime
// functions of launch_probe.hip, which print a line per launch.
#define main launch_probe_main
#include "launch_probe.hip"
#undef main

// pages_probe refuse         a line "NAME CODE" for every call below, launches between them
// pages_probe plan bf16 heads kv_heads head_dim pages B L cap max_rows      rows of a tile, most splits
// pages_probe turns theta head_dim      2^-64 turns a position of every pair
int main(int argc, char **argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  int v[8] = {};
  for (int i = 0; i < 8 && i + 2 < argc; ++i) v[i] = atoi(argv[2 + i]);
  dyllm_layer_cfg cfg{};
  cfg.hidden = 256; cfg.ffn_dim = 256; cfg.rms_eps = 1e-5f; cfg.rope_theta = 1e4f;
  cfg.dtype = DYLLM_BF16; cfg.n_heads = 4; cfg.n_kv_heads = 2; cfg.head_dim = 64; cfg.max_batch = 2; cfg.max_seq = 32; cfg.max_rows = 8;
  if (what == "plan") {
    cfg.dtype = v[0] ? DYLLM_BF16 : DYLLM_F32; cfg.n_heads = v[1]; cfg.n_kv_heads = v[2]; cfg.head_dim = v[3];
    cfg.max_batch = 1; cfg.max_seq = cfg.max_rows = atoi(argv[9]);
    if (argc != 10) return 2;
  }
  if (what == "turns") { cfg.rope_theta = (float)atof(argv[2]); cfg.head_dim = v[1]; }
  dyllm_ctx *ctx = nullptr;
  if (dyllm_create(&cfg, &ctx) != DYLLM_OK) return 3;
  if (what == "turns") {
    for (int p = 0; p < cfg.head_dim / 2; ++p) printf("%llu\n", (unsigned long long)ctx->turns[p]);
    return 0;
  }
  if (what == "plan") {
    ScoredAttn a = scored_args(ctx, nullptr, nullptr, nullptr);
    int32_t some = 0;
    a.pages.table = v[4] ? &some : nullptr;
    a.offsets = &some; a.B = v[5]; a.L = v[6]; a.cap = cfg.max_rows;
    scored_plan(dt(ctx), &a);
    printf("%d %d\n", a.bq, a.splits);
    return 0;
  }
  if (what != "refuse") return 4;
  alignas(16) static char mem[32][256];  // addresses that nothing follows
  int n = 0;
  auto any = [&]() { return (void *)mem[n++]; };
  auto words = [&]() { return (int32_t *)any(); };
  const dyllm_pages good{any(), any(), words(), 4, 16, 3};
  const dyllm_page_rows rows{words(), words(), words(), 8};
  dyllm_page_rows mine = rows;
  int32_t *len = words(), *now = words(), *num = words(), *free_list = words(), *n_free = words(), *len_out = words(), *n_out = words(), *kv = words();
  void *x = any(), *q = any(), *out = any();
  uint8_t axis[32] = {};
  auto off = [](const void *p) { return (void *)((char *)p + 4); };
  auto odd = [](const void *p) { return (int32_t *)((char *)p + 2); };
  auto say = [&](const char *name, int rc) { printf("%s %d\n", name, rc); };
  auto plan = [&](const dyllm_pages &p, int R) { mine = rows; return dyllm_page_plan(ctx, &p, R, len, now, num, free_list, n_free, &mine, len_out, n_out, nullptr); };
  auto attend = [&](const dyllm_pages &p, const dyllm_page_rows &r, int R, const dyllm_scores *s = nullptr) { return dyllm_paged_attention(ctx, q, &p, &r, R, kv, s, out, nullptr); };
  auto heads = [&](const dyllm_pages &p, const dyllm_page_rows &r, int64_t ld, const int32_t *at = nullptr, int axes = 0, const uint8_t *ax = nullptr) {
    return dyllm_head_norm_rope_paged(ctx, x, ld, nullptr, nullptr, &r, 2, at, axes, ax, &p, q, nullptr);
  };
  auto with = [&](auto set) { dyllm_pages p = good; set(p); return p; };
  auto row = [&](auto set) { dyllm_page_rows r = rows; set(r); return r; };
  say("plan", plan(good, 2));
  say("attend", attend(good, rows, 2));
  say("heads", heads(good, rows, 512));
  say("masked", dyllm_partial_attention_masked(ctx, q, x, x, nullptr, nullptr, 1, 8, nullptr, out, nullptr));
  // pages
  say("no requests -1", plan(good, 0));
  say("too many requests -3", plan(good, DYLLM_MAX_REQUESTS + 1));
  say("too many requests -3", attend(good, rows, DYLLM_MAX_REQUESTS + 1));
  for (int size : {1, 8, 17, 48, 2048}) {
    const dyllm_pages p = with([&](auto &p) { p.page_size = size; });
    say("page size -3", plan(p, 2)); say("page size -3", attend(p, rows, 2)); say("page size -3", heads(p, rows, 512));
  }
  for (int size : {0, -16}) say("page size -1", attend(with([&](auto &p) { p.page_size = size; }), rows, 2));
  say("no pages -1", attend(with([&](auto &p) { p.n_pages = 0; }), rows, 2));
  say("no entries -1", attend(with([&](auto &p) { p.max_pages = 0; }), rows, 2));
  say("slots -3", attend(with([&](auto &p) { p.n_pages = 1 << 27; }), rows, 2));
  say("long rows -3", plan(with([&](auto &p) { p.max_pages = (1 << 26) + 1; }), 2));
  say("no table -1", plan(with([&](auto &p) { p.table = nullptr; }), 2));
  say("odd table -1", attend(with([&](auto &p) { p.table = odd(p.table); }), rows, 2));
  say("heads without a table 0", heads(with([&](auto &p) { p.table = nullptr; p.max_pages = 0; }), rows, 512));
  say("plan without pages 0", plan(with([&](auto &p) { p.k = p.v = nullptr; }), 2));
  say("no keys -1", attend(with([&](auto &p) { p.k = nullptr; }), rows, 2));
  say("odd values -1", heads(with([&](auto &p) { p.v = off(p.v); }), rows, 512));
  // rows
  say("no offsets -1", attend(good, row([&](auto &r) { r.offsets = nullptr; }), 2));
  say("no positions -1", attend(good, row([&](auto &r) { r.pos = nullptr; }), 2));
  say("attend without slots 0", attend(good, row([&](auto &r) { r.slot = nullptr; }), 2));
  say("no slots -1", heads(good, row([&](auto &r) { r.slot = nullptr; }), 512));
  say("odd positions -1", heads(good, row([&](auto &r) { r.pos = odd(r.pos); }), 512));
  say("negative capacity -1", heads(good, row([&](auto &r) { r.cap = -1; }), 512));
  say("nothing 0", heads(good, dyllm_page_rows{rows.offsets, nullptr, nullptr, 0}, 512));
  say("nothing 0", attend(good, dyllm_page_rows{rows.offsets, nullptr, nullptr, 0}, 2));
  say("capacity of attention 0", attend(good, row([&](auto &r) { r.cap = 9; }), 2));
  say("capacity of heads 0", heads(good, row([&](auto &r) { r.cap = 9; }), 512));
  // heads
  say("short rows -2", heads(good, rows, 504));
  say("odd rows -2", heads(good, rows, 516));
  say("no axis -1", heads(good, rows, 512, len, 1, nullptr));
  say("axes -1", heads(good, rows, 512, len, 9, axis));
  say("axes -1", heads(good, rows, 512, len, 0, axis));
  axis[31] = 2;
  say("axis -1", heads(good, rows, 512, len, 2, axis));
  say("axes 0", heads(good, rows, 512, len, 3, axis));
  say("positions of axes alone 0", heads(good, row([&](auto &r) { r.pos = nullptr; }), 512, len, 3, axis));
  say("odd gain -1", dyllm_head_norm_rope_paged(ctx, x, 512, off(x), nullptr, &rows, 2, nullptr, 0, nullptr, &good, q, nullptr));
  // scores
  auto score = [&](auto set) { dyllm_scores s{}; set(s); return attend(good, rows, 2, &s); };
  say("cap -1", score([&](auto &s) { s.cap = -1.f; }));
  say("cap -1", score([&](auto &s) { s.cap = INFINITY; }));
  say("cap -1", score([&](auto &s) { s.cap = NAN; }));
  say("cap -3", score([&](auto &s) { s.cap = 1e-7f; }));
  say("cap -3", score([&](auto &s) { s.cap = 4097.f; }));
  say("cap 0", score([&](auto &s) { s.cap = 4096.f; }));
  say("block -1", score([&](auto &s) { s.block = -1; }));
  say("odd slopes -1", score([&](auto &s) { s.slopes = (const float *)odd(x); }));
  say("documents -3", score([&](auto &s) { s.doc = len; }));
  // the plan's lists
  mine = rows;
  say("same length -1", dyllm_page_plan(ctx, &good, 2, len, now, num, free_list, n_free, &mine, len, n_out, nullptr));
  say("same count -1", dyllm_page_plan(ctx, &good, 2, len, now, num, free_list, n_free, &mine, len_out, n_free, nullptr));
  say("same offsets -1", dyllm_page_plan(ctx, &good, 2, len, rows.offsets, num, free_list, n_free, &mine, len_out, n_out, nullptr));
  say("no list -1", dyllm_page_plan(ctx, &good, 2, len, now, num, nullptr, n_free, &mine, len_out, n_out, nullptr));
  say("odd list -1", dyllm_page_plan(ctx, &good, 2, odd(len), now, num, free_list, n_free, &mine, len_out, n_out, nullptr));
  say("no context -1", dyllm_page_plan(nullptr, &good, 2, len, now, num, free_list, n_free, &mine, len_out, n_out, nullptr));
  say("all tokens 0", dyllm_partial_attention_masked(ctx, q, x, x, nullptr, nullptr, 2, 32, nullptr, out, nullptr));
  say("sequences -2", dyllm_partial_attention_masked(ctx, q, x, x, nullptr, nullptr, 3, 2, nullptr, out, nullptr));
  say("odd keys -1", dyllm_partial_attention_masked(ctx, q, off(x), x, nullptr, nullptr, 1, 8, nullptr, out, nullptr));
  say("odd lengths -1", dyllm_partial_attention_masked(ctx, q, x, x, odd(kv), nullptr, 1, 8, nullptr, out, nullptr));
  return 0;
}
