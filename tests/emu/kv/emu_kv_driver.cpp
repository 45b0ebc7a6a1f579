// TEST INFRASTRUCTURE ONLY: runs calls of the 4-bit key/value cache's C ABI on the CPU emulation, from a script on standard input.
// Every buffer is an allocation of exactly its size, so that the sanitizer sees an access that strays.
//   buf NAME BYTES [FILE]          "device memory", filled from FILE or with 0xA5
//   cache PAGES LAYERS N_PAGES KV_HEADS HEAD_DIM PAGE_TOKENS
//   rows TABLE LENGTHS ROWS PAGES_PER_ROW
//   pool_init N POOL | reserve WANT POOL | fork PARENT POOL | free KEEP POOL | compact POOL
//   append LAYER BEGIN TOKENS K V DTYPE TOKEN_STRIDE HEAD_STRIDE
//   read LAYER BEGIN FIRST|- TOKENS K V DTYPE TOKEN_STRIDE HEAD_STRIDE
//   attention LAYER BEGIN TOKENS Q OUT DTYPE TOKEN_STRIDE HEAD_STRIDE Q_HEADS SCALE CAUSAL WINDOW   (a workspace of its own)
//   dump NAME FILE
// Each call's status goes to standard output.
#include <hip/hip_runtime.h>

#include <fstream>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

#include "quantpipe.h"

namespace emu {
h8 mfma_a[16][2][64], mfma_b[16][2][64];
}

struct Buf { char *p; size_t bytes; };
static std::map<std::string, Buf> bufs;
static char *at(const std::string &name)
{
    const auto i = bufs.find(name);
    if (i == bufs.end()) { fprintf(stderr, "no buffer %s\n", name.c_str()); exit(3); }
    return i->second.p;
}
static char *alloc(size_t bytes)
{
    char *p = (char *)aligned_alloc(16, (bytes + 15) / 16 * 16);
    if (!p) exit(3);
    memset(p, 0xA5, (bytes + 15) / 16 * 16);
    return p;
}

int main()
{
    qp_kv_cache_t cache{};
    qp_kv_rows_t rows{};
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string op;
        in >> op;
        auto word = [&] { std::string s; in >> s; return s; };
        auto num = [&] { unsigned long long v = 0; in >> v; return v; };
        auto pool = [&](const std::string &n) { return std::pair<void *, size_t>(at(n), bufs[n].bytes); };
        int rc = 0;
        if (op == "buf") {
            const std::string name = word();
            const size_t bytes = num();
            const std::string file = word();
            bufs[name] = Buf{alloc(bytes), bytes};
            if (!file.empty()) {
                std::ifstream f(file, std::ios::binary);
                if (!f.read(bufs[name].p, (std::streamsize)bytes)) { fprintf(stderr, "%s: short\n", file.c_str()); return 3; }
            }
            continue;
        } else if (op == "cache") {
            const std::string n = word();
            cache.pages_dev = at(n);
            cache.pages_bytes = bufs[n].bytes;
            cache.layers = (uint32_t)num();
            cache.n_pages = (uint32_t)num();
            cache.kv_heads = (uint32_t)num();
            cache.head_dim = (uint32_t)num();
            cache.page_tokens = (uint32_t)num();
            continue;
        } else if (op == "rows") {
            rows.table_dev = (int32_t *)at(word());
            rows.lengths_dev = (int32_t *)at(word());
            rows.rows = (uint32_t)num();
            rows.pages_per_row = (uint32_t)num();
            continue;
        } else if (op == "dump") {
            const std::string n = word(), file = word();
            std::ofstream f(file, std::ios::binary);
            f.write(at(n), (std::streamsize)bufs[n].bytes);
            continue;
        } else if (op == "pool_init") {
            const uint32_t n = (uint32_t)num();
            const auto p = pool(word());
            rc = qp_kv_pool_init(n, p.first, p.second, nullptr);
        } else if (op == "reserve" || op == "fork" || op == "free") {
            const int32_t *a = (const int32_t *)at(word());
            const auto p = pool(word());
            rc = op == "reserve" ? qp_kv_reserve(&cache, &rows, a, p.first, p.second, nullptr)
               : op == "fork" ? qp_kv_fork(&cache, &rows, a, p.first, p.second, nullptr)
                              : qp_kv_free(&cache, &rows, a, p.first, p.second, nullptr);
        } else if (op == "compact") {
            const auto p = pool(word());
            rc = qp_kv_compact(&cache, &rows, p.first, p.second, nullptr);
        } else if (op == "append" || op == "read" || op == "attention") {
            const uint32_t layer = (uint32_t)num();
            const int32_t *begin = (const int32_t *)at(word());
            const int32_t *first = nullptr;
            if (op == "read") {
                const std::string f = word();
                if (f != "-") first = (const int32_t *)at(f);
            }
            const uint64_t tokens = num();
            qp_kv_view_t a{}, b{};
            a.data_dev = at(word());
            b.data_dev = at(word());
            a.dtype = b.dtype = (uint32_t)num();
            a.token_stride = b.token_stride = num();
            a.head_stride = b.head_stride = num();
            if (op == "append") rc = qp_kv_append(&cache, &rows, layer, begin, tokens, &a, &b, nullptr);
            else if (op == "read") rc = qp_kv_read(&cache, &rows, layer, begin, first, tokens, &a, &b, nullptr);
            else {
                qp_kv_attn_cfg_t cfg{};
                cfg.q_heads = (uint32_t)num();
                in >> cfg.scale;
                cfg.causal = (uint32_t)num();
                cfg.window = (uint32_t)num();
                b.token_stride = (uint64_t)cfg.q_heads * cache.head_dim;      // the answer is dense
                b.head_stride = cache.head_dim;
                const size_t wb = qp_kv_attention_workspace_bytes(&cache, &rows, tokens, cfg.q_heads);
                char *ws = alloc(wb);
                rc = qp_kv_attention(&cache, &rows, layer, begin, tokens, &a, &b, &cfg, ws, wb, nullptr);
                free(ws);
            }
        } else {
            fprintf(stderr, "unknown: %s\n", line.c_str());
            return 3;
        }
        printf("%d\n", rc);
        fflush(stdout);
    }
    for (auto &b : bufs) free(b.second.p);
    return 0;
}
