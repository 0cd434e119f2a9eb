// Host-side test driver of attention: the library's own host code over the HIP runtime that fake_layers_driver.cpp makes up, so no GPU is touched and no
// kernel runs.  Reads calls from standard input, one a line, and prints for each what it returned, the work memory it asks for, and its launches.
//
//   g++ -std=c++17 -rdynamic -o driver tests/fake_blocks_driver.cpp libalpa_dp.so
//
//   attention back dtype seqs heads kv_heads dim causal k_step rows k_rows cap slopes need      (need: 1 dq, 2 dk, 4 dv)
//   kernels                                                     (all there are, as if they were launched)
#define main layers_main
#include "fake_layers_driver.cpp"
#undef main

#include "../include/alpa_blocks.h"

static alpa_heads_t heads(int n, int64_t count, int64_t dim, bool there = true) { return there ? alpa_heads_t{place(n), count * dim, dim} : alpa_heads_t{nullptr, 0, 0}; }

int main()
{
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string op;
        in >> op;
        launches.clear();
        int rc = -99;
        int64_t need = 0;
        if (op == "attention") {
            int back, slopes, wanted;
            alpa_attention_t a{};
            in >> back >> a.dtype >> a.seqs >> a.heads >> a.kv_heads >> a.dim >> a.causal >> a.k_step >> a.rows >> a.k_rows >> a.cap >> slopes >> wanted;
            a.scale = 0.125f;
            a.offsets = (const int32_t *)place(1);
            a.k_offsets = (const int32_t *)place(2);
            a.slopes = slopes ? (const float *)place(3) : nullptr;
            auto *lse = (float *)place(4);
            const alpa_heads_t q = heads(5, a.heads, a.dim), k = heads(6, a.kv_heads, a.dim), v = heads(7, a.kv_heads, a.dim), y = heads(8, a.heads, a.dim);
            if (back) {
                const alpa_heads_t dy = heads(9, a.heads, a.dim), dq = heads(10, a.heads, a.dim, wanted & 1), dk = heads(11, a.kv_heads, a.dim, wanted & 2),
                                   dv = heads(12, a.kv_heads, a.dim, wanted & 4);
                need = alpa_attention_backward_work(&a, dy, q, k, v, y);
                rc = alpa_attention_backward(&a, dy, q, k, v, y, lse, dq, dk, dv, place(13), need, nullptr);
            } else {
                need = alpa_attention_forward_work(&a, q, k, v);
                rc = alpa_attention_forward(&a, q, k, v, y, lse, place(13), need, nullptr);
            }
        }
        if (op == "kernels")
            for (auto &k : kernels()) launches += " " + k.second + " 0 0 0 0;";
        printf("%d %lld%s\n", rc, (long long)need, launches.c_str());
    }
    return 0;
}
