// Host-side test driver of the layer operators: the library's own host code over a HIP runtime that is made up here, so no
// GPU is touched and no kernel runs.  Reads calls from standard input, one a line, and prints for each what it returned, the
// work memory it asks for, and its launches with their sizes; a launch of a shape that HIP refuses is refused here too.
//
//   g++ -std=c++17 -rdynamic -o driver tests/fake_layers_driver.cpp libalpa_dp.so
//
//   forward  dtype act rows experts n_in n_out ldx ldy bias residual z
//   backward dtype act rows experts n_in n_out ldx lddx bias dx dw        experts -1: a dense layer
//   loss     dtype rows n_in words
//   gradient dtype rows n_in words
//   kernels                                     (all there are, as if they were launched)
#include "../include/alpa_layers.h"

#include <cstdio>
#include <cstring>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

struct Dim3 { uint32_t x, y, z; };
static std::map<const void *, std::string> &kernels() { static std::map<const void *, std::string> m; return m; }
static Dim3 the_grid, the_block;
static int last_error = 0;
static std::string launches;

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *stub, char *, const char *name, unsigned, void *, void *, void *, void *, int *)
{
    kernels()[stub] = name;
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t, void *) { the_grid = grid; the_block = block; return 0; }
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *shared, void **st)
{
    *grid = the_grid; *block = the_block; *shared = 0; *st = nullptr;
    return 0;
}
int hipLaunchKernel(const void *stub, Dim3 g, Dim3 b, void **, size_t, void *)
{
    // threads of a dimension of the grid are counted in 32 bits, the other two dimensions' workgroups in 16
    const bool fits = g.x && g.y && g.z && (uint64_t)g.x * b.x <= 0xffffffffu && g.y <= 65535 && g.z <= 65535;
    if (!fits) return last_error = 9;                                     // hipErrorInvalidConfiguration
    char text[64];
    snprintf(text, sizeof text, " %u %u %u %u;", g.x, g.y, g.z, b.x);
    launches += " " + kernels()[stub] + text;
    return 0;
}
int hipGetLastError(void) { const int e = last_error; last_error = 0; return e; }
const char *hipGetErrorString(int) { return "invalid configuration"; }
}

// addresses that nothing follows, far apart
static void *place(int n) { return (void *)((uintptr_t)1 << 40 | (uintptr_t)n << 48); }
static alpa_mat_t mat(int n, int64_t ld) { return ld ? alpa_mat_t{place(n), ld} : alpa_mat_t{nullptr, 0}; }

int main()
{
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string op;
        in >> op;
        int dtype = 0, act = 0, experts = -1, bias = 0, residual = 0, z = 0, dx = 0, dw = 0;
        int64_t rows = 0, n_in = 0, n_out = 0, ldx = 0, ldo = 0, need = 0;
        int rc = -99;
        launches.clear();
        auto *off = (const int32_t *)place(1);
        auto *target = (const int64_t *)place(2);
        auto *f = (float *)place(3);
        if (op == "forward") {
            in >> dtype >> act >> rows >> experts >> n_in >> n_out >> ldx >> ldo >> bias >> residual >> z;
            const alpa_mat_t x = mat(4, ldx), w = mat(5, n_in), y = mat(6, ldo), k = mat(7, z ? n_out : 0), r = mat(8, residual ? n_out : 0);
            void *b = bias ? place(9) : nullptr;
            if (experts < 0) {
                need = alpa_linear_forward_work(dtype, rows, n_in, n_out, x, w);
                rc = alpa_linear_forward(dtype, act, rows, n_in, n_out, x, w, b, r, y, k, place(10), need, nullptr);
            } else {
                need = alpa_experts_forward_work(dtype, rows, experts, n_in, n_out, x, w);
                rc = alpa_experts_forward(dtype, act, rows, experts, n_in, n_out, off, x, w, b, r, y, k, place(10), need, nullptr);
            }
        } else if (op == "backward") {
            in >> dtype >> act >> rows >> experts >> n_in >> n_out >> ldx >> ldo >> bias >> dx >> dw;
            const alpa_mat_t dy = mat(4, n_out), k = mat(5, act ? n_out : 0), x = mat(6, ldx), w = mat(7, n_in), gx = mat(8, dx ? ldo : 0),
                             gw = mat(9, dw ? n_in : 0);
            void *b = bias ? place(10) : nullptr;
            if (experts < 0) {
                need = alpa_linear_backward_work(dtype, act, rows, n_in, n_out, dy, x, w);
                rc = alpa_linear_backward(dtype, act, rows, n_in, n_out, dy, k, x, w, gx, gw, b, place(11), need, nullptr);
            } else {
                need = alpa_experts_backward_work(dtype, act, rows, experts, n_in, n_out, dy, x, w);
                rc = alpa_experts_backward(dtype, act, rows, experts, n_in, n_out, off, dy, k, x, w, gx, gw, b, place(11), need, nullptr);
            }
        } else if (op == "loss" || op == "gradient") {
            in >> dtype >> rows >> n_in >> n_out;
            const alpa_mat_t x = mat(4, n_in), w = mat(5, n_in);
            if (op == "loss") {
                need = alpa_vocab_loss_forward_work(dtype, rows, n_in, n_out, x, w);
                rc = alpa_vocab_loss_forward(dtype, rows, n_in, n_out, x, w, target, f, f, place(6), need, nullptr);
            } else {
                need = alpa_vocab_loss_backward_work(dtype, rows, n_in, n_out, x, w);
                rc = alpa_vocab_loss_backward(dtype, rows, n_in, n_out, f, x, w, target, f, mat(6, n_in), mat(7, n_in), place(8), need, nullptr);
            }
        }
        if (op == "kernels")
            for (auto &k : kernels()) launches += " " + k.second + " 0 0 0 0;";
        printf("%d %lld%s\n", rc, (long long)need, launches.c_str());
    }
    return 0;
}
