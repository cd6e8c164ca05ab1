// Runs one call of the library's C ABI on host buffers: reads its arguments from files, writes its outputs to files (tests/test_cpu_lm.py).
//   driver CALL DIR key=value ...   inputs DIR/<name>.in (absent: NULL), outputs DIR/<name>.out of the sizes given as name:bytes
// Buffers are heap blocks of exactly their size; the workspace is filled with ones bits first.
#include "stl.h"
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

asm(R"(
.text
.globl emu_switch
emu_switch:
    pushq %rbp
    pushq %rbx
    pushq %r12
    pushq %r13
    pushq %r14
    pushq %r15
    movq %rsp, (%rdi)
    movq %rsi, %rsp
    popq %r15
    popq %r14
    popq %r13
    popq %r12
    popq %rbx
    popq %rbp
    ret
)");

// what the library has in stl_api.hip
static thread_local char error_buffer[512] = "";
namespace stl {
char *error_text() { return error_buffer; }
}
extern "C" const char *stl_last_error(void) { return error_buffer; }

static std::string dir;
static std::map<std::string, double> num;
static std::map<std::string, std::pair<void *, size_t>> outs;
static void *in(const char *name)
{
    FILE *f = fopen((dir + "/" + name + ".in").c_str(), "rb");
    if (!f) return nullptr;
    fseek(f, 0, SEEK_END);
    const size_t n = ftell(f);
    rewind(f);
    void *p = nullptr;
    if (posix_memalign(&p, 16, n ? n : 1)) abort();
    if (fread(p, 1, n, f) != n) abort();
    fclose(f);
    return p;
}
static void *out(const char *name)
{
    auto it = outs.find(name);
    return it == outs.end() ? nullptr : it->second.first;
}
static void *block(size_t n)
{
    void *p = nullptr;
    if (posix_memalign(&p, 16, n ? n : 16)) abort();
    memset(p, 0xff, n);
    return p;
}
int main(int argc, char **argv)
{
    const std::string call = argv[1];
    dir = argv[2];
    for (int i = 3; i < argc; ++i) {
        std::string a = argv[i];
        const size_t eq = a.find('='), co = a.find(':');
        if (eq != std::string::npos) num[a.substr(0, eq)] = atof(a.c_str() + eq + 1);
        else {
            const size_t n = strtoull(a.c_str() + co + 1, nullptr, 10);
            outs[a.substr(0, co)] = {block(n), n};
        }
    }
    int st = -1;
    if (call == "residual_forward" || call == "residual_backward") {
        const stl_residual_t p = {(int64_t)num["rows"], (int64_t)num["n"], (int64_t)num["per"], (float)num["skip"], (float)num["scale"], 1e-6f, (int)num["dtype"]};
        const int flags = (int)num["flags"];
        if (call == "residual_forward") {
            st = stl_residual_norm_forward(&p, in("X"), in("H"), in("gate"), in("w_post"), in("b_post"), in("w_pre"), in("b_pre"), out("Xout"), out("Z"), flags, nullptr);
        } else {
            const size_t n = stl_residual_norm_workspace_bytes(&p, flags);
            st = stl_residual_norm_backward(&p, in("Xout"), in("H"), in("gate"), in("w_post"), in("b_post"), in("w_pre"), in("dXout"), in("dZ"), out("dX"), out("dH"),
                                            (float *)out("dgate"), (float *)out("dw_post"), (float *)out("db_post"), (float *)out("dw_pre"),
                                            (float *)out("db_pre"), 0, block(n), n, flags, nullptr);
        }
    } else if (call == "vocab_forward" || call == "vocab_backward") {
        const stl_vocab_t p = {(int64_t)num["rows"], (int64_t)num["d"], (int64_t)num["vocab"], (int64_t)num["ntop"], (float)num["tau"], (int)num["dtype"]};
        const bool back = call == "vocab_backward";
        const size_t n = stl_vocab_loss_workspace_bytes(&p, back ? STL_OP_BACKWARD : STL_OP_FORWARD);
        const int64_t *label = (const int64_t *)in("label"), *top_id = (const int64_t *)in("top_id");
        const float *top_logit = (const float *)in("top_logit");
        if (back)
            st = stl_vocab_loss_backward(&p, in("X"), in("W"), label, top_id, top_logit, (const float *)in("dlabel"), (const float *)in("dtop"),
                                         (float *)out("label_loss"), (float *)out("top_loss"), out("dX"), out("dW"), block(n), n, nullptr);
        else
            st = stl_vocab_loss_forward(&p, in("X"), in("W"), label, top_id, top_logit, (float *)out("label_loss"), (float *)out("top_loss"), block(n), n, nullptr);
    }
    if (st) {
        fprintf(stderr, "status %d: %s\n", st, stl_last_error());
        return 2;
    }
    for (auto &o : outs) {
        FILE *f = fopen((dir + "/" + o.first + ".out").c_str(), "wb");
        if (fwrite(o.second.first, 1, o.second.second, f) != o.second.second) abort();
        fclose(f);
    }
    printf("ok\n");
}
