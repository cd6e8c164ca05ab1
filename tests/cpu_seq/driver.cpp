// Runs one call of the library's C ABI on host buffers (tests/test_cpu_seq.py): as tests/cpu_emu/driver.cpp does, for the entry points of csrc_seq.
//   driver CALL DIR key=value ... name:bytes ...   inputs DIR/<name>.in (absent: NULL), outputs DIR/<name>.out
// An output starts as DIR/<name>.was where there is one, as ones bits otherwise.  The workspace is of exactly its size, filled with ones bits.
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

static thread_local char error_buffer[512] = "";
namespace stl {
char *error_text() { return error_buffer; }
}
extern "C" const char *stl_last_error(void) { return error_buffer; }

static std::string dir;
static std::map<std::string, double> num;
static std::map<std::string, std::pair<void *, size_t>> outs;
static void *file(const std::string &path)
{
    FILE *f = fopen(path.c_str(), "rb");
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
static void *in(const char *name) { return file(dir + "/" + name + ".in"); }
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
static int64_t whole(const char *k) { return (int64_t)num[k]; }
int main(int argc, char **argv)
{
    const std::string call = argv[1];
    dir = argv[2];
    for (int i = 3; i < argc; ++i) {
        std::string a = argv[i];
        const size_t eq = a.find('='), co = a.find(':');
        if (eq != std::string::npos) {
            num[a.substr(0, eq)] = atof(a.c_str() + eq + 1);
        } else {
            const std::string name = a.substr(0, co);
            const size_t n = strtoull(a.c_str() + co + 1, nullptr, 10);
            void *was = file(dir + "/" + name + ".was");
            outs[name] = {was ? was : block(n), n};
        }
    }
    const int dtype = (int)num["dtype"], acc = (int)num["accumulate"], flags = (int)num["flags"];
    int st = -1;
    if (call == "embed_forward" || call == "embed_backward") {
        const stl_embed_t p = {whole("rows"), whole("d"), whole("vocab"), (float)num["scale"], dtype};
        const int64_t *token = (const int64_t *)in("token");
        const size_t n = stl_embed_workspace_bytes(&p);
        st = call == "embed_forward" ? stl_embed_forward(&p, token, in("W"), out("X"), nullptr) : stl_embed_backward(&p, token, in("dX"), out("dW"), acc, block(n), n, nullptr);
    } else if (call == "head_forward" || call == "head_backward") {
        const stl_head_norm_t p = {whole("rows"), whole("heads"), whole("kv_heads"), whole("d"), whole("rot"), whole("ld_q"), whole("ld_k"), whole("ld_qout"), whole("ld_kout"),
                                   (float)num["base"], 1e-6f, dtype};
        const int64_t *position = (const int64_t *)in("position");
        const size_t n = stl_head_norm_workspace_bytes(&p, flags);
        st = call == "head_forward" ? stl_head_norm_forward(&p, in("Q"), in("K"), in("w_q"), in("w_k"), position, out("Qout"), out("Kout"), flags, nullptr)
                                    : stl_head_norm_backward(&p, in("Q"), in("K"), in("w_q"), in("w_k"), position, in("dQout"), in("dKout"), out("dQ"), out("dK"),
                                                             (float *)out("dw_q"), (float *)out("dw_k"), acc, block(n), n, flags, nullptr);
    } else if (call == "decay_forward" || call == "decay_backward") {
        const stl_decay_attention_t p = {whole("rows"), whole("sequences"), whole("length"), whole("heads"), whole("kv_heads"), whole("dk"), whole("dv"), whole("seq_step"),
                                         whole("token_step"), whole("ld_q"), whole("ld_k"), whole("ld_v"), whole("ld_o"), (float)num["scale"], dtype};
        const float *decay = (const float *)in("log_decay"), *state = (const float *)in("state");
        const int64_t *offset = (const int64_t *)in("offset");
        const bool back = call == "decay_backward";
        const size_t n = stl_decay_attention_workspace_bytes(&p, back ? STL_OP_BACKWARD : STL_OP_FORWARD);
        if (!back) {
            float *after = (float *)out("state_out");
            if (num["in_place"] && after) memcpy(after, state, outs["state_out"].second);
            if (num["step"]) {                                  // one sequence, so many tokens a call, whose state goes on in its place
                stl_decay_attention_t some = p;
                char *q = (char *)in("Q"), *k = (char *)in("K"), *v = (char *)in("V"), *o = (char *)out("O");
                const int64_t size = dtype ? 2 : 4;
                void *ws = block(n);
                some.rows = some.length = whole("step");
                for (st = 0; st == 0 && some.rows <= p.rows; some.rows += some.length) {
                    stl_decay_attention_t one = some;
                    const int64_t row = some.rows - some.length;
                    one.rows = some.length;
                    st = stl_decay_attention_forward(&one, q + row * p.ld_q * size, k + row * p.ld_k * size, v + row * p.ld_v * size, decay, nullptr, after,
                                                     o + row * p.ld_o * size, after, ws, n, nullptr);
                }
            } else {
                st = stl_decay_attention_forward(&p, in("Q"), in("K"), in("V"), decay, offset, num["in_place"] ? after : state, out("O"), after, block(n), n, nullptr);
            }
        } else {
            st = stl_decay_attention_backward(&p, in("Q"), in("K"), in("V"), decay, offset, state, in("dO"), (const float *)in("dstate_out"), out("dQ"), out("dK"), out("dV"),
                                              (float *)out("dstate_in"), block(n), n, nullptr);
        }
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
