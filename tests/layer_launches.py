"""What the layer operators would launch for given shapes: the library's own host
code, compiled with launchers that only write down their arguments, so no GPU is
needed."""
import json
import math
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Shapes that between them take every path (`paths`) that at least 3 of 30000 drawn
# ones (`draw`) take, and large ones.  The GPU tests check their results.
SHAPES = [
    ("ffn", 1, 0, 42, 2158, 2088, 1, 0), ("ffn", 1, 0, 92, 4176, 6792, 0, 0), ("ffn", 1, 0, 3042, 64, 4160, 1, 1),
    ("ffn", 1, 0, 3520, 425, 843, 1, 0), ("ffn", 1, 0, 4096, 512, 384, 1, 1), ("ffn", 1, 0, 7076, 2474, 1269, 1, 0),
    ("ffn", 1, 0, 7744, 2947, 3725, 1, 0), ("ffn", 1, 0, 8064, 640, 6336, 0, 0), ("ffn", 1, 0, 8192, 512, 752, 1, 1),
    ("ffn", 1, 0, 8192, 4096, 10944, 1, 0), ("ffn", 1, 1, 64, 471, 8145, 0, 0), ("ffn", 1, 1, 316, 72, 9976, 1, 1),
    ("ffn", 1, 1, 802, 3024, 4696, 1, 1), ("ffn", 1, 1, 810, 2480, 10127, 1, 0),
    ("ffn", 1, 1, 2013, 3432, 5624, 0, 0), ("ffn", 1, 1, 2454, 3693, 6838, 0, 1), ("ffn", 1, 1, 4087, 136, 256, 1, 1),
    ("ffn", 1, 1, 4096, 64, 4032, 0, 0), ("ffn", 1, 1, 4565, 2880, 5824, 0, 0), ("ffn", 1, 1, 7360, 1232, 8488, 1, 0),
    ("ffn", 1, 1, 8358, 2560, 2368, 0, 1), ("ffn", 1, 1, 8461, 3776, 128, 1, 1), ("ffn", 1, 1, 8518, 501, 107, 0, 1),
    ("ffn", 1, 2, 33, 64, 64, 0, 0), ("ffn", 1, 2, 1024, 1784, 2008, 0, 1), ("ffn", 1, 2, 2008, 3008, 10120, 0, 1),
    ("ffn", 1, 2, 2035, 4194, 5709, 1, 1), ("ffn", 1, 2, 2048, 4056, 168, 1, 1), ("ffn", 1, 2, 3095, 4096, 192, 1, 0),
    ("ffn", 1, 2, 5063, 203, 3181, 0, 1), ("ffn", 1, 2, 5568, 1600, 4160, 1, 0), ("ffn", 1, 2, 6311, 349, 451, 0, 0),
    ("ffn", 1, 2, 7744, 775, 9841, 0, 1), ("ffn", 1, 2, 8192, 192, 1024, 1, 0), ("ffn", 1, 2, 8303, 672, 5008, 1, 1),
    ("ffn", 1, 2, 8760, 4000, 1920, 1, 1), ("ffn", 2, 0, 660, 864, 2648, 2, 1), ("ffn", 2, 0, 1828, 2561, 2227, 0, 0),
    ("ffn", 2, 0, 2304, 704, 10944, 0, 0), ("ffn", 2, 0, 5919, 64, 2240, 2, 1), ("ffn", 2, 0, 6796, 4038, 4220, 2, 0),
    ("ffn", 2, 0, 8144, 86, 253, 0, 1), ("ffn", 2, 0, 8192, 4096, 10944, 2, 0), ("ffn", 2, 0, 8384, 3584, 128, 2, 1),
    ("ffn", 2, 1, 33, 64, 64, 2, 1), ("ffn", 2, 1, 512, 88, 5184, 0, 0), ("ffn", 2, 1, 2752, 3328, 192, 0, 0),
    ("ffn", 2, 1, 4096, 73, 997, 2, 0), ("ffn", 2, 1, 4302, 64, 3200, 0, 0), ("ffn", 2, 1, 5568, 2880, 6848, 2, 1),
    ("ffn", 2, 1, 5632, 80, 8792, 0, 1), ("ffn", 2, 1, 6336, 2880, 8192, 0, 0), ("ffn", 2, 1, 7104, 1240, 7832, 2, 0),
    ("ffn", 2, 1, 8320, 384, 384, 0, 1), ("ffn", 2, 2, 33, 3640, 2712, 0, 1), ("ffn", 2, 2, 64, 960, 4096, 2, 1),
    ("ffn", 2, 2, 479, 2496, 4096, 2, 0), ("ffn", 2, 2, 4288, 512, 448, 0, 1), ("ffn", 2, 2, 5504, 904, 368, 2, 0),
    ("ffn", 2, 2, 5588, 1016, 9352, 0, 0), ("ffn", 2, 2, 6073, 3728, 3104, 2, 1),
    ("ffn", 2, 2, 6464, 123, 2265, 0, 1), ("ffn", 2, 2, 6656, 3580, 286, 2, 1), ("ffn", 2, 2, 8318, 1491, 981, 0, 0),
    ("update", 0, 1, 960, 4032), ("update", 0, 1, 1104, 4329), ("update", 0, 1, 1124, 1037),
    ("update", 0, 1, 2018, 3736), ("update", 0, 1, 2944, 4800), ("update", 0, 1, 2991, 2702),
    ("update", 0, 1, 3523, 4763), ("update", 0, 1, 3982, 901), ("update", 0, 1, 4000, 4000),
    ("update", 0, 1, 4179, 4875), ("update", 0, 1, 4425, 1101), ("update", 0, 1, 5056, 4224),
    ("update", 0, 1, 5133, 3224), ("update", 0, 1, 5568, 1600), ("update", 0, 1, 7892, 4647),
    ("update", 0, 1, 8515, 2278), ("update", 0, 1, 10944, 4096), ("update", 0, 2, 1165, 75),
    ("update", 0, 2, 3440, 986), ("update", 0, 2, 4911, 4626), ("update", 0, 2, 5312, 1152),
    ("update", 0, 2, 7413, 4233), ("update", 0, 3, 2344, 2532), ("update", 0, 3, 2488, 2507),
    ("update", 0, 3, 3638, 3462), ("update", 0, 3, 3648, 2304), ("update", 0, 3, 3658, 3269),
    ("update", 0, 3, 9346, 2367), ("update", 0, 8, 75, 2016), ("update", 0, 8, 352, 3035),
    ("update", 0, 8, 453, 3822), ("update", 0, 8, 458, 340), ("update", 0, 8, 677, 4782), ("update", 0, 8, 1000, 777),
    ("update", 0, 8, 1398, 1348), ("update", 0, 8, 1728, 1280), ("update", 0, 8, 2000, 2000),
    ("update", 0, 8, 2019, 475), ("update", 0, 8, 2480, 1971), ("update", 0, 8, 4792, 974),
    ("update", 0, 8, 6583, 2164), ("update", 0, 8, 8201, 2019), ("update", 0, 8, 9442, 1432),
    ("update", 0, 1, 64, 64), ("update", 0, 8, 2022, 81), ("update", 0, 1, 4655, 451), ("update", 0, 3, 333, 2909),
]

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "arena_layer_host.cpp"
using namespace arena::mm;
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
static int at;
static void say(const char* fn, const GemmArgs& A, int dtype, int what, const Cut& c, bool second)
{
    static const char* const products[] = {"rows rows", "rows cols", "cols cols", "gate up", "gate up back", "rows rows rest", "rows cols rest"};
    static const char* const kinds[] = {"256", "128", "128 deep", "64"};
    const bool sym = A.sym, dual = what == kGateUp;
    const int64_t side = kTileSide[c.main], tm = (A.M + side - 1) / side, cols = dual ? side / 2 : side;
    const int64_t tn = (A.N + cols - 1) / cols, all = (sym ? tm * (tm + 1) / 2 : tm * tn) * A.batch;
    printf("{\"shape\": %d, \"call\": \"%s\", \"product\": \"%s\", \"dtype\": %d, \"act\": %d, \"sym\": %s, \"batch\": %d, "
           "\"out\": %d, \"adds\": %s, \"segments\": %d, \"steps\": %d, \"main\": \"%s\", \"whole\": %lld, \"tail\": \"%s\", "
           "\"rest\": %lld, \"ratio\": %d, \"splits\": %d}\n",
           at, fn, products[what], dtype, A.act, sym ? "true" : "false", A.batch, A.out, A.beta != 0.0f ? "true" : "false",
           A.nseg, A.nseg * ((A.K + kBK - 1) / kBK), kinds[c.main], (long long)c.first, kinds[c.tail],
           (long long)(all - c.first), (int)(side / kTileSide[c.tail]), second ? 1 : c.splits);
}
namespace arena {
int ctx_device(const arena_ctx*) { return 0; }
void ctx_clear(arena_ctx*) {}
arena_status ctx_fail(arena_ctx*, arena_status s, const char* fmt, ...) { fprintf(stderr, "%s\n", fmt); return s; }
void norm_plan(int64_t, int64_t, int, int*, int*) {}
hipError_t launch_norm_forward(const NormArgs&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(const NormArgs&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_update_sum(const UpdateArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_update_scale(const UpdateArgs&, int, hipStream_t) { return hipSuccess; }
namespace mm {
hipError_t launch_gemm(const GemmArgs& A, int dtype, Product what, const Cut& cut, hipStream_t)
{
    say("one", A, dtype, what, cut, false);
    return hipSuccess;
}
hipError_t launch_pair(const GemmArgs& A, int dtype, Product what, const GemmArgs& B, const Cut& cut, hipStream_t)
{
    say("pair", A, dtype, what, cut, false);
    say("second of pair", B, dtype, kColsCols, cut, true);
    return hipSuccess;
}
hipError_t launch_skinny(const GemmArgs& A, int dtype, bool dual, hipStream_t)
{
    printf("{\"shape\": %d, \"call\": \"skinny\", \"product\": \"%s\", \"dtype\": %d, \"act\": %d}\n", at,
           dual ? "gate up" : "rows rows", dtype, A.act);
    return hipSuccess;
}
hipError_t launch_packs(const Pack*, int, hipStream_t) { return hipSuccess; }
}
}
static void check(arena_status s) { if (s) exit(10 + s); }
int main()
{
    void* const p = (void*)0x10000;
    arena_ctx* const c = (arena_ctx*)p;
    char kind[16];
    for (at = 0; scanf("%15s", kind) == 1; ++at) {
        if (kind[0] == 'f') {
            int dtype, act, model, inner, grad, accumulate;
            long long tokens;
            if (scanf("%d %d %lld %d %d %d %d", &dtype, &act, &tokens, &model, &inner, &grad, &accumulate) != 7) return 1;
            arena_ffn_desc d;
            memset(&d, 0, sizeof(d));
            d.dtype = dtype; d.activation = act; d.tokens = tokens; d.model = model; d.inner = inner;
            d.x = d.w_gate = d.w_up = d.w_down = p;
            d.g = d.u = d.h = d.y = p;
            d.ld_x = d.ld_gate = d.ld_up = d.ld_y = model;
            d.ld_down = inner; d.ld_inner = (inner + 7) / 8 * 8;
            d.workspace = p;
            check(arena_ffn_forward_workspace(c, &d, &d.workspace_bytes));
            check(arena_ffn_forward(c, &d, nullptr));
            arena_ffn_grads g;
            memset(&g, 0, sizeof(g));
            g.grad_dtype = grad; g.accumulate = accumulate;
            g.dy = p; g.dx = g.dw_gate = g.dw_up = g.dw_down = p;
            g.ld_dy = g.ld_dx = g.ld_dw_gate = g.ld_dw_up = model; g.ld_dw_down = inner;
            check(arena_ffn_backward_workspace(c, &d, &g, &d.workspace_bytes));
            check(arena_ffn_backward(c, &d, &g, nullptr));
        } else {
            arena_update_desc d;
            memset(&d, 0, sizeof(d));
            const float k[9] = {1.5f, -0.5f, 0.0f, 1.5f, -0.5f, 0.0f, 1.5f, -0.5f, 0.0f};
            if (scanf("%d %d %d %d", &d.dtype, &d.batch, &d.rows, &d.cols) != 4) return 1;
            d.out_dtype = ARENA_BF16; d.steps = 3; d.eps = 1e-7f; d.scale = 1.0f;
            d.coefficients = k;
            d.grad = d.out = p;
            d.ld_grad = d.ld_out = d.cols;
            d.stride_grad = d.stride_out = (int64_t)d.rows * d.cols;
            d.workspace = p;
            check(arena_orthogonal_update_workspace(c, &d, &d.workspace_bytes));
            check(arena_orthogonal_update(c, &d, nullptr));
        }
    }
    return 0;
}
"""


def build(folder):
    """Path of the program."""
    src, exe = os.path.join(folder, "launches.cpp"), os.path.join(folder, "launches")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2403_16125_amd", "csrc"), "-I",
                    os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"), src, "-o", exe], check=True)
    return exe


def launches(exe, shapes):
    """One dict a product, in order.  shapes: ("ffn", dtype, act, tokens, model, inner,
    gradients' dtype, accumulate) or ("update", dtype, batch, rows, cols), in the ABI's
    codes; "shape" in a dict is the index into them.  Updates are of three steps: the
    first hands on what its 16 bits leave out, the last writes the result."""
    text = "\n".join(" ".join(str(int(v)) if not isinstance(v, str) else v for v in s) for s in shapes)
    done = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
    return [json.loads(line) for line in done.stdout.splitlines()]


def draw(rng, most):
    """A shape of the ranges that the operators are used over, of at most `most` operations."""
    def size(low, high, step):
        return max(low, int(math.exp(rng.uniform(math.log(low), math.log(high)))) // step * step)

    while True:
        if rng.random() < 0.6:
            step, typ = rng.choice((1, 8, 64)), rng.choice((1, 2))
            s = ("ffn", typ, rng.choice((0, 1, 2)), size(33, 9000, rng.choice((1, 64))), size(64, 4200, step),
                 size(64, 11000, step), rng.choice((typ, 0)), rng.choice((0, 1)))
            work = 18 * s[3] * s[4] * s[5]
        else:
            step = rng.choice((1, 64))
            s = ("update", 0, rng.choice((1, 1, 2, 3, 8)), size(64, 11000, step), size(64, 5000, step))
            n, m = sorted(s[3:])
            work = s[2] * (3 * n * n * m + n ** 3)
        if work <= most and 3072 not in s:
            return s


def paths(launch):
    """The paths through the kernels that a launch takes: which tile of which product,
    how it is cut, and what its epilogue does."""
    if launch["call"] == "skinny":
        return []
    what, split = (launch["product"], launch["dtype"]), "split" if launch["splits"] > 1 else "unsplit"
    sym, batch = "mirrored" if launch["sym"] else "", "batch" if launch["sym"] and launch["batch"] > 1 else ""
    out = []
    if launch["call"] != "one":
        out.append((launch["call"], *what, split))
    else:
        if launch["whole"]:
            out.append((*what, launch["main"], "whole rounds", sym, batch))
        if launch["rest"]:
            out.append((*what, launch["tail"], "after whole rounds" if launch["whole"] else "alone",
                        "smaller tiles" if launch["ratio"] > 1 else "", split, sym, batch))
    if launch["product"] == "cols cols" and not launch["sym"]:
        out.append(("weight gradient", launch["call"], launch["out"], launch["adds"], split))
    if launch["product"].startswith("gate up"):
        out.append((*what, launch["act"], launch["tail"] if launch["rest"] else launch["main"]))
    return out
