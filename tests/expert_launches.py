"""What the operators of a layer of experts and of the loss would launch for given shapes:
the library's own host code, compiled with launchers that only write down their
arguments, so no GPU is needed."""
import json
import math
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Shapes that between them take every path (`paths`) that at least 2 of 45000 drawn ones
# (`draw`) take, and a large one of each type.  The GPU tests check their results.
SHAPES = [
    ("experts", 1, 0, 15, 704, 64, 2, 1, 1), ("experts", 1, 0, 22, 908, 334, 2, 1, 1),
    ("experts", 1, 0, 62, 66, 65, 3, 0, 1), ("experts", 1, 0, 364, 1748, 2457, 47, 1, 1),
    ("experts", 1, 0, 754, 3712, 2304, 21, 1, 0), ("experts", 1, 0, 3983, 4104, 160, 6, 0, 1),
    ("experts", 1, 0, 4132, 129, 1478, 3, 1, 1), ("experts", 1, 0, 4705, 64, 64, 10, 0, 1),
    ("experts", 1, 0, 5625, 2880, 4992, 2, 1, 1), ("experts", 1, 0, 6974, 2528, 3360, 5, 1, 0),
    ("experts", 1, 0, 8162, 400, 1440, 2, 1, 0), ("experts", 1, 0, 9627, 5068, 68, 5, 1, 0),
    ("experts", 1, 0, 12482, 64, 448, 4, 1, 0), ("experts", 1, 1, 5, 704, 64, 2, 1, 1),
    ("experts", 1, 1, 204, 665, 86, 2, 0, 1), ("experts", 1, 1, 3943, 141, 65, 6, 1, 1),
    ("experts", 1, 1, 5060, 4082, 136, 8, 1, 1), ("experts", 1, 1, 5430, 64, 2048, 5, 0, 0),
    ("experts", 1, 1, 9765, 2400, 176, 2, 0, 0), ("experts", 1, 1, 9988, 1856, 2048, 3, 1, 0),
    ("experts", 1, 1, 12063, 87, 473, 6, 1, 1), ("experts", 1, 1, 13405, 960, 64, 3, 1, 0),
    ("experts", 1, 1, 13911, 64, 448, 5, 0, 1), ("experts", 1, 2, 2, 64, 128, 2, 0, 1),
    ("experts", 1, 2, 510, 70, 68, 4, 0, 1), ("experts", 1, 2, 1121, 136, 5320, 5, 1, 0),
    ("experts", 1, 2, 2788, 1728, 64, 2, 0, 1), ("experts", 1, 2, 5867, 170, 2468, 4, 0, 0),
    ("experts", 1, 2, 6566, 4416, 64, 4, 1, 0), ("experts", 1, 2, 6574, 64, 2240, 3, 1, 1),
    ("experts", 1, 2, 7226, 3292, 177, 4, 1, 1), ("experts", 1, 2, 9035, 1972, 105, 3, 1, 1),
    ("experts", 1, 2, 9421, 232, 2984, 2, 1, 1), ("experts", 1, 2, 12303, 751, 4695, 5, 1, 1),
    ("experts", 2, 0, 3, 64, 1664, 13, 0, 1), ("experts", 2, 0, 182, 1625, 2969, 51, 0, 0),
    ("experts", 2, 0, 1691, 88, 154, 6, 0, 0), ("experts", 2, 0, 4622, 1479, 90, 2, 2, 1),
    ("experts", 2, 0, 6209, 2591, 129, 13, 0, 1), ("experts", 2, 0, 7153, 64, 672, 2, 2, 0),
    ("experts", 2, 0, 8752, 2072, 160, 3, 0, 1), ("experts", 2, 0, 8972, 2056, 104, 3, 0, 0),
    ("experts", 2, 0, 12423, 168, 4008, 2, 0, 1), ("experts", 2, 0, 14080, 73, 1107, 2, 0, 1),
    ("experts", 2, 0, 15391, 1088, 4864, 3, 0, 1), ("experts", 2, 1, 7, 1216, 64, 2, 0, 1),
    ("experts", 2, 1, 16, 956, 69, 3, 2, 1), ("experts", 2, 1, 825, 1104, 5000, 65, 2, 0),
    ("experts", 2, 1, 907, 159, 67, 109, 2, 0), ("experts", 2, 1, 2311, 4942, 280, 3, 0, 1),
    ("experts", 2, 1, 4593, 64, 2688, 3, 0, 1), ("experts", 2, 1, 6872, 64, 2496, 4, 0, 1),
    ("experts", 2, 1, 8357, 1984, 3584, 2, 0, 1), ("experts", 2, 1, 11210, 172, 587, 2, 2, 0),
    ("experts", 2, 1, 12232, 2448, 80, 9, 2, 0), ("experts", 2, 1, 13967, 576, 64, 6, 2, 0),
    ("experts", 2, 2, 4, 882, 89, 2, 2, 1), ("experts", 2, 2, 15, 904, 1544, 3, 2, 1),
    ("experts", 2, 2, 48, 107, 715, 2, 0, 0), ("experts", 2, 2, 2305, 144, 2304, 12, 0, 0),
    ("experts", 2, 2, 2427, 3346, 4354, 2, 0, 0), ("experts", 2, 2, 3479, 1995, 544, 5, 0, 0),
    ("experts", 2, 2, 5493, 134, 3067, 4, 0, 0), ("experts", 2, 2, 10437, 64, 64, 15, 0, 0),
    ("experts", 2, 2, 13795, 64, 3008, 3, 0, 1), ("experts", 2, 2, 14111, 2432, 64, 2, 2, 0),
    ("experts", 2, 2, 16260, 192, 2048, 4, 0, 0), ("loss", 1, 1, 64, 257, 0, 1), ("loss", 1, 22, 142, 20064, 1, 0),
    ("loss", 1, 71, 257, 130417, 1, 1), ("loss", 1, 72, 136, 43080, 1, 0), ("loss", 1, 1366, 6040, 272, 1, 1),
    ("loss", 1, 2915, 2940, 459, 0, 1), ("loss", 1, 3199, 832, 1664, 0, 0), ("loss", 1, 4954, 64, 30784, 1, 1),
    ("loss", 1, 6598, 1728, 23808, 0, 1), ("loss", 1, 6844, 320, 21440, 1, 0), ("loss", 1, 6924, 940, 56727, 0, 0),
    ("loss", 1, 7087, 82, 1139, 0, 0), ("loss", 1, 7322, 152, 11936, 0, 1), ("loss", 1, 7711, 67, 18046, 1, 1),
    ("loss", 2, 1, 64, 896, 0, 0), ("loss", 2, 1, 69, 506, 2, 0), ("loss", 2, 1, 137, 16822, 0, 1),
    ("loss", 2, 1, 143, 46273, 0, 0), ("loss", 2, 1, 160, 35987, 0, 1), ("loss", 2, 75, 293, 92999, 2, 1),
    ("loss", 2, 84, 320, 86080, 0, 0), ("loss", 2, 1459, 6032, 320, 2, 1), ("loss", 2, 2372, 1910, 267, 0, 1),
    ("loss", 2, 3361, 64, 84096, 2, 0), ("loss", 2, 4073, 448, 2560, 2, 0), ("loss", 2, 4618, 144, 16584, 0, 0),
    ("loss", 2, 5049, 512, 5568, 2, 0), ("loss", 2, 5702, 2240, 46656, 2, 1), ("loss", 2, 6597, 192, 23424, 2, 1),
    ("loss", 2, 7081, 152, 48024, 0, 1), ("loss", 2, 7626, 520, 257, 2, 0),
    ("experts", 1, 0, 9000, 4096, 10944, 4, 1, 0), ("experts", 2, 1, 9000, 4096, 10944, 4, 2, 0),
    ("loss", 1, 8192, 4096, 40000, 1, 0), ("loss", 2, 5000, 4000, 50001, 0, 1),
]

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "arena_experts_host.cpp"
#define is_float is_float_of_loss
#include "arena_loss_host.cpp"
using namespace arena::mm;
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
static int at;
static void say(const char* fn, const GroupArgs& A, int dtype, int what, int kind)
{
    static const char* const products[] = {"rows rows", "rows cols", "cols cols", "gate up", "gate up back", "", "", "logits", "logits back"};
    static const char* const kinds[] = {"256", "128", "64 x 128", "streamed"};
    printf("{\"shape\": %d, \"call\": \"%s\", \"product\": \"%s\", \"dtype\": %d, \"act\": %d, \"kind\": \"%s\", \"any\": %s, "
           "\"splits\": %d, \"tail\": %d, \"out\": %d, \"adds\": %s, \"wide\": %s, \"pairs\": %d, \"M\": %d, \"N\": %d, \"K\": %d, "
           "\"saves\": %s}\n",
           at, fn, products[what], dtype, A.act, kinds[kind], A.any ? "true" : "false", A.splits, A.tail, A.out,
           A.beta != 0.0f ? "true" : "false", A.e_f32 ? "true" : "false", A.pairs, A.M, A.N, A.K, A.g ? "true" : "false");
}
namespace arena {
int ctx_device(const arena_ctx*) { return 0; }
void ctx_clear(arena_ctx*) {}
arena_status ctx_fail(arena_ctx*, arena_status s, const char* fmt, ...) { fprintf(stderr, "%s\n", fmt); return s; }
void sort_plan(int64_t, int*, int*) {}
hipError_t launch_route_forward(const RouteArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_route_backward(const RouteArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_sort(const SortArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_dispatch(const MoveArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_combine(const MoveArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_combine_backward(const MoveArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_loss_join(const LossArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_loss_rows(const LossArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_loss_fold(const float*, void*, int64_t, int64_t, int, int, hipStream_t) { return hipSuccess; }
namespace mm {
hipError_t launch_groups(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t)
{
    say("groups", A, dtype, what, kind);
    return hipSuccess;
}
hipError_t launch_skinny_groups(const GroupArgs& A, int dtype, Product what, hipStream_t)
{
    say(A.offsets ? "groups" : "loss", A, dtype, what, 3);
    return hipSuccess;
}
hipError_t launch_loss(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t)
{
    say("loss", A, dtype, what, kind);
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
        int dtype, act, model, inner, grad, accumulate;
        long long rows;
        if (kind[0] == 'e') {
            arena_experts_desc d;
            memset(&d, 0, sizeof(d));
            if (scanf("%d %d %lld %d %d %d %d %d", &dtype, &act, &rows, &model, &inner, &d.experts, &grad, &accumulate) != 8) return 1;
            d.dtype = dtype; d.activation = act; d.rows = rows; d.model = model; d.inner = inner;
            d.offsets = (int32_t*)p;
            d.x = d.w_gate = d.w_up = d.w_down = p;
            d.g = d.u = d.h = d.y = p;
            d.ld_x = d.ld_gate = d.ld_up = d.ld_y = model;
            d.ld_down = inner; d.ld_inner = (inner + 7) / 8 * 8;
            d.stride_gate = d.stride_up = d.stride_down = (int64_t)model * inner;
            d.workspace = p;
            check(arena_experts_forward_workspace(c, &d, &d.workspace_bytes));
            check(arena_experts_forward(c, &d, nullptr));
            arena_experts_grads g;
            memset(&g, 0, sizeof(g));
            g.grad_dtype = grad; g.accumulate = accumulate;
            g.dy = p; g.dx = g.dw_gate = g.dw_up = g.dw_down = p;
            g.ld_dy = g.ld_dx = g.ld_dw_gate = g.ld_dw_up = model; g.ld_dw_down = inner;
            g.stride_dw_gate = g.stride_dw_up = g.stride_dw_down = (int64_t)model * inner;
            check(arena_experts_backward_workspace(c, &d, &g, &d.workspace_bytes));
            check(arena_experts_backward(c, &d, &g, nullptr));
        } else {
            arena_loss_desc d;
            memset(&d, 0, sizeof(d));
            if (scanf("%d %lld %d %d %d %d", &dtype, &rows, &model, &d.vocabulary, &grad, &accumulate) != 6) return 1;
            d.dtype = dtype; d.target_dtype = ARENA_I64; d.tokens = rows; d.model = model;
            d.x = d.w = d.target = p;
            d.ld_x = d.ld_w = model;
            d.loss = d.lse = (float*)p;
            d.workspace = p;
            check(arena_cross_entropy_forward_workspace(c, &d, &d.workspace_bytes));
            check(arena_cross_entropy_forward(c, &d, nullptr));
            arena_loss_grads g;
            memset(&g, 0, sizeof(g));
            g.grad_dtype = grad; g.accumulate = accumulate;
            g.dloss = (float*)p; g.stride_dloss = 1;
            g.dx = g.dw = p;
            g.ld_dx = g.ld_dw = model;
            check(arena_cross_entropy_backward_workspace(c, &d, &g, &d.workspace_bytes));
            check(arena_cross_entropy_backward(c, &d, &g, nullptr));
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
    """One dict a product, in order.  shapes: ("experts", dtype, act, rows, model, inner, experts,
    gradients' dtype, accumulate) or ("loss", dtype, tokens, model, vocabulary, gradients' dtype,
    accumulate), in the ABI's codes, rows dense; "shape" in a dict is the index into them."""
    text = "\n".join(" ".join(str(v) for v in s) for s in shapes)
    done = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
    return [json.loads(line) for line in done.stdout.splitlines()]


def draw(rng, most, weights):
    """A shape of the ranges that the operators are used over, of at most `most` operations and
    `weights` values of weights."""
    def size(low, high, step):
        return max(low, int(math.exp(rng.uniform(math.log(low), math.log(high)))) // step * step)

    while True:
        step, typ = rng.choice((1, 8, 64, 64)), rng.choice((1, 2))
        grad, accumulate = rng.choice((typ, 0)), rng.choice((0, 1))
        if rng.random() < 0.6:
            s = ("experts", typ, rng.choice((0, 1, 2)), size(1, 16384, 1), size(64, 6144, step), size(64, 12288, step),
                 size(2, 128, 1), grad, accumulate)
            work, held = 18 * s[3] * s[4] * s[5], 3 * s[4] * s[5] * s[6]
        else:
            s = ("loss", typ, size(1, 8192, 1), size(64, 6144, step), size(257, 131072, step), grad, accumulate)
            work, held = 8 * s[2] * s[3] * s[4], s[3] * s[4]
        if work <= most and held <= weights:
            return s


def counts(rows, experts):
    """Rows of each expert, uneven and some of none: the same for the same numbers."""
    rng = random.Random(rows * 1031 + experts)
    share = [0.0 if rng.random() < 0.1 else math.exp(rng.gauss(0.0, 0.5)) for _ in range(experts)]
    if not any(share):
        share[0] = 1.0
    out = [int(rows * s / sum(share)) for s in share]
    out[share.index(max(share))] += rows - sum(out)
    return out


ROWS, COLS, BLOCKS = {"256": 256, "128": 128, "64 x 128": 64}, {"256": 256, "128": 128, "64 x 128": 128}, {"256": 256}


def shared_out(launch, shape):
    """Whether a last round of tiles goes out in parts, which the device decides from the groups' rows."""
    if launch["tail"] < 2 or launch["splits"] > 1:
        return False
    n, rows = -(-launch["N"] // COLS[launch["kind"]]), ROWS[launch["kind"]]
    blocks = BLOCKS.get(launch["kind"], 512)
    if (shape[3] // rows + min(shape[3], shape[6])) * n < blocks:
        return False
    rest = sum(-(-c // rows) for c in counts(shape[3], shape[6])) * n % blocks
    return rest > 0 and min(launch["tail"], blocks // rest) > 1


def paths(launch, shape):
    """The paths through the kernels that a launch takes: which tile of which product, how it
    is cut, and what its epilogue does."""
    what = (launch["call"], launch["product"], launch["dtype"], launch["kind"], "uneven" if launch["any"] else "even")
    if launch["kind"] == "streamed":
        what = what[:4]
    cut = "split" if launch["splits"] > 1 else "last round in parts" if shared_out(launch, shape) else "whole"
    out = [(*what, cut)]
    if launch["product"].startswith("gate up"):
        out.append((*what, cut, "activation", launch["act"]))
    if launch["product"] == "cols cols" or (launch["call"] == "loss" and launch["product"] == "rows cols"):
        out.append((launch["call"], launch["product"], launch["kind"], cut, "out", launch["out"], launch["adds"], launch["wide"]))
    return out
