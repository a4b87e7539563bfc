"""Which kernels the student nets' operators launch, from the calls that the library makes on the host (no kernel runs)."""
import re
import subprocess

from tests import host_hip

# Reads cases, one a line, and prints for each the launched kernels with their numbers of workgroups and of a workgroup's threads.
#   norm rows cols type out                     the layer norm's forward pass; out: "-" (the type), "e4m3", "e4m3_128"
#   norm_back rows cols type sum wanted         its backward pass; sum: "-" or "e4m3"; wanted: "dx", "all"
#   save rows cols type kind which              into blocks of 128; kind: "rows", "tiles"; which: "out", "out_t", "both"
#   load rows cols type kind
#   product rows outputs inputs type x y        x: "-" or "e4m3_128"; y (and z): "-" or "e4m3_128"
#   product_back rows outputs inputs type wanted    wanted: "dx", "dw", "all"
#   distil rows classes top type wanted         wanted: "loss", "all"
#   all                                         every kernel that the library has
MAIN = r"""
#include "lf_operators.h"
#include <iostream>
int main() {
    std::string what;
    const auto number = [] { long long n; std::cin >> n; return (int)n; };
    const auto word = [] { std::string w; std::cin >> w; return w; };
    const auto type_of = [](const std::string& w) { return w == "f32" ? LF_MATRIX_F32 : LF_MATRIX_BF16; };
    const auto matrix = [](lf_matrix_type type, int cols) {
        const long long group = type == LF_MATRIX_E4M3 ? 32 : 128, groups = (cols + group - 1) / group;
        if (type == LF_MATRIX_F32 || type == LF_MATRIX_BF16) return lf_matrix{some_input, cols, nullptr, 0, type};
        return lf_matrix{some_input, groups * group, (unsigned char*)some_input, type == LF_MATRIX_E4M3 ? groups : (groups + 3) / 4 * 4, type};
    };
    const auto kind_of = [](const std::string& w, lf_matrix_type type) {
        return w == "-" ? type : w == "e4m3" ? LF_MATRIX_E4M3 : w == "tiles" ? LF_MATRIX_E4M3_TILES : LF_MATRIX_E4M3_128;
    };
    float* const vector = (float*)some_input;
    const size_t most = (size_t)1 << 50;
    while (std::cin >> what) {
        if (what == "all") {
            for (const auto& k : kernels()) std::printf("%s ", k.second.c_str());
            std::printf("\n");
            continue;
        }
        const int rows = number(), a = number();
        used.clear();
        lf_status st = LF_OK;
        if (what == "norm") {
            const lf_matrix_type type = type_of(word());
            const lf_matrix x = matrix(type, a), y = matrix(kind_of(word(), type), a);
            st = lf_layer_norm_forward(rows, a, &x, &x, vector, vector, 1e-5f, &x, &y, vector, vector, &caller_1);
        } else if (what == "norm_back") {
            const lf_matrix_type type = type_of(word());
            const lf_matrix x = matrix(type, a), sum = matrix(kind_of(word(), type), a);
            float* const grad = word() == "all" ? vector : nullptr;
            st = lf_layer_norm_backward(rows, a, &x, &sum, vector, vector, vector, &x, &x, grad, grad, some_input, most, &caller_1);
        } else if (what == "save") {
            const lf_matrix x = matrix(type_of(word()), a);
            const lf_matrix_type kind = kind_of(word(), LF_MATRIX_BF16);
            const lf_matrix out = matrix(kind, a), out_t = matrix(kind, rows);
            const std::string which = word();
            st = lf_block_save(rows, a, &x, which == "out_t" ? nullptr : &out, which == "out" ? nullptr : &out_t, &caller_1);
        } else if (what == "load") {
            const lf_matrix out = matrix(type_of(word()), a), in = matrix(kind_of(word(), LF_MATRIX_BF16), a);
            st = lf_block_load(rows, a, &in, &out, &caller_1);
        } else if (what == "product") {
            const int inputs = number();
            const lf_matrix_type type = type_of(word());
            const lf_matrix x = matrix(kind_of(word(), type), inputs), w = matrix(LF_MATRIX_E4M3_TILES, inputs), y = matrix(kind_of(word(), type), a);
            st = lf_block_linear_forward(rows, a, inputs, &x, &w, vector, LF_ACT_RELU, nullptr, &y, &y, nullptr, some_input, most, &caller_1);
        } else if (what == "product_back") {
            const int inputs = number();
            const lf_matrix_type type = type_of(word());
            const std::string wanted = word();
            const lf_matrix dy = matrix(type, a), x_t = matrix(LF_MATRIX_E4M3_128, rows), w_t = matrix(LF_MATRIX_E4M3_TILES, a), d = matrix(type, inputs);
            st = lf_block_linear_backward(rows, a, inputs, &dy, &dy, LF_ACT_RELU, &x_t, &w_t, wanted == "dw" ? nullptr : &d, wanted == "dx" ? nullptr : &d,
                                          wanted == "all" ? vector : nullptr, some_input, most, &caller_1);
        } else {
            const int top = number();
            const lf_matrix_type type = type_of(word());
            const lf_matrix z = matrix(type, a), t = matrix(LF_MATRIX_F32, top);
            st = lf_distil(rows, a, top, &z, &t, (const int*)some_input, top, 1.0f, vector, vector, word() == "all" ? &z : nullptr, &caller_1);
        }
        if (st != LF_OK) std::printf("%s\n", lf_operator_error());
        CHECK(st == LF_OK && used.size() == 1 && *used.begin() == (stream_t)&caller_1);
        for (size_t i = 0; i < launched.size(); ++i) std::printf("%s:%llu:%llu ", launched[i].c_str(), workgroups[i], threads[i]);
        std::printf("\n");
        launched.clear();
        workgroups.clear();
        threads.clear();
    }
    return failures != 0;
}
"""


def _with_sizes(prologue):
    """The host's HIP entry points, which also write down a launch's workgroups and their threads."""
    for old, new in (("int __hipPushCallConfiguration(dim3, dim3, size_t, stream_t s) { launch_stream = s;",
                      "static unsigned long long grid, block;\nstatic std::vector<unsigned long long> workgroups, threads;\n"
                      "int __hipPushCallConfiguration(dim3 g, dim3 b, size_t, stream_t s) {\n"
                      "    launch_stream = s; grid = 1ull * g.x * g.y * g.z; block = 1ull * b.x * b.y * b.z;"),
                     ("int hipLaunchKernel(const void* f, dim3, dim3, void**, size_t, stream_t s) {",
                      "int hipLaunchKernel(const void* f, dim3, dim3, void**, size_t, stream_t s) {\n"
                      "    workgroups.push_back(grid); threads.push_back(block);")):
        assert old in prologue
        prologue = prologue.replace(old, new)
    return prologue


def build(directory, monkeypatch):
    monkeypatch.setattr(host_hip, "PROLOGUE", _with_sizes(host_hip.PROLOGUE))
    return host_hip.build(directory, MAIN)


def name_of(symbol):
    """(kernel, (template arguments)): numbers and truth values as integers."""
    m = re.match(r"_ZN2lf3ops\d+_GLOBAL__N_1\d+(k_[a-z_]+)(?:I((?:Lin?\d+E|Lb[01]E)+)E)?", symbol)
    return m.group(1), tuple(int(v.replace("n", "-")) for v in re.findall(r"L[ib](n?\d+)E", m.group(2) or ""))


def _run(program, lines):
    out = subprocess.run([program], input=lines, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-2000:]
    return out.stdout.splitlines()


def kernels(program, cases):
    """For each case the launches: (kernel, template arguments, workgroups, threads of one)."""
    found = []
    for line in _run(program, "".join(" ".join(map(str, c)) + "\n" for c in cases)):
        launches = [launch.split(":") for launch in line.split()]
        found.append([(*name_of(symbol), int(groups), int(threads)) for symbol, groups, threads in launches])
    return found


# Backward passes of products that take every way that a pass may go, each with ends in every direction: (rows, outputs, inputs), and the launches
# that follow the one that makes dz and db's partial sums, tiles and splits of dx and of dw among them.  The sizes follow from the choice of
# the tiles; where that changes, they do.
BACKWARD = [
    ((17, 8200, 2100), ["both 128, dx split", "join"]), ((3000, 130, 3333), ["both 128, dw split", "join"]),
    ((3000, 3333, 130), ["both 128, dx split, dw split", "join"]), ((300, 1100, 2050), ["both 128"]),
    ((3, 8190, 8187), ["dx few", "dw 256"]), ((2100, 5003, 2050), ["join", "dx 128", "dw 256"]), ((3001, 2050, 4100), ["join", "dx 256", "dw 256"]),
    ((9000, 2050, 2050), ["join", "dx 128", "dw 256, split", "join"]),
]


def describe_backward(sizes, launches):
    """The launches of a whole backward pass behind the first."""
    rows, outputs, inputs = sizes

    def tiles(use, tile):
        m, n = (rows, inputs) if use == "dx" else (outputs, inputs)
        return -(-m // tile) * -(-n // tile)
    assert launches[0][0] == "k_block_save"
    found, uses = [], iter(("dx", "dw"))
    for kernel, args, groups, _ in launches[1:]:
        if kernel == "k_block_join":
            found.append("join")
        elif kernel == "k_block_few":
            found.append(f"{next(uses)} few")
        elif kernel == "k_block_product":
            use = next(uses)
            found.append(f"{use} {args[0]}" + ", split" * (groups > tiles(use, args[0])))
        else:                              # (the workgroups of both products and, 512 columns each, of db's sums over more than 128 rows)
            assert kernel == "k_block_both"
            rest, x, w = groups - (-(-outputs // 512) if rows > 128 else 0), tiles("dx", 128), tiles("dw", 128)
            ways = [(i, j) for i in range(1, 257) for j in range(1, 257) if i * x + j * w == rest]
            assert ways
            found.append(f"both {args[0]}" + (", dx split" * all(i > 1 for i, _ in ways) + ", dw split" * all(j > 1 for _, j in ways)))
    return found


# Layer norms' backward passes over many rows, by the kernel that they take beside those of tests/test_gpu_layer_norm.py: (rows, columns).
NORM_BACK = {"k_layer_backward, 64 threads": [(1300, 1023), (1300, 5)], "k_layer_backward, 256 threads": [(700, 2500), (1100, 4095)],
             "k_layer_backward, 512 threads": [(1030, 5000), (1100, 8191)], "k_layer_backward_few, 512 threads": [(1024, 4097)],
             "k_layer_gradients, 256 threads": [(600, 9001)]}
