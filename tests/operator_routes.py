"""Which kernels the product's passes launch, from the calls that the library makes on the host (no kernel runs)."""
import re
import subprocess

from tests import host_hip

# Reads cases, one a line: "forward", "dx", "dw" or "backward" (both and db), rows, outputs, inputs, "f32" or "bf16", and which of x and
# z are in 8 bits ("-", "x", "z", "xz").  Prints for each the launched kernels with their numbers of workgroups (of both products of a backward
# pass: with those of the first).  "all": every kernel that the library has.
MAIN = r"""
#include "lf_operators.h"
#include <iostream>
int main() {
    std::string what, type_name;
    while (std::cin >> what) {
        if (what == "all") {
            for (const auto& k : kernels()) std::printf("%s ", k.second.c_str());
            std::printf("\n");
            continue;
        }
        int rows, outputs, inputs;
        std::string kept;
        std::cin >> rows >> outputs >> inputs >> type_name >> kept;
        const lf_matrix_type type = type_name == "bf16" ? LF_MATRIX_BF16 : LF_MATRIX_F32;
        auto dense = [&](int cols) { return lf_matrix{some_input, cols, nullptr, 0, type}; };
        auto either = [&](char name, int cols) {
            const long long groups = (cols + 31) / 32;
            return kept.find(name) != std::string::npos ? lf_matrix{some_input, groups * 32, (unsigned char*)some_input, groups, LF_MATRIX_E4M3} : dense(cols);
        };
        const lf_matrix x = either('x', inputs), w = dense(inputs), y = dense(outputs), z = either('z', outputs), dx = dense(inputs);
        const size_t most = (size_t)1 << 50;
        used.clear();
        if (what == "forward") {
            CHECK(lf_linear_forward(rows, outputs, inputs, &x, &w, (float*)some_input, LF_ACT_RELU, nullptr, &y, &z, some_input, most,
                                    &caller_1) == LF_OK);
        } else {
            CHECK(lf_linear_backward(rows, outputs, inputs, &y, &z, LF_ACT_RELU, &x, &w, what == "dw" ? nullptr : &dx,
                                     what == "dx" ? nullptr : &w, what == "backward" ? (float*)some_input : nullptr, some_input, most,
                                     &caller_1) == LF_OK);
        }
        CHECK(used.size() == 1 && *used.begin() == (stream_t)&caller_1);
        for (size_t i = 0; i < launched.size(); ++i)
            std::printf("%s:%u:%u ", launched[i].c_str(), workgroups[i], first_workgroups[i]);
        std::printf("\n");
        launched.clear();
        workgroups.clear();
        first_workgroups.clear();
    }
    return failures != 0;
}
"""


def _with_workgroups(prologue):
    """The host's HIP entry points, which also write down a launch's workgroups and, of two products in one launch, the first's."""
    for old, new in (("int __hipPushCallConfiguration(dim3, dim3, size_t, stream_t s) { launch_stream = s;",
                      "static unsigned grid_x;\nstatic std::vector<unsigned> workgroups, first_workgroups;\n"
                      "int __hipPushCallConfiguration(dim3 g, dim3, size_t, stream_t s) { launch_stream = s; grid_x = g.x * g.y;"),
                     ("int hipLaunchKernel(const void* f, dim3, dim3, void**, size_t, stream_t s) {",
                      "int hipLaunchKernel(const void* f, dim3, dim3, void** args, size_t, stream_t s) {\n"
                      "    workgroups.push_back(grid_x);\n"
                      "    first_workgroups.push_back(kernels()[f].find(\"k_both\") != std::string::npos ? *(unsigned*)args[2] : 0);")):
        assert old in prologue
        prologue = prologue.replace(old, new)
    return prologue


def build(directory, monkeypatch):
    monkeypatch.setattr(host_hip, "PROLOGUE", _with_workgroups(host_hip.PROLOGUE))
    return host_hip.build(directory, MAIN)


def name_of(symbol):
    """(kernel, [template arguments]): types by their names, numbers and truth values as digits."""
    m = re.match(r"_ZN2lf3ops\d+_GLOBAL__N_1\d+(k_[a-z_]+)(?:I((?:DF16b|f|Li\d+E|Lb[01]E)+)E)?", symbol)
    arguments = re.findall(r"DF16b|f|\d+(?=E)", m.group(2) or "")
    return m.group(1), [{"DF16b": "bf16", "f": "f32"}.get(a, a) for a in arguments]


def kernels(program, cases):
    """For each case the launches: (kernel, template arguments, workgroups, the first product's of two)."""
    lines = "".join(" ".join(map(str, c)) + "\n" for c in cases)
    out = subprocess.run([program], input=lines, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-2000:]
    found = []
    for line in out.stdout.splitlines():
        launches = []
        for launch in line.split():
            symbol, all_, first = launch.split(":")
            launches.append((*name_of(symbol), int(all_), int(first)))
        found.append(launches)
    return found


def of_library(program):
    """Every kernel of the operators that the library has: (kernel, template arguments)."""
    out = subprocess.run([program], input="all\n", capture_output=True, text=True, timeout=120)
    return [name_of(s) for s in out.stdout.split() if s.startswith("_ZN2lf3ops")]


def tiles(m, n, tile):
    return -(-m // tile) * -(-n // tile)


def describe(case, launches):
    """The products among a case's launches: use, tile, groups of waves, and whether the contraction is split."""
    what, rows, outputs, inputs = case[:4]
    sizes = {"forward": (rows, outputs), "dx": (rows, inputs), "dw": (outputs, inputs)}
    found = []
    for kernel, args, workgroups, first in launches:
        if kernel == "k_few":
            found.append(f"forward {args[2]} rows, {args[3]} waves")
        elif kernel == "k_product":
            use = "forward" if args[4] == "0" else "dx" if args[3] == "0" else "dw"
            split = workgroups > tiles(*sizes[use], int(args[5]))
            found.append(f"{use} {args[5]}, {args[9]} groups" + " narrow" * (args[11] == "1") + " split" * split)
        elif kernel == "k_both":
            splits = [n > tiles(*sizes[use], int(args[3])) for use, n in (("dx", first), ("dw", workgroups - first))]
            found.append(f"both {args[3]}, {args[4]} groups" + " dx split" * splits[0] + " dw split" * splits[1])
    return found


# Cases that take every kernel of the products, each with ends in every direction (no size is a multiple of any tile's, nor of a vector).
# The sizes follow from the choice of the tiles; where that changes, they do.
CASES = [
    *[(("forward", rows, 333, 777, dtype, kept), [f"forward {rows if rows < 3 else 4} rows, {16 if 'z' in kept else 4} waves"])
      for rows in (1, 2, 3) for dtype in ("bf16", "f32") for kept in ("-", "x", "z", "xz")],
    *[((*sizes, dtype, kept), [want])
      for dtype in ("bf16", "f32") for kept in ("-", "xz")
      for sizes, want in [
          (("forward", 130, 257, 7), "forward 64, 1 groups narrow"), (("dx", 130, 257, 5), "dx 64, 1 groups narrow"),
          (("dx", 300, 7, 201), "dx 64, 1 groups narrow"), (("dw", 301, 6, 131), "dw 64, 1 groups narrow"),
          (("dw", 301, 131, 6), "dw 64, 2 groups" if kept == "xz" else "dw 64, 1 groups narrow"),      # (8 bits come in whole groups)
          (("dw", 5, 131, 203), "dw 64, 2 groups"),
          (("forward", 301, 259, 103), "forward 64, 2 groups"), (("dx", 301, 103, 259), "dx 64, 2 groups"),
          (("dw", 103, 301, 259), "dw 64, 2 groups"),
          (("forward", 101, 131, 2051), "forward 64, 2 groups split"), (("dx", 101, 2051, 131), "dx 64, 2 groups split"),
          (("dw", 2051, 101, 131), "dw 64, 2 groups split"),
          (("forward", 131, 6101, 77), "forward 64, 1 groups"), (("dx", 131, 77, 6101), "dx 64, 1 groups"),
          (("dw", 77, 131, 6101), "dw 64, 1 groups"),
          (("backward", 45, 101, 77), "both 64, 2 groups"), (("backward", 1541, 45, 39), "both 64, 2 groups dw split"),
          (("backward", 45, 1541, 39), "both 64, 2 groups dx split"),
          (("backward", 131, 67, 6101), "both 64, 1 groups"),
      ]],
    *[((*sizes, "bf16", kept), want)
      for kept in ("-", "xz")
      for sizes, want in [
          (("forward", 421, 7001, 77), ["forward 128, 2 groups"]), (("dx", 421, 77, 7001), ["dx 128, 2 groups"]),
          (("dw", 77, 421, 7001), ["dw 128, 2 groups"]),
          (("forward", 901, 1101, 3003), ["forward 128, 2 groups split"]), (("dx", 901, 3003, 1101), ["dx 128, 2 groups split"]),
          (("dw", 3003, 901, 1101), ["dw 128, 2 groups split"]),
          (("forward", 2051, 3003, 131), ["forward 128, 1 groups"]), (("dx", 2051, 131, 3003), ["dx 128, 1 groups"]),
          (("dw", 131, 2051, 3003), ["dw 128, 1 groups"]),
          (("forward", 2051, 6101, 333), ["forward 256, 1 groups"]), (("dx", 2051, 333, 6101), ["dx 256, 1 groups"]),
          (("dw", 333, 2051, 6101), ["dw 256, 1 groups"]),
          (("forward", 1541, 2603, 5003), ["forward 256, 1 groups split"]), (("dx", 1541, 5003, 2603), ["dx 256, 1 groups split"]),
          (("dw", 5003, 1541, 2603), ["dw 256, 1 groups split"]),
          (("backward", 257, 421, 7001), ["both 128, 1 groups"]), (("backward", 2051, 517, 1803), ["both 128, 1 groups dw split"]),
          (("backward", 517, 2051, 1803), ["both 128, 1 groups dx split"]),
          (("backward", 3003, 3003, 333), ["both 128, 1 groups dx split dw split"]),
          (("backward", 2051, 2043, 2021), ["dx 64, 1 groups", "dw 128, 2 groups"]),
          (("backward", 4091, 8181, 8171), ["dx 256, 1 groups", "dw 256, 1 groups"]),
      ]],
]
