"""The plans of full attention's calls, from the library's own host code compiled for the CPU (full_plan_host.cpp)."""
import functools
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.path.dirname(os.path.dirname(os.path.realpath(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"))))


@functools.lru_cache(maxsize=None)
def _program():
    keep = tempfile.TemporaryDirectory()
    path = os.path.join(keep.name, "plans")
    subprocess.run(["g++", "-O1", "-std=c++17", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I", "/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2604_03815_amd", "csrc"),
                    os.path.join(HERE, "full_plan_host.cpp"), "-o", path], check=True)
    return keep, path


def call(bwd, H, Hk, d, dv, causal, nq, nk, graph_offsets=None, key_offsets=None, key_lengths=None):
    """A line for the program."""
    line = [int(bwd), H, Hk, d, dv, int(causal), nq, nk]
    if graph_offsets is None:
        return " ".join(map(str, line + [0]))
    ko = graph_offsets if key_offsets is None else key_offsets
    lens = [b - a for a, b in zip(ko, ko[1:])] if key_lengths is None else key_lengths
    return " ".join(map(str, [*line, len(graph_offsets) - 1, *graph_offsets, *ko, *lens]))


def plans(calls):
    """For each call a dict: "fwd", or "dq" and "dkv", -> (rows, halves, split, jobs, launches); "keys"; "status"."""
    got = subprocess.run([_program()[1]], input="\n".join(calls) + "\n", capture_output=True, text=True, check=True).stdout
    rows = []
    for line in got.splitlines():
        words, row = line.split(), {}
        while words:
            name, n = words[0], 5 if words[0] in ("fwd", "dq", "dkv") else 1
            values = tuple(map(int, words[1:1 + n]))
            row[name] = values if n > 1 else values[0]
            words = words[1 + n:]
        rows.append(row)
    assert len(rows) == len(calls)
    return rows
