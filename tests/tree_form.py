"""The rule for the columns of the attention of drafted trees (csrc/pq_tree_form.cuh) compiled for the host with g++, for tests that choose their calls by it."""
import ctypes
import functools
import os
import subprocess
import tempfile

import paper_2410_05265_b200

CSRC = os.path.join(os.path.dirname(paper_2410_05265_b200.__file__), "csrc")
SHIM = r"""
#include "pq_tree_form.cuh"
extern "C" {
int columns(int own, int n_prefix, int sms, int B, int Hkv, int G, int max_new, long long max_len, int window, int n_sink) {
  return pq_tree::columns_of(own != 0, n_prefix, sms, B, Hkv, G, max_new, max_len, window, n_sink);
}
int ctas(int columns, int own, int n_prefix) { return pq_tree::ctas_of_sm(columns, own != 0, n_prefix); }
}
"""


@functools.lru_cache(maxsize=1)
def rule():
    folder = tempfile.mkdtemp()
    src, lib = os.path.join(folder, "form.cpp"), os.path.join(folder, "form.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-x", "c++", src, "-I", CSRC, "-o", lib])
    lib = ctypes.CDLL(lib)
    lib.columns.argtypes = [ctypes.c_int] * 7 + [ctypes.c_longlong] + [ctypes.c_int] * 2
    return lib


def columns(own, n_prefix, B, Hkv, G, max_new, max_len, window=0, n_sink=0, sms=148):
    return rule().columns(int(own), n_prefix, sms, B, Hkv, G, max_new, max_len, window, n_sink)


def call_for(want, own, n_prefix, B, Hkv, G, rows, longest, window=0, n_sink=0, sms=148):
    """(max_new, max_len, sequences without rows to add) with which a call of these sizes takes so many columns. max_new and max_len are bounds that a caller may give; they
    choose the columns, whatever the rows and lengths below them are. None where no such call takes them."""
    for more in (0, 8, 30, 60, 120, 250, 500, 1000):
        for max_len in (60000, 20000, 8000, 4000, 2000, 1000, 500, 1):
            for max_new in (128, 96, 64, 48, 32, 24, 16, 8, 4, 2):
                if max_new >= rows and max_len >= longest and (not window or window >= max_new) and \
                        columns(own, n_prefix, B + more, Hkv, G, max_new, max_len, window, n_sink, sms) == want:
                    return max_new, max_len, more
    return None
