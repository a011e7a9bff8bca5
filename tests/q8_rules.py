"""The split rules of the 8-bit decode steps as the library has them: csrc/decode_plan.h compiled for the host, so that a test can state
the route of each of its cases."""
import atexit
import ctypes as C
import functools
import os
import shutil
import subprocess
import tempfile
from types import SimpleNamespace

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("whole", "rb_max", "chunk_a", "splits_a", "chunk_b", "splits_b", "items_a", "items_b", "off_ml", "bytes")
SHIM = r"""
#include "decode_plan.h"
extern "C" int q8_rules(const dag_decode_desc_t* d, int hq, int hkv, int D, double* out) {
  Q8Plan p{};
  const int rc = make_q8_plan(d, hq, hkv, D, &p);
  const double v[] = {(double)p.whole, (double)p.rb_max, (double)p.chunk_a, (double)p.splits_a, (double)p.chunk_b, (double)p.splits_b,
                      (double)p.items_a, (double)p.items_b, (double)p.off_ml, (double)p.bytes};
  for (int i = 0; i < 10; ++i) out[i] = v[i];
  return rc;
}
extern "C" int q8_segment_rules(const dag_decode_seg_desc_t* d, int hkv, int D) { return q8_whole_segments(d, hkv, D); }
"""


@functools.lru_cache(maxsize=None)
def _lib():
    folder = tempfile.mkdtemp()
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    src, so = os.path.join(folder, "rules.cpp"), os.path.join(folder, "rules.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2602_07529_amd", "csrc"), src, "-o", so], check=True)
    return C.CDLL(so)


def plan(desc, hq, hkv, d):
    """Plan of dag_attn_decode_q8 for a dag_decode_desc_t."""
    out = (C.c_double * len(NAMES))()
    rc = _lib().q8_rules(C.byref(desc), hq, hkv, d, out)
    return SimpleNamespace(rc=rc, **{n: int(v) for n, v in zip(NAMES, out)})


def segments_whole(desc, hkv, d):
    return bool(_lib().q8_segment_rules(C.byref(desc), hkv, d))
