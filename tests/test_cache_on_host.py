"""The kernels of the quantized cache, of the attention over it and of the rotation of queries and keys run on the host, thread by
thread, under the address and undefined-behaviour sanitizers, against float64 loops: every access of rings that wrap, ragged
batches, odd heads and tiles with both ends inside is checked against buffers of exactly their size."""
import os
import subprocess

import pytest

from test_kernels_on_host import HERE, ROOT, cut, read, rule


def spliced():
    def kernels(name, space, until):
        src = read(name).replace("namespace aqt {\nnamespace {", "namespace aqt {\nnamespace %s {" % space, 1)
        return src[:src.index(until)] + "}\n}\n"

    layout = read("cache.h")
    layout = layout[:layout.index("bool cache_shape_ok")] + rule("cache.hip", "CacheGeom cache_geom(") + "}\n"
    shared = cut(read("attention_cached.h"), "// part: the splits' rows", "namespace {")
    helpers = "namespace aqt {\n" + "".join(rule_line + "\n" for rule_line in (
        "inline int qmax_of(int bits) { return (1 << (bits - 1)) - 1; }", "inline bool packed4(int bits_w) { return bits_w <= 4; }")) + "}\n"
    shim = ('#define AQT_ON_HOST 1\n#include "vectors_on_host.h"\n#include "aqt.h"\n'
            "inline int __builtin_amdgcn_readlane(int v, int lane) { return lane_value(v, (unsigned)lane); }\n"
            # the data-parallel primitives of a maximum over the wavefront: row_shr:n, row_bcast:15, row_bcast:31
            "inline int __builtin_amdgcn_update_dpp(int old, int v, int ctrl, int rows, int, bool) {\n"
            "  const unsigned l = threadIdx.x & 63u;\n"
            # moves that every lane takes part in: a permutation of four, mirror images in 16 and in 8
            "  if (ctrl < 0x100) return lane_value(v, (l & ~3u) | ((unsigned)ctrl >> 2 * (l & 3u) & 3u));\n"
            "  if (ctrl == 0x140 || ctrl == 0x141) return lane_value(v, l ^ (ctrl == 0x140 ? 15u : 7u));\n"
            "  const bool shift = ctrl < 0x120, on = (rows >> (l >> 4) & 1) && (shift ? (l & 15u) >= (unsigned)(ctrl & 15) : ctrl == 0x142 ? l >= 16u : l >= 32u);\n"
            "  const int from = lane_value(v, on ? (shift ? l - (unsigned)(ctrl & 15) : ctrl == 0x142 ? (l & 48u) - 1u : 31u) : l);\n"
            "  return on ? from : old;\n}\n"
            "template <class V> inline V __builtin_nontemporal_load(const V *p) { return *p; }\n"
            "inline float __builtin_amdgcn_rsqf(float x) { return 1.0f / sqrtf(x); }\n"
            "inline float __shfl(float v, int lane) { return lane_value(v, (unsigned)lane); }\n")
    # a vector of two or four ints, by its length
    shim += "template <int N> struct key_piece_of { typedef v4i type; };\ntemplate <> struct key_piece_of<2> { typedef v2i type; };\n"
    return (shim + helpers + layout + read("lanes.h").replace('#include "aqt_internal.h"', "") + read("quant_code.h") + kernels("cache.hip", "cache_", "}  // namespace\n\nbool cache_shape_ok") +
            shared + kernels("attention_cached_few.hip", "few", "template <int DT, bool PACKED>\naqt_status launch_rows").replace(
                "typedef int key_piece __attribute__((ext_vector_type(KEYS)));", "typedef typename key_piece_of<KEYS>::type key_piece;") +
            kernels("attention_cached.hip", "attend", "constexpr int64_t kSplitTiles").replace(
                "typedef int key_piece __attribute__((ext_vector_type(KEYS)));", "typedef typename key_piece_of<KEYS>::type key_piece;") +
            kernels("rotate.hip", "turn", "__global__ void rotation_turns_kernel") +
            open(os.path.join(HERE, "host_emulation", "cache_driver.cpp")).read())


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    path = tmp_path_factory.mktemp("cache_on_host")
    (path / "cache.cpp").write_text(spliced())
    r = subprocess.run(["g++", "-O0", "-g1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
                        "-std=c++20", "-pthread", "-I", os.path.join(HERE, "host_emulation"), "-I", os.path.join(ROOT, "include"),
                        str(path / "cache.cpp"), "-o", str(path / "cache")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return str(path / "cache")


@pytest.mark.parametrize("what", [[], ["rotate"]], ids=["cache", "rotate"])
def test_kernels_in_bounds_and_correct_on_host(exe, what):
    r = subprocess.run([exe, *what], capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"), timeout=900)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-3000:], r.stderr[-3000:])
