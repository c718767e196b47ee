"""Where the loads of the pipeline over dense keys start, and that every kernel's buffer loads are looked at (no GPU needed).

The pipeline runs to a multiple of four tiles and brings keys four tiles ahead: up to seven tiles behind the last one.  Their
scalar offsets have to stop at the descriptor's end like any other, and no product on the way may leave 31 bits."""
import os
import re
import subprocess

from paper_2510_21270_amd import build
from test_load_places_cpu import SCALAR_OFFSET, WITHIN as LOOKED_AT, _arguments


def _source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_tiles_behind_the_last_key_start_at_the_end(tmp_path):
    # the loop that the places below follow
    text = _source("key_pipeline.h")
    assert "where = src.at(t + (wave == 0 ? 4 : 3));" in text and "if (t + 4 >= tiles) break;" in text
    assert "else return {tile_start(t, tiles, tile_bytes, size)};" in text
    # factors beside the rows: parts of 1024 keys at most, rows of 256 bytes, and seven tiles
    assert "if constexpr (F) return {scalar_offset(t * tile_bytes, size)};" in text
    prefix = _source("prefix_attn.hip")
    assert "s.tile_bytes = KS * D * 2;" in prefix and "Rows<D, true> s;" in prefix and "Rows<D, false>" not in prefix
    assert "if (a.p_chunk > 1024) a.p_chunk = 1024;" in _source("decode_attn.hip")
    assert "if (!rows_have_places(p->total_k, prompt::KS, stride * 2, p->d * 2)) return PBS_ERR_UNSUPPORTED;" in _source("prompt_attn.hip")
    code = """
#include <cstdio>
#include <initializer_list>
#include "load_places.h"
typedef long long i64;
constexpr int KS = 32;
// every tile that is brought for `keys` keys, step bytes apart
static int walk(i64 keys, i64 step, int row)
{
    const int tile_bytes = (int)(KS * step), size = (int)((keys - 1) * step + row), tiles = (int)((keys + KS - 1) / KS);
    auto look = [&](int t) {
        if (t < tiles && (i64)t * tile_bytes > 0x7fffffffll) return 1;
        const int at = pbs::tile_start(t, tiles, tile_bytes, size);
        if (at < 0 || at > size) return 2;
        if (t < tiles && at != (i64)t * tile_bytes) return 3;                   // the tiles that hold keys are themselves
        if (t >= tiles && at != size) return 4;                                 // the others are nothing
        return 0;
    };
    for (int t = 0; t < 4; ++t)
        if (const int bad = look(t)) return bad;
    const int from = tiles > 40 ? (tiles - 40) / 4 * 4 : 0;                     // (the tiles between are in order)
    for (int t = from;; t += 4) {
        for (int k = 0; k < 4; ++k)
            for (int ahead = 3; ahead <= 4; ++ahead)
                if (const int bad = look(t + k + ahead)) return bad;
        if (t + 4 >= tiles) break;
    }
    return 0;
}
int main()
{
    int looked = 0;
    for (int row = 128; row <= 256; row += 128)
        for (i64 step : {(i64)row, (i64)row + 16, (i64)4 * row, (i64)8 * row, (i64)32 * row, (i64)12288, (i64)1 << 16, (i64)1 << 21, (i64)5000016,
                         (i64)1 << 24, (i64)0x7fffffff / 66 / 16 * 16}) {
            i64 most = 0x7fffffffll / step + 2;                                  // the longest accepted
            while (most > 0 && !pbs::rows_have_places(most, KS, step, row)) --most;
            if (most < 1 || pbs::rows_have_places(most + 1, KS, step, row)) return 9;
            for (i64 keys = most > 600 ? most - 600 : 1; keys <= most; ++keys, ++looked)
                if (const int bad = walk(keys, step, row)) {
                    std::printf("%d: %lld keys, %lld bytes apart\\n", bad, keys, step);
                    return bad;
                }
            for (i64 keys = 1; keys <= 300 && keys <= most; ++keys, ++looked)
                if (const int bad = walk(keys, step, row)) return bad;
        }
    std::printf("all places hold, %d lengths\\n", looked);
}
"""
    src, exe = str(tmp_path / "places.cpp"), str(tmp_path / "places")
    with open(src, "w") as f:
        f.write(code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, src, "-o", exe], check=True)
    out = subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout
    assert "all places hold" in out


# scalar offsets by which no load of the pipeline starts behind its descriptor, and why; the other files' stand in
# test_load_places_cpu.py
WITHIN = {
    "key_pipeline.h": {
        "w.rows": "Rows::at forms it by tile_start, or scalar_offset",
        "scalar_offset(t * KS * 4, factors_size)": "stops at the end",
    },
    "prefix_attn.hip": {},                                 # a descriptor to every tile
}


def test_no_load_of_the_pipeline_starts_behind_its_descriptor():
    for name, known in WITHIN.items():
        text, found = _source(name), 0
        for m in re.finditer(r"\b(%s)\(" % "|".join(SCALAR_OFFSET), text):
            offset = " ".join(_arguments(text, m.end() - 1)[SCALAR_OFFSET[m.group(1)]].split())
            found += 1
            assert offset == "0" or offset in known, (name, offset)
        assert found, name


def test_every_file_with_buffer_loads_is_looked_at():
    for name in sorted(os.listdir(build.CSRC)):
        if not name.endswith((".hip", ".h")):
            continue
        loads = set(re.findall(r"\b__builtin_amdgcn_(?:raw|struct)_\w*buffer_load\w*", _source(name)))
        assert not loads or name in WITHIN or name in LOOKED_AT, name
        assert loads <= set(SCALAR_OFFSET), (name, loads)  # each with a known place of its scalar offset
        assert "buffer_load" not in re.sub(r"__builtin_amdgcn_\w+", "", _source(name)), name
