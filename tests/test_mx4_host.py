"""The arithmetic of the 4-bit matrices' kernels that needs no GPU (csrc/flashoptim_mx4.h), compiled into a small program."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def _run(tmp_path, body):
    """Compiles `body` as main()'s statements behind the header and returns the lines that it prints."""
    src, exe = tmp_path / "mx4.cpp", tmp_path / "mx4"
    src.write_text('#include <cstdio>\n#include <initializer_list>\n#include "flashoptim_mx4.h"\nint main() {\n' + body + "\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-I",
                    os.path.join(ROOT, "paper_2602_23349_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()


@pytest.mark.parametrize("edge,stages", [(64, 4), (128, 2), (256, 2)])
def test_copies_of_a_tile_stay_within_the_matrix(tmp_path, edge, stages):
    # every lane of every copy, those for steps behind the last one among them, of tiles of one to all rows and of sums that end
    # within a group of scales: what is fetched (16 bytes at a place below the buffer's size) lies in the tile's rows, and of
    # steps that there are it is the piece that the lane's place in LDS stands for
    out = _run(tmp_path, f"""
    const int edge = {edge}, stages = {stages};
    long long fetched = 0, outside = 0, wrong = 0, absent = 0;
    for (uint32_t rows : {{1, 2, 31, 33, edge - 1, edge}})
        for (uint32_t segments = 1; segments <= 13; ++segments) {{
            const uint32_t last = rows - 1, pitch = segments * fo::kSegmentBytes, scale_pitch = (segments + 1) / 2 * 16;
            for (uint32_t step = 0; step < segments + stages - 1; ++step) {{
                const fo::CopyBuffer b = fo::copy_buffer(rows * pitch, step * fo::kSegmentBytes, step < segments);
                for (int copy = 0; copy < edge / 8; ++copy)
                    for (int lane = 0; lane < 64; ++lane) {{
                        const uint32_t place = fo::code_place(copy, lane, last, pitch);
                        if (place >= b.bytes) {{ absent += step < segments; continue; }}
                        ++fetched;
                        outside += place + 16 > b.bytes || b.begin + b.bytes > (uint64_t)rows * pitch;
                        const uint32_t row = copy * 8 + lane / 8, piece = (lane % 8) ^ fo::code_swizzle(row);
                        wrong += b.begin + place != (row < last ? row : last) * pitch + step * fo::kSegmentBytes + piece * 16;
                    }}
            }}
            const uint32_t groups = (segments + fo::kScaleSteps - 1) / fo::kScaleSteps;
            for (uint32_t group = 0; group <= groups; ++group) {{
                const fo::CopyBuffer b = fo::copy_buffer(rows * scale_pitch, group * fo::kScaleBytes, group < groups);
                for (int copy = 0; copy < edge / 32; ++copy)
                    for (int lane = 0; lane < 64; ++lane) {{
                        const uint32_t place = fo::scale_place(copy, lane, last, scale_pitch);
                        const uint32_t row = copy * 32 + lane / 2, piece = (lane % 2) ^ fo::scale_swizzle(row), own = row < last ? row : last;
                        const bool used = group < groups && group * fo::kScaleBytes + piece * 16 < scale_pitch;
                        if (place >= b.bytes) {{ absent += used; continue; }}
                        ++fetched;
                        outside += place + 16 > b.bytes || b.begin + b.bytes > (uint64_t)rows * scale_pitch;
                        if (used) wrong += b.begin + place != own * scale_pitch + group * fo::kScaleBytes + piece * 16;
                    }}
            }}
        }}
    std::printf("%lld %lld %lld %lld\\n", fetched, outside, wrong, absent);
    """)
    fetched, outside, wrong, absent = (int(x) for x in out[0].split())
    assert fetched > 100000 and outside == 0 and wrong == 0 and absent == 0


def test_quantisation_beyond_one_launch_is_refused(tmp_path):
    # out_t alone admits a matrix of up to 2^31 rows of a few columns, whose tiles would be more than 2^32 lanes
    import paper_2602_23349_amd as fo
    from paper_2602_23349_amd import binding as B
    call = fo.load_library().flashoptim_mx4_quantize
    for rows, cols in ((1 << 29, 1), (1 << 30, 1), (1 << 30, 8), ((1 << 31) - 1, 1), (1 << 29, 63)):
        x, out_t = B._Matrix(4096, rows, cols, cols, 0), B._Mx4(4096, 4096, cols, rows)
        assert call(x, None, None, None, out_t, None) == -3, (rows, cols)
        assert call(x, None, 4096, None, out_t, None) == -3, (rows, cols)
    # and whatever is accepted, by itself or with `out` (2^27 segments at most in either direction), fits
    out = _run(tmp_path, """
    long long accepted = 0, wrong = 0;
    for (int r = 0; r <= 31; ++r)
        for (int c = 0; c <= 31; ++c)
            for (int d = -1; d <= 1; ++d) {
                const int64_t rows = ((int64_t)1 << r) + d, cols = ((int64_t)1 << c) + d;
                if (rows < 1 || cols < 1 || rows >= (int64_t)1 << 31 || cols >= (int64_t)1 << 31) continue;
                const bool fits = fo::quantize_fits(rows, cols), lanes = fo::quantize_tiles(rows, cols) * 256 < (int64_t)1 << 32;
                wrong += fits != lanes;
                if (fo::quantize_tile_rows(rows, cols) == 64) wrong += fits != (fo::up(rows, 256) * fo::up(cols, 256) < 1 << 21);
                else wrong += !fits;
                const bool both = rows * (fo::up(cols, 256) + 1) <= 1 << 27 && cols * (fo::up(rows, 256) + 1) <= 1 << 27;
                wrong += both && !fits;
                accepted += fits;
            }
    std::printf("%lld %lld\\n", accepted, wrong);
    """)
    accepted, wrong = (int(x) for x in out[0].split())
    assert accepted > 1000 and wrong == 0


def test_sizes_of_the_tests_reach_every_way_of_dispatch(tmp_path):
    import mx4_sizes as S
    rows = "".join(f"product({m}, {n}, {k});\n" for _, m, n, k in S.PRODUCTS)
    rows += "".join(f"product({m}, {k}, {n}); product({n}, {k}, {m});\n" for _, m, n, k in S.GRADIENTS)
    rows += "".join(f"few({m}, {n}, {k});\n" for _, m, n, k in S.FEW) + "".join(f"quantised({r}, {c});\n" for _, r, c in S.QUANTISED)
    out = _run(tmp_path, """
    auto product = [](int64_t m, int64_t n, int64_t k) {
        const fo::Shape s = fo::product_shape(m, n, k);
        if (s == fo::kTiny) std::printf("16, %d wavefronts\\n", fo::sum_waves(fo::up(k, fo::kSegment)));
        else std::printf("%d\\n", s == fo::kTile64 ? 64 : s == fo::kTile128 ? 128 : 256);
    };
    auto few = [](int64_t m, int64_t n, int64_t k) {
        const fo::FewPlan p = fo::plan_few(m, n, k);
        const int64_t segments = fo::up(k, fo::kSegment), units = m * segments * (fo::kSegment / 8);
        if (!fo::takes_few_rows(m, n, k)) std::printf("no ");
        std::printf("%d x %d%s%s%s\\n", p.waves, p.tiles, segments > fo::kFewAhead * p.waves ? ", w" : "",
                    units > 64 * p.waves * fo::kFewBatch ? ", x" : "", p.workgroups > 256 ? ", 2 each" : "");
    };
    auto quantised = [](int64_t r, int64_t c) { std::printf("%d%s\\n", fo::quantize_tile_rows(r, c), r > 1024 ? ", bands" : ""); };
    """ + rows)
    pairs = [out.pop(len(S.PRODUCTS)) for _ in range(2 * len(S.GRADIENTS))]
    joined = [a if a == b else f"{a}, {b}" for a, b in zip(pairs[0::2], pairs[1::2])]
    assert joined == [g[0] for g in S.GRADIENTS]
    assert out == [s[0] for s in S.PRODUCTS + S.FEW + S.QUANTISED]
    # all there are: a sum's wavefronts and the tiles, each tile alone and in joint launches; wavefronts by tiles of few rows, with
    # further rounds where there can be any; both tiles of the quantisation
    assert {s[0] for s in S.PRODUCTS} == {f"16, {w} wavefronts" for w in (4, 8, 16)} | {"64", "128", "256"}
    assert {"64", "128", "256"} < set(joined)
    ways = {s[0] for s in S.FEW}
    assert {way.split(",")[0] for way in ways} == {f"{w} x {t}" for w in (4, 8, 16) for t in (1, 2)}
    assert {"16 x 1, w, x", "16 x 2, w, x", "8 x 2, x, 2 each", "8 x 2, w, x, 2 each"} <= ways
    assert {s[0] for s in S.QUANTISED} == {"32", "32, bands", "64", "64, bands"}
