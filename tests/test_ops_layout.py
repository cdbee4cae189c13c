"""What of the model operators' kernels can be checked without a GPU: the index arithmetic of the
tile order, of the clusters' shares and of the swizzled transposition, written out again here, and
the header as plain C99."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("tiles_m", [1, 2, 7, 8, 9, 16, 33])
@pytest.mark.parametrize("tiles_n", [1, 3, 32])
def test_every_tile_of_a_product_is_visited_once(tiles_m, tiles_n):
    group = 8
    seen = set()
    for t in range(tiles_m * tiles_n):
        per = group * tiles_n
        g, r = divmod(t, per)
        h = min(group, tiles_m - g * group)
        tm, tn = g * group + r % h, r // h
        assert 0 <= tm < tiles_m and 0 <= tn < tiles_n
        seen.add((tm, tn))
    assert len(seen) == tiles_m * tiles_n


@pytest.mark.parametrize("bn", [16, 32, 64, 128])
@pytest.mark.parametrize("splits", range(2, 9))
def test_clusters_share_the_columns_without_gap_or_overlap(bn, splits):
    groups = bn // 4
    first = [(groups * o + splits - 1) // splits for o in range(9)]
    share = (groups + splits - 1) // splits
    warps = 2 if bn >= 64 else 1
    places = set()
    for g0 in range(0, groups, groups // warps):
        owner = g0 * splits // groups
        nxt, at = first[owner + 1], (owner, g0 - first[owner])
        for g in range(g0, g0 + groups // warps):
            while g == nxt:
                owner += 1
                nxt, at = first[owner + 1], (owner, 0)
            assert owner < splits and first[owner] <= g < first[owner + 1]
            assert at == (owner, g - first[owner]) and at[1] < share
            places.add(at)
            at = (at[0], at[1] + 1)
    assert len(places) == groups
    # every CTA's part for one owner fits the owner's buffer
    assert splits * share * 2048 <= (groups + 8) * 2048


def test_swizzled_transposition_is_a_bijection_without_bank_conflicts():
    def at(r, k):
        return r * 128 + ((k ^ (r >> 3)) & 15) * 8

    assert len({at(r, k) for r in range(128) for k in range(16)}) == 128 * 16
    # a half-warp's writes (16 rows apart by 8, one 8-byte piece each, two pieces per warp): 64 banks'
    # worth of 4-byte words in two passes of 32
    for j in range(8):
        for ry in range(0, 16, 2):
            words = [at(cx * 8 + j, ry + h) // 4 % 32 for cx in range(16) for h in range(2)]
            assert all(words.count(w) == 2 for w in set(words))


def test_header_of_the_operators_is_plain_c99(tmp_path):
    from paper_2608_02611_b200 import build
    lib_path = build.build()
    src = tmp_path / "use_ops.c"
    src.write_text('#include "kb_ops.h"\n'
                   "int main(void) {\n"
                   "  return (int)kb_matmul_blocks(0, 0, 0, KB_F8E4M3, 0, 0, 0, KB_F8E4M3, 0, KB_SCALE_ROWS, 1, 1, 1, 0, 0,\n"
                   "                               KB_F32, 0) == KB_ERR_INVALID_ARG ? 0 : 1;\n"
                   "}\n")
    exe = tmp_path / "use_ops"
    cmd = ["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), lib_path,
           "-o", str(exe), "-Wl,-rpath," + os.path.dirname(lib_path), "-Wl,--allow-shlib-undefined"]
    done = subprocess.run(cmd, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr


def test_a_null_context_is_refused_without_a_device():
    from paper_2608_02611_b200 import binding
    L = binding.load()
    assert L.kb_quantize_blocks(None, None, 1, 1, 1, 0, 0, 0, None, 1, 3, None, None) == 1
    assert L.kb_layernorm(None, None, 1, 1, 1, 0, None, None, 0, 1e-5, None, 1, None, None, None, 0, 3, None, None) == 1
    assert L.kb_layernorm_backward(None, None, 1, None, 1, 1, 1, 0, None, 0, None, None, None, 1, None, None, None) == 1
    assert L.kb_matmul_blocks(None, None, 1, 3, None, None, 1, 3, None, 0, 1, 1, 1, None, 1, 0, None) == 1
