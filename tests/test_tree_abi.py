"""CPU: what the operators on trees and on 8-bit pages refuse, before anything reaches a GPU; page addressing and plain
implementations by hand."""
import ctypes as C

import numpy as np
import pytest

import paper_2407_19947_amd as pkg
import trees_util as tu

P = 1 << 20                        # an aligned address nobody reads: the calls are refused


def cache(**kw):
    return pkg.StairsPagedCache(**dict(dict(k=P, v=P, dtype=pkg.DTYPE_BF16, n_pages=8, page_size=64, n_kv_heads=4, head_dim=128, held=pkg.DTYPE_E4M3, scale=P), **kw))


def rows(**kw):
    return pkg.StairsPagedRows(**dict(dict(rows=3, n_heads=8, q=P, k=P, v=P, q_out=P, q_stride=1024, k_stride=512, v_stride=512, q_out_stride=1024,
                                           position=P, slot=P, rope_theta=1e4), **kw))


def attn(**kw):
    return pkg.StairsPagedAttention(**dict(dict(n_seqs=2, max_blocks=4, rows=4, n_heads=8, max_fresh=2, q=P, out=2 * P, q_stride=1024, out_stride=1024,
                                                block_table=P, row_start=P, seq_len=P, scale=0.0, workspace=P, workspace_bytes=1 << 40), **kw))


def read(**kw):
    return pkg.StairsPagedRead(**dict(dict(rows=3, k=P, v=P, k_stride=512, v_stride=512, slot=P), **kw))


def tree(**kw):
    return pkg.StairsTree(**dict(dict(n_seqs=2, rows=9, row_start=P, seq_len=P, parent=P, position=P, sees=P), **kw))


def walk(**kw):
    return pkg.StairsTreeWalk(**dict(dict(n_seqs=2, rows=9, row_start=P, seq_len=P, parent=P, token=P, predicted=P, kept=P, cached=P, path=P, emitted=P), **kw))


def path(**kw):
    return pkg.StairsPagedPath(**dict(dict(n_seqs=2, max_blocks=4, rows=9, block_table=P, row_start=P, seq_len=P, path=P, kept=P), **kw))


def refused(call, code=-1):
    with pytest.raises(pkg.StairsError) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("bad", [dict(scale=None), dict(scale=P + 8), dict(held=1), dict(held=-1), dict(held=pkg.DTYPE_FP16), dict(dtype=pkg.DTYPE_E4M3),
                                 dict(dtype=pkg.DTYPE_FP32), dict(k=P + 8), dict(page_size=48), dict(head_dim=96)])
def test_a_pool_that_is_none_is_refused(bad):
    for call in (lambda c: pkg.stairs_paged_append(c, rows()), lambda c: pkg.stairs_paged_attention(c, attn()), lambda c: pkg.stairs_paged_read(c, read()),
                 lambda c: pkg.stairs_paged_attention_workspace(c, attn()), lambda c: pkg.stairs_paged_compact([c], path()),
                 lambda c: pkg.stairs_paged_compact([cache(), c], path())):
        refused(lambda: call(cache(**bad)))


@pytest.mark.parametrize("bad", [dict(sees=P + 4), dict(q=P + 8), dict(n_heads=6), dict(out=P), dict(workspace=None)])
def test_attention_refuses(bad):
    refused(lambda: pkg.stairs_paged_attention(cache(), attn(**bad)))
    refused(lambda: pkg.stairs_paged_attention(cache(held=0, scale=None), attn(**dict(dict(sees=P), **bad))))


def test_attention_refuses_a_workspace_that_is_too_small():
    need = pkg.stairs_paged_attention_workspace(cache(), attn())
    refused(lambda: pkg.stairs_paged_attention(cache(), attn(workspace_bytes=need - 1)), -2)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 29) - 31), dict(slot=None), dict(k=P + 8), dict(v=P + 2), dict(k_stride=504), dict(v_stride=516),
                                 dict(k_stride=-512)])
def test_read_refuses(bad):
    refused(lambda: pkg.stairs_paged_read(cache(), read(**bad)))
    refused(lambda: pkg.stairs_paged_read(cache(held=0), read(**bad)))


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=1025), dict(rows=-1), dict(row_start=None), dict(seq_len=None), dict(parent=None), dict(sees=None),
                                 dict(sees=P + 4)])
def test_tree_plan_refuses(bad):
    refused(lambda: pkg.stairs_tree_plan(tree(**bad)))


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=1025), dict(rows=-1)] + [{k: None} for k in ("row_start", "seq_len", "parent", "token", "predicted",
                                                                                                         "kept", "cached", "path", "emitted")])
def test_tree_walk_refuses(bad):
    refused(lambda: pkg.stairs_tree_walk(walk(**bad)))


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=1025), dict(rows=-1), dict(max_blocks=0), dict(max_blocks=1 << 25)] +
                         [{k: None} for k in ("block_table", "row_start", "seq_len", "path", "kept")])
def test_compact_refuses(bad):
    refused(lambda: pkg.stairs_paged_compact([cache()], path(**bad)))


@pytest.mark.parametrize("other", [dict(n_pages=9), dict(page_size=32), dict(n_kv_heads=2), dict(head_dim=64), dict(dtype=pkg.DTYPE_FP16), dict(held=0)])
def test_compact_refuses_pools_of_different_shapes(other):
    refused(lambda: pkg.stairs_paged_compact([cache(), cache(k=2 * P, v=2 * P, scale=2 * P), cache(**dict(dict(k=3 * P, v=3 * P, scale=3 * P), **other))], path()))


@pytest.mark.parametrize("twice", [dict(v=3 * P, scale=3 * P), dict(k=3 * P, scale=3 * P), dict(k=3 * P, v=3 * P), dict()])
def test_compact_refuses_a_pool_twice(twice):
    refused(lambda: pkg.stairs_paged_compact([cache(), cache(k=2 * P, v=2 * P, scale=2 * P), cache(**twice)], path()))
    pkg.stairs_paged_compact([cache(), cache(k=2 * P, v=2 * P, scale=2 * P)], path(rows=0))


def test_null_arguments_and_nothing_to_do():
    L = pkg.lib()
    assert L.stairs_paged_read(None, read(), None) == -1 and L.stairs_paged_read(cache(), None, None) == -1
    assert L.stairs_tree_plan(None, None) == -1 and L.stairs_tree_walk(None, None) == -1
    assert L.stairs_paged_compact(cache(), 1, None, None) == -1 and L.stairs_paged_compact(None, 1, path(), None) == -1
    assert L.stairs_paged_compact(cache(), -1, path(), None) == -1 and L.stairs_paged_compact(cache(), 4097, path(), None) == -1
    assert L.stairs_paged_compact(None, 0, path(), None) == 0
    pkg.stairs_paged_read(cache(), read(rows=0))
    pkg.stairs_paged_read(cache(), read(k=None, v=None))
    pkg.stairs_tree_plan(tree(rows=0))
    pkg.stairs_tree_walk(walk(rows=0, n_seqs=0))
    pkg.stairs_paged_compact([], path())
    pkg.stairs_paged_compact([cache()], path(n_seqs=0))
    pkg.stairs_paged_compact([cache()], path(rows=0))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ps", [32, 64, 256])
def test_every_number_of_an_8_bit_page_has_a_place_of_its_own(ps, hd):
    p, e = np.meshgrid(np.arange(ps), np.arange(hd), indexing="ij")
    for at in (tu.held_key_at, tu.held_value_at):
        assert np.array_equal(np.sort(at(p, e, hd).ravel()), np.arange(ps * hd))
    p = np.arange(ps)
    assert np.array_equal(np.sort(np.concatenate([tu.held_scale_at(p, 0), tu.held_scale_at(p, 1)])), np.arange(2 * ps))


def test_the_8_bit_format_by_hand():
    assert tu.DECODE[0x7E] == 448 and tu.DECODE[0x38] == 1 and tu.DECODE[1] == 2.0 ** -9 and tu.DECODE[0x08] == 2.0 ** -6 and np.isnan(tu.DECODE[0xFF])
    assert tu.DECODE[tu.encode(np.array([17.0, 19.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 448.0, 1.0625, 1.1875]))].tolist() == [
        16, 20, -16, 0, 2.0 ** -8, 448, 1, 1.25]             # halfway: the even code
    x = np.array([[1.0, -3.5], [0.0, 0.0], [448.0, 1.0], [449.0, 1.0], [np.inf, 2.0], [2.0 ** -140, 0.0]])
    assert tu.scale_byte(x).tolist() == [120, 1, 127, 128, 120, 1]     # (3.5 = 448 / 128; 2 needs 2^-7 too: 448 / 256 = 1.75)
    codes, b = tu.quantise(x)
    got = tu.values_of(codes, b)
    assert tu.values_of(*tu.quantise(np.array([[65504.0, -57344.0, 63000.0, np.inf]]), "fp16"))[0, :3].tolist() == [61440, -57344, 61440]
    assert got[0].tolist() == [1.0, -3.5] and got[3].tolist() == [448.0, 1.0] and np.isnan(got[4, 0]) and got[4, 1] == 2.0


def test_the_8_bit_rounding_is_torchs():
    import torch
    y = torch.linspace(-448, 448, 40001, dtype=torch.float64)
    y = torch.cat([y, y / 3000, torch.from_numpy((tu.DECODE[:126] + tu.DECODE[1:127]) / 2)])
    want = y.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(tu.encode(y.float().double().numpy()), want)


def test_the_trees_references_by_hand():
    #   0 - 1 - 3      (a chain beside: 5, whose parent is none)
    #     - 2 - 4
    parent = [-1, 0, 0, 1, 2, 7]
    position, sees = tu.tree_reference([0, 6], [16], parent, 7)
    assert position.tolist() == [10, 11, 11, 12, 12, 10, -1] and sees.tolist() == [1, 3, 5, 11, 21, 32, 0]
    kept, cached, path, emitted = tu.walk_reference([0, 6], [16], parent, [9, 4, 5, 6, 7, 8], [5, 0, 7, 0, 3, 0], 7, [10])
    assert kept == [3] and cached == [13] and path.tolist() == [0, 2, 4, -1, -1, -1, -1] and emitted.tolist() == [5, 7, 3, -1, -1, -1, -1]


def test_structures_lie_as_the_header_has_them(tmp_path):
    """Sizes and offsets of the operators' structures, by a C compiler; built from zeros, members that were added last mean what was before them."""
    import os
    import subprocess
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    classes = [pkg.StairsPagedCache, pkg.StairsPagePlan, pkg.StairsPagedRows, pkg.StairsPagedAttention, pkg.StairsPagedRead, pkg.StairsTree, pkg.StairsTreeWalk,
               pkg.StairsPagedPath, pkg.StairsSampling]
    lines, want = [], []
    for c in classes:
        name = c.__doc__.split(":")[0]
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        want.append(f"{name} {C.sizeof(c)}")
        for field, _ in c._fields_:
            lines.append(f'printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
            want.append(f"{name}.{field} {getattr(c, field).offset}")
    zeros = "stairs_paged_cache c = {0}; stairs_paged_attn a = {0}; if (c.held || c.scale || a.sees) return 1;"
    (tmp_path / "layout.c").write_text("#include <stddef.h>\n#include <stdio.h>\n#include <string.h>\n#include \"stairs.h\"\nint main(void) {" + zeros + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", include, "-o", tmp_path / "layout", tmp_path / "layout.c"], check=True)
    out = subprocess.run([tmp_path / "layout"], check=True, capture_output=True, text=True).stdout
    assert out.split("\n")[:-1] == want
