"""Host-side behaviour of the rotary and block-sparse entry points, without a GPU: struct layouts, workspace sizes, launches of
nothing, and what is refused before anything touches the device."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2608_26523_b200 import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = api.VPP_ERR_INVALID_ARG, api.VPP_ERR_UNSUPPORTED, api.VPP_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2608_26523_b200 import build
    build.build()                      # nvcc cross-compiles without a GPU
    return api.load_library()


STRUCTS = [("vpp_rope_spec", api.RopeSpec, None), ("vpp_rope_args", api.RopeArgs, api._PACK_ROPE),
           ("vpp_kv_append_rope_args", api.KvAppendRopeArgs, api._PACK_APPEND_ROPE), ("vpp_block_means_args", api.BlockMeansArgs, api._PACK_MEANS),
           ("vpp_block_select_args", api.BlockSelectArgs, api._PACK_SELECT)]


@pytest.mark.parametrize("name, mirror, pack", STRUCTS)
def test_layouts_match_the_header(tmp_path, name, mirror, pack):
    """Sizes and every field's offset as a C compiler lays the header's struct out; the packed form has the fields in the same places."""
    fields = [f[0] for f in mirror._fields_]
    lines = ["printf(\"%%zu\\n\", offsetof(%s, %s));" % (name, f) for f in fields]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "vpp.h"\nint main(void){printf("%%zu\\n", sizeof(%s));%s return 0;}\n'
                   % (name, "".join(lines)))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    c = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert c == [ctypes.sizeof(mirror)] + [getattr(mirror, f).offset for f in fields]
    if pack is None:
        return
    assert ctypes.sizeof(mirror) - 8 < pack.size <= ctypes.sizeof(mirror)          # (but for the padding behind the last field)

    def leaves(cls, at=0):
        for f, t in cls._fields_:
            where = at + getattr(cls, f).offset
            if issubclass(t, ctypes.Structure):
                yield from leaves(t, where)
            else:
                yield where, t
    kinds = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f", ctypes.c_size_t: "N"}
    found = list(leaves(mirror))
    long = {"P", "q", "N"}
    codes = pack.format
    assert len(codes) == len(found)
    for i, (where, t) in enumerate(found):
        assert codes[i] == kinds[t] or {codes[i], kinds[t]} <= long
        assert struct_offset(codes, i) == where


def struct_offset(codes, i):
    """Where field i of a format string stands."""
    import struct
    before = struct.calcsize(codes[:i])
    size = struct.calcsize(codes[i])
    return (before + size - 1) // size * size


# ---- refusals: a good call's arguments, one of them changed -----------------------------------------------------------------------

buffer = torch.zeros(1 << 16, dtype=torch.uint8)
P = buffer.data_ptr() + -buffer.data_ptr() % 256


def spec(**kw):
    return api.RopeSpec(**{**dict(inv_freq=P, rot_dim=64, rot_offset=0, layout=0, amplitude=1.0), **kw})


def rope_args():
    return api.RopeArgs(x=P, out=P, x_token_stride=512, x_head_stride=128, out_token_stride=512, out_head_stride=128, prefix_len=P, chunk_len=P, num_reqs=2,
                        total_q=5, num_heads=4, head_dim=128, rope=spec())


def append_args():
    a = api.KvAppendArgs(k_new=P, v_new=P, k_cache=P, v_cache=P, k_block_stride=8192, k_token_stride=512, k_head_stride=128, v_block_stride=8192, v_token_stride=512,
                         v_head_stride=128, block_table=P, prefix_len=P, chunk_len=P, num_reqs=2, max_blocks_per_req=4, block_size=16, num_blocks=8, total_q=5,
                         max_seq_len=64, num_kv_heads=4, head_dim_qk=128, head_dim_v=128)
    return api.KvAppendRopeArgs(append=a, k_new_token_stride=512, k_new_head_stride=128, v_new_token_stride=512, v_new_head_stride=128, q=P, q_out=P,
                                q_token_stride=2048, q_head_stride=128, q_out_token_stride=2048, q_out_head_stride=128, num_q_heads=16, rope=spec())


def means_args():
    return api.BlockMeansArgs(k_cache=P, k_block_stride=8192, k_token_stride=512, k_head_stride=128, k_means=P, block_table=P, prefix_len=P, chunk_len=P, num_reqs=2,
                              max_blocks_per_req=4, block_size=16, num_blocks=8, total_q=5, num_kv_heads=4, head_dim=128)


def select_args():
    return api.BlockSelectArgs(q=P, k_means=P, block_table=P, prefix_len=P, chunk_len=P, num_reqs=2, max_blocks_per_req=4, block_size=16, num_blocks=8, total_q=5,
                               max_seq_len=64, num_q_heads=16, num_kv_heads=4, head_dim=128, topk=8, num_first=1, num_last=2, indices=P, workspace=P,
                               workspace_bytes=1 << 40)


def attn_args():
    a = api.ChunkAttnArgs()
    for f, v in dict(q=P, k_cache=P, v_cache=P, k_block_stride=8192, k_token_stride=512, k_head_stride=128, v_block_stride=8192, v_token_stride=512, v_head_stride=128,
                     block_table=P, prefix_len=P, chunk_len=P, num_reqs=2, max_blocks_per_req=4, block_size=16, num_blocks=8, total_q=5, max_seq_len=64,
                     num_q_heads=16, num_kv_heads=4, head_dim_qk=128, head_dim_v=128, softmax_scale=0.1, num_kv_splits=0, out=P, workspace=P,
                     workspace_bytes=1 << 40).items():
        setattr(a, f, v)
    return a


def call(lib, a):
    if isinstance(a, api.ChunkAttnArgs):
        return lib.vpp_block_attn_fwd(ctypes.byref(a), getattr(a, "lists", P), getattr(a, "topk", 8), 0)
    f = {api.RopeArgs: lib.vpp_rope, api.KvAppendRopeArgs: lib.vpp_kv_append_rope, api.BlockMeansArgs: lib.vpp_block_means, api.BlockSelectArgs: lib.vpp_block_select}
    return f[type(a)](bytes(a), 0)


SPEC = [(dict(inv_freq=None), INVALID), (dict(layout=2), INVALID), (dict(layout=-1), INVALID), (dict(amplitude=float("nan")), INVALID),
        (dict(amplitude=float("inf")), INVALID), (dict(rot_dim=0), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=-16), UNSUPPORTED),
        (dict(rot_dim=2048), UNSUPPORTED), (dict(rot_dim=144), INVALID), (dict(rot_offset=4), UNSUPPORTED), (dict(rot_offset=-8), UNSUPPORTED),
        (dict(rot_offset=72), INVALID), (dict(rot_offset=2 ** 31 - 8), INVALID)]
LENGTHS = [(dict(num_reqs=-1), INVALID), (dict(total_q=-1), INVALID), (dict(num_reqs=8193), UNSUPPORTED), (dict(prefix_len=None), INVALID),
           (dict(chunk_len=None), INVALID)]
PAGES = [(dict(block_table=None), UNSUPPORTED), (dict(block_size=24), UNSUPPORTED), (dict(block_size=0), UNSUPPORTED), (dict(max_blocks_per_req=0), INVALID),
         (dict(num_blocks=0), INVALID)]
HEADS = [(dict(num_kv_heads=0), INVALID), (dict(num_kv_heads=3), INVALID), (dict(num_q_heads=0), INVALID), (dict(num_q_heads=4 * 129), UNSUPPORTED)]
CASES = (
    [(rope_args, dict(rope=spec(**kw)), st) for kw, st in SPEC]
    + [(rope_args, kw, st) for kw, st in LENGTHS + [
        (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(x=P + 8), INVALID), (dict(out=P + 2), INVALID), (dict(num_heads=0), INVALID),
        (dict(head_dim=0), INVALID), (dict(head_dim=120), UNSUPPORTED), (dict(head_dim=1040), UNSUPPORTED), (dict(num_heads=65537), UNSUPPORTED),
        (dict(x_token_stride=-512), INVALID), (dict(x_head_stride=12), INVALID), (dict(out_token_stride=515), INVALID), (dict(out_head_stride=-8), INVALID)]]
    + [(append_args, dict(rope=spec(**kw)), st) for kw, st in SPEC]
    + [(append_args, {"append." + k: v for k, v in kw.items()}, st) for kw, st in LENGTHS + [
        (dict(k_new=None), INVALID), (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(k_new=P + 4), INVALID), (dict(v_cache=P + 8), INVALID),
        (dict(block_size=24), UNSUPPORTED), (dict(max_blocks_per_req=0), INVALID), (dict(num_blocks=0), INVALID), (dict(block_table=None, max_seq_len=0), INVALID),
        (dict(num_kv_heads=0), INVALID), (dict(head_dim_qk=100), UNSUPPORTED), (dict(head_dim_v=72), UNSUPPORTED), (dict(head_dim_v=1040), UNSUPPORTED),
 (dict(k_block_stride=-8), INVALID), (dict(v_token_stride=4), INVALID)]]
    + [(append_args, kw, st) for kw, st in [
        (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(num_q_heads=0), INVALID), (dict(num_q_heads=65537), UNSUPPORTED), (dict(q=P + 2), INVALID),
        (dict(k_new_token_stride=-512), INVALID), (dict(v_new_head_stride=4), INVALID), (dict(q_head_stride=100), INVALID), (dict(q_out_token_stride=-8), INVALID),
        # (the rotated part has to lie within the keys, whose heads may be narrower than the values')
        ({"append.head_dim_qk": 64, "rope": spec(rot_offset=32)}, INVALID)]]
    + [(means_args, kw, st) for kw, st in LENGTHS + PAGES + [
        (dict(k_cache=None), INVALID), (dict(k_means=None), INVALID), (dict(k_cache=P + 8), INVALID), (dict(k_means=P + 2), INVALID), (dict(num_kv_heads=0), INVALID),
        (dict(head_dim=64), UNSUPPORTED), (dict(k_block_stride=-8), INVALID), (dict(k_token_stride=4), INVALID), (dict(k_head_stride=1), INVALID)]]
    + [(select_args, kw, st) for kw, st in LENGTHS + PAGES + HEADS + [
        (dict(q=None), INVALID), (dict(k_means=None), INVALID), (dict(indices=None), INVALID), (dict(q=P + 8), INVALID), (dict(k_means=P + 8), INVALID),
        (dict(head_dim=64), UNSUPPORTED), (dict(topk=0), UNSUPPORTED), (dict(topk=257), UNSUPPORTED), (dict(num_first=-1), INVALID), (dict(num_last=0), INVALID),
        (dict(num_first=7), INVALID), (dict(num_first=2 ** 31 - 1, num_last=2 ** 31 - 1), INVALID), (dict(max_seq_len=-1), INVALID), (dict(workspace=None), WORKSPACE),
        (dict(workspace_bytes=0), WORKSPACE), (dict(workspace=P + 16), INVALID), (dict(block_size=1, max_seq_len=2 ** 31 - 1, num_reqs=8000, total_q=9000), UNSUPPORTED)]]
    + [(attn_args, kw, st) for kw, st in LENGTHS + PAGES + HEADS + [
        (dict(q=None), INVALID), (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(out=None), INVALID), (dict(lists=None), INVALID),
        (dict(q=P + 8), INVALID), (dict(out=P + 2), INVALID), (dict(v_cache=P + 4), INVALID), (dict(head_dim_qk=64), UNSUPPORTED), (dict(head_dim_v=64), UNSUPPORTED),
        (dict(head_dim_qk=576, head_dim_v=512), UNSUPPORTED), (dict(block_size=8), UNSUPPORTED), (dict(block_size=256), UNSUPPORTED), (dict(topk=0), UNSUPPORTED),
        (dict(topk=1025), UNSUPPORTED), (dict(softmax_scale=0.0), INVALID), (dict(softmax_scale=float("nan")), INVALID), (dict(softmax_scale=float("inf")), INVALID),
        (dict(num_kv_splits=-1), INVALID), (dict(num_kv_splits=65), INVALID), (dict(k_block_stride=0), INVALID), (dict(k_token_stride=100), INVALID),
        (dict(v_head_stride=-128), INVALID), (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE), (dict(workspace=P + 128), INVALID)]]
)


@pytest.mark.parametrize("make, change, status", CASES, ids=["%s-%s" % (c[0].__name__, "-".join(c[1])) for c in CASES])
def test_refusals(lib, make, change, status):
    a = make()
    for name, v in change.items():
        at, _, field = name.rpartition(".")
        setattr(getattr(a, at) if at else a, field, v)
    assert call(lib, a) == status
    assert lib.vpp_last_error()


@pytest.mark.parametrize("make", [rope_args, append_args, means_args, select_args, attn_args])
@pytest.mark.parametrize("none", ["num_reqs", "total_q"])
def test_launches_of_nothing(lib, make, none):
    """No requests or no tokens: nothing is read or written (there is no status word here to zero)."""
    a = make()
    setattr(a.append if isinstance(a, api.KvAppendRopeArgs) else a, none, 0)
    assert call(lib, a) == api.VPP_OK


@pytest.mark.parametrize("name", ["vpp_rope", "vpp_kv_append_rope", "vpp_block_means", "vpp_block_select"])
def test_null_args(lib, name):
    assert getattr(lib, name)(None, 0) == INVALID
    assert lib.vpp_block_attn_fwd(None, P, 8, 0) == INVALID
    assert lib.vpp_block_attn_workspace_size(None, 8) == 0 and lib.vpp_block_select_workspace_size(None) == 0


def test_workspace_sizes():
    size = api.vpp_block_select_workspace_size
    assert 0 < size(16, 16, 64, 8, 64, 131072) < 1 << 24
    assert size(8192, 1, 64, 4, 64, 73728) < 1 << 28
    # bounded, however long the chunk is
    assert size(1 << 20, 1, 64, 4, 64, 1 << 20) < 1 << 28
    assert size(100, 4, 8, 8, 16, 5000) == max(size(100, 4, 8, 8, 16, 5000, topk=k) for k in range(1, 257))
    assert size(10, 1, 7, 2, 16, 100, topk=8) == 0 and size(10, 1, 8, 2, 24, 100, topk=8) == 0 and size(10, 1, 8, 2, 16, 100, topk=300) == 0
    a = attn_args()
    a.num_kv_splits = 1
    one = api.vpp_block_attn_workspace_size(a, 8)
    a.num_kv_splits = 2
    a.max_seq_len = 1 << 16
    two = api.vpp_block_attn_workspace_size(a, 64)
    assert 0 < one < two and two >= 2 * 5 * 16 * 129 * 4
    assert api.vpp_block_attn_workspace_size(a, 0) == 0


def test_the_bindings_check_types_and_shapes():
    bf16 = torch.bfloat16
    x, freq, lens = torch.zeros(5, 4, 128, dtype=bf16), torch.ones(32), torch.zeros(2, dtype=torch.int32)
    cache, means = torch.zeros(8, 16, 4, 128, dtype=bf16), torch.zeros(8, 4, 128, dtype=bf16)
    table, lists = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(5, 4, 8, dtype=torch.int32)
    bad = [lambda: api.vpp_rope(x.float(), x, lens, lens, freq), lambda: api.vpp_rope(x, x[:4], lens, lens, freq),
           lambda: api.vpp_rope(x, x, lens, lens, freq.double()), lambda: api.vpp_rope(x.transpose(1, 2), x.transpose(1, 2), lens, lens, freq),
           lambda: api.vpp_kv_append_rope(x, x[:3], cache, cache, table, lens, lens, 16, 64, freq),
           lambda: api.vpp_kv_append_rope(x, x, cache, cache, table, lens, lens, 16, 64, freq, q_out=x),
           lambda: api.vpp_kv_append_rope(x, x, cache, cache, table, lens, lens, 16, 64, freq, q=x[:4], q_out=x[:4]),
           lambda: api.vpp_block_means(cache, means[:4], table, lens, lens, 16, 5), lambda: api.vpp_block_means(cache, means.float(), table, lens, lens, 16, 5),
           lambda: api.vpp_block_select(x, means, table, lens, lens, 16, 64, lists.long(), buffer),
           lambda: api.vpp_block_select(x, means, table, lens, lens, 16, 64, lists[:4], buffer),
           lambda: api.vpp_block_attn_fwd(attn_args(), lists[:, :2]), lambda: api.vpp_block_attn_fwd(attn_args(), lists.float())]
    for f in bad:
        with pytest.raises(AssertionError):
            f()
    with pytest.raises(KeyError):
        api.vpp_rope(x, x, lens, lens, freq, layout="other")
