"""What the long-context calls refuse, on the host and before any launch; layouts of their parameter structs."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import build as svbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                            # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    svbuild.build()
    return sv.load()


class FakePool(C.Structure):
    """The head of a registered pool as the library holds it (tests make one where no driver can build tensor maps)."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int64), ("page_size", C.c_int32), ("hkv", C.c_int32), ("head_dim", C.c_int32),
                ("strides", C.c_int64 * 4), ("has_maps", C.c_bool), ("pad", C.c_uint8 * 512)]


def pool(head_dim=128, hkv=2, page_size=16):
    return FakePool(P, P, 100, page_size, hkv, head_dim, (C.c_int64 * 4)(hkv * 16 * head_dim, 16 * head_dim, head_dim, 1), True)


def made(cls, base, **change):
    p = cls()
    for k, v in {**base, **change}.items():
        setattr(p, k, v)
    return p


def attn(pl, **change):
    return made(sv.AttnParams, dict(q=P, o=P, pool=C.addressof(pl), block_table=P, block_table_stride=10, seq_len=P, gamma=P, cu_q=P, batch=3, gamma_max=4,
                                    hq=8, hkv=2, head_dim=128, max_seq_len=160, sm_scale=0.1), **change)


def test_bounds(lib):
    pl = pool()
    base = dict(pool=C.addressof(pl), bounds=P, scales=P, block_table=P, block_table_stride=10, seq_len=P, gamma=P, batch=3, max_new=5)
    call = lambda **kw: lib.spec_page_bounds_update(C.byref(made(sv.PageBoundsParams, base, **kw)), None)  # noqa: E731
    assert lib.spec_page_bounds_update(None, None) == sv.SV_EINVAL
    for name in ("pool", "bounds", "scales", "block_table", "seq_len", "gamma"):
        assert call(**{name: None}) == sv.SV_EINVAL, name
    assert call(first=P) == sv.SV_EINVAL                                  # gamma and first
    for name in ("batch", "max_new", "block_table_stride"):
        assert call(**{name: 0}) == sv.SV_EINVAL, name
    assert call(bounds=P + 8) == sv.SV_EALIGN and call(scales=P + 2) == sv.SV_EALIGN
    other = pool(head_dim=96)
    assert call(pool=C.addressof(other)) == sv.SV_EUNSUPPORTED


def test_select(lib):
    base = dict(q=P, bounds=P, scales=P, n_pages=100, block_table=P, block_table_stride=10, seq_len=P, gamma=P, cu_q=P, batch=3, gamma_max=4, hq=8, hkv=2,
                head_dim=128, max_seq_len=160, n_select=4, n_first=1, n_last=2, page_list=P, row_mask=P, n_list=P, list_stride=10)
    size = lib.spec_page_select_workspace_bytes(3, 4, 2, 160)
    assert size > 0 and [lib.spec_page_select_workspace_bytes(*a) for a in ((0, 4, 2, 160), (3, -1, 2, 160), (3, 64, 2, 160), (3, 4, 0, 160), (3, 4, 2, 0))] == [0] * 5
    call = lambda ws=P, n=size, **kw: lib.spec_page_select(C.byref(made(sv.PageSelectParams, base, **kw)), ws, n, None)  # noqa: E731
    assert lib.spec_page_select(None, P, size, None) == sv.SV_EINVAL
    for name in ("q", "bounds", "scales", "block_table", "seq_len", "gamma", "cu_q", "page_list", "row_mask", "n_list"):
        assert call(**{name: None}) == sv.SV_EINVAL, name
    for change in (dict(batch=0), dict(gamma_max=-1), dict(n_pages=0), dict(max_seq_len=0), dict(n_last=0), dict(n_first=-1), dict(n_select=2), dict(n_first=3),
                   dict(block_table_stride=9), dict(list_stride=9), dict(hq=0)):
        assert call(**change) == sv.SV_EINVAL, change
    for change in (dict(hq=7), dict(hq=516), dict(gamma_max=64), dict(head_dim=96)):
        assert call(**change) == sv.SV_EUNSUPPORTED, change
    for change in (dict(q=P + 8), dict(bounds=P + 4), dict(row_mask=P + 4), dict(ws=P + 8)):
        assert call(**change) == sv.SV_EALIGN, change
    assert call(ws=None) == sv.SV_EWORKSPACE and call(n=size - 1) == sv.SV_EWORKSPACE


def attention_refusals(call, pl):
    for name in ("q", "o", "pool", "block_table", "seq_len", "gamma", "cu_q"):
        assert call(attn=attn(pl, **{name: None})) == sv.SV_EINVAL, name
    for change in (dict(batch=0), dict(gamma_max=-1), dict(max_seq_len=0), dict(block_table_stride=9), dict(hkv=4), dict(sm_scale=0.0), dict(sm_scale=float("nan"))):
        assert call(attn=attn(pl, **change)) == sv.SV_EINVAL, change
    assert call(attn=attn(pl, hq=7)) == sv.SV_EUNSUPPORTED and call(attn=attn(pl, hq=258)) == sv.SV_EUNSUPPORTED
    assert call(attn=attn(pl, q=P + 8)) == sv.SV_EALIGN and call(ws=P + 8) == sv.SV_EALIGN
    small = pool(head_dim=96)
    assert call(attn=attn(small, head_dim=96)) == sv.SV_EUNSUPPORTED


def test_listed_pages(lib):
    pl = pool()
    size = lib.spec_verify_attn_pages_workspace_bytes(3, 4, 8, 2, 128)
    assert size > 0 and [lib.spec_verify_attn_pages_workspace_bytes(*a) for a in ((0, 4, 8, 2, 128), (3, 64, 8, 2, 128), (3, 4, 7, 2, 128), (3, 4, 8, 2, 96))] == [0] * 4
    base = dict(attn=attn(pl), page_list=P, row_mask=P, n_list=P, list_stride=10)
    call = lambda ws=P, n=size, **kw: lib.spec_verify_attn_pages(C.byref(made(sv.AttnPagesParams, base, **kw)), ws, n, None)  # noqa: E731
    assert lib.spec_verify_attn_pages(None, P, size, None) == sv.SV_EINVAL
    attention_refusals(call, pl)
    for change in (dict(page_list=None), dict(row_mask=None), dict(n_list=None), dict(list_stride=0)):
        assert call(**change) == sv.SV_EINVAL, change
    assert call(attn=attn(pl, gamma_max=64)) == sv.SV_EUNSUPPORTED
    assert call(row_mask=P + 4) == sv.SV_EALIGN
    assert call(ws=None) == sv.SV_EWORKSPACE and call(n=size - 1) == sv.SV_EWORKSPACE


def test_shared_prefixes(lib):
    pl = pool()
    size = lib.spec_verify_attn_prefix_workspace_bytes(3, 4, 8, 2, 128, 2)
    assert size > 0 and [lib.spec_verify_attn_prefix_workspace_bytes(*a) for a in ((0, 4, 8, 2, 128, 1), (8193, 4, 8, 2, 128, 1), (3, 4, 8, 2, 128, 4),
                                                                                  (3, 4, 8, 2, 128, 0), (3, 4, 8, 2, 96, 1))] == [0] * 5
    base = dict(attn=attn(pl), group=P, prefix_len=P, n_groups=2)
    call = lambda ws=P, n=size, **kw: lib.spec_verify_attn_prefix(C.byref(made(sv.AttnPrefixParams, base, **kw)), ws, n, None)  # noqa: E731
    assert lib.spec_verify_attn_prefix(None, P, size, None) == sv.SV_EINVAL
    attention_refusals(call, pl)
    for change in (dict(group=None), dict(prefix_len=None), dict(n_groups=0), dict(n_groups=4)):
        assert call(**change) == sv.SV_EINVAL, change
    assert call(attn=attn(pl, batch=8193)) == sv.SV_EUNSUPPORTED
    assert call(ws=None) == sv.SV_EWORKSPACE and call(n=size - 1) == sv.SV_EWORKSPACE


def test_more_tiles_than_31_bits_number(lib):
    """64 tokens a tile: 2^31 - 1 of them over all pairs (of up to 256 rows of a sequence and kv head)."""
    pl = pool(hkv=1)
    last = 2 ** 31 - 1
    big = dict(batch=64, hq=128, hkv=1, max_seq_len=last, block_table_stride=(last + 15) // 16)
    size = lib.spec_verify_attn_prefix_workspace_bytes(64, 4, 128, 1, 128, 2)
    args = dict(group=P, prefix_len=P, n_groups=2)
    assert lib.spec_verify_attn_prefix(C.byref(made(sv.AttnPrefixParams, dict(attn=attn(pl, **big), **args))), P, size, None) == sv.SV_EUNSUPPORTED
    lists = dict(page_list=P, row_mask=P, n_list=P, list_stride=1 << 26)
    size = lib.spec_verify_attn_pages_workspace_bytes(128, 4, 128, 1, 128)
    assert lib.spec_verify_attn_pages(C.byref(made(sv.AttnPagesParams, dict(attn=attn(pl, **{**big, "batch": 128}), **lists))), P, size, None) == sv.SV_EUNSUPPORTED


def test_parameter_structs_are_laid_out_as_the_header_has_them(tmp_path):
    classes = {"sv_page_bounds_params": sv.PageBoundsParams, "sv_page_select_params": sv.PageSelectParams, "sv_attn_pages_params": sv.AttnPagesParams,
               "sv_attn_prefix_params": sv.AttnPrefixParams}
    lines = []
    for name, cls in classes.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "specverify.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True).stdout.split()]
    want = []
    for cls in classes.values():
        want.append(C.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_packed_arguments_fill_the_structs():
    """The packers of the binding write what the ctypes structures hold (nested structs and padding too)."""
    values = iter(range(1, 1000))

    def fill(cls):
        s, flat = cls(), []
        for name, ty in cls._fields_:
            if issubclass(ty, C.Structure):
                inner, more = fill(ty)
                setattr(s, name, inner)
                flat += more
            else:
                v = next(values)
                setattr(s, name, v)
                flat.append(v)
        return s, flat

    for cls, pack in ((sv.PageBoundsParams, sv._pack_page_bounds), (sv.PageSelectParams, sv._pack_page_select), (sv.AttnPagesParams, sv._pack_attn_pages),
                      (sv.AttnPrefixParams, sv._pack_attn_prefix)):
        s, flat = fill(cls)
        packed = pack(*flat)
        assert len(packed) == C.sizeof(cls) and packed == bytes(s), cls.__name__
