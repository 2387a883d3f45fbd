"""What the binding of the long-context calls refuses: tensors that are not what the call reads, before anything is launched."""
import numpy as np
import pytest
import torch

from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev_bf16
from tests.longctx import config

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, GMAX, MOST = 3, 8, 2, 128, 2, 64


def arguments():
    kv = synth.make_kv(config("lb", B, HQ, HKV, D, 160), np.full(B, MOST, np.int32))
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    q = torch.zeros((B * 3, HQ, D), dtype=torch.bfloat16, device=DEV)
    byte = lambda n: torch.zeros(n, dtype=torch.uint8, device=DEV)  # noqa: E731
    return dict(pool=pool, q=q, o=torch.zeros_like(q), lse=torch.zeros(B * 3, HQ, device=DEV), block_table=i32(B, 4), seq_len=i32(B) + 3, gamma=i32(B),
                cu_q=i32(B + 1), gamma_max=GMAX, max_seq_len=MOST, device_status=i32(1),
                bounds=torch.zeros((pool.n_pages, HKV, 2, D), dtype=torch.int8, device=DEV), scales=torch.zeros((pool.n_pages, HKV), device=DEV),
                page_list=i32(B, HKV, 4), row_mask=torch.zeros((B, HKV, 4), dtype=torch.int64, device=DEV), n_list=i32(B, HKV),
                n_select=4, n_first=1, n_last=1, group=i32(B), prefix_len=i32(2), max_new=3,
                select_ws=byte(sv.spec_page_select_workspace_bytes(B, GMAX, HKV, MOST)),
                pages_ws=byte(sv.spec_verify_attn_pages_workspace_bytes(B, GMAX, HQ, HKV, D)),
                prefix_ws=byte(sv.spec_verify_attn_prefix_workspace_bytes(B, GMAX, HQ, HKV, D, 2)))


CALLS = {
    "bounds": (sv.spec_page_bounds_update, "pool bounds scales block_table seq_len gamma max_new device_status", None),
    "select": (sv.spec_page_select, "q bounds scales block_table seq_len gamma cu_q gamma_max max_seq_len n_select n_first n_last page_list row_mask n_list "
                                    "device_status", "select_ws"),
    "pages": (sv.spec_verify_attn_pages, "q o pool block_table seq_len gamma cu_q gamma_max max_seq_len page_list row_mask n_list lse device_status", "pages_ws"),
    "prefix": (sv.spec_verify_attn_prefix, "q o pool block_table seq_len gamma cu_q gamma_max max_seq_len group prefix_len lse device_status", "prefix_ws"),
}


def call(name, a, **change):
    fn, names, ws = CALLS[name]
    kw = {k: a[k] for k in names.split()}
    if ws:
        kw["workspace"] = a[ws]
    fn(**{**kw, **change})


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_of_another_kind(name):
    a = arguments()
    call(name, a)
    before = sv.sv_launch_count()
    for k in CALLS[name][1].split() + (["workspace"] if CALLS[name][2] else []):
        t = a[CALLS[name][2] if k == "workspace" else k]
        if not torch.is_tensor(t):
            continue
        wrong = [t.cpu()]
        if k != "workspace":
            wrong.append(t.double())
        if t.numel() > 1:
            wrong.append(torch.stack((t, t), -1)[..., 0])              # not contiguous
        if t.dim() and k not in ("q", "o", "prefix_len", "seq_len"):
            wrong.append(t[:-1] if k != "device_status" else t[:0].cpu())
        for w in wrong:
            with pytest.raises((ValueError, sv.SpecVerifyError)):
                call(name, a, **{k: w})
    for k in ("q", "o", "page_list", "row_mask", "bounds"):
        if k in CALLS[name][1].split():
            with pytest.raises(ValueError):
                call(name, a, **{k: a[k][0]})                          # a dimension short
    assert sv.sv_launch_count() == before
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["bounds", "pages", "prefix"])
def test_pools(name):
    a = arguments()
    other = sv.spec_kv_pool_register(*(torch.zeros((5, 4, 16, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    before = sv.sv_launch_count()
    with pytest.raises((ValueError, sv.SpecVerifyError)):
        call(name, a, pool=other)
    a["pool"].release()
    with pytest.raises(ValueError):
        call(name, a)
    assert sv.sv_launch_count() == before


@pytest.mark.parametrize("name", ["select", "pages", "prefix"])
def test_workspaces(name):
    a = arguments()
    ws = a[CALLS[name][2]]
    before = sv.sv_launch_count()
    for w in (None, ws[:-1], torch.empty(ws.numel() + 8, dtype=torch.uint8, device=DEV)[8:]):
        with pytest.raises((ValueError, sv.SpecVerifyError)):
            call(name, a, workspace=w)
    assert sv.sv_launch_count() == before
