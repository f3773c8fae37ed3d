"""What the token-scoring entry points refuse, before anything is enqueued: statuses of the C ABI and errors of the
binding (no compute call is made here), and the layout of their structs."""
import ctypes as C
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = ("adwin_opd_quant_rows", "adwin_opd_quant_logits", "adwin_opd_quant_logits_workspace_bytes", "adwin_opd_token_logp",
         "adwin_opd_token_logp_workspace_bytes", "adwin_opd_token_logp_grad")
PTR = 4096          # never dereferenced on the paths below


@pytest.fixture(scope="module")
def B():
    from paper_2605_28396_amd import binding
    return binding


def test_header_library_and_binding_agree(B):
    header = open(os.path.join(ROOT, "include", "adwin_opd.h")).read()
    for name in CALLS:
        assert re.search(r"\bint %s\(" % name, header) and hasattr(B.lib, name) and hasattr(B, name), name
    for struct in ("adwin_opd_quant_problem", "adwin_opd_quant_logits_problem", "adwin_opd_logp_problem",
                   "adwin_opd_logp_grad_problem"):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), header, re.S).group(1)
        names = []
        for decl in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
            names += [re.findall(r"(\w+)\s*$", x)[0] for x in decl.split(",") if x.strip()]
        assert names == [f[0] for f in getattr(B, struct)._fields_], struct
    assert [int(re.search(r"#define %s +(\d+)" % k, header).group(1)) for k in (
        "ADWIN_QUANT_MAX_H", "ADWIN_MAX_GIVEN", "ADWIN_MAX_TOP")] == [B.ADWIN_QUANT_MAX_H, B.ADWIN_MAX_GIVEN, B.ADWIN_MAX_TOP]
    assert [B.ADWIN_QUANT_PITCH(H) for H in (1, 128, 129, 4096)] == [128, 128, 256, 4096]


def _struct(cls, base, over):
    p = cls()
    p.struct_bytes = C.sizeof(cls)
    for k, v in {**base, **over}.items():
        setattr(p, k, v)
    return p


def test_quant_rows_refusals(B):
    base = dict(N=5, ld_x=64, H=64, x_dtype=0, x=PTR, q=PTR, scale=PTR)

    def st(**over):
        return B.lib.adwin_opd_quant_rows(C.byref(_struct(B.adwin_opd_quant_problem, base, over)), None)
    assert B.lib.adwin_opd_quant_rows(None, None) == B.ADWIN_E_NULL
    assert st(struct_bytes=8) == B.ADWIN_E_MODE and st(x_dtype=2) == B.ADWIN_E_MODE
    for over in (dict(H=0), dict(H=B.ADWIN_QUANT_MAX_H + 1, ld_x=1 << 20), dict(N=-1), dict(N=1 << 24), dict(N=1 << 31), dict(ld_x=63)):
        assert st(**over) == B.ADWIN_E_SHAPE, over
    for over in (dict(x=None), dict(q=None), dict(scale=None)):
        assert st(**over) == B.ADWIN_E_NULL, over
    assert st(x=PTR + 1) == B.ADWIN_E_ALIGN and st(q=PTR + 8) == B.ADWIN_E_ALIGN
    assert st(x=PTR + 2, x_dtype=1) == B.ADWIN_E_ALIGN
    assert st(N=0, x=None, q=None, scale=None) == B.ADWIN_OK


def test_quant_logits_refusals(B):
    base = dict(T=5, ld_h=64, ld_z=1000, V=1000, H=64, h_dtype=0, z_dtype=0, h=PTR, W_q=PTR, W_scale=PTR, z=PTR)

    def p(**over):
        return _struct(B.adwin_opd_quant_logits_problem, base, over)

    def st(ws=PTR, ws_bytes=1 << 30, **over):
        return B.lib.adwin_opd_quant_logits(C.byref(p(**over)), ws, ws_bytes, None)
    need = B.adwin_opd_quant_logits_workspace_bytes(p())
    assert need >= 5 * 128 + 5 * 4 and need % 256 == 0
    assert B.lib.adwin_opd_quant_logits(None, PTR, need, None) == B.ADWIN_E_NULL
    assert B.lib.adwin_opd_quant_logits_workspace_bytes(C.byref(p()), None) == B.ADWIN_E_NULL
    assert st(struct_bytes=8) == st(h_dtype=5) == st(z_dtype=-1) == B.ADWIN_E_MODE
    for over in (dict(H=0), dict(V=0), dict(V=(1 << 28) + 1, ld_z=1 << 29), dict(T=-1), dict(T=1 << 24), dict(T=1 << 31), dict(ld_h=63),
                 dict(ld_z=999), dict(H=B.ADWIN_QUANT_MAX_H + 1, ld_h=1 << 20)):
        assert st(**over) == B.ADWIN_E_SHAPE, over
    for name in ("h", "W_q", "W_scale", "z"):
        assert st(**{name: None}) == B.ADWIN_E_NULL, name
    assert st(h=PTR + 1) == st(W_q=PTR + 8) == st(z=PTR + 1) == st(z=PTR + 2, z_dtype=1) == B.ADWIN_E_ALIGN
    assert st(ws=None) == st(ws=PTR + 16) == st(ws_bytes=need - 1) == B.ADWIN_E_WORKSPACE
    assert st(T=0, ws=None, ws_bytes=0, h=None, z=None) == B.ADWIN_OK


def test_token_logp_refusals(B):
    base = dict(T=5, ld_z=1000, V=1000, G=2, top=3, z_dtype=0, temperature=1.0, z=PTR, ids=PTR, logp=PTR, norm=PTR)

    def p(**over):
        return _struct(B.adwin_opd_logp_problem, base, over)

    def st(ws=PTR, ws_bytes=1 << 30, **over):
        return B.lib.adwin_opd_token_logp(C.byref(p(**over)), ws, ws_bytes, None)
    assert B.lib.adwin_opd_token_logp(None, PTR, 0, None) == B.ADWIN_E_NULL
    assert B.lib.adwin_opd_token_logp_workspace_bytes(C.byref(p()), None) == B.ADWIN_E_NULL
    assert st(struct_bytes=8) == st(z_dtype=2) == B.ADWIN_E_MODE
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        assert st(temperature=t) == B.ADWIN_E_MODE, t
    for over in (dict(V=0), dict(V=(1 << 28) + 1, ld_z=1 << 29), dict(T=-1), dict(T=1 << 24), dict(T=1 << 31), dict(ld_z=999), dict(G=-1),
                 dict(G=B.ADWIN_MAX_GIVEN + 1), dict(top=-1), dict(top=B.ADWIN_MAX_TOP + 1)):
        assert st(**over) == B.ADWIN_E_SHAPE, over
    assert st(z=None) == st(ids=None) == B.ADWIN_E_NULL
    assert st(z=PTR + 1) == st(z=PTR + 2, z_dtype=1) == B.ADWIN_E_ALIGN
    assert st(T=0, z=None, ids=None, ws=None, ws_bytes=0) == B.ADWIN_OK
    need = B.adwin_opd_token_logp_workspace_bytes(p(T=1, V=151936, ld_z=151936))
    if need:
        big = dict(T=1, V=151936, ld_z=151936)
        assert st(ws=None, **big) == st(ws=PTR + 16, **big) == st(ws_bytes=need - 1, **big) == B.ADWIN_E_WORKSPACE


def test_token_logp_grad_refusals(B):
    base = dict(T=5, ld_z=1000, ld_dz=1000, V=1000, G=2, z_dtype=0, dz_dtype=0, temperature=1.0, z=PTR, ids=PTR, norm=PTR,
                g_logp=PTR, entropy=PTR, g_entropy=PTR, dz=PTR)

    def st(**over):
        return B.lib.adwin_opd_token_logp_grad(C.byref(_struct(B.adwin_opd_logp_grad_problem, base, over)), None)
    assert B.lib.adwin_opd_token_logp_grad(None, None) == B.ADWIN_E_NULL
    assert st(struct_bytes=8) == st(z_dtype=2) == st(dz_dtype=2) == st(temperature=0.0) == B.ADWIN_E_MODE
    for over in (dict(V=0), dict(T=-1), dict(T=1 << 24), dict(ld_z=999), dict(ld_dz=999), dict(G=-1), dict(G=B.ADWIN_MAX_GIVEN + 1)):
        assert st(**over) == B.ADWIN_E_SHAPE, over
    for name in ("z", "ids", "norm", "g_logp", "entropy", "dz"):
        assert st(**{name: None}) == B.ADWIN_E_NULL, name
    assert st(z=PTR + 1) == st(dz=PTR + 1) == st(dz=PTR + 2, dz_dtype=1) == B.ADWIN_E_ALIGN
    assert st(T=0, z=None, dz=None, norm=None) == B.ADWIN_OK


def test_binding_refuses_what_the_library_could_not_read(B):
    """Host memory, other types, other strides and other sizes: an error before the library is called."""
    z, ids, f = torch.zeros(4, 10), torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4)
    for bad in (z, z.half(), z.t(), z[0], z[:, ::2]):
        with pytest.raises(ValueError):
            B.adwin_opd_token_logp(bad, ids)
        with pytest.raises(ValueError):
            B.adwin_opd_quant_rows(bad)
        with pytest.raises(ValueError):
            B.adwin_opd_quant_logits(bad, torch.zeros(7, 128, dtype=torch.int8), torch.zeros(7))
        with pytest.raises(ValueError):
            B.adwin_opd_token_logp_grad(bad, ids, torch.zeros(4, 2), f)
