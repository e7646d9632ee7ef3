"""Refusals of the calls on rows, paged caches and logits: error codes of the C calls and the binding's checks, on the host."""
import ctypes as C
import re

import pytest
import torch

import paper_2409_16560_amd as dsbd
import paper_2409_16560_amd.binding as b

P = 1 << 20          # a pointer that nothing reads: every call here is refused, or has nothing to do


def rows(ptr=P, ts=1024, hs=128):
    return C.byref(b._Rows(ptr, ts, hs))


def prep(**kw):
    f = dict(q_weight=None, k_weight=None, inv_freq=P, eps=1e-6, rot_scale=1.0, rot_dim=128, norm=1, per_head=0, interleaved=0)
    f.update(kw)
    return C.byref(b._QKPrep(*[f[n] for n, _ in b._QKPrep._fields_]))


def cache(**kw):
    f = dict(k_pages=P, v_pages=P, page_table=P, ctx_len=P, q_off=P, page_stride=16384, token_stride=1024, head_stride=128, n_pages=10,
             page_size=16, table_stride=4, n_seqs=2, max_new=1, max_len=64)
    f.update(kw)
    return C.byref(b._PagedKV(*[f[n] for n, _ in b._PagedKV._fields_]))


def test_structs_match_the_header():
    import os
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dsbd.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    for cname, cls in (("dsbd_rows", b._Rows), ("dsbd_qk_prep", b._QKPrep), ("dsbd_paged_kv", b._PagedKV), ("dsbd_logit_rules", b._LogitRules)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cname, cname), src, flags=re.S).group(1)
        fields = []
        for decl in filter(None, (d.strip() for d in body.split(";"))):
            fields += [re.findall(r"([A-Za-z_][A-Za-z_0-9]*)\s*$", n.strip())[0] for n in decl.split(",")]
        assert fields == [n for n, _ in cls._fields_], cname


@pytest.mark.parametrize("code,kw", [
    (-2, dict(D=100)), (-2, dict(D=272)), (-2, dict(D=0)), (-2, dict(dtype=2)), (-2, dict(dtype=-1)), (-1, dict(n=-1)), (-1, dict(Hq=0)),
    (-1, dict(Hkv=0)), (-2, dict(q=rows(ts=1020))), (-1, dict(q=rows(ptr=P + 8))), (-1, dict(q=rows(ts=-1024))), (-1, dict(q_out=None)),
    (-1, dict(q=None)), (-1, dict(positions=None)), (-1, dict(prep=prep(rot_dim=256))), (-2, dict(prep=prep(rot_dim=24))),
    (-1, dict(prep=prep(inv_freq=None))), (-1, dict(prep=prep(eps=-1.0))), (-1, dict(prep=prep(eps=float("nan")))),
    (-1, dict(prep=prep(q_weight=P + 2))), (-2, dict(Hq=70000)), (0, dict(n=0)), (0, dict(n=0, positions=None))])
def test_rows(code, kw):
    a = dict(n=4, Hq=8, Hkv=2, D=128, dtype=0, q=rows(), k=rows(), v=rows(), positions=P, prep=prep(), q_out=rows(), k_out=rows(), v_out=rows())
    a.update(kw)
    assert b.load_library().dsbd_qk_norm_rope(a["n"], a["Hq"], a["Hkv"], a["D"], a["dtype"], a["q"], a["k"], a["v"], a["positions"],
                                              a["prep"], a["q_out"], a["k_out"], a["v_out"], None) == code


CACHES = [(-1, dict(page_size=0)), (-1, dict(n_pages=-1)), (-1, dict(n_seqs=-1)), (-1, dict(max_new=-1)), (-1, dict(max_len=-1)),
          (-1, dict(table_stride=-1)), (-2, dict(page_stride=16380)), (-2, dict(token_stride=12)), (-1, dict(head_stride=-128)),
          (-1, dict(k_pages=None)), (-1, dict(v_pages=P + 8)), (-1, dict(page_table=None)), (-1, dict(ctx_len=None)), (-1, dict(q_off=None)),
          (-2, dict(max_len=(1 << 30) + 1)), (0, dict(n_seqs=0))]


@pytest.mark.parametrize("code,kw", CACHES + [(-1, "k"), (-1, "fault"), (-1, "cache"), (-1, "q_out"), (-2, "D"), (-1, "n"), (0, "none")])
def test_append(code, kw):
    c = cache(**kw) if isinstance(kw, dict) else cache()
    lib = b.load_library()
    got = lib.dsbd_paged_append(None if kw == "cache" else c, -1 if kw == "n" else 0 if kw == "none" else 2, 8, 2, 96 + 8 if kw == "D" else 128, 0,
                                rows(), None if kw == "k" else rows(), rows(), None, prep(), None if kw == "q_out" else rows(),
                                None if kw == "fault" else P, None)
    assert got == code


@pytest.mark.parametrize("code,kw", CACHES + [(-1, "q"), (-1, "out"), (-1, "fault"), (-1, "cache"), (-1, "ws"), (-3, "small"), (-2, "D"), (-2, "dtype"),
                                              (-1, "heads"), (-2, "anc"), (0, "none")])
def test_attention(code, kw):
    c = cache(**kw) if isinstance(kw, dict) else cache(max_new=65) if kw == "anc" else cache()
    lib = b.load_library()
    n, Hq, D = 0 if kw == "none" else 2, 7 if kw == "heads" else 8, 96 if kw == "D" else 128
    need = lib.dsbd_paged_attention_workspace_bytes(c, n, Hq, 2, D)
    assert (need > 0) == (not isinstance(kw, str) or kw not in ("heads", "D")) or isinstance(kw, dict)
    got = lib.dsbd_paged_attention(None if kw == "cache" else c, n, Hq, 2, D, 2 if kw == "dtype" else 0, None if kw == "q" else rows(), 0.0,
                                   P if kw == "anc" else None, None if kw == "out" else rows(), None, None if kw == "ws" else P,
                                   need - 1 if kw == "small" else need, None if kw == "fault" else P, None)
    assert got == code


def test_workspace_goes_by_the_arguments_alone():
    lib = b.load_library()
    for Hq, Hkv, D in ((8, 2, 128), (4, 4, 64), (28, 4, 128)):
        for n, s in ((1, 1), (7, 3), (64, 64), (300, 2), (8000, 1), (100000, 200)):
            need = lib.dsbd_paged_attention_workspace_bytes(cache(n_seqs=s, max_new=n), n, Hq, Hkv, D)
            assert 256 <= need <= 1 << 28 and need % 256 == 0
            assert need == lib.dsbd_paged_attention_workspace_bytes(cache(n_seqs=s, max_new=n, max_len=9999, k_pages=None), n, Hq, Hkv, D)


def forest(**kw):
    f = dict(n_prompts=1, n_trees=1, n_nodes=3, tree_prompt=P, tree_off=P, parent=P, token=P, draft_rank=None, max_tree_nodes=3, max_depth=2,
             max_prompt_trees=1)
    f.update(kw)
    return C.byref(b._Forest(*[f[n] for n, _ in b._Forest._fields_]))


def rules(**kw):
    f = {n: None for n, _ in b._LogitRules._fields_[:12]}
    f.update(mask_stride=0, n_masks=0, n_hist=0, n_bias=0)
    f.update(kw)
    return C.byref(b._LogitRules(*[f[n] for n, _ in b._LogitRules._fields_]))


@pytest.mark.parametrize("code,kw", [
    (-1, dict(forest=None)), (-1, dict(rules=None)), (-1, dict(fault=None)), (-1, dict(n=-1)), (-2, dict(V=0)), (-2, dict(V=(1 << 30) + 1)),
    (-2, dict(dtype=3)), (-1, dict(stride=99)), (-1, dict(out_stride=99)), (-2, dict(forest=forest(max_tree_nodes=65))), (-1, dict(n=2)),
    (0, dict(n=0, row_node=P)), (-1, dict(logits=None)), (-1, dict(out=None)), (-1, dict(forest=forest(token=None))),
    (-1, dict(rules=rules(hist_off=P, n_hist=5))), (-1, dict(rules=rules(bias_off=P, n_bias=2))), (-1, dict(rules=rules(mask=P, mask_stride=3))),
    (-1, dict(rules=rules(n_masks=-1))), (-1, dict(logits=P + 2)), (-1, dict(dtype=0, logits=P + 64, out=P + 64)),
    (-1, dict(logits=P + 64, out=P + 64, stride=104))])
def test_logits(code, kw):
    a = dict(forest=forest(), row_node=None, n=3, V=100, dtype=2, logits=P, stride=100, rules=rules(), out=P + 65536, out_stride=100, fault=P)
    a.update(kw)
    assert b.load_library().dsbd_process_logits(a["forest"], a["row_node"], a["n"], a["V"], a["dtype"], a["logits"], a["stride"], a["rules"],
                                                a["out"], a["out_stride"], a["fault"], None) == code


# ------------------------------------------------------------------------------------------------ the binding's own checks

def cpu_cache(dtype=torch.bfloat16, **kw):
    a = dict(k_pages=torch.zeros(4, 16, 2, 64, dtype=dtype), v_pages=torch.zeros(4, 16, 2, 64, dtype=dtype), page_table=[[0, 1]], ctx_len=[3],
             q_off=[0, 2])
    a.update(kw)
    return dsbd.PagedKV(a["k_pages"], a["v_pages"], a["page_table"], a["ctx_len"], a["q_off"], max_new=2, max_len=32)


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_rows():
    pos, pr = torch.zeros(3, dtype=torch.int32), dsbd.QKPrep(inv_freq=torch.ones(32, dtype=torch.float64))
    call = dsbd.dsbd_qk_norm_rope
    with pytest.raises(ValueError, match="GPU"):
        call(z(3, 4, 64), z(3, 2, 64), pos, pr)
    bad = [(z(3, 4, 64), z(3, 2, 64), pos[:2], pr), (z(3, 4, 64), z(3, 2, 64), pos.long(), pr), (z(3, 4, 64), z(2, 2, 64), pos, pr),
           (z(3, 4, 64), z(3, 2, 64, dtype=torch.float16), pos, pr), (z(3, 4, 64).transpose(1, 2), None, pos, pr),
           (z(3, 4, 64), None, pos, dsbd.QKPrep(inv_freq=torch.ones(33, dtype=torch.float64))),
           (z(3, 4, 64), None, pos, dsbd.QKPrep(inv_freq=torch.ones(32))),
           (z(3, 4, 64), None, pos, dsbd.QKPrep(norm=True, q_weight=z(32))), (z(3, 4, 64), None, pos, dsbd.QKPrep(norm=True, q_weight=z(5, 64))),
           (z(3, 4, 64), None, pos, dsbd.QKPrep(norm=True, q_weight=torch.ones(64))),
           (z(3, 4, 64), z(3, 2, 64), pos, dsbd.QKPrep(norm=True, q_weight=z(64), k_weight=z(2, 64)))]
    for args in bad:
        with pytest.raises(AssertionError):
            call(*args)
    with pytest.raises(AssertionError):
        call(z(3, 4, 64), None, pos, pr, q_out=z(3, 1, 64).expand(3, 4, 64))       # rows on top of each other
    with pytest.raises(AssertionError):
        call(z(3, 4, 64), None, pos, pr, k_out=z(3, 2, 64))
    with pytest.raises(StopIteration):
        call(None, None, pos, pr)


def test_binding_cache():
    ap, at, k, q = dsbd.dsbd_paged_append, dsbd.dsbd_paged_attention, z(2, 2, 64), z(2, 4, 64)
    with pytest.raises(ValueError, match="GPU"):
        ap(cpu_cache(), k, k, q=q)
    with pytest.raises(ValueError, match="GPU"):
        at(cpu_cache(), q)
    for c in (cpu_cache(page_table=[[0, 1], [0, 1]]), cpu_cache(q_off=[0, 1, 2]), cpu_cache(v_pages=z(4, 16, 2, 32)),
              cpu_cache(v_pages=z(4, 2, 16, 64).transpose(1, 2)), cpu_cache(v_pages=z(4, 16, 2, 64, dtype=torch.float16)),
              cpu_cache(dtype=torch.float16)):
        with pytest.raises(AssertionError):
            ap(c, k, k)
        with pytest.raises(AssertionError):
            at(c, q)
    for args in ((cpu_cache(), z(2, 3, 64), z(2, 3, 64)), (cpu_cache(), k, z(3, 2, 64)), (cpu_cache(), z(2, 2, 32), z(2, 2, 32))):
        with pytest.raises(AssertionError):
            ap(*args)
    with pytest.raises(AssertionError):
        ap(cpu_cache(), k, k, positions=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(AssertionError):
        ap(cpu_cache(), k, k, q_out=q)
    for kw in (dict(anc_mask=torch.zeros(2, dtype=torch.int32)), dict(anc_mask=torch.zeros(3, dtype=torch.int64)), dict(out=z(2, 4, 32)),
               dict(lse=torch.zeros(2, 3)), dict(lse=z(2, 4)), dict(out=z(2, 4, 64, dtype=torch.float16))):
        with pytest.raises(AssertionError):
            at(cpu_cache(), q, **kw)
    with pytest.raises(dsbd.DsbdError):
        at(cpu_cache(), z(2, 3, 64))                 # three query heads on two
    assert dsbd.dsbd_paged_attention_workspace_bytes(cpu_cache(), 2, 4) > 0


def test_binding_logits():
    f = dsbd.Forest([0], [0, 3], [-1, 0, 0], [5, 6, 7], n_prompts=1, max_tree_nodes=3, max_depth=1, max_prompt_trees=1, device=torch.device("cpu"))
    call, logits, i32 = dsbd.dsbd_process_logits, torch.zeros(3, 40), lambda *a: torch.tensor(a, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        call(f, logits, dsbd.LogitRules())
    one = torch.ones(1)
    for r in (dict(hist=i32(1, 2)), dict(hist=i32(1), hist_off=i32(0, 1, 1)), dict(prompt_len=i32(1, 1)), dict(repetition=torch.ones(2)),
              dict(repetition=one.double()), dict(bias_off=i32(0, 1), bias_token=i32(4)), dict(bias_off=i32(0, 1), bias_token=i32(4), bias_value=torch.ones(2)),
              dict(bias_token=i32(4), bias_value=one), dict(mask=torch.zeros(3, 1, dtype=torch.int32)), dict(mask=torch.zeros(2, 2, dtype=torch.int32)),
              dict(mask=torch.zeros(3, 2, dtype=torch.int64)), dict(mask=torch.zeros(2, 2, dtype=torch.int32), mask_row=i32(0, 1))):
        with pytest.raises(AssertionError):
            call(f, logits, dsbd.LogitRules(**r))
    for args, kw in (((f, torch.zeros(2, 40), dsbd.LogitRules()), {}), ((f, logits.double(), dsbd.LogitRules()), {}),
                     ((f, logits, dsbd.LogitRules()), dict(row_node=i32(0))), ((f, logits, dsbd.LogitRules()), dict(out=torch.zeros(3, 39))),
                     ((f, logits, dsbd.LogitRules()), dict(out=torch.zeros(3, 40).bfloat16())),
                     ((f, logits, dsbd.LogitRules()), dict(out=torch.zeros(1, 40).expand(3, 40)))):
        with pytest.raises(AssertionError):
            call(*args, **kw)
    f.token = None
    with pytest.raises(ValueError, match="tokens"):
        call(f, logits, dsbd.LogitRules())


def test_frequencies():
    import math
    f, s = dsbd.rope_inv_freq(64, 10000.0, device="cpu")
    assert s == 1.0 and f.dtype == torch.float64
    want = torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    assert torch.allclose(f, want, rtol=1e-14)
    assert torch.allclose(dsbd.rope_inv_freq(64, 10000.0, "linear", 8.0, device="cpu")[0], want / 8, rtol=1e-14)
    g = dsbd.rope_inv_freq(64, 10000.0, "base", 8.0, device="cpu")[0]
    assert float(g[0]) == 1.0 and abs(float(g[-1] * 8 / want[-1]) - 1) < 1e-12
    for kind in ("by_parts", "by_turns"):
        g, s = dsbd.rope_inv_freq(64, 10000.0, kind, 8.0, orig_len=4096, low=1.0, high=32.0, device="cpu")
        turns = 4096 * want / (2 * math.pi)
        ratio = g / want
        assert bool((ratio[turns >= 40] == 1).all()) and bool((ratio[turns < 0.7] - 1 / 8).abs().max() < 1e-12)
        assert bool((ratio[1:] <= ratio[:-1] + 1e-12).all())
        assert abs(s - (0.1 * math.log(8.0) + 1 if kind == "by_parts" else 1.0)) < 1e-12
        assert torch.allclose(dsbd.rope_inv_freq(64, 10000.0, kind, 1.0, orig_len=4096, device="cpu")[0], want, rtol=1e-14)
    for bad in (dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.0), dict(rot_dim=64, scaling="other"),
                dict(rot_dim=64, scaling="by_parts", factor=2.0), dict(rot_dim=2, scaling="base", factor=2.0)):
        with pytest.raises(ValueError):
            dsbd.rope_inv_freq(device="cpu", **bad)
