"""Refusals of the operators of a step over drafted tokens: on the host, before anything touches a device (addresses here are never read)."""
import ctypes as C

import pytest

import paper_2410_12513_amd as P
from paper_2410_12513_amd import binding as B

BIG = 1 << 40                 # room enough, were it read
A16 = 1 << 20                 # an address on 16 bytes


@pytest.fixture(scope="module")
def lib():
    return P.load_library()


def _refused(lib, rc, code, word):
    assert rc == code and word in lib.first_last_error(None).decode(), (rc, lib.first_last_error(None))


LORA = dict(stream=None, dtype=1, A=A16, W=A16, La=A16, Lb=A16, adapter=A16, scale=A16, C=A16, m=4, n=4, k=8, ads=1, r=8, acc=0, ws=A16, size=BIG)


@pytest.mark.parametrize("change,code,word", [
    ({"dtype": 2}, -1, "dtype"), ({"m": -1}, -1, "negative"), ({"n": 0}, -1, "n < 1"), ({"k": 12}, -1, "multiple of 8"), ({"k": 0}, -1, "multiple of 8"), ({"r": 0}, -1, "rank"),
    ({"r": 65}, -1, "rank"), ({"ads": 0}, -1, "adapters"), ({"A": 0}, -1, "null"), ({"C": 0}, -1, "null"), ({"ws": 0}, -1, "null"), ({"W": A16 + 2}, -1, "16 bytes"),
    ({"Lb": A16 + 8}, -1, "16 bytes"), ({"C": A16 + 2}, -1, "on 4"), ({"size": 0}, -3, "workspace"), ({"m": (1 << 20) + 1}, -3, "rows")])
def test_lora(lib, change, code, word):
    _refused(lib, lib.first_op_gemm_nt_lora(*{**LORA, **change}.values()), code, word)


def test_lora_workspace(lib):
    assert lib.first_op_gemm_nt_lora_workspace(1, 16, 64, 64, 8) > 0
    assert lib.first_op_gemm_nt_lora_workspace(1, 16, 64, 64, 65) == -1


ROPE_DESC = dict(dtype=1, n_heads=4, head_dim=64, rot_dim=64, layout=0, scaling=2, inverse=0, original_len=8192, base=1e4, factor=8.0, low=1.0, high=4.0, amplitude=1.0)


@pytest.mark.parametrize("change,word", [
    ({"dtype": 3}, "dtype"), ({"n_heads": 0}, "heads"), ({"head_dim": 258}, "head_dim"), ({"rot_dim": 63}, "rot_dim"), ({"rot_dim": 66}, "rot_dim"), ({"rot_dim": 0}, "rot_dim"),
    ({"layout": 2}, "layout"), ({"scaling": 3}, "scaling"), ({"base": 0.0}, "base"), ({"base": float("nan")}, "base"), ({"factor": 0.0}, "factor"), ({"factor": float("inf")}, "factor"),
    ({"low": 4.0}, "low"), ({"original_len": 0}, "original_len"), ({"amplitude": float("nan")}, "finite")])
def test_rope_description(lib, change, word):
    d = B._RopeDesc(**{**ROPE_DESC, **change})
    _refused(lib, lib.first_op_rope(None, C.byref(d), A16, 256, BIG, 256, A16, 4), -1, word)


@pytest.mark.parametrize("args,word", [
    ((0, 256, BIG, 256, A16, 4), "null"), ((A16, 255, BIG, 256, A16, 4), "pitch"), ((A16, 256, BIG, 255, A16, 4), "pitch"), ((A16, 1 << 31, BIG, 256, A16, 4), "pitch"),
    ((A16, 256, BIG, 256, A16, -1), "negative"), ((A16 + 1, 256, BIG, 256, A16, 4), "element"), ((A16, 256, A16 + 2, 256, A16, 4), "overlap"),
    ((A16, 512, A16, 256, A16, 4), "overlap"), ((A16, 512, A16 + 512 - 2, 512, A16, 4), "overlap")])
def test_rope_arguments(lib, args, word):
    d = B._RopeDesc(**ROPE_DESC)
    _refused(lib, lib.first_op_rope(None, C.byref(d), *args), -1, word)
    assert lib.first_op_rope(None, None, A16, 256, BIG, 256, A16, 4) == -1


TREE_DESC = dict(dtype=1, n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, max_pages=4, mask_words=1, scale=0.125)
TREE = dict(q=A16, k=A16, v=A16, pool=A16, table=A16, lens=A16, offs=A16, mask=A16, out=A16, lse=A16, B=2, N=4, nodes=4, length=64, ws=A16, size=BIG)


@pytest.mark.parametrize("change,code,word", [
    ({"dtype": 2}, -1, "dtype"), ({"n_q_heads": 7}, -1, "heads"), ({"n_q_heads": 0}, -1, "heads"), ({"n_kv_heads": 0}, -1, "heads"), ({"n_q_heads": 2048}, -1, "heads"),
    ({"head_dim": 96}, -1, "head_dim"), ({"page_tokens": 32}, -1, "16 tokens"), ({"n_pages": -1}, -1, "negative"), ({"scale": float("inf")}, -1, "scale"), ({"mask_words": 0}, -1, "mask_words"),
    ({"q": 0}, -1, "null"), ({"pool": 0}, -1, "null"), ({"table": 0}, -1, "null"), ({"offs": 0}, -1, "null"), ({"out": 0}, -1, "null"), ({"k": A16 + 8}, -1, "aligned"), ({"mask": A16 + 4}, -1, "aligned"),
    ({"B": -1}, -1, "negative"), ({"N": -1}, -1, "negative"), ({"nodes": -1}, -1, "negative"), ({"length": -1}, -1, "negative"), ({"B": 65536}, -3, "sequences"), ({"nodes": 2049, "mask_words": 64}, -3, "2048"), ({"nodes": 65}, -1, "mask_words")])
def test_tree_attention(lib, change, code, word):
    d = B._TreeAttnDesc(**{**TREE_DESC, **{k: v for k, v in change.items() if k in TREE_DESC}})
    _refused(lib, lib.first_op_tree_attn(None, C.byref(d), *{**TREE, **{k: v for k, v in change.items() if k not in TREE_DESC}}.values()), code, word)


def test_tree_attention_workspace(lib):
    d = B._TreeAttnDesc(**TREE_DESC)
    need = lib.first_op_tree_attn_workspace(C.byref(d), 1, 8, 8, 1 << 20)
    assert need >= 0
    if need > 0:
        args = {**TREE, "B": 1, "N": 8, "nodes": 8, "length": 1 << 20}
        _refused(lib, lib.first_op_tree_attn(None, C.byref(d), *{**args, "size": need - 1}.values()), -3, "workspace")
        _refused(lib, lib.first_op_tree_attn(None, C.byref(d), *{**args, "ws": 0}.values()), -1, "null")
    assert lib.first_op_tree_attn_workspace(None, 1, 8, 8, 64) == -1


SAMPLE = dict(stream=None, logits=A16, pitch=100, rows=3, vocab=100, u=A16, t=A16, k=A16, p=A16, mp=A16, token=A16, lp=A16, kept=A16, ws=A16, size=BIG)


@pytest.mark.parametrize("change,word", [
    ({"logits": 0}, "null"), ({"u": 0}, "null"), ({"token": 0}, "null"), ({"rows": -1}, "rows"), ({"vocab": 0}, "vocab"), ({"pitch": 99}, "pitch"), ({"pitch": 1 << 31}, "pitch"),
    ({"logits": A16 + 2}, "aligned"), ({"kept": A16 + 1}, "aligned"), ({"ws": A16 + 4}, "aligned")])
def test_sample(lib, change, word):
    _refused(lib, lib.first_sample(*{**SAMPLE, **change}.values()), -1, word)


def test_sample_workspace(lib):
    need = lib.first_sample_workspace(1, 128256)
    assert need >= 0 and lib.first_sample_workspace(1, 0) == -1 and lib.first_sample_workspace(-1, 5) == -1
    if need > 0:
        args = {**SAMPLE, "rows": 1, "vocab": 128256, "pitch": 128256}
        _refused(lib, lib.first_sample(*{**args, "size": need - 1}.values()), -3, "workspace")


def test_sizes_beyond_the_limits(lib):
    d = B._TreeAttnDesc(**TREE_DESC)
    assert lib.first_op_tree_attn_workspace(C.byref(d), 2, (1 << 27) + 1, 4, 1 << 20) == -3
    _refused(lib, lib.first_op_tree_attn(None, C.byref(d), *{**TREE, "N": (1 << 27) + 1}.values()), -3, "2^27")
    assert lib.first_sample_workspace(1, (1 << 30) + 1) == -3
    _refused(lib, lib.first_sample(*{**SAMPLE, "vocab": (1 << 30) + 1, "pitch": (1 << 30) + 1}.values()), -3, "2^30")


def test_tree_attention_without_a_context(lib):
    assert lib.first_tree_attn_workspace(None, 4, 4) == -1
    assert lib.first_tree_attn(None, 0, A16, A16, A16, A16, None, 0, A16, None, 4, 4, A16, BIG) == -1


def test_nothing_to_do_is_no_error(lib):
    assert lib.first_op_gemm_nt_lora(*{**LORA, "m": 0, "A": 0, "C": 0, "ws": 0, "size": 0}.values()) == 0
    d = B._RopeDesc(**ROPE_DESC)
    assert lib.first_op_rope(None, C.byref(d), 0, 256, 0, 256, 0, 0) == 0
    t = B._TreeAttnDesc(**TREE_DESC)
    for change in ({"B": 0}, {"N": 0}, {"nodes": 0}):
        assert lib.first_op_tree_attn(None, C.byref(t), *{**TREE, "q": 0, "k": 0, "ws": 0, "size": 0, **change}.values()) == 0
    assert lib.first_sample(*{**SAMPLE, "rows": 0, "logits": 0, "token": 0, "ws": 0, "size": 0}.values()) == 0


def test_the_binding_refuses_what_it_can_see():
    import torch
    cpu = torch.zeros(4, 100)
    with pytest.raises(ValueError):
        P.sample(cpu, torch.zeros(4), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.sample(cpu.double(), torch.zeros(4), torch.zeros(4, dtype=torch.int32))
    x = torch.zeros(2, 3, 64)
    with pytest.raises(ValueError):
        P.op_rope(x, torch.zeros(2, dtype=torch.int32), x, layout="other")
    with pytest.raises(ValueError):
        P.op_rope(x.transpose(0, 1), torch.zeros(3, dtype=torch.int32), x.transpose(0, 1))
    with pytest.raises(ValueError):
        P.op_gemm_nt_lora(torch.zeros(2, 8), torch.zeros(4, 8), torch.zeros(1, 8, 8), torch.zeros(1, 4, 9), torch.zeros(2, dtype=torch.int32), torch.zeros(1), torch.zeros(2, 4))
