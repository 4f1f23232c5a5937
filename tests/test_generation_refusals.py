"""What the candidate generator's operators refuse before anything is enqueued: at the C-ABI with made-up
pointers that nothing follows (no GPU), and in the Python calls."""
import math
import os
import subprocess

import pytest

from paper_2603_02565_gb300 import binding as B, build as fe_build
from paper_2603_02565_gb300 import generation as G

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a pointer's value, aligned to anything

APPEND = ["dtype", "n_pages", "page_rows", "kv_heads", "head_dim", "kc", "vc", "n_seqs", "n_rows", "page_cols",
          "q_heads", "rope_rows", "rot_dim", "pairs", "reserved", "row_start", "first", "shift", "pages", "k", "v", "q",
          "k_row", "k_head", "v_row", "v_head", "q_row", "q_head", "q_out", "rope", "status"]
PREFIX = ["dtype", "n_pages", "page_rows", "kv_heads", "head_dim", "kc", "vc", "n_groups", "n_seqs", "n_rows",
          "q_heads", "prefix_cols", "page_cols", "scale", "reserved", "group_start", "prefix_len", "prefix_pages",
          "row_start", "seq_len", "pages", "q", "q_row", "q_head", "out", "lse", "workspace", "workspace_bytes", "status"]
POLICY = ["dtype", "rows", "vocab", "clip_low", "clip_high", "beta", "temperature", "grad_scale", "logits", "logits_row",
          "grad_row", "tokens", "advantages", "weights", "old_logp", "ref_logp", "loss", "terms", "logp", "lse", "coef",
          "grad", "status"]
KV = dict(dtype=B.FE_IO_BF16, n_pages=64, page_rows=64, kv_heads=2, head_dim=64, kc=P, vc=2 * P)
GOOD = {
    "append": dict(KV, n_seqs=3, n_rows=5, page_cols=4, q_heads=4, rope_rows=100, rot_dim=64, pairs=0, reserved=0,
                   row_start=P, first=P, shift=0, pages=P, k=P, v=P, q=P, k_row=512, k_head=64, v_row=512, v_head=64,
                   q_row=512, q_head=64, q_out=3 * P, rope=P, status=0),
    "prefix": dict(KV, n_groups=2, n_seqs=3, n_rows=5, q_heads=4, prefix_cols=4, page_cols=4, scale=0.125, reserved=0,
                   group_start=P, prefix_len=P, prefix_pages=P, row_start=P, seq_len=P, pages=P, q=P, q_row=256, q_head=64,
                   out=3 * P, lse=0, workspace=P, workspace_bytes=0, status=0),
    "policy": dict(dtype=B.FE_IO_BF16, rows=5, vocab=100, clip_low=0.2, clip_high=0.2, beta=0.1, temperature=1.0,
                   grad_scale=1.0, logits=P, logits_row=100, grad_row=100, tokens=P, advantages=P, weights=0, old_logp=0,
                   ref_logp=0, loss=P, terms=P, logp=P, lse=P, coef=P, grad=2 * P, status=0),
}
PACK = {"append": (G._APPEND, APPEND), "prefix": (G._PREFIX, PREFIX), "policy": (G._POLICY, POLICY)}
INVALID, UNSUPPORTED = B.FE_ERR_INVALID_ARG, B.FE_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    fe_build.build()
    return B.load_library()


def packed(kind, **kw):
    form, names = PACK[kind]
    a = dict(GOOD[kind], **kw)
    assert len(a) == len(names)
    return form.pack(*(a[n] for n in names))


def call(lib, kind, **kw):
    a = packed(kind, **kw)
    if kind == "append":
        return lib.fe_kv_append(a, None)
    if kind == "prefix":
        return lib.fe_prefix_attention(a, None)
    return lib.fe_policy_loss(a, None)


def test_python_packs_the_structures_of_the_header(tmp_path):
    """Sizes and every field's offset, as a C compiler sees them."""
    fields = {"append": ("fe_append_args", {"kc": "kv.k", "vc": "kv.v"}), "prefix": ("fe_prefix_args", {"kc": "kv.k", "vc": "kv.v"}),
              "policy": ("fe_policy_args", {})}
    src = ['#include <stddef.h>', '#include <stdio.h>', '#include "fe.h"', "int main(void) {"]
    for kind, (name, other) in fields.items():
        src.append(f'printf("%zu\\n", sizeof({name}));')
        for f in PACK[kind][1]:
            f = other.get(f, f"kv.{f}" if kind != "policy" and f in KV else f)
            src.append(f'printf("%zu\\n", offsetof({name}, {f}));')
    (tmp_path / "a.c").write_text("\n".join(src + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "a")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for kind in fields:
        form, names = PACK[kind]
        want.append(form.size)
        zero = form.pack(*([0] * len(names)))
        for i in range(len(names)):
            one = form.pack(*([0] * i + [1] + [0] * (len(names) - i - 1)))
            at = next(j for j in range(form.size) if one[j] != zero[j])
            # (a float's 1 has its bits at its end)
            want.append(at - at % 4)
    assert got == want


@pytest.mark.parametrize("kind", ["append", "prefix"])
@pytest.mark.parametrize("change,code", [
    (dict(kc=0), INVALID), (dict(vc=0), INVALID), (dict(kc=P + 64), INVALID), (dict(vc=P + 2), INVALID),
    (dict(n_pages=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=-1), INVALID),
    (dict(dtype=B.FE_IO_F32), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(page_rows=8), UNSUPPORTED),
    (dict(page_rows=48), UNSUPPORTED), (dict(page_rows=256), UNSUPPORTED), (dict(head_dim=16), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(n_pages=1 << 24), UNSUPPORTED),  # 2^31 rows of 2 heads
    (dict(n_seqs=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(page_cols=0), INVALID), (dict(n_seqs=0), INVALID),
    (dict(row_start=0), INVALID), (dict(pages=0), INVALID), (dict(q=P + 8), UNSUPPORTED), (dict(q_row=260), UNSUPPORTED),
    (dict(q_head=4), UNSUPPORTED),
])
def test_pages_and_rows(lib, kind, change, code):
    assert call(lib, kind, **change) == code
    assert lib.fe_last_error_message().decode()


@pytest.mark.parametrize("change,code", [
    (dict(first=0), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(q_out=0), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_out=P), INVALID),  # in place, and the queries not contiguous
    (dict(k=P + 8), UNSUPPORTED), (dict(v_row=132), UNSUPPORTED), (dict(k_head=2), UNSUPPORTED), (dict(q_out=P + 2), UNSUPPORTED),
    (dict(pairs=2), INVALID), (dict(pairs=-1), INVALID), (dict(rope_rows=0), INVALID), (dict(rope=P + 4), INVALID),
    (dict(rot_dim=0), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=128), UNSUPPORTED),
])
def test_append(lib, change, code):
    assert call(lib, "append", **change) == code
    assert lib.fe_last_error_message().decode()


@pytest.mark.parametrize("change,code", [
    (dict(n_groups=-1), INVALID), (dict(n_groups=0), INVALID), (dict(prefix_cols=0), INVALID),
    (dict(q_heads=0), INVALID), (dict(q_heads=3), INVALID), (dict(q_heads=4096), UNSUPPORTED),
    (dict(n_rows=1 << 30), UNSUPPORTED), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(scale=-1.0), INVALID), (dict(group_start=0), INVALID), (dict(prefix_len=0), INVALID),
    (dict(prefix_pages=0), INVALID), (dict(seq_len=0), INVALID), (dict(out=0), INVALID), (dict(out=3 * P + 8), UNSUPPORTED), (dict(out=3 * P + 16), UNSUPPORTED),
    (dict(out=P), INVALID), (dict(workspace=0), INVALID), (dict(workspace=P + 128), INVALID),
])
def test_attention(lib, change, code):
    assert call(lib, "prefix", **change) == code
    assert lib.fe_last_error_message().decode()
    if "workspace" not in change:
        assert lib.fe_prefix_attention_workspace(packed("prefix", **change)) == 0


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(temperature=0.0), INVALID), (dict(temperature=-1.0), INVALID), (dict(temperature=math.nan), INVALID),
    (dict(temperature=math.inf), INVALID), (dict(temperature=1e-44), INVALID), (dict(grad_scale=math.inf), INVALID),
    (dict(logits=0), INVALID), (dict(tokens=0), INVALID), (dict(lse=0), INVALID), (dict(coef=0), INVALID),
    (dict(logits=P + 1), INVALID), (dict(grad=P + 1), INVALID), (dict(logits_row=99), INVALID), (dict(grad_row=99), INVALID),
    (dict(grad=P, grad_row=104), INVALID),
])
def test_policy(lib, change, code):
    assert call(lib, "policy", **change) == code
    assert lib.fe_policy_loss_backward(packed("policy", **change), None, None) == code
    assert lib.fe_last_error_message().decode()


@pytest.mark.parametrize("change", [
    dict(loss=0), dict(advantages=0), dict(terms=0), dict(logp=0), dict(clip_low=-0.1), dict(clip_low=1.5),
    dict(clip_low=math.nan), dict(clip_high=-0.1), dict(clip_high=math.nan), dict(beta=math.inf), dict(beta=math.nan),
])
def test_policy_forward(lib, change):
    assert call(lib, "policy", **change) == INVALID


def test_policy_backward_needs_a_gradient(lib):
    assert lib.fe_policy_loss_backward(packed("policy", grad=0), None, None) == INVALID


def test_null_and_empty_calls(lib):
    for f in (lib.fe_kv_append, lib.fe_prefix_attention, lib.fe_policy_loss):
        assert f(None, None) == INVALID
    assert lib.fe_policy_loss_backward(None, None, None) == INVALID
    assert lib.fe_prefix_attention_workspace(None) == 0
    assert call(lib, "append", n_rows=0, n_seqs=0) == B.FE_OK  # nothing to do, nothing enqueued
    assert call(lib, "prefix", n_rows=0, n_seqs=0, n_groups=0) == B.FE_OK
    assert lib.fe_policy_loss_backward(packed("policy", rows=0), None, None) == B.FE_OK


def test_tensors_that_are_not_on_a_gpu():
    x = torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        G.PagedKV(x, x.clone())
    with pytest.raises(ValueError):
        G.policy_loss(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2))


# ---------------------------------------------------------------------------
# the Python calls
# ---------------------------------------------------------------------------
def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda:0")


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda:0")


@pytest.mark.gpu
@pytest.mark.parametrize("make", [
    lambda: G.PagedKV(gpu(4, 2, 64), gpu(4, 2, 64)),
    lambda: G.PagedKV(gpu(4, 2, 64, 64), gpu(4, 2, 64, 32)),
    lambda: G.PagedKV(gpu(4, 2, 64, 64), gpu(4, 2, 64, 64, dtype=torch.float16)),
    lambda: G.PagedKV(gpu(4, 2, 64, 64, dtype=torch.float32), gpu(4, 2, 64, 64, dtype=torch.float32)),
    lambda: G.PagedKV(gpu(4, 64, 2, 64).transpose(1, 2), gpu(4, 64, 2, 64).transpose(1, 2)),
])
def test_pages_that_python_refuses(make):
    with pytest.raises(ValueError):
        make()


@pytest.mark.gpu
@pytest.mark.parametrize("change", [
    dict(k="type"), dict(k="heads"), dict(k="dim"), dict(v="rows"), dict(q="type"), dict(row_start="long"),
    dict(row_start="short"), dict(first="cpu"), dict(pages="rows"), dict(pages="float"), dict(pairs="even"), dict(rope="flat"),
    dict(rope="half"), dict(shift="short"), dict(q_out="shape"), dict(status="long"),
])
def test_append_calls_that_python_refuses(change):
    pages = G.PagedKV(gpu(4, 2, 64, 64), gpu(4, 2, 64, 64))
    a = dict(k=gpu(3, 2, 64), v=gpu(3, 2, 64), row_start=ints(0, 1, 3), first=ints(0, 0), pages=ints(0, 1).view(2, 1),
             q=gpu(3, 4, 64), rope=gpu(8, 32, 2, dtype=torch.float32))
    pages.append(**a)
    (name, what), = change.items()
    bad = {("k", "type"): gpu(3, 2, 64, dtype=torch.float16), ("k", "heads"): gpu(3, 1, 64), ("k", "dim"): gpu(3, 2, 32),
           ("v", "rows"): gpu(2, 2, 64), ("q", "type"): gpu(3, 4, 64, dtype=torch.float32),
           ("row_start", "long"): torch.tensor([0, 1, 3], device="cuda:0"), ("row_start", "short"): ints(0, 3),
           ("first", "cpu"): torch.zeros(2, dtype=torch.int32), ("pages", "rows"): ints(0).view(1, 1),
           ("pages", "float"): gpu(2, 1, dtype=torch.float32), ("pairs", "even"): "even",
           ("rope", "flat"): gpu(8, 64, dtype=torch.float32), ("rope", "half"): gpu(8, 32, 2), ("shift", "short"): ints(0),
           ("q_out", "shape"): gpu(3, 2, 64), ("status", "long"): torch.zeros(1, dtype=torch.int64, device="cuda:0")}
    with pytest.raises(ValueError):
        pages.append(**dict(a, **{name: bad[name, what]}))


@pytest.mark.gpu
def test_attention_calls_that_python_or_the_library_refuses():
    pages = G.PagedKV(gpu(4, 2, 64, 64), gpu(4, 2, 64, 64))
    a = dict(q=gpu(3, 4, 64), row_start=ints(0, 1, 3), lengths=ints(1, 2), pages=ints(0, 1).view(2, 1), group_start=ints(0, 2),
             prefix_lengths=ints(0), prefix_pages=ints(2).view(1, 1))
    pages.attend(**a)
    need = pages.workspace_bytes(1, 2, 3, 4)
    pages.attend(**a, workspace=gpu(need, dtype=torch.uint8))
    for bad in (dict(q=gpu(3, 4, 32)), dict(q=gpu(3, 64, 4).transpose(1, 2)), dict(row_start=ints(0, 3)), dict(lengths=ints(1, 2, 3)),
                dict(group_start=ints(0)), dict(prefix_pages=ints(2)), dict(pages=ints(0, 1)), dict(out=gpu(3, 4, 32)),
                dict(out=gpu(4, 3, 64).transpose(0, 1)), dict(workspace=gpu(need // 2))):
        with pytest.raises(ValueError):
            pages.attend(**dict(a, **bad))
    for bad, code in ((dict(q=gpu(3, 3, 64)), INVALID), (dict(out=a["q"]), INVALID), (dict(scale=-1.0), INVALID),
                      (dict(q=gpu(3, 4, 68)[..., 4:]), UNSUPPORTED),
                      (dict(workspace=gpu(need - 256, dtype=torch.uint8)), B.FE_ERR_WORKSPACE)):
        with pytest.raises(B.FeError) as e:
            pages.attend(**dict(a, **bad))
        assert e.value.code == code
    with pytest.raises(B.FeError):
        pages.workspace_bytes(1, 2, 3, 5)
    pages.attend(**a)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_loss_calls_that_python_or_the_library_refuses():
    f32 = torch.float32
    a = dict(logits=gpu(3, 40), tokens=ints(1, 2, 3), advantages=gpu(3, dtype=f32))
    r = G.policy_loss(**a)
    for bad in (dict(logits=gpu(3, 40, 1)), dict(logits=gpu(40, 3).t()), dict(logits=gpu(3, 40, dtype=torch.float64)),
                dict(tokens=ints(1, 2)), dict(tokens=torch.zeros(3, dtype=torch.int64, device="cuda:0")),
                dict(advantages=gpu(3)), dict(advantages=gpu(2, dtype=f32)), dict(weights=gpu(4, dtype=f32)),
                dict(old_logp=torch.zeros(3)), dict(ref_logp=gpu(6, dtype=f32)[::2]), dict(grad=gpu(3, 41)),
                dict(grad=gpu(3, 40, dtype=f32)), dict(grad=gpu(40, 3).t()), dict(status=gpu(1))):
        with pytest.raises(ValueError):
            G.policy_loss(**dict(a, **bad))
    for bad in (dict(temperature=0.0), dict(clip=(2.0, 0.2)), dict(beta=float("nan")), dict(grad_scale=float("inf"))):
        with pytest.raises(B.FeError) as e:
            G.policy_loss(**dict(a, **bad))
        assert e.value.code == INVALID
    with pytest.raises(ValueError):
        G.policy_loss_backward(a["logits"], a["tokens"], r, upstream=gpu(2, dtype=f32))
    with pytest.raises(ValueError):
        G.policy_loss_backward(gpu(2, 40), ints(1, 2), r)  # statistics of other rows
    G.policy_loss(**a)
    torch.cuda.synchronize()
