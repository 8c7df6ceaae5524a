"""Refusals of the losses over a vocabulary: everything is checked before any work is enqueued, so no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2306_09342_amd import binding as B

GOOD = dict(rows=40, d_model=64, vocab=1001, mode="bf16", grad_mode="fp32", bias=True, top_k=4, temperature=2.0)
P = 0x100000                       # never dereferenced


def _cfg(**more):
    return B.make_vocab_cfg(**dict(GOOD, **more))


def test_sizes():
    c = _cfg()
    assert B.rev_vocab_check_cfg(c) == 0
    assert B.rev_vocab_param_count(c) == 1001 * 64 + 1001
    assert B.rev_vocab_param_count(_cfg(bias=False)) == 1001 * 64
    n = B.rev_vocab_workspace_bytes(c)
    assert n > 0 and n % 256 == 0


@pytest.mark.parametrize("rows,d,vocab", [(1 << 20, 8, 1), (1, 8192, 1 << 20), (65536, 1024, 131072), (1, 8, 1), (1 << 20, 8192, 1 << 20)])
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_the_workspace_never_holds_the_logits(rows, d, vocab, mode):
    """At the limits its size is that of the rows and the weights, and a bounded number of bytes besides."""
    n = B.rev_vocab_workspace_bytes(_cfg(rows=rows, d_model=d, vocab=vocab, mode=mode))
    assert 0 < n
    rows_up, d_up, e = rows + 256, d + 128, 2 if mode == "bf16" else 6
    # the rows' copy and dx, W laid out, statistics and dz of a piece (256 MB and 512 MB, or 256 entries of all rows), small tables of rows and teachers
    assert n <= rows_up * (e * d_up + 4 * (d_up + 256) + 64 + 4 * 5) + e * (vocab + 256) * d_up + max(1 << 28, 6144 * rows_up // 256 * 4) + max(
        1 << 29, 256 * e * rows_up) + (1 << 28) + 300 * 4 * min(rows, 512) * (vocab + d_up)


@pytest.mark.parametrize("bad", [dict(rows=0), dict(rows=-1), dict(d_model=0), dict(d_model=12), dict(d_model=8200), dict(vocab=0), dict(vocab=(1 << 20) + 1),
                                 dict(rows=(1 << 20) + 1), dict(mode=2), dict(grad_mode=3), dict(mode="fp32", grad_mode="bf16"), dict(bias=2),
                                 dict(top_k=-1), dict(top_k=257), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
                                 dict(temperature=float("inf"))])
def test_bad_configs(bad):
    c = _cfg(**bad)
    assert B.rev_vocab_check_cfg(c) == -1 and B.rev_last_error()
    with pytest.raises(B.RevError):
        B.rev_vocab_workspace_bytes(c)


def test_null_config():
    assert B.lib().rev_vocab_check_cfg(None) == -1
    assert B.lib().rev_vocab_param_count(None) == -1


# pointers of each call, in order; those that may be null
CALLS = {"rev_xent_forward": ("params", "X", "labels", "loss", "lse"),
         "rev_xent_backward": ("params", "X", "labels", "lse", "dloss", "dX", "dparams"),
         "rev_distill_forward": ("params", "X", "labels", "teacher_idx", "teacher_logits", "loss_ce", "loss_kd", "lse"),
         "rev_distill_backward": ("params", "X", "labels", "teacher_idx", "teacher_logits", "lse", "dloss_ce", "dloss_kd", "dX", "dparams")}


def _call(name, cfg, pointers, ws=P, bytes_=None):
    n = B.rev_vocab_workspace_bytes(cfg) if bytes_ is None else bytes_
    return getattr(B.lib(), name)(ctypes.byref(cfg), *[ctypes.c_void_p(p) for p in pointers], ctypes.c_void_p(ws), n, None)


@pytest.mark.parametrize("name", list(CALLS))
def test_null_and_misaligned_pointers(name):
    c, names = _cfg(), CALLS[name]
    for k, n in enumerate(names):
        p = [P] * len(names)
        if n not in ("dX", "dparams"):
            p[k] = None
            assert _call(name, c, p) == -1, n
        p[k] = P + (8 if n in ("params", "X", "dX", "dparams") else 2)
        assert _call(name, c, p) == -1 and "aligned" in B.rev_last_error(), n
    if "dX" in names:
        p = [None if n in ("dX", "dparams") else P for n in names]
        assert _call(name, c, p) == -1 and "both null" in B.rev_last_error()


@pytest.mark.parametrize("name", list(CALLS))
def test_workspace(name):
    c, p = _cfg(), [P] * len(CALLS[name])
    assert _call(name, c, p, ws=None) == -1
    assert _call(name, c, p, ws=P + 128) == -1
    n = B.rev_vocab_workspace_bytes(c)
    assert _call(name, c, p, bytes_=n - 1) == -2 and "workspace too small" in B.rev_last_error()


@pytest.mark.parametrize("name", ["rev_distill_forward", "rev_distill_backward"])
def test_distillation_needs_a_teacher_and_labels_go_with_their_loss(name):
    names = CALLS[name]
    assert _call(name, _cfg(top_k=0), [P] * len(names)) == -1 and "top_k" in B.rev_last_error()
    ce = "loss_ce" if "loss_ce" in names else "dloss_ce"
    for missing in ("labels", ce):
        p = [None if n == missing else P for n in names]
        assert _call(name, _cfg(), p) == -1 and "go together" in B.rev_last_error()


def test_the_binding_refuses_other_types_and_shapes():
    c = _cfg()
    with pytest.raises(AssertionError):
        B.rev_xent_forward(c, torch.zeros(B.rev_vocab_param_count(c), dtype=torch.bfloat16), torch.zeros(40, 64, dtype=torch.bfloat16),
                           torch.zeros(40, dtype=torch.int32))            # CPU tensors


MB = 1 << 20


@pytest.mark.parametrize("mode,rows,d,vocab,most", [("bf16", 129, 64, 200, 2 * MB), ("bf16", 129, 128, 1000, 4 * MB), ("bf16", 300, 64, 17000, 60 * MB),
                                                    ("fp32", 129, 64, 200, 2 * MB), ("fp32", 900, 64, 5001, 100 * MB)])
def test_small_problems_have_small_workspaces(mode, rows, d, vocab, most):
    """No more places for ranges of dX than the ranges that there can be."""
    assert B.rev_vocab_workspace_bytes(_cfg(rows=rows, d_model=d, vocab=vocab, mode=mode)) <= most


@pytest.mark.parametrize("rows,d,vocab", [(64, 8192, 1 << 20), (64, 4096, 131072), (33, 8192, 300000), (1, 8192, 1 << 20), (64, 2048, 32000), (768, 8, 81380),
                                          (512, 976, 1000)])
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_the_workspace_of_few_rows_is_bounded(rows, d, vocab, mode):
    """Rows' copy and tables, named logits, dz of the whole vocabulary or of a piece, statistics, fragments of dX and dW, and W where tiles need it laid out."""
    n = B.rev_vocab_workspace_bytes(_cfg(rows=rows, d_model=d, vocab=vocab, mode=mode))
    rows_up, d_up = (rows + 255) // 256 * 256, (d + 127) // 128 * 128
    few = mode == "fp32"                                         # (bf16 of these sizes goes through tiles, and W as it lies)
    fixed = rows_up * (6 * d_up + 64) + 4 * rows * 5 + 4096
    assert n <= fixed + (256 * MB if few else 512 * MB) + 32 * MB + 256 * MB + (0 if few else 256 * MB) + (2 * vocab * d_up if d % 128 else 0)


@pytest.mark.parametrize("rows,d,vocab", [(8192, 1024, 131072), (65536, 1024, 131072), (4096, 64, 1 << 20), (1 << 20, 8, 50265), (1 << 20, 8192, 1 << 20), (16384, 768, 50265),
                                          (2500, 200, 1 << 20), (769, 128, 900000), (1000, 8192, 300), (129, 64, 50265)])
@pytest.mark.parametrize("top_k", [0, 256])
@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_the_workspace_is_what_the_header_says(rows, d, vocab, top_k, mode):
    """Its parts one by one, each at its bound; where the logits of all rows would be larger than that, they are not in it."""
    n = B.rev_vocab_workspace_bytes(_cfg(rows=rows, d_model=d, vocab=vocab, mode=mode, top_k=top_k))
    rows_up, d_up, e = (rows + 255) // 256 * 256, (d + 127) // 128 * 128, 2 if mode == "bf16" else 6
    copies = rows_up * e * d_up + (e * vocab * d_up if mode == "fp32" or d % 128 else 0) + 4 * rows_up * ((d + 255) // 256 * 256)
    tables = 64 * rows_up + 4 * rows * (top_k + 1) + 4096
    pieces = max(512 * MB, 256 * e * rows_up) + max(256 * MB, 24 * rows_up)
    assert n <= copies + tables + pieces + 2 * 256 * MB
    # the logits at two bytes each would not fit beside what goes with the elements
    if 2 * rows * vocab > pieces + 2 * 256 * MB:
        assert n < copies + tables + 2 * rows * vocab
