"""Refusals of the operators that keep no logits, no mask and no copy of a norm's input, without a GPU: bad arguments are answered with
a status before anything is launched."""
import os
import subprocess

import pytest
import torch

import paper_2505_05086_amd as asi
from paper_2505_05086_amd import binding as B

P = 0x10000          # non-null, 256-aligned, never dereferenced by validation
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
MANY = 1 << 50


def _of(cls, values, changed):
    values.update(changed)
    return cls(*[values[n] for n, _ in cls._fields_])


def _head(**kw):
    return _of(B.LinearLogprobDesc, dict(rows=40, dim=64, vocab=100, hidden_stride=64, weight_stride=64, ignore_index=-100, dtype=1, scale=1.0,
                                         any_address=0, reserved=0), kw)


def _values(d, h=P, w=P, t=P, logprob=P, entropy=P, stats=P, ws=P, size=MANY):
    return B.lib().asi_linear_logprobs(d, h, w, t, logprob, entropy, stats, ws, size, None)


def _grad(d, given=0, h=P, w=P, t=P, stats=P, logprob=P, entropy=P, a=P, b=P, dh=P, dw=P, ws=P, size=MANY):
    return B.lib().asi_linear_logprobs_grad(d, given, h, w, t, stats, logprob, entropy, a, b, dh, dw, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(vocab=0), INVALID), (dict(hidden_stride=63), INVALID), (dict(weight_stride=63), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=1e-30), UNSUPPORTED), (dict(scale=1e30), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(any_address=2), INVALID), (dict(reserved=1), INVALID), (dict(rows=1 << 24), UNSUPPORTED),
    (dict(dim=1 << 18, hidden_stride=1 << 18, weight_stride=1 << 18), UNSUPPORTED), (dict(vocab=1 << 28), UNSUPPORTED), (dict(rows=1 << 20, vocab=1 << 20), UNSUPPORTED),
    (dict(rows=(1 << 24) - 1, dim=(1 << 18) - 1, hidden_stride=1 << 18, weight_stride=1 << 18), UNSUPPORTED)])
def test_head_descriptors(bad, status):
    d = _head(**bad)
    assert _values(d) == status and _grad(d) == status
    assert B.lib().asi_linear_logprobs_workspace_bytes(d) == 0 and B.lib().asi_linear_logprobs_grad_workspace_bytes(d) == 0


def test_head_arguments():
    assert _values(None) == INVALID and _grad(None) == INVALID
    d = _head()
    for kw in (dict(h=None), dict(w=None), dict(t=None), dict(h=P + 1), dict(w=P + 8), dict(t=P + 4), dict(logprob=P + 2), dict(entropy=P + 1), dict(stats=P + 3)):
        assert _values(d, **kw) == INVALID, kw
        assert _grad(d, **kw) == INVALID or "stats" in kw and kw["stats"] is None, kw
    for kw in (dict(given=2), dict(given=1, stats=None), dict(given=1, entropy=None), dict(dh=P + 1), dict(dw=P + 1), dict(a=P + 2), dict(b=P + 1), dict(t=None, logprob=None)):
        assert _grad(d, **kw) == INVALID, kw
    for size, f in ((B.lib().asi_linear_logprobs_workspace_bytes(d), _values), (B.lib().asi_linear_logprobs_grad_workspace_bytes(d), _grad)):
        assert size > 0 and size % 256 == 0
        for kw in (dict(ws=None), dict(ws=P + 64), dict(size=size - 1)):
            assert f(d, **kw) == WORKSPACE, kw
    assert _values(_head(rows=0), h=None, w=None, t=None) == OK and _grad(_head(rows=0), h=None, w=None, dw=None) == OK


def test_head_scratch_holds_no_more_than_a_piece_of_the_logits():
    need = B.lib().asi_linear_logprobs_grad_workspace_bytes
    small, large = (need(_head(rows=4096, dim=1024, vocab=v, hidden_stride=1024, weight_stride=1024)) for v in (20000, 200000))
    assert large - small < 4096 * 180000 * 2 / 8                          # the values of the tiles alone grow
    assert need(_head(any_address=1)) > need(_head())


HEAD_PLAN = """
#include <stdio.h>
#include <stdlib.h>
#include "asi_head_plan.h"
using namespace asi;
// what a call writes in its workspace; dz may lie where the parts were
struct Region { const char* name; size_t at, bytes; };
int main() {
    unsigned long long state = 1;
    auto random = [&](long long lo, long long hi) {          // spread over the logarithm
        state = state * 6364136223846793005ull + 1442695040888963407ull;
        double x = (double)lo;
        const double f = (double)(state >> 40) / (1 << 24);
        double ratio = (double)hi / lo;
        return (long long)(x * __builtin_pow(ratio, f) + 0.5);
    };
    long long several = 0, small = 0, kept = 0;
    for (int n = 0; n < 400000; ++n) {
        asi_linear_logprob_desc d{};
        d.rows = random(1, n % 2 ? 1 << 23 : 2000); d.dim = random(1, (1 << 18) - 1); d.vocab = random(1, n % 2 ? (1 << 28) - 1 : 300000);
        if (n % 3 == 0) d.dim = (d.dim + 63) / 64 * 64;
        if (n % 5 == 0) d.vocab = (d.vocab + 255) / 256 * 256;
        d.hidden_stride = d.dim; d.weight_stride = d.dim + random(1, 9) - 1;
        d.dtype = n % 7 < 4 ? ASI_F32 : ASI_BF16; d.scale = 1.f; d.any_address = n % 11 == 0;
        if (up(d.rows, 128) / 128 * (up(d.vocab, 128) / 128) > (1 << 23) || up(d.dim, 128) / 128 * (up(d.vocab, 128) / 128) > (1 << 23)) continue;
        for (int grad = 0; grad < 2; ++grad) {
            const Plan p = plan(&d, grad);
            bool fine = true;
            const int planes = d.dtype == ASI_F32 ? 3 : 1;
            if (!p.few) {
                long long token = 0, part = 0, pieces = 0;
                each_piece(p, [&](long long first, long long count, int tile, long long first_part) {
                    fine = fine && first == token && count > 0 && (count + (p.staged ? 0 : p.piece) <= p.piece || !p.staged) && first_part == part && (tile == 128 || tile == 256);
                    token += count;
                    part += (count + tile - 1) / tile;
                    ++pieces;
                    small += pieces > 1 && tile != p.tile;
                    if (p.keep) fine = fine && pieces == 1;
                });
                fine = fine && token == d.vocab && part == p.parts;
                several += pieces > 1;
                kept += p.keep;
            }
            Region r[12];
            int count = 0;
            auto add = [&](const char* name, size_t at, long long bytes) { r[count++] = Region{name, at, (size_t)bytes}; };
            add("target", p.target, d.rows * 4);
            if (grad) add("info", p.info, d.rows * 32);
            const int part = count;
            add("part", p.part, p.parts * 16 * d.rows);
            int dz = -1;
            if (!p.few) {
                const long long packed = (d.dim + 63) / 64 * 64, rows_up = up(d.rows, p.tile);
                add("split", p.split, 16); add("live", p.live, d.rows * 4); add("place", p.place, d.rows * 4);
                add("hidden", p.hidden, planes * d.rows * packed * 2);
                if (p.staged) add("weights", p.weights, planes * p.piece * packed * 2);
                if (grad) {
                    dz = count;
                    add("dz", p.dz, (planes == 3 ? 3 : 2) * rows_up * p.piece * 2);
                    add("sums", p.sums, d.rows * p.most_splits * d.dim * 4);
                    fine = fine && p.most_splits >= 1 && p.most_sums == d.rows * p.most_splits && p.piece % 256 == 0;
                    if (p.keep) add("kept", p.kept, rows_up * up(d.vocab, p.tile) * 4);
                }
            } else if (grad) {
                add("logits", p.logits, up(d.rows, 16) * d.vocab * 4);
                add("sums", p.sums, p.few_blocks * d.rows * d.dim * 4);
            }
            const char* what = "";
            for (int i = 0; i < count; ++i) {
                if (r[i].at % 256 || r[i].at + r[i].bytes > p.bytes) { fine = false; what = r[i].name; }
                for (int j = 0; j < i; ++j)
                    if (r[i].at < r[j].at + r[j].bytes && r[j].at < r[i].at + r[i].bytes && !(i == dz && j == part)) { fine = false; what = r[i].name; }
            }
            if (!fine) {
                printf("%lld x %lld x %lld, type %d, gradients %d: tile %d, piece %lld, parts %lld %s\\n", (long long)d.rows, (long long)d.dim, (long long)d.vocab, d.dtype, grad, p.tile, p.piece, p.parts, what);
                return 1;
            }
        }
    }
    printf("%d %d %d\\n", several > 1000, small > 100, kept > 1000);
    return 0;
}
"""


def test_head_pieces_and_what_they_write_lie_beside_each_other(tmp_path):
    """The parts of the pieces' tiles follow each other without a gap and end where their memory does, and no two regions of the workspace
    overlap or reach behind its end: over random sizes of the whole range, pieces in tiles smaller than the call's among them."""
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(HEAD_PLAN)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_05086_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I" + csrc, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.split() == ["1", "1", "1"], res.stdout


def _drop(**kw):
    return _of(B.DropoutDesc, dict(rows=4, dim=10, x_stride=10, y_stride=10, seed=1, offset=2, p=0.1, dtype=0, reserved=0), kw)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(x_stride=9), INVALID), (dict(y_stride=9), INVALID), (dict(p=-0.1), INVALID), (dict(p=1.0), INVALID),
    (dict(p=0.999999), INVALID), (dict(p=float("nan")), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(reserved=1), INVALID),
    (dict(dim=1 << 31, x_stride=(1 << 31) + 1, y_stride=1 << 31), UNSUPPORTED), (dict(rows=1 << 30, dim=1 << 30, x_stride=1 << 30, y_stride=1 << 30), UNSUPPORTED)])
def test_dropout_descriptors(bad, status):
    assert B.lib().asi_dropout(_drop(**bad), P, None, 2 * P, None) == status


def test_dropout_arguments():
    f = B.lib().asi_dropout
    assert f(None, P, None, P, None) == INVALID and f(_drop(), None, None, P, None) == INVALID and f(_drop(), P, None, None, None) == INVALID
    assert f(_drop(), P + 2, None, P, None) == INVALID and f(_drop(), P, None, P + 2, None) == INVALID and f(_drop(), P, P + 4, P, None) == INVALID
    assert f(_drop(x_stride=12), P, None, P, None) == INVALID              # in place with another stride
    assert f(_drop(rows=0), None, None, None, None) == OK


def _edge(**kw):
    return _of(B.ResidualDesc, dict(rows=12, dim=64, x_stride=64, y_stride=64, gate_rows=3, seed=1, offset=0, p=0.1, stream_dtype=0, dtype=0, gain_dtype=0,
                                    post_norm=1, scale=1.0, eps=1e-6), kw)


def _forward(d, x=P, y=P, post=P, gate=P, pre=P, seed=None, s=2 * P, out=P):
    return B.lib().asi_residual_norm(d, x, y, post, gate, pre, seed, s, out, None)


def _backward(d, ds=P, do=P, s=P, y=P, post=P, gate=P, pre=P, seed=None, dx=P, dy=P, dpost=P, dgate=P, dpre=P, ws=P, size=MANY):
    return B.lib().asi_residual_norm_grad(d, ds, do, s, y, post, gate, pre, seed, dx, dy, dpost, dgate, dpre, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(x_stride=63), INVALID), (dict(y_stride=63), INVALID), (dict(gate_rows=-1), INVALID), (dict(gate_rows=5), INVALID),
    (dict(gate_rows=24), INVALID), (dict(post_norm=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(p=1.0), INVALID), (dict(p=-1.0), INVALID), (dict(stream_dtype=2), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(gain_dtype=2), UNSUPPORTED), (dict(stream_dtype=1), UNSUPPORTED), (dict(dim=16385, x_stride=16385, y_stride=16385), UNSUPPORTED), (dict(rows=3 << 40), UNSUPPORTED)])
def test_residual_descriptors(bad, status):
    d = _edge(**bad)
    assert _forward(d) == status and _backward(d) == status and B.lib().asi_residual_norm_grad_workspace_bytes(d) == 0


def test_residual_arguments():
    assert _forward(None) == INVALID and _backward(None) == INVALID
    d = _edge()
    for kw in (dict(x=None), dict(y=None), dict(s=None), dict(gate=None), dict(x=P + 2), dict(y=P + 1), dict(post=P + 2), dict(gate=P + 1), dict(pre=P + 3), dict(seed=P + 4),
               dict(s=P + 2), dict(out=P + 1)):
        assert _forward(d, **kw) == INVALID, kw
    assert _forward(_edge(post_norm=0)) == INVALID and _forward(_edge(gate_rows=0)) == INVALID
    assert _forward(_edge(gate_rows=0), y=None, post=None, gate=None, s=None, out=None) == INVALID
    assert _forward(_edge(x_stride=80), s=P) == INVALID                    # in place with another stride
    for kw in (dict(ds=None, do=None), dict(s=None), dict(y=None), dict(dy=None), dict(gate=None), dict(ds=P + 2), dict(do=P + 1), dict(dx=P + 2), dict(dy=P + 2),
               dict(dpost=P + 2), dict(dgate=P + 1), dict(dpre=P + 3)):
        assert _backward(d, **kw) == INVALID, kw
    size = B.lib().asi_residual_norm_grad_workspace_bytes(d)
    assert size > 0 and size % 256 == 0
    for kw in (dict(ws=None), dict(ws=P + 64), dict(size=size - 1)):
        assert _backward(d, **kw) == WORKSPACE, kw
    none = _edge(rows=0, gate_rows=0)
    assert _forward(none, x=None, y=None) == OK


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x = torch.zeros(4, 64)
    for bad in (lambda: asi.dropout(x, 0.1, 1), lambda: asi.residual_norm(x, x), lambda: asi.linear_logprobs(x, x)):
        with pytest.raises(ValueError):
            bad()


def test_the_version_tells_libraries_with_these_entry_points_apart():
    assert B.asi_version() >= 1004
