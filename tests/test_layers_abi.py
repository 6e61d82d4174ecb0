"""The layers' and the gradient norm's entry points without a GPU: struct layouts, refusals before any device work, and the plans' arithmetic."""
import ctypes as C
import subprocess
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def L(amlib):
    from paper_2601_22442_amd import layers
    return layers


def _table(*vals):
    return C.addressof(_table.keep.setdefault(vals, (C.c_void_p * len(vals))(*vals)))


_table.keep = {}


def test_structs_mirror_the_header(L, tmp_path):
    src = tmp_path / "abi.c"
    src.write_text(r"""
#include <stddef.h>
#include <stdio.h>
#include "asyncmesh.h"
int main(void) {
    printf("%zu %zu %zu\n", sizeof(am_linear_config), offsetof(am_linear_config, in), offsetof(am_linear_config, dx_stride));
    printf("%zu %zu %zu\n", sizeof(am_linear_buffers), offsetof(am_linear_buffers, pre), offsetof(am_linear_buffers, workspace_bytes));
    printf("%zu %zu %zu\n", sizeof(am_norm_config), offsetof(am_norm_config, dtype), offsetof(am_norm_config, max_norm));
    printf("%zu %zu %zu\n", sizeof(am_qk_config), offsetof(am_qk_config, rotated), offsetof(am_qk_config, eps));
    printf("%zu %zu %zu\n", sizeof(am_qk_buffers), offsetof(am_qk_buffers, positions), offsetof(am_qk_buffers, workspace_bytes));
    return 0;
}
""")
    exe = tmp_path / "abi"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", str(ROOT / "include"), "-o", str(exe), str(src)], check=True)
    lines = [list(map(int, line.split())) for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    for got, cls, a, b in zip(lines, (L.LinearConfig, L.LinearBuffers, L.NormConfig, L.QkConfig, L.QkBuffers), ("in_", "pre", "dtype", "rotated", "positions"),
                              ("dx_stride", "workspace_bytes", "max_norm", "eps", "workspace_bytes")):
        assert got == [C.sizeof(cls), getattr(cls, a).offset, getattr(cls, b).offset], cls


def _linear(L, **kw):
    base = dict(replicas=2, dtype=1, grad_dtype=1, act=0, rows=8, in_=16, out=32)
    base.update(kw)
    return L.LinearConfig(**base)


def _message(L):
    return L.lib.am_last_error().decode()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(replicas=0), -1, "replicas"), (dict(replicas=33), -1, "replicas"), (dict(dtype=2), -1, "dtype"), (dict(dtype=0), -1, "grad_dtype"),
    (dict(act=5), -1, "act"), (dict(in_=0), -1, "in="), (dict(out=1 << 31), -1, "out="), (dict(rows=1 << 31), -1, "rows="),
    (dict(x_stride=15), -1, "x_stride"), (dict(y_stride=31), -1, "y_stride"), (dict(residual_stride=1 << 31), -1, "residual_stride"),
])
def test_linear_refuses_bad_configs(L, kw, status, needle):
    cfg, good = _linear(L, **kw), _table(0x10000, 0x20000)
    buf, need = L.LinearBuffers(x=good, w=good, y=good, dy=good, dx=good, dw=good, db=good), C.c_uint64(0)
    assert L.lib.am_linear(C.byref(cfg), C.byref(buf), None) == status and needle in _message(L)
    assert L.lib.am_linear_backward(C.byref(cfg), C.byref(buf), 0, None) == status and needle in _message(L)
    assert L.lib.am_linear_workspace(C.byref(cfg), C.byref(buf), 0, C.byref(need)) == status


def test_linear_refuses_bad_buffers(L):
    cfg, good, odd, hole = _linear(L), _table(0x10000, 0x20000), _table(0x10000, 0x20001), _table(0x10000, 0)
    ref = C.byref(cfg)
    assert L.lib.am_linear(None, None, None) == -1 and L.lib.am_linear(ref, None, None) == -1
    for kw, status, needle in ((dict(w=good, y=good), -1, "x is NULL"), (dict(x=good, y=good), -1, "w is NULL"), (dict(x=good, w=good), -1, "y is NULL"),
                               (dict(x=good, w=hole, y=good), -1, "w[1]"), (dict(x=odd, w=good, y=good), -2, "x[1]"),
                               (dict(x=good, w=good, y=good, bias=odd), -2, "bias[1]"), (dict(x=good, w=good, y=good, pre=hole), -1, "pre[1]")):
        assert L.lib.am_linear(ref, C.byref(L.LinearBuffers(**kw)), None) == status and needle in _message(L), kw
    assert L.lib.am_linear_backward(ref, C.byref(L.LinearBuffers(dy=good, x=good, w=good)), 0, None) == -1 and "no gradient" in _message(L)
    assert L.lib.am_linear_backward(ref, C.byref(L.LinearBuffers(dy=good, x=good, w=good, db=odd)), 0, None) == -2 and "db[1]" in _message(L)
    cfg.act = 2
    assert L.lib.am_linear_backward(ref, C.byref(L.LinearBuffers(dy=good, x=good, w=good, dx=good)), 0, None) == -1 and "pre" in _message(L)
    # a workspace that is needed and missing, misaligned or too small: never reached without a check
    buf, need = L.LinearBuffers(dy=good, x=good, w=good, dx=good, pre=good), C.c_uint64(0)
    assert L.lib.am_linear_workspace(ref, C.byref(buf), 1, C.byref(need)) == 0 and need.value > 0
    assert L.lib.am_linear_backward(ref, C.byref(buf), 0, None) == -1 and "workspace is NULL" in _message(L)
    buf.workspace, buf.workspace_bytes = 0x100010, need.value
    assert L.lib.am_linear_backward(ref, C.byref(buf), 0, None) == -2
    buf.workspace, buf.workspace_bytes = 0x100000, need.value - 1
    assert L.lib.am_linear_backward(ref, C.byref(buf), 0, None) == -3


def test_norm_refusals(L):
    numel, dtype = (C.c_uint64 * 2)(5, 7), (C.c_uint32 * 2)(0, 1)
    grads, out, need = _table(0x1000, 0x2000, 0x3000, 0x4000), _table(0x5000, 0x6000), C.c_uint64(0)

    def cfg(**kw):
        base = dict(replicas=2, tensors=2, numel=C.addressof(numel), dtype=C.addressof(dtype), out_dtype=0, max_norm=1.0)
        base.update(kw)
        return L.NormConfig(**base)

    for kw, needle in ((dict(replicas=0), "replicas"), (dict(tensors=(1 << 20) + 1), "tensors"), (dict(numel=None), "numel"), (dict(out_dtype=2), "out_dtype"),
                       (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=float("nan")), "max_norm")):
        c = cfg(**kw)
        assert L.lib.am_norm_workspace(C.byref(c), C.byref(need)) == -1 and needle in _message(L), kw
    c = cfg()
    assert L.lib.am_norm_workspace(C.byref(c), C.byref(need)) == 0 and need.value == 8 * 2 * 2
    call = L.lib.am_clip_grads
    assert call(C.byref(c), None, None, 0x100, 0x200, 0x10000, 32, None) == -1 and "grads" in _message(L)
    assert call(C.byref(c), grads, None, None, 0x200, 0x10000, 32, None) == -1
    assert call(C.byref(c), grads, None, 0x102, 0x200, 0x10000, 32, None) == -2
    assert call(C.byref(c), grads, out, 0x100, 0x200, None, 0, None) == -1 and "workspace" in _message(L)
    assert call(C.byref(c), grads, out, 0x100, 0x200, 0x10000, 31, None) == -3
    assert call(C.byref(c), _table(0x1000, 0x2000, 0x3002, 0x4000), None, 0x100, 0x200, 0x10000, 32, None) == -2 and "replica 1, tensor 0" in _message(L)
    assert call(C.byref(c), _table(0x1000, 0x2000, 0x3000, 0), None, 0x100, 0x200, 0x10000, 32, None) == -1
    numel[0] = 1 << 40
    assert L.lib.am_norm_workspace(C.byref(c), C.byref(need)) == -1 and "2^40" in _message(L)


def test_qk_refusals(L):
    good = _table(0x10000, 0x20000)

    def call(status, needle, drop=(), backward=False, **kw):
        base = dict(replicas=2, dtype=1, grad_dtype=1, interleaved=0, tokens=4, q_heads=2, k_heads=1, head_dim=64, rotated=64, table_rows=4, eps=1e-6)
        base.update(kw)
        names = ["q", "k", "q_gain", "k_gain", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk"]
        buf = L.QkBuffers(**{n: good for n in names if n not in drop}, cos=0 if "cos" in drop else 0x100, sin=0x200)
        if "dq_gain" in drop:
            buf.dq_gain = good
        cfg = L.QkConfig(**base)
        f = (lambda: L.lib.am_qk_norm_backward(C.byref(cfg), C.byref(buf), 0, None)) if backward else (lambda: L.lib.am_qk_norm(C.byref(cfg), C.byref(buf), None))
        assert f() == status and needle in _message(L), (drop, kw, _message(L))

    for kw, needle in ((dict(replicas=33), "replicas"), (dict(dtype=0), "grad_dtype"), (dict(interleaved=2), "interleaved"), (dict(head_dim=65), "head_dim"),
                       (dict(head_dim=514), "head_dim"), (dict(rotated=66), "rotated"), (dict(rotated=31), "rotated"), (dict(table_rows=0), "table_rows"),
                       (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(q_heads=0, k_heads=0), "heads"), (dict(q_stride=127), "q_stride"),
                       (dict(tokens=1 << 31), "tokens")):
        call(-1, needle, **kw)
        call(-1, needle, backward=True, **kw)
    call(-1, "q is NULL", drop=("q",))
    call(-1, "k_gain is NULL", drop=("k_gain",))
    call(-1, "cos", drop=("cos",))
    call(-1, "dk_out", drop=("dk_out",), backward=True)
    call(-1, "workspace", drop=("dq_gain",), backward=True)


def test_the_binding_refuses_before_any_launch(L):
    x, w = [torch.zeros(4, 8)], [torch.zeros(3, 8)]
    for call in (lambda: L.linear(x, w), lambda: L.linear([], []), lambda: L.linear_backward(x, x, w), lambda: L.grad_norm([x]), lambda: L.grad_norm([[]]),
                 lambda: L.grad_norm([[1.0]]), lambda: L.qk_norm(x, x, x, x, x[0], x[0]), lambda: L.linear([torch.zeros(4, 8)] * 33, w * 33)):
        with pytest.raises(ValueError):
            call()


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """am_product_plan.h compiled for the host."""
    d = tmp_path_factory.mktemp("plans")
    (d / "plans.cpp").write_text(f'#include "{ROOT}/paper_2601_22442_amd/csrc/am_product_plan.h"\n' + r"""
extern "C" int plan(int bf16, int direct, uint64_t r, uint64_t m, uint64_t n, uint64_t k, uint32_t *out)
{
    double us;
    const am_host::ProductPlan p = am_host::product_plan(bf16, direct, r, m, n, k, &us);
    out[0] = p.tile; out[1] = p.stages; out[2] = p.splits; out[3] = p.split_k;
    return us > 0.;
}
extern "C" int pair(int bf16, int direct, uint64_t r, const uint64_t *a, const uint64_t *b, uint32_t *out)
{
    am_host::ProductPlan p, q;
    double us;
    if (!am_host::pair_plan(bf16, direct, r, {a[0], a[1], a[2]}, {b[0], b[1], b[2]}, &p, &q, &us)) return 0;
    out[0] = p.tile; out[1] = p.stages; out[2] = p.splits; out[3] = p.split_k;
    out[4] = q.tile; out[5] = q.stages; out[6] = q.splits; out[7] = q.split_k;
    return us > 0.;
}
extern "C" void columns(uint64_t r, uint64_t m, uint64_t n, uint32_t *out) { am_host::column_parts(r, m, n, out, out + 1); }
""")
    lib = d / "plans.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", "-o", str(lib), str(d / "plans.cpp")], check=True)
    so = C.CDLL(str(lib))
    so.plan.argtypes = [C.c_int, C.c_int] + [C.c_uint64] * 4 + [C.c_void_p]
    so.pair.argtypes = [C.c_int, C.c_int, C.c_uint64] + [C.c_void_p] * 3
    so.columns.argtypes = [C.c_uint64] * 3 + [C.c_void_p]
    return so


def test_every_split_of_a_product_has_work_and_together_they_cover_it(plans):
    import random
    rng = random.Random(1)
    out = (C.c_uint32 * 8)()
    for _ in range(3000):
        bf16, direct = rng.randint(0, 1), rng.randint(0, 1)
        step = 64 if bf16 else 32
        r, m, n, k = rng.randint(1, 32), *(int(2 ** rng.uniform(0, 17)) for _ in range(3))
        assert plans.plan(bf16, direct, r, m, n, k, out)
        tile, stages, splits, split_k = out[:4]
        assert (tile, stages) in {(256, 2), (128, 2), (64, 2), (64, 4)} and (bf16 or tile < 256) and (direct or stages == 2)
        assert split_k % step == 0 and (splits - 1) * split_k < k <= splits * split_k
        a, b = (C.c_uint64 * 3)(m, k, n), (C.c_uint64 * 3)(n, k, m)
        assert plans.pair(bf16, direct, r, a, b, out)
        assert out[0] == out[4] and out[1] == out[5] and out[2] == out[6] == 1 and out[3] >= n and out[7] >= m and (direct or out[1] == 2)
        plans.columns(r, m, n, out)
        assert (out[1] - 1) * out[0] < m <= out[1] * out[0] and out[1] <= 65535
