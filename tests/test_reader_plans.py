"""Which form of the kernels a call of the reader's attention gets: the shapes of the GPU tests reach every one of them.  The rules are
compiled into assertions; nothing runs."""
import os
import shutil
import subprocess

import pytest

from test_build_properties import CSRC, HIPCC, ROOT
from test_gpu_reader_forms import CACHED, CROSS

HEAD = """
constexpr plaid_attention call(int n, int heads, int kv_heads, int dim, long long queries, long long keys, bool bias)
{
    plaid_attention a = {};
    a.n = n, a.heads = heads, a.kv_heads = kv_heads, a.head_dim = dim, a.num_queries = queries, a.num_keys = keys;
    a.key_bias = bias ? &a : nullptr;
    return a;
}
constexpr Plan forward(plaid_attention a, bool bias)
{
    return plan_forward(a, bias ? PLAID_SOURCE_BIAS : PLAID_SOURCE_DENSE, a.num_keys, a.num_keys, ceil_div(a.num_keys, a.n));
}
"""


def _flag(x):
    return "true" if x else "false"


def _claims():
    for name, (q, k, heads, kv_heads, dim, waves, parts, k_waves, q_parts, k_parts) in CROSS.items():
        for bias in (False, True):
            a = f"call({len(q)}, {heads}, {kv_heads}, {dim}, {sum(q)}, {sum(k)}, false)"
            f = f"forward({a}, {_flag(bias)})"
            if waves:
                yield f"!{f}.few && {f}.waves == {waves} && ({f}.splits > 1) == {_flag(parts)}", name
            yield f"plan_backward({a}).k_waves == {k_waves} && (plan_backward({a}).q_splits > 1) == {_flag(q_parts)}", name
            yield f"(plan_backward({a}).k_splits > 1) == {_flag(k_parts)}", name
    for name, (q, k, heads, kv_heads, dim, bs, width, waves, parts) in CACHED.items():
        assert width * bs >= max(max(q), max(k))
        f = f"plan_cached(call({len(q)}, {heads}, {kv_heads}, {dim}, {sum(q)}, 0, false), {width}, {bs})"
        yield f"!{f}.few && {f}.waves == {waves} && ({f}.splits > 1) == {_flag(parts)}", name


def test_the_shapes_are_of_every_form():
    assert {(c[4], c[5], c[6]) for c in CROSS.values()} >= {(d, w, p) for d in (64, 128) for w in (4, 8) for p in (False, True)}
    assert {(c[4], c[7], c[8]) for c in CACHED.values()} == {(d, w, p) for d in (64, 128) for w in (4, 8) for p in (False, True)}
    assert {(c[4], c[7]) for c in CROSS.values()} == {(64, 4), (128, 4), (128, 8)}
    assert {(c[4], c[8]) for c in CROSS.values()} == {(c[4], c[9]) for c in CROSS.values()} == {(d, p) for d in (64, 128) for p in (False, True)}


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not installed")
def test_the_shapes_get_their_forms(tmp_path):
    unit = tmp_path / "plans.hip"
    unit.write_text('#include "reader_api.hip"\n' + HEAD + "".join(f'static_assert({c}, "{name}");\n' for c, name in _claims()))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "--cuda-host-only",
                        "-fsyntax-only", str(unit)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
