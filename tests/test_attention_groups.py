"""Large groups of query heads on long sequences: the row of a pair (row, head of the group) is right for every group and every number of rows, on the host for all of them
and on the GPU where pairs are many."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_1902_01064_amd import attention
from test_layers import DEV, U, close, holes, rounded

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"), reason="needs g++ and the HIP headers")
def test_quotients_of_all_groups_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "attention_quotient_driver")
    csrc = os.path.join(ROOT, "paper_1902_01064_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
           "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "attention_quotient_driver.cpp"), os.path.join(csrc, "hop_attention.cpp"), os.path.join(csrc, "hop_sim.cpp"),
           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    subprocess.run(cmd, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0")
    out = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    told = dict(p.split("=") for p in out.stdout.split()[1:])
    assert out.stdout.startswith("ok ") and int(told["launches"]) == 4 * attention.HOP_MAX_HEADS and int(told["looked"]) > 10 ** 7, out.stdout


def of_a_head(q, k, v, causal, scale):
    """(o, lse) of one head, all rows at once."""
    nq, nk = len(q), len(k)
    s = np.where(oa.seen(nq, nk, causal), scale * q @ k.T, -np.inf)
    top = np.where(np.isfinite(s.max(1)), s.max(1), 0.0)[:, None]
    e = np.exp(s - top)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.where(total > 0, e @ v / np.where(total > 0, total, 1.0), 0.0), (top + np.log(total))[:, 0]


# 1023 heads of one group from row 4120 on, 1016 from 4227 on: where an inverse of 32 bits gave the next row.  Rows further apart than their columns; queries that see nothing
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,nq,nk,causal", [("bf16", 1023, 4200, 24, False), ("f32", 1016, 4300, 4290, True), ("bf16", 1000, 6200, 7, True)])
def test_many_heads_on_many_rows(dtype, hq, nq, nk, causal):
    D, first = 4, 4090 if nq < 6000 else 6080
    r = np.random.default_rng(hq)
    q, q64 = rounded(r.standard_normal((nq, hq * D)), dtype)
    k, k64 = rounded(r.standard_normal((nk, D)), dtype)
    v, v64 = rounded(r.standard_normal((nk, D)), dtype)
    do, do64 = rounded(r.standard_normal((nq, hq * D)), dtype)
    o, unharmed = holes(nq, hq * D, dtype, 8, 0)
    lses, fine = holes(hq, nq, "f32", 0, 4)
    how = dict(q_heads=hq, k_heads=1, causal=causal)
    attention.attention(q, k, v, out=o, out_lse=lses, **how)
    assert unharmed() and fine()
    # as a statement the last rows of a few heads are a call of their own: where causal they see the same keys
    heads = [0, 1, hq // 2, hq - 2, hq - 1]
    pick = np.concatenate([np.arange(h * D, h * D + D) for h in heads])
    Q, DO, n = q64[first:, pick], do64[first:, pick], nq - first
    rest = (len(heads), 1, [0, n], [0, nk], causal, D ** -0.5)
    want, want_lse = np.empty_like(Q), np.empty((len(heads), n))
    for i in range(len(heads)):
        want[:, i * D:i * D + D], want_lse[i] = of_a_head(Q[:, i * D:i * D + D], k64, v64, causal, D ** -0.5)
    got, got_lse = o[first:][:, torch.from_numpy(pick).to(DEV)], lses[torch.tensor(heads, device=DEV)][:, first:]
    rounding = 2.0 ** -8 if dtype == "bf16" else 0.0
    bounds = oa.attention_bounds(DO, want, want_lse, Q, k64, v64, *rest, U, rounding)
    close(got, want, bounds[0], dtype, "o")
    see = np.isfinite(want_lse)
    assert np.array_equal(np.isfinite(got_lse.double().cpu().numpy()), see)
    close(torch.where(torch.from_numpy(see).to(DEV), got_lse, 0.0), np.where(see, want_lse, 0.0), np.where(see, bounds[1], 0.0), "f32", "lse")
    dq, unharmed = holes(nq, hq * D, dtype, 8, 0)
    dq, dk, dv = attention.attention_grad(do, o, lses.contiguous(), q, k, v, dq=dq, **how)
    assert unharmed()
    o64, lse64 = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    bounds = oa.attention_bounds(DO, o64, lse64, Q, k64, v64, *rest, U, rounding, want)
    close(dq[first:][:, torch.from_numpy(pick).to(DEV)], oa.attention_grad(DO, o64, lse64, Q, k64, v64, *rest)[0], bounds[2], dtype, "dq")
    # the keys' gradients are sums over all pairs
    all_o, all_lse = o.double().cpu().numpy(), lses.double().cpu().numpy()
    rest = (hq, 1, [0, nq], [0, nk], causal, D ** -0.5)
    if nk < 100:
        exact = np.concatenate([of_a_head(q64[:, h * D:h * D + D], k64, v64, causal, D ** -0.5)[0] for h in range(hq)], 1)
        wants = oa.attention_grad(do64, all_o, all_lse, q64, k64, v64, *rest)
        bounds = oa.attention_bounds(do64, all_o, all_lse, q64, k64, v64, *rest, U, rounding, exact)
        close(dk, wants[1], bounds[3], dtype, "dk")
        close(dv, wants[2], bounds[4], dtype, "dv")
