"""The token operators' kernels on the host, in lock step (tests/emu): the GPU tests' own functions on host memory whose
neighbouring pages cannot be touched, so that an access outside a buffer ends the run."""
import ctypes
import os
import subprocess

import pytest
import torch

import emu_build
import paper_1805_04170_amd.binding as binding
import test_gpu_tokens as g

pytestmark = pytest.mark.skipif(emu_build.CLANG is None, reason="no host clang++ for the emulation build")
UNITS = ["emu_lib_embed.cpp", "emu_lib_policy.cpp", "emu_lib_pack8.cpp"]


@pytest.fixture(scope="module")
def emulated_tokens(emulators, tmp_path_factory):
    """the token operators built for the host, linked with the emulated library"""
    out = str(tmp_path_factory.mktemp("emu_tokens"))
    jobs = []
    for u in UNITS:
        o = os.path.join(out, u + ".o")
        cmd = [emu_build.CLANG] + emu_build.BASE + emu_build.LIBRARY_FLAGS + emu_build.INCLUDES + ["-c", os.path.join(emu_build.EMU, u), "-o", o]
        jobs.append((o, subprocess.Popen(cmd, stderr=subprocess.PIPE, text=True)))
    for _, p in jobs:
        err = p.communicate()[1]
        assert p.returncode == 0, err[-4000:]
    base = emulators.get("library")
    so = os.path.join(out, "libtokens_emulated.so")
    subprocess.run([emu_build.CLANG, "-shared", "-o", so] + [o for o, _ in jobs] + [base, "-Wl,-rpath," + os.path.dirname(base)], check=True)
    return so


@pytest.fixture(autouse=True, params=["end", "front"])
def on_host(request, emulated_tokens, monkeypatch):
    monkeypatch.setattr(binding, "LIB_PATH", emulated_tokens)
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_stream", lambda stream: ctypes.c_void_p(0))
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a, **k: None)
    monkeypatch.setattr(g, "DEV", "cpu")
    monkeypatch.setattr(g, "GUARD", request.param)


@pytest.mark.parametrize("T,V,D,dt", [(1, 1, 1, "bf16"), (7, 40, 33, "bf16"), (65, 130, 20, "f32"), (70, 9, 250, "bf16")])
def test_embedding(T, V, D, dt):
    g.run_embed(T, V, D, dt, seed=T)


@pytest.mark.parametrize("T,V,D,dt,tW,tX", [(40, 20, 600, "bf16", "", ""), (45, 3, 1031, "f32", "", ""), (40, 8, 1200, "bf16", "C", "R"), (36, 6, 532, "f32", "rC", "CR")])
def test_embedding_of_wide_rows(T, V, D, dt, tW, tX):
    g.run_embed(T, V, D, dt, tW, tX, seed=D)


@pytest.mark.parametrize("tW,tX,dt,D", [("R", "C", "bf16", 64), ("RC", "CR", "f32", 24), ("rC", "Cr", "bf16", 40), ("RCr", "CCC", "bf16", 40)])
def test_embedding_tiled(tW, tX, dt, D):
    g.run_embed(40, 48, D, dt, tW, tX, "i32", seed=len(tW) + D)


@pytest.mark.parametrize("what", ["one", "none", "two", "huge", "long_runs"])
def test_embedding_token_patterns(what):
    g.test_embedding_token_patterns(what)


def test_embedding_without_tokens():
    g.test_embedding_without_tokens_is_a_gradient_of_zeros()


@pytest.mark.parametrize("T,V,dt,masked", [(1, 1, "f32", False), (3, 7, "bf16", False), (16, 333, "bf16", True), (14, 1031, "f32", True), (2, 8200, "bf16", False)])
def test_policy_loss(T, V, dt, masked):
    g.run_policy(T, V, dt, seed=T + V, masked=masked, scale=1.3)


@pytest.mark.parametrize("tX,tG,dt,V", [("C", "R", "bf16", 512), ("CC", "RC", "f32", 328), ("CR", "rr", "bf16", 104), ("rC", "Cr", "f32", 36), ("CCC", "RRC", "bf16", 104)])
def test_policy_loss_tiled(tX, tG, dt, V):
    g.run_policy(16, V, dt, tX, tG, "i32", seed=len(tX), masked=True, scale=0.7)


@pytest.mark.parametrize("tX,tG,dt,V", [("", "", "bf16", 17000), ("C", "R", "bf16", 1100), ("RC", "CC", "f32", 2084), ("CCCCC", "RRCCC", "f32", 17600)])
def test_policy_loss_of_long_rows(tX, tG, dt, V):
    g.run_policy(4, V, dt, tX, tG, "i32", seed=V, masked=True)


def test_policy_special_rows():
    g.test_policy_rows_that_count_show_their_nan()
    g.test_policy_loss_of_no_tokens_is_zero()
    g.test_policy_loss_without_gradient_and_log_probabilities_alone()


@pytest.mark.parametrize("mask", [-5e9, -1e10, -1e30, None])
@pytest.mark.parametrize("V,dt,tX,tG,scale", [(40, "f32", "", "", 1.0), (600, "bf16", "", "", 0.5), (9, "f32", "", "", 1e-30), (24, "bf16", "CC", "CC", 2.0),
                                              (600, "f32", "CCC", "RRr", 4.0)])
def test_policy_loss_of_large_finite_masks(V, dt, tX, tG, scale, mask):
    g.run_policy_of_large_logits(V, dt, mask, scale, tX, tG)


def test_policy_loss_of_large_finite_masks_in_cut_rows():
    g.run_policy_of_large_logits(17000, "bf16", -1e10, 1.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_policy_loss_of_large_logits_a_few_steps_apart(dt):
    g.test_policy_loss_of_large_logits_a_few_steps_apart(dt)


def test_policy_loss_at_the_ends_of_the_scale():
    g.test_policy_loss_at_the_ends_of_the_scale()


@pytest.mark.parametrize("T,V,dt,tX", [(1, 1, "f32", ""), (1, 4099, "bf16", ""), (8, 640, "bf16", "CC"), (6, 36, "bf16", "CR")])
def test_token_logp(T, V, dt, tX):
    g.run_logp(T, V, dt, tX, scale=0.8)


@pytest.mark.parametrize("T,scale", [(40, float("inf")), (40, -2.0), (300, float("inf")), (300, -2.0)])
def test_table_gradient_rows_without_tokens_are_zeros(T, scale):
    g.test_table_gradient_rows_without_tokens_are_zeros(T, scale)


@pytest.mark.parametrize("T,V,D", [(0, 6, 5), (5, 0, 5), (0, 0, 5), (5, 6, 0)])
def test_tensors_without_values(T, V, D):
    g.test_embedding_of_tensors_without_values(T, V, D)
    g.test_policy_loss_of_tensors_without_values(T, V if T == 0 else 0, torch.bfloat16)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pack8(dt):
    for rows, cols in [(1, 1), (3, 31), (5, 33), (2, 200), (9, 47)]:
        g.run_pack(rows, cols, dt, seed=cols)
    for t in ["R", "C", "RC", "CCr"]:
        g.run_pack(16, 88, dt, t)
    g.test_pack8_values_at_the_edges(dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [64, 40])
def test_unpack8_takes_any_step(cols, dt):
    g.test_unpack8_takes_any_step(cols, dt)


@pytest.mark.parametrize("t", [("", "", "", "", ""), ("CC", "RR", "CR", "RC", "Cr")])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_packed_backward(t, dt):
    g.run_packed_backward(16, 64, 72, dt, True, *t)


def test_packed_backward_gates_out_what_is_not_a_number():
    g.test_packed_backward_gates_out_what_is_not_a_number()
