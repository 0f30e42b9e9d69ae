"""The mixer operators' host side on the CPU: the places of a launch's threads, and calls
that the binding and the C ABI take or refuse."""
from __future__ import annotations

import os
import subprocess

import pytest
import torch

import paper_2607_17419_amd as kata
from test_mixer_cpu import _conv_fwd


# ---- places of threads ----------------------------------------------------------------

PLACES = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "kata_index.hpp"
// argv: tokens, channels in groups of one, sequences; runs of 16 tokens
int main(int, char** argv) {
  const int T = atoi(argv[1]), groups = atoi(argv[2]), B = atoi(argv[3]), runs = (T + 15) / 16;
  const long long per = 1LL * groups * runs, all = per * B;
  long long bad = 0;
  const auto check = [&](long long id) {
    const kata::ConvPlace p = kata::conv_place(id, groups, runs);
    if (p.b < 0 || p.b >= B || p.run < 0 || p.run >= runs || p.group < 0 || p.group >= groups) ++bad;
    if ((1LL * p.b * runs + p.run) * groups + p.group != id) ++bad;
  };
  for (long long id = 0; id < all; id += 65537) check(id);
  for (int b = 0; b < B; ++b)
    for (long long at : {0LL, 1LL, groups - 1LL, 1LL * groups, per / 2, (1LL << 31) - 1, 1LL << 31, per - 1})
      if (at < per) check(b * per + at);
  printf("%lld\n", bad);
}
"""


def test_conv_places_of_sequences_past_2_31_threads(tmp_path):
    """The threads of a launch that the host's check admits, up to 2^32 - 512 of one sequence, have
    places inside the tensors, each its own: samples all over, and around 2^31."""
    src = tmp_path / "places.cpp"
    src.write_text(PLACES)
    csrc = os.path.join(os.path.dirname(kata.__file__), "csrc")
    exe = str(tmp_path / "places")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fsanitize=undefined", "-I", csrc, str(src), "-o", exe],
                   check=True)
    for T, D, B in ((1 << 20, 32769, 1), (32784, (1 << 20) - 1, 1), (16, 7, 3), (1 << 20, 32769, 2),
                    (1 << 16, (1 << 20) - 1, 1)):
        threads = (T + 15) // 16 * D * B
        sizes = dict(B=B, T=T, D=D, xb=T * D, xt=D, yb=T * D, yt=D)
        if threads > (1 << 32) - 512:
            assert _conv_fwd(**sizes) == 2
            continue
        out = subprocess.run([exe, str(T), str(D), str(B)], check=True, capture_output=True, text=True)
        assert out.stdout.strip() == "0" and not out.stderr, (T, D, B, out.stdout, out.stderr)


# ---- sources --------------------------------------------------------------------------

def test_mixer_operators_stand_in_a_source_of_their_own():
    """bench.py reports counted traffic for sources whose hash its record holds: a header of
    other operators in one of them would drop the record though its kernels are the same."""
    import bench
    from paper_2607_17419_amd import build
    assert "kata_mixer.hip" in build.SOURCES
    for name in {*bench.M1_SOURCES, *bench.LIN_SOURCES, "kata_fp32.hip"}:
        with open(os.path.join(os.path.dirname(kata.__file__), "csrc", name)) as f:
            text = f.read()
        for header in ("kata_conv.hpp", "kata_qknorm.hpp", "kata_ssm.hpp", "kata_rows.hpp", "kata_mixer"):
            assert header not in text, (name, header)


# ---- the binding ------------------------------------------------------------------------

def test_first_argument_by_name_or_missing():
    """A host tensor is refused as one, given by position or by name; none at all is a TypeError."""
    x, w = torch.zeros(2, 8, 16), torch.zeros(16, 4)
    for args, named in (((x,), dict(w=w)), ((), dict(x=x, w=w)), ((), dict(w=w, x=x))):
        with pytest.raises(ValueError, match="device tensors"):
            kata.conv_fwd(*args, **named)
    for call, name in ((kata.conv_step, "state"), (kata.conv_bwd, "x"), (kata.qk_norm_fwd, "q"),
                       (kata.qk_norm_bwd, "q"), (kata.ssm_fwd, "x"), (kata.ssm_step, "S"), (kata.ssm_bwd, "x")):
        with pytest.raises(ValueError, match="device tensors"):
            call(**{name: x})
        with pytest.raises(TypeError, match=name):
            call()
