"""The turns of the attention kernel's two issuing warps: whatever pieces a
block has and however its two warps run, no turn is given before the last one
has been taken (a barrier's parity tells two phases apart, not three), none is
missed, and none is taken early.  The program walks every interleaving of the
rules that the kernel itself is compiled with."""
import os
import subprocess

from paper_2608_13255_gb300 import build as gbuild

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "c", "attention_turns.cpp")


def test_every_interleaving_of_the_turns(tmp_path):
    exe = str(tmp_path / "turns")
    res = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-I", gbuild.CSRC, SRC, "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, "unsound for the pieces (goes of tile 0, of tile 1): " + res.stdout


def test_plans_keep_what_the_turns_rely_on():
    """In no piece of two tiles has tile 0 more key tiles than tile 1."""
    import numpy as np
    gbuild.build()
    from paper_2608_13255_gb300 import geocache as gc
    rng = np.random.default_rng(11)
    pairs = 0
    for _ in range(60):
        n = int(rng.integers(1, 5))
        q, k = ([int(x) for x in rng.integers(0, 900, n)] for _ in range(2))
        Hk = int(rng.choice([1, 2]))
        info, schedule = gc.plan_attention_host(q, k, Hk * int(rng.choice([1, 3, 8])), Hk, 128, bool(rng.integers(2)),
                                                int(rng.choice([1, 9, 152])))
        at = (info.n_ctas + 1 + 15) // 16 * 16
        for it in schedule.numpy()[at:at + 16 * info.n_items].reshape(-1, 16):
            n_tok, n_kv = it[6:8], it[8:10]
            assert n_kv[0] == 0 or n_tok[1] == 0 or n_kv[0] <= n_kv[1]
            assert n_kv[1] == 0 or n_tok[1] > 0
            pairs += bool(n_kv.all())
    assert pairs > 100
