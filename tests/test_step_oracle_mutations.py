"""The pins of the decode-step oracle must notice a mistake: each plausible slip is planted in a copy of the oracle's source (on the CPU,
never in the CUDA path) and the pins are run against that copy in a child process; they have to fail."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILE = "vt_step_oracle.py"
PINS = [os.path.join(ROOT, "tests", f) for f in ("test_step_oracle_pins.py", "test_step_oracle_more_pins.py")]

# name: (text in the oracle, the slip)
MUTANTS = {
    "frequencies_of_whole_pairs": ("f = base ** (-2.0 * i / rot)", "f = base ** (-1.0 * i / rot)"),
    "linear_multiplied": ("            w = f / factor\n        elif", "            w = f * factor\n        elif"),
    "base_exponent": ("factor ** (rot / (rot - 2.0))", "factor ** (rot / (rot + 2.0))"),
    "base_exponent_lost": ("factor ** (rot / (rot - 2.0))", "factor"),
    "wavelength_without_whole_turn": ("turns = original_len * f / (2 * math.pi)", "turns = original_len * f"),
    "wavelength_sides_swapped": ("w = f * s + f / factor * (1 - s)", "w = f * (1 - s) + f / factor * s"),
    "wavelength_range": ("s = min(max((turns - low) / (high - low), 0.0), 1.0)", "s = min(max((turns - low) / high, 0.0), 1.0)"),
    "ramp_sides_swapped": ("w = f * (1 - s) + f / factor * s", "w = f * s + f / factor * (1 - s)"),
    "ramp_ends_swapped": ("max(math.floor(pair_that_makes(high)), 0), min(math.ceil(pair_that_makes(low)), rot - 1)",
                          "max(math.floor(pair_that_makes(low)), 0), min(math.ceil(pair_that_makes(high)), rot - 1)"),
    "ramp_pair_of_elements": ("(2 * math.log(base))", "math.log(base)"),
    "ramp_not_rounded": ("max(math.floor(pair_that_makes(high)), 0)", "max(pair_that_makes(high), 0)"),
    "ramp_default_of_wavelength": ("high = 32.0 if scaling == \"ramp\" else 4.0", "high = 4.0"),
    "turned_the_other_way": ("x[n][:, a] * c - x[n][:, b] * s", "x[n][:, a] * c + x[n][:, b] * s"),
    "inverse_forgotten": ("s = -s", "s = s"),
    "amplitude_on_one_part": ("c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)", "c, s = amplitude * np.cos(angle), np.sin(angle)"),
    "pairs_always_in_halves": ("a = np.arange(half) * 2 if interleaved else np.arange(half)", "a = np.arange(half)"),
    "partner_next_to_it": ("b = a + 1 if interleaved else a + half", "b = a + 1"),
    "own_bit_lost": ("at, d = t, 0\n            while True:\n", "at, d = max(parents[cu[b] + t], 0), 0\n            while True:\n"),
    "bit_of_the_wrong_word": ("mask[cu[b] + t, at // 32] |= 1 << (at % 32)", "mask[cu[b] + t, 0] |= 1 << (at % 32)"),
    "parent_that_comes_later": ("if not 0 <= up < at:", "if not 0 <= up < len(parents) or up == at or d > 40:"),
    "depth_from_one": ("at, d = t, 0\n", "at, d = t, 1\n"),
    "scale_forgotten": ("x = scale * (kb[sees, kh] @ q[row, h])", "x = kb[sees, kh] @ q[row, h]"),
    "weights_not_normalised": ("wgt = e / e.sum()", "wgt = e"),
    "lse_without_maximum": ("lse[row, h] = top + math.log(e.sum())", "lse[row, h] = math.log(e.sum())"),
    "chain_does_not_see_itself": ("sees[i] = u <= t if mask is None", "sees[i] = u < t if mask is None"),
    "mask_of_another_row": ("int(mask[row, u // 32])", "int(mask[int(cu[b]), u // 32])"),
    "earlier_positions_lost": ("sees = at < L\n", "sees = at < 0\n"),
    "pages_in_order": ("ids = table[b, at // page]", "ids = at // page"),
    "heads_dealt_out": ("kh = h // (Hq // heads)", "kh = h % heads"),
    "empty_row_of_zero_lse": ("out[row, h], absolute[row, h], lse[row, h] = 0.0, 0.0, -np.inf", "out[row, h], absolute[row, h], lse[row, h] = 0.0, 0.0, 0.0"),
    "what_is_left_not_normalised": ("float(u_accept[row + c]) * qc * Z < left[y]", "float(u_accept[row + c]) * qc < left[y]"),
    "accepted_without_q": ("float(u_accept[row + c]) * qc * Z < left[y]", "float(u_accept[row + c]) * Z < left[y]"),
    "rejected_child_stays": ("                    left[y] = 0.0\n", "                    left[y] = left[y]\n"),
    "rejections_not_counted": ("                    S += Z\n", "                    S = 1.0\n"),
    "left_of_another_row": ("left = np.maximum(p - S * q, 0.0)", "left = np.maximum(left - q, 0.0)"),
    "children_of_the_root_alone": ("if not fits(c) or parents[row + c] != x:", "if not fits(c) or parents[row + c] != 0:"),
    "draft_index_unchecked": ("return draft_probs is None or 0 <= draft_ids[row + c] < draft_probs.shape[1]", "return True"),
    "draft_map_forgotten": ("to = i if d2t is None else int(d2t[i])", "to = i"),
    "sampled_from_the_whole_row": ("target, y, cum = max(float(u_sample[b]), 0.0) * math.fsum(left), -1, 0.0", "left = p\n        target, y, cum = max(float(u_sample[b]), 0.0) * math.fsum(left), -1, 0.0"),
    "sampled_one_early": ("if cum > target:", "if cum >= target * 0.9:"),
    "following_token_of_the_next_place": ("out[b, len(taken)] = y", "out[b, -1] = y"),
}

CHILD = """
import sys
sys.path.insert(0, {tmp!r})
import oracle, oracle.vt_step_oracle
assert oracle.__file__.startswith({tmp!r}), oracle.__file__
sys.path.insert(1, {root!r})
import pytest
sys.exit(pytest.main({pins!r} + ["-x", "-q", "-p", "no:cacheprovider"]))
"""


def run_pins(tmp):
    code = CHILD.format(tmp=str(tmp), root=ROOT, pins=PINS)
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600,
                          env={**os.environ, "PYTEST_DISABLE_PLUGIN_AUTOLOAD": "1"})


def copy_oracle(tmp_path):
    dst = tmp_path / "oracle"
    dst.mkdir()
    for f in os.listdir(os.path.join(ROOT, "oracle")):
        if f.endswith(".py"):
            shutil.copy(os.path.join(ROOT, "oracle", f), dst / f)
    return dst


@pytest.mark.parametrize("name", sorted(MUTANTS))
def test_pins_catch_planted_mistake(name, tmp_path):
    old, new = MUTANTS[name]
    dst = copy_oracle(tmp_path)
    text = (dst / FILE).read_text()
    assert text.count(old) == 1, f"mutation site for {name} not found exactly once"
    (dst / FILE).write_text(text.replace(old, new))
    r = run_pins(tmp_path)
    assert r.returncode == 1 and "failed" in r.stdout, f"the pins passed with the mistake '{name}' planted:\n{r.stdout[-1500:]}"


def test_unmodified_copy_passes(tmp_path):
    copy_oracle(tmp_path)
    r = run_pins(tmp_path)
    assert r.returncode == 0, r.stdout[-1500:] + r.stderr[-800:]
