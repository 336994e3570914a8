"""The pins of the scoring and feed-forward oracles must notice a mistake: each plausible slip is planted in a copy of the
oracle's source (on the CPU, never in the CUDA path) and the pins are run against that copy in a child process; they have to
fail."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCORE, FFN = "vt_score_oracle.py", "vt_ffn_oracle.py"

# name: (file, text in the oracle, the slip)
MUTANTS = {
    "negative_token_scored": (SCORE, "return (tokens >= 0) & (tokens < V)", "return tokens < V"),
    "token_past_the_end_scored": (SCORE, "return (tokens >= 0) & (tokens < V)", "return (tokens >= 0) & (tokens <= V)"),
    "scale_forgotten": (SCORE, "z = scale * (h @ W.T)", "z = h @ W.T"),
    "maximum_counted_twice": (SCORE, "rest[np.arange(len(z)), z.argmax(1)] = 0.0", "rest[np.arange(len(z)), z.argmax(1)] = 1.0"),
    "lse_without_maximum": (SCORE, "lse = mx[:, 0] + log_s", "lse = log_s"),
    "entropy_sign": (SCORE, "entropy = -(p * ", "entropy = (p * "),
    "worst_instead_of_best": (SCORE, "np.argsort(-z, axis=1, kind=\"stable\")", "np.argsort(z, axis=1, kind=\"stable\")"),
    "ties_to_higher_id": (SCORE, "np.argsort(-z, axis=1, kind=\"stable\")[:, :k]", "(z.shape[1] - 1 - np.argsort(-z[:, ::-1], axis=1, kind=\"stable\"))[:, :k]"),
    "alternatives_as_logits": (SCORE, "np.take_along_axis(logp, order, 1)", "np.take_along_axis(z, order, 1)"),
    "gradient_without_scale": (SCORE, "G[keep] = scale * (", "G[keep] = 1.0 * ("),
    "gradient_sign": (SCORE, "(gl * (hot - p) - ge", "(gl * (p - hot) - ge"),
    "entropy_gradient_without_entropy": (SCORE, "- ge * p * (logp + entropy[:, None]))", "- ge * p * logp)"),
    "entropy_gradient_sign": (SCORE, "- ge * p * (logp + entropy[:, None]))", "+ ge * p * (logp + entropy[:, None]))"),
    "unscored_rows_reach_the_weights": (SCORE, "G[keep].T @ h[keep]", "G.T @ h"),
    "silu_without_gate": (FFN, "return g / (1.0 + np.exp(-g))", "return 1.0 / (1.0 + np.exp(-g))"),
    "silu_slope_term_lost": (FFN, "return s + g * s * (1.0 - s)", "return s"),
    "gelu_cubic_factor": (FFN, "0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)))", "0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.44715 * g ** 3)))"),
    "gelu_slope_factor": (FFN, "(1.0 + 3 * 0.044715 * g * g)", "(1.0 + 0.044715 * g * g)"),
    "gate_and_up_swapped": (FFN, "g, u = x @ Wg.T, x @ Wu.T", "u, g = x @ Wg.T, x @ Wu.T"),
    "activation_on_the_product": (FFN, "a = act(g, kind) * u", "a = act(g * u, kind)"),
    "input_gradient_of_one_branch": (FFN, "dg @ Wg + du @ Wu", "dg @ Wg"),
    "down_gradient_from_gate": (FFN, "dy.T @ f[\"a\"]", "dy.T @ f[\"g\"]"),
    "branch_gradients_swapped": (FFN, "du, dg = da", "dg, du = da"),
}

CHILD = """
import sys
sys.path.insert(0, {tmp!r})
import oracle, oracle.vt_score_oracle, oracle.vt_ffn_oracle
assert oracle.__file__.startswith({tmp!r}), oracle.__file__
sys.path.insert(1, {root!r})
import pytest
sys.exit(pytest.main([{pins!r}, "-x", "-q", "-p", "no:cacheprovider"]))
"""


def run_pins(tmp):
    code = CHILD.format(tmp=str(tmp), root=ROOT, pins=os.path.join(ROOT, "tests", "test_score_ffn_oracle_pins.py"))
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)


def copy_oracle(tmp_path):
    dst = tmp_path / "oracle"
    dst.mkdir()
    for f in os.listdir(os.path.join(ROOT, "oracle")):
        if f.endswith(".py"):
            shutil.copy(os.path.join(ROOT, "oracle", f), dst / f)
    return dst


@pytest.mark.parametrize("name", sorted(MUTANTS))
def test_pins_catch_planted_mistake(name, tmp_path):
    fname, old, new = MUTANTS[name]
    dst = copy_oracle(tmp_path)
    text = (dst / fname).read_text()
    assert text.count(old) == 1, f"mutation site for {name} not found exactly once"
    (dst / fname).write_text(text.replace(old, new))
    r = run_pins(tmp_path)
    assert r.returncode == 1 and "failed" in r.stdout, f"the pins passed with the mistake '{name}' planted:\n{r.stdout[-1500:]}"


def test_unmodified_copy_passes(tmp_path):
    copy_oracle(tmp_path)
    r = run_pins(tmp_path)
    assert r.returncode == 0, r.stdout[-1500:] + r.stderr[-800:]
