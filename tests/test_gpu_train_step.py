"""The example that trains a policy on BLEU with every loss: it learns."""
import pytest

pytestmark = pytest.mark.gpu


def test_policy_learns_from_bleu():
    from paper_2510_05485_amd.example import train_step
    lines = []
    means = train_step.run(say=lines.append)
    assert len(means) == 4 and len(lines) == 5
    # the teacher is right at seven positions of ten; samples that are right everywhere have a BLEU of 1
    assert means[0] < 0.1 and means[1] > means[0] + 0.1
    assert means[3] > means[1] + 0.1
