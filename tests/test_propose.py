"""Pose corrections of the proposals (CPU): a correction leads to its target."""
import numpy as np

from paper_2210_10108_amd import propose, synth


def test_corrections_lead_to_their_target():
    w = synth.WORKLOADS["tiny32"]
    gt = synth.ground_truth_pose(w, 0)
    poses = synth.perturb_poses(gt, 50, 60.0, 0.4, 1).astype(np.float64)
    c = propose.corrections(poses, np.broadcast_to(gt, poses.shape))
    moved = propose.corrected(poses, c)
    assert np.allclose(moved, gt, atol=1e-6)
    r, t = propose.errors(moved, gt)
    assert r < 1e-3 and t < 1e-6
    assert propose.errors(poses, gt)[0] > 1.0
    assert np.allclose(propose.corrected(poses, np.zeros((50, 6))), poses)
