"""A group-normed student that learns from a teacher's kept logits, one iteration of calls as a training program makes them: teacher
logits -> logits_topk; convolution -> group norm + ReLU -> average pooling -> fully connected -> distill_ce, backward through all of them,
and the update.  Against the oracle's functions chained in float64 on the same inputs."""
import numpy as np
import pytest
import torch

from oracle import ops as orc
from paper_1711_04325_amd import binding as rn
from paper_1711_04325_amd import synth
from tests.gpu_util import DEV, assert_close, empty, nchw, nhwc, to_dev, ws_bytes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,c,h,k,groups,classes,t", [(4, 32, 14, 64, 32, 1000, 10), (1, 64, 9, 128, 8, 37, 5)])
def test_student_iteration(n, c, h, k, groups, classes, t):
    g = synth.rng(9)
    x, w = synth.normal(g, (n, c, h, h)), synth.he_normal(g, (k, c, 3, 3))
    gamma, beta = synth.normal(g, k, 0.1, 1.0), synth.normal(g, k, 0.1)
    fw, fb = synth.normal(g, (classes, k), 0.2), synth.normal(g, classes, 0.1)
    teacher, labels = synth.normal(g, (n, classes), 2.0), g.integers(0, classes, n).astype(np.int32)
    alpha, tau, scale, eps = 0.5, 4.0, 1.0 / n, 1e-5

    d = rn.conv_desc(n, c, h, h, k, 3, 3, 1, 1)
    dx, dw, dgam, dbet, dfw = nhwc(x), nhwc(w), to_dev(gamma), to_dev(beta), to_dev(fw)
    ws = ws_bytes(max(rn.rn50_gn_workspace_bytes(n, k, h, h, groups), rn.rn50_topk_workspace_bytes(n, classes, t),
                      rn.rn50_distill_workspace_bytes(n, classes, t), *[rn.rn50_conv_workspace_bytes(d, op) for op in (rn.OP_FWD, rn.OP_BWD_WEIGHT)]))
    val, idx = empty(n, t), empty(n, t, dtype=torch.int32)
    rn.logits_topk(n, classes, t, to_dev(teacher), classes, val, idx, ws)
    conv, y, mean, inv = empty(n, h, h, k), empty(n, h, h, k), empty(n, groups), empty(n, groups)
    rn.conv2d_fwd(d, dx, dw, conv, ws)
    rn.gn_fwd(n, k, h, h, groups, conv, dgam, dbet, eps, None, rn.ACT_RELU, y, mean, inv, ws)
    f, logits, loss, dlogits = empty(n, k), empty(n, classes), empty(3), empty(n, classes)
    rn.avgpool_fwd(n, k, h, h, y, f)
    rn.fc_fwd(n, k, classes, f, dfw, to_dev(fb), logits)
    rn.distill_ce(n, classes, t, logits, classes, to_dev(labels, torch.int32), idx, val, alpha, tau, scale, loss, dlogits, classes, ws)
    df, dfw_, dfb, dy, dconv, dg, db, dwt = empty(n, k), empty(classes, k), empty(classes), empty(n, h, h, k), empty(n, h, h, k), empty(k), empty(k), empty(k, 3, 3, c)
    rn.fc_bwd(n, k, classes, f, dfw, dlogits, df, dfw_, dfb)
    rn.avgpool_bwd(n, k, h, h, df, dy)
    rn.gn_bwd(n, k, h, h, groups, conv, dy, None, None, dgam, dbet, mean, inv, rn.ACT_RELU, dconv, None, dg, db, ws)
    rn.conv2d_bwd_weight(d, dx, dconv, dwt, ws)
    theta, delta, m = dw.clone(), torch.zeros_like(dw), torch.zeros_like(dw)
    rn.opt_update(theta.numel(), theta, delta, m, dwt, None, None, rn.opt_hparams(0.1, 0.9, 0.99, 1e-8, 0.5, 1e-4))
    torch.cuda.synchronize()

    rval, ridx = orc.topk(teacher, t)
    np.testing.assert_array_equal(idx.cpu().numpy(), ridx)
    rconv = orc.conv2d_fwd(x, w, 1, 1)
    # a ReLU decision within rounding of the corner may go either way: the oracle takes the device's where it is that near
    pre, rmean, rinv = orc.gn_fwd(rconv, groups, gamma, beta, eps)
    near = np.abs(pre) < 1e-5
    on = np.where(near, nchw(y) > 0, pre > 0)
    ry = pre * on
    rlogits = orc.fc_fwd(orc.avgpool_fwd(ry), fw, fb)
    rloss, rdl = orc.distill_ce(rlogits, labels, ridx, rval, alpha, tau, scale)
    rdf, rdfw, rdfb = orc.fc_bwd(orc.avgpool_fwd(ry), fw, rdl)
    rdconv, _, rdg, rdb = orc.gn_bwd(rconv, orc.avgpool_bwd(rdf, h, h) * on, groups, gamma, beta, rmean, rinv)
    rdw = orc.conv2d_bwd_weight(x, rdconv, 3, 3, 1, 1)
    # every call alone is good to 1e-6 and the chain to some times that: the library's bar of 1e-4 leaves room for the filter gradient,
    # a sum of many gradients that nearly cancel (the group's means are taken out of dconv)
    for what, got, ref, bar in (("conv", nchw(conv), rconv, 2e-6), ("y", nchw(y), ry, 4e-6), ("logits", logits.cpu(), rlogits, 1e-5), ("loss", loss.cpu(), rloss, 1e-5),
                                ("dlogits", dlogits.cpu(), rdl, 2e-5), ("dfc", dfw_.cpu(), rdfw, 4e-5), ("dconv", nchw(dconv), rdconv, 1e-4),
                                ("dgamma", dg.cpu(), rdg, 1e-4), ("dbeta", db.cpu(), rdb, 1e-4), ("dw", nchw(dwt), rdw, 1e-4)):
        assert_close(np.asarray(got), ref, bar, what)
    gw = nchw(dwt)
    rth, _, _ = orc.opt_update(w.ravel(), 0 * w.ravel(), 0 * w.ravel(), gw.ravel(), 0.1, 0.9, 0.99, 1e-8, 0.5, 1e-4)
    assert_close(nchw(theta).ravel(), rth, 1e-6, "theta")
