// What lists of tensors ask of the HIP runtime, on the stand-in for it (fake_hip.h).
#include "fake_hip.h"
#include "ptchunk.h"

extern "C" hipError_t hipSetDevice(int d) {
  fake::device = d;
  fake::note(d ? "device 1" : "device 0");
  return hipSuccess;
}

#define EXPECT(c) do { if (!(c)) { fprintf(stderr, "line %d: %s\n%s", __LINE__, #c, fake::text().c_str()); return 1; } } while (0)

// A list belongs to the device that was current when it was made: that one's work is waited for before its memory goes, whichever is current then.
static int destroyed_from_another_device() {
  for (int own = 0; own < 2; ++own)
    for (int current = 0; current < 2; ++current) {
      fake::device = own;
      pt_tensor t = {};
      float* a = nullptr;
      EXPECT(hipMalloc((void**)&a, 4096) == hipSuccess);
      t.grad = a; t.master = a + 64; t.m = a + 128; t.v = a + 192; t.elems = 10;
      pt_tensors* l = nullptr;
      EXPECT(pt_tensors_create(&l, PT_BF16, &t, 1, 32, nullptr, 0) == PT_OK);
      const size_t held = fake::memory.size();
      fake::device = current;
      const size_t from = fake::ops.size();
      EXPECT(pt_tensors_destroy(l) == PT_OK);
      EXPECT(fake::memory.size() == held - 1);
      EXPECT(fake::device == current);                       // as the caller left it
      int at = current;
      bool waited = false;
      for (size_t i = from; i < fake::ops.size(); ++i) {
        const std::string& what = fake::ops[i].what;
        if (what.rfind("device ", 0) == 0) at = what.back() - '0';
        if (what == "sync device" && at == own) waited = true;
      }
      EXPECT(waited);
    }
  return 0;
}

// The powers of beta are those of the update that is launched, also behind one with other betas whose launch has failed.
static int betas_behind_an_update_that_failed() {
  fake::device = 0;
  float* a = nullptr;
  EXPECT(hipMalloc((void**)&a, 4096) == hipSuccess);
  pt_tensor t = {};
  t.grad = a; t.master = a + 64; t.m = a + 128; t.v = a + 192; t.elems = 10;
  pt_tensors* l = nullptr;
  EXPECT(pt_tensors_create(&l, PT_BF16, &t, 1, 32, nullptr, 0) == PT_OK);
  pt_hparams first = {1e-3, 0.9, 0.95, 1e-8, 0.0, 1.0}, other = first;
  other.beta1 = 0.8;
  EXPECT(pt_tensors_grad_sqnorm(l, nullptr) == PT_OK);       // with the first ones' powers
  fake::fail_kernel = "k_list_adamw";
  fake::fail_after = 0;
  EXPECT(pt_tensors_adamw_step(l, &other, nullptr) == PT_ERR_HIP);
  fake::fail_kernel = "";
  EXPECT(fake::launches("k_list_betas").size() == 1);
  EXPECT(pt_tensors_adamw_step(l, &first, nullptr) == PT_OK);
  EXPECT(fake::launches("k_list_betas").size() == 2);        // theirs again
  EXPECT(pt_tensors_grad_sqnorm(l, nullptr) == PT_OK);
  EXPECT(pt_tensors_adamw_step(l, &first, nullptr) == PT_OK);
  EXPECT(fake::launches("k_list_betas").size() == 2 && fake::launches("k_list_adamw").size() == 2);
  EXPECT(pt_tensors_destroy(l) == PT_OK);
  return 0;
}

int main(int argc, char** argv) {
  const std::string check = argc == 2 ? argv[1] : "";
  const int rc = check == "destroyed_from_another_device"        ? destroyed_from_another_device()
                 : check == "betas_behind_an_update_that_failed" ? betas_behind_an_update_that_failed()
                                                                 : 2;
  if (rc == 0) puts("held");
  return rc;
}
