// What the paged-cache translation units share.
#pragma once

namespace ra {

constexpr int kMaxPage = 1024;   // tokens a page
constexpr int kMaxRequests = 4096;
constexpr int kMaxHeads = 1024;  // heads of q, or of k and v

// Checks of a cache's shape and of its type and scales; they set the error text.
int check_pages(int page_size, int n_pages, int Hkv, int D);
int check_kv(int kv_type, const void* k_scales, const void* v_scales);

}  // namespace ra
